// Attention over chosen pages, few query rows a tile (include/dkv.h: dkv_cache_attend_chosen): O = softmax(scale Q K^T) V
// over the positions of the pages that a tile's list names.
//
// A unit is 8 query rows of one tile and key head, row = token * G + head.  The listed pages, in steps of 16 positions, are
// shared out evenly to the warps of a cluster; each keeps a running maximum, sum and outputs in registers, and
// the parts are joined in shared memory, over the cluster by reading the neighbours' (no scratch, no second launch).
// HBM bounds it (4 d bytes a listed position in bf16, 2 d + 2 in e4m3), and for a single token the chain of dependent
// reads before the first key: lengths, list, table.
//
// The products are turned round, as in the other few-row kernel: keys (columns of the values) are the 16 rows of mma.sync
// m16n8k16, the query rows its 8 columns.  Keys go from memory to the product's registers by plain 16-byte loads, without
// shared memory: the order in which d is summed is free, so lane (g, t) takes the 8 (16) numbers that its load brings as
// its own share of the steps of 16, and the queries are laid out the same way.  The values' 8 x 8 blocks become operands by one
// transposing move each; which d a column then stands for follows from the loads.
#include "attn_math.cuh"
#include "cache_internal.h"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace dkv {
namespace cache {

namespace {

using namespace tc;

constexpr int WARPS = 6, THREADS = WARPS * 32, MAX_WIDTH = 1024;
constexpr float RAISE_LOG2 = 8.0f;   // how far a score may pass the running maximum before that is raised

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// A row's numbers with one lane of its four: NW registers of bf16 pairs.  bf16: load p of 16 bytes holds d = 32 p + 8 t ..;
// codes: load p holds d = 64 p + 16 t ..
template <int D>
struct Frag {
  uint32_t w[D / 8];
};

// d of number e of register r.
template <bool E4M3>
__device__ __forceinline__ int dim_of(int r, int t, int e) {
  return E4M3 ? (r >> 3) * 64 + t * 16 + (r & 7) * 2 + e : (r >> 2) * 32 + t * 8 + (r & 3) * 2 + e;
}

template <int D, bool E4M3>
struct Raw {
  uint4 v[E4M3 ? D / 64 : D / 32];
  uint32_t scale;
};

template <int D, bool E4M3>
__device__ __forceinline__ Raw<D, E4M3> fetch(const void* pool, const uint8_t* scales, int64_t at, int t) {
  Raw<D, E4M3> x;
  x.scale = 127u;
  if (at < 0) {   // nobody's
#pragma unroll
    for (int p = 0; p < (int)(sizeof(x.v) / 16); ++p) x.v[p] = make_uint4(0, 0, 0, 0);
    return x;
  }
  const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(pool) + at * (E4M3 ? D : 2 * D)) + t;
#pragma unroll
  for (int p = 0; p < (int)(sizeof(x.v) / 16); ++p) x.v[p] = __ldg(src + 4 * p);
  if (E4M3) x.scale = __ldg(scales + at);
  return x;
}

// Four bf16 from four codes: a code's bits in bf16's fields are its value times 2^-120; f holds 2^120 times the scale.
__device__ __forceinline__ void widen(uint32_t w, __nv_bfloat162 f, uint32_t& a, uint32_t& b) {
  const uint32_t hi = (w & 0x80808080u) | ((w >> 4) & 0x07070707u), lo = (w << 4) & 0xf0f0f0f0u;
  const uint32_t x = __byte_perm(lo, hi, 0x5140), y = __byte_perm(lo, hi, 0x7362);
  const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&x), f);
  const __nv_bfloat162 q = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&y), f);
  a = *reinterpret_cast<const uint32_t*>(&p);
  b = *reinterpret_cast<const uint32_t*>(&q);
}
__device__ __forceinline__ __nv_bfloat162 bf2(uint32_t bits) { return *reinterpret_cast<const __nv_bfloat162*>(&bits); }

template <int D, bool E4M3>
__device__ __forceinline__ Frag<D> numbers(const Raw<D, E4M3>& x) {
  Frag<D> y;
  if (!E4M3) {
#pragma unroll
    for (int p = 0; p < D / 32; ++p) {
      y.w[4 * p] = x.v[p].x;
      y.w[4 * p + 1] = x.v[p].y;
      y.w[4 * p + 2] = x.v[p].z;
      y.w[4 * p + 3] = x.v[p].w;
    }
    return y;
  }
  // one factor where 2^120 times the scale is a bf16 number; else two, the scale by itself (255: NaN)
  const uint32_t s = x.scale;
  const __nv_bfloat162 f = bf2((s > 134u ? 247u : s + 120u) * 0x00800080u);
#pragma unroll
  for (int p = 0; p < (int)(sizeof(x.v) / 16); ++p) {
    widen(x.v[p].x, f, y.w[8 * p], y.w[8 * p + 1]);
    widen(x.v[p].y, f, y.w[8 * p + 2], y.w[8 * p + 3]);
    widen(x.v[p].z, f, y.w[8 * p + 4], y.w[8 * p + 5]);
    widen(x.v[p].w, f, y.w[8 * p + 6], y.w[8 * p + 7]);
  }
  if (__any_sync(0xffffffffu, s > 134u)) {
    const __nv_bfloat162 f2 = bf2(s == 255u ? 0x7fff7fffu : (s > 134u ? s : 127u) * 0x00800080u);
#pragma unroll
    for (int r = 0; r < D / 8; ++r) {
      const __nv_bfloat162 z = __hmul2(bf2(y.w[r]), f2);
      y.w[r] = *reinterpret_cast<const uint32_t*>(&z);
    }
  }
  return y;
}

// Clears what is not finite in a pair; true where there was any.
__device__ __forceinline__ bool clear_wild(uint32_t& x) {
  const uint32_t bad = ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  x &= ~(((bad >> 15) & 0x00010001u) * 0xffffu);
  return bad != 0;
}

template <int D, bool E4M3>
__device__ __noinline__ float value_at(const Pool& c, int64_t at, int d) {
  if (!E4M3) return __bfloat162float(static_cast<const __nv_bfloat16*>(c.v)[at * D + d]);
  return c.vs[at] == 255 ? __int_as_float(0x7fffffff) : 0.f;   // (a code is finite)
}

template <int D>
struct Smem {
  int page[MAX_WIDTH], entry[MAX_WIDTH];
  float part[WARPS][8][D + 4];   // outputs, maximum, sum
  float joined[8][D + 4];
  int count;
};

template <int D, bool E4M3>
__global__ void __launch_bounds__(THREADS, 2) chosen_rows(Pool c, Seqs s, Packed qp, Packed op, int G, Mask m, Chosen how, int blocks) {
  __shared__ Smem<D> w;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = cluster.num_blocks(), rank = cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int unit = blockIdx.x / C, slot = unit / blocks, r0 = (unit - slot * blocks) * 8, h = blockIdx.y;
  if (blockIdx.x == 0 && h == 0)
    for (int b = tid; b < s.n; b += THREADS) seq_at(c, s, b);
  const int b = seq_of_slot_warp(s, how.tile, slot);
  const Seq q = seq_at(c, s, b);
  const int i0 = (slot - first_slot(s, how.tile, b)) * how.tile;
  const int tokens = min(how.tile, q.n - i0), R = tokens * G;
  if (i0 < 0 || r0 >= R) return;   // (the whole cluster)
  const int rows = min(8, R - r0), p0 = q.len - q.n + i0;
  auto end_of = [&](int r) {
    const int p = p0 + min(r0 + r, R - 1) / G;
    return p < 0 ? 0 : visible_end(m, p, q.len);
  };
  const int all_end = end_of(0), any_end = end_of(rows - 1);
  // the list: pages of the pool
  const int32_t* line = how.lists + ((int64_t)h * how.slots + slot) * how.width;
  if (tid == 0) w.count = how.width;
  __syncthreads();
  for (int k = tid; k < how.width; k += THREADS) {
    const int e = __ldg(line + k), before = k ? __ldg(line + k - 1) : -1;
    int page = -1;
    if (e < 0) {
      atomicMin(&w.count, k);
    } else if ((k && before >= 0 && e <= before) || e >= (q.len + c.page_len - 1) >> c.page_log2) {
      fail(c.status, DEV_INCONSISTENT, SITE_LIST);
    } else if ((e << c.page_log2) < any_end) {
      const int64_t row = pool_row(c, s, b, h, e << c.page_log2);
      if (row >= 0) page = (int)(row >> c.page_log2);   // page * H + h
    }
    w.entry[k] = e;
    w.page[k] = page;
  }
  __syncthreads();
  const int sub = c.page_log2 - 4, total = w.count << sub, warps = C * WARPS, gw = rank * WARPS + warp;
  const int first = (int)((int64_t)total * gw / warps), last = (int)((int64_t)total * (gw + 1) / warps);
  // queries: row g's numbers, laid out as the keys'
  Frag<D> Q;
  {
    const int r = r0 + g, i = r / G, hq = h * G + r - i * G;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(qp.p) + hq * qp.head + (int64_t)(q.r0 + i0 + i) * qp.row;
#pragma unroll
    for (int k = 0; k < D / 8; k += 4) {
      const uint4 x = g < rows ? __ldg(reinterpret_cast<const uint4*>(src + dim_of<E4M3>(k, t, 0))) : make_uint4(0, 0, 0, 0);
      Q.w[k] = x.x;
      Q.w[k + 1] = x.y;
      Q.w[k + 2] = x.z;
      Q.w[k + 3] = x.w;
    }
  }
  const int end[2] = {2 * t < rows ? end_of(2 * t) : 0, 2 * t + 1 < rows ? end_of(2 * t + 1) : 0};
  float o[D / 16][4], mrun[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < D / 16; ++k) o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.f;
  // a step's place: its first position, and lane g's row of the pool (-1: nothing to be read)
  auto place = [&](int st, int& pos0, int64_t& at) {
    pos0 = 0x40000000;
    at = -1;
    if (st >= last) return;
    const int k = st >> sub, in = (st & ((1 << sub) - 1)) * 16;
    if (w.page[k] < 0) return;
    pos0 = (w.entry[k] << c.page_log2) + in;
    at = ((int64_t)w.page[k] << c.page_log2) + in + g;
  };
  // Keys (values) of the next step are asked for as soon as this one's have gone into their product.  (Positions
  // that nobody sees may lie behind the sequence: keys there are read, the page is there, and masked.)
  int pos0, next0;
  int64_t at, next;
  place(first, pos0, at);
  Raw<D, E4M3> k0 = fetch<D, E4M3>(c.k, c.ks, at, t), k1 = fetch<D, E4M3>(c.k, c.ks, at < 0 ? at : at + 8, t);
  Raw<D, E4M3> v0 = fetch<D, E4M3>(c.v, c.vs, pos0 + g < any_end ? at : -1, t);
  Raw<D, E4M3> v1 = fetch<D, E4M3>(c.v, c.vs, pos0 + g + 8 < any_end ? at + 8 : -1, t);
#pragma unroll 1
  for (int st = first; st < last; ++st, pos0 = next0, at = next) {
    place(st + 1, next0, next);
    float sc[4] = {0.f, 0.f, 0.f, 0.f}, sd[4] = {0.f, 0.f, 0.f, 0.f};
    {
      const Frag<D> a = numbers<D, E4M3>(k0), z = numbers<D, E4M3>(k1);
#pragma unroll
      for (int i = 0; i < D / 16; i += 2) {
        mma(sc, a.w[2 * i], z.w[2 * i], a.w[2 * i + 1], z.w[2 * i + 1], Q.w[2 * i], Q.w[2 * i + 1]);
        mma(sd, a.w[2 * i + 2], z.w[2 * i + 2], a.w[2 * i + 3], z.w[2 * i + 3], Q.w[2 * i + 2], Q.w[2 * i + 3]);
      }
    }
    k0 = fetch<D, E4M3>(c.k, c.ks, next, t);
    k1 = fetch<D, E4M3>(c.k, c.ks, next < 0 ? next : next + 8, t);
#pragma unroll
    for (int e = 0; e < 4; ++e) sc[e] += sd[e];
    const bool partial = pos0 + 16 > all_end;
    if (partial) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (pos0 + g + (e >> 1) * 8 >= end[e & 1]) sc[e] = -INFINITY;
    }
    float mx[2] = {fmaxf(sc[0], sc[2]), fmaxf(sc[1], sc[3])};
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
      mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], x));
      mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], x));
    }
    bool raise[2];
    float alpha[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      mx[e] *= m.sl2;
      raise[e] = mx[e] > mrun[e] + RAISE_LOG2 || (mrun[e] == -INFINITY && mx[e] > -INFINITY);
      alpha[e] = raise[e] ? (mrun[e] == -INFINITY ? 0.f : ex2(mrun[e] - mx[e])) : 1.f;
      if (raise[e]) mrun[e] = mx[e];
    }
    if (__any_sync(0xffffffffu, raise[0] || raise[1])) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[e] *= alpha[e];
#pragma unroll
        for (int k2 = 0; k2 < D / 16; ++k2) {
          o[k2][e] *= alpha[e];
          o[k2][2 + e] *= alpha[e];
        }
      }
    }
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[e] = ex2(fmaf(sc[e], m.sl2, mrun[e & 1] == -INFINITY ? 0.f : -mrun[e & 1]));
      l[e & 1] += p[e];
    }
    const uint32_t b0 = transpose(pack_bf16(p[0], p[1])), b1 = transpose(pack_bf16(p[2], p[3]));
    Frag<D> a = numbers<D, E4M3>(v0), z = numbers<D, E4M3>(v1);
    bool wild = false;
    if (partial) {
#pragma unroll
      for (int r = 0; r < D / 8; ++r) {
        wild = clear_wild(a.w[r]) || wild;
        wild = clear_wild(z.w[r]) || wild;
      }
    }
#pragma unroll
    for (int k2 = 0; k2 < D / 16; ++k2)
      mma(o[k2], transpose(a.w[2 * k2]), transpose(a.w[2 * k2 + 1]), transpose(z.w[2 * k2]), transpose(z.w[2 * k2 + 1]), b0, b1);
    v0 = fetch<D, E4M3>(c.v, c.vs, next0 + g < any_end ? next : -1, t);
    v1 = fetch<D, E4M3>(c.v, c.vs, next0 + g + 8 < any_end ? next + 8 : -1, t);
    // values that are not finite, where some row may not see them: to the rows that do
    if (partial && __any_sync(0xffffffffu, wild)) {
#pragma unroll 1
      for (int x = 0; x < 16 && pos0 + x < any_end; ++x) {
#pragma unroll
        for (int k2 = 0; k2 < D / 16; ++k2) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float y = value_at<D, E4M3>(c, at - g + x, dim_of<E4M3>(2 * k2 + half, g >> 1, g & 1));
            if (isfinite(y)) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (pos0 + x < end[e]) o[k2][2 * half + e] += y;
          }
        }
      }
    }
  }
  // ---- parts into shared memory, joined
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) l[e] += __shfl_xor_sync(0xffffffffu, l[e], x);
    float* to = w.part[warp][2 * t + e];
#pragma unroll
    for (int k2 = 0; k2 < D / 16; ++k2) {
      to[dim_of<E4M3>(2 * k2, g >> 1, g & 1)] = o[k2][e];
      to[dim_of<E4M3>(2 * k2 + 1, g >> 1, g & 1)] = o[k2][2 + e];
    }
    if (g == 0) {
      to[D] = mrun[e];
      to[D + 1] = l[e];
    }
  }
  __syncthreads();
  // a part of weight: something was seen, or a NaN
  auto join = [&](auto at, int n, float& M, float& L, float (&x)[D / 32]) {
    M = -INFINITY;
    L = 0.f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) x[k] = 0.f;
    for (int i = 0; i < n; ++i) M = fmaxf(M, at(i)[D]);
    for (int i = 0; i < n; ++i) {
      const float* y = at(i);
      const float mi = y[D], li = y[D + 1];
      if (mi == -INFINITY && li == 0.f) continue;
      const float f = mi == M || mi == -INFINITY ? 1.f : ex2(mi - M);
      L = fmaf(f, li, L);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) x[k] = fmaf(f, y[lane * (D / 32) + k], x[k]);
    }
  };
  auto store = [&](int row, float L, const float (&x)[D / 32]) {
    if (row >= rows) return;
    const float inv = L == 0.f ? 0.f : 1.0f / L;   // (a NaN stays one)
    const int r = r0 + row, i = r / G, hq = h * G + r - i * G;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(op.p) + hq * op.head + (int64_t)(q.r0 + i0 + i) * op.row + lane * (D / 32);
    if (D == 128) {
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[D / 32 - 2] * inv, x[D / 32 - 1] * inv));
    } else {
      *reinterpret_cast<uint32_t*>(dst) = pack_bf16(x[0] * inv, x[1] * inv);
    }
  };
  float M, L, x[D / 32];
  for (int row = warp; row < rows; row += WARPS) {
    join([&](int i) -> const float* { return w.part[i][row]; }, WARPS, M, L, x);
    if (C == 1) {
      store(row, L, x);
      continue;
    }
#pragma unroll
    for (int k = 0; k < D / 32; ++k) w.joined[row][lane * (D / 32) + k] = x[k];
    if (lane == 0) {
      w.joined[row][D] = M;
      w.joined[row][D + 1] = L;
    }
  }
  if (C == 1) return;
  cluster.sync();
  for (int row = rank + C * warp; row < rows; row += C * WARPS) {   // (the CTAs share the rows)
    join([&](int i) -> const float* { return cluster.map_shared_rank(&w, i)->joined[row]; }, C, M, L, x);
    store(row, L, x);
  }
  cluster.sync();
}

}  // namespace

cudaError_t launch_chosen_rows(const Pool& c, const Seqs& s, const Packed& q, const Packed& o, int Hq, const Mask& m,
                               const Chosen& how, cudaStream_t st) {
  const int n_sm = sm_count(), G = Hq / c.H;
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const int blocks = (how.tile * G + 7) / 8;
  // a cluster for each unit, as large as leaves two CTAs an SM and a warp a step or more
  int C = 1;
  const int64_t units = (int64_t)std::min(how.slots, s.rows) * blocks * c.H;   // (a tile has a row or more)
  while (C < 8 && units * C <= n_sm && how.width * (c.page_len / 16) >= 2 * C * WARPS) C *= 2;
  if ((int64_t)how.slots * blocks * C > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(how.slots * blocks * C, c.H);
  auto* f = c.d == 128 ? (c.e4m3 ? chosen_rows<128, true> : chosen_rows<128, false>)
                       : (c.e4m3 ? chosen_rows<64, true> : chosen_rows<64, false>);
  return launch_kernel(f, grid, THREADS, 0, C, false, st, c, s, q, o, G, m, how, blocks);
}

}  // namespace cache
}  // namespace dkv
