// Attention over chosen pages, few query rows a tile (include/dkv.h: dkv_cache_attend_chosen): O = softmax(scale Q K^T) V
// over the positions of the pages that a tile's list names.
//
// A unit is 8 query rows of one tile and key head, row = token * G + head.  The listed pages, in steps of 16 positions, are
// shared out evenly to the warps of a cluster; each keeps a running maximum, sum and outputs in registers, and
// the parts are joined in shared memory, over the cluster by reading the neighbours' (no scratch, no second launch).
// HBM bounds it (4 d bytes a listed position in bf16, 2 d + 2 in e4m3), and for a single token the chain of dependent
// reads before the first key: sequence, table, key.
//
// The products are turned round, as in the other few-row kernel: keys (columns of the values) are the 16 rows of mma.sync
// m16n8k16, the query rows its 8 columns.  Keys go from memory to the product's registers by plain 16-byte loads, without
// shared memory: the order in which d is summed is free, so lane (g, t) takes the 8 (16) numbers that its load brings as
// its own share of the steps of 16, and the queries are laid out the same way.  The values' 8 x 8 blocks become operands by one
// transposing move each; which d a column then stands for follows from the loads.  The next step's loads are issued as soon as
// their registers are free.
//
// e4m3: the keys' codes become fp16, one conversion for two, and meet queries in fp16; their scales join the scores.  The values'
// codes are transposed two at a time, a pair of columns in the place of one, and become bf16 with their scales in them.
//
// Weights are rounded to bf16 where they meet the values (mma.sync's other operand would have to be fp32 too, at a fraction of the rate);
// their sum takes them unrounded.
//
// Measured: 32 tokens of 40 on 8 heads over 32 pages of 64 in e4m3 36 us (136 MB; 12 us of it with 3 pages: launch, chain, joining), in
// bf16 49 (269 MB, 5.5 TB/s; 6.8 is a copy's); one token over as many pages of 131,001 positions, 8 heads, 10 to 12.  (By asynchronous copies
// into shared memory, two or three steps ahead: 45.)
#include "attn_math.cuh"
#include "cache_internal.h"

#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

namespace cg = cooperative_groups;

namespace dkv {
namespace cache {

namespace {

using namespace tc;

constexpr int MAX_WIDTH = 1024;
// Warps of a CTA, CTAs of an SM (registers), times 16 positions of a warp's step.  (32 tokens over 32 pages: e4m3 8 warps 39 us, 6
// 43, 12 in one CTA 49; bf16 6 warps 50, 8 70; d = 64, e4m3: two times 16 positions 25, one 27; bf16 one 29, two 31.)
// NARROW: two warps a CTA and as many warps an SM, where there are many units.
template <int D, bool E4M3, bool NARROW>
struct Cfg {
  static constexpr int ALL = !E4M3 && D == 128 ? 12 : 16;   // warps of an SM
  static constexpr int WARPS = NARROW ? 2 : ALL / 2, CTAS = ALL / WARPS, NH = E4M3 ? 128 / D : 1;
  static constexpr int THREADS = 32 * WARPS;
};
constexpr float RAISE_LOG2 = 8.0f;   // how far a score may pass the running maximum before that is raised

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// A row's numbers with one lane of its four: registers of pairs.  bf16: load p of 16 bytes holds d = 32 p + 8 t ..;
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

// d of row g (half 1: g + 8) of outputs block i.  bf16: words 2 i and 2 i + 1 were transposed, whose columns 2 t' + e are d of
// lane t''s number e.  Codes: word i, whose columns t' .. are pairs: row g is the pair of lane g / 2, the two numbers of which
// (word halves) are columns 2 (g / 2) and 2 (g / 2) + 1 of the block; the pair's first code goes to row g, its second to g + 8.
template <bool E4M3>
__device__ __forceinline__ int column(int i, int half, int g) {
  return E4M3 ? dim_of<E4M3>(2 * i + (g & 1), g >> 1, half) : dim_of<E4M3>(2 * i + half, g >> 1, g & 1);
}

template <int D, bool E4M3>
struct Raw {
  uint4 v[E4M3 ? D / 64 : D / 32];
};

// Row `at` (of d numbers) of a pool: lane t's share.
template <int D, bool E4M3>
__device__ __forceinline__ Raw<D, E4M3> fetch(const void* pool, int64_t at, int t) {
  Raw<D, E4M3> x;
  const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(pool) + at * (E4M3 ? D : 2 * D)) + t;
#pragma unroll
  for (int p = 0; p < (int)(sizeof(x.v) / 16); ++p) x.v[p] = __ldg(src + 4 * p);
  return x;
}
template <int D, bool E4M3>
__device__ __forceinline__ uint32_t word(const Raw<D, E4M3>& x, int i) {
  const uint4& v = x.v[i >> 2];
  return (i & 3) == 0 ? v.x : (i & 3) == 1 ? v.y : (i & 3) == 2 ? v.z : v.w;
}

// Four fp16 from four codes (exact).
__device__ __forceinline__ void widen_f16(uint32_t w, uint32_t& a, uint32_t& b) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(a), "=r"(b) : "r"(w));
}

// Two positions of two neighbouring columns (bytes: position 0: d, d + 1, position 1: d, d + 1) as bf16, a register for each
// column: a code's bits in bf16's fields (its sign spread over a byte above it, all but one of those bits cleared) are its
// value times 2^-120; f holds 2^120 times the positions' scales.
__device__ __forceinline__ void widen_values(uint32_t w, __nv_bfloat162 f, uint32_t& d0, uint32_t& d1) {
  uint32_t a, b;
  asm("prmt.b32 %0, %1, 0, 0xa280;" : "=r"(a) : "r"(w));   // (a selector's upper bit: that byte's sign, eight times)
  asm("prmt.b32 %0, %1, 0, 0xb391;" : "=r"(b) : "r"(w));
  a = (a << 4) & 0x87f087f0u;
  b = (b << 4) & 0x87f087f0u;
  const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), f);
  const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&b), f);
  d0 = *reinterpret_cast<const uint32_t*>(&x);
  d1 = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ __nv_bfloat162 bf2(uint32_t bits) { return *reinterpret_cast<const __nv_bfloat162*>(&bits); }
// 2^120 times the scales of two bytes (low and high half), as far as bf16 holds it; the rest (255: NaN).
__device__ __forceinline__ __nv_bfloat162 factor(uint32_t s0, uint32_t s1) {
  return bf2((s0 > 134u ? 247u : s0 + 120u) << 7 | (s1 > 134u ? 247u : s1 + 120u) << 23);
}
__device__ __forceinline__ __nv_bfloat162 factor_rest(uint32_t s0, uint32_t s1) {
  auto one = [](uint32_t s) { return s == 255u ? 0x7fffu : (s > 134u ? s : 127u) << 7; };
  return bf2(one(s0) | one(s1) << 16);
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

__device__ __forceinline__ uint32_t times(uint32_t x, __nv_bfloat162 f) {
  const __nv_bfloat162 y = __hmul2(bf2(x), f);
  return *reinterpret_cast<const uint32_t*>(&y);
}
// Element i of a small array in registers.
template <typename T, int N>
__device__ __forceinline__ T place_of(const T (&x)[N], int i) {
  T y = x[0];
#pragma unroll
  for (int k = 1; k < N; ++k)
    if (i == k) y = x[k];
  return y;
}

template <int D, int WARPS>
struct Smem {
  int page[MAX_WIDTH], entry[MAX_WIDTH];
  float part[WARPS][8][D + 4];   // outputs, maximum, sum
  float joined[8][D + 4];
  int count;
  int bad;   // least faulty entry: twice its place, odd: its page
};

template <int D, bool E4M3, bool NARROW>
__global__ void __launch_bounds__(Cfg<D, E4M3, NARROW>::THREADS, (Cfg<D, E4M3, NARROW>::CTAS)) chosen_rows(Pool c, Seqs s, Packed qp, Packed op, int G, Mask m, Chosen how, int blocks) {
  using K = Cfg<D, E4M3, NARROW>;
  constexpr int WARPS = K::WARPS, THREADS = K::THREADS, NH = K::NH;
  __shared__ Smem<D, WARPS> w;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = cluster.num_blocks(), rank = cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int unit = blockIdx.x / C, slot = unit / blocks, r0 = (unit - slot * blocks) * 8, h = blockIdx.y;
  if (blockIdx.x == 0 && h == 0)
    for (int b = tid; b < s.n; b += THREADS) seq_at(c, s, b);
  // (the list's first entries are asked for before the sequence is known)
  const int32_t* line = how.lists + ((int64_t)h * how.slots + slot) * how.width;
  const int early = tid < how.width ? __ldg(line + tid) : -1, early_before = tid && tid < how.width ? __ldg(line + tid - 1) : -1;
  Seq q;
  const int b = seq_of_slot_warp(c, s, how.tile, slot, q);
  const int i0 = (slot - q.r0 / how.tile - b) * how.tile;
  const int tokens = min(how.tile, q.n - i0), R = tokens * G;
  if (i0 < 0 || r0 >= R) return;   // (the whole cluster)
  const int rows = min(8, R - r0), p0 = q.len - q.n + i0;
  auto end_of = [&](int r) {
    const int p = p0 + min(r0 + r, R - 1) / G;
    return p < 0 ? 0 : visible_end(m, p, q.len);
  };
  const int all_end = end_of(0), any_end = end_of(rows - 1);
  // the list: pages of the pool
  if (tid == 0) {
    w.count = how.width;
    w.bad = 0x7fffffff;
  }
  __syncthreads();
  for (int k = tid; k < how.width; k += THREADS) {
    const int e = k == tid ? early : __ldg(line + k), before = k == tid ? early_before : __ldg(line + k - 1);
    int page = -1;
    if (e < 0) {
      atomicMin(&w.count, k);
    } else if ((k && before >= 0 && e <= before) || e >= (q.len + c.page_len - 1) >> c.page_log2) {
      atomicMin(&w.bad, 2 * k);
    } else if ((e << c.page_log2) < any_end) {
      const int at = s.table[(int64_t)b * s.max_pages + e];
      if ((unsigned)at < (unsigned)c.n_pages) page = at * c.H + h;   // (memory holds fewer than 2^31)
      else atomicMin(&w.bad, 2 * k + 1);
    }
    w.entry[k] = e;
    w.page[k] = page;
  }
  __syncthreads();
  if (tid == 0 && w.bad >> 1 < w.count) fail(c.status, DEV_INCONSISTENT, w.bad & 1 ? SITE_PAGE : SITE_LIST);   // (what is behind the end is nothing)
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
  // codes are met by queries in fp16, each row times a power of two that brings its largest magnitude to 2^14 .. 2^15: what is
  // 2^-28 of that or more stays exact, smaller numbers are off by 2^-39 of it at most
  float mul[2] = {m.sl2, m.sl2};   // of the columns' scores, into exponents of 2
  if constexpr (E4M3) {
    uint32_t top = 0;   // (bits of magnitudes order like the magnitudes)
#pragma unroll
    for (int k = 0; k < D / 8; ++k) top = __vmaxu2(top, Q.w[k] & 0x7fff7fffu);
    top = max(top & 0xffffu, top >> 16);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int x = top >= 0x7f80u ? 14 : max((int)(top >> 7) - 127, -100);
    const float f = __uint_as_float((uint32_t)(127 + 14 - x) << 23);
#pragma unroll
    for (int k = 0; k < D / 8; ++k) {
      const __half2 y = __floats2half2_rn(__uint_as_float(Q.w[k] << 16) * f, __uint_as_float(Q.w[k] & 0xffff0000u) * f);
      Q.w[k] = *reinterpret_cast<const uint32_t*>(&y);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) mul[e] *= __uint_as_float((uint32_t)(127 - 14 + __shfl_sync(0xffffffffu, x, 4 * (2 * t + e))) << 23);
  }
  const int end[2] = {2 * t < rows ? end_of(2 * t) : 0, 2 * t + 1 < rows ? end_of(2 * t + 1) : 0};
  float o[D / 16][4], mrun[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < D / 16; ++k) o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.f;
  // the place of 16 positions: the first one, and its row of the pool (nothing to be read: a position that nobody sees, and
  // whatever row is there)
  auto place = [&](int st, int& pos0, int64_t& at) {
    pos0 = 0x40000000;
    at = -1;
    if (st >= last) return;
    const int k = st >> sub, in = (st & ((1 << sub) - 1)) * 16;
    if (w.page[k] < 0) return;
    pos0 = (w.entry[k] << c.page_log2) + in;
    at = ((int64_t)w.page[k] << c.page_log2) + in;
  };
  // A warp takes NH times 16 positions a step: as many as the registers hold.  Keys (values) of the next step are asked for as
  // soon as this one's have gone into their product.  (Positions that nobody sees are read, their page is there, and masked.)
  int pos0[NH], next0[NH];
  int64_t at[NH], next[NH];
  using R1 = Raw<D, E4M3>;
  R1 k0[NH]{}, k1[NH]{}, v0[NH]{}, v1[NH]{};
  uint32_t ks0[NH]{}, ks1[NH]{}, vs0[NH]{}, vs1[NH]{};   // scale bytes: keys g, g + 8; values 2 t, 2 t + 1 and those + 8
  auto load_keys = [&](const int64_t (&x)[NH]) {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      if (x[n] < 0) continue;
      k0[n] = fetch<D, E4M3>(c.k, x[n] + g, t);
      k1[n] = fetch<D, E4M3>(c.k, x[n] + g + 8, t);
    }
  };
  auto load_values = [&](const int64_t (&x)[NH]) {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      if (x[n] < 0) continue;
      v0[n] = fetch<D, E4M3>(c.v, x[n] + g, t);
      v1[n] = fetch<D, E4M3>(c.v, x[n] + g + 8, t);
    }
  };
  auto load_scales = [&](const int64_t (&x)[NH]) {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      if (x[n] < 0) continue;
      ks0[n] = __ldg(c.ks + x[n] + g);
      ks1[n] = __ldg(c.ks + x[n] + g + 8);
      vs0[n] = __ldg(reinterpret_cast<const uint16_t*>(c.vs + x[n]) + t);
      vs1[n] = __ldg(reinterpret_cast<const uint16_t*>(c.vs + x[n] + 8) + t);
    }
  };
#pragma unroll
  for (int n = 0; n < NH; ++n) place(first + n, pos0[n], at[n]);
  load_keys(at);
  load_values(at);
  if constexpr (E4M3) load_scales(at);
#pragma unroll 1
  for (int st = first; st < last; st += NH) {
    bool partial = false;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      place(st + NH + n, next0[n], next[n]);
      partial = partial || pos0[n] + 16 > all_end;
    }
    // scores in exponents of 2, rounded before the maximum goes off them: of large ones the rounding alone passes fp32 as an
    // exponent.  (A scale is multiplied by its row's factor first: the sum of products times one of them may pass fp32 too.)
    float sc[NH][4];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float sd[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
      if constexpr (E4M3) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {   // a word of codes: a step of 16
          uint32_t a0, a2, a1, a3;
          widen_f16(word(k0[n], i), a0, a2);
          widen_f16(word(k1[n], i), a1, a3);
          mma_f16(i & 1 ? sd : sc[n], a0, a1, a2, a3, Q.w[2 * i], Q.w[2 * i + 1]);
        }
        const float f0 = scale_of(ks0[n]), f1 = scale_of(ks1[n]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] = (sc[n][e] + sd[e]) * ((e < 2 ? f0 : f1) * mul[e & 1]);
      } else {
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
          mma(i & 1 ? sd : sc[n], word(k0[n], 2 * i), word(k1[n], 2 * i), word(k0[n], 2 * i + 1), word(k1[n], 2 * i + 1), Q.w[2 * i], Q.w[2 * i + 1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] = (sc[n][e] + sd[e]) * m.sl2;
      }
    }
    load_keys(next);
    if (partial) {
#pragma unroll
      for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (pos0[n] + g + (e >> 1) * 8 >= end[e & 1]) sc[n][e] = -INFINITY;
    }
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      mx[0] = max3(mx[0], sc[n][0], sc[n][2]);
      mx[1] = max3(mx[1], sc[n][1], sc[n][3]);
    }
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
      mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], x));
      mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], x));
    }
    bool raise[2];
    float alpha[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      raise[e] = mx[e] > mrun[e] + RAISE_LOG2 || (mrun[e] == -INFINITY && mx[e] > -INFINITY);
      alpha[e] = raise[e] ? (mrun[e] == -INFINITY ? 0.f : ex2(mrun[e] - mx[e])) : 1.f;
      if (raise[e]) mrun[e] = mx[e];
    }
    if (__any_sync(0xffffffffu, raise[0] || raise[1])) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[e] *= alpha[e];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          o[i][e] *= alpha[e];
          o[i][2 + e] *= alpha[e];
        }
      }
    }
    uint32_t b0[NH], b1[NH];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = ex2(sc[n][e] - (mrun[e & 1] == -INFINITY ? 0.f : mrun[e & 1]));
        l[e & 1] += p[e];
      }
      b0[n] = transpose(pack_bf16(p[0], p[1]));
      b1[n] = transpose(pack_bf16(p[2], p[3]));
    }
    bool wild = false;
    uint32_t large = 0;
    if constexpr (E4M3) {
#pragma unroll
      for (int n = 0; n < NH; ++n) large = max(large, max(max(vs0[n] & 0xffu, vs0[n] >> 8), max(vs1[n] & 0xffu, vs1[n] >> 8)));
    }
    const bool two = E4M3 && __any_sync(0xffffffffu, large > 134u);
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      __nv_bfloat162 f0 = bf2(0), f1 = f0;
      if constexpr (E4M3) {
        f0 = factor(vs0[n] & 0xffu, vs0[n] >> 8);
        f1 = factor(vs1[n] & 0xffu, vs1[n] >> 8);
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t a0, a1, a2, a3;
        if constexpr (E4M3) {
          widen_values(transpose(word(v0[n], i)), f0, a0, a1);
          widen_values(transpose(word(v1[n], i)), f1, a2, a3);
          if (two) {
            const __nv_bfloat162 h0 = factor_rest(vs0[n] & 0xffu, vs0[n] >> 8), h1 = factor_rest(vs1[n] & 0xffu, vs1[n] >> 8);
            a0 = times(a0, h0);
            a1 = times(a1, h0);
            a2 = times(a2, h1);
            a3 = times(a3, h1);
          }
        } else {
          a0 = transpose(word(v0[n], 2 * i));
          a1 = transpose(word(v0[n], 2 * i + 1));
          a2 = transpose(word(v1[n], 2 * i));
          a3 = transpose(word(v1[n], 2 * i + 1));
        }
        if (partial) {
          wild = clear_wild(a0) || wild;
          wild = clear_wild(a1) || wild;
          wild = clear_wild(a2) || wild;
          wild = clear_wild(a3) || wild;
        }
        mma(o[i], a0, a1, a2, a3, b0[n], b1[n]);
      }
    }
    load_values(next);
    if constexpr (E4M3) load_scales(next);
    // values that are not finite, where some row may not see them: to the rows that do
    if (partial && __any_sync(0xffffffffu, wild)) {
#pragma unroll 1
      for (int x = 0; x < 16 * NH; ++x) {
        const int p = NH == 1 || x < 16 ? pos0[0] : place_of(pos0, x >> 4);
        const int64_t row = NH == 1 || x < 16 ? at[0] : place_of(at, x >> 4);
        if (p + (x & 15) >= any_end) continue;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float y = value_at<D, E4M3>(c, row + (x & 15), column<E4M3>(i, half, g));
            if (isfinite(y)) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (p + (x & 15) < end[e]) o[i][2 * half + e] += y;
          }
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      pos0[n] = next0[n];
      at[n] = next[n];
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
      to[column<E4M3>(k2, 0, g)] = o[k2][e];
      to[column<E4M3>(k2, 1, g)] = o[k2][2 + e];
    }
    if (g == 0) {
      to[D] = mrun[e];
      to[D + 1] = l[e];
    }
  }
  __syncthreads();
  // (a part that has seen nothing adds zeros; one whose scores are all -infinity the values that are not finite)
  auto join = [&](auto at, int n, float& M, float& L, float (&x)[D / 32]) {
    M = -INFINITY;
    L = 0.f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) x[k] = 0.f;
    for (int i = 0; i < n; ++i) M = fmaxf(M, at(i)[D]);
    for (int i = 0; i < n; ++i) {
      const float* y = at(i);
      const float mi = y[D], li = y[D + 1];
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
  const int blocks = (how.tokens * G + 7) / 8;
  // few units: a cluster for each, while its CTAs have 16 steps or more (8 units: 8 CTAs each 12.5 us, 4 14.4, 1 24.7; 64 units: 4 18.5 us, 8
  // 27, 2 23; 256 units: 1 35, 2 45)
  int C = 1;
  const int64_t units = (int64_t)std::min(how.slots, s.rows) * blocks * c.H;   // (a tile has a row or more)
  while (C < 8 && units * C <= n_sm && how.width * (c.page_len / 16) >= 16 * C) C *= 2;
  if ((int64_t)how.slots * blocks * C > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(how.slots * blocks * C, c.H);
  // many short lists: two warps a CTA (8 pages of 64 in e4m3, 800 units 35 us, wide CTAs 43, 3,200 116 and 146; 29,384 lists of up to
  // 4 pages in bf16 387 and 647; but 32 pages, 3,200 units 337 and 314)
  const bool narrow = C == 1 && units > 4 * n_sm && how.width * (c.page_len / 16) <= 64;
  auto launch = [&](auto d, auto e4m3) {
    constexpr int D = decltype(d)::value;
    constexpr bool E = decltype(e4m3)::value;
    return narrow ? launch_kernel(chosen_rows<D, E, true>, grid, Cfg<D, E, true>::THREADS, 0, 1, false, st, c, s, q, o, G, m, how, blocks)
                  : launch_kernel(chosen_rows<D, E, false>, grid, Cfg<D, E, false>::THREADS, 0, C, false, st, c, s, q, o, G, m, how, blocks);
  };
  using D128 = std::integral_constant<int, 128>;
  using D64 = std::integral_constant<int, 64>;
  if (c.d == 128) return c.e4m3 ? launch(D128(), std::true_type()) : launch(D128(), std::false_type());
  return c.e4m3 ? launch(D64(), std::true_type()) : launch(D64(), std::false_type());
}

}  // namespace cache
}  // namespace dkv
