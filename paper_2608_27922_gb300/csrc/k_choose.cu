// Summaries of pages and the choice of pages by them (include/dkv.h: dkv_cache_summarise, dkv_cache_choose).
//
// A summary is the mean key of a page and head in 8 bits, so a page costs d + 1 bytes instead of its page_len rows.  The
// score of a query row and a page is a product of whole numbers (magnitudes up to 127, sums of d of them below 2^21) times
// a power of two: fp16 holds the numbers, the tensor cores' fp32 sums of them are exact in whatever order, and so
// the choice does not depend on how the work is split.
#include "cache_internal.h"

#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace dkv {
namespace cache {

namespace {

constexpr int SMIN = -50;            // least exponent of 8-bit codes
constexpr float WILD = 0x1p40f;      // magnitudes from here on have no codes

// The smallest e >= SMIN with a <= 127 2^e (0 <= a < 2^40).  127 = (2 - 2^-6) 2^6: a = f 2^x, 1 <= f < 2.
__device__ __forceinline__ int exponent_of(float a) {
  const uint32_t u = __float_as_uint(a);
  const int x = (int)(u >> 23) - 127;
  return max(x - 6 + ((u & 0x7fffffu) > 0x7e0000u ? 1 : 0), SMIN);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// ------------------------------------------------------------------ summaries
// A number as hi + lo, |lo| <= ulp(hi) / 2: sums exact to some 45 bits.
struct Two {
  float hi, lo;
};
__device__ __forceinline__ void add(Two& s, float x) {
  const float t = __fadd_rn(s.hi, x), b = __fsub_rn(t, s.hi);
  s.lo = __fadd_rn(s.lo, __fadd_rn(__fsub_rn(s.hi, __fsub_rn(t, b)), __fsub_rn(x, b)));
  s.hi = t;
}
__device__ __forceinline__ Two settled(Two s) {   // hi = hi + lo rounded
  const float t = __fadd_rn(s.hi, s.lo);
  return Two{t, __fsub_rn(s.lo, __fsub_rn(t, s.hi))};
}

__device__ __forceinline__ float scaled(uint32_t code, float f) {   // an e4m3 code's value times f
  const uint32_t m = code & 7, e = (code >> 3) & 15;
  const float x = e ? __uint_as_float(((e + 120) << 23) | (m << 20)) : (float)m * 0x1p-9f;
  return (code & 0x80u ? -x : x) * f;
}

constexpr int SUM_THREADS = 256;

__device__ __forceinline__ void add(Two& s, const Two& y) {
  add(s, y.hi);
  s.lo = __fadd_rn(s.lo, y.lo);
}

// Block: pages of one sequence (blockIdx.y), each with one head, in turn.  A row lies with d / 8 threads; the rows' sums
// go over the warp, then one thread a column joins the warps'.
template <int D, bool E4M3>
__global__ void __launch_bounds__(SUM_THREADS) summarise(Pool c, Seqs s, const int32_t* first, int8_t* code, uint8_t* scale) {
  constexpr int LANES = D / 8, ROWS = SUM_THREADS / LANES, WARPS = SUM_THREADS / 32;
  __shared__ Two part[WARPS][D];
  __shared__ float tops[D / 32];
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid % LANES, r0 = tid / LANES;
  const Seq q = seq_at(c, s, b);
  const int from = max(first ? first[b] : q.len - q.n, 0) >> c.page_log2, pages = (q.len + c.page_len - 1) >> c.page_log2;
  if (!first && q.n == 0) return;
  const int64_t units = (int64_t)max(pages - from, 0) * c.H;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int h = (int)(u % c.H), k = from + (int)(u / c.H);
    const int64_t at = pool_row(c, s, b, h, k << c.page_log2);   // (the same for all threads)
    if (at < 0) continue;
    const int held = min(c.page_len, q.len - (k << c.page_log2));
    Two sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = Two{0.f, 0.f};
#pragma unroll 4
    for (int r = r0; r < held; r += ROWS) {
      float x[8];
      if (E4M3) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(c.k) + (at + r) * D) + lane);
        const float f = scale_of(c.ks[at + r]);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = scaled((i < 4 ? v.x >> (8 * i) : v.y >> (8 * i - 32)) & 0xffu, f);
      } else {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(c.k) + (at + r) * D) + lane);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[2 * i] = __uint_as_float(w[i] << 16);
          x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) add(sum[i], x[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int o = LANES; o < 32; o <<= 1)
        add(sum[i], Two{__shfl_xor_sync(0xffffffffu, sum[i].hi, o), __shfl_xor_sync(0xffffffffu, sum[i].lo, o)});
    }
    __syncthreads();   // (the last unit's sums have been read)
    if (tid % 32 < LANES) {
#pragma unroll
      for (int i = 0; i < 8; ++i) part[tid / 32][lane * 8 + i] = sum[i];
    }
    __syncthreads();
    Two m{0.f, 0.f};
    if (tid < D) {
      m = part[0][tid];
#pragma unroll
      for (int w = 1; w < WARPS; ++w) add(m, part[w][tid]);
      m = settled(m);
      if ((held & (held - 1)) == 0) {
        const float f = 1.0f / (float)held;
        m.hi *= f;
        m.lo *= f;
      } else {
        const double y = ((double)m.hi + (double)m.lo) / (double)held;
        m.hi = (float)y;
        m.lo = (float)(y - (double)m.hi);
      }
      // a magnitude that lies above hi's counts as the next float; one without codes as an infinity
      const float a = fabsf(m.hi);
      const bool above = m.hi < 0.f ? m.lo < 0.f : m.lo > 0.f;
      float top = above && (__float_as_uint(a) & 0x7fffffu) == 0x7e0000u ? __uint_as_float(__float_as_uint(a) + 1) : a;
      if (!(a < WILD)) top = INFINITY;
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (tid % 32 == 0) tops[tid / 32] = top;
    }
    __syncthreads();
    if (tid < D) {
      float top = tops[0];
#pragma unroll
      for (int w = 1; w < D / 32; ++w) top = fmaxf(top, tops[w]);
      const bool fine = top < INFINITY;
      const int e = fine ? exponent_of(top) : 0;
      const float y = m.hi * pow2(-e);
      float r = rintf(y);
      if (fabsf(y - r) == 0.5f && m.lo != 0.f) r = m.lo > 0.f ? floorf(y) + 1.f : floorf(y);   // no tie
      const int64_t row = at >> c.page_log2;   // page * H + h
      code[row * D + tid] = fine ? (int8_t)(int)r : 0;
      if (tid == 0) scale[row] = fine ? (uint8_t)(e + 127) : 255;
    }
  }
}

// ------------------------------------------------------------------ choice
constexpr int CH_THREADS = 256;
constexpr int CAP = 2048;        // pages looked at in one go
constexpr int MAX_TOP = 1024;
constexpr int PLACES = CAP + MAX_TOP;

// Order of scores as unsigned numbers; 0: not to be listed.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <int D>
struct Work {
  static constexpr int STRIDE = D + 4;   // halves of a row: 8-byte reads of 4 lanes x 4 rows touch every bank once
  __half q[64][STRIDE];
  float unit[64];            // 2^e of a row, 0: none
  alignas(16) uint32_t key[PLACES];      // what has been kept so far, then this part's pages (first their best scores)
  int page[PLACES];          //   ascending
  int at[CAP];               // of this part's pages: place in the pool
  float scale[CAP];          //   and 2^e of the summary, 0: not to be listed
  uint32_t kept_key[MAX_TOP];
  int kept_page[MAX_TOP];
  uint32_t lo[8], hi[8];
  int total[8];
  int kept, below;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Four signed bytes as two pairs of fp16: 1024 + (byte ^ 128) lies in the fields of 0x6400, less 1152.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& a, uint32_t& b) {
  w ^= 0x80808080u;
  const uint32_t x = __byte_perm(w, 0x64646464u, 0x4140), y = __byte_perm(w, 0x64646464u, 0x4342);
  const __half2 k = __float2half2_rn(1152.0f);
  const __half2 p = __hsub2(*reinterpret_cast<const __half2*>(&x), k), q = __hsub2(*reinterpret_cast<const __half2*>(&y), k);
  a = *reinterpret_cast<const uint32_t*>(&p);
  b = *reinterpret_cast<const uint32_t*>(&q);
}

// The `top` largest of key[0 .. n), equal ones: the first, in their order, into kept_key and kept_page.  Thread t holds
// places t PER ..; halving the range of the keys with counts over the block finds a bound with `top` keys above
// it, or the top-th key itself where others equal it.
template <int PER, typename W>
__device__ __forceinline__ void keep_best(W& w, int n, int top) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t k[PER], least = 0xffffffffu, most = 0;
  int valid = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    k[i] = tid * PER + i < n ? w.key[tid * PER + i] : 0;
    if (k[i]) {
      least = min(least, k[i]);
      most = max(most, k[i]);
      ++valid;
    }
  }
  least = __reduce_min_sync(0xffffffffu, least);
  most = __reduce_max_sync(0xffffffffu, most);
  valid = __reduce_add_sync(0xffffffffu, valid);
  if (lane == 0) {
    w.lo[warp] = least;
    w.hi[warp] = most;
    w.total[warp] = valid;
  }
  __syncthreads();
  valid = 0;
#pragma unroll
  for (int x = 0; x < CH_THREADS / 32; ++x) {
    least = min(least, w.lo[x]);
    most = max(most, w.hi[x]);
    valid += w.total[x];
  }
  // keys > T are kept, and `need` of those equal to T
  uint32_t T = 0;
  int need = 0;
  if (valid > top) {
    // lo: more than `top` keys >= lo; hi: at most `top` keys >= hi
    uint32_t lo = least, hi = most + 1;   // (no key is 0xffffffff: that would be a NaN)
    int above = 0;                        // keys >= hi
#pragma unroll 1
    while (hi - lo > 1 && above != top) {
      const uint32_t mid = lo + (hi - lo) / 2;
      int c = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) c += k[i] >= mid;
      c = __reduce_add_sync(0xffffffffu, c);
      __syncthreads();
      if (lane == 0) w.total[warp] = c;
      __syncthreads();
      c = 0;
#pragma unroll
      for (int x = 0; x < CH_THREADS / 32; ++x) c += w.total[x];
      if (c > top) {
        lo = mid;
      } else {
        hi = mid;
        above = c;
      }
    }
    T = hi - 1;
    need = top - above;   // (0 unless hi = lo + 1: then T = lo is the top-th key)
  }
  int eq = 0, gt = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    eq += T && k[i] == T;
    gt += k[i] > T;
  }
  // sums over the threads before: equal ones in the upper half
  const int mine = eq << 16 | gt;
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 31) w.total[warp] = incl;
  __syncthreads();
  int before = incl - mine, all = 0;
#pragma unroll
  for (int x = 0; x < CH_THREADS / 32; ++x) {
    if (x < warp) before += w.total[x];
    all += w.total[x];
  }
  int eq_before = before >> 16, gt_before = before & 0xffff;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool same = T && k[i] == T;
    if (k[i] > T || (same && eq_before < need)) {
      const int at = gt_before + min(eq_before, need);
      w.kept_key[at] = k[i];
      w.kept_page[at] = w.page[tid * PER + i];
    }
    eq_before += same;
    gt_before += k[i] > T;
  }
  if (tid == 0) w.kept = (all & 0xffff) + min(all >> 16, need);
  __syncthreads();
}
template <typename W>
__device__ __forceinline__ void keep_best(W& w, int n, int top) {
  if (n <= 4 * CH_THREADS) keep_best<4>(w, n, top);
  else keep_best<PLACES / CH_THREADS>(w, n, top);
}

// Cluster: one list (slot blockIdx.x / CTAs of the cluster, head blockIdx.y); its CTAs share the seen pages.
template <int D>
__global__ void __launch_bounds__(CH_THREADS) choose(Pool c, Seqs s, const int8_t* code, const uint8_t* scale, Packed qp, int G,
                                                     Choose how, int32_t* lists) {
  extern __shared__ __align__(16) uint8_t raw[];
  Work<D>& w = *reinterpret_cast<Work<D>*>(raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int C = cluster.num_blocks(), rank = cluster.block_rank();
  const int slot = blockIdx.x / C, h = blockIdx.y, slots = gridDim.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  if (blockIdx.x == 0 && h == 0)
    for (int b = tid; b < s.n; b += CH_THREADS) seq_at(c, s, b);
  const int b = seq_of_slot_warp(s, how.tile, slot);
  const Seq q = seq_at(c, s, b);
  const int i0 = (slot - first_slot(s, how.tile, b)) * how.tile;
  int32_t* line = lists + ((int64_t)h * slots + slot) * how.width;
  const int m = min(how.tile, q.n - i0), p1 = q.len - q.n + i0 + m - 1;
  if (i0 < 0 || m <= 0 || p1 < 0) {   // no tile, or one that sees nothing (the whole cluster)
    if (rank == 0)
      for (int k = tid; k < how.width; k += CH_THREADS) line[k] = -1;
    return;
  }
  const int p0 = max(p1 - m + 1, 0);
  const Mask mask{0.f, 0, 0, how.block, how.inverse};
  const int end = visible_end(mask, p0, q.len);
  const int whole = end == q.len ? (q.len + c.page_len - 1) >> c.page_log2 : end >> c.page_log2;
  const int own = p1 >> c.page_log2, lo = max(0, (p0 >> c.page_log2) - (how.local - 1)), sinks = min(how.sinks, whole);
  const int R = m * G;
  // this CTA's share of the seen pages
  const int per = (whole + C - 1) / C, a = min(rank * per, whole), z = min(a + per, whole);
  int kept = 0;
  if (how.top > 0) {
#pragma unroll 1
    for (int k0 = a; k0 < z; k0 += CAP) {
      const int n = min(CAP, z - k0);
      float* score = reinterpret_cast<float*>(w.key + kept);
      for (int i = tid; i < n; i += CH_THREADS) {
        const int k = k0 + i;
        const int64_t row = pool_row(c, s, b, h, k << c.page_log2);
        const int64_t at = row >> c.page_log2;   // page * H + h
        const uint32_t byte = row >= 0 ? scale[at] : 255u;
        const bool listed = k < sinks || (k >= lo && k <= own);
        w.at[i] = row >= 0 ? (int)(at / c.H) : -1;
        w.scale[i] = listed || byte == 255u ? 0.f : scale_of(byte);
        w.page[kept + i] = k;
        score[i] = -INFINITY;
      }
      for (int i = tid; i < kept; i += CH_THREADS) {
        w.key[i] = w.kept_key[i];
        w.page[i] = w.kept_page[i];
      }
#pragma unroll 1
      for (int r0 = 0; r0 < R; r0 += 64) {
        const int rows = min(64, R - r0), used = (rows + 15) & ~15;
        __syncthreads();   // (the last rows have been used)
#pragma unroll 4
        for (int r = warp; r < used; r += CH_THREADS / 32) {   // codes of the rows
          float x[D / 32];
          if (r < rows) {
            const int i = (r0 + r) / G, hq = h * G + (r0 + r) - i * G;
            const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(qp.p) + hq * qp.head + (int64_t)(q.r0 + i0 + i) * qp.row + lane * (D / 32);
            if (D == 128) {
              const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
              x[0] = __uint_as_float(v.x << 16);
              x[1] = __uint_as_float(v.x & 0xffff0000u);
              x[D / 32 - 2] = __uint_as_float(v.y << 16);
              x[D / 32 - 1] = __uint_as_float(v.y & 0xffff0000u);
            } else {
              const uint32_t v = __ldg(reinterpret_cast<const uint32_t*>(p));
              x[0] = __uint_as_float(v << 16);
              x[1] = __uint_as_float(v & 0xffff0000u);
            }
          } else {
#pragma unroll
            for (int k = 0; k < D / 32; ++k) x[k] = __int_as_float(0x7fffffff);
          }
          uint32_t top = 0;   // (bits of magnitudes order like the magnitudes, NaN above infinity)
#pragma unroll
          for (int k = 0; k < D / 32; ++k) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
          top = __reduce_max_sync(0xffffffffu, top);
          const bool fine = top < __float_as_uint(WILD);
          const int e = fine ? exponent_of(__uint_as_float(top)) : 0;
          const float f = fine ? pow2(-e) : 0.f;
#pragma unroll
          for (int k = 0; k < D / 32; ++k) w.q[r][lane * (D / 32) + k] = __float2half_rn(fine ? rintf(x[k] * f) : 0.f);
          if (lane == 0) w.unit[r] = fine ? pow2(e) : 0.f;
        }
        __syncthreads();
        // eight pages a warp: page j + g's codes, 16 bytes at 16 t (and at 64 + 16 t), the next eight's on their way
        auto codes = [&](int j, uint4 (&v)[D / 64]) {
          const int at = j + g < n ? w.at[j + g] : -1;
#pragma unroll
          for (int x = 0; x < D / 64; ++x)
            v[x] = at >= 0 ? __ldg(reinterpret_cast<const uint4*>(code + ((int64_t)at * c.H + h) * D + x * 64) + t) : make_uint4(0, 0, 0, 0);
        };
        uint4 v[D / 64];
        codes(warp * 8, v);
#pragma unroll 1
        for (int j0 = warp * 8; j0 < n; j0 += CH_THREADS / 32 * 8) {
          uint32_t B[D / 8];
#pragma unroll
          for (int x = 0; x < D / 64; ++x) {
            widen4(v[x].x, B[8 * x], B[8 * x + 1]);
            widen4(v[x].y, B[8 * x + 2], B[8 * x + 3]);
            widen4(v[x].z, B[8 * x + 4], B[8 * x + 5]);
            widen4(v[x].w, B[8 * x + 6], B[8 * x + 7]);
          }
          codes(j0 + CH_THREADS / 32 * 8, v);
          float best[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
          for (int mt = 0; mt < used; mt += 16) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f}, ac2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              const int col = (i >> 2) * 64 + t * 16 + (i & 3) * 4;
              const uint2 x = *reinterpret_cast<const uint2*>(&w.q[mt + g][col]);
              const uint2 y = *reinterpret_cast<const uint2*>(&w.q[mt + g + 8][col]);
              const uint32_t A[4] = {x.x, y.x, x.y, y.y};
              mma_f16(i & 1 ? ac2 : acc, A, B[2 * i], B[2 * i + 1]);
            }
            const float u0 = w.unit[mt + g], u1 = w.unit[mt + g + 8];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              if (u0 != 0.f) best[x] = fmaxf(best[x], (acc[x] + ac2[x]) * u0);
              if (u1 != 0.f) best[x] = fmaxf(best[x], (acc[2 + x] + ac2[2 + x]) * u1);
            }
          }
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) {
            best[0] = fmaxf(best[0], __shfl_xor_sync(0xffffffffu, best[0], o));
            best[1] = fmaxf(best[1], __shfl_xor_sync(0xffffffffu, best[1], o));
          }
          if (g < 2) {   // page 2 t + g of the eight
            const int x = j0 + 2 * t + g;
            if (x < n) {
              const float y = fmaxf(score[x], best[g]);
              if (r0 + 64 < R) score[x] = y;
              else w.key[kept + x] = w.scale[x] != 0.f && y > -INFINITY ? key_of(y * w.scale[x]) : 0;   // the last rows
            }
          }
        }
      }
      __syncthreads();
      keep_best(w, kept + n, how.top);
      kept = w.kept;
    }
  }
  if (C > 1) {
    if (tid == 0) w.kept = kept;
    cluster.sync();
    if (rank == 0) {   // the shares' best, in their order, and the best of those
      int n = 0;
      for (int r = 0; r < C; ++r) {
        Work<D>* o = cluster.map_shared_rank(&w, r);
        const int m2 = o->kept;
        for (int i = tid; i < m2; i += CH_THREADS) {
          w.key[n + i] = o->kept_key[i];
          w.page[n + i] = o->kept_page[i];
        }
        n += m2;
      }
      __syncthreads();
      keep_best(w, n, how.top);
      kept = w.kept;
    }
    cluster.sync();
    if (rank) return;
  }
  // sinks, then the chosen pages and the local ones as they ascend
  const int l0 = max(lo, sinks), locals = max(own - l0 + 1, 0);
  int before = 0;   // chosen pages before the local ones: a halving search
  for (int top = kept; before < top;) {
    const int mid = (before + top) / 2;
    if (w.kept_page[mid] < l0) before = mid + 1; else top = mid;
  }
  const int count = sinks + kept + locals;
  for (int i = tid; i < sinks; i += CH_THREADS) line[i] = i;
  for (int i = tid; i < locals; i += CH_THREADS) line[sinks + before + i] = l0 + i;
  for (int i = tid; i < kept; i += CH_THREADS) line[sinks + i + (i < before ? 0 : locals)] = w.kept_page[i];
  for (int i = count + tid; i < how.width; i += CH_THREADS) line[i] = -1;
}

}  // namespace

cudaError_t choose_set_smem_limits() {
  cudaError_t e = taken(cudaFuncSetAttribute(choose<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Work<128>)));
  if (e == cudaSuccess)
    e = taken(cudaFuncSetAttribute(choose<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Work<64>)));
  return e;
}

cudaError_t launch_summarise(const Pool& c, const Seqs& s, const int32_t* first, int8_t* code, uint8_t* scale, cudaStream_t st) {
  const int n_sm = sm_count();
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const int64_t units = (int64_t)s.max_pages * c.H;
  const dim3 grid((unsigned)std::min<int64_t>(units, std::max(1, 8 * n_sm / s.n)), s.n);
  auto* f = c.d == 128 ? (c.e4m3 ? summarise<128, true> : summarise<128, false>)
                       : (c.e4m3 ? summarise<64, true> : summarise<64, false>);
  return launch_kernel(f, grid, SUM_THREADS, 0, 1, false, st, c, s, first, code, scale);
}

cudaError_t launch_choose(const Pool& c, const Seqs& s, const int8_t* code, const uint8_t* scale, const Packed& q, int Hq,
                          const Choose& how, int32_t* lists, cudaStream_t st) {
  const int n_sm = sm_count();
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const int slots = s.rows / how.tile + s.n;
  int C = 1;
  const int64_t lines = (int64_t)std::min(slots, s.rows) * c.H;   // (a tile has a row or more)
  while (C < 8 && lines * C <= n_sm && s.max_pages / C > 128 && 2 * C * how.top <= MAX_TOP + CAP) C *= 2;
  const dim3 grid(slots * C, c.H);
  if (c.d == 128)
    return launch_kernel(choose<128>, grid, CH_THREADS, sizeof(Work<128>), C, false, st, c, s, code, scale, q, Hq / c.H, how, lists);
  return launch_kernel(choose<64>, grid, CH_THREADS, sizeof(Work<64>), C, false, st, c, s, code, scale, q, Hq / c.H, how, lists);
}

}  // namespace cache
}  // namespace dkv
