// Summaries of pages and the choice of pages by them (include/dkv.h: dkv_cache_summarise, dkv_cache_choose).
//
// A summary is the mean key of a page and head in 8 bits, so a page costs d + 1 bytes instead of its page_len rows.  The
// score of a query row and a page is a product of whole numbers (magnitudes up to 127, sums of d of them below 2^21) times
// a power of two: fp16 holds the numbers, the tensor cores' fp32 sums of them are exact in whatever order, and so
// the choice does not depend on how the work is split.  (In products of 8-bit whole numbers this GPU's tensor cores make 150 TOP/s,
// mma.sync in fp16 594.)  The means' sums are kept as pairs of fp32 numbers, exact to some 45 bits, so that
// their rounding to codes does not depend on the order either.
//
// Bound by latency: 32 tokens of 40 heads over up to 469 pages take 21 us in a graph (summaries 9, choice 16 by themselves), a chain of
// reads (sequence, table, scale, codes), three rounds of counting and two launches.  A block of 4,680 tokens in
// tiles of 64 over 732 pages, 12 heads: 55.5 us, 52 of them the choice: widening the codes for each tile of tokens 23 (shared memory is
// 50% busy, 33 KB in and out a tile of 128 pages), the queries' codes, looking for the best 48 4, the start of 888 CTAs and the
// summaries the rest.
#include "attn_math.cuh"
#include "cache_internal.h"
#include "tc_ptx.cuh"

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

// Units, a page and a head each, one sequence's behind the other's, go round the blocks (so many that all run at once; which
// sequence a unit is of, every warp finds from 32 sequences at a time).  A row lies with d / 8 threads; the rows' sums
// go over the warp, then one thread a column joins the warps'.  A whole past, 46,800 positions of 12 heads in pages of 64: 51 us in bf16 (HBM's
// share 21; the pair sums' instructions, 69% of the issue slots, and the waits of the joining), 79 in e4m3.
constexpr int SUM_BLOCKS = 6;   // of an SM

template <int D, bool E4M3>
__global__ void __launch_bounds__(SUM_THREADS, SUM_BLOCKS) summarise(Pool c, Seqs s, const int32_t* first, int8_t* code, uint8_t* scale) {
  constexpr int LANES = D / 8, ROWS = SUM_THREADS / LANES, WARPS = SUM_THREADS / 32;
  __shared__ Two part[WARPS][D];
  __shared__ float tops[D / 32];
  const int tid = threadIdx.x, lane = tid % LANES, r0 = tid / LANES;
  int64_t u = blockIdx.x;   // the block's next unit
#pragma unroll 1
  for (int b0 = 0; b0 < s.n; b0 += 32) {
    const int mine = b0 + (tid & 31);
    int from = 0, len = 0, pages = 0;
    if (mine < s.n) {
      const Seq q = seq_at(c, s, mine);
      len = q.len;
      from = max(first ? first[mine] : q.len - q.n, 0) >> c.page_log2;
      if (first || q.n > 0) pages = max(((len + c.page_len - 1) >> c.page_log2) - from, 0);
    }
    unsigned incl = pages;   // (32 of up to 2^26)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned y = __shfl_up_sync(0xffffffffu, incl, o);
      if ((tid & 31) >= o) incl += y;
    }
    const int64_t units = (int64_t)__shfl_sync(0xffffffffu, incl, 31) * c.H;
#pragma unroll 1
    for (; u < units; u += gridDim.x) {
      const int h = (int)(u % c.H);
      const unsigned place = (unsigned)(u / c.H);
      const int src = __ffs(__ballot_sync(0xffffffffu, incl > place)) - 1, b = b0 + src;
      const int k = (int)(place - __shfl_sync(0xffffffffu, incl - pages, src)) + __shfl_sync(0xffffffffu, from, src);
      const int page = s.table[(int64_t)b * s.max_pages + k];   // (the same for all threads; negative: given back)
      if (page >= c.n_pages) fail(c.status, DEV_INCONSISTENT, SITE_PAGE);
      const int64_t at = (unsigned)page < (unsigned)c.n_pages ? ((int64_t)page * c.H + h) << c.page_log2 : -1;
      const int held = min(c.page_len, __shfl_sync(0xffffffffu, len, src) - (k << c.page_log2));
      if (at < 0) continue;
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
    u -= units;
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

// A CTA's pages in shared memory.  `cap` pages are looked at in one go, behind what has been kept so far.
struct Work {
  uint32_t* key;      // [places] what has been kept, then this part's pages (first their best scores)
  int* page;          // [places]   ascending
  int* at;            // [cap] of this part's pages: place in the pool, -1
  float* scale;       // [cap]   and 2^e of the summary, 0: not to be listed
  float* other;       // [cap]   and the best scores of the second half of the rows (tensor cores)
  uint32_t* kept_key;   // [top]
  int* kept_page;
  struct Sums {
    uint32_t lo[8], hi[8];
    int total[8];
    int kept, step, here, above;
  }* sums;
  int* hist;          // [256]
};
struct Sizes {
  int cap, places, top;   // each a multiple of 4
};
__host__ __device__ inline size_t work_bytes(const Sizes& z) { return 8 * (size_t)z.places + 12 * (size_t)z.cap + 8 * (size_t)z.top + 128 + 1024; }
__device__ __forceinline__ Work work_in(uint8_t* p, const Sizes& z) {
  Work w;
  w.sums = reinterpret_cast<Work::Sums*>(p);
  w.hist = reinterpret_cast<int*>(p + 128);
  w.key = reinterpret_cast<uint32_t*>(p + 128 + 1024);
  w.page = reinterpret_cast<int*>(w.key + z.places);
  w.at = w.page + z.places;
  w.scale = reinterpret_cast<float*>(w.at + z.cap);
  w.other = w.scale + z.cap;
  w.kept_key = reinterpret_cast<uint32_t*>(w.other + z.cap);
  w.kept_page = reinterpret_cast<int*>(w.kept_key + z.top);
  return w;
}

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

// Four signed bytes c as two pairs of fp16 numbers (c + 128) 2^-24: the byte is the mantissa of a subnormal number.  (Sums of d of
// them times whole numbers up to 127 stay below 2^22 2^-24, exact in fp32; 128 times the other factors' sum goes off again.)
__device__ __forceinline__ void biased4(uint32_t w, uint32_t& a, uint32_t& b) {
  w ^= 0x80808080u;
  a = __byte_perm(w, 0u, 0x4140);
  b = __byte_perm(w, 0u, 0x4342);
}

// The `top` largest of key[0 .. n), equal ones: the first, in their order, into kept_key and kept_page.  Thread t holds
// places t PER ..; counts of the keys in 256 even steps between the least and the largest, then in 256 steps of the one that the
// top-th key lies in, and so on (two or three rounds as a rule), end at a bound with `top` keys above it, or at the top-th key
// itself where others equal it.
template <int THREADS, int PER>
__device__ __forceinline__ void keep_best(const Work& w, int n, int top) {
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
    w.sums->lo[warp] = least;
    w.sums->hi[warp] = most;
    w.sums->total[warp] = valid;
  }
  for (int i = tid; i < 256; i += THREADS) w.hist[i] = 0;
  __syncthreads();
  valid = 0;
#pragma unroll
  for (int x = 0; x < THREADS / 32; ++x) {
    least = min(least, w.sums->lo[x]);
    most = max(most, w.sums->hi[x]);
    valid += w.sums->total[x];
  }
  // keys > T are kept, and `need` of those equal to T
  uint32_t T = 0;
  int need = 0;
  if (valid > top) {
    uint32_t lo = least, span = most - least;   // (as a difference: what lies above lo may pass 32 bits)
    int shift = max(0, 24 - __clz(span)), left = top;   // (most - least) >> shift < 256; keys wanted from lo .. on
#pragma unroll 1
    for (;;) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (k[i] >= lo && k[i] - lo <= span) atomicAdd(&w.hist[(k[i] - lo) >> shift], 1);
      __syncthreads();
      if (warp == 0) {   // lane: steps 255 - 8 lane, .. downwards
        int own = 0, c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) own += c[i] = w.hist[255 - lane * 8 - i];
        int incl = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += y;
        }
        if (lane == __ffs(__ballot_sync(0xffffffffu, incl >= left)) - 1) {   // (there is one)
          int above = incl - own, step = 255 - lane * 8, here = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {   // (not by an index that varies)
            if (above + c[i] >= left) {
              here = c[i];
              break;
            }
            above += c[i];
            --step;
          }
          w.sums->step = step;
          w.sums->here = here;
          w.sums->above = above;
        }
      }
      __syncthreads();
      const int step = w.sums->step, here = w.sums->here;
      left -= w.sums->above;   // wanted of the step's
      lo += (uint32_t)step << shift;
      if (here == left) {      // all of them
        T = lo - 1;
        need = 0;
        break;
      }
      if (shift == 0) {        // equal ones
        T = lo;
        need = left;
        break;
      }
      span = (1u << shift) - 1;
      shift = max(0, shift - 8);
      for (int i = tid; i < 256; i += THREADS) w.hist[i] = 0;
      __syncthreads();
    }
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
  if (lane == 31) w.sums->total[warp] = incl;
  __syncthreads();
  int before = incl - mine, all = 0;
#pragma unroll
  for (int x = 0; x < THREADS / 32; ++x) {
    if (x < warp) before += w.sums->total[x];
    all += w.sums->total[x];
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
  if (tid == 0) w.sums->kept = (all & 0xffff) + min(all >> 16, need);
  __syncthreads();
}
template <int THREADS>
__device__ __forceinline__ void keep_best(const Work& w, int n, int top) {
  if (THREADS < CH_THREADS || n <= 4 * THREADS) keep_best<THREADS, 4>(w, n, top);
  else keep_best<THREADS, PLACES / THREADS>(w, n, top);
}

// One list: its tile of tokens and the pages that are listed anyway.
struct Line {
  int b, i0, m;       // sequence, first token, tokens
  Seq q;
  int whole;          // seen pages
  int lo, own;        // local pages
  int sinks;
  bool any;           // false: no tile, or one that sees nothing
};
__device__ __forceinline__ Line line_of(const Pool& c, const Seqs& s, const Choose& how, int slot) {
  Line l{};
  l.b = seq_of_slot_warp(c, s, how.tile, slot, l.q);
  l.i0 = (slot - l.q.r0 / how.tile - l.b) * how.tile;
  l.m = min(how.tile, l.q.n - l.i0);
  const int p1 = l.q.len - l.q.n + l.i0 + l.m - 1, p0 = max(p1 - l.m + 1, 0);
  l.any = l.i0 >= 0 && l.m > 0 && p1 >= 0;
  if (!l.any) return l;
  const Mask mask{0.f, 0, 0, how.block, how.inverse};
  const int end = visible_end(mask, p0, l.q.len);
  l.whole = end == l.q.len ? (l.q.len + c.page_len - 1) >> c.page_log2 : end >> c.page_log2;
  l.own = p1 >> c.page_log2;
  l.lo = max(0, (p0 >> c.page_log2) - (how.local - 1));
  l.sinks = min(how.sinks, l.whole);
  return l;
}

// Pages k0 .. k0 + n - 1 looked up, behind the `kept` ones.
template <int THREADS>
__device__ __forceinline__ void look_up(const Pool& c, const Seqs& s, const Work& w, const Line& l, const uint8_t* scale, int h,
                                        int k0, int n, int kept) {
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int k = k0 + i;
    int page = s.table[(int64_t)l.b * s.max_pages + k];   // (negative: given back)
    if (page >= c.n_pages) {
      fail(c.status, DEV_INCONSISTENT, SITE_PAGE);
      page = -1;
    }
    page = max(page, -1);
    const uint32_t byte = page >= 0 ? __ldg(scale + (int64_t)page * c.H + h) : 255u;
    const bool listed = k < l.sinks || (k >= l.lo && k <= l.own);
    w.at[i] = page;
    w.scale[i] = listed || byte == 255u ? 0.f : scale_of(byte);
    w.other[i] = -INFINITY;
    w.page[kept + i] = k;
    reinterpret_cast<float*>(w.key)[kept + i] = -INFINITY;
  }
  for (int i = threadIdx.x; i < kept; i += THREADS) {
    w.key[i] = w.kept_key[i];
    w.page[i] = w.kept_page[i];
  }
}

struct Job {
  Pool c;
  Seqs s;
  const int8_t* code;
  const uint8_t* scale;
  Packed q;
  int G;
  uint32_t g_inverse;   // ceil(2^32 / G): r / G is the high half of r times it (G > 1, r < 2^14)
  Choose how;
  int32_t* lists;
  Sizes z;
};

// A warp's query row r of the tile (row = token * G + head), lane's D / 32 numbers of it; a row behind the last: infinities.
template <int D>
__device__ __forceinline__ uint2 row_load(const Job& j, const Line& l, int h, int r, int R) {
  const int lane = threadIdx.x & 31;
  const Packed& qp = j.q;
  if (r >= R) return make_uint2(0x7f807f80u, 0x7f807f80u);
  const int i = j.G == 1 ? r : (int)__umulhi((uint32_t)r, j.g_inverse), hq = h * j.G + r - i * j.G;
  const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(qp.p) + hq * qp.head + (int64_t)(l.q.r0 + l.i0 + i) * qp.row + lane * (D / 32);
  if (D == 128) return __ldg(reinterpret_cast<const uint2*>(p));
  return make_uint2(__ldg(reinterpret_cast<const uint32_t*>(p)), 0u);
}
// The numbers as whole ones, and the row's power of two (0: no codes).
template <int D>
__device__ __forceinline__ float row_codes(const uint2& v, float (&x)[D / 32]) {
  x[0] = __uint_as_float(v.x << 16);
  x[1] = __uint_as_float(v.x & 0xffff0000u);
  if (D == 128) {
    x[D / 32 - 2] = __uint_as_float(v.y << 16);
    x[D / 32 - 1] = __uint_as_float(v.y & 0xffff0000u);
  }
  uint32_t top = 0;   // (bits of magnitudes order like the magnitudes, NaN above infinity)
#pragma unroll
  for (int k = 0; k < D / 32; ++k) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
  top = __reduce_max_sync(0xffffffffu, top);
  const bool fine = top < __float_as_uint(WILD);
  const int e = fine ? exponent_of(__uint_as_float(top)) : 0;
  const float f = fine ? pow2(-e) : 0.f;
#pragma unroll
  for (int k = 0; k < D / 32; ++k) x[k] = fine ? rintf(x[k] * f) : 0.f;
  return fine ? pow2(e) : 0.f;
}

// The cluster's shares joined, and the list written: sinks, then the chosen pages and the local ones as they ascend.
template <int THREADS>
__device__ __forceinline__ void finish(const Work& w, const Line& l, int kept, int top, int32_t* line, int width) {
  cg::cluster_group cluster = cg::this_cluster();
  const int C = cluster.num_blocks(), rank = cluster.block_rank(), tid = threadIdx.x;
  if (C > 1) {
    if (tid == 0) w.sums->kept = kept;
    cluster.sync();
    if (rank == 0) {   // the shares' best, in their order, and the best of those
      int n = 0;
      for (int r = 0; r < C; ++r) {
        const uint32_t* key = cluster.map_shared_rank(w.kept_key, r);
        const int* page = cluster.map_shared_rank(w.kept_page, r);
        const int m2 = cluster.map_shared_rank(w.sums, r)->kept;
        for (int i = tid; i < m2; i += THREADS) {
          w.key[n + i] = key[i];
          w.page[n + i] = page[i];
        }
        n += m2;
      }
      __syncthreads();
      keep_best<THREADS>(w, n, top);
      kept = w.sums->kept;
    }
    cluster.sync();
    if (rank) return;
  }
  const int l0 = max(l.lo, l.sinks), locals = max(l.own - l0 + 1, 0);
  int before = 0;   // chosen pages before the local ones: a halving search
  for (int z = kept; before < z;) {
    const int mid = (before + z) / 2;
    if (w.kept_page[mid] < l0) before = mid + 1; else z = mid;
  }
  const int count = l.sinks + kept + locals;
  for (int i = tid; i < l.sinks; i += THREADS) line[i] = i;
  for (int i = tid; i < locals; i += THREADS) line[l.sinks + before + i] = l0 + i;
  for (int i = tid; i < kept; i += THREADS) line[l.sinks + i + (i < before ? 0 : locals)] = w.kept_page[i];
  for (int i = count + tid; i < width; i += THREADS) line[i] = -1;
}

// Cluster: one list (slot blockIdx.x / CTAs of the cluster, head blockIdx.y); its CTAs share the seen pages.  (CTAs of fewer
// threads hold up to 4 pages a thread, and come without a cluster.)  Few query rows (a single token's group): mma.sync, the rows its 16, the pages its 8 columns.
constexpr int FEW = 16;

template <int D, int THREADS>
__global__ void __launch_bounds__(THREADS, 3 * (CH_THREADS / THREADS)) choose(const __grid_constant__ Job j) {
  constexpr int STRIDE = D + 4;   // halves of a row: 8-byte reads of 4 lanes x 4 rows touch every bank once
  extern __shared__ __align__(16) uint8_t raw[];
  __half* qs = reinterpret_cast<__half*>(raw);                              // [FEW][STRIDE]
  float* unit = reinterpret_cast<float*>(raw + FEW * STRIDE * 2);           // 2^e of a row, 0: none
  const Work w = work_in(raw + FEW * STRIDE * 2 + FEW * 4, j.z);
  const Pool& c = j.c;
  const int C = cg::this_cluster().num_blocks(), rank = cg::this_cluster().block_rank();
  const int slot = blockIdx.x / C, h = blockIdx.y, slots = gridDim.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  if (blockIdx.x == 0 && h == 0)
    for (int b = tid; b < j.s.n; b += THREADS) seq_at(c, j.s, b);
  const Line l = line_of(c, j.s, j.how, slot);
  int32_t* line = j.lists + ((int64_t)h * slots + slot) * j.how.width;
  if (!l.any) {   // (the whole cluster)
    if (rank == 0)
      for (int k = tid; k < j.how.width; k += THREADS) line[k] = -1;
    return;
  }
  const int R = l.m * j.G;   // <= FEW
  // this CTA's share of the seen pages
  const int per = (l.whole + C - 1) / C, a = min(rank * per, l.whole), z = min(a + per, l.whole);
  int kept = 0;
  if (j.how.top > 0) {
    for (int r = warp; r < FEW; r += THREADS / 32) {   // (their codes made after the pages are looked up: 47,888 lists 170 us, 160 so)
      float x[D / 32];
      const float u = row_codes<D>(row_load<D>(j, l, h, r, R), x);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) qs[r * STRIDE + lane * (D / 32) + k] = __float2half_rn(x[k]);
      if (lane == 0) unit[r] = u;
    }
#pragma unroll 1
    for (int k0 = a; k0 < z; k0 += j.z.cap) {
      const int n = min(j.z.cap, z - k0);
      look_up<THREADS>(c, j.s, w, l, j.scale, h, k0, n, kept);
      __syncthreads();
      // eight pages a warp: page i + g's codes, 16 bytes at 16 t (and at 64 + 16 t), the next eight's on their way
      auto codes = [&](int i, uint4 (&v)[D / 64]) {
        const int at = i + g < n ? w.at[i + g] : -1;
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
          v[x] = at >= 0 ? __ldg(reinterpret_cast<const uint4*>(j.code + ((int64_t)at * c.H + h) * D + x * 64) + t) : make_uint4(0, 0, 0, 0);
      };
      uint4 v[D / 64];
      codes(warp * 8, v);
      const float u0 = unit[g], u1 = unit[g + 8];
#pragma unroll 1
      for (int i0 = warp * 8; i0 < n; i0 += THREADS / 32 * 8) {
        uint32_t B[D / 8];
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          widen4(v[x].x, B[8 * x], B[8 * x + 1]);
          widen4(v[x].y, B[8 * x + 2], B[8 * x + 3]);
          widen4(v[x].z, B[8 * x + 4], B[8 * x + 5]);
          widen4(v[x].w, B[8 * x + 6], B[8 * x + 7]);
        }
        codes(i0 + THREADS / 32 * 8, v);
        float acc[4] = {0.f, 0.f, 0.f, 0.f}, ac2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const int col = (i >> 2) * 64 + t * 16 + (i & 3) * 4;
          const uint2 x = *reinterpret_cast<const uint2*>(qs + g * STRIDE + col);
          const uint2 y = *reinterpret_cast<const uint2*>(qs + (g + 8) * STRIDE + col);
          const uint32_t A[4] = {x.x, y.x, x.y, y.y};
          mma_f16(i & 1 ? ac2 : acc, A, B[2 * i], B[2 * i + 1]);
        }
        float best[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (u0 != 0.f) best[x] = (acc[x] + ac2[x]) * u0;
          if (u1 != 0.f) best[x] = fmaxf(best[x], (acc[2 + x] + ac2[2 + x]) * u1);
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          best[0] = fmaxf(best[0], __shfl_xor_sync(0xffffffffu, best[0], o));
          best[1] = fmaxf(best[1], __shfl_xor_sync(0xffffffffu, best[1], o));
        }
        if (g < 2) {   // page 2 t + g of the eight
          const int x = i0 + 2 * t + g;
          if (x < n) w.key[kept + x] = w.scale[x] != 0.f && best[g] > -INFINITY ? key_of(best[g] * w.scale[x]) : 0;
        }
      }
      __syncthreads();
      keep_best<THREADS>(w, kept + n, j.how.top);
      kept = w.sums->kept;
    }
  }
  finish<THREADS>(w, l, kept, j.how.top, line, j.how.width);
}

// The same for many query rows on the tensor cores, turned round: 128 pages are the rows of tcgen05.mma, 64 or 128 query rows its
// columns, so that a thread's part of the result is one page, whose best score it finds by itself.  Two halves of the
// threads take half of the query rows each.  Codes are widened to fp16 by all threads; a tile's product runs
// while the last one's result is looked through.
template <int D, int ROWS>
struct TcLay {
  static constexpr int NP = D / 64;
  static constexpr int A = 0;                            // [NP][128 pages][64] swizzled
  static constexpr int B = NP * 128 * 128;               // [NP][ROWS][64]
  static constexpr int UNIT = B + NP * ROWS * 128;             // [ROWS] 2^e, [ROWS] 0 or -inf
  static constexpr int CTRL = UNIT + 8 * ROWS;
  static constexpr int WORK = CTRL + 32;
};

template <int D, int ROWS>
__global__ void __launch_bounds__(CH_THREADS, ROWS == 64 ? 3 : 2) choose_tc(const __grid_constant__ Job j) {
  using namespace tc;
  using L = TcLay<D, ROWS>;
  constexpr uint32_t TMEM = 2 * ROWS;   // columns: two results
  extern __shared__ __align__(1024) uint8_t tile[];
  const Work w = work_in(tile + L::WORK, j.z);
  float* unit = reinterpret_cast<float*>(tile + L::UNIT);
  uint64_t* done = reinterpret_cast<uint64_t*>(tile + L::CTRL);
  uint32_t* holder = reinterpret_cast<uint32_t*>(done + 1);
  const Pool& c = j.c;
  const int C = cg::this_cluster().num_blocks(), rank = cg::this_cluster().block_rank();
  const int slot = blockIdx.x / C, h = blockIdx.y, slots = gridDim.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (blockIdx.x == 0 && h == 0)
    for (int b = tid; b < j.s.n; b += CH_THREADS) seq_at(c, j.s, b);
  const Line l = line_of(c, j.s, j.how, slot);
  int32_t* line = j.lists + ((int64_t)h * slots + slot) * j.how.width;
  if (!l.any) {   // (the whole cluster)
    if (rank == 0)
      for (int k = tid; k < j.how.width; k += CH_THREADS) line[k] = -1;
    return;
  }
  if ((smem_u32(tile) & 1023u) != 0u) {   // 128-byte-swizzled tiles need 1024-byte alignment
    if (tid == 0) fail(c.status, DEV_INCONSISTENT, 9905);
    return;
  }
  if (tid == 0) {
    mbar_init(done, 1);
    fence_barrier_init();
  }
  if (warp == 0) tmem_alloc(holder, TMEM);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *holder;
  constexpr uint32_t idesc = idesc_bf16(128, ROWS) & ~((1u << 7) | (1u << 10));   // fp16
  const uint64_t ad = desc_sw128(smem_u32(tile + L::A)), bd = desc_sw128(smem_u32(tile + L::B));
  const int R = l.m * j.G;
  const int per = (l.whole + C - 1) / C, a = min(rank * per, l.whole), z = min(a + per, l.whole);
  const int half = warp >> 2;
  const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
  volatile int no_abort = 0;
  int kept = 0;
  uint32_t phase = 0;
  bool ok = true;
  if (j.how.top > 0) {
#pragma unroll 1
    for (int k0 = a; ok && k0 < z; k0 += j.z.cap) {
      const int n = min(j.z.cap, z - k0);
      float* score = half ? w.other : reinterpret_cast<float*>(w.key) + kept;
#pragma unroll 1
      for (int r0 = 0; ok && r0 < R; r0 += ROWS) {
        // rows, then the pages, then their first codes are asked for before the rows' codes are made
        constexpr int PER = 8;   // of a warp in one go
        uint2 rows[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) rows[k] = row_load<D>(j, l, h, r0 + warp + k * (CH_THREADS / 32), R);
        if (r0 == 0) {
          look_up<CH_THREADS>(c, j.s, w, l, j.scale, h, k0, n, kept);
          __syncthreads();
        }
        // 16-byte parts of a tile's codes: eight threads take four parts (64 columns) of two neighbouring rows, so that their
        // stores, swizzled by the row, touch every bank once
        constexpr int V = 128 * (D / 16) / CH_THREADS, STEP = CH_THREADS / 4 / L::NP;
        const int part = tid & 3, panel = (tid >> 3) % L::NP, p0 = (tid >> 3) / L::NP * 2 + ((tid >> 2) & 1);
        const int8_t* const from = j.code + (int64_t)h * D + panel * 64 + part * 16;
        auto codes = [&](int i0, uint4 (&v)[V]) {
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const int i = i0 + p0 + k * STEP, at = i < n ? w.at[i] : -1;
            v[k] = at >= 0 ? __ldg(reinterpret_cast<const uint4*>(from + (int64_t)at * (c.H * D))) : make_uint4(0, 0, 0, 0);
          }
        };
        uint4 v[V];
        codes(0, v);
        // (the products that read the last rows are complete, and nobody looks through their result any more)
#pragma unroll 1
        for (int k0 = 0;; k0 += PER) {
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            const int r = warp + (k0 + k) * (CH_THREADS / 32);
            float x[D / 32];
            const float u = row_codes<D>(rows[k], x);
            const int col = lane * (D / 32), at = (col >> 6) * (ROWS * 128) + r * 128 + ((((col & 63) >> 3) ^ (r & 7)) << 4) + (col & 7) * 2;
            const __half2 y = __floats2half2_rn(x[0], x[1]);
            if (D == 128) {
              const __half2 y2 = __floats2half2_rn(x[D / 32 - 2], x[D / 32 - 1]);
              *reinterpret_cast<uint2*>(tile + L::B + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&y), *reinterpret_cast<const uint32_t*>(&y2));
            } else {
              *reinterpret_cast<uint32_t*>(tile + L::B + at) = *reinterpret_cast<const uint32_t*>(&y);
            }
            float sum = 0.f;   // (whole numbers)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) sum += x[i];
            sum = (float)__reduce_add_sync(0xffffffffu, (int)sum);
            if (lane == 0) {
              unit[r] = u * 0x1p24f;
              unit[ROWS + r] = u != 0.f ? -128.f * sum * u : -INFINITY;
            }
          }
          if (k0 + PER >= ROWS / (CH_THREADS / 32)) break;
#pragma unroll
          for (int k = 0; k < PER; ++k) rows[k] = row_load<D>(j, l, h, r0 + warp + (k0 + PER + k) * (CH_THREADS / 32), R);
        }
        auto look = [&](int i0, uint32_t buf) {   // the best of the half's rows for this thread's page
          float best = -INFINITY;
#pragma unroll 1
          for (int k0 = half * (ROWS / 2); k0 < (half + 1) * (ROWS / 2) && k0 < R - r0; k0 += 32) {
            float x[32];
            tmem_ld32(tmem + lane_off + buf * ROWS + k0, x);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const float4 u = *reinterpret_cast<const float4*>(unit + k0 + k), o = *reinterpret_cast<const float4*>(unit + ROWS + k0 + k);
              const float2 y = __ffma2_rn(make_float2(x[k], x[k + 1]), make_float2(u.x, u.y), make_float2(o.x, o.y));
              const float2 y2 = __ffma2_rn(make_float2(x[k + 2], x[k + 3]), make_float2(u.z, u.w), make_float2(o.z, o.w));
              best = max3(max3(best, y.x, y.y), y2.x, y2.y);
            }
          }
          const int i = i0 + (warp & 3) * 32 + lane;
          if (i < n) score[i] = fmaxf(score[i], best);
        };
        uint32_t buf = 0;
#pragma unroll 1
        for (int i0 = 0; ok && i0 < n; i0 += 128, buf ^= 1) {
          uint8_t* const to = tile + L::A + panel * (128 * 128) + p0 * 128;
#pragma unroll
          for (int k = 0; k < V; ++k) {
            uint32_t x[8];
            biased4(v[k].x, x[0], x[1]);
            biased4(v[k].y, x[2], x[3]);
            biased4(v[k].z, x[4], x[5]);
            biased4(v[k].w, x[6], x[7]);
            static_assert(STEP % 8 == 0, "a thread's rows share their swizzle");
            *reinterpret_cast<uint4*>(to + k * STEP * 128 + (((2 * part) ^ (p0 & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<uint4*>(to + k * STEP * 128 + (((2 * part + 1) ^ (p0 & 7)) << 4)) = make_uint4(x[4], x[5], x[6], x[7]);
          }
          fence_async_smem();
          fence_before_sync();   // (results looked through before they are overwritten)
          __syncthreads();
          if (warp == 0) {
            fence_after_sync();
            if (elect_one()) {
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk)
                mma_bf16(tmem + buf * ROWS, desc_add(ad, (kk >> 2) * (128 * 128) + (kk & 3) * 32),
                         desc_add(bd, (kk >> 2) * (ROWS * 128) + (kk & 3) * 32), idesc, kk > 0);
              mma_commit(done);
            }
            __syncwarp();
          }
          codes(i0 + 128, v);
          if (i0 > 0) {
            fence_after_sync();
            look(i0 - 128, buf ^ 1);
          }
          ok = mbar_wait(done, phase, &no_abort);
          phase ^= 1;
          ok = __syncthreads_and(ok) != 0;
          fence_after_sync();
        }
        if (ok) look((n - 1) / 128 * 128, buf ^ 1);
        fence_before_sync();
        __syncthreads();
      }
      for (int i = tid; i < n; i += CH_THREADS) {
        const float x = fmaxf(reinterpret_cast<float*>(w.key)[kept + i], w.other[i]);
        w.key[kept + i] = w.scale[i] != 0.f && x > -INFINITY ? key_of(x * w.scale[i]) : 0;
      }
      __syncthreads();
      keep_best<CH_THREADS>(w, kept + n, j.how.top);
      kept = w.sums->kept;
    }
  }
  if (!ok && tid == 0) fail(c.status, DEV_TIMEOUT, SITE_WAIT + 20);
  __syncthreads();
  if (warp == 0) {
    fence_after_sync();
    tmem_dealloc(tmem, TMEM);
  }
  finish<CH_THREADS>(w, l, kept, j.how.top, line, j.how.width);
}

}  // namespace

namespace {
template <int D>
size_t few_bytes(const Sizes& z) {
  return FEW * (D + 4) * 2 + FEW * 4 + work_bytes(z);
}
template <int D, int ROWS>
size_t tc_bytes(const Sizes& z) {
  return TcLay<D, ROWS>::WORK + work_bytes(z);
}
template <int D>
cudaError_t choose_limits() {
  const Sizes z{CAP, PLACES, MAX_TOP};
  cudaError_t e = taken(cudaFuncSetAttribute(choose<D, CH_THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_bytes<D>(z)));
  if (e == cudaSuccess)
    e = taken(cudaFuncSetAttribute(choose_tc<D, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc_bytes<D, 64>(z)));
  if (e == cudaSuccess)
    e = taken(cudaFuncSetAttribute(choose_tc<D, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc_bytes<D, 128>(z)));
  return e;
}
template <int D>
cudaError_t launch_choose_d(const Job& job, int slots, int C, bool few, int threads, cudaStream_t st) {
  const dim3 grid(slots * C, job.c.H);
  if (few && threads == 32) return launch_kernel(choose<D, 32>, grid, 32, few_bytes<D>(job.z), 1, false, st, job);
  if (few && threads == 64) return launch_kernel(choose<D, 64>, grid, 64, few_bytes<D>(job.z), 1, false, st, job);
  if (few) return launch_kernel(choose<D, CH_THREADS>, grid, CH_THREADS, few_bytes<D>(job.z), C, false, st, job);
  // More than 128 rows: 128 a product, so that the codes are widened half as often, but two CTAs an SM (4,680 tokens over 732 pages: 768
  // rows 62 us, 101 by 64; 256 rows of d = 64 36 and 50; 320 rows 154 and 182; 128 rows 55 and 49).
  if ((int64_t)std::min(job.how.tile, job.s.rows) * job.G > 128)
    return launch_kernel(choose_tc<D, 128>, grid, CH_THREADS, tc_bytes<D, 128>(job.z), C, false, st, job);
  return launch_kernel(choose_tc<D, 64>, grid, CH_THREADS, tc_bytes<D, 64>(job.z), C, false, st, job);
}
}  // namespace

cudaError_t choose_set_smem_limits() {
  const cudaError_t e = choose_limits<128>();
  return e == cudaSuccess ? choose_limits<64>() : e;
}

cudaError_t launch_summarise(const Pool& c, const Seqs& s, const int32_t* first, int8_t* code, uint8_t* scale, cudaStream_t st) {
  const int n_sm = sm_count();
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const int64_t most = (int64_t)s.max_pages * c.H * s.n;
  const dim3 grid((unsigned)std::min<int64_t>(most, SUM_BLOCKS * n_sm));
  auto* f = c.d == 128 ? (c.e4m3 ? summarise<128, true> : summarise<128, false>)
                       : (c.e4m3 ? summarise<64, true> : summarise<64, false>);
  return launch_kernel(f, grid, SUM_THREADS, 0, 1, false, st, c, s, first, code, scale);
}

cudaError_t launch_choose(const Pool& c, const Seqs& s, const int8_t* code, const uint8_t* scale, const Packed& q, int Hq,
                          const Choose& how, int32_t* lists, cudaStream_t st) {
  const int n_sm = sm_count();
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const int slots = s.rows / how.tile + s.n, G = Hq / c.H;
  const int64_t lines = (int64_t)std::min(slots, s.rows) * c.H;   // (a tile has a row or more)
  // few lists: a cluster each (one token over 2,047 pages, 8 heads: 8 CTAs a list 21 us, 1 29; 256 lists of 469 pages: 1 CTA 21,
  // 2 29)
  int C = 1;
  while (C < 8 && lines * C <= n_sm && s.max_pages / C > 128 && 2 * C * how.top <= PLACES) C *= 2;
  auto four = [](int x) { return (x + 3) / 4 * 4; };
  Sizes z;
  z.top = four(how.top);
  z.cap = std::min(CAP, four((s.max_pages + C - 1) / C));
  z.places = std::max(z.cap + z.top, four(C * how.top));
  const Job job{c, s, code, scale, q, G, (uint32_t)((0x100000000ull + G - 1) / G), how, lists, z};
  // (32 tokens of 5 or of 16 rows: the kernel for few rows 21 us, the other 26)
  const bool few = (int64_t)std::min(how.tile, s.rows) * G <= FEW;
  // many short lists: a warp or two each, so that 24 or 12 run on an SM instead of 3 (47,888 lists of up to 94 pages 160 us with one warp, 221
  // with two, 554 with eight; 3,200 of up to 146 62 with two, 91 with eight; 480 18.7 and 20.6, 256 18.5 and 16.5)
  int threads = CH_THREADS;
  if (C == 1 && lines > 3 * n_sm) threads = z.places <= 4 * 32 ? 32 : z.places <= 4 * 64 ? 64 : CH_THREADS;
  return c.d == 128 ? launch_choose_d<128>(job, slots, C, few, threads, st) : launch_choose_d<64>(job, slots, C, few, threads, st);
}

}  // namespace cache
}  // namespace dkv
