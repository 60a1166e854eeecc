// Attention of few query rows over the paged cache (include/dkv.h: dkv_cache_attend): single tokens
// and a handful of drafted ones.  Every key and value is read once and used by at most 16 rows, so
// HBM bounds it (4 d bytes a position and key head in bf16, 2 d + 2 in e4m3); the arithmetic only
// has to keep out of the way.
//
// A unit is 8 or 16 query rows of one sequence and one key head, row = token * G + head.  The visible
// positions of all units, in stages of KT, form one range, and each of the GPU's warps
// takes an equal stretch of it, whatever units it belongs to: no warp waits for another, and the
// split over a long cache, over many sequences and over ragged lengths is the same one.  A unit inside one
// stretch is finished there; one that a boundary cuts leaves a partial result for each warp that
// holds some of it: a CTA joins its own warps' parts, and of the CTAs that share a unit the one that is
// done last joins theirs, in the order of the CTAs (a second kernel for it took 2 us of the GPU's time
// and 3 of the host's, as long as the rest of a small call).
//
// A warp streams its stages through a ring of its own (TMA boxes of one page, 128-byte swizzled;
// a lane issues each, a barrier a slot) and works on them with mma.sync m16n8k16, turned round: the 16 rows
// of a product are keys or columns of the values and its 8 columns the query rows,
//   S^T = K Q^T,   O^T += V^T P^T,
// so that 8 query rows (a single token's group of heads) fill a product; with the query rows as its 16 rows
// every product, weight and register was at least half empty (and the tensor cores' tiles of 128 rows
// would be empty but for a sixteenth).  The weights' registers become an operand by one
// transposing move for 8 keys.  Running maximum, sum and outputs stay in registers.
//
// e4m3: the keys' codes become fp16 in the registers, one conversion for two; the scales join the scores.  A key row's 128
// codes lie with four lanes, 32 neighbouring ones each, and the queries' registers are loaded in that order of d
// instead of the product's own.  The values become bf16 with their scales in them, by bit operations (widen_values), for
// weights in bf16 as a bf16 cache has them: in fp16 the weights would have to carry the scales, relative to the largest such
// product, and what is 2^-24 below that would be lost (beside a row of zeros, whose scale is 2^0, all of a row of ordinary
// size).  Of the values, a transposed load gives pairs of d of one position, which widen into the even and the odd ones of 16.
// (With fp16 weights, whose sums had to be kept apart, 32 tokens of 40 on 8 heads took as long: 70.6 us a call for 70.4.)
//
// Measured: one token of 12 heads over 131,001 positions in bf16 127 us, 6.3 TB/s of the 6.8 that a copy reaches (in
// e4m3 75 us, 5.4); 32 tokens of 40 on 8 heads over up to 9,360 positions in e4m3 68 us (5.1 TB/s), in bf16 115 (6.0).
// About 9 us of each are fixed (reading the arrays, the first keys' way, the joining): one token over 1,561 positions 11 us.
#include "attn_math.cuh"
#include "cache_internal.h"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

namespace dkv {

bool make_map_4d(CUtensorMap* m, const void* base, int elem_bytes, const int64_t (&dim)[4], const int64_t (&stride)[3],
                 const int (&box)[4], int swizzle);

namespace cache {

namespace {

using namespace tc;

constexpr int MAX_CTAS = 152;
constexpr int MAX_WARPS = 12;
constexpr int WORKERS = MAX_WARPS * MAX_CTAS;
constexpr float RESCALE_LOG2 = 8.0f;
constexpr int MIN_STAGES = 1;    // stages of a warp, at least (one token over 1,561 positions: with 1 11 us, 2 15, 4 19)

// What a worker's stretch leaves unfinished.
struct Stretch {
  int head;            // 1: a part of a unit that began before it
  int head_smem;       //   and its part is in the warp's ring: the stretch's last unit, nothing follows
  int head_ends;       //   that ends in it
  int tail;            // 1: a first part of a unit that goes on behind it
  int first, last;     // CTAs of the head's unit's first stage and of the tail's unit's last one
  int hlast;           // CTA of the head's unit's last stage
  int h, tile, rows, r0;      // of the tail's unit
  int hh, htile, hrows, hr0;  // of the head's
};

template <int D, bool E4M3, int NR>
struct Lay {
  static constexpr int ES = E4M3 ? 1 : 2;
  static constexpr int KT = !E4M3 && D == 128 ? 16 : 32;   // positions of a stage
  static constexpr int PANEL = KT * (E4M3 ? D : 128);      // bytes of a panel (64 columns; codes: all)
  static constexpr int TILE = KT * D * ES;                 // bytes of a stage's keys
  static constexpr int WARPS = NR == 1 ? 12 : 8;           // (as many as the registers allow)
  static constexpr int SLOTS = NR == 1 ? 2 : 3;
  static constexpr int SLOT = 2 * TILE;                    // keys, values
  static constexpr int RING = SLOTS * SLOT;                // a warp's
  static constexpr int SCALES = WARPS * RING;              // [warps][slots][2][KT] scale bytes
  static constexpr int BARS = SCALES + (E4M3 ? WARPS * SLOTS * 2 * KT : 0);
  static constexpr int INFO = BARS + WARPS * SLOTS * 8;
  static constexpr int BYTES = INFO + WARPS * (int)sizeof(Stretch) + 16;
  static_assert(BYTES <= 227 * 1024, "shared memory per CTA");
  static_assert(16 * (D + 4) * 4 <= RING, "a part in the ring");
};

struct Job {
  Pool c;
  Seqs s;
  Mask m;
  Packed q, o;
  int G, max_rows;
  uint32_t g_inverse;   // ceil(2^32 / G): i / G is the high half of i times it (i < 2^24)
  int unit;          // rows of a unit
  int part_rows;     // rows of a partial result
  float* parts;      // partial results, [part_rows][D + 4] each (outputs, then the logarithm of a row's sum): one of every
                     //   worker (a unit that its stretch begins in the middle of and goes on behind; its last unit's
                     //   stays in shared memory), then two of every CTA (a unit from before it, one that goes on behind)
  unsigned long long* arrived;   // [MAX_CTAS] CTAs that are done with the unit that begins in a CTA and goes on behind it: the
                     //   call's number << ROWS_COUNT_BITS | their count; anything else counts as none (the scratch comes as it is)
  unsigned long long call;
};

// One sequence's share of the range.
struct Span {
  int r0, n, len;
  int tiles;         // row tiles of a key head
  int ns, w0, stages;   // stages 0 .. ns - 1 (sinks), then w0, w0 + 1, ..; at least one
  int lo, end, sk;   // positions that some token sees
  int all_end, all_lo;  // positions that every token sees: [all_lo, all_end) and below all_sk
};

template <int KT>
__device__ __forceinline__ Span span_of(const Job& j, int b) {
  Span x{};
  const Seq q = seq_at(j.c, j.s, b);
  x.r0 = q.r0;
  x.n = q.n;
  x.len = q.len;
  if (q.n == 0) return x;
  x.tiles = (q.n * j.G + j.unit - 1) >> (j.unit == 8 ? 3 : 4);
  x.stages = 1;
  const int p0 = q.len - q.n, pl = q.len - 1;
  if (pl < 0) return x;
  const int e0 = visible_end(j.m, max(p0, 0), q.len);
  x.end = visible_end(j.m, pl, q.len);
  x.lo = window_first(j.m, e0);
  x.sk = j.m.window ? min(j.m.sinks, x.end) : 0;
  x.all_end = p0 >= 0 ? e0 : 0;
  x.all_lo = window_first(j.m, x.end);
  x.ns = (x.sk + KT - 1) / KT;
  x.w0 = max(x.ns, x.lo / KT);
  x.stages = max(1, x.ns + max(0, (x.end + KT - 1) / KT - x.w0));
  return x;
}

__device__ __forceinline__ int token_of(const Job& j, int i) { return j.G == 1 ? i : (int)__umulhi((uint32_t)i, j.g_inverse); }

__device__ __forceinline__ int stages_of(const Job& j, const Span& x) { return x.tiles * j.c.H * x.stages; }

// Stages of the whole range; `first`: the span of sequence `lane`.  All lanes of a warp.  None where a row_start that goes
// back and forth gives the sequences more rows than the call has.
template <int KT>
__device__ __forceinline__ int total_stages(const Job& j, Span& first) {
  const int lane = threadIdx.x & 31;
  int64_t mine = 0;
  unsigned claimed = 0;
  first = Span{};
  for (int b = lane; b < j.s.n; b += 32) {
    const Span x = span_of<KT>(j, b);
    if (b == lane) first = x;
    if (x.n > j.max_rows) fail(j.c.status, DEV_INCONSISTENT, SITE_CHUNK);
    claimed += (unsigned)x.n;
    mine += (int64_t)x.tiles * j.c.H * x.stages;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if (__reduce_add_sync(0xffffffffu, claimed) > (unsigned)j.s.rows) {
    fail(j.c.status, DEV_INCONSISTENT, SITE_ROWS);
    return 0;
  }
  if (mine > 0x7fffffff) {   // 2^31 stages: more than 17 TB of keys and values
    fail(j.c.status, DEV_INCONSISTENT, SITE_LEN);
    return 0;
  }
  return (int)mine;
}

// Sequence that holds stage `at` of the range, and where its stages begin.  All lanes of a warp; the search goes on from
// the 32 sequences where the last one ended (stretches are walked upwards), this lane's of them in x.
struct Cursor {
  int b0, begin;
  Span x;
};
struct Place {
  int b, begin;
  Span x;
};
template <int KT>
__device__ __forceinline__ Place find(const Job& j, int at, Cursor& c) {
  const int lane = threadIdx.x & 31;
  for (;;) {
    const int mine = stages_of(j, c.x);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    const unsigned past = __ballot_sync(0xffffffffu, c.begin + incl > at);
    if (past || c.b0 + 32 >= j.s.n) {
      const int k = past ? __ffs(past) - 1 : 31;   // (there is one: `at` lies in the range)
      Place p;
      p.b = min(c.b0 + k, j.s.n - 1);
      p.begin = c.begin + __shfl_sync(0xffffffffu, incl - mine, k);
      int* to = reinterpret_cast<int*>(&p.x);
      const int* from = reinterpret_cast<const int*>(&c.x);
#pragma unroll
      for (int i = 0; i < (int)(sizeof(Span) / 4); ++i) to[i] = __shfl_sync(0xffffffffu, from[i], k);
      return p;
    }
    c.begin += __shfl_sync(0xffffffffu, incl, 31);
    c.b0 += 32;
    c.x = c.b0 + lane < j.s.n ? span_of<KT>(j, c.b0 + lane) : Span{};
  }
}

__device__ __forceinline__ void ldsm(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// An 8 x 8 matrix of 16-bit elements, a row's pairs with four lanes, to its transpose.
__device__ __forceinline__ uint32_t transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two fp16 from the two codes in the low or the high half of x.
__device__ __forceinline__ uint32_t widen_lo(uint32_t x) {
  uint32_t y;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t x) {
  uint32_t y;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// The two bf16 of x times f, as fp16.
__device__ __forceinline__ uint32_t to_f16(uint32_t x, float f) {
  const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x));
  return pack_f16(v.x * f, v.y * f);
}

// Four codes of the values, two positions of two neighbouring columns d, d + 1 (bytes: position 0: d, d + 1, position 1:
// d, d + 1), as bf16: a code's bits in bf16's fields (its sign spread over a byte above it, all but one of those bits cleared)
// are its value times 2^-120, subnormal codes included; f holds 2^120 times the positions' scales.
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

// Byte offset of 16-byte chunk c of row r in a tile.
template <int D, bool E4M3>
__device__ __forceinline__ int chunk_at(int r, int c) {
  if (!E4M3) return (c >> 3) * Lay<D, E4M3, 1>::PANEL + r * 128 + (((c & 7) ^ (r & 7)) << 4);
  return D == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}

__device__ __forceinline__ bool sees(int p, int end, int lo, int sk) { return p < end && (p >= lo || p < sk); }

// A unit's count of CTAs that are done with it: call << ROWS_COUNT_BITS | count once somebody has put it there, before that
// whatever the memory held.  begin_count, early: the CTA in which the unit begins does so; should another be done
// before that, it sees that the number is not the call's.
__device__ __forceinline__ void begin_count(unsigned long long* at, unsigned long long call) {
  const unsigned long long old = *reinterpret_cast<volatile unsigned long long*>(at);
  if ((old >> ROWS_COUNT_BITS) != call) atomicCAS(at, old, call << ROWS_COUNT_BITS);
}
// One more of n; true for the last one, which leaves nothing behind.  (One trip to L2 as a rule; taking turns with
// compare and swap instead cost 13 CTAs 6 us.)
__device__ __forceinline__ bool arrive(unsigned long long* at, unsigned long long call, int n) {
  for (;;) {
    unsigned long long old = atomicAdd(at, 1ull);
    if ((old >> ROWS_COUNT_BITS) == call) {
      if ((int)(old & ((1u << ROWS_COUNT_BITS) - 1u)) + 1 < n) return false;
      atomicExch(at, 0ull);
      return true;
    }
    // nobody's count yet: the number that was added to was not one; put the call's there, or see that it is
    old = *reinterpret_cast<volatile unsigned long long*>(at);
    while ((old >> ROWS_COUNT_BITS) != call) {
      const unsigned long long got = atomicCAS(at, old, call << ROWS_COUNT_BITS);
      if (got == old) break;
      old = got;
    }
  }
}

// One warp's sum of parts p = first, first + step, .. < n of a row (at(p): outputs [D], then the row's logarithm at
// `log`): m, l and o (columns c * 32 + lane) as a softmax over them, in their order.  Short loops: these
// instructions run once or twice, and fetching them is most of what they cost.
template <int D, typename At>
__device__ __forceinline__ void sum_parts(At at, int first, int n, int step, int log, float& m, float& l, float (&o)[D / 32]) {
  const int lane = threadIdx.x & 31;
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) o[c] = 0.f;
#pragma unroll 1
  for (int p0 = first; p0 < n; p0 += 32 * step) {
    const int mine = p0 + lane * step, count = min(32, (n - p0 + step - 1) / step);
    const float z = mine < n ? __ldcg(at(mine) + log) : -INFINITY;
    float top = fmaxf(m, z);
#pragma unroll
    for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    const float a = m == -INFINITY ? 0.f : exp2f(m - top);
    const float weight = z == -INFINITY ? 0.f : exp2f(z - top);   // (nothing seen: 0; a NaN stays one)
    m = top;
    l *= a;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[c] *= a;
#pragma unroll 4
    for (int k = 0; k < count; ++k) {
      const float w = __shfl_sync(0xffffffffu, weight, k);
      const float* x = at(p0 + k * step) + lane;
      l += w;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const float v = __ldcg(x + c * 32);
        if (w != 0.f) o[c] = fmaf(w, v, o[c]);
      }
    }
  }
}

template <int D>
__device__ __forceinline__ void store_row(const Job& j, int h, int tile, int r0, int r, float l, const float (&o)[D / 32]) {
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int lane = threadIdx.x & 31, i = tile * j.unit + r, tok = token_of(j, i), hq = i - tok * j.G;
  __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(j.o.p) + (int64_t)(h * j.G + hq) * j.o.head + (int64_t)(r0 + tok) * j.o.row;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) dst[c * 32 + lane] = __float2bfloat16_rn(o[c] * inv);
}

// Joins the n CTAs' parts of a unit, the first one's from CTA `first`, in the CTAs' order: a row a warp, or, where the
// parts are many for one warp, all warps at a row.  All threads of the CTA; room: shared memory.
template <int D, int WARPS>
__device__ __forceinline__ void join(const Job& j, int h, int tile, int rows, int r0, int first, int n, float* room) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool shared = n > 32;
  auto at = [&](int p) { return j.parts + (int64_t)(WORKERS + 2 * (first + p) + (p == 0 ? 1 : 0)) * j.part_rows * (D + 4); };
#pragma unroll 1
  for (int r = shared ? 0 : warp; r < rows; r += shared ? 1 : WARPS) {
    float m, l, o[D / 32];
    auto row_at = [&](int p) { return at(p) + r * D; };
    sum_parts<D>(row_at, shared ? warp : 0, n, shared ? WARPS : 1, j.part_rows * D + r - r * D, m, l, o);
    if (shared) {                          // the warps' sums, as parts again
      __syncthreads();
      const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) room[warp * (D + 1) + c * 32 + lane] = o[c] * inv;
      if (lane == 0) room[warp * (D + 1) + D] = l == 0.f ? -INFINITY : m + log2f(l);
      __syncthreads();
      if (warp != 0) continue;
      m = -INFINITY;
      const float z = lane < WARPS ? room[lane * (D + 1) + D] : -INFINITY;
      float top = z;
#pragma unroll
      for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
      const float weight = z == -INFINITY ? 0.f : exp2f(z - top);
      l = 0.f;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) o[c] = 0.f;
#pragma unroll 1
      for (int w = 0; w < WARPS; ++w) {
        const float a = __shfl_sync(0xffffffffu, weight, w);
        l += a;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
          if (a != 0.f) o[c] = fmaf(a, room[w * (D + 1) + c * 32 + lane], o[c]);
      }
    }
    store_row<D>(j, h, tile, r0, r, l, o);
  }
  __syncthreads();
}

template <int D, bool E4M3, int NR>
__global__ void __launch_bounds__((Lay<D, E4M3, NR>::WARPS * 32), 1)
    cache_attend_rows(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ Job j) {
  using L = Lay<D, E4M3, NR>;
  constexpr int WARPS = L::WARPS, KT = L::KT, KS = D / 16, NB = KT / 8, UNIT = 8 * NR;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
  if ((smem_u32(smem) & 1023u) != 0u) {
    if (threadIdx.x == 0) fail(j.c.status, DEV_INCONSISTENT, 9904);
    return;
  }
  uint8_t* ring = smem + warp * L::RING;
  uint8_t* scales = smem + L::SCALES + warp * (L::SLOTS * 2 * KT);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::BARS) + warp * L::SLOTS;
  Stretch* info = reinterpret_cast<Stretch*>(smem + L::INFO);
  if (lane == 0) {
    for (int i = 0; i < L::SLOTS; ++i) mbar_init(bars + i, 1);
    fence_barrier_init();
  }
  if (threadIdx.x == 0) begin_count(j.arrived + blockIdx.x, j.call);
  __syncwarp();

  // The CTAs' stretches follow one another, a CTA's warps' too, so that a unit's parts are joined in the CTA
  // first; where there are few stages, few warps of every CTA have one.
  Cursor cursor{};
  const int total = total_stages<KT>(j, cursor.x);
  const int per = min(WARPS, max(1, total / (MIN_STAGES * (int)gridDim.x)));   // warps at work
  const int workers = min(total, per * (int)gridDim.x);
  const int worker = (int)blockIdx.x * per + warp;
  // the first `more` stretches have one stage more than the others
  const int least = workers > 0 ? (int)((unsigned)total / (unsigned)workers) : 0, more = total - least * workers;
  int at = 0, stop = 0;
  if (warp < per && worker < workers) {
    at = worker * least + min(worker, more);
    stop = at + least + (worker < more ? 1 : 0);
  }
  if (lane == 0) info[warp].head = info[warp].tail = 0;
  uint32_t issued = 0, used = 0;          // stages, over all segments: slot and phase of the ring
  volatile int no_abort = 0;
  bool ok = true;

  while (ok && at < stop) {
    // ---- the segment: stages [k0, k1) of a unit's list
    const Place pl = find<KT>(j, at, cursor);
    const Span& x = pl.x;
    const int unit = (int)((unsigned)(at - pl.begin) / (unsigned)x.stages), k0 = at - pl.begin - unit * x.stages;
    const int h = (int)((unsigned)unit / (unsigned)x.tiles), tile = unit - h * x.tiles;
    const int k1 = min(x.stages, k0 + (stop - at));
    const int rows = min(UNIT, x.n * j.G - tile * UNIT);
    const int boxr = min(KT, j.c.page_len), box_log2 = min(KT == 16 ? 4 : 5, j.c.page_log2);
    const int nbox_log2 = (KT == 16 ? 4 : 5) - box_log2, nbox = 1 << nbox_log2;   // boxes of a stage: 1 or 2

    // first position of box i of the segment, and whether some token sees into it
    auto place_of = [&](int i) {
      const int k = k0 + (i >> nbox_log2);
      return (k < x.ns ? k : x.w0 + (k - x.ns)) * KT + ((i & (nbox - 1)) << box_log2);
    };
    auto wanted = [&](int p) { return p < x.end && (p + boxr > x.lo || p < x.sk); };
    // its page, 32 boxes at a time with the lanes (looked at when the box is issued)
    auto entry_of = [&](int i) -> int {
      const int p = place_of(i);
      return k0 + (i >> nbox_log2) < k1 && wanted(p) ? __ldg(j.s.table + (int64_t)pl.b * j.s.max_pages + (p >> j.c.page_log2)) : 0;
    };
    int pages = entry_of(lane), pages_next = entry_of(32 + lane), base = 0;

    // ---- the queries: operand columns gr + 8 u, in the order of d that the keys' registers have
    uint32_t qb[NR][KS][2];
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int r = gr + 8 * u, i = tile * UNIT + r, tok = token_of(j, i), hq = i - tok * j.G;
      const bool on = r < rows;
      const uint32_t* src = reinterpret_cast<const uint32_t*>(
          static_cast<const __nv_bfloat16*>(j.q.p) + (int64_t)(h * j.G + hq) * j.q.head + (int64_t)(x.r0 + tok) * j.q.row);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const int w0 = E4M3 ? t * (D / 8) + 2 * kk : kk * 8 + t, w1 = E4M3 ? w0 + 1 : w0 + 4;
        qb[u][kk][0] = on ? __ldg(src + w0) : 0u;
        qb[u][kk][1] = on ? __ldg(src + w1) : 0u;
      }
    }
    // the rows whose scores and outputs this thread holds: 2 t, 2 t + 1 (and 8 more), what they see
    int end[NR][2], lo[NR][2];
#pragma unroll
    for (int u = 0; u < NR; ++u)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * u + 2 * t + e, p = x.len - x.n + token_of(j, tile * UNIT + r);
        end[u][e] = r < rows && p >= 0 ? visible_end(j.m, p, x.len) : 0;
        lo[u][e] = window_first(j.m, end[u][e]);
      }
    // stage k0 + k into the ring, a lane a copy: of keys and values (lane bit 0), boxes and panels
    auto issue = [&](int k) {
      const int slot = issued % L::SLOTS;
      ++issued;
      if ((k << nbox_log2) - base >= 32) {   // (32 is a multiple of nbox)
        base += 32;
        pages = pages_next;
        pages_next = entry_of(base + 32 + lane);
      }
      const int c = lane >> 1, box = c & (nbox - 1), panel = c >> nbox_log2;
      const int p = place_of((k << nbox_log2) + box), sl = p & (j.c.page_len - 1);
      int page = __shfl_sync(0xffffffffu, pages, ((k << nbox_log2) - base + box) & 31);
      const bool mine = panel < (E4M3 ? 1 : D / 64);
      if (!wanted(p)) {
        page = j.c.n_pages;                  // nobody's: zeros
      } else if ((unsigned)page >= (unsigned)j.c.n_pages) {
        fail(j.c.status, DEV_INCONSISTENT, SITE_PAGE);
        page = j.c.n_pages;
      }
      uint32_t bytes = 2 * L::TILE;
      if (E4M3) bytes += __popc(__ballot_sync(0xffffffffu, mine && page < j.c.n_pages)) << box_log2;
      if (lane == 0) mbar_arrive_expect_tx(bars + slot, bytes);
      __syncwarp();
      if (!mine) return;
      const CUtensorMap* map = lane & 1 ? &tmV : &tmK;
      uint8_t* dst = ring + slot * L::SLOT + (lane & 1) * L::TILE;
      if (E4M3) {
        tma_load_4d(dst + (box << box_log2) * D, map, bars + slot, 0, sl, h, page);
        if (page < j.c.n_pages)
          bulk_load(scales + slot * 2 * KT + (lane & 1) * KT + (box << box_log2),
                    (lane & 1 ? j.c.vs : j.c.ks) + (((int64_t)page * j.c.H + h) << j.c.page_log2) + sl, boxr, bars + slot);
      } else {
        tma_load_4d(dst + panel * L::PANEL + (box << box_log2) * 128, map, bars + slot, panel * 64, sl, h, page);
      }
    };
    const int count = k1 - k0;
    for (int k = 0; k < min(count, L::SLOTS); ++k) issue(k);

    const int sk = j.m.window ? j.m.sinks : 0;
    // e4m3: the products are fp16, which holds every code exactly; a row of queries too, times the power of
    // two that puts its largest magnitude at 2^7 .. 2^8 (what lies 2^-24 below that is rounded, to within 2^-32 of it: fp16's
    // steps are 2^-24 there)
    float rs[NR][2];                        // of a row's products, in the exponent of 2
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      rs[u][0] = rs[u][1] = j.m.sl2;
      if constexpr (E4M3) {
        uint32_t big = 0;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) big = __vmaxu2(__vmaxu2(big, qb[u][kk][0] & 0x7fff7fffu), qb[u][kk][1] & 0x7fff7fffu);
        big = __vmaxu2(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = __vmaxu2(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const int e = max((int)(max(big & 0xffffu, big >> 16) >> 7), 16) - 134;   // (-118 .. 121)
        const float f = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          qb[u][kk][0] = to_f16(qb[u][kk][0], f);
          qb[u][kk][1] = to_f16(qb[u][kk][1], f);
        }
        const float back = __uint_as_float((uint32_t)(127 + e) << 23);   // row gr's; rows 2 t, 2 t + 1 lie with lanes 8 t, 8 t + 4
        rs[u][0] *= __shfl_sync(0xffffffffu, back, 8 * t);
        rs[u][1] *= __shfl_sync(0xffffffffu, back, 8 * t + 4);
      }
    }
    // o[c][u]: columns of the values 16 c + gr, + 8 (e4m3: 16 c + 2 gr, + 1) of rows 8 u + 2 t, + 1
    float o[D / 16][NR][4], mrun[NR][2], l[NR][2];
#pragma unroll
    for (int u = 0; u < NR; ++u) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mrun[u][e] = -INFINITY;
        l[u][e] = 0.f;
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c][u][e] = 0.f;
    }

    for (int k = 0; k < count; ++k) {
      const int slot = used % L::SLOTS;
      if (!(ok = mbar_wait_warp(bars + slot, (used / L::SLOTS) & 1, &no_abort))) break;
      ++used;
      const int kk0 = k0 + k, p0 = (kk0 < x.ns ? kk0 : x.w0 + (kk0 - x.ns)) * KT;
      const bool partial = !(p0 + KT <= x.all_end && (p0 >= x.all_lo || p0 + KT <= sk));
      uint8_t* kt = ring + slot * L::SLOT;
      uint8_t* vt = kt + L::TILE;
      const uint32_t ka = smem_u32(kt), va = smem_u32(vt);
      const uint8_t* sc = scales + slot * 2 * KT;

      // ---- scores: s[g][u][e]: position 16 g + gr (e < 2) or 8 more, row 8 u + 2 t + (e & 1)
      float s[KT / 16][NR][4];
#pragma unroll
      for (int g = 0; g < KT / 16; ++g)
#pragma unroll
        for (int u = 0; u < NR; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[g][u][e] = 0.f;
      if constexpr (E4M3) {
        uint32_t w[NB][D / 16];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < D / 64; ++i) {
            const uint4 y = *reinterpret_cast<const uint4*>(kt + chunk_at<D, E4M3>(n * 8 + gr, t * (D / 64) + i));
            w[n][4 * i] = y.x; w[n][4 * i + 1] = y.y; w[n][4 * i + 2] = y.z; w[n][4 * i + 3] = y.w;
          }
#pragma unroll
        for (int kk = 0; kk < KS; ++kk)
#pragma unroll
          for (int g = 0; g < KT / 16; ++g) {
            const uint32_t a[4] = {widen_lo(w[2 * g][kk]), widen_lo(w[2 * g + 1][kk]), widen_hi(w[2 * g][kk]), widen_hi(w[2 * g + 1][kk])};
#pragma unroll
            for (int u = 0; u < NR; ++u) mma_f16(s[g][u], a, qb[u][kk][0], qb[u][kk][1]);
          }
      } else {
        float s2[KT / 16][NR][4];            // (two sums of half the products each: shorter chains)
#pragma unroll
        for (int g = 0; g < KT / 16; ++g)
#pragma unroll
          for (int u = 0; u < NR; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s2[g][u][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk)
#pragma unroll
          for (int g = 0; g < KT / 16; ++g) {
            uint32_t a[4];
            const int m = lane >> 3, key = g * 16 + (m & 1) * 8 + (lane & 7);
            ldsm(ka + chunk_at<D, E4M3>(key, kk * 2 + (m >> 1)), a);
#pragma unroll
            for (int u = 0; u < NR; ++u) mma(kk & 1 ? s2[g][u] : s[g][u], a, qb[u][kk][0], qb[u][kk][1]);
          }
#pragma unroll
        for (int g = 0; g < KT / 16; ++g)
#pragma unroll
          for (int u = 0; u < NR; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[g][u][e] += s2[g][u][e];
      }
      // e4m3: 2^120 times the values' scales (positions 16 g + 8 v + 2 t and the next).  Where that is more than bf16 holds
      // (far: scales above 2^7), as much of it as bf16 does hold; the rest goes to the weights.  A row of byte 255 is NaN to
      // those that see it by its score; its codes are left finite for the others, whose weight is 0.
      uint32_t vf[KT / 16][2];
      bool far = false;
      if constexpr (E4M3) {
        uint32_t most = 0;
#pragma unroll
        for (int g = 0; g < KT / 16; ++g)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const uint32_t b = __byte_perm(*reinterpret_cast<const uint16_t*>(sc + KT + g * 16 + v * 8 + 2 * t), 0, 0x4140);
            most = __vmaxu2(most, b);
            vf[g][v] = (b + 0x00780078u) << 7;
          }
        far = __any_sync(0xffffffffu, max(most & 0xffffu, most >> 16) > 134u);
      }
      // into exponents of 2, with the keys' scales
#pragma unroll
      for (int g = 0; g < KT / 16; ++g)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const float ck = E4M3 ? scale_of(sc[g * 16 + v * 8 + gr]) : 1.0f;
#pragma unroll
          for (int u = 0; u < NR; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) s[g][u][2 * v + e] *= E4M3 ? ck * rs[u][e] : j.m.sl2;
        }
      if (E4M3 && far) {
#pragma unroll
        for (int g = 0; g < KT / 16; ++g)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            vf[g][v] = (__vminu2(vf[g][v] >> 7, 0x00fe00feu)) << 7;
            if (sc[KT + g * 16 + v * 8 + gr] != 255u) continue;
#pragma unroll
            for (int u = 0; u < NR; ++u) s[g][u][2 * v] = s[g][u][2 * v + 1] = __int_as_float(0x7fffffff);
          }
      }
      if (partial) {
#pragma unroll
        for (int g = 0; g < KT / 16; ++g)
#pragma unroll
          for (int u = 0; u < NR; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!sees(p0 + g * 16 + (e >> 1) * 8 + gr, end[u][e & 1], lo[u][e & 1], sk)) s[g][u][e] = -INFINITY;
      }
      // ---- running maximum of a row (the eight lanes of the same t)
      float nm[NR][2], alpha[NR][2];
      bool raised = false;
#pragma unroll
      for (int u = 0; u < NR; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = -INFINITY;
#pragma unroll
          for (int g = 0; g < KT / 16; ++g) mx = max3(mx, s[g][u][e], s[g][u][2 + e]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          const float before = mrun[u][e];
          const bool raise = mx > before + RESCALE_LOG2 || (before == -INFINITY && mx > -INFINITY);
          alpha[u][e] = raise ? (before == -INFINITY ? 0.f : ex2(before - mx)) : 1.f;
          if (raise) {
            raised |= before != -INFINITY;   // (nothing to scale before the first visible key)
            l[u][e] *= alpha[u][e];
            mrun[u][e] = mx;
          }
          nm[u][e] = mrun[u][e] == -INFINITY ? 0.f : -mrun[u][e];
        }
      if (__any_sync(0xffffffffu, raised)) {
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
          for (int u = 0; u < NR; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][u][e] *= alpha[u][e & 1];
      }
      // ---- weights, as an operand: pb[g][u]: positions 16 g + 2 t, + 1 (and 8 more) of row 8 u + gr
      uint32_t pb[KT / 16][NR][2];
#pragma unroll
      for (int g = 0; g < KT / 16; ++g)
#pragma unroll
        for (int u = 0; u < NR; ++u)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            float a = ex2(s[g][u][2 * v] + nm[u][0]), b = ex2(s[g][u][2 * v + 1] + nm[u][1]);
            l[u][0] += a;
            l[u][1] += b;
            if (E4M3 && far) {              // (a weight is 2^8 at most, the rest of a scale 2^113)
              const uint32_t y = sc[KT + g * 16 + v * 8 + gr];
              const float rest = y > 134u && y != 255u ? __uint_as_float((y - 7u) << 23) : 1.0f;
              a *= rest;
              b *= rest;
            }
            pb[g][u][v] = transpose(pack_bf16(a, b));
          }
      // ---- values that are not finite, in a stage that some row does not see whole: into the outputs of the rows
      // that see them, and out of the tile (their weight elsewhere is 0, and 0 times them NaN)
      if (!E4M3 && partial) {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < KT * D / 8 / 32; ++i) {
          const uint4 y = *reinterpret_cast<const uint4*>(vt + (i * 32 + lane) * 16);
          any |= ((y.x & 0x7f807f80u) + 0x00800080u) | ((y.y & 0x7f807f80u) + 0x00800080u) |
                 ((y.z & 0x7f807f80u) + 0x00800080u) | ((y.w & 0x7f807f80u) + 0x00800080u);
        }
        if (__any_sync(0xffffffffu, (any & 0x80008000u) != 0)) {
          for (int key = 0; key < KT; ++key)
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
#pragma unroll
              for (int v = 0; v < 2; ++v) {
                const float y = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(vt + chunk_at<D, E4M3>(key, 2 * c + v) + gr * 2));
                if (!isfinite(y)) {
#pragma unroll
                  for (int u = 0; u < NR; ++u)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                      if (sees(p0 + key, end[u][e], lo[u][e], sk)) o[c][u][2 * v + e] += y;
                }
              }
          __syncwarp();
          for (int i = 0; i < KT * D / 2 / 32; ++i) {
            uint32_t* w = reinterpret_cast<uint32_t*>(vt) + i * 32 + lane;
            const uint32_t bad = ((*w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
            *w &= ~(((bad >> 15) & 0x00010001u) * 0xffffu);
          }
          fence_async_smem();               // (the next copy into the slot follows)
          __syncwarp();
        }
      }
      // ---- outputs
#pragma unroll
      for (int g = 0; g < KT / 16; ++g) {
        const int m = lane >> 3;
        if constexpr (E4M3) {
#pragma unroll
          for (int c2 = 0; c2 < D / 32; ++c2) {
            uint32_t b[4];
            ldsm_t(va + chunk_at<D, E4M3>(g * 16 + (m & 1) * 8 + (lane & 7), c2 * 2 + (m >> 1)), b);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t a[4];
              widen_values(b[2 * i], *reinterpret_cast<const __nv_bfloat162*>(&vf[g][0]), a[0], a[1]);
              widen_values(b[2 * i + 1], *reinterpret_cast<const __nv_bfloat162*>(&vf[g][1]), a[2], a[3]);
#pragma unroll
              for (int u = 0; u < NR; ++u) mma(o[2 * c2 + i][u], a, pb[g][u][0], pb[g][u][1]);
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            uint32_t a[4];
            ldsm_t(va + chunk_at<D, E4M3>(g * 16 + (m >> 1) * 8 + (lane & 7), c * 2 + (m & 1)), a);
#pragma unroll
            for (int u = 0; u < NR; ++u) mma(o[c][u], a, pb[g][u][0], pb[g][u][1]);
          }
        }
      }
      __syncwarp();                       // all lanes have read the slot
      if (k + L::SLOTS < count) issue(k + L::SLOTS);
    }
    if (!ok) break;

    // ---- the segment's result
#pragma unroll
    for (int u = 0; u < NR; ++u)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int w = 4; w <= 16; w <<= 1) l[u][e] += __shfl_xor_sync(0xffffffffu, l[u][e], w);
    const bool whole = count == x.stages;
    if (!whole && lane == 0) {
      Stretch& y = info[warp];
      auto cta_of = [&](int stage) {        // who has it
        return (stage < more * (least + 1) ? stage / (least + 1) : more + (stage - more * (least + 1)) / least) / per;
      };
      const int begin = pl.begin + unit * x.stages, last = begin + x.stages - 1;
      if (k0 == 0) {                      // the unit's first part
        y.tail = 1;
        y.last = cta_of(last);
        y.h = h; y.tile = tile; y.rows = rows; y.r0 = x.r0;
      } else {
        y.head = 1;
        y.head_ends = k1 == x.stages;
        y.head_smem = at + count >= stop;
        y.first = cta_of(begin);
        y.hlast = cta_of(last);
        y.hh = h; y.htile = tile; y.hrows = rows; y.hr0 = x.r0;
      }
    }
    // a part goes where the stages were (the last one: the ring is the warp's own and empty), or into the scratch
    float* part = at + count >= stop ? reinterpret_cast<float*>(ring) : j.parts + (int64_t)worker * j.part_rows * (D + 4);
#pragma unroll
    for (int u = 0; u < NR; ++u)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * u + 2 * t + e;
        if (r >= rows || (!whole && r >= j.part_rows)) continue;
        const float inv = l[u][e] == 0.f ? 0.f : 1.0f / l[u][e];
        const int i = tile * UNIT + r, tok = token_of(j, i), hq = i - tok * j.G;
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(j.o.p) + (int64_t)(h * j.G + hq) * j.o.head + (int64_t)(x.r0 + tok) * j.o.row;
        float* pd = part + r * D;
        if (!whole && gr == 0) part[j.part_rows * D + r] = l[u][e] == 0.f ? -INFINITY : mrun[u][e] + log2f(l[u][e]);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          const float a = o[c][u][e] * inv, b = o[c][u][2 + e] * inv;
          if (E4M3 && whole) {
            *reinterpret_cast<uint32_t*>(dst + 16 * c + 2 * gr) = pack_bf16(a, b);
          } else if (E4M3) {
            *reinterpret_cast<float2*>(pd + 16 * c + 2 * gr) = make_float2(a, b);
          } else if (whole) {
            dst[16 * c + gr] = __float2bfloat16_rn(a);
            dst[16 * c + 8 + gr] = __float2bfloat16_rn(b);
          } else {
            pd[16 * c + gr] = a;
            pd[16 * c + 8 + gr] = b;
          }
        }
      }
    at += count;
  }
  if (!ok) {
    if (lane == 0) fail(j.c.status, DEV_TIMEOUT, SITE_WAIT + 4);
    const uint64_t t0 = globaltimer_ns();   // copies may be in flight: far longer than one takes
    while (globaltimer_ns() - t0 < 50000ull) {
    }
    if (lane == 0) info[warp].tail = info[warp].head = 0;
  }

  // ---- the CTA's parts joined: one chain for each tail, and one for a unit from before the CTA.  A chain's
  // parts are a tail (or the first warp's head) and the heads of the warps behind it up to the unit's end.
  __syncthreads();
  auto worker_part = [&](int w, bool tail) -> const float* {
    return tail || info[w].head_smem ? reinterpret_cast<const float*>(smem + w * L::RING)
                                     : j.parts + (int64_t)((int)blockIdx.x * per + w) * j.part_rows * (D + 4);
  };
  // (a bit a warp: has a head, its head ends in it, has a tail)
  const unsigned heads = __ballot_sync(0xffffffffu, lane < per && info[lane < per ? lane : 0].head);
  const unsigned ending = __ballot_sync(0xffffffffu, lane < per && info[lane < per ? lane : 0].head_ends) & heads;
  const unsigned tails = __ballot_sync(0xffffffffu, lane < per && info[lane < per ? lane : 0].tail);
  int open = -1;                          // the chain of a unit that goes on behind the CTA
  int todo = 0;                           // (chain, row) pairs so far: warps take them in turn
#pragma unroll 1
  for (unsigned left = (tails << 1) | (heads & 1u); left; left &= left - 1) {
    const int c = __ffs(left) - 2, c0 = max(c, 0);   // -1: the first warp's head
    const Stretch& y = info[c0];
    const int h = c < 0 ? y.hh : y.h, tile = c < 0 ? y.htile : y.tile;
    const int rows = min(c < 0 ? y.hrows : y.rows, j.part_rows), r0 = c < 0 ? y.hr0 : y.r0;
    // parts: up to the first warp behind whose head ends there, or before the first without a head
    const int after = c < 0 ? 0 : c + 1, stop = __ffs((~heads | ending) >> after) - 1 + after;
    const bool ends = stop < per && ((ending >> stop) & 1u);
    const int n = min(stop, per) - c0 + (ends ? 1 : 0);
    if (c >= 0 && !ends) open = c;        // (one at most: the last chain)
    // rows in turn with the other chains' (a warp's first: warp - todo, modulo their number)
#pragma unroll 1
    for (int r = (warp + 16 * WARPS - todo % WARPS) % WARPS; r < rows; r += WARPS) {
      float m, l, o[D / 32];
      // (every part's address by itself: some are in shared memory)
      const int log = j.part_rows * D + r;
      const float z = lane < n ? worker_part(max(c, 0) + lane, lane == 0 && c >= 0)[log] : -INFINITY;
      m = z;
#pragma unroll
      for (int w = 16; w; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
      const float weight = z == -INFINITY ? 0.f : exp2f(z - m);   // (nothing seen: 0; a NaN stays one)
      l = 0.f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
#pragma unroll 1
      for (int p = 0; p < n; ++p) {
        const float w = __shfl_sync(0xffffffffu, weight, p);
        const float* x = worker_part(max(c, 0) + p, p == 0 && c >= 0) + r * D + lane;
        l += w;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
          if (w != 0.f) o[i] = fmaf(w, x[i * 32], o[i]);
      }
      if (c >= 0 && ends) {
        store_row<D>(j, h, tile, r0, r, l, o);
      } else {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        float* part = j.parts + (int64_t)(WORKERS + 2 * (int)blockIdx.x + (c < 0 ? 0 : 1)) * j.part_rows * (D + 4);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) part[r * D + i * 32 + lane] = o[i] * inv;
        if (lane == 0) part[log] = l == 0.f ? -INFINITY : m + log2f(l);
      }
    }
    todo += rows;
  }

  // ---- units that other CTAs hold parts of: the last of them to come joins the parts
  const bool from_before = info[0].head != 0;
  if (!from_before && open < 0) return;   // uniform
  __syncthreads();
  int* last = reinterpret_cast<int*>(info + WARPS);   // [2]
  if (lane == 0 && warp < 2) {            // (both trips at once)
    __threadfence();
    const Stretch& y = info[max(open, 0)];
    last[warp] = (warp == 0 ? from_before : open >= 0) &&
                 arrive(j.arrived + (warp == 0 ? info[0].first : (int)blockIdx.x), j.call,
                        warp == 0 ? info[0].hlast - info[0].first + 1 : y.last - (int)blockIdx.x + 1);
    __threadfence();
  }
  __syncthreads();
  float* room = reinterpret_cast<float*>(smem);
  if (last[0])
    join<D, WARPS>(j, info[0].hh, info[0].htile, min(info[0].hrows, j.part_rows), info[0].hr0, info[0].first,
            info[0].hlast - info[0].first + 1, room);
  if (last[1]) {
    const Stretch& y = info[max(open, 0)];
    join<D, WARPS>(j, y.h, y.tile, min(y.rows, j.part_rows), y.r0, blockIdx.x, y.last - (int)blockIdx.x + 1, room);
  }
}

template <int D, bool E4M3, int NR>
cudaError_t launch_n(const Maps& maps, const Job& job, int ctas, cudaStream_t st) {
  using L = Lay<D, E4M3, NR>;
  return launch_kernel(cache_attend_rows<D, E4M3, NR>, dim3(ctas), L::WARPS * 32, L::BYTES, 1, false, st, maps.rk, maps.rv, job);
}
template <int D, bool E4M3>
cudaError_t launch_d(const Maps& maps, const Job& job, int ctas, cudaStream_t st) {
  return job.unit == 8 ? launch_n<D, E4M3, 1>(maps, job, ctas, st) : launch_n<D, E4M3, 2>(maps, job, ctas, st);
}

template <int D, bool E4M3, int NR>
cudaError_t set_limit_n() {
  return taken(cudaFuncSetAttribute(cache_attend_rows<D, E4M3, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    Lay<D, E4M3, NR>::BYTES));
}
template <int D, bool E4M3>
cudaError_t set_limit() {
  const cudaError_t e = set_limit_n<D, E4M3, 1>();
  return e != cudaSuccess ? e : set_limit_n<D, E4M3, 2>();
}

template <int D, bool E4M3>
bool make_d(const Pool& c, Maps* m) {
  using L = Lay<D, E4M3, 1>;
  const int64_t dim[4] = {D, c.page_len, c.H, c.n_pages};
  const int64_t stride[3] = {(int64_t)D * L::ES, (int64_t)c.page_len * D * L::ES, (int64_t)c.H * c.page_len * D * L::ES};
  const int box[4] = {E4M3 ? D : 64, std::min(c.page_len, L::KT), 1, 1};
  const int swizzle = E4M3 ? D : 128;
  return make_map_4d(&m->rk, c.k, L::ES, dim, stride, box, swizzle) && make_map_4d(&m->rv, c.v, L::ES, dim, stride, box, swizzle);
}

// Query rows of a unit, and of a partial result.
int unit_rows(int G, int max_rows) { return (int64_t)max_rows * G <= 8 ? 8 : 16; }
int part_rows(int G, int max_rows) { return (int)std::min<int64_t>(unit_rows(G, max_rows), (int64_t)max_rows * G); }

}  // namespace

cudaError_t attend_rows_set_smem_limits() {
  cudaError_t e = set_limit<128, false>();
  if (e == cudaSuccess) e = set_limit<128, true>();
  if (e == cudaSuccess) e = set_limit<64, false>();
  if (e == cudaSuccess) e = set_limit<64, true>();
  return e;
}

bool make_rows_maps(const Pool& c, Maps* m) {
  if (c.d == 128) return c.e4m3 ? make_d<128, true>(c, m) : make_d<128, false>(c, m);
  return c.e4m3 ? make_d<64, true>(c, m) : make_d<64, false>(c, m);
}

size_t attend_rows_scratch(const Pool& c, int G, int max_rows) {
  return sizeof(unsigned long long) * MAX_CTAS + sizeof(float) * (size_t)(WORKERS + 2 * MAX_CTAS) * part_rows(G, max_rows) * (c.d + 4);
}

cudaError_t launch_attend_rows(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                               int max_rows, const Mask& m, void* scratch, cudaStream_t st) {
  const int n_sm = std::min(sm_count(), MAX_CTAS), G = Hq / c.H;
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  // numbers the calls, so that a count that another call left in the same memory is not taken for this one's (a captured
  // call keeps its number: its replays, one after the other, each find the count cleared by the one before)
  static std::atomic<uint64_t> calls{0};
  unsigned long long* const arrived = static_cast<unsigned long long*>(scratch);
  const Job job{c, s, m, q, o, G, max_rows, (uint32_t)((0xffffffffull + G) / G), unit_rows(G, max_rows), part_rows(G, max_rows), reinterpret_cast<float*>(arrived + MAX_CTAS), arrived,
                rows_number(calls.fetch_add(1))};
  if (c.d == 128)
    return c.e4m3 ? launch_d<128, true>(maps, job, n_sm, st) : launch_d<128, false>(maps, job, n_sm, st);
  return c.e4m3 ? launch_d<64, true>(maps, job, n_sm, st) : launch_d<64, false>(maps, job, n_sm, st);
}

}  // namespace cache
}  // namespace dkv
