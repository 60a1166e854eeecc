// Attention of few query rows over the paged cache (include/dkv.h: dkv_cache_attend): single tokens
// and a handful of drafted ones.  Every key and value is read once and used by at most 16 rows, so
// HBM bounds it (4 d bytes a position and key head in bf16, 2 d + 2 in e4m3); the arithmetic only
// has to keep out of the way.
//
// A unit is 16 query rows of one sequence and one key head, row = token * G + head.  The visible
// positions of all units, in stages of KT, form one range, and each of the GPU's 8 x 152 warps
// takes an equal stretch of it, whatever units it belongs to: no warp waits for another, and the
// split over a long cache, over many sequences and over ragged lengths is the same one.  A unit inside one
// stretch is finished there; one that a boundary cuts leaves a partial result for each warp that
// holds some of it, joined by rows_merge.
//
// A warp streams its stages through a ring of its own (TMA boxes of one page, 128-byte swizzled;
// one lane issues, a barrier a slot), scores them with mma.sync m16n8k16 (16 rows fill one such
// product; the tensor cores' tile of 128 rows would be an eighth full at best and add its latencies), and
// keeps the running maximum, sum and 16 x d outputs in registers.  Scores' accumulators are the
// weights' operand layout, so weights never leave the registers.
//
// e4m3: the codes become bf16 in the registers.  A key row's 128 codes lie with four lanes, 32
// neighbouring ones each, and the queries' registers are loaded in that order of d instead of the product's own; of the
// values, a transposed load gives pairs of d of one position, which widen into the even and the odd
// columns of 16.
#include "attn_math.cuh"
#include "cache_internal.h"
#include "tc_ptx.cuh"

#include <algorithm>

namespace dkv {

bool make_map_4d(CUtensorMap* m, const void* base, int elem_bytes, const int64_t (&dim)[4], const int64_t (&stride)[3],
                 const int (&box)[4], int swizzle);

namespace cache {

namespace {

using namespace tc;

constexpr int WARPS = 8;
constexpr int MAX_CTAS = 152;
constexpr int WORKERS = WARPS * MAX_CTAS;
constexpr int ROWS = 16;
constexpr float RESCALE_LOG2 = 8.0f;
constexpr int MIN_STAGES = 4;    // stages of a stretch, at least: below that the joining costs more

template <int D, bool E4M3>
struct Lay {
  static constexpr int ES = E4M3 ? 1 : 2;
  static constexpr int KT = !E4M3 && D == 128 ? 16 : 32;   // positions of a stage
  static constexpr int PANEL = KT * (E4M3 ? D : 128);      // bytes of a panel (64 columns; codes: all)
  static constexpr int TILE = KT * D * ES;                 // bytes of a stage's keys
  static constexpr int SLOTS = 3;
  static constexpr int SLOT = 2 * TILE;                    // keys, values
  static constexpr int RING = SLOTS * SLOT;                // a warp's
  static constexpr int SCALES = WARPS * RING;              // [warps][slots][2][KT] scale bytes
  static constexpr int BARS = SCALES + (E4M3 ? WARPS * SLOTS * 2 * KT : 0);
  static constexpr int BYTES = BARS + WARPS * SLOTS * 8;
  static_assert(BYTES <= 227 * 1024, "shared memory per CTA");
};

struct Job {
  Pool c;
  Seqs s;
  Mask m;
  Packed q, o;
  int G, max_rows;
  int part_rows;     // rows of a partial result
  int4* meta;        // [WORKERS][2] the unit that is cut first in the worker's stretch: {sequence, key head, row tile,
                     //   its last worker}, {rows, -, -, -}; .w < 0: none
  float* parts;      // [2 WORKERS][part_rows][D + 4] (outputs, then a sum's logarithm a row): a stretch's first unit,
                     //   its last one
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
  x.tiles = (q.n * j.G + ROWS - 1) / ROWS;
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

__device__ __forceinline__ int64_t stages_of(const Job& j, const Span& x) { return (int64_t)x.tiles * j.c.H * x.stages; }

// All lanes of a warp.
template <int KT>
__device__ int64_t total_stages(const Job& j) {
  int64_t mine = 0;
  for (int b = threadIdx.x & 31; b < j.s.n; b += 32) {
    const Span x = span_of<KT>(j, b);
    if (x.n > j.max_rows) fail(j.c.status, DEV_INCONSISTENT, SITE_CHUNK);
    mine += stages_of(j, x);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  return mine;
}

// Sequence that holds stage `at` of the range, and where its stages begin.  All lanes of a warp.
struct Place {
  int b;
  int64_t begin;
  Span x;
};
template <int KT>
__device__ Place find(const Job& j, int64_t at) {
  const int lane = threadIdx.x & 31;
  int64_t begin = 0;
  for (int b0 = 0;; b0 += 32) {
    const int b = b0 + lane;
    Span x{};
    if (b < j.s.n) x = span_of<KT>(j, b);
    const int64_t mine = stages_of(j, x);
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    const unsigned past = __ballot_sync(0xffffffffu, b < j.s.n && begin + incl > at);
    if (past || b0 + 32 >= j.s.n) {
      const int k = past ? __ffs(past) - 1 : 31;   // (there is one: `at` lies in the range)
      Place p;
      p.b = min(b0 + k, j.s.n - 1);
      p.begin = begin + __shfl_sync(0xffffffffu, incl - mine, k);
      int* to = reinterpret_cast<int*>(&p.x);
      const int* from = reinterpret_cast<const int*>(&x);
#pragma unroll
      for (int i = 0; i < (int)(sizeof(Span) / 4); ++i) to[i] = __shfl_sync(0xffffffffu, from[i], k);
      return p;
    }
    begin += __shfl_sync(0xffffffffu, incl, 31);
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

__device__ __forceinline__ __nv_bfloat162 bf2(uint32_t bits) { return *reinterpret_cast<const __nv_bfloat162*>(&bits); }
__device__ __forceinline__ uint32_t times(uint32_t x, __nv_bfloat162 f) {
  const __nv_bfloat162 y = __hmul2(bf2(x), f);
  return *reinterpret_cast<const uint32_t*>(&y);
}
// Four codes as bf16 fields (their values times 2^-120) in two pairs, taken by the byte selectors.
template <uint32_t S0, uint32_t S1>
__device__ __forceinline__ void widen(uint32_t w, __nv_bfloat162 f, uint32_t& a, uint32_t& b) {
  const uint32_t hi = (w & 0x80808080u) | ((w >> 4) & 0x07070707u), lo = (w << 4) & 0xf0f0f0f0u;
  a = times(__byte_perm(lo, hi, S0), f);
  b = times(__byte_perm(lo, hi, S1), f);
}

// Byte offset of 16-byte chunk c of row r in a tile.
template <int D, bool E4M3>
__device__ __forceinline__ int chunk_at(int r, int c) {
  if (!E4M3) return (c >> 3) * Lay<D, E4M3>::PANEL + r * 128 + (((c & 7) ^ (r & 7)) << 4);
  return D == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}

__device__ __forceinline__ bool sees(int p, int end, int lo, int sk) { return p < end && (p >= lo || p < sk); }

template <int D, bool E4M3>
__global__ void __launch_bounds__(WARPS * 32, 1)
    cache_attend_rows(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ Job j) {
  using L = Lay<D, E4M3>;
  constexpr int KT = L::KT, KS = D / 16, NB = KT / 8;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
  if ((smem_u32(smem) & 1023u) != 0u) {
    if (threadIdx.x == 0) fail(j.c.status, DEV_INCONSISTENT, 9904);
    return;
  }
  uint8_t* ring = smem + warp * L::RING;
  uint8_t* scales = smem + L::SCALES + warp * (L::SLOTS * 2 * KT);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::BARS) + warp * L::SLOTS;
  if (lane == 0) {
    for (int i = 0; i < L::SLOTS; ++i) mbar_init(bars + i, 1);
    fence_barrier_init();
  }
  __syncwarp();
  pdl_trigger();

  // neighbouring stretches on different SMs: where there are few, each has an SM to itself
  const int worker = warp * gridDim.x + blockIdx.x;
  const int64_t total = total_stages<KT>(j);
  const int64_t most = (total + MIN_STAGES - 1) / MIN_STAGES;
  const int workers = (int)min(most, (int64_t)(WARPS * gridDim.x));
  int64_t at = 0, stop = 0;
  if (worker < workers) {
    at = total * worker / workers;
    stop = total * (worker + 1) / workers;
  }
  int4 cut0 = make_int4(0, 0, 0, -1), cut1 = make_int4(0, 0, 0, 0);
  uint32_t issued = 0, used = 0;          // stages, over all segments: slot and phase of the ring
  volatile int no_abort = 0;
  bool ok = true;

  while (ok && at < stop) {
    // ---- the segment: stages [k0, k1) of a unit's list
    const Place pl = find<KT>(j, at);
    const Span& x = pl.x;
    const int64_t rel = at - pl.begin;
    const int unit = (int)(rel / x.stages), k0 = (int)(rel % x.stages);
    const int h = unit / x.tiles, tile = unit % x.tiles;
    const int k1 = (int)min((int64_t)x.stages, k0 + (stop - at));
    const int rows = min(ROWS, x.n * j.G - tile * ROWS);
    const int boxr = min(KT, j.c.page_len), nbox = KT / boxr;

    // page of box i of the segment, 32 at a time with the lanes; nobody's where no token sees into it
    auto page_of = [&](int i) -> int {
      const int k = k0 + i / nbox;
      const int p = (k < x.ns ? k : x.w0 + (k - x.ns)) * KT + (i % nbox) * boxr;
      if (k >= k1 || p >= x.end || !(p + boxr > x.lo || p < x.sk)) return j.c.n_pages;
      const int page = __ldg(j.s.table + (int64_t)pl.b * j.s.max_pages + (p >> j.c.page_log2));
      if ((unsigned)page >= (unsigned)j.c.n_pages) {
        fail(j.c.status, DEV_INCONSISTENT, SITE_PAGE);
        return j.c.n_pages;
      }
      return page;
    };
    int pages = page_of(lane), pages_next = page_of(32 + lane), base = 0;
    auto issue = [&](int k) {             // stage k0 + k into the ring
      const int slot = issued % L::SLOTS;
      ++issued;
      const int first = k * nbox;
      if (first - base >= 32) {           // (32 is a multiple of nbox)
        base += 32;
        pages = pages_next;
        pages_next = page_of(base + 32 + lane);
      }
      int pg[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) pg[i] = i < nbox ? __shfl_sync(0xffffffffu, pages, first - base + i) : j.c.n_pages;
      if (lane != 0) return;
      const int kk = k0 + k, p = (kk < x.ns ? kk : x.w0 + (kk - x.ns)) * KT;
      uint32_t bytes = 2 * L::TILE;
      if (E4M3)
        for (int i = 0; i < nbox; ++i) bytes += pg[i] < j.c.n_pages ? 2 * boxr : 0;
      mbar_arrive_expect_tx(bars + slot, bytes);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i >= nbox) break;
        const int sl = (p + i * boxr) & (j.c.page_len - 1);
        uint8_t* dst = ring + slot * L::SLOT;
        if (E4M3) {
          tma_load_4d(dst + i * boxr * D, &tmK, bars + slot, 0, sl, h, pg[i]);
          tma_load_4d(dst + L::TILE + i * boxr * D, &tmV, bars + slot, 0, sl, h, pg[i]);
          if (pg[i] < j.c.n_pages) {
            const int64_t row = (((int64_t)pg[i] * j.c.H + h) << j.c.page_log2) + sl;
            bulk_load(scales + slot * 2 * KT + i * boxr, j.c.ks + row, boxr, bars + slot);
            bulk_load(scales + slot * 2 * KT + KT + i * boxr, j.c.vs + row, boxr, bars + slot);
          }
        } else {
#pragma unroll
          for (int n = 0; n < D / 64; ++n) {
            tma_load_4d(dst + n * L::PANEL + i * boxr * 128, &tmK, bars + slot, n * 64, sl, h, pg[i]);
            tma_load_4d(dst + L::TILE + n * L::PANEL + i * boxr * 128, &tmV, bars + slot, n * 64, sl, h, pg[i]);
          }
        }
      }
    };
    const int count = k1 - k0;
    for (int k = 0; k < min(count, L::SLOTS); ++k) issue(k);

    // ---- the queries, in the order of d that the keys' registers have
    uint32_t qa[KS][4];
    int end[2], lo[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = gr + 8 * u, i = tile * ROWS + r, tok = i / j.G, hq = i - tok * j.G;
      const bool on = r < rows;
      const int p = x.len - x.n + tok;
      end[u] = on && p >= 0 ? visible_end(j.m, p, x.len) : 0;
      lo[u] = window_first(j.m, end[u]);
      const uint32_t* src = reinterpret_cast<const uint32_t*>(
          static_cast<const __nv_bfloat16*>(j.q.p) + (int64_t)(h * j.G + hq) * j.q.head + (int64_t)(x.r0 + tok) * j.q.row);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const int w0 = E4M3 ? t * (D / 8) + 2 * kk : kk * 8 + t, w1 = E4M3 ? w0 + 1 : w0 + 4;
        qa[kk][u] = on ? __ldg(src + w0) : 0u;
        qa[kk][2 + u] = on ? __ldg(src + w1) : 0u;
      }
    }
    const int sk = j.m.window ? j.m.sinks : 0;
    float o[D / 8][4], mrun[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][e] = 0.f;

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

      // ---- scores
      float s[NB][4];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
      if (E4M3) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const int key = n * 8 + gr;
          const uint32_t b = sc[key];
          uint32_t w[D / 16];
#pragma unroll
          for (int i = 0; i < D / 64; ++i) {
            const uint4 y = *reinterpret_cast<const uint4*>(kt + chunk_at<D, E4M3>(key, t * (D / 64) + i));
            w[4 * i] = y.x; w[4 * i + 1] = y.y; w[4 * i + 2] = y.z; w[4 * i + 3] = y.w;
          }
          // 2^120 times the scale in one factor where it is a bf16 number, else by itself on the sums' side
          const bool two = b > 134u;
          const __nv_bfloat162 f = bf2((two ? 247u : b + 120u) * 0x00800080u);
#pragma unroll
          for (int kk = 0; kk < KS; ++kk) {
            uint32_t b0, b1;
            widen<0x5140, 0x7362>(w[kk], f, b0, b1);
            mma(s[n], qa[kk], b0, b1);
          }
          if (__any_sync(0xffffffffu, two)) {   // columns 2t, 2t + 1 of this block
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t c = sc[n * 8 + 2 * t + e];
              const float g = c > 134u ? scale_of(c) : 1.0f;
              s[n][e] *= g;
              s[n][2 + e] *= g;
            }
          }
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < KS; ++kk)
#pragma unroll
          for (int n2 = 0; n2 < NB / 2; ++n2) {
            uint32_t b[4];
            const int m = lane >> 3, key = n2 * 16 + (m >> 1) * 8 + (lane & 7);
            ldsm(ka + chunk_at<D, E4M3>(key, kk * 2 + (m & 1)), b);
            mma(s[2 * n2], qa[kk], b[0], b[1]);
            mma(s[2 * n2 + 1], qa[kk], b[2], b[3]);
          }
      }
      if (partial) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!sees(p0 + n * 8 + 2 * t + (e & 1), end[e >> 1], lo[e >> 1], sk)) s[n][e] = -INFINITY;
      }
      // ---- running maximum of rows gr and gr + 8 (four lanes each)
      float nm[2];
      bool raised = false;
      float alpha[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < NB; ++n) mx = fmaxf(mx, fmaxf(s[n][2 * u], s[n][2 * u + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        mx *= j.m.sl2;
        const bool raise = mx > mrun[u] + RESCALE_LOG2 || (mrun[u] == -INFINITY && mx > -INFINITY);
        alpha[u] = raise ? (mrun[u] == -INFINITY ? 0.f : ex2(mrun[u] - mx)) : 1.f;
        if (raise) {
          raised |= mrun[u] != -INFINITY;   // (nothing to scale before the first visible key)
          l[u] *= alpha[u];
          mrun[u] = mx;
        }
        nm[u] = mrun[u] == -INFINITY ? 0.f : -mrun[u];
      }
      if (__any_sync(0xffffffffu, raised)) {
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[n][0] *= alpha[0]; o[n][1] *= alpha[0];
          o[n][2] *= alpha[1]; o[n][3] *= alpha[1];
        }
      }
      // ---- weights
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][e] = ex2(fmaf(s[n][e], j.m.sl2, nm[e >> 1]));
          l[e >> 1] += s[n][e];
        }
      if (E4M3) {   // the values' scales (a hidden row's may be NaN)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float g = scale_of(sc[KT + n * 8 + 2 * t + e]);
            s[n][e] = s[n][e] == 0.f ? 0.f : s[n][e] * g;
            s[n][2 + e] = s[n][2 + e] == 0.f ? 0.f : s[n][2 + e] * g;
          }
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
            for (int n = 0; n < D / 8; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float v = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(vt + chunk_at<D, E4M3>(key, n) + (2 * t + e) * 2));
                if (!isfinite(v)) {
                  if (sees(p0 + key, end[0], lo[0], sk)) o[n][e] += v;
                  if (sees(p0 + key, end[1], lo[1], sk)) o[n][2 + e] += v;
                }
              }
          __syncwarp();
          for (int i = 0; i < KT * D / 2 / 32; ++i) {
            uint32_t* w = reinterpret_cast<uint32_t*>(vt) + i * 32 + lane;
            const uint32_t bad = ((*w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
            *w &= ~(((bad >> 15) & 0x00010001u) * 0xffffu);
          }
          fence_async_smem();             // (the next copy into the slot follows)
          __syncwarp();
        }
      }
      // ---- outputs
#pragma unroll
      for (int g2 = 0; g2 < KT / 16; ++g2) {
        const uint32_t pa[4] = {pack_bf16(s[2 * g2][0], s[2 * g2][1]), pack_bf16(s[2 * g2][2], s[2 * g2][3]),
                                pack_bf16(s[2 * g2 + 1][0], s[2 * g2 + 1][1]), pack_bf16(s[2 * g2 + 1][2], s[2 * g2 + 1][3])};
        if (E4M3) {
          const __nv_bfloat162 f = bf2(247u * 0x00800080u);
#pragma unroll
          for (int c2 = 0; c2 < D / 32; ++c2) {
            uint32_t b[4];
            const int m = lane >> 3, key = g2 * 16 + (m & 1) * 8 + (lane & 7);
            ldsm_t(va + chunk_at<D, E4M3>(key, c2 * 2 + (m >> 1)), b);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t e0, o0, e1, o1;
              widen<0x6240, 0x7351>(b[2 * i], f, e0, o0);
              widen<0x6240, 0x7351>(b[2 * i + 1], f, e1, o1);
              mma(o[4 * c2 + 2 * i], pa, e0, e1);
              mma(o[4 * c2 + 2 * i + 1], pa, o0, o1);
            }
          }
        } else {
#pragma unroll
          for (int c2 = 0; c2 < D / 16; ++c2) {
            uint32_t b[4];
            const int m = lane >> 3, key = g2 * 16 + (m & 1) * 8 + (lane & 7);
            ldsm_t(va + chunk_at<D, E4M3>(key, c2 * 2 + (m >> 1)), b);
            mma(o[2 * c2], pa, b[0], b[1]);
            mma(o[2 * c2 + 1], pa, b[2], b[3]);
          }
        }
      }
      __syncwarp();                       // all lanes have read the slot
      if (k + L::SLOTS < count) issue(k + L::SLOTS);
    }
    if (!ok) break;

    // ---- the segment's result
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 1);
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 2);
    }
    const bool whole = count == x.stages;
    if (!whole && k0 == 0) {              // the unit's first part
      const int64_t last = pl.begin + (int64_t)(unit + 1) * x.stages;
      cut0 = make_int4(pl.b, h, tile, (int)((last * workers + total - 1) / total) - 1);
      cut1 = make_int4(rows, x.r0, 0, 0);
    }
    float* part = j.parts + (int64_t)(2 * worker + (k0 == 0 ? 1 : 0)) * j.part_rows * (D + 4);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = gr + 8 * u;
      if (r >= rows || (!whole && r >= j.part_rows)) continue;
      const float inv = l[u] == 0.f ? 0.f : 1.0f / l[u];
      const int i = tile * ROWS + r, tok = i / j.G, hq = i - tok * j.G;
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(j.o.p) + (int64_t)(h * j.G + hq) * j.o.head + (int64_t)(x.r0 + tok) * j.o.row;
      float* pd = part + r * D;
      if (!whole && t == 0) part[j.part_rows * D + r] = l[u] == 0.f ? -INFINITY : mrun[u] + log2f(l[u]);
      if (E4M3) {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {   // columns 16 c + 4 t ..
          const float4 y = make_float4(o[2 * c][2 * u] * inv, o[2 * c + 1][2 * u] * inv, o[2 * c][2 * u + 1] * inv,
                                       o[2 * c + 1][2 * u + 1] * inv);
          if (whole)
            *reinterpret_cast<uint2*>(dst + 16 * c + 4 * t) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
          else
            *reinterpret_cast<float4*>(pd + 16 * c + 4 * t) = y;
        }
      } else {
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          const float a = o[n][2 * u] * inv, b = o[n][2 * u + 1] * inv;
          if (whole)
            *reinterpret_cast<uint32_t*>(dst + 8 * n + 2 * t) = pack_bf16(a, b);
          else
            *reinterpret_cast<float2*>(pd + 8 * n + 2 * t) = make_float2(a, b);
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
    cut0.w = -1;
  }
  if (lane == 0) {
    j.meta[2 * worker] = cut0;
    j.meta[2 * worker + 1] = cut1;
  }
}

// Joins the parts of cut units: O = sum 2^(lse - max) O_part / sum 2^(lse - max).  Block (x, y) looks at
// the eight workers x, x + gridDim.x, .. and takes the rows y, y + gridDim.y, .. of the units whose first part
// they hold; its warps share a row's parts.
constexpr int MERGE_Y = 4;

template <int D>
__global__ void __launch_bounds__(256) rows_merge(const __grid_constant__ Job j) {
  pdl_wait();
  constexpr int N = D / 32;
  __shared__ float so[8][D], sm[8], sl[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int k = 0; k < WARPS; ++k) {
    const int first = k * gridDim.x + blockIdx.x;
    const int4 u = j.meta[2 * first];
    if (u.w < first || u.w >= WARPS * (int)gridDim.x) continue;
    const int4 v = j.meta[2 * first + 1];
    const int rows = min(v.x, j.part_rows), n = u.w - first + 1;
    for (int r = blockIdx.y; r < rows; r += MERGE_Y) {
      float m = -INFINITY, l = 0.f, o[N];
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = 0.f;
      constexpr int UN = 4;
      for (int p0 = warp; p0 < n; p0 += 8 * UN) {
        float x[UN][N], z[UN];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
          const int p = p0 + 8 * i;
          z[i] = -INFINITY;
          if (p < n) {
            const float* part = j.parts + (int64_t)(p == 0 ? 2 * first + 1 : 2 * (first + p)) * j.part_rows * (D + 4);
            z[i] = part[j.part_rows * D + r];
#pragma unroll
            for (int c = 0; c < N; ++c) x[i][c] = part[r * D + c * 32 + lane];
          }
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) {
          if (z[i] == -INFINITY) continue;   // nothing seen
          if (z[i] > m) {
            const float a = exp2f(m - z[i]);
            m = z[i];
            l *= a;
#pragma unroll
            for (int c = 0; c < N; ++c) o[c] *= a;
          }
          const float w = exp2f(z[i] - m);   // (a NaN stays one)
          l += w;
#pragma unroll
          for (int c = 0; c < N; ++c) o[c] = fmaf(w, x[i][c], o[c]);
        }
      }
#pragma unroll
      for (int c = 0; c < N; ++c) so[warp][c * 32 + lane] = o[c];
      if (lane == 0) {
        sm[warp] = m;
        sl[warp] = l;
      }
      __syncthreads();
      if (threadIdx.x < D) {
        float mx = -INFINITY, den = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) mx = fmaxf(mx, sm[w]);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          if (sl[w] == 0.f) continue;
          const float a = exp2f(sm[w] - mx);
          den = fmaf(a, sl[w], den);
          y = fmaf(a, so[w][threadIdx.x], y);
        }
        const int i = u.z * ROWS + r, tok = i / j.G, hq = i - tok * j.G;
        static_cast<__nv_bfloat16*>(j.o.p)[(int64_t)(u.y * j.G + hq) * j.o.head + (int64_t)(v.y + tok) * j.o.row + threadIdx.x] =
            __float2bfloat16_rn(den == 0.f ? 0.f : y / den);
      }
      __syncthreads();
    }
  }
}

template <int D, bool E4M3>
cudaError_t launch_d(const Maps& maps, const Job& job, int ctas, cudaStream_t st) {
  cudaError_t e = launch_kernel(cache_attend_rows<D, E4M3>, dim3(ctas), WARPS * 32, Lay<D, E4M3>::BYTES, 1, false, st,
                                maps.rk, maps.rv, job);
  if (e == cudaSuccess)
    e = launch_kernel(rows_merge<D>, dim3(ctas, std::min(MERGE_Y, job.part_rows)), 256, 0, 1, true, st, job);
  return e;
}

template <int D, bool E4M3>
cudaError_t set_limit() {
  return taken(cudaFuncSetAttribute(cache_attend_rows<D, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    Lay<D, E4M3>::BYTES));
}

template <int D, bool E4M3>
bool make_d(const Pool& c, Maps* m) {
  using L = Lay<D, E4M3>;
  const int64_t dim[4] = {D, c.page_len, c.H, c.n_pages};
  const int64_t stride[3] = {(int64_t)D * L::ES, (int64_t)c.page_len * D * L::ES, (int64_t)c.H * c.page_len * D * L::ES};
  const int box[4] = {E4M3 ? D : 64, std::min(c.page_len, L::KT), 1, 1};
  const int swizzle = E4M3 ? D : 128;
  return make_map_4d(&m->rk, c.k, L::ES, dim, stride, box, swizzle) && make_map_4d(&m->rv, c.v, L::ES, dim, stride, box, swizzle);
}

int part_rows(int G, int max_rows) { return std::min(ROWS, std::min(max_rows, ROWS) * G); }

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
  return sizeof(int4) * 2 * WORKERS + sizeof(float) * 2 * (size_t)WORKERS * part_rows(G, max_rows) * (c.d + 4);
}

cudaError_t launch_attend_rows(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                               int max_rows, const Mask& m, void* scratch, cudaStream_t st) {
  const int n_sm = std::min(sm_count(), MAX_CTAS), G = Hq / c.H;
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const Job job{c, s, m, q, o, G, max_rows, part_rows(G, max_rows), static_cast<int4*>(scratch),
                reinterpret_cast<float*>(static_cast<int4*>(scratch) + 2 * WORKERS)};
  if (c.d == 128)
    return c.e4m3 ? launch_d<128, true>(maps, job, n_sm, st) : launch_d<128, false>(maps, job, n_sm, st);
  return c.e4m3 ? launch_d<64, true>(maps, job, n_sm, st) : launch_d<64, false>(maps, job, n_sm, st);
}

}  // namespace cache
}  // namespace dkv
