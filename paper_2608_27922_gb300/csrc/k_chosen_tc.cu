// Attention over chosen pages on the tensor cores (include/dkv.h: dkv_cache_attend_chosen), many query rows a tile.
//
// A unit is 128 query rows of one tile of tokens and one key head, row = token * G + head, TQ = 128 / G tokens.  The pages that
// the tile's list names, one behind the other, form the unit's keys; in tiles of 128 they stream past the query rows:
//   S = Q K^T             tcgen05.mma into TMEM; thread = query row
//   P = exp2(S scale log2(e) - m)   packed bf16 over S in TMEM; what a row does not see is 0
//   O += P V              tcgen05.mma with A = P from TMEM
// with the running maximum raised only when a tile's exceeds it by more than 2^8 (O is then rescaled in TMEM).  The product of a
// tile's first 64 keys with V runs while the last 64's weights are worked out.
//
// One CTA a unit (or a cluster, whose CTAs share its key tiles and join their parts on chip) and two CTAs an SM: while one's
// softmax runs, the other's products do, and one's first loads hide behind the other's work, without a schedule of
// items.  Each has half of the SM's memory (a tile of Q, one of K and one of V at d = 128) and of its TMEM.
//
// bf16 pages come in by TMA, one box a page and 64-column panel.  (Asking the tile after next into L2 ahead of it: 278 us for
// 276.)  Codes come by plain loads, one tile ahead in the registers of warps of their own, which write them as bf16 with their
// scales in them: code bits in bf16's fields are the value times 2^-120, one product with 2^120 times the scale makes it
// exact.
//
// Weights are rounded to bf16 for the second product, whose values are bf16 and whose rate fp32 weights would cut to a part; their sum takes
// them unrounded.  A weight is off by 2^-8 of it at most: over a case outputs are 0.0023 from float64, where 32 bits throughout and
// the outputs' own rounding make 0.0017.
//
// Values in places that a row does not see meet its weight 0, and 0 times a NaN or an infinity is NaN: in the tiles that some
// row does not see whole, the softmax threads clear what is not finite in V's tile, and rows that do see such a value get
// it back at the end (wild_in).
//
// Measured: 4,680 tokens of 40 heads in tiles of 128, 28 pages of 128 each, in bf16 276 us, 1.24 PFLOP/s of 1.89.  Every tile of
// tokens reads its own keys, so a key tile serves 128 rows instead of 256 or more: 2.7 GB come through L2 (at 9.7 TB/s; 1.0 GB of
// it from HBM), and shared memory moves 1,280 cycles' worth of operands and copies a tile and CTA, 2,560 of the 3,200 that two CTAs' tiles
// take.  A CTA's start and end are 8 of its 50 us.  In e4m3 436 us: the conversion (5,200 of 8,000 instructions a tile).  d = 64: 224 and
// 300.  Chunks of 333 to 700 tokens of a small model in tiles of 16 (48 of 128 rows used) 47 us, in e4m3 57.5: three rounds of CTAs of 11 us.
// (Tiles of 64 keys, two of them in TMEM, so that a tile's softmax overlaps the next one's scores: 290 at d = 128, 212 at 64.)
#include "attn_math.cuh"
#include "cache_internal.h"
#include "tc_ptx.cuh"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace dkv {

bool make_map_4d(CUtensorMap* m, const void* base, int elem_bytes, const int64_t (&dim)[4], const int64_t (&stride)[3],
                 const int (&box)[4], int swizzle);

namespace cache {

namespace {

using namespace tc;

constexpr int BQ = 128, BK = 128;
constexpr int PANEL = 128 * 128;         // bytes of a 64-column panel of 128 rows
constexpr uint32_t TMEM_COLS = 256;      // S [0, 128), O [128, 128 + d)
constexpr float RESCALE_LOG2 = 8.0f;
constexpr int MAX_WIDTH = 1024;
constexpr int SITE = 10;                 // of waits, beside the other kernels'

template <int D, bool E4M3>
struct Lay {
  static constexpr int NP = D / 64;
  static constexpr int TB = NP * PANEL;                // bytes of a 128-row tile
  static constexpr int N = D == 128 ? 1 : 2;           // tiles of K, and of V
  static constexpr int Q = 0;
  static constexpr int K = TB;
  static constexpr int V = K + N * TB;
  static constexpr int LIST = V + N * TB;              // [MAX_WIDTH] entries, [MAX_WIDTH] pages
  static constexpr int CTRL = LIST + 2 * MAX_WIDTH * 4;
  static constexpr int STATS = CTRL + 256;             // [128] maximum, sum (a cluster's join)
  static constexpr size_t BYTES = STATS + 128 * 8;
  static constexpr int JOIN = K;                       // a part's outputs, [D / 4][128 rows] of 16 bytes
  // converting warps (a block of 40 heads: 8 warps 526 us, 4 569; at d = 64 358 and 321)
  static constexpr int CONV = !E4M3 ? 0 : D == 128 ? 8 : 4;
  static constexpr int THREADS = (8 + CONV) * 32;
  // registers a thread: the first four warps, the softmax, the conversion; the launch gives each
  // thread REGS.  (The softmax does with
  // 128 or 96; the first warps, with 56 or 40, kept their descriptors in local memory: a block of 40 heads 303 us for 280.)
  static constexpr int REGS = CONV == 8 ? 64 : CONV == 4 ? 80 : 128;
  static constexpr int REGS_IO = CONV == 8 ? 64 : CONV == 4 ? 72 : 88, REGS_SOFT = E4M3 ? 96 : 168, REGS_CONV = CONV == 8 ? 48 : 72;
  static_assert(REGS_IO + REGS_SOFT + CONV / 4 * REGS_CONV <= (2 + CONV / 4) * REGS, "register split");
  static_assert(REGS_IO <= REGS && (CONV == 0 || REGS_CONV <= REGS) && REGS_SOFT >= REGS, "lowered ones are, raised ones are");
  static_assert(2 * N * TB >= D * BQ * 4, "a part in the tiles' place");
  static_assert(2 * (BYTES + 1024) <= 228 * 1024, "two CTAs an SM");
};

struct Job {
  Pool c;
  Seqs s;
  Mask m;
  Packed o;
  Chosen how;
  int G, TQ, tiles;   // query tiles of a slot
  int wide;           // rows of the outputs 32-byte aligned
};

// The unit's keys: the first `count` entries of its list, page by page.
struct Keys {
  const int* entry;   // shared memory
  const int* page;    // -1: not to be read
  int count;
  int log2, len;      // of a page
  // position of place u of the keys; -1: none
  __device__ __forceinline__ int pos(int u) const {
    const int k = u >> log2;
    return k < count && page[k] >= 0 ? (entry[k] << log2) + (u & (len - 1)) : -1;
  }
};

__device__ __forceinline__ uint32_t below(int x) { return x <= 0 ? 0u : x >= 32 ? 0xffffffffu : (1u << x) - 1u; }

// Which of the places u .. u + 31 a row that sees up to `end` sees.
__device__ __forceinline__ uint32_t seen32(const Keys& k, int u, int end) {
  const int a = k.pos(u);
  if (k.len >= 32) return a < 0 ? 0u : below(end - a);
  const int z = k.pos(u + 16);
  return (a < 0 ? 0u : below(end - a) & 0xffffu) | (z < 0 ? 0u : (below(end - z) & 0xffffu) << 16);
}

// P = 2^(s sl2 + nm) over 32 scores as 16 packed bf16 pairs; lab accumulates the even and the odd columns.
__device__ __forceinline__ void weights(const float (&a)[32], float sl2, float nm, float2& lab, uint32_t (&pk)[16]) {
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const float2 x = __ffma2_rn(make_float2(a[2 * k], a[2 * k + 1]), make_float2(sl2, sl2), make_float2(nm, nm));
    const float2 p = make_float2(ex2(x.x), ex2(x.y));
    lab = __fadd2_rn(lab, p);
    pk[k] = pack_bf16(p.x, p.y);
  }
}
// 16 consecutive 32-bit columns of this warp's 32 TMEM lanes.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
               "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}

__device__ __forceinline__ void mask_row(float (&v)[32], uint32_t see) {
#pragma unroll
  for (int k = 0; k < 32; ++k)
    if (!((see >> k) & 1u)) v[k] = -INFINITY;
}

// Clears what is not finite in one bf16 row (128-byte swizzled panels), and says so in *met.
template <int D>
__device__ __forceinline__ void clear_row(uint8_t* tile, int row, volatile int* met) {
  uint32_t any = 0;
#pragma unroll
  for (int c = 0; c < D / 8; ++c) {
    const uint4 x = *reinterpret_cast<uint4*>(tile + (c >> 3) * PANEL + row * 128 + (((c & 7) ^ (row & 7)) << 4));
    any |= ((x.x & 0x7f807f80u) + 0x00800080u) | ((x.y & 0x7f807f80u) + 0x00800080u) |
           ((x.z & 0x7f807f80u) + 0x00800080u) | ((x.w & 0x7f807f80u) + 0x00800080u);
  }
  if ((any & 0x80008000u) == 0) return;
  *met = 1;
#pragma unroll 1
  for (int c = 0; c < D / 2; ++c) {
    uint32_t* p = reinterpret_cast<uint32_t*>(tile + (c >> 5) * PANEL + row * 128 + ((((c >> 2) & 7) ^ (row & 7)) << 4)) + (c & 3);
    const uint32_t x = *p, bad = ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    if (bad) *p = x & ~(((bad >> 15) & 0x00010001u) * 0xffffu);
  }
}

// The columns [c0, c0 + 32) in which a row that sees up to `end` meets a NaN, +inf, -inf in the places [u0, u1).
struct Wild {
  uint32_t nan, pos, neg;
};
template <int D, bool E4M3>
__device__ __noinline__ Wild wild_in(const Pool& c, const Keys& keys, int h, int u0, int u1, int end, int c0) {
  Wild w{0, 0, 0};
#pragma unroll 1
  for (int u = u0; u < u1; ++u) {
    const int p = keys.pos(u);
    if (p < 0 || p >= end) continue;
    const int64_t page = keys.page[u >> keys.log2], at = ((E4M3 ? page : page * c.H + h) << c.page_log2) + (p & (c.page_len - 1));
    if (E4M3) {
      if (c.vs[at] == 255) w.nan = 0xffffffffu;
      continue;
    }
    const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(c.v) + at * D + c0;
#pragma unroll 1
    for (int k = 0; k < 32; ++k) {
      const float x = __bfloat162float(v[k]);
      if (isnan(x)) w.nan |= 1u << k;
      if (x == INFINITY) w.pos |= 1u << k;
      if (x == -INFINITY) w.neg |= 1u << k;
    }
  }
  return w;
}

__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// Four bf16 from four codes (the sign spread over a byte above each, all but one of those bits cleared); f holds 2^120 times
// the scale.
__device__ __forceinline__ uint2 widen(uint32_t w, __nv_bfloat162 f) {
  uint32_t a, b;
  asm("prmt.b32 %0, %1, 0, 0x9180;" : "=r"(a) : "r"(w));   // (a selector's upper bit: that byte's sign, eight times)
  asm("prmt.b32 %0, %1, 0, 0xb3a2;" : "=r"(b) : "r"(w));
  a = (a << 4) & 0x87f087f0u;
  b = (b << 4) & 0x87f087f0u;
  const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), f);
  const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&b), f);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
}
__device__ __forceinline__ __nv_bfloat162 bf2(uint32_t bits) { return *reinterpret_cast<const __nv_bfloat162*>(&bits); }
__device__ __forceinline__ uint32_t times(uint32_t x, __nv_bfloat162 f) {
  const __nv_bfloat162 y = __hmul2(bf2(x), f);
  return *reinterpret_cast<const uint32_t*>(&y);
}

// Codes into bf16, CONV warps: eight neighbouring threads take four 16-byte parts (64 columns) of two neighbouring rows, so that
// their stores, swizzled by the row, touch every bank once.  A thread has N such parts, rows STEP apart; each is asked for
// again, for the tile after, as soon as it has been used.  (Two sets of registers did not fit: a block of 40 heads took 2,005 us.)
template <int D, int CONV>
struct Codes {
  static constexpr int NP = D / 64, STEP = CONV * 8 / NP, N = 128 / STEP;
  static_assert(STEP % 8 == 0, "a thread's rows share their swizzle");
  uint4 x[N];
  uint32_t s[N];
};

template <int D, bool E4M3>
__global__ void __launch_bounds__(Lay<D, E4M3>::THREADS, 2)
    chosen_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
              const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Job j) {
  using L = Lay<D, E4M3>;
  extern __shared__ __align__(1024) uint8_t smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int C = cluster.num_blocks(), rank = cluster.block_rank();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // ---- the unit (its list's first entries are asked for before the sequence is known)
  const int unit = blockIdx.x / C, slot = unit / j.tiles, qt = unit - slot * j.tiles, h = blockIdx.y;
  if (blockIdx.x == 0 && h == 0)
    for (int b = tid; b < j.s.n; b += L::THREADS) seq_at(j.c, j.s, b);
  const int32_t* const line = j.how.lists + ((int64_t)h * j.how.slots + slot) * j.how.width;
  const int early = tid < j.how.width ? __ldg(line + tid) : -1, early_before = tid && tid < j.how.width ? __ldg(line + tid - 1) : -1;
  Seq q;
  const int b = seq_of_slot_warp(j.c, j.s, j.how.tile, slot, q);
  const int i0 = (slot - q.r0 / j.how.tile - b) * j.how.tile;
  const int first = i0 + qt * j.TQ;                                        // its first token
  const int tokens = i0 < 0 ? 0 : min(min(j.how.tile - qt * j.TQ, j.TQ), q.n - first);
  if (tokens <= 0) return;                                                 // (the whole cluster)
  if ((smem_u32(smem) & 1023u) != 0u) {   // 128-byte-swizzled tiles need 1024-byte alignment
    if (tid == 0) fail(j.c.status, DEV_INCONSISTENT, 9904);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::CTRL);
  uint64_t* q_full = bars + 0;
  uint64_t* k_full = bars + 1;      // [N]
  uint64_t* k_empty = bars + 3;     // [N]
  uint64_t* v_full = bars + 5;      // [N]
  uint64_t* v_empty = bars + 7;     // [N]
  uint64_t* s_full = bars + 9;
  uint64_t* p_full = bars + 10;     // [2] weights of a tile's first and last 64 keys
  uint64_t* o_full = bars + 12;
  uint64_t* over = bars + 13;       // every role but the producer has ended
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 14);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 15);
  volatile int* wild = abort_flag + 1;
  // entries to be read, leading ones that all rows see whole, the list's end, its least faulty entry (twice its place, odd: its page)
  int* bounds = reinterpret_cast<int*>(bars + 16);
  int* entry = reinterpret_cast<int*>(smem + L::LIST);
  int* page = entry + MAX_WIDTH;
  if (tid == 64) {
    mbar_init(q_full, 1);
    for (int i = 0; i < L::N; ++i) {
      mbar_init(k_full + i, E4M3 ? L::CONV : 1);
      mbar_init(k_empty + i, 1);
      mbar_init(v_full + i, E4M3 ? L::CONV : 1);
      mbar_init(v_empty + i, 1);
    }
    mbar_init(s_full, 1);
    mbar_init(p_full + 0, 4);
    mbar_init(p_full + 1, 4);
    mbar_init(o_full, 1);
    mbar_init(over, 1 + 4 + L::CONV);
    *abort_flag = 0;
    *wild = 0;
    bounds[0] = bounds[1] = bounds[2] = j.how.width;
    bounds[3] = 0x7fffffff;
    fence_barrier_init();
    // Q is on its way while the list is looked through
    mbar_arrive_expect_tx(q_full, L::NP * j.TQ * j.G * 128);
    for (int p = 0; p < L::NP; ++p) tma_load_4d(smem + L::Q + p * PANEL, &tmQ, q_full, p * 64, 0, q.r0 + first, h);
  }
  if (warp == 1) tmem_alloc(tmem_holder, TMEM_COLS);
  auto end_of = [&](int token) {
    const int p = q.len - q.n + first + token;
    return p < 0 ? 0 : visible_end(j.m, p, q.len);
  };
  const int all_end = end_of(0), any_end = end_of(tokens - 1);
  __syncthreads();
  {
    for (int k = tid; k < j.how.width; k += L::THREADS) {
      const int e = k == tid ? early : __ldg(line + k), before = k == tid ? early_before : __ldg(line + k - 1);
      int at = -1;
      if (e < 0) {
        atomicMin(bounds, k);
        atomicMin(bounds + 2, k);
      } else if ((k && before >= 0 && e <= before) || e >= (q.len + j.c.page_len - 1) >> j.c.page_log2) {
        atomicMin(bounds + 3, 2 * k);
      } else if (((int64_t)e << j.c.page_log2) >= any_end) {
        atomicMin(bounds, k);   // (the rest of an ascending list lies behind it)
      } else {
        at = j.s.table[(int64_t)b * j.s.max_pages + e];
        if ((unsigned)at >= (unsigned)j.c.n_pages) {
          atomicMin(bounds + 3, 2 * k + 1);
          at = -1;
        }
      }
      if (at < 0 || ((int64_t)e + 1) << j.c.page_log2 > all_end) atomicMin(bounds + 1, k);
      entry[k] = e;
      page[k] = E4M3 && at >= 0 ? at * j.c.H + h : at;   // (codes: place of the head's rows; memory holds fewer than 2^31)
    }
  }
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *tmem_holder;
  if (tid == 64 && bounds[3] >> 1 < bounds[2])   // (what is behind the end is nothing)
    fail(j.c.status, DEV_INCONSISTENT, bounds[3] & 1 ? SITE_PAGE : SITE_LIST);
  const Keys keys{entry, page, bounds[0], j.c.page_log2, j.c.page_len};
  const int whole_to = min(bounds[1], bounds[0]) << j.c.page_log2;   // places that every row sees
  const int NT = ((keys.count << j.c.page_log2) + BK - 1) / BK;
  const int t0 = (int)((int64_t)NT * rank / C), t1 = (int)((int64_t)NT * (rank + 1) / C), n = t1 - t0;

  auto give_up = [&](int site) {
    *abort_flag = 1;
    fail(j.c.status, DEV_TIMEOUT, SITE_WAIT + SITE + site);
  };
  // of the softmax threads, kept for the join
  float mrun = -INFINITY, l = 0.f;
  bool ok = true;
  const int r = tid & 127, tok = r / j.G, hq = r - tok * j.G;   // row of a softmax thread
  const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t sc = tmem + lane_off, oc = sc + 128;
  const bool mine = tok < j.TQ && tok < tokens;
  const int end = mine ? end_of(tok) : 0;

  if (warp < 4) {
    regs_lower<L::REGS_IO>();
    if (warp == 0) {
      // ---------------- producer: K(0), V(0), K(1), ..  It also watches the time for all roles' waits.
      const int rows = min(j.c.page_len, BK), np = BK / rows;   // rows and boxes of a tile
      if constexpr (!E4M3) {
        const int box = lane / L::NP, panel = lane % L::NP;
        auto place = [&](int i, int& at, int& slot_in) {   // the lane's box of tile t0 + i
          const int u = (t0 + i) * BK + box * rows, k = u >> j.c.page_log2;
          at = box < np && i < n && k < keys.count ? page[k] : -1;
          slot_in = u & (j.c.page_len - 1);
        };
        auto load = [&](bool is_k, int i) -> bool {
          const int sl = i % L::N;
          uint64_t* bar = (is_k ? k_full : v_full) + sl;
          if (i >= L::N && !mbar_wait_warp((is_k ? k_empty : v_empty) + sl, (i / L::N - 1) & 1, abort_flag)) return false;
          if (lane == 0) mbar_arrive_expect_tx(bar, L::TB);
          __syncwarp();
          int at, in;
          place(i, at, in);
          if (box < np)   // (nobody's page: zeros)
            tma_load_4d(smem + (is_k ? L::K : L::V) + sl * L::TB + panel * PANEL + box * rows * 128, is_k ? &tmK : &tmV, bar,
                        panel * 64, in, h, at < 0 ? j.c.n_pages : at);
          __syncwarp();
          return true;
        };
        if (n > 0) ok = load(true, 0);
        for (int i = 0; ok && i < n; ++i) {
          ok = load(false, i);
          if (ok && i + 1 < n) ok = load(true, i + 1);
        }
      }
      if (ok) ok = mbar_wait_warp(over, 0, abort_flag);
      if (!ok) {
        if (lane == 0) give_up(0);
        // copies may be in flight that nobody waits for any more: far longer than one takes
        const uint64_t since = globaltimer_ns();
        while (globaltimer_ns() - since < 50000ull) {
        }
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer (the whole warp, one elected lane issues)
      constexpr uint32_t id_s = idesc_bf16(BQ, BK), id_o = idesc_bf16(BQ, D, /*b_mn_major=*/true);
      const uint64_t qd = desc_sw128(smem_u32(smem + L::Q)), kd0 = desc_sw128(smem_u32(smem + L::K));
      const uint64_t vd0 = desc_sw128_mn(smem_u32(smem + L::V), PANEL, 1024);
      ok = mbar_wait_warp_short(q_full, 0, abort_flag);   // (also where there are no keys: the copy ends before the CTA)
      for (int i = 0; ok && i < n; ++i) {
        const int sl = i % L::N;
        if (!(ok = mbar_wait_warp_short(k_full + sl, (i / L::N) & 1, abort_flag))) break;
        fence_after_sync();
        // (S's place holds the last tile's P: its product was issued before)
        const uint64_t kd = desc_add(kd0, sl * L::TB);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = (kk >> 2) * PANEL + (kk & 3) * 32;
            mma_bf16(tmem, desc_add(qd, off), desc_add(kd, off), id_s, kk > 0);
          }
          mma_commit(s_full);
          mma_commit(k_empty + sl);
        }
        __syncwarp();
        if (!(ok = mbar_wait_warp_short(v_full + sl, (i / L::N) & 1, abort_flag))) break;
        const uint64_t vd = desc_add(vd0, sl * L::TB);
        // (the first half's product runs while the last half's weights are worked out)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(ok = mbar_wait_warp_short(p_full + half, i & 1, abort_flag))) break;
          fence_after_sync();
          if (elect_one()) {
#pragma unroll
            for (int kk = half * 4; kk < half * 4 + 4; ++kk)
              mma_bf16_ts(tmem + 128, tmem + kk * 8, desc_add(vd, kk * 2048), id_o, i > 0 || kk > 0 ? 1u : 0u);
            if (half) {
              mma_commit(v_empty + sl);
              if (i + 1 == n) mma_commit(o_full);
            }
          }
          __syncwarp();
        }
      }
      if (!ok && lane == 0) give_up(1);
      if (!ok) {   // every product complete before TMEM is freed
        if (elect_one()) mma_commit(o_full);
        __syncwarp();
        volatile int no_abort = 0;
        mbar_wait(o_full, 0, &no_abort);
      }
      if (lane == 0) mbar_arrive(over);
    }
  } else if (warp < 8) {
    regs_raise<L::REGS_SOFT>();
    // ---------------- softmax, thread = query row = TMEM lane
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int sl = i % L::N, u0 = (t0 + i) * BK;
      const bool partial = u0 + BK > whole_to;
      if (!(ok = mbar_wait_warp_short(s_full, i & 1, abort_flag))) break;
      if (partial) {   // (after the scores: before them the values' barrier may still be a phase behind)
        if (!(ok = mbar_wait_warp_short(v_full + sl, (i / L::N) & 1, abort_flag))) break;
        clear_row<D>(smem + L::V + sl * L::TB, r, wild);
        fence_async_smem();
      }
      fence_after_sync();
      float tmax;
      {
        float t[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = -INFINITY;
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          float a[32], z[32];
          tmem_ld32(sc + half * 64, a);
          tmem_ld32(sc + half * 64 + 32, z);
          tmem_wait_ld();
          if (partial) {
            mask_row(a, seen32(keys, u0 + half * 64, end));
            mask_row(z, seen32(keys, u0 + half * 64 + 32, end));
            tmem_st32(sc + half * 64, reinterpret_cast<uint32_t(&)[32]>(a));
            tmem_st32(sc + half * 64 + 32, reinterpret_cast<uint32_t(&)[32]>(z));
          }
          max_acc(t, a);
          max_acc(t, z);
        }
        if (partial) tmem_wait_st();
        tmax = fmaxf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])), fmaxf(fmaxf(t[4], t[5]), fmaxf(t[6], t[7])));
      }
      tmax *= j.m.sl2;
      // S of this tile complete implies O of the one before complete (issued earlier by one thread)
      const bool raise = tmax > mrun + RESCALE_LOG2 || (mrun == -INFINITY && tmax > -INFINITY);
      const float mprev = mrun;
      if (raise) {
        l *= i > 0 ? ex2(mrun - tmax) : 0.f;
        mrun = tmax;
      }
      if (i > 0 && __any_sync(0xffffffffu, raise)) {
        const float alpha = raise ? ex2(mprev - mrun) : 1.0f;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          float v[32];
          tmem_ld32(oc + c * 32, v);
          tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] *= alpha;
          tmem_st32(oc + c * 32, reinterpret_cast<uint32_t(&)[32]>(v));
        }
      }
      const float nm = mrun == -INFINITY ? 0.f : -mrun;   // (a row that has seen nothing yet: all weights 0)
      // large scores are rounded before the maximum goes off them: in one step the maximum's own rounding, 2^-24 of it, stays
      // in the exponent
      const bool large = __any_sync(0xffffffffu, fabsf(nm) > 0x1p24f);
      const float sl2 = large ? 1.f : j.m.sl2;
      if (large) {
#pragma unroll 1
        for (int k0 = 0; k0 < BK; k0 += 32) {
          float a[32];
          tmem_ld32(sc + k0, a);
          tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 32; ++k) a[k] *= j.m.sl2;
          tmem_st32(sc + k0, reinterpret_cast<uint32_t(&)[32]>(a));
        }
        tmem_wait_st();
      }
      float2 lab = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        float a[32], z[32];
        uint32_t pk[16];
        tmem_ld32(sc + half * 64, a);
        tmem_ld32(sc + half * 64 + 32, z);
        tmem_wait_ld();
        weights(a, sl2, nm, lab, pk);
        tmem_st16(sc + half * 32, pk);
        weights(z, sl2, nm, lab, pk);
        tmem_st16(sc + half * 32 + 16, pk);
        tmem_wait_st();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + half);
      }
      l += lab.x + lab.y;
    }
    if (ok && n > 0) ok = mbar_wait_warp_short(o_full, 0, abort_flag);
    fence_after_sync();
    if (!ok && lane == 0) give_up(2);
    // ---- outputs, or a part of them into the tiles' place
    if (ok) {
      const bool fix = *wild != 0;
      const float f = C > 1 ? 1.f : l == 0.f ? 0.f : 1.0f / l;         // (a NaN stays one; what is not finite shows where all weights are 0 too)
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float v[32];
        if (n > 0) {
          tmem_ld32(oc + c * 32, v);
          tmem_wait_ld();
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = n > 0 ? fmaf(v[k], f, 0.f) : 0.f;
        if (fix) {
          const Wild w = wild_in<D, E4M3>(j.c, keys, h, max(t0 * BK, whole_to / BK * BK), t1 * BK, end, c * 32);
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            if ((w.pos >> k) & 1u) v[k] += INFINITY;
            if ((w.neg >> k) & 1u) v[k] -= INFINITY;
            if ((w.nan >> k) & 1u) v[k] = __int_as_float(0x7fffffff);
          }
        }
        if (C > 1) {
          float4* dst = reinterpret_cast<float4*>(smem + L::JOIN) + (c * 8) * BQ + r;
#pragma unroll
          for (int k = 0; k < 8; ++k) dst[k * BQ] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        } else if (mine) {
          uint32_t w[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) w[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
          __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(j.o.p) + (int64_t)(h * j.G + hq) * j.o.head +
                               (int64_t)(q.r0 + first + tok) * j.o.row + c * 32;
          if (j.wide) {
            store32(dst, w);
            store32(dst + 16, w + 8);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(dst)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
          }
        }
      }
    }
    if (C > 1) reinterpret_cast<float2*>(smem + L::STATS)[r] = ok ? make_float2(mrun, l) : make_float2(-INFINITY, 0.f);
    fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(over);
  } else if constexpr (E4M3) {
    regs_lower<L::REGS_CONV>();
    // ---------------- codes into bf16: K(0), V(0), K(1), ..; the next tile's codes are on their way meanwhile
    using W = Codes<D, L::CONV>;
    const int ct = tid - 256, part = ct & 3, panel = (ct >> 3) % W::NP, r0 = (ct >> 3) / W::NP * 2 + ((ct >> 2) & 1);
    const uint32_t page_bytes = (uint32_t)D << j.c.page_log2;   // of a head
    const uint8_t* const kp = static_cast<const uint8_t*>(j.c.k) + panel * 64 + part * 16;
    const uint8_t* const vp = static_cast<const uint8_t*>(j.c.v) + panel * 64 + part * 16;
    W w;
    // (a place behind the last, or of no page: what the registers hold stays, and is masked)
    auto fetch = [&](const uint8_t* pool, const uint8_t* scales, int u, int k) {
      const int e = u >> j.c.page_log2, in = u & (j.c.page_len - 1);
      const int at = e < keys.count ? page[e] : -1;   // (page * H + head: see where it is set)
      if (at >= 0) {
        w.x[k] = __ldg(reinterpret_cast<const uint4*>(pool + (int64_t)at * page_bytes + in * D));
        w.s[k] = __ldg(scales + ((int64_t)at << j.c.page_log2) + in);
      }
    };
    uint8_t* const to = smem + panel * PANEL + r0 * 128;
    const int at0 = ((2 * part) ^ (r0 & 7)) << 4, at1 = ((2 * part + 1) ^ (r0 & 7)) << 4;
#pragma unroll
    for (int k = 0; k < W::N; ++k) {
      w.x[k] = make_uint4(0, 0, 0, 0);
      w.s[k] = 127;
      if (n > 0) fetch(kp, j.c.ks, t0 * BK + r0 + k * W::STEP, k);
    }
#pragma unroll 1
    for (int turn = 0; turn < 2 * n; ++turn) {
      const bool is_k = (turn & 1) == 0;
      const int i = turn >> 1, sl = i % L::N;
      if (i >= L::N && !(ok = mbar_wait_warp_short((is_k ? k_empty : v_empty) + sl, (i / L::N - 1) & 1, abort_flag))) break;
      uint8_t* const tile = to + (is_k ? L::K : L::V) + sl * L::TB;
      const uint8_t* const next = is_k ? vp : kp;
      const uint8_t* const next_scales = is_k ? j.c.vs : j.c.ks;
      const int u0 = (t0 + ((turn + 1) >> 1)) * BK + r0;
      uint32_t big = 0;
#pragma unroll
      for (int k = 0; k < W::N; ++k) big = max(big, w.s[k]);
      const bool two = __any_sync(0xffffffffu, big > 134u);
#pragma unroll
      for (int k = 0; k < W::N; ++k) {
        const uint32_t s = w.s[k];
        const __nv_bfloat162 f = bf2((two && s > 134u ? 247u : s + 120u) * 0x00800080u);
        uint2 y0 = widen(w.x[k].x, f), y1 = widen(w.x[k].y, f), y2 = widen(w.x[k].z, f), y3 = widen(w.x[k].w, f);
        if (two) {
          const __nv_bfloat162 f2 = bf2(s == 255u ? 0x7fff7fffu : (s > 134u ? s : 127u) * 0x00800080u);
          y0 = make_uint2(times(y0.x, f2), times(y0.y, f2));
          y1 = make_uint2(times(y1.x, f2), times(y1.y, f2));
          y2 = make_uint2(times(y2.x, f2), times(y2.y, f2));
          y3 = make_uint2(times(y3.x, f2), times(y3.y, f2));
        }
        *reinterpret_cast<uint4*>(tile + k * W::STEP * 128 + at0) = make_uint4(y0.x, y0.y, y1.x, y1.y);
        *reinterpret_cast<uint4*>(tile + k * W::STEP * 128 + at1) = make_uint4(y2.x, y2.y, y3.x, y3.y);
        fetch(next, next_scales, u0 + k * W::STEP, k);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive((is_k ? k_full : v_full) + sl);
    }
    if (!ok && lane == 0) give_up(3);
    if (lane == 0) mbar_arrive(over);
  }
  fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    fence_after_sync();
    tmem_dealloc(tmem, TMEM_COLS);
  }
  if (C == 1) return;
  // ---- the cluster's parts: each CTA joins its share of the rows, a thread a row and D / C columns
  cluster.sync();
  if (warp >= 4 && warp < 8) {
    const int share = BQ / C, row = rank * share + r % share, g = r / share, cols = D / C;
    const int t2 = row / j.G, h2 = row - t2 * j.G;
    if (t2 < j.TQ && t2 < tokens) {
      float M = -INFINITY, sum = 0.f;
      for (int x = 0; x < C; ++x) M = fmaxf(M, cluster.map_shared_rank(reinterpret_cast<float2*>(smem + L::STATS), x)[row].x);
      float f[8];   // (0 times what is not finite is NaN, as it should be; a part that has seen nothing adds zeros, one whose
                    // scores are all -infinity the values that are not finite)
      for (int x = 0; x < C; ++x) {
        const float2 y = cluster.map_shared_rank(reinterpret_cast<float2*>(smem + L::STATS), x)[row];
        f[x] = y.x == M || y.x == -INFINITY ? 1.f : ex2(y.x - M);
        sum = fmaf(f[x], y.y, sum);
      }
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(j.o.p) + (int64_t)(h * j.G + h2) * j.o.head +
                           (int64_t)(q.r0 + first + t2) * j.o.row + g * cols;
      for (int c = 0; c < cols; c += 8) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int x = 0; x < C; ++x) {
          const float4* src = cluster.map_shared_rank(reinterpret_cast<float4*>(smem + L::JOIN), x) + ((g * cols + c) / 4) * BQ + row;
          const float4 a = src[0], z = src[BQ];
          v[0] = fmaf(f[x], a.x, v[0]); v[1] = fmaf(f[x], a.y, v[1]); v[2] = fmaf(f[x], a.z, v[2]); v[3] = fmaf(f[x], a.w, v[3]);
          v[4] = fmaf(f[x], z.x, v[4]); v[5] = fmaf(f[x], z.y, v[5]); v[6] = fmaf(f[x], z.z, v[6]); v[7] = fmaf(f[x], z.w, v[7]);
        }
        *reinterpret_cast<uint4*>(dst + c) = make_uint4(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv),
                                                        pack_bf16(v[4] * inv, v[5] * inv), pack_bf16(v[6] * inv, v[7] * inv));
      }
    }
  }
  cluster.sync();
}

template <int D, bool E4M3>
cudaError_t launch_d(const Maps& maps, const Job& job, const CUtensorMap& mq, dim3 grid, int C, cudaStream_t st) {
  using L = Lay<D, E4M3>;
  return launch_kernel(chosen_tc<D, E4M3>, grid, L::THREADS, L::BYTES, C, false, st, mq, maps.k, maps.v, job);
}

template <int D, bool E4M3>
cudaError_t set_limit() {
  return taken(cudaFuncSetAttribute(chosen_tc<D, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Lay<D, E4M3>::BYTES));
}

}  // namespace

cudaError_t chosen_tc_set_smem_limits() {
  cudaError_t e = set_limit<128, false>();
  if (e == cudaSuccess) e = set_limit<128, true>();
  if (e == cudaSuccess) e = set_limit<64, false>();
  if (e == cudaSuccess) e = set_limit<64, true>();
  return e;
}

cudaError_t launch_chosen_tc(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                             const Mask& m, const Chosen& how, cudaStream_t st) {
  const int G = Hq / c.H, TQ = BQ / G, n_sm = sm_count(), tiles = (how.tokens + TQ - 1) / TQ;
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  CUtensorMap mq;
  const int64_t dim[4] = {c.d, G, s.rows, c.H};
  const int64_t head = q.head ? q.head : c.d, row = q.row ? q.row : c.d;   // (one head or row: any stride)
  const int64_t stride[3] = {head * 2, row * 2, G * head * 2};
  const int box[4] = {64, G, TQ, 1};
  if (!make_map_4d(&mq, q.p, 2, dim, stride, box, 128)) return cudaErrorInvalidValue;
  const Job job{c, s, m, o, how, G, TQ, tiles, (uintptr_t)o.p % 32 == 0 && o.head % 16 == 0 && o.row % 16 == 0};
  // few units: a cluster each, while its CTAs have four key tiles or more (37 units of 28 tiles: 4 CTAs each 28 us, 2 33, 1 45)
  const int64_t units = (int64_t)std::min(how.slots, s.rows) * tiles * c.H, key_tiles = (int64_t)how.width * c.page_len / BK;
  int C = 1;
  while (C < 4 && units * C <= n_sm && key_tiles >= 8 * C) C *= 2;
  if ((int64_t)how.slots * tiles * C > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(how.slots * tiles * C, c.H);
  if (c.d == 128)
    return c.e4m3 ? launch_d<128, true>(maps, job, mq, grid, C, st) : launch_d<128, false>(maps, job, mq, grid, C, st);
  return c.e4m3 ? launch_d<64, true>(maps, job, mq, grid, C, st) : launch_d<64, false>(maps, job, mq, grid, C, st);
}

}  // namespace cache
}  // namespace dkv
