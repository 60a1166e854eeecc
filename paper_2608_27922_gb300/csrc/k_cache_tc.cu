// Attention of chunks of tokens over the paged cache on the tensor cores (include/dkv.h: dkv_cache_attend).
//
// A unit is two tiles of 128 query rows of one sequence and one key head.  With G query heads on a
// key head a tile holds TQ = 128 / G tokens, row = token * G + head, so that all of a group's
// queries meet a key tile in one product.  The unit's visible keys, in tiles of 128 positions (the sinks'
// tiles, then the window's), stream past both query tiles:
//   S_g = Q_g K^T            tcgen05.mma into TMEM, one softmax warpgroup a tile, thread = query row
//   P_g = exp2(S_g scale log2(e) - m_g)   packed bf16 over S_g in TMEM; what a row does not see is 0
//   O_g += P_g V             tcgen05.mma with A = P_g from TMEM
// with the running maximum raised only when a tile's exceeds it by more than 2^8 (O_g is then
// rescaled in TMEM).  Bound by the tensor pipe (4 d flops a row and key) and close to it by the exponentials.
//
// Pages come in by TMA, one box a page and 64-column panel, in the layout that the products read.
// A quantised cache's codes land beside that layout and eight warps turn them into bf16 in place
// of the copy: code bits shifted into bf16's fields are the value times 2^-120, one product with
// 2^120 times the row's scale makes it exact (bf16 holds every code times its scale).
//
// Persistent: one CTA an SM takes items, the first by its number and then whichever is next: whole units, or,
// where there are few of them, parts of C key tiles each, joined by cache_merge.  A sequence's last
// tokens come first, which see most, so that the last items are short ones.  The producer warp runs one item
// ahead and every barrier runs on from item to item, so that an item's first products are
// issued while the previous one's outputs are still being stored.
//
// Values in places that a row does not see meet its weight 0, and 0 times a NaN or an infinity
// is NaN.  So in a tile that some row of either query tile does not see whole, the softmax warps first clear what is
// not finite in V's tile, those of both (each before its own product); rows that do see such a value get it back at
// the end (wild_masks).
//
// Measured: 4,680 tokens of 40 heads over 14,040 keys in bf16 817 us, 1.65 PFLOP/s of 1.92 (tensor pipe 70% active; of a
// key tile's 2,960 cycles the issuing warp waits 480; back to back 880, at the power limit).  12 heads' block over its
// window of 14,040 keys in e4m3 343 us, 1.18 PFLOP/s (pipe 52%, issue slots 59%), in bf16 271.  A call of one item a
// CTA takes about 13 us beside its key tiles, and an item after another 3,000 cycles of outputs.
#include "attn_math.cuh"
#include "cache_internal.h"
#include "cache_plan.cuh"
#include "tc_ptx.cuh"

#include <algorithm>
#include <atomic>

namespace dkv {

bool make_map_4d(CUtensorMap* m, const void* base, int elem_bytes, const int64_t (&dim)[4], const int64_t (&stride)[3],
                 const int (&box)[4], int swizzle);

namespace cache {

namespace {

using namespace tc;
using namespace chunk;

constexpr int PANEL = 128 * 128;         // bytes of a 64-column panel of 128 rows
constexpr uint32_t TMEM_COLS = 512;      // S_0 [0,128), O_0 [128,256), S_1 [256,384), O_1 [384,512)
constexpr float RESCALE_LOG2 = 8.0f;

template <int D, bool E4M3>
struct Lay {
  static constexpr int NP = D / 64;                    // panels of a row
  static constexpr int TB = NP * PANEL;                // bytes of a 128-row tile
  static constexpr int NK = 2, NV = E4M3 ? 2 : 3;
  static constexpr int Q = 0;                          // [2 groups]
  static constexpr int K = 2 * TB;                     // [NK]
  static constexpr int V = K + NK * TB;                // [NV]
  static constexpr int CODES = V + NV * TB;            // [2] tiles of codes, [128][D]
  static constexpr int SCALES = CODES + (E4M3 ? 2 * 128 * D : 0);   // [2][128]
  static constexpr int CTRL = SCALES + (E4M3 ? 256 : 0);
  static constexpr size_t BYTES = CTRL + 512;          // base 1024-aligned (checked)
  static constexpr int SOFT0 = 4;                      // first softmax warp (warps 2 and 3 idle)
  static constexpr int CONV0 = SOFT0 + 8;              // first converting warp
  static constexpr int CONV = E4M3 ? 8 : 0;            // converting warps
  static constexpr int THREADS = (12 + CONV) * 32;
  // registers a thread of the first four warps, of the softmax warps and of the converting ones; the
  // launch gives every thread 96 (640 threads) or 168 (384)
  static constexpr int REGS_IO = E4M3 ? 80 : 88, REGS_SOFT = E4M3 ? 144 : 208, REGS_CONV = 56;
  static_assert(REGS_IO + 2 * REGS_SOFT + (E4M3 ? 2 * REGS_CONV : 0) <= (E4M3 ? 5 * 96 : 3 * 168), "register split");
  static constexpr int READERS = 1 + 8 + CONV;   // warps that follow the producer's items
  static_assert(BYTES <= 227 * 1024, "shared memory per CTA");
};

// ------------------------------------------------------------------ the items
// A count in scratch memory that nobody has cleared: call << CHUNK_COUNT_BITS | count once somebody has put that there.  One more;
// the count before it.
__device__ __forceinline__ void begin_count(unsigned long long* at, unsigned long long call) {
  const unsigned long long old = *reinterpret_cast<volatile unsigned long long*>(at);
  if ((old >> CHUNK_COUNT_BITS) != call) atomicCAS(at, old, call << CHUNK_COUNT_BITS);
}
__device__ __forceinline__ int taken_as(unsigned long long* at, unsigned long long call, unsigned long long old) {   // (old: of the addition)
  for (;; old = atomicAdd(at, 1ull)) {
    if ((old >> CHUNK_COUNT_BITS) == call) return (int)(old & ((1u << CHUNK_COUNT_BITS) - 1u));
    // what was added to was no count of this call's yet: put it there, or see that it is
    old = *reinterpret_cast<volatile unsigned long long*>(at);
    while ((old >> CHUNK_COUNT_BITS) != call) {
      const unsigned long long got = atomicCAS(at, old, call << CHUNK_COUNT_BITS);
      if (got == old) break;
      old = got;
    }
  }
}
__device__ __forceinline__ int take(unsigned long long* at, unsigned long long call) {
  return taken_as(at, call, atomicAdd(at, 1ull));
}

// ------------------------------------------------------------------ values that are not finite
// Clears what is not finite in one bf16 row (128-byte swizzled panels), and says so in *met before it does: the other
// query tile's products may meet the cleared row at once, and its outputs wait for nothing else.
template <int D>
__device__ __forceinline__ void clear_row(uint8_t* tile, int row, volatile int* met, int item) {
  uint32_t any = 0;
#pragma unroll
  for (int c = 0; c < D / 8; ++c) {
    uint4* p = reinterpret_cast<uint4*>(tile + (c >> 3) * PANEL + row * 128 + (((c & 7) ^ (row & 7)) << 4));
    const uint4 x = *p;
    // an exponent field of ones plus one carries into the (cleared) sign
    any |= ((x.x & 0x7f807f80u) + 0x00800080u) | ((x.y & 0x7f807f80u) + 0x00800080u) |
           ((x.z & 0x7f807f80u) + 0x00800080u) | ((x.w & 0x7f807f80u) + 0x00800080u);
  }
  if ((any & 0x80008000u) == 0) return;
  *met = item;
  __threadfence_block();
#pragma unroll 1
  for (int c = 0; c < D / 2; ++c) {
    uint32_t* p = reinterpret_cast<uint32_t*>(tile + (c >> 5) * PANEL + row * 128 + ((((c >> 2) & 7) ^ (row & 7)) << 4)) + (c & 3);
    const uint32_t x = *p, bad = ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    if (bad) *p = x & ~(((bad >> 15) & 0x00010001u) * 0xffffu);
  }
}

// The columns [c0, c0 + 32) in which row (position range [lo, end) and sinks) meets a NaN, +inf, -inf in the tiles
// of this item that clear_row may have been at.
struct Wild {
  uint32_t nan, pos, neg;
};
template <int D, bool E4M3>
__device__ __noinline__ Wild wild_masks(const Job& j, const Item& it, int end, int lo, int c0) {
  Wild w{0, 0, 0};
  const Span a = span_of(j.m, it.n, it.p0, it.len, 0, j.TQ), z = span_of(j.m, it.n, it.p0, it.len, 1, j.TQ);
#pragma unroll 1
  for (int i = it.i0; i < it.i1; ++i) {
    const int kt = tile_of(it, i);
    if ((!active(a, kt) || all_seen(a, kt)) && (!active(z, kt) || all_seen(z, kt))) continue;
#pragma unroll 1
    for (int p = kt * BK; p < min(end, kt * BK + BK); ++p) {
      if (p < lo && !(j.m.window && p < j.m.sinks)) continue;
      const int64_t at = pool_row(j.c, j.s, it.b, it.h, p);
      if (at < 0) continue;
      if (E4M3) {
        if (j.c.vs[at] == 255) w.nan = 0xffffffffu;
        continue;
      }
      const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(j.c.v) + at * D + c0;
#pragma unroll 1
      for (int k = 0; k < 32; ++k) {
        const float x = __bfloat162float(v[k]);
        if (isnan(x)) w.nan |= 1u << k;
        if (x == INFINITY) w.pos |= 1u << k;
        if (x == -INFINITY) w.neg |= 1u << k;
      }
    }
  }
  return w;
}

// 32 bytes in one store.  (A row a thread, a warp's store is 32 lines whatever its width, a cycle each, and what
// else the SM's load and store unit has to do waits: as 16-byte stores an item's outputs took 5,000 cycles.)
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// 16 bytes to shared memory (the first `bytes` of them copied, the rest zeros); copies_arrive: an arrival at bar when
// the thread's copies so far are there.
__device__ __forceinline__ void copy16(void* to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Bits k < x.
__device__ __forceinline__ uint32_t below(int x) { return x <= 0 ? 0u : x >= 32 ? 0xffffffffu : (1u << x) - 1u; }

// Scores of what the row does not see become -inf (columns k0 .. k0 + 31 of the positions).
__device__ __forceinline__ void mask_row(float (&v)[32], int k0, int end, int lo, int sk) {
  const uint32_t see = below(end - k0) & (~below(lo - k0) | below(sk - k0));
#pragma unroll
  for (int k = 0; k < 32; ++k)
    if (!((see >> k) & 1u)) v[k] = -INFINITY;
}

// ------------------------------------------------------------------ codes into bf16
// Four bf16 (two pairs) from four codes: a code's bits in bf16's fields (sign; three zero bits and the first
// of the exponent above; the rest below) are its value times 2^-120, subnormal codes included; f
// holds 2^120 times the scale.
__device__ __forceinline__ uint2 widen(uint32_t w, __nv_bfloat162 f) {
  const uint32_t hi = (w & 0x80808080u) | ((w >> 4) & 0x07070707u), lo = (w << 4) & 0xf0f0f0f0u;
  const uint32_t a = __byte_perm(lo, hi, 0x5140), b = __byte_perm(lo, hi, 0x7362);
  const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), f);
  const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&b), f);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
}
__device__ __forceinline__ __nv_bfloat162 bf2(uint32_t bits) { return *reinterpret_cast<const __nv_bfloat162*>(&bits); }
__device__ __forceinline__ uint32_t times(uint32_t x, __nv_bfloat162 f) {
  const __nv_bfloat162 y = __hmul2(bf2(x), f);
  return *reinterpret_cast<const uint32_t*>(&y);
}

// A [128][D] tile of codes and its rows' scales into a swizzled bf16 tile (W warps); whether a row of
// the warp's is NaN.  Eight neighbouring threads take 64 columns of two rows, chosen so that neither the 16-byte loads (128-byte
// swizzled codes at D = 128, plain ones at 64) nor the 16-byte stores of a quarter warp share a bank: rows r
// and r ^ 5 at D = 128, two adjacent ones at 64.
template <int D, int W>
__device__ __forceinline__ bool widen_tile(const uint8_t* codes, const uint8_t* scales, uint8_t* tile, int t) {
  constexpr int PANELS = D / 64, UNITS = 16 * PANELS / W;   // units of (8 rows, 64 columns): a warp's
  static_assert(W % PANELS == 0, "a warp stays in its panel");
  constexpr int ROWS = W / PANELS * 8;                // rows from one of them to the next
  const int warp = t >> 5, quarter = (t & 31) >> 3, half = (t >> 2) & 1, c = t & 3;
  const int r8 = D == 128 ? (half ? quarter ^ 5 : quarter) : 2 * quarter + half;
  const int row = (warp / PANELS) * 8 + r8, panel = warp % PANELS;
  codes += row * D + (D == 128 ? (((panel * 4 + c) ^ r8) << 4) : c * 16);
  uint8_t* lo = tile + panel * PANEL + row * 128 + (((2 * c) ^ r8) << 4);
  uint8_t* hi = tile + panel * PANEL + row * 128 + (((2 * c + 1) ^ r8) << 4);
  uint32_t s[UNITS], big = 0;
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    s[k] = scales[row + k * ROWS];
    big = max(big, s[k]);
  }
  // one factor where 2^120 times the scale is a bf16 number; else two, the scale by itself (255: NaN)
  if (__any_sync(0xffffffffu, big > 134u)) {
#pragma unroll 1
    for (int k = 0; k < UNITS; ++k) {
      const uint32_t sk = scales[row + k * ROWS];
      const uint4 x = *reinterpret_cast<const uint4*>(codes + k * ROWS * D);
      const __nv_bfloat162 f = bf2((sk > 134u ? 247u : sk + 120u) * 0x00800080u);
      const __nv_bfloat162 f2 = bf2(sk == 255u ? 0x7fff7fffu : (sk > 134u ? sk : 127u) * 0x00800080u);
      const uint2 y0 = widen(x.x, f), y1 = widen(x.y, f), y2 = widen(x.z, f), y3 = widen(x.w, f);
      *reinterpret_cast<uint4*>(lo + k * ROWS * 128) = make_uint4(times(y0.x, f2), times(y0.y, f2), times(y1.x, f2), times(y1.y, f2));
      *reinterpret_cast<uint4*>(hi + k * ROWS * 128) = make_uint4(times(y2.x, f2), times(y2.y, f2), times(y3.x, f2), times(y3.y, f2));
    }
    return __any_sync(0xffffffffu, big == 255u);
  } else {
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
      const uint4 x = *reinterpret_cast<const uint4*>(codes + k * ROWS * D);
      const __nv_bfloat162 f = bf2((s[k] + 120u) * 0x00800080u);
      const uint2 y0 = widen(x.x, f), y1 = widen(x.y, f), y2 = widen(x.z, f), y3 = widen(x.w, f);
      *reinterpret_cast<uint4*>(lo + k * ROWS * 128) = make_uint4(y0.x, y0.y, y1.x, y1.y);
      *reinterpret_cast<uint4*>(hi + k * ROWS * 128) = make_uint4(y2.x, y2.y, y3.x, y3.y);
    }
    return false;
  }
}

// ------------------------------------------------------------------ the kernel
template <int D, bool E4M3>
__global__ void __launch_bounds__(Lay<D, E4M3>::THREADS, 1)
    cache_attend_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Job j) {
  using L = Lay<D, E4M3>;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0u) {   // 128-byte-swizzled tiles need 1024-byte alignment
    if (threadIdx.x == 0) fail(j.c.status, DEV_INCONSISTENT, 9903);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::CTRL);
  uint64_t* q_full = bars + 0;
  uint64_t* q_empty = bars + 1;     // all score products of the item complete
  uint64_t* k_full = bars + 2;      // [2]
  uint64_t* k_empty = bars + 4;     // [2]
  uint64_t* v_full = bars + 6;      // [3]
  uint64_t* v_empty = bars + 9;     // [3]
  uint64_t* c_full = bars + 12;     // [2] tiles of codes
  uint64_t* c_empty = bars + 14;    // [2]
  uint64_t* s_full = bars + 16;     // [2] by group
  uint64_t* p_full = bars + 18;     // [2]
  uint64_t* o_full = bars + 20;     // [2]
  uint64_t* it_full = bars + 22;    // [2] items
  uint64_t* it_empty = bars + 24;   // [2]
  uint64_t* done = bars + 26;
  uint64_t* over = bars + 27;       // every role but the producer has ended
  Item* items = reinterpret_cast<Item*>(bars + 28);                        // [2]
  volatile int* wild = reinterpret_cast<volatile int*>(items + 2);         // [2] number of the last item with values cleared
  // [2] e4m3: a byte a widening warp, not 0 where it met a NaN row of the slot's values
  volatile unsigned long long* nan_rows = reinterpret_cast<volatile unsigned long long*>(items + 2) + 1;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(items + 2) + 6;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  static_assert(28 * 8 + 2 * sizeof(Item) + 32 <= 512, "control block");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 64) {
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full + i, E4M3 ? L::CONV : 1);
      mbar_init(k_empty + i, 1);
      mbar_init(c_full + i, 1 + 32);   // the codes', and each of the producer's lanes for its scales
      mbar_init(c_empty + i, E4M3 ? L::CONV : 1);
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, 4);
      mbar_init(o_full + i, 1);
      mbar_init(it_full + i, 1);
      mbar_init(it_empty + i, L::READERS);
      wild[i] = 0;
    }
    for (int i = 0; i < 3; ++i) {
      mbar_init(v_full + i, E4M3 ? L::CONV : 1);
      mbar_init(v_empty + i, 1);
    }
    mbar_init(done, 1);
    mbar_init(over, 1 + 8 + L::CONV);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(tmem_holder, TMEM_COLS);
  if (blockIdx.x == 0 && threadIdx.x < 3) begin_count(j.count + threadIdx.x, j.call);
  pdl_trigger();   // cache_merge's blocks start as SMs free up, and wait there
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *tmem_holder;

  auto give_up = [&](int site) {
    *abort_flag = 1;
    fail(j.c.status, DEV_TIMEOUT, SITE_WAIT + site);
  };
  // Reader warps: the next item (state 0: none, or the CTA has given up).
  auto next_item = [&](uint32_t n) -> Item {
    Item x;
    x.state = 0;
    if (mbar_wait_warp_short(it_full + (n & 1), (n >> 1) & 1, abort_flag)) {
      x = items[n & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(it_empty + (n & 1));
    }
    return x;
  };

  if (warp < L::SOFT0) {
    regs_lower<L::REGS_IO>();
    if (warp == 0) {
      // ---------------- producer: items; Q, then K(0), V(0), K(1), ..  It also watches the time for all roles' waits: its
      // own wait for their work, tile by tile, and at last for their end.
      Cursor cursor{};
      const Plan plan = make_plan(j, gridDim.x, cursor.k);
      if (plan.C == 0 && j.s.n > 1 && j.s.n <= 32) order(cursor.k, j.s.n);
      if (blockIdx.x == 0 && lane == 0) *j.plan = stored_plan(plan);
      const int rows = min(j.c.page_len, BK), np = BK / rows;   // rows and boxes of a tile
      uint32_t tc = 0, nq = 0, ni = 0, cc = 0;
      bool ok = true;
      // the next item's number: asked for (and waited for only where it is wanted), wanted
      unsigned long long ticket = 0;
      auto ask = [&]() {
        if (lane == 0) ticket = atomicAdd(j.count, 1ull);
      };
      auto next = [&]() {
        int i = 0;
        if (lane == 0) i = (int)gridDim.x + taken_as(j.count, j.call, ticket);
        return __shfl_sync(0xffffffffu, i, 0);
      };
#pragma unroll 1
      for (int it = blockIdx.x;; ++ni) {
        Item x;
        x.state = 0;
        List l{};
#pragma unroll 1
        while (it < plan.items) {
          x = make_item(j, plan, it, cursor, l);
          if (x.state) break;
          ask();
          it = next();
        }
        if (x.state) {
          if (x.part >= 0) {
            int slot = 0;
            if (lane == 0) {
              slot = min(take(j.count + 2, j.call), MAX_PARTS - 1);
              j.slot[it] = slot;
            }
            x.part = __shfl_sync(0xffffffffu, slot, 0);
          }
        }
        if (ni >= 2) ok = mbar_wait_warp(it_empty + (ni & 1), ((ni >> 1) & 1) ^ 1, abort_flag);
        if (!ok) break;
        if (lane == 0) {
          items[ni & 1] = x;
          mbar_arrive(it_full + (ni & 1));
        }
        __syncwarp();
        if (x.state == 0) break;
        const int n = x.i1 - x.i0;
        if (n <= 0) {
          ask();
          it = next();
          continue;
        }
        // pages of the list's tiles, 32 boxes at a time with the lanes: box (i - base) np + .. of tile i
        const int np_log2 = __ffs(np) - 1, batch = 32 >> np_log2;
        auto entry_of = [&](int first) -> int {
          const int i = first + (lane >> np_log2), k0 = tile_of(x, i) * BK + (lane & (np - 1)) * rows;
          return i < x.i1 && k0 < l.end && (k0 + rows > l.lo || k0 < l.sk)
                     ? __ldg(j.s.table + (int64_t)x.b * j.s.max_pages + (k0 >> j.c.page_log2)) : 0;
        };
        int base = x.i0, pages = entry_of(base), pages_next = entry_of(base + batch);
        if (nq > 0 && !(ok = mbar_wait_warp(q_empty, (nq - 1) & 1, abort_flag))) break;
        ++nq;
        if (lane == 0) {
          const int groups = x.n > j.TQ ? 2 : 1, bytes = j.TQ * j.G * 128;
          mbar_arrive_expect_tx(q_full, groups * L::NP * bytes);
          for (int g = 0; g < groups; ++g)
            for (int p = 0; p < L::NP; ++p)
              tma_load_4d(smem + L::Q + g * L::TB + p * PANEL, &tmQ, q_full, p * 64, 0, x.r0 + g * j.TQ, x.h);
        }
        __syncwarp();
        // one tile of K or V: a lane a box
        auto load = [&](bool is_k, int i) -> bool {
          const int kt = tile_of(x, i);
          const uint32_t t = tc + (uint32_t)(i - x.i0);
          const int box = E4M3 ? lane : lane / L::NP, panel = E4M3 ? 0 : lane % L::NP;
          if (i - base >= batch) {          // (K comes first to a tile)
            base += batch;
            pages = pages_next;
            pages_next = entry_of(base + batch);
          }
          // the box's page; nobody's (zeros) where no row of the unit sees into it
          const int k0 = kt * BK + box * rows;
          int page = __shfl_sync(0xffffffffu, pages, (((i - base) << np_log2) + box) & 31);
          if (!(box < np && k0 < l.end && (k0 + rows > l.lo || k0 < l.sk))) {
            page = j.c.n_pages;
          } else if ((unsigned)page >= (unsigned)j.c.n_pages) {
            fail(j.c.status, DEV_INCONSISTENT, SITE_PAGE);
            page = j.c.n_pages;
          }
          const int slot = k0 & (j.c.page_len - 1);
          if (E4M3) {
            const uint32_t c = cc++;
            uint64_t* bar = c_full + (c & 1);
            if (c >= 2 && !mbar_wait_warp(c_empty + (c & 1), ((c >> 1) & 1) ^ 1, abort_flag)) return false;
            if (lane == 0) mbar_arrive_expect_tx(bar, BK * D);
            __syncwarp();
            if (box < np)
              tma_load_4d(smem + L::CODES + (c & 1) * 128 * D + box * rows * D, is_k ? &tmK : &tmV, bar, 0, slot, x.h, page);
            // the scales, 16 bytes a lane (zeros where the page is nobody's)
            page = __shfl_sync(0xffffffffu, page, (lane * 16) >> (7 - np_log2) & 31);
            if (lane < 8)
              copy16(smem + L::SCALES + (c & 1) * 128 + lane * 16,
                     (is_k ? j.c.ks : j.c.vs) + (page < j.c.n_pages
                         ? (((int64_t)page * j.c.H + x.h) << j.c.page_log2) + ((kt * BK + lane * 16) & (j.c.page_len - 1)) : 0),
                     page < j.c.n_pages ? 16 : 0);
            copies_arrive(bar);
          } else {
            const uint32_t nb = is_k ? L::NK : L::NV, sl = t % nb;
            uint64_t* bar = (is_k ? k_full : v_full) + sl;
            if (t >= nb && !mbar_wait_warp((is_k ? k_empty : v_empty) + sl, (t / nb - 1) & 1, abort_flag)) return false;
            if (lane == 0) mbar_arrive_expect_tx(bar, L::TB);
            __syncwarp();
            if (box < np)
              tma_load_4d(smem + (is_k ? L::K : L::V) + sl * L::TB + panel * PANEL + box * rows * 128, is_k ? &tmK : &tmV,
                          bar, panel * 64, slot, x.h, page);
          }
          __syncwarp();
          return true;
        };
        ok = load(true, x.i0);
        for (int i = x.i0; ok && i < x.i1; ++i) {
          if (i == max(x.i0, x.i1 - 2)) ask();
          ok = load(false, i);
          if (ok && i + 1 < x.i1) ok = load(true, i + 1);
        }
        tc += n;
        if (!ok) break;
        it = next();
      }
      // the last CTA to run out of items clears the counts (a replayed graph's next call has the same number)
      if (lane == 0 && take(j.count + 1, j.call) == (int)gridDim.x - 1)
        for (int i = 0; i < 3; ++i) atomicExch(j.count + i, 0ull);
      if (ok) ok = mbar_wait_warp(over, 0, abort_flag);
      if (!ok) {
        if (lane == 0) give_up(0);
        // copies may be in flight that nobody waits for any more: far longer than one takes
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 50000ull) {
        }
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer (the whole warp, one elected lane issues)
      constexpr uint32_t id_s = idesc_bf16(BQ, BK), id_o = idesc_bf16(BQ, D, /*b_mn_major=*/true);
      const uint64_t qd0 = desc_sw128(smem_u32(smem + L::Q)), kd0 = desc_sw128(smem_u32(smem + L::K));
      const uint64_t vd0 = desc_sw128_mn(smem_u32(smem + L::V), PANEL, 1024);
      uint32_t nq = 0, ks = 0, kph = 0, vs = 0, vph = 0, pph[2] = {0, 0};   // slots and phases
      bool ok = true;
      auto step = [](uint32_t& slot, uint32_t& phase, uint32_t n) {
        if (++slot == n) {
          slot = 0;
          phase ^= 1;
        }
      };
      auto issue_s = [&](int g, uint32_t slot) {
        const uint64_t qd = desc_add(qd0, g * L::TB), kd = desc_add(kd0, slot * L::TB);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = (kk >> 2) * PANEL + (kk & 3) * 32;
            mma_bf16(tmem + g * 256, desc_add(qd, off), desc_add(kd, off), id_s, kk > 0);
          }
          mma_commit(s_full + g);
        }
        __syncwarp();
      };
      auto issue_pv = [&](int g, uint32_t slot, bool first) {
        const uint64_t vd = desc_add(vd0, slot * L::TB);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            mma_bf16_ts(tmem + g * 256 + 128, tmem + g * 256 + kk * 8, desc_add(vd, kk * 2048), id_o,
                        first && kk == 0 ? 0u : 1u);
        }
        __syncwarp();
      };
      auto commit = [&](uint64_t* bar) {
        if (elect_one()) mma_commit(bar);
        __syncwarp();
      };
      // (lane 0's copy of the item for all: loop bounds, slots and descriptors stay warp-uniform, where the
      // tensor instructions take them from)
      auto uni = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
      for (uint32_t ni = 0; ok; ++ni) {
        Item x = next_item(ni);
        if (uni(x.state) == 0) break;
        x.i0 = uni(x.i0);
        x.i1 = uni(x.i1);
        x.ns = uni(x.ns);
        x.w0 = uni(x.w0);
        const int n = x.i1 - x.i0;
        if (n <= 0) continue;
        Span sp[2];
        int last[2];            // list index of the group's last active tile
        bool fresh[2] = {true, true};
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          sp[g] = span_of(j.m, uni(x.n), uni(x.p0), uni(x.len), g, j.TQ);
          const int kt = sp[g].any_end - 1;
          last[g] = kt < x.ns ? kt : x.ns + (kt - x.w0);
        }
        ok = mbar_wait_warp_short(q_full, nq & 1, abort_flag) &&
             mbar_wait_warp_short(k_full + ks, kph, abort_flag);
        ++nq;
        if (!ok) break;
        fence_after_sync();
        int kt = tile_of(x, x.i0);
        bool act[2] = {active(sp[0], kt), active(sp[1], kt)};
        if (act[0]) issue_s(0, ks);
        if (act[1]) issue_s(1, ks);
        commit(k_empty + ks);
        if (n == 1) commit(q_empty);
        step(ks, kph, L::NK);
        for (int i = x.i0; i < x.i1; ++i) {
          const bool next = i + 1 < x.i1;
          kt = tile_of(x, i + 1);
          const bool actn[2] = {next && active(sp[0], kt), next && active(sp[1], kt)};
          if (!(ok = mbar_wait_warp_short(v_full + vs, vph, abort_flag))) break;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (act[g]) {
              if (!(ok = mbar_wait_warp_short(p_full + g, pph[g], abort_flag))) break;
              pph[g] ^= 1;
              fence_after_sync();
              issue_pv(g, vs, fresh[g]);
              fresh[g] = false;
              if (i == last[g]) commit(o_full + g);
            }
            if (g == 0 && next) {
              if (!(ok = mbar_wait_warp_short(k_full + ks, kph, abort_flag))) break;
              fence_after_sync();
            }
            if (actn[g]) issue_s(g, ks);
            act[g] = actn[g];
          }
          if (!ok) break;
          commit(v_empty + vs);
          if (next) {
            commit(k_empty + ks);
            if (i + 2 == x.i1) commit(q_empty);
            step(ks, kph, L::NK);
          }
          step(vs, vph, L::NV);
        }
        if (!ok) break;
#pragma unroll
        for (int g = 0; g < 2; ++g)   // a part that ends before the group's last tile
          if (!fresh[g] && last[g] >= x.i1) commit(o_full + g);
      }
      if (!ok && lane == 0) give_up(1);
      // every product complete before TMEM is freed
      commit(done);
      volatile int no_abort = 0;
      mbar_wait(done, 0, &no_abort);
      if (lane == 0) mbar_arrive(over);
    }
  } else if (warp < L::CONV0) {
    regs_raise<L::REGS_SOFT>();
    // ---------------- softmax group g over query tile g, thread = query row = TMEM lane
    const int g = (warp - L::SOFT0) >> 2, qd = warp & 3, r = qd * 32 + lane;
    const uint32_t lane_off = (uint32_t)(qd * 32) << 16;
    const uint32_t sc = tmem + lane_off + g * 256, oc = sc + 128;
    const int tok = r / j.G, hq = r - tok * j.G;
    uint32_t ns = 0, no = 0, tc = 0;
    bool ok = true;
    for (uint32_t ni = 0; ok; ++ni) {
      // (the item stays in its slot until its outputs are stored: fewer registers)
      if (!mbar_wait_warp_short(it_full + (ni & 1), (ni >> 1) & 1, abort_flag)) break;
      const Item& x = items[ni & 1];
      if (x.state == 0) break;
      const Span sp = span_of(j.m, x.n, x.p0, x.len, g, j.TQ);
      const Edges others = edges_of(span_of(j.m, x.n, x.p0, x.len, 1 - g, j.TQ), g);
      const int p = x.p0 + g * j.TQ + tok;                // the row's position
      const int end = p >= 0 ? visible_end(j.m, p, x.len) : 0, lo = window_first(j.m, end);
      const int sk = j.m.window ? j.m.sinks : 0;
      float mrun = -INFINITY, l = 0.f;
      bool some = false;
      for (int i = x.i0; i < x.i1; ++i) {
        const int kt = tile_of(x, i);
        if (!active(sp, kt)) continue;
        const bool partial = !all_seen(sp, kt);
        if (partial || in(others, kt)) {
          const uint32_t t = tc + (uint32_t)(i - x.i0);
          if (!(ok = mbar_wait_warp_short(v_full + t % L::NV, (t / L::NV) & 1, abort_flag))) break;
          if (!E4M3 || nan_rows[t % L::NV] != 0) clear_row<D>(smem + L::V + (t % L::NV) * L::TB, r, wild + (ni & 1), (int)ni + 1);
          fence_async_smem();
        }
        if (!(ok = mbar_wait_warp_short(s_full + g, ns & 1, abort_flag))) break;
        ++ns;
        fence_after_sync();
        // the row's 128 scores, 64 at a time and read twice (maximum, weights): fewer registers and
        // half the instructions than the whole row at once, which the instruction caches repay.  Masked ones go
        // back into their place in between.
        const int k0 = kt * BK;
        float tmax;
        {
          float t[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] = -INFINITY;
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            float a[32], b[32];
            tmem_ld32(sc + half * 64, a);
            tmem_ld32(sc + half * 64 + 32, b);
            tmem_wait_ld();
            if (partial) {
              mask_row(a, k0 + half * 64, end, lo, sk);
              mask_row(b, k0 + half * 64 + 32, end, lo, sk);
              tmem_st32(sc + half * 64, reinterpret_cast<uint32_t(&)[32]>(a));
              tmem_st32(sc + half * 64 + 32, reinterpret_cast<uint32_t(&)[32]>(b));
            }
            max_acc(t, a);
            max_acc(t, b);
          }
          if (partial) tmem_wait_st();
          tmax = fmaxf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])), fmaxf(fmaxf(t[4], t[5]), fmaxf(t[6], t[7])));
        }
        tmax *= j.m.sl2;
        // S_g of this tile complete implies O_g of the one before complete (issued earlier by one thread)
        const bool raise = tmax > mrun + RESCALE_LOG2 || (mrun == -INFINITY && tmax > -INFINITY);
        const float mprev = mrun;
        if (raise) {
          l *= some ? ex2(mrun - tmax) : 0.f;
          mrun = tmax;
        }
        const float nm = mrun == -INFINITY ? 0.f : -mrun;   // (a row that has seen nothing yet: all weights 0)
        float2 lab = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          float a[32], b[32];
          uint32_t pk[32];
          tmem_ld32(sc + half * 64, a);
          tmem_ld32(sc + half * 64 + 32, b);
          tmem_wait_ld();
          exp_pack(a, b, j.m.sl2, nm, lab, pk);
          tmem_st32(sc + half * 32, pk);
        }
        if (__any_sync(0xffffffffu, raise && some)) {
          const float alpha = raise ? ex2(mprev - mrun) : 1.0f;
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            float v[32];
            tmem_ld32(oc + c * 32, v);
            tmem_wait_ld();
            uint32_t w32[32];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const float2 y = __fmul2_rn(make_float2(v[2 * k], v[2 * k + 1]), make_float2(alpha, alpha));
              w32[2 * k] = __float_as_uint(y.x);
              w32[2 * k + 1] = __float_as_uint(y.y);
            }
            tmem_st32(oc + c * 32, w32);
          }
        }
        some = true;
        l += lab.x + lab.y;
        tmem_wait_st();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + g);
      }
      tc += (uint32_t)max(0, x.i1 - x.i0);
      if (ok && some) {
        ok = mbar_wait_warp_short(o_full + g, no & 1, abort_flag);
        ++no;
      }
      if (!ok) break;
      fence_after_sync();
      // ---- outputs
      const int token = g * j.TQ + tok;
      const bool mine = tok < j.TQ && token < x.n;
      const bool whole = x.part < 0;
      const bool fix = wild[ni & 1] == (int)ni + 1;
      const float inv = l == 0.f ? 0.f : 1.0f / l;         // (a NaN stays one)
      float* part = whole ? nullptr : j.parts + (int64_t)x.part * (256 * (D + 1));
      if (!whole) part[256 * D + g * BQ + r] = l == 0.f ? -INFINITY : mrun + log2f(l);
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float v[32];
        if (some) {   // warp-uniform
          tmem_ld32(oc + c * 32, v);
          tmem_wait_ld();
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = some ? v[k] * inv : 0.f;
        if (fix) {
          const Wild w = wild_masks<D, E4M3>(j, x, mine ? end : 0, lo, c * 32);
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            if ((w.pos >> k) & 1u) v[k] += INFINITY;
            if ((w.neg >> k) & 1u) v[k] -= INFINITY;
            if ((w.nan >> k) & 1u) v[k] = __int_as_float(0x7fffffff);
          }
        }
        if (!whole) {
          float4* dst = reinterpret_cast<float4*>(part) + (c * 8) * 256 + g * BQ + r;
#pragma unroll
          for (int k = 0; k < 8; ++k) dst[k * 256] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        } else if (mine) {
          uint32_t w[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) w[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
          __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(j.o.p) + (int64_t)(x.h * j.G + hq) * j.o.head +
                               (int64_t)(x.r0 + token) * j.o.row + c * 32;
          if (j.wide) {
            store32(dst, w);
            store32(dst + 16, w + 8);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(dst)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
          }
        }
      }
      fence_before_sync();   // O_g read before the next item's products overwrite it (they wait for its weights)
      __syncwarp();
      if (lane == 0) mbar_arrive(it_empty + (ni & 1));
    }
    if (!ok && lane == 0) give_up(2);
    if (lane == 0) mbar_arrive(over);
  } else if constexpr (E4M3) {
    regs_lower<L::REGS_CONV>();
    // ---------------- codes into bf16, in the order of the copies: K(0), V(0), K(1), V(1), .. (V(i) is wanted
    // half a step before K(i + 1))
    const int tid = threadIdx.x - L::CONV0 * 32;
    uint32_t tc = 0, cc = 0;
    bool ok = true;
    auto turn = [&](bool is_k, uint32_t t) -> bool {
      const uint32_t c = cc++;
      const uint32_t nb = is_k ? L::NK : L::NV, sl = t % nb;
      if (!mbar_wait_warp_short(c_full + (c & 1), (c >> 1) & 1, abort_flag)) return false;
      if (t >= nb && !mbar_wait_warp_short((is_k ? k_empty : v_empty) + sl, (t / nb - 1) & 1, abort_flag)) return false;
      const bool nan = widen_tile<D, L::CONV>(smem + L::CODES + (c & 1) * 128 * D, smem + L::SCALES + (c & 1) * 128,
                    smem + (is_k ? L::K : L::V) + sl * L::TB, tid);
      if (!is_k && lane == 0) reinterpret_cast<volatile uint8_t*>(nan_rows + sl)[warp - L::CONV0] = nan;
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive((is_k ? k_full : v_full) + sl);
        mbar_arrive(c_empty + (c & 1));
      }
      return true;
    };
    for (uint32_t ni = 0; ok; ++ni) {
      const Item x = next_item(ni);
      if (x.state == 0) break;
      const int n = x.i1 - x.i0;
      if (n <= 0) continue;
#pragma unroll 1
      for (int k = 0; ok && k < 2 * n; ++k) ok = turn((k & 1) == 0, tc + (k >> 1));
      tc += n;
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
}

// Joins the parts of cut units: O = sum_s 2^(lse_s - max) O_s / sum_s 2^(lse_s - max), parts in
// order.  Block (unit, 32 rows), thread = (row, D / 8 columns).
constexpr int MG_ROWS = 32;

template <int D>
__global__ void __launch_bounds__(256) cache_merge(const __grid_constant__ Job j) {
  pdl_wait();
  const int4 p = *j.plan;
  __shared__ float lse[MAX_CUT][MG_ROWS];
  __shared__ int slots[MAX_CUT];
  __shared__ Unit su;
  __shared__ int sS;
  const int units = min(p.x, CUT_ROUNDS * (int)gridDim.x);   // (no call that cuts has more)
  for (int unit = max(p.z, 0) + blockIdx.x; unit < units; unit += gridDim.x) {   // uniform
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    const Joined x = joined(j, p, unit);
    if (x.n > 1 && lane < x.n) {
      slots[lane] = slot_of(j.slot, x.at + lane * x.step);
      if (slots[lane] < 0) fail(j.c.status, DEV_INCONSISTENT, SITE_PART);
    }
    if (lane == 0) {
      su = x.u;
      sS = x.n;
    }
  }
  __syncthreads();
  const int S = sS, row0 = blockIdx.y * MG_ROWS;
  if (S < 2) continue;
  auto part = [&](int s) { return j.parts + (int64_t)slots[s] * (256 * (D + 1)); };
  for (int e = threadIdx.x; e < S * MG_ROWS; e += 256)
    lse[e / MG_ROWS][e % MG_ROWS] = slots[e / MG_ROWS] < 0 ? -INFINITY : part(e / MG_ROWS)[256 * D + row0 + e % MG_ROWS];
  __syncthreads();
  const Unit u = su;
  const int rl = threadIdx.x % MG_ROWS, row = row0 + rl, q = threadIdx.x / MG_ROWS;   // 8 column groups
  const int g = row / BQ, r = row % BQ, tok = r / j.G, token = g * j.TQ + tok;
  if (tok >= j.TQ || u.t * 2 * j.TQ + token >= u.q.n) continue;
  float mx = -INFINITY, den = 0.f;
  for (int s = 0; s < S; ++s) mx = fmaxf(mx, lse[s][rl]);
  float o[D / 8];
#pragma unroll
  for (int k = 0; k < D / 8; ++k) o[k] = 0.f;
  for (int s = 0; s < S; ++s) {
    const float z = lse[s][rl];
    if (z == -INFINITY) continue;                          // the part saw nothing of this row's
    const float w = exp2f(z - mx);
    den += w;
    const float4* src = reinterpret_cast<const float4*>(part(s)) + row;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const float4 x = src[(q * (D / 32) + k) * 256];
      o[4 * k] = fmaf(w, x.x, o[4 * k]);
      o[4 * k + 1] = fmaf(w, x.y, o[4 * k + 1]);
      o[4 * k + 2] = fmaf(w, x.z, o[4 * k + 2]);
      o[4 * k + 3] = fmaf(w, x.w, o[4 * k + 3]);
    }
  }
  const float inv = den == 0.f ? 0.f : 1.0f / den;
  uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(j.o.p) +
                                              (int64_t)(u.h * j.G + r - tok * j.G) * j.o.head +
                                              (int64_t)(u.q.r0 + u.t * 2 * j.TQ + token) * j.o.row + q * (D / 8));
#pragma unroll
  for (int k = 0; k < D / 16; ++k) dst[k] = pack_bf16(o[2 * k] * inv, o[2 * k + 1] * inv);
  }
}

template <int D, bool E4M3>
cudaError_t launch_d(const Maps& maps, const Job& job, const CUtensorMap& mq, int ctas, cudaStream_t st) {
  using L = Lay<D, E4M3>;
  cudaError_t e = launch_kernel(cache_attend_tc<D, E4M3>, dim3(ctas), L::THREADS, L::BYTES, 1, false, st, mq, maps.k,
                                maps.v, job);
  if (e == cudaSuccess && job.cut)
    e = launch_kernel(cache_merge<D>, dim3(ctas, 256 / MG_ROWS), 256, 0, 1, true, st, job);
  return e;
}

template <int D, bool E4M3>
cudaError_t set_limit() {
  return taken(cudaFuncSetAttribute(cache_attend_tc<D, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)Lay<D, E4M3>::BYTES));
}

}  // namespace

cudaError_t attend_tc_set_smem_limits() {
  cudaError_t e = set_limit<128, false>();
  if (e == cudaSuccess) e = set_limit<128, true>();
  if (e == cudaSuccess) e = set_limit<64, false>();
  if (e == cudaSuccess) e = set_limit<64, true>();
  return e;
}

bool make_tc_maps(const Pool& c, Maps* m) {
  const int es = c.e4m3 ? 1 : 2;
  const int64_t dim[4] = {c.d, c.page_len, c.H, c.n_pages};
  const int64_t stride[3] = {(int64_t)c.d * es, (int64_t)c.page_len * c.d * es, (int64_t)c.H * c.page_len * c.d * es};
  const int box[4] = {c.e4m3 ? c.d : 64, std::min(c.page_len, BK), 1, 1};
  const int swizzle = !c.e4m3 || c.d == 128 ? 128 : 0;   // (see widen_tile)
  return make_map_4d(&m->k, c.k, es, dim, stride, box, swizzle) && make_map_4d(&m->v, c.v, es, dim, stride, box, swizzle);
}

size_t attend_tc_scratch(const Pool& c) {
  return 256 + sizeof(int) * (size_t)MAX_ITEMS + sizeof(float) * (size_t)MAX_PARTS * 256 * (c.d + 1);
}

cudaError_t launch_attend_tc(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                             int max_rows, const Mask& m, void* scratch, cudaStream_t st) {
  const int G = Hq / c.H, TQ = BQ / G, n_sm = std::min(sm_count(), MAX_CTAS);
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  // items are counted in CHUNK_COUNT_BITS bits (only outputs whose rows overlap could make more: 2.3e9 rows of 64 fill the
  // memory, a unit has 130 rows or more but for a sequence's last, and there are 4,096 x 4,096 of those)
  if ((int64_t)c.H * (s.rows / (2 * TQ) + s.n) >= (1ll << CHUNK_COUNT_BITS) - 4096) return cudaErrorInvalidValue;
  CUtensorMap mq;
  const int64_t dim[4] = {c.d, G, s.rows, c.H};
  const int64_t head = q.head ? q.head : c.d, row = q.row ? q.row : c.d;   // (one head or row: any stride)
  const int64_t stride[3] = {head * 2, row * 2, G * head * 2};
  const int box[4] = {64, G, TQ, 1};
  if (!make_map_4d(&mq, q.p, 2, dim, stride, box, 128)) return cudaErrorInvalidValue;
  // numbers the calls, so that what another call left in the same memory is not taken for a count of this one's (a
  // captured call keeps its number: its replays, one after the other, each find the counts cleared by the one before)
  static std::atomic<uint64_t> calls{0};
  char* const at = static_cast<char*>(scratch);
  // (several sequences make more units than one with all their rows)
  const bool cut = (int64_t)c.H * ((s.rows + 2 * TQ - 1) / (2 * TQ)) < CUT_ROUNDS * n_sm;
  const Job job{c, s, m, o, G, TQ, max_rows, cut ? 1 : 0,
                (uintptr_t)o.p % 32 == 0 && o.head % 16 == 0 && o.row % 16 == 0, chunk_number(calls.fetch_add(1)), reinterpret_cast<unsigned long long*>(at),
                reinterpret_cast<int4*>(at + 64), reinterpret_cast<int*>(at + 256),
                reinterpret_cast<float*>(at + 256 + sizeof(int) * MAX_ITEMS)};
  if (c.d == 128)
    return c.e4m3 ? launch_d<128, true>(maps, job, mq, n_sm, st) : launch_d<128, false>(maps, job, mq, n_sm, st);
  return c.e4m3 ? launch_d<64, true>(maps, job, mq, n_sm, st) : launch_d<64, false>(maps, job, mq, n_sm, st);
}

}  // namespace cache
}  // namespace dkv
