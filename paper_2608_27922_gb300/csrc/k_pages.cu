// Pages of several sequences (include/dkv.h): dkv_cache_fork, dkv_cache_extend, dkv_cache_release, dkv_cache_compact.
//
// Tables and counts are whole numbers in device memory; the calls change them there, so that a program forks and
// grows its sequences without asking the host (or inside a graph).  Counts go up and down by atomics, whose
// order does not show in the result.  Fresh pages are the lowest free ones in the order of who asks: a cluster of
// PLANNERS CTAs counts the free pages of its parts of refs, sums over the cluster say which free page goes to whom, and
// only then is anything written: a call that finds a fault or too few pages leaves everything as it was.
// A second kernel, launched beside the first, moves the rows: HBM bounds it (each byte read once and written once).
#include "cache_internal.h"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace dkv {
namespace cache {

namespace {

constexpr int PLANNERS = 8;       // CTAs of a cluster that plan a call
constexpr int PLAN_THREADS = 1024;
constexpr int MAX_SEQS = 4096;
constexpr int COPY_THREADS = 256;

__device__ __forceinline__ int pages_of(const Pool& c, int len) { return (len + c.page_len - 1) >> c.page_log2; }
__device__ __forceinline__ bool in_pool(const Pool& c, int page) { return (unsigned)page < (unsigned)c.n_pages; }

// ------------------------------------------------------------------ fork
// Blocks 0 .. from.n - 1: the counts of a parent's pages; then a block for each child's row of the table.
__global__ void __launch_bounds__(256) cache_fork(Pool c, int32_t* refs, Table from, const int32_t* parent, Table to) {
  const int b = blockIdx.x;
  const int64_t cap = (int64_t)from.max_pages << c.page_log2;
  if (b < from.n) {
    __shared__ int children;
    if (threadIdx.x == 0) children = 0;
    __syncthreads();
    int mine = 0;
    for (int i = threadIdx.x; i < to.n; i += 256) mine += parent[i] == b;
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (threadIdx.x % 32 == 0 && mine) atomicAdd(&children, mine);
    __syncthreads();
    const int change = children - 1;
    for (int k = threadIdx.x; k < from.max_pages; k += 256) {
      const int page = from.table[(int64_t)b * from.max_pages + k];
      if (page < 0) continue;
      if (!in_pool(c, page)) {
        fail(c.status, DEV_INCONSISTENT, SITE_PAGE);
      } else if (change && atomicAdd(refs + page, change) <= 0) {   // held, and counted as free
        atomicSub(refs + page, change);
        fail(c.status, DEV_INCONSISTENT, SITE_REFS);
      }
    }
    return;
  }
  const int i = b - from.n, p = parent[i];
  const bool on = p >= 0 && p < from.n;
  int len = on ? from.len[p] : 0;
  if (threadIdx.x == 0) {
    if (p < -1 || p >= from.n) fail(c.status, DEV_INCONSISTENT, SITE_ROWS);
    if (len < 0 || len > cap) fail(c.status, DEV_INCONSISTENT, SITE_LEN);
    to.len[i] = len < 0 || len > cap ? 0 : len;
  }
  for (int k = threadIdx.x; k < to.max_pages; k += 256) {
    int page = on && k < from.max_pages ? from.table[(int64_t)p * from.max_pages + k] : -1;
    if (!in_pool(c, page)) page = -1;
    to.table[(int64_t)i * to.max_pages + k] = page;
  }
}

// ------------------------------------------------------------------ release
__global__ void __launch_bounds__(128) cache_release(Pool c, int32_t* refs, Table s, const int32_t* first, const int32_t* last) {
  const int b = blockIdx.x, len = s.len[b], lo = max(first[b], 0), hi = last[b];
  if (len < 0 || len > ((int64_t)s.max_pages << c.page_log2)) {
    if (threadIdx.x == 0) fail(c.status, DEV_INCONSISTENT, SITE_LEN);
    return;
  }
  if (hi <= lo || lo >= len) return;
  for (int k = threadIdx.x; k < s.max_pages; k += 128) {
    const int64_t a = (int64_t)k << c.page_log2, z = min((int64_t)len, a + c.page_len);
    if (a < lo || a >= len || z > hi) continue;
    int32_t* at = s.table + (int64_t)b * s.max_pages + k;
    const int page = *at;
    if (page < 0) continue;   // (given back before)
    if (!in_pool(c, page)) {
      fail(c.status, DEV_INCONSISTENT, SITE_PAGE);
      continue;
    }
    if (atomicSub(refs + page, 1) <= 0) {
      atomicAdd(refs + page, 1);
      fail(c.status, DEV_INCONSISTENT, SITE_REFS);
      continue;
    }
    *at = -1;
  }
  __syncthreads();   // (every thread has read the length)
  if (threadIdx.x == 0 && hi >= len) s.len[b] = lo;
}

// ------------------------------------------------------------------ fresh pages
// What a sequence asks for in a plan: `fresh` pages for the entries k0, k0 + 1, ..
struct Ask {
  int k0, fresh;
};

// Inclusive sum over the block; every thread gets its own.  `part`: 32 numbers of shared memory.
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int64_t y = lane < PLAN_THREADS / 32 ? part[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t z = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) y += z;
    }
    part[lane] = y;
  }
  __syncthreads();
  return warp ? x + part[warp - 1] : x;
}

struct Planner {
  int64_t part[32];
  int64_t before[MAX_SEQS + 1];   // fresh pages of the sequences before
  int k0[MAX_SEQS];
  alignas(16) int held[MAX_SEQS]; // extend: the shared page that the sequence's new positions begin on, -1; compact: pages kept
  long long counted;              // free pages of this CTA's part
  int fault;                      // of this CTA: site, 0 none
};

// One CTA of a cluster: sums of what the sequences ask for (thread t has those of sequences 4 t .. 4 t + 3 in ask), the
// free pages counted, and if all is well each of them to whom it is due: give(b, k, page).  False: nothing was given.
template <typename Give>
__device__ __forceinline__ bool give_pages(const Pool& c, int32_t* refs, Planner& m, const Ask (&ask)[4], Give give) {
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank();
  int64_t mine = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) mine += ask[i].fresh;
  const int64_t incl = block_sum(mine, m.part);
  int64_t at = incl - mine;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = threadIdx.x * 4 + i;
    m.before[b] = at;
    m.k0[b] = ask[i].k0;
    at += ask[i].fresh;
  }
  if (threadIdx.x == PLAN_THREADS - 1) m.before[MAX_SEQS] = incl;
  // this CTA's part of refs
  const int per = ((c.n_pages + PLANNERS - 1) / PLANNERS + 3) / 4 * 4;
  const int64_t p0 = min((int64_t)rank * per, (int64_t)c.n_pages), p1 = min(p0 + per, (int64_t)c.n_pages);
  // a thread looks at 4 pages a round, its neighbours at the next ones
  auto free4 = [&](int64_t p) -> int {
    if (p + 4 <= p1) {
      const int4 x = *reinterpret_cast<const int4*>(refs + p);
      return (x.x == 0) | (x.y == 0) << 1 | (x.z == 0) << 2 | (x.w == 0) << 3;
    }
    int f = 0;
    for (int i = 0; p + i < p1; ++i) f |= (refs[p + i] == 0) << i;
    return f;
  };
  int64_t free_pages = 0;
  for (int64_t p = p0 + threadIdx.x * 4; p < p1; p += PLAN_THREADS * 4) free_pages += __popc(free4(p));
  const int64_t upto = block_sum(free_pages, m.part);
  if (threadIdx.x == PLAN_THREADS - 1) m.counted = upto;
  cluster.sync();   // every CTA has read what the plan goes by, and counted
  int64_t first = 0, total = 0;
  int fault = 0;
  for (int r = 0; r < PLANNERS; ++r) {
    const Planner* o = cluster.map_shared_rank(&m, r);
    if (r < rank) first += o->counted;
    total += o->counted;
    if (o->fault) fault = o->fault;
  }
  cluster.sync();   // (nobody's shared memory is looked at any more)
  const int64_t need = m.before[MAX_SEQS];
  if (fault || need > total) {
    if (rank == 0 && threadIdx.x == 0) {
      if (fault) fail(c.status, DEV_INCONSISTENT, fault);
      else fail(c.status, DEV_NO_PAGES, SITE_PAGE);
    }
    return false;
  }
  for (int64_t base = p0; base < p1 && first < need; base += PLAN_THREADS * 4) {
    const int64_t p = base + threadIdx.x * 4;
    const int f = p < p1 ? free4(p) : 0;
    const int64_t incl4 = block_sum(__popc(f), m.part);
    int64_t rank_of = first + incl4 - __popc(f);
    first += m.part[31];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!((f >> i) & 1)) continue;
      if (rank_of < need) {
        int lo = 0, hi = MAX_SEQS;   // the last sequence with before <= rank_of that asks for any
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (m.before[mid] <= rank_of) lo = mid; else hi = mid;
        }
        refs[p + i] = 1;
        give(lo, m.k0[lo] + (int)(rank_of - m.before[lo]), (int)(p + i));
      }
      ++rank_of;
    }
  }
  return true;
}

// What the second kernel moves for a sequence.
struct Move {
  int src, dst, rows, pad;
};

// ------------------------------------------------------------------ extend
__global__ void __cluster_dims__(PLANNERS, 1, 1) __launch_bounds__(PLAN_THREADS)
    extend_plan(Pool c, int32_t* refs, Table s, const int32_t* add, Move* moves) {
  extern __shared__ __align__(16) uint8_t raw[];
  Planner& m = *reinterpret_cast<Planner*>(raw);
  const int rank = cg::this_cluster().block_rank();
  pdl_trigger();
  if (threadIdx.x == 0) m.fault = 0;
  for (int b = threadIdx.x; b < MAX_SEQS; b += PLAN_THREADS) m.held[b] = -1;
  __syncthreads();
  const int64_t cap = (int64_t)s.max_pages << c.page_log2;
  Ask ask[4];
  int len4[4], add4[4], page4[4], refs4[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = threadIdx.x * 4 + i;
    ask[i] = Ask{0, 0};
    len4[i] = add4[i] = refs4[i] = 0;
    page4[i] = -1;
    if (b >= s.n) continue;
    const int len = s.len[b], more = add[b];
    if (len < 0 || len > cap || more < 0 || (int64_t)len + more > cap) {
      m.fault = SITE_LEN;
      continue;
    }
    if (more == 0) continue;
    len4[i] = len;
    add4[i] = more;
    ask[i] = Ask{pages_of(c, len), pages_of(c, len + more) - pages_of(c, len)};
    if (len & (c.page_len - 1)) {
      const int page = s.table[(int64_t)b * s.max_pages + (len >> c.page_log2)];
      if (!in_pool(c, page)) {
        m.fault = SITE_PAGE;
        continue;
      }
      page4[i] = page;
      refs4[i] = refs[page];
      if (refs4[i] < 1) m.fault = SITE_REFS;
      if (refs4[i] > 1) m.held[b] = page;
    }
  }
  __syncthreads();
  // A shared page: the last of its sequences keeps it, if nobody else holds it.
  int moved4[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    moved4[i] = 0;
    if (refs4[i] <= 1) continue;
    const int b = threadIdx.x * 4 + i, page = page4[i];
    int holders = 0, last = b;
    for (int k = 0; k < (s.n + 3) / 4; ++k) {
      const int4 x = reinterpret_cast<const int4*>(m.held)[k];
      if (x.x == page) ++holders, last = max(last, 4 * k);
      if (x.y == page) ++holders, last = max(last, 4 * k + 1);
      if (x.z == page) ++holders, last = max(last, 4 * k + 2);
      if (x.w == page) ++holders, last = max(last, 4 * k + 3);
    }
    if (holders > refs4[i]) m.fault = SITE_REFS;
    if (holders == refs4[i] && last == b) continue;
    moved4[i] = 1;
    ask[i].k0 -= 1;
    ask[i].fresh += 1;
  }
  // the entries that pages are to go to hold none (a warp a sequence, the cluster's CTAs taking turns)
  for (int b = rank + PLANNERS * (threadIdx.x >> 5); b < s.n; b += PLANNERS * (PLAN_THREADS / 32)) {
    const int len = s.len[b], more = add[b];
    if (len < 0 || more <= 0 || (int64_t)len + more > cap) continue;
    for (int k = pages_of(c, len) + (threadIdx.x & 31); k < pages_of(c, len + more); k += 32)
      if (s.table[(int64_t)b * s.max_pages + k] >= 0) m.fault = SITE_PAGE;
  }
  __syncthreads();
  const bool ok = give_pages(c, refs, m, ask, [&](int b, int k, int page) { s.table[(int64_t)b * s.max_pages + k] = page; });
  cg::this_cluster().sync();   // (the tables are written)
  if (rank) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = threadIdx.x * 4 + i;
    if (b >= s.n) continue;
    Move v{0, 0, 0, 0};
    if (ok && add4[i] > 0) {
      s.len[b] = len4[i] + add4[i];
      if (moved4[i]) {
        v = Move{page4[i], s.table[(int64_t)b * s.max_pages + (len4[i] >> c.page_log2)], len4[i] & (c.page_len - 1), 0};
        atomicSub(refs + page4[i], 1);
      }
    }
    moves[b] = v;
  }
}

// A sequence's shared page into its own: block (parts of a head's rows, head, sequence).
__device__ __forceinline__ void copy_bytes(void* to, const void* from, int bytes, int t, int n) {
  uint4* d = static_cast<uint4*>(to);
  const uint4* s = static_cast<const uint4*>(from);
  const int m = bytes / 16;
  int i = t;
  for (; i + 3 * n < m; i += 4 * n) {
    const uint4 a = __ldcs(s + i), b = __ldcs(s + i + n), x = __ldcs(s + i + 2 * n), y = __ldcs(s + i + 3 * n);
    d[i] = a;
    d[i + n] = b;
    d[i + 2 * n] = x;
    d[i + 3 * n] = y;
  }
  for (; i < m; i += n) d[i] = __ldcs(s + i);
}

__global__ void __launch_bounds__(COPY_THREADS) extend_copy(Pool c, const Move* moves, int n) {
  pdl_wait();
  const int h = blockIdx.x;
  const int row = c.d * (c.e4m3 ? 1 : 2);
  for (int b = blockIdx.y; b < n; b += gridDim.y) {
    const Move v = moves[b];
    if (v.rows == 0) continue;
    const int64_t from = ((int64_t)v.src * c.H + h) << c.page_log2, to = ((int64_t)v.dst * c.H + h) << c.page_log2;
    copy_bytes(static_cast<char*>(c.k) + to * row, static_cast<char*>(c.k) + from * row, v.rows * row, threadIdx.x, COPY_THREADS);
    copy_bytes(static_cast<char*>(c.v) + to * row, static_cast<char*>(c.v) + from * row, v.rows * row, threadIdx.x, COPY_THREADS);
    if (c.e4m3 && threadIdx.x < v.rows) {   // (at most 255 rows)
      c.ks[to + threadIdx.x] = c.ks[from + threadIdx.x];
      c.vs[to + threadIdx.x] = c.vs[from + threadIdx.x];
    }
  }
}

// ------------------------------------------------------------------ compact
// same[b]: positions from the first on that stay where they are; -1: a fault.  A block a sequence.
__global__ void __launch_bounds__(256) compact_look(Pool c, Table from, const int32_t* keep, int n_keep, const int32_t* keep_start,
                                                    Table to, int32_t* same) {
  pdl_trigger();
  const int b = blockIdx.x, len = from.len[b], a = keep_start[b], z = keep_start[b + 1];
  __shared__ int stay, wrong;
  if (threadIdx.x == 0) {
    stay = z - a;
    wrong = a < 0 || z < a || z > n_keep || z - a > ((int64_t)to.max_pages << c.page_log2) || (b == 0 && a != 0) ? SITE_ROWS :
            len < 0 || len > ((int64_t)from.max_pages << c.page_log2) ? SITE_LEN : 0;
  }
  __syncthreads();
  if (wrong == 0) {
    int mine = z - a, bad = 0;
    for (int i = threadIdx.x; i < z - a; i += 256) {
      const int j = keep[a + i];
      if (j != i) mine = min(mine, i);
      if (j < 0 || j >= len) {
        bad = SITE_LEN;
      } else if (!in_pool(c, from.table[(int64_t)b * from.max_pages + (j >> c.page_log2)])) {
        bad = SITE_PAGE;
      }
    }
    if (mine < z - a) atomicMin(&stay, mine);
    if (bad) wrong = bad;
    // every page that is given up has to be one
    for (int k = threadIdx.x; k < from.max_pages; k += 256)
      if (from.table[(int64_t)b * from.max_pages + k] >= c.n_pages) wrong = SITE_PAGE;
  }
  __syncthreads();
  if (threadIdx.x == 0) same[b] = wrong ? -wrong : stay;
}

__global__ void __cluster_dims__(PLANNERS, 1, 1) __launch_bounds__(PLAN_THREADS)
    compact_plan(Pool c, int32_t* refs, Table from, const int32_t* keep_start, Table to, int32_t* same) {
  extern __shared__ __align__(16) uint8_t raw[];
  Planner& m = *reinterpret_cast<Planner*>(raw);
  const int rank = cg::this_cluster().block_rank();
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x == 0) m.fault = 0;
  __syncthreads();
  Ask ask[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = threadIdx.x * 4 + i;
    ask[i] = Ask{0, 0};
    m.held[b] = 0;
    if (b >= from.n) continue;
    const int stay = same[b];
    if (stay < 0) {
      m.fault = -stay;
      continue;
    }
    const int n = keep_start[b + 1] - keep_start[b], all = pages_of(c, n);
    const int kept = stay == n ? all : stay >> c.page_log2;   // pages that stay
    ask[i] = Ask{kept, all - kept};
    m.held[b] = kept;
  }
  __syncthreads();
  // refs of pages held: none free (a warp a sequence)
  for (int b = rank + PLANNERS * (threadIdx.x >> 5); b < from.n; b += PLANNERS * (PLAN_THREADS / 32))
    for (int k = threadIdx.x & 31; k < from.max_pages; k += 32) {
      const int page = from.table[(int64_t)b * from.max_pages + k];
      if (in_pool(c, page) && refs[page] < 1) m.fault = SITE_REFS;
    }
  __syncthreads();
  const bool ok = give_pages(c, refs, m, ask, [&](int b, int k, int page) { to.table[(int64_t)b * to.max_pages + k] = page; });
  if (!ok) {
    if (rank == 0)
      for (int b = threadIdx.x; b < from.n; b += PLAN_THREADS) same[b] = -1;   // nothing to move
    return;
  }
  cg::this_cluster().sync();   // (nobody counts free pages any more)
  for (int b = rank + PLANNERS * (threadIdx.x >> 5); b < from.n; b += PLANNERS * (PLAN_THREADS / 32)) {
    const int kept = m.held[b], n = keep_start[b + 1] - keep_start[b], all = pages_of(c, n);
    for (int k = threadIdx.x & 31; k < max(from.max_pages, to.max_pages); k += 32) {
      const int page = k < from.max_pages ? from.table[(int64_t)b * from.max_pages + k] : -1;
      if (k < kept) to.table[(int64_t)b * to.max_pages + k] = page;
      else if (page >= 0) atomicSub(refs + page, 1);
      if (k >= all && k < to.max_pages) to.table[(int64_t)b * to.max_pages + k] = -1;
    }
    if ((threadIdx.x & 31) == 0) to.len[b] = n;
  }
}

// Rows [blockIdx.x * ROWS, ..) of keep, head blockIdx.y.
constexpr int MOVE_ROWS = 64;
__global__ void __launch_bounds__(COPY_THREADS) compact_copy(Pool c, Table from, const int32_t* keep, int n_keep,
                                                             const int32_t* keep_start, Table to, const int32_t* same) {
  pdl_wait();
  __shared__ int64_t src[MOVE_ROWS], dst[MOVE_ROWS];   // rows of the pool for head 0, -1: stays
  const int i0 = blockIdx.x * MOVE_ROWS;
  if (threadIdx.x < MOVE_ROWS) {
    const int i = i0 + threadIdx.x;
    int64_t a = -1, z = -1;
    if (same[0] != -1 && i < n_keep && i < keep_start[from.n] && i >= keep_start[0]) {
      int lo = 0, hi = from.n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (keep_start[mid] <= i) lo = mid; else hi = mid;
      }
      const int pos = i - keep_start[lo], n = keep_start[lo + 1] - keep_start[lo], stay = same[lo];
      const int kept = stay == n ? pages_of(c, n) : stay >> c.page_log2;
      if ((pos >> c.page_log2) >= kept) {
        const int j = keep[i];
        a = (((int64_t)from.table[(int64_t)lo * from.max_pages + (j >> c.page_log2)] * c.H) << c.page_log2) + (j & (c.page_len - 1));
        z = (((int64_t)to.table[(int64_t)lo * to.max_pages + (pos >> c.page_log2)] * c.H) << c.page_log2) + (pos & (c.page_len - 1));
      }
    }
    src[threadIdx.x] = a;
    dst[threadIdx.x] = z;
  }
  __syncthreads();
  const int row16 = c.d * (c.e4m3 ? 1 : 2) / 16;   // 4, 8 or 16 threads a row
  const int64_t head = (int64_t)blockIdx.y << c.page_log2;
  const int t = threadIdx.x % row16, per = COPY_THREADS / row16;
  const uint4* k = static_cast<const uint4*>(c.k);
  const uint4* v = static_cast<const uint4*>(c.v);
#pragma unroll 2
  for (int r = threadIdx.x / row16; r < MOVE_ROWS; r += per) {
    if (src[r] < 0) continue;
    const int64_t a = src[r] + head, z = dst[r] + head;
    const uint4 x = __ldcs(k + a * row16 + t), y = __ldcs(v + a * row16 + t);
    static_cast<uint4*>(c.k)[z * row16 + t] = x;
    static_cast<uint4*>(c.v)[z * row16 + t] = y;
  }
  if (c.e4m3 && threadIdx.x < MOVE_ROWS && src[threadIdx.x] >= 0) {
    const int64_t a = src[threadIdx.x] + head, z = dst[threadIdx.x] + head;
    c.ks[z] = c.ks[a];
    c.vs[z] = c.vs[a];
  }
}

}  // namespace

cudaError_t pages_set_smem_limits() {
  cudaError_t e = taken(cudaFuncSetAttribute(extend_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Planner)));
  if (e == cudaSuccess)
    e = taken(cudaFuncSetAttribute(compact_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Planner)));
  return e;
}

size_t extend_scratch(int n_seq) { return sizeof(Move) * (size_t)n_seq; }
size_t compact_scratch(int n_seq) { return sizeof(int32_t) * (size_t)n_seq; }

cudaError_t launch_fork(const Pool& c, int32_t* refs, const Table& from, const int32_t* parent, const Table& to, cudaStream_t st) {
  return launch_kernel(cache_fork, dim3(from.n + to.n), 256, 0, 1, false, st, c, refs, from, parent, to);
}

cudaError_t launch_release(const Pool& c, int32_t* refs, const Table& s, const int32_t* first, const int32_t* last, cudaStream_t st) {
  return launch_kernel(cache_release, dim3(s.n), 128, 0, 1, false, st, c, refs, s, first, last);
}

cudaError_t launch_extend(const Pool& c, int32_t* refs, const Table& s, const int32_t* add, void* scratch, cudaStream_t st) {
  Move* moves = static_cast<Move*>(scratch);
  const cudaError_t e = launch_kernel(extend_plan, dim3(PLANNERS), PLAN_THREADS, sizeof(Planner), 1, false, st, c, refs, s, add, moves);
  if (e != cudaSuccess) return e;
  return launch_kernel(extend_copy, dim3(c.H, std::min(s.n, 1024)), COPY_THREADS, 0, 1, true, st, c, moves, s.n);
}

cudaError_t launch_compact(const Pool& c, int32_t* refs, const Table& from, const int32_t* keep, int n_keep,
                           const int32_t* keep_start, const Table& to, void* scratch, cudaStream_t st) {
  int32_t* same = static_cast<int32_t*>(scratch);
  cudaError_t e = launch_kernel(compact_look, dim3(from.n), 256, 0, 1, false, st, c, from, keep, n_keep, keep_start, to, same);
  if (e == cudaSuccess)
    e = launch_kernel(compact_plan, dim3(PLANNERS), PLAN_THREADS, sizeof(Planner), 1, true, st, c, refs, from, keep_start, to, same);
  if (e == cudaSuccess && n_keep > 0)
    e = launch_kernel(compact_copy, dim3((n_keep + MOVE_ROWS - 1) / MOVE_ROWS, c.H), COPY_THREADS, 0, 1, true, st, c, from, keep,
                      n_keep, keep_start, to, same);
  return e;
}

}  // namespace cache
}  // namespace dkv
