// Pages of several sequences (include/dkv.h): dkv_cache_fork, dkv_cache_extend, dkv_cache_release, dkv_cache_compact.
//
// Tables and counts are whole numbers in device memory; the calls change them there, so that a program forks and
// grows its sequences without asking the host (or inside a graph).  Counts go up and down by atomics, whose
// order does not show in the result.  Fresh pages are the lowest free ones in the order of who asks: a cluster of
// PLANNERS CTAs counts the free pages of its parts of refs, sums over the cluster say which free page goes to whom, and
// only then is anything written: a call that finds a fault or too few pages leaves everything as it was.
// A second kernel, launched beside the first, moves the rows: HBM bounds it (each byte read once and written once).
//
// Measured: 48 continuations forked (3.6 us) and grown (plan 8.5, copies 3.7) 14.5 us in a graph; three prompts on pages of
// 256, 40 heads, into 64 continuations 50 us, of which the copies 33 (160 MB, read mostly from L2, where the 61 copies of three pages
// find them); a window of 9,360 positions of two sequences, 40 heads, e4m3, moved together 64 us (look 5, plan 7, rows 49: 6.6 TB/s); half of the
// pages of 48 sequences given back 1.6 us among other launches, of 4,096 sequences of 64 pages 3.6.
#include "cache_internal.h"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace dkv {
namespace cache {

namespace {

constexpr int PLANNERS = 8;       // CTAs that plan a call on a large pool
constexpr int PLAN_THREADS = 512;
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
// (Short loops, not unrolled: these kernels are one CTA that runs its instructions once or twice, and fetching them is much of
// what they cost.)
struct Planner {
  int part[32];
  int base;                // fresh pages of the chunks of sequences before
  int64_t need, counted;   // fresh pages asked for; free pages of this CTA's part
  int fault;               // of this CTA: site, 0 none
  int before[MAX_SEQS];    // fresh pages of the sequences before (where the sum is no more than there are)
  int k0[MAX_SEQS];        // the entry that a sequence's first one is for
  int fresh[MAX_SEQS];     // how many it asks for
  alignas(16) int held[MAX_SEQS];   // extend: the shared page that the sequence's new positions begin on, -1
  int given[MAX_SEQS];     // extend: how many hold that page; then, in the cluster's first CTA, the page that takes its place
};

// Inclusive sum over the block.
__device__ __forceinline__ int block_sum(int x, int* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += a;
  }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  const int y = lane < warp ? part[lane] : 0;
  return x + __reduce_add_sync(0xffffffffu, y);
}

// A thread's run of refs: per pages from p0 on.
__device__ __forceinline__ int free4(const int32_t* refs, int64_t p, int64_t end) {
  if (p + 4 <= end) {
    const int4 x = *reinterpret_cast<const int4*>(refs + p);
    return (x.x == 0) | (x.y == 0) << 1 | (x.z == 0) << 2 | (x.w == 0) << 3;
  }
  int f = 0;
  for (int i = 0; p + i < end; ++i) f |= (refs[p + i] == 0) << i;
  return f;
}
struct Run {
  int64_t p0, p1;
  int free;   // free pages in it
};
__device__ __forceinline__ Run count_free(const Pool& c, const int32_t* refs, int ctas, int rank) {
  const int64_t threads = (int64_t)ctas * PLAN_THREADS, per = ((c.n_pages + threads - 1) / threads + 3) / 4 * 4;
  Run r;
  r.p0 = min(((int64_t)rank * PLAN_THREADS + threadIdx.x) * per, (int64_t)c.n_pages);
  r.p1 = min(r.p0 + per, (int64_t)c.n_pages);
  r.free = 0;
#pragma unroll 4
  for (int64_t p = r.p0; p < r.p1; p += 4) r.free += __popc(free4(refs, p, r.p1));
  return r;
}

// All CTAs of a cluster: what the sequences ask for (k0, fresh) summed up, the free pages likewise, and if all is well each fresh
// page to whom it is due: give(b, k, page).  False: nothing was given.  Every read of what a plan goes by lies
// before the cluster's first barrier here.
template <typename Give>
__device__ __forceinline__ bool give_pages(const Pool& c, int32_t* refs, int n_seq, Planner& m, const Run& run, Give give) {
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), tid = threadIdx.x;
  if (tid == 0) {
    m.base = 0;
    m.need = 0;
  }
#pragma unroll 1
  for (int b0 = 0; b0 < n_seq; b0 += PLAN_THREADS) {
    const int b = b0 + tid, x = b < n_seq ? m.fresh[b] : 0;
    const int incl = block_sum(x, m.part);   // (wraps only where the 64-bit sum below says that there are too few pages)
    if (b < n_seq) m.before[b] = m.base + incl - x;
    const int lo = __reduce_add_sync(0xffffffffu, x & 0xffff), hi = __reduce_add_sync(0xffffffffu, (int)((unsigned)x >> 16));
    if (tid % 32 == 0) atomicAdd(reinterpret_cast<unsigned long long*>(&m.need), ((unsigned long long)hi << 16) + lo);
    __syncthreads();
    if (tid == PLAN_THREADS - 1) m.base += incl;
  }
  const int upto = block_sum(run.free, m.part);
  if (tid == PLAN_THREADS - 1) m.counted = upto;
  int64_t first = upto - run.free, total = 0;
  int fault = 0;
  if (ctas == 1) {
    __syncthreads();
    total = m.counted;
    fault = m.fault;
  } else {
    cluster.sync();
#pragma unroll 1
    for (int r = 0; r < ctas; ++r) {
      const Planner* o = cluster.map_shared_rank(&m, r);
      const int64_t x = o->counted;
      if (r < rank) first += x;
      total += x;
      if (o->fault) fault = o->fault;
    }
    cluster.sync();   // (nobody's shared memory is looked at any more)
  }
  const int64_t need = m.need;
  if (fault || need > total) {
    if (rank == 0 && tid == 0) fail(c.status, fault ? DEV_INCONSISTENT : DEV_NO_PAGES, fault ? fault : SITE_PAGE);
    return false;
  }
  if (run.free == 0) return true;
#pragma unroll 1
  for (int64_t p = run.p0; p < run.p1 && first < need; p += 4) {
#pragma unroll 1
    for (int f = free4(refs, p, run.p1); f && first < need; f &= f - 1, ++first) {
      const int at = (int)p + __ffs(f) - 1;
      int lo = 0, hi = n_seq;   // the last sequence with before <= first: one that asks for some
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (m.before[mid] <= first) lo = mid; else hi = mid;
      }
      refs[at] = 1;
      give(lo, m.k0[lo] + (int)first - m.before[lo], at);
    }
  }
  return true;
}

// One CTA plans for small pools, a cluster for large ones.  48 sequences grown on pools three quarters full, one CTA against a
// cluster: 2,048 pages 4.2 us against 8.2, 8,192 10.3 against 8.2, 131,072 55 against 21; 2,000 sequences on 32,768 pages 64 against 23.
constexpr int ALONE_MOST = 4096;
int planners(const Pool& c) { return c.n_pages <= ALONE_MOST ? 1 : PLANNERS; }

// What the second kernel moves for a sequence.
struct Move {
  int src, dst, rows, pad;
};

// ------------------------------------------------------------------ extend
__global__ void __launch_bounds__(PLAN_THREADS, 1) extend_plan(Pool c, int32_t* refs, Table s, const int32_t* add, Move* moves) {
  extern __shared__ __align__(16) uint8_t raw[];
  Planner& m = *reinterpret_cast<Planner*>(raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), tid = threadIdx.x;
  pdl_trigger();
  const Run run = count_free(c, refs, ctas, rank);
  if (tid == 0) m.fault = 0;
  __syncthreads();
  const int64_t cap = (int64_t)s.max_pages << c.page_log2;
  bool any_long = false, any_shared = false;
#pragma unroll 1
  for (int b = tid; b < (s.n + 3) / 4 * 4; b += PLAN_THREADS) {
    int k0 = 0, fresh = 0, held = -1, count = 0;
    const int len = b < s.n ? s.len[b] : 0, more = b < s.n ? add[b] : 0;
    if (len < 0 || len > cap || more < 0 || (int64_t)len + more > cap) {
      m.fault = SITE_LEN;
    } else if (more) {
      const int32_t* row = s.table + (int64_t)b * s.max_pages;
      k0 = pages_of(c, len);
      fresh = pages_of(c, len + more) - k0;
      if (len & (c.page_len - 1)) {
        const int page = row[k0 - 1];
        if (!in_pool(c, page)) {
          m.fault = SITE_PAGE;
        } else {
          count = refs[page];
          if (count < 1) m.fault = SITE_REFS;
          if (count > 1) held = page;
        }
      }
      // the entries that pages are to go to hold none (the many of a long growth: below)
      for (int k = 0; k < min(fresh, 4); ++k)
        if (row[k0 + k] >= 0) m.fault = SITE_PAGE;
      any_long = any_long || fresh > 4;
    }
    m.k0[b] = k0;
    m.fresh[b] = fresh;
    m.held[b] = held;
    m.given[b] = count;
    any_shared = any_shared || held >= 0;
  }
  any_shared = __syncthreads_or(any_shared);
  if (__syncthreads_or(any_long)) {   // a warp a sequence, the cluster's CTAs taking turns
#pragma unroll 1
    for (int b = rank + ctas * (tid >> 5); b < s.n; b += ctas * (PLAN_THREADS / 32))
      for (int k = m.k0[b] + 4 + (tid & 31); k < m.k0[b] + m.fresh[b]; k += 32)
        if (s.table[(int64_t)b * s.max_pages + k] >= 0) m.fault = SITE_PAGE;
    __syncthreads();
  }
  // A shared page: the last of its sequences keeps it, if nobody else holds it.
  if (any_shared) {
#pragma unroll 1
    for (int b = tid; b < s.n; b += PLAN_THREADS) {
      const int page = m.held[b];
      if (page < 0) continue;
      int holders = 0, last = b;
#pragma unroll 4
      for (int k = 0; k < (s.n + 3) / 4; ++k) {
        const int4 x = reinterpret_cast<const int4*>(m.held)[k];
        holders += (x.x == page) + (x.y == page) + (x.z == page) + (x.w == page);
        last = x.w == page ? 4 * k + 3 : x.z == page ? 4 * k + 2 : x.y == page ? 4 * k + 1 : x.x == page ? 4 * k : last;
      }
      if (holders > m.given[b]) m.fault = SITE_REFS;
      if (holders == m.given[b] && last == b) {
        m.given[b] = 0;   // stays
      } else {
        --m.k0[b];
        ++m.fresh[b];
      }
    }
    __syncthreads();
  }
  int* given = cluster.map_shared_rank(m.given, 0);
  const bool ok = give_pages(c, refs, s.n, m, run, [&](int b, int k, int p) {
    s.table[(int64_t)b * s.max_pages + k] = p;
    if (k == m.k0[b] && m.held[b] >= 0 && m.given[b] != 0) given[b] = ~p;   // (counts are positive)
  });
  if (ctas == 1) __syncthreads();
  else cluster.sync();   // (the first CTA has all pages given)
  if (rank) return;
#pragma unroll 1
  for (int b = tid; b < s.n; b += PLAN_THREADS) {
    int4 v = make_int4(0, 0, 0, 0);
    const int more = add[b];
    if (ok && more > 0) {
      const int len = s.len[b];
      s.len[b] = len + more;
      if (m.given[b] < 0) {
        v = make_int4(m.held[b], ~m.given[b], len & (c.page_len - 1), 0);
        atomicSub(refs + v.x, 1);
      }
    }
    *reinterpret_cast<int4*>(moves + b) = v;
  }
}

// A sequence's shared page into its own: block (head, sequence), keys and values side by side.
__global__ void __launch_bounds__(COPY_THREADS) extend_copy(Pool c, const Move* moves, int n) {
  pdl_wait();
  const int h = blockIdx.x, row16 = c.d * (c.e4m3 ? 1 : 2) / 16;
  for (int b = blockIdx.y; b < n; b += gridDim.y) {
    const int4 v = *reinterpret_cast<const int4*>(moves + b);
    if (v.z == 0) continue;
    const int64_t from = ((int64_t)v.x * c.H + h) << c.page_log2, to = ((int64_t)v.y * c.H + h) << c.page_log2;
    const uint4* ks = static_cast<const uint4*>(c.k) + from * row16;
    const uint4* vs = static_cast<const uint4*>(c.v) + from * row16;
    uint4* kd = static_cast<uint4*>(c.k) + to * row16;
    uint4* vd = static_cast<uint4*>(c.v) + to * row16;
    const int m = v.z * row16;
    for (int i = threadIdx.x; i < m; i += 4 * COPY_THREADS) {
      uint4 x[4], y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k * COPY_THREADS < m) {
          x[k] = __ldcs(ks + i + k * COPY_THREADS);
          y[k] = __ldcs(vs + i + k * COPY_THREADS);
        }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k * COPY_THREADS < m) {
          kd[i + k * COPY_THREADS] = x[k];
          vd[i + k * COPY_THREADS] = y[k];
        }
    }
    if (c.e4m3 && threadIdx.x < v.z) {   // (at most 255 rows)
      c.ks[to + threadIdx.x] = c.ks[from + threadIdx.x];
      c.vs[to + threadIdx.x] = c.vs[from + threadIdx.x];
    }
  }
}

// ------------------------------------------------------------------ compact
// Block (sequence, part): same[b * parts + part] := the first place of the part's (every parts-th group of
// LOOK_THREADS places) whose position moves, or the number of places; minus a site: a fault.
constexpr int LOOK_THREADS = 256, MAX_LOOKS = 32;
__global__ void __launch_bounds__(LOOK_THREADS) compact_look(Pool c, const int32_t* refs, Table from, const int32_t* keep,
                                                             int n_keep, const int32_t* keep_start, Table to, int32_t* same) {
  pdl_trigger();
  const int b = blockIdx.x, part = blockIdx.y, parts = gridDim.y;
  const int len = from.len[b], a = keep_start[b], z = keep_start[b + 1], n = z - a;
  const int32_t* row = from.table + (int64_t)b * from.max_pages;
  int wrong = a < 0 || z < a || z > n_keep || n > ((int64_t)to.max_pages << c.page_log2) || (b == 0 && a != 0) ? SITE_ROWS :
              len < 0 || len > ((int64_t)from.max_pages << c.page_log2) ? SITE_LEN : 0;
  int mine = n;
  if (wrong == 0) {
#pragma unroll 4
    for (int i = part * LOOK_THREADS + threadIdx.x; i < n; i += parts * LOOK_THREADS) {
      const int j = keep[a + i];
      if (j != i) mine = min(mine, i);
      if (j < 0 || j >= len) {
        wrong = SITE_LEN;
      } else if (!in_pool(c, row[j >> c.page_log2])) {
        wrong = SITE_PAGE;
      }
    }
    // the pages that are given up are pages, and held
#pragma unroll 4
    for (int k = part * LOOK_THREADS + threadIdx.x; k < from.max_pages; k += parts * LOOK_THREADS) {
      const int page = row[k];
      if (page >= c.n_pages) wrong = SITE_PAGE;
      else if (page >= 0 && refs[page] < 1) wrong = SITE_REFS;
    }
  }
  __shared__ int best[LOOK_THREADS / 32], site[LOOK_THREADS / 32];
  mine = __reduce_min_sync(0xffffffffu, mine);
  wrong = __reduce_max_sync(0xffffffffu, wrong);
  if (threadIdx.x % 32 == 0) {
    best[threadIdx.x / 32] = mine;
    site[threadIdx.x / 32] = wrong;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int x = 1; x < LOOK_THREADS / 32; ++x) {
      mine = min(mine, best[x]);
      wrong = max(wrong, site[x]);
    }
    same[(int64_t)b * parts + part] = wrong ? -wrong : mine;
  }
}

// kept[b] := leading pages of sequence b that stay; kept[0] = -1: nothing is done.
__global__ void __launch_bounds__(PLAN_THREADS, 1) compact_plan(Pool c, int32_t* refs, Table from, const int32_t* keep_start, Table to,
                                                                const int32_t* same, int parts, int32_t* kept) {
  extern __shared__ __align__(16) uint8_t raw[];
  Planner& m = *reinterpret_cast<Planner*>(raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ctas = cluster.num_blocks();
  const Run run = count_free(c, refs, ctas, rank);   // (the kernel before this one does not change them)
  if (threadIdx.x == 0) m.fault = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
#pragma unroll 1
  for (int b = threadIdx.x; b < from.n; b += PLAN_THREADS) {
    const int n = keep_start[b + 1] - keep_start[b], all = pages_of(c, n);
    int stay = 0x7fffffff;
#pragma unroll 4
    for (int x = 0; x < parts; ++x) stay = min(stay, same[(int64_t)b * parts + x]);
    if (stay < 0) m.fault = -stay;
    m.k0[b] = stay < 0 ? 0 : stay == n ? all : stay >> c.page_log2;
    m.fresh[b] = stay < 0 ? 0 : all - m.k0[b];
  }
  __syncthreads();
  const bool ok = give_pages(c, refs, from.n, m, run, [&](int b, int k, int p) { to.table[(int64_t)b * to.max_pages + k] = p; });
  if (rank == 0)
    for (int b = threadIdx.x; b < from.n; b += PLAN_THREADS) kept[b] = ok ? m.k0[b] : -1;
}

// Block x: rows [x % groups * MOVE_ROWS, ..) of keep, head x / groups; behind those, one block a sequence, the tables and counts (the
// pages that stay, the entries behind the last page, what is given up).
constexpr int MOVE_ROWS = 64;
__global__ void __launch_bounds__(COPY_THREADS) compact_copy(Pool c, int32_t* refs, Table from, const int32_t* keep, int n_keep,
                                                             const int32_t* keep_start, Table to, const int32_t* kept, int groups) {
  pdl_wait();
  if (kept[0] == -1) return;
  if ((int)blockIdx.x >= groups * c.H) {
    const int b = blockIdx.x - groups * c.H, stay = kept[b], n = keep_start[b + 1] - keep_start[b], all = pages_of(c, n);
    for (int k = threadIdx.x; k < max(from.max_pages, to.max_pages); k += COPY_THREADS) {
      const int page = k < from.max_pages ? from.table[(int64_t)b * from.max_pages + k] : -1;
      if (k < stay) {
        to.table[(int64_t)b * to.max_pages + k] = page;
      } else if (page >= 0 && atomicSub(refs + page, 1) <= 0) {   // given up more often than counted
        atomicAdd(refs + page, 1);
        fail(c.status, DEV_INCONSISTENT, SITE_REFS);
      }
      if (k >= all && k < to.max_pages) to.table[(int64_t)b * to.max_pages + k] = -1;
    }
    if (threadIdx.x == 0) to.len[b] = n;
    return;
  }
  __shared__ int64_t src[MOVE_ROWS], dst[MOVE_ROWS];   // rows of the pool for head 0, -1: stays
  const int h = blockIdx.x / groups, i0 = (blockIdx.x - h * groups) * MOVE_ROWS;
  if (threadIdx.x < MOVE_ROWS) {
    const int i = i0 + threadIdx.x;
    int64_t a = -1, z = -1;
    if (i < n_keep && i < keep_start[from.n]) {
      int lo = 0, hi = from.n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (keep_start[mid] <= i) lo = mid; else hi = mid;
      }
      const int pos = i - keep_start[lo];
      if ((pos >> c.page_log2) >= kept[lo]) {
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
  const int64_t head = (int64_t)h << c.page_log2;
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
size_t compact_scratch(int n_seq) { return sizeof(int32_t) * (size_t)n_seq * (MAX_LOOKS + 1); }

cudaError_t launch_fork(const Pool& c, int32_t* refs, const Table& from, const int32_t* parent, const Table& to, cudaStream_t st) {
  return launch_kernel(cache_fork, dim3(from.n + to.n), 256, 0, 1, false, st, c, refs, from, parent, to);
}

cudaError_t launch_release(const Pool& c, int32_t* refs, const Table& s, const int32_t* first, const int32_t* last, cudaStream_t st) {
  return launch_kernel(cache_release, dim3(s.n), 128, 0, 1, false, st, c, refs, s, first, last);
}

cudaError_t launch_extend(const Pool& c, int32_t* refs, const Table& s, const int32_t* add, void* scratch, cudaStream_t st) {
  Move* moves = static_cast<Move*>(scratch);
  const int P = planners(c);
  const cudaError_t e = launch_kernel(extend_plan, dim3(P), PLAN_THREADS, sizeof(Planner), P, false, st, c, refs, s, add, moves);
  if (e != cudaSuccess) return e;
  return launch_kernel(extend_copy, dim3(c.H, std::min(s.n, 1024)), COPY_THREADS, 0, 1, true, st, c, moves, s.n);
}

cudaError_t launch_compact(const Pool& c, int32_t* refs, const Table& from, const int32_t* keep, int n_keep,
                           const int32_t* keep_start, const Table& to, void* scratch, cudaStream_t st) {
  const int n_sm = sm_count(), P = planners(c);
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  int32_t* const kept = static_cast<int32_t*>(scratch);
  int32_t* const same = kept + from.n;
  // parts of a sequence: four blocks an SM in all, and no more than the work is good for
  const int most = std::max(n_keep, from.max_pages) / (4 * LOOK_THREADS) + 1;
  const int parts = std::max(1, std::min({MAX_LOOKS, 4 * n_sm / from.n, most}));
  const int groups = (n_keep + MOVE_ROWS - 1) / MOVE_ROWS;
  if ((int64_t)groups * c.H + from.n > 0x7fffffff) return cudaErrorInvalidValue;   // (more than any memory holds)
  cudaError_t e = launch_kernel(compact_look, dim3(from.n, parts), LOOK_THREADS, 0, 1, false, st, c, refs, from, keep, n_keep,
                                keep_start, to, same);
  if (e == cudaSuccess)
    e = launch_kernel(compact_plan, dim3(P), PLAN_THREADS, sizeof(Planner), P, true, st, c, refs, from, keep_start, to, same, parts, kept);
  if (e == cudaSuccess)
    e = launch_kernel(compact_copy, dim3(groups * c.H + from.n), COPY_THREADS, 0, 1, true, st, c, refs, from, keep, n_keep,
                      keep_start, to, kept, groups);
  return e;
}

}  // namespace cache
}  // namespace dkv
