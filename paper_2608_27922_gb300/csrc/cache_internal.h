// The paged cache (include/dkv.h): what its host API and kernels share.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dkv_device.cuh"
#include "dkv_internal.h"

namespace dkv {
namespace cache {

// Pages, [n_pages][H][page_len][d] codes (bf16 or e4m3) and [n_pages][H][page_len] scale bytes.
struct Pool {
  void* k;
  void* v;
  uint8_t* ks;
  uint8_t* vs;
  int32_t* status;   // sticky error word, first failing site
  int H, d, page_len, page_log2, n_pages;
  int e4m3;
};

// The sequences of a call (device arrays).
struct Seqs {
  const int32_t* table;
  const int32_t* len;
  const int32_t* row_start;
  int n, max_pages;
  int rows;   // packed rows of the call's tensors
};

// A table that calls change.
struct Table {
  int32_t* table;
  int32_t* len;
  int n, max_pages;
};

// Packed tensors [heads][rows][d].
struct Packed {
  void* p;
  int64_t head, row;   // strides in elements
};

struct Mask {
  float sl2;   // scale * log2(e)
  int window, sinks, block;
  uint64_t inverse;   // ceil(2^64 / block), block >= 2: p / block is the high half of p times it (p < 2^32)
};
inline uint64_t inverse_of(int block) { return block >= 2 ? ~(uint64_t)0 / (uint64_t)block + 1 : 0; }

enum : int { SITE_ROWS = 1, SITE_LEN = 2, SITE_PAGE = 3, SITE_CHUNK = 4, SITE_PART = 5, SITE_REFS = 6, SITE_LIST = 7, SITE_WAIT = 400 };

// Counts in scratch memory that nobody has cleared: a word is the call's number << COUNT_BITS | a count once a block of
// the call has put that there, and whatever else it holds is no count yet.  A call clears its counts or leaves them at 0, so
// that what an earlier call of the same kernel left is taken for no more than that even where the number comes round again;
// what anybody else left must not look like a number at all.  So the upper 16 bits of the few-row kernel's words are 0x7f81 ..
// 0x7fbe and those of the chunks' 0xff81 .. 0xffbe: never the other kernel's, and as the upper half of an fp32, as bf16 or
// as fp16 NaNs that no arithmetic gives (infinities and the usual NaNs, 0x7f80, 0x7fc0, 0x7fff and their negatives, lie
// outside), as integers far from small ones of either sign.  Beside them 38 bits or more have to agree.
constexpr int ROWS_COUNT_BITS = 16;    // CTAs that share a unit
constexpr int CHUNK_COUNT_BITS = 26;   // items of a call, CTAs, partial results
constexpr uint64_t NUMBER_TOPS = 62;
constexpr uint64_t rows_number(uint64_t call) {
  return (0x7f81ull << (48 - ROWS_COUNT_BITS)) + call % (NUMBER_TOPS << (48 - ROWS_COUNT_BITS));
}
constexpr uint64_t chunk_number(uint64_t call) {
  return (0xff81ull << (48 - CHUNK_COUNT_BITS)) + call % (NUMBER_TOPS << (48 - CHUNK_COUNT_BITS));
}

#ifdef __CUDACC__
// (The index arithmetic below also compiles for the host, where a test walks its bounds.)
__host__ __device__ __forceinline__ void fail(int32_t* status, int32_t code, int32_t site) {
#ifdef __CUDA_ARCH__
  if (atomicCAS(status, 0, code) == 0) atomicExch(status + 1, site);
#else
  if (status[0] == 0) {
    status[0] = code;
    status[1] = site;
  }
#endif
}

__host__ __device__ __forceinline__ int clamp(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// One sequence as the call may use it: its rows inside the tensors, its length inside the table.
struct Seq {
  int r0, n, len;
};

__host__ __device__ __forceinline__ Seq seq_at(const Pool& c, const Seqs& s, int b) {
  Seq q;
  const int a = s.row_start[b], z = s.row_start[b + 1], len = s.len[b];
  const int64_t cap = (int64_t)s.max_pages << c.page_log2;
  q.r0 = clamp(a, 0, s.rows);
  q.n = clamp(z, q.r0, s.rows) - q.r0;
  q.len = clamp(len, 0, (int)cap);
  if (a < 0 || z < a || z > s.rows) fail(c.status, DEV_INCONSISTENT, SITE_ROWS);
  if (len < 0 || len > cap) fail(c.status, DEV_INCONSISTENT, SITE_LEN);
  return q;
}

// Tiles of new tokens: the slots of sequence b begin at row_start[b] / tile + b, which ascends by 1 or more.
__host__ __device__ __forceinline__ int slot_at(const Seqs& s, int tile, int b, int start) { return clamp(start, 0, s.rows) / tile + b; }
inline int first_slot(const Seqs& s, int tile, int b) { return slot_at(s, tile, b, s.row_start[b]); }   // (host)

// The search for the sequence whose tiles a slot may be one of, the last b with first_slot(b) <= slot, by 32 lanes that look at
// sequences evenly apart: it is among [lo, lo + n), and step() == 1 is the last round.  (Row starts that do not ascend give some
// sequence.)
struct SlotSearch {
  int lo, n;
  __host__ __device__ __forceinline__ int step() const { return (n + 31) / 32; }
  __host__ __device__ __forceinline__ int at(int lane) const { return lane * step() < n ? lo + lane * step() : lo; }
  __host__ __device__ __forceinline__ bool past(const Seqs& s, int tile, int slot, int lane, int start) const {
    return lane * step() < n && slot_at(s, tile, at(lane), start) <= slot;
  }
  // mask: the lanes that are past; the one whose sequences are left.
  __host__ __device__ __forceinline__ int narrow(uint32_t mask) {
#ifdef __CUDA_ARCH__
    const int ones = __popc(mask);
#else
    const int ones = __builtin_popcount(mask);
#endif
    const int k = ones > 0 ? ones - 1 : 0, every = step();   // (k * every < n, whatever the starts hold)
    lo += k * every;
    n = every < n - k * every ? every : n - k * every;
    return k;
  }
};

// The search lane by lane, on the host.
inline int seq_of_slot(const Seqs& s, int tile, int slot) {
  SlotSearch w{0, s.n};
  for (;;) {
    const bool last = w.step() == 1;
    uint32_t mask = 0;
    for (int lane = 0; lane < 32; ++lane) mask |= (uint32_t)w.past(s, tile, slot, lane, s.row_start[w.at(lane)]) << lane;
    w.narrow(mask);
    if (last) return w.lo;
  }
}

#ifdef __CUDACC__
// By a warp, and the sequence itself as the call may use it (one or two dependent reads instead of one a halving, and the length
// comes with the last).
__device__ __forceinline__ int seq_of_slot_warp(const Pool& c, const Seqs& s, int tile, int slot, Seq& q) {
  const int lane = threadIdx.x & 31;
  SlotSearch w{0, s.n};
  int start = 0, end = 0, len = 0;
  for (;;) {
    const bool last = w.step() == 1;
    const int b = w.at(lane);
    start = __ldg(s.row_start + b);
    if (last) {
      end = __ldg(s.row_start + b + 1);
      len = __ldg(s.len + b);
    }
    const int k = w.narrow(__ballot_sync(0xffffffffu, w.past(s, tile, slot, lane, start)));
    if (last) {
      start = __shfl_sync(0xffffffffu, start, k);
      end = __shfl_sync(0xffffffffu, end, k);
      len = __shfl_sync(0xffffffffu, len, k);
      break;
    }
  }
  const int64_t cap = (int64_t)s.max_pages << c.page_log2;
  q.r0 = clamp(start, 0, s.rows);
  q.n = clamp(end, q.r0, s.rows) - q.r0;
  q.len = clamp(len, 0, (int)cap);
  if (start < 0 || end < start || end > s.rows) fail(c.status, DEV_INCONSISTENT, SITE_ROWS);
  if (len < 0 || len > cap) fail(c.status, DEV_INCONSISTENT, SITE_LEN);
  return w.lo;
}
#endif

// The sequence of a packed row (row < row_start[n]): the last b with row_start[b] <= row.
__host__ __device__ __forceinline__ int seq_of_row(const Seqs& s, int row) {
  int lo = 0, hi = s.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.row_start[mid] <= row) lo = mid; else hi = mid;
  }
  return lo;
}

// Row of position pos (0 <= pos < table's positions) of sequence b and head h in the pool, -1
// where the table names no page of it.
__host__ __device__ __forceinline__ int64_t pool_row(const Pool& c, const Seqs& s, int b, int h, int pos) {
  const int page = s.table[(int64_t)b * s.max_pages + (pos >> c.page_log2)];
  if ((unsigned)page >= (unsigned)c.n_pages) {
    fail(c.status, DEV_INCONSISTENT, SITE_PAGE);
    return -1;
  }
  return (((int64_t)page * c.H + h) << c.page_log2) + (pos & (c.page_len - 1));
}

// 2^(byte - 127); the byte 255 is NaN.  Bytes are at least 17 (e >= -110) in rows that the cache wrote.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return byte == 255u ? __int_as_float(0x7fffffff) : __uint_as_float(byte << 23);
}

// end(p) of include/dkv.h.
__host__ __device__ __forceinline__ int visible_end(const Mask& m, int p, int len) {
  if (m.block == 0) return len;
  if (m.block == 1) return p < len ? p + 1 : len;
#ifdef __CUDA_ARCH__
  const int q = (int)__umul64hi((uint64_t)(uint32_t)p, m.inverse);
#else
  const int q = (int)(((unsigned __int128)(uint32_t)p * m.inverse) >> 64);
#endif
  const int64_t e = ((int64_t)q + 1) * m.block;
  return e < len ? (int)e : len;
}
// First position of the window that ends there (the sinks before it are visible too).
__host__ __device__ __forceinline__ int window_first(const Mask& m, int end) {
  return m.window == 0 || m.window > end ? 0 : end - m.window;
}
#endif

// Boxes of the pages as the two attention kernels load them, made once for a handle.
struct Maps {
  CUtensorMap k, v;     // chunks of tokens: 128 positions a tile
  CUtensorMap rk, rv;   // few rows: a stage
};

cudaError_t launch_write(const Pool& c, const Seqs& s, const Packed& k, const Packed& v, cudaStream_t st);
cudaError_t launch_read(const Pool& c, const Seqs& s, const int32_t* first, const Packed& k, const Packed& v,
                        cudaStream_t st);

// norm and rotation (dkv_norm_rope_t as the kernel takes it)
struct RopeHow {
  const int32_t* coord;   // [axes][rows], or null: positions
  const float* theta;
  const float* q_weight;
  const float* k_weight;
  float eps;
  int norm, half;
  int pair_end[3];   // pairs of the axes up to 0, 1, 2 (d / 2 past the last one)
};
// (dense: of c only d counts, of s only rows; ko takes the keys.  Else the pages take keys and values)
cudaError_t launch_norm_rope(const Pool& c, const Seqs& s, bool dense, const RopeHow& how, int Hq, const Packed& q,
                             const Packed& qo, int Hk, const Packed& k, const Packed& ko, const Packed& v, cudaStream_t st);

// pages
cudaError_t pages_set_smem_limits();   // on the current device
size_t extend_scratch(int n_seq);
size_t compact_scratch(int n_seq);
cudaError_t launch_fork(const Pool& c, int32_t* refs, const Table& from, const int32_t* parent, const Table& to, cudaStream_t st);
cudaError_t launch_release(const Pool& c, int32_t* refs, const Table& s, const int32_t* first, const int32_t* last, cudaStream_t st);
cudaError_t launch_extend(const Pool& c, int32_t* refs, const Table& s, const int32_t* add, void* scratch, cudaStream_t st);
cudaError_t launch_compact(const Pool& c, int32_t* refs, const Table& from, const int32_t* keep, int n_keep,
                           const int32_t* keep_start, const Table& to, void* scratch, cudaStream_t st);

// choice of pages and attention over them
struct Choose {
  int tile, block, sinks, local, top, width;
  uint64_t inverse;   // of the block, as Mask's
};
struct Chosen {
  const int32_t* lists;
  int tile, width, slots;
  int tokens;   // most of a tile in the call
};
cudaError_t choose_set_smem_limits();   // on the current device
cudaError_t launch_summarise(const Pool& c, const Seqs& s, const int32_t* first, int8_t* code, uint8_t* scale, cudaStream_t st);
cudaError_t launch_choose(const Pool& c, const Seqs& s, const int8_t* code, const uint8_t* scale, const Packed& q, int Hq,
                          const Choose& how, int32_t* lists, cudaStream_t st);

cudaError_t chosen_tc_set_smem_limits();   // on the current device
cudaError_t launch_chosen_tc(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                             const Mask& m, const Chosen& how, cudaStream_t st);
cudaError_t launch_chosen_rows(const Pool& c, const Seqs& s, const Packed& q, const Packed& o, int Hq, const Mask& m,
                               const Chosen& how, cudaStream_t st);

// chunks of tokens, on the tensor cores
bool make_tc_maps(const Pool& c, Maps* m);
cudaError_t attend_tc_set_smem_limits();     // on the current device
size_t attend_tc_scratch(const Pool& c);
cudaError_t launch_attend_tc(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                             int max_rows, const Mask& m, void* scratch, cudaStream_t st);
// few query rows a sequence and key head
bool make_rows_maps(const Pool& c, Maps* m);
cudaError_t attend_rows_set_smem_limits();   // on the current device
size_t attend_rows_scratch(const Pool& c, int G, int max_rows);
cudaError_t launch_attend_rows(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                               int max_rows, const Mask& m, void* scratch, cudaStream_t st);

}  // namespace cache
}  // namespace dkv
