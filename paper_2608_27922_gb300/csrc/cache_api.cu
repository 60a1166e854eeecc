// Host implementation of the paged cache's calls (include/dkv.h).
#include "../../include/dkv.h"
#include <nvtx3/nvToolsExt.h>
#include "cache_internal.h"

#include <atomic>
#include <cmath>
#include <new>

using namespace dkv;

struct dkv_cache_s {
  cache::Pool pool{};
  cache::Maps maps{};
  int device = 0;
  std::atomic<cudaStream_t> last{nullptr};   // (calls may come from several threads)
};

namespace {

constexpr int kMaxHeads = 4096;
constexpr int kMaxSeqs = 4096;
constexpr int kMaxRows = 1 << 20;
constexpr int kMaxGroup = 128;
constexpr int64_t kMaxPositions = 1 << 30;

struct Range {
  explicit Range(const char* name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
};

// The handle's device is the current one for the length of a call.
struct OnDevice {
  int back = -1;
  bool ok = false;
  explicit OnDevice(int device) {
    int cur = 0;
    if (taken(cudaGetDevice(&cur)) != cudaSuccess) return;
    if (cur != device) {
      if (taken(cudaSetDevice(device)) != cudaSuccess) return;
      back = cur;
    }
    ok = true;
  }
  ~OnDevice() {
    if (back >= 0) taken(cudaSetDevice(back));
  }
};

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Which attention kernel: the one for few rows where a sequence's tokens and the heads that share a key head make
// no more than ROWS_MOST, the most rows that read a key once there (16 rows a unit).  32 sequences of 5,000
// positions, 8 key heads, few rows against tensor cores: with 16 rows 125 us against 126 in bf16 and 88 against 156 in
// e4m3, with 25 or 32 rows 225 against 127 and 157 against 158 (the keys are read twice); a single such sequence 27
// to 30 us either way.
constexpr int ROWS_MOST = 16;
bool few_rows(const cache::Pool& c, int Hq, int max_rows) { return (int64_t)max_rows * (Hq / c.H) <= ROWS_MOST; }

size_t scratch_of(const cache::Pool& c, int Hq, int max_rows) {
  return few_rows(c, Hq, max_rows) ? cache::attend_rows_scratch(c, Hq / c.H, max_rows) : cache::attend_tc_scratch(c);
}

dkv_status_t status_of(cudaError_t e) { return e == cudaSuccess ? DKV_OK : DKV_ERR_CUDA; }

dkv_status_t check_seqs(const cache::Pool& c, const dkv_cache_seqs_t* s, int32_t rows, cache::Seqs* out) {
  if (!s || !s->block_table || !s->seq_len || !s->row_start) return DKV_ERR_ARG;
  if (!aligned(s->block_table, 4) || !aligned(s->seq_len, 4) || !aligned(s->row_start, 4)) return DKV_ERR_ARG;
  if (s->n_seq < 1 || s->n_seq > kMaxSeqs || s->max_pages < 1 || rows < 1 || rows > kMaxRows) return DKV_ERR_SHAPE;
  if ((int64_t)s->max_pages * c.page_len > kMaxPositions) return DKV_ERR_SHAPE;
  *out = cache::Seqs{s->block_table, s->seq_len, s->row_start, s->n_seq, s->max_pages, rows};
  return DKV_OK;
}

// A packed tensor's address and strides, the least of which is `least`; a stride between one row or head says nothing.
// Inputs of the write may be broadcast (0), queries come by TMA, whose strides are not 0, and the rows of outputs lie apart.
dkv_status_t check_packed(const void* p, int heads, int rows, int64_t head, int64_t row, int64_t least, cache::Packed* out) {
  if (!p || !aligned(p, 16)) return DKV_ERR_ARG;
  if (heads == 1) head = 0;
  if (rows == 1) row = 0;
  if (head < 0 || row < 0 || head % 8 || row % 8) return DKV_ERR_ARG;
  if ((heads > 1 && head < least) || (rows > 1 && row < least)) return DKV_ERR_ARG;
  *out = cache::Packed{const_cast<void*>(p), head, row};
  return DKV_OK;
}

}  // namespace

extern "C" {

dkv_status_t dkv_cache_create(dkv_cache_t* out, int32_t H, int32_t d, int32_t page_len, int32_t n_pages,
                              int32_t format, const dkv_cache_buffers_t* buf) {
  if (!out || !buf) return DKV_ERR_ARG;
  *out = nullptr;
  if (format != DKV_CACHE_BF16 && format != DKV_CACHE_E4M3) return DKV_ERR_ARG;
  if (H < 1 || H > kMaxHeads || (d != 64 && d != 128) || n_pages < 1 || n_pages > (1 << 30)) return DKV_ERR_SHAPE;
  if (page_len != 16 && page_len != 32 && page_len != 64 && page_len != 128 && page_len != 256) return DKV_ERR_SHAPE;
  if (!buf->k || !buf->v || !buf->status || !aligned(buf->k, 128) || !aligned(buf->v, 128) || !aligned(buf->status, 8))
    return DKV_ERR_ARG;
  const bool e4m3 = format == DKV_CACHE_E4M3;
  if (e4m3 && (!buf->k_scale || !buf->v_scale || !aligned(buf->k_scale, 16) || !aligned(buf->v_scale, 16)))
    return DKV_ERR_ARG;
  int dev = 0;
  cudaDeviceProp prop;
  if (taken(cudaGetDevice(&dev)) != cudaSuccess) return DKV_ERR_CUDA;
  if (taken(cudaGetDeviceProperties(&prop, dev)) != cudaSuccess) return DKV_ERR_CUDA;
  if (prop.major != 10 || prop.minor != 3) return DKV_ERR_UNSUPPORTED;   // built for sm_103a only
  if (cache::attend_tc_set_smem_limits() != cudaSuccess || cache::attend_rows_set_smem_limits() != cudaSuccess)
    return DKV_ERR_CUDA;
  if (taken(cudaMemset(buf->status, 0, 2 * sizeof(int32_t))) != cudaSuccess) return DKV_ERR_CUDA;
  dkv_cache_s* c = new (std::nothrow) dkv_cache_s();
  if (!c) return DKV_ERR_ARG;
  int log2 = 4;
  while ((1 << log2) < page_len) ++log2;
  c->pool = cache::Pool{buf->k, buf->v, e4m3 ? buf->k_scale : nullptr, e4m3 ? buf->v_scale : nullptr, buf->status,
                        H, d, page_len, log2, n_pages, e4m3 ? 1 : 0};
  c->device = dev;
  if (!cache::make_tc_maps(c->pool, &c->maps) || !cache::make_rows_maps(c->pool, &c->maps)) {
    delete c;
    return DKV_ERR_CUDA;
  }
  *out = c;
  return DKV_OK;
}

void dkv_cache_destroy(dkv_cache_t c) { delete c; }

dkv_status_t dkv_cache_write(dkv_cache_t c, const dkv_cache_seqs_t* seqs, const void* K, const void* V, int32_t rows,
                             int64_t k_head, int64_t k_row, int64_t v_head, int64_t v_row, void* stream) {
  Range range("dkv_cache_write");
  if (!c) return DKV_ERR_ARG;
  cache::Seqs s;
  cache::Packed k, v;
  dkv_status_t st = check_seqs(c->pool, seqs, rows, &s);
  if (st == DKV_OK) st = check_packed(K, c->pool.H, rows, k_head, k_row, 0, &k);
  if (st == DKV_OK) st = check_packed(V, c->pool.H, rows, v_head, v_row, 0, &v);
  if (st != DKV_OK) return st;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_write(c->pool, s, k, v, (cudaStream_t)stream));
}

dkv_status_t dkv_cache_read(dkv_cache_t c, const dkv_cache_seqs_t* seqs, const int32_t* first, void* K, void* V,
                            int32_t rows, int64_t k_head, int64_t k_row, int64_t v_head, int64_t v_row, void* stream) {
  Range range("dkv_cache_read");
  if (!c || !first || !aligned(first, 4)) return DKV_ERR_ARG;
  cache::Seqs s;
  cache::Packed k, v;
  dkv_status_t st = check_seqs(c->pool, seqs, rows, &s);
  if (st == DKV_OK) st = check_packed(K, c->pool.H, rows, k_head, k_row, c->pool.d, &k);
  if (st == DKV_OK) st = check_packed(V, c->pool.H, rows, v_head, v_row, c->pool.d, &v);
  if (st != DKV_OK) return st;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_read(c->pool, s, first, k, v, (cudaStream_t)stream));
}

size_t dkv_cache_attend_scratch_size(dkv_cache_t c, int32_t n_seq, int32_t H_q, int32_t rows, int32_t max_rows) {
  if (!c || n_seq < 1 || n_seq > kMaxSeqs || rows < 1 || rows > kMaxRows || max_rows < 1) return 0;
  if (H_q < c->pool.H || H_q % c->pool.H || H_q / c->pool.H > kMaxGroup) return 0;
  return scratch_of(c->pool, H_q, max_rows < rows ? max_rows : rows);
}

dkv_status_t dkv_cache_attend(dkv_cache_t c, const dkv_cache_seqs_t* seqs, const void* Q, int32_t H_q, int32_t rows,
                              int64_t q_head, int64_t q_row, void* O, int64_t o_head, int64_t o_row,
                              const dkv_cache_attend_t* how, void* scratch, size_t scratch_bytes, void* stream) {
  Range range("dkv_cache_attend");
  if (!c || !how || !scratch || !aligned(scratch, 256)) return DKV_ERR_ARG;
  cache::Seqs s;
  cache::Packed q, o;
  dkv_status_t st = check_seqs(c->pool, seqs, rows, &s);
  if (st != DKV_OK) return st;
  if (H_q < c->pool.H || H_q % c->pool.H || H_q / c->pool.H > kMaxGroup) return DKV_ERR_SHAPE;
  if (how->window < 0 || how->sinks < 0 || how->block < 0 || how->max_rows < 1 || !std::isfinite(how->scale))
    return DKV_ERR_ARG;
  st = check_packed(Q, H_q, rows, q_head, q_row, 8, &q);
  if (st == DKV_OK) st = check_packed(O, H_q, rows, o_head, o_row, c->pool.d, &o);
  if (st != DKV_OK) return st;
  const int max_rows = how->max_rows < rows ? how->max_rows : rows;
  if (scratch_bytes < scratch_of(c->pool, H_q, max_rows)) return DKV_ERR_NOMEM;
  const float scale = how->scale > 0.f ? how->scale : 1.0f / std::sqrt((float)c->pool.d);
  const cache::Mask m{scale * 1.4426950408889634f, how->window, how->sinks, how->block, cache::inverse_of(how->block)};
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  auto* launch = few_rows(c->pool, H_q, max_rows) ? cache::launch_attend_rows : cache::launch_attend_tc;
  return status_of(launch(c->pool, c->maps, s, q, o, H_q, max_rows, m, scratch, (cudaStream_t)stream));
}

dkv_status_t dkv_cache_sync(dkv_cache_t c) {
  if (!c) return DKV_ERR_ARG;
  OnDevice on(c->device);
  if (!on.ok || taken(cudaStreamSynchronize(c->last.load())) != cudaSuccess) return DKV_ERR_CUDA;
  int32_t err = 0;
  if (taken(cudaMemcpy(&err, c->pool.status, sizeof(err), cudaMemcpyDeviceToHost)) != cudaSuccess) return DKV_ERR_CUDA;
  if (err == 0) return DKV_OK;
  if (taken(cudaMemset(c->pool.status, 0, 2 * sizeof(int32_t))) != cudaSuccess) return DKV_ERR_CUDA;
  return err == DEV_TIMEOUT ? DKV_ERR_TIMEOUT : DKV_ERR_DEVICE;
}

}  // extern "C"
