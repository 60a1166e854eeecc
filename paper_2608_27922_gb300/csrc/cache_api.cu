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
constexpr int kMaxKeep = 1 << 26;
constexpr int kMaxTile = 128;
constexpr int kMaxWidth = 1024;

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

// The same over chosen pages, where the few-row kernel takes 8 rows at a time: 32 tiles over 32 pages of 64 on 8 key heads, few
// rows against tensor cores: 8 rows 50 us against 53 in bf16 and 36 against 80 in e4m3, 16 rows 93 against 54 and 63
// against 81, 32 rows 145 against 55 and 116 against 82.  (Small tiles of 12 rows, d = 64, bf16: 181 against 158.)
bool few_chosen_rows(const cache::Pool& c, int Hq, int tokens) {
  return (int64_t)tokens * (Hq / c.H) <= (c.e4m3 ? 16 : 8);
}

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

// An input and its output: one and the same, or (as far as addresses tell) apart.
dkv_status_t check_pair(const void* in, int64_t in_head, int64_t in_row, void* out, int64_t out_head, int64_t out_row, int heads,
                        int rows, int d, cache::Packed* a, cache::Packed* z) {
  dkv_status_t st = check_packed(in, heads, rows, in_head, in_row, 0, a);
  if (st == DKV_OK) st = check_packed(out, heads, rows, out_head, out_row, d, z);
  if (st == DKV_OK && in == out && (a->head != z->head || a->row != z->row)) st = DKV_ERR_ARG;
  return st;
}

dkv_status_t check_how(const dkv_norm_rope_t* how, int d, const int32_t* coord, cache::RopeHow* out) {
  if (!how || !how->theta || !aligned(how->theta, 4) || !aligned(how->q_weight, 4) || !aligned(how->k_weight, 4)) return DKV_ERR_ARG;
  if (how->norm != 0 && how->norm != 1) return DKV_ERR_ARG;
  if (how->norm && !(how->eps > 0.f && std::isfinite(how->eps))) return DKV_ERR_ARG;
  if (how->layout != DKV_ROPE_INTERLEAVED && how->layout != DKV_ROPE_HALF) return DKV_ERR_ARG;
  if (how->n_axes < 1 || how->n_axes > 4) return DKV_ERR_ARG;
  int64_t sum = 0;
  *out = cache::RopeHow{coord, how->theta, how->q_weight, how->k_weight, how->eps, how->norm, how->layout == DKV_ROPE_HALF,
                        {d / 2, d / 2, d / 2}};
  for (int a = 0; a < how->n_axes; ++a) {
    if (how->axis_pairs[a] < 0) return DKV_ERR_ARG;
    sum += how->axis_pairs[a];
    if (a < 3 && a < how->n_axes - 1) out->pair_end[a] = (int)(sum < d / 2 ? sum : d / 2);
  }
  return sum == d / 2 ? DKV_OK : DKV_ERR_ARG;
}

dkv_status_t check_table(const cache::Pool& c, const dkv_cache_table_t* t, cache::Table* out) {
  if (!t || !t->block_table || !t->seq_len || !aligned(t->block_table, 4) || !aligned(t->seq_len, 4)) return DKV_ERR_ARG;
  if (t->n_seq < 1 || t->n_seq > kMaxSeqs || t->max_pages < 1 || (int64_t)t->max_pages * c.page_len > kMaxPositions)
    return DKV_ERR_SHAPE;
  *out = cache::Table{t->block_table, t->seq_len, t->n_seq, t->max_pages};
  return DKV_OK;
}
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}
bool overlap(const cache::Table& a, const cache::Table& b) {
  const size_t ta = sizeof(int32_t) * (size_t)a.n * a.max_pages, tb = sizeof(int32_t) * (size_t)b.n * b.max_pages;
  const size_t la = sizeof(int32_t) * (size_t)a.n, lb = sizeof(int32_t) * (size_t)b.n;
  return overlap(a.table, ta, b.table, tb) || overlap(a.len, la, b.len, lb) || overlap(a.table, ta, b.len, lb) ||
         overlap(a.len, la, b.table, tb);
}

dkv_status_t check_summaries(const dkv_cache_summaries_t* s) {
  return s && s->code && s->scale && aligned(s->code, 16) ? DKV_OK : DKV_ERR_ARG;
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
  if (cache::attend_tc_set_smem_limits() != cudaSuccess || cache::attend_rows_set_smem_limits() != cudaSuccess ||
      cache::pages_set_smem_limits() != cudaSuccess || cache::choose_set_smem_limits() != cudaSuccess ||
      cache::chosen_tc_set_smem_limits() != cudaSuccess)
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
  return err == DEV_TIMEOUT ? DKV_ERR_TIMEOUT : err == DEV_NO_PAGES ? DKV_ERR_NOMEM : DKV_ERR_DEVICE;
}

// ------------------------------------------------------------------ norm and rotation
dkv_status_t dkv_norm_rope(int32_t d, const dkv_norm_rope_t* how, const int32_t* coord, int32_t rows, int32_t H_q, const void* Q,
                           int64_t q_head, int64_t q_row, void* Qo, int64_t qo_head, int64_t qo_row, int32_t H_k, const void* K,
                           int64_t k_head, int64_t k_row, void* Ko, int64_t ko_head, int64_t ko_row, void* stream) {
  Range range("dkv_norm_rope");
  if (!coord || !aligned(coord, 4)) return DKV_ERR_ARG;
  if ((d != 64 && d != 128) || rows < 1 || rows > kMaxRows) return DKV_ERR_SHAPE;
  if (H_q < 0 || H_q > kMaxHeads || H_k < 0 || H_k > kMaxHeads || H_q + H_k == 0) return DKV_ERR_SHAPE;
  cache::RopeHow r;
  dkv_status_t st = check_how(how, d, coord, &r);
  cache::Packed q{}, qo{}, k{}, ko{};
  if (st == DKV_OK && H_q) st = check_pair(Q, q_head, q_row, Qo, qo_head, qo_row, H_q, rows, d, &q, &qo);
  if (st == DKV_OK && H_k) st = check_pair(K, k_head, k_row, Ko, ko_head, ko_row, H_k, rows, d, &k, &ko);
  if (st != DKV_OK) return st;
  cache::Pool c{};
  c.d = d;
  cache::Seqs s{};
  s.rows = rows;
  return status_of(cache::launch_norm_rope(c, s, true, r, H_q, q, qo, H_k, k, ko, cache::Packed{}, (cudaStream_t)stream));
}

dkv_status_t dkv_cache_write_norm_rope(dkv_cache_t c, const dkv_cache_seqs_t* seqs, const dkv_norm_rope_t* how,
                                       const int32_t* coord, int32_t rows, int32_t H_q, const void* Q, int64_t q_head,
                                       int64_t q_row, void* Qo, int64_t qo_head, int64_t qo_row, const void* K, int64_t k_head,
                                       int64_t k_row, const void* V, int64_t v_head, int64_t v_row, void* stream) {
  Range range("dkv_cache_write_norm_rope");
  if (!c || !aligned(coord, 4)) return DKV_ERR_ARG;
  cache::Seqs s;
  cache::RopeHow r;
  cache::Packed q{}, qo{}, k, v;
  dkv_status_t st = check_seqs(c->pool, seqs, rows, &s);
  if (st == DKV_OK && (H_q < 0 || H_q > kMaxHeads)) st = DKV_ERR_SHAPE;
  if (st == DKV_OK) st = check_how(how, c->pool.d, coord, &r);
  if (st == DKV_OK && !coord && how->n_axes != 1) st = DKV_ERR_ARG;
  if (st == DKV_OK && H_q) st = check_pair(Q, q_head, q_row, Qo, qo_head, qo_row, H_q, rows, c->pool.d, &q, &qo);
  if (st == DKV_OK) st = check_packed(K, c->pool.H, rows, k_head, k_row, 0, &k);
  if (st == DKV_OK) st = check_packed(V, c->pool.H, rows, v_head, v_row, 0, &v);
  if (st != DKV_OK) return st;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_norm_rope(c->pool, s, false, r, H_q, q, qo, c->pool.H, k, cache::Packed{}, v, (cudaStream_t)stream));
}

// ------------------------------------------------------------------ pages
dkv_status_t dkv_cache_fork(dkv_cache_t c, int32_t* refs, const dkv_cache_table_t* from, const int32_t* parent,
                            const dkv_cache_table_t* to, void* stream) {
  Range range("dkv_cache_fork");
  if (!c || !refs || !aligned(refs, 16) || !parent || !aligned(parent, 4)) return DKV_ERR_ARG;
  cache::Table a, z;
  dkv_status_t st = check_table(c->pool, from, &a);
  if (st == DKV_OK) st = check_table(c->pool, to, &z);
  if (st == DKV_OK && overlap(a, z)) st = DKV_ERR_ARG;
  if (st == DKV_OK && z.max_pages < a.max_pages) st = DKV_ERR_SHAPE;
  if (st != DKV_OK) return st;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_fork(c->pool, refs, a, parent, z, (cudaStream_t)stream));
}

size_t dkv_cache_extend_scratch_size(dkv_cache_t c, int32_t n_seq) {
  return !c || n_seq < 1 || n_seq > kMaxSeqs ? 0 : cache::extend_scratch(n_seq);
}

dkv_status_t dkv_cache_extend(dkv_cache_t c, int32_t* refs, const dkv_cache_table_t* seqs, const int32_t* add, void* scratch,
                              size_t scratch_bytes, void* stream) {
  Range range("dkv_cache_extend");
  if (!c || !refs || !aligned(refs, 16) || !add || !aligned(add, 4) || !scratch || !aligned(scratch, 256)) return DKV_ERR_ARG;
  cache::Table s;
  const dkv_status_t st = check_table(c->pool, seqs, &s);
  if (st != DKV_OK) return st;
  if (scratch_bytes < cache::extend_scratch(s.n)) return DKV_ERR_NOMEM;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_extend(c->pool, refs, s, add, scratch, (cudaStream_t)stream));
}

dkv_status_t dkv_cache_release(dkv_cache_t c, int32_t* refs, const dkv_cache_table_t* seqs, const int32_t* first,
                               const int32_t* last, void* stream) {
  Range range("dkv_cache_release");
  if (!c || !refs || !aligned(refs, 16) || !first || !last || !aligned(first, 4) || !aligned(last, 4)) return DKV_ERR_ARG;
  cache::Table s;
  const dkv_status_t st = check_table(c->pool, seqs, &s);
  if (st != DKV_OK) return st;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_release(c->pool, refs, s, first, last, (cudaStream_t)stream));
}

size_t dkv_cache_compact_scratch_size(dkv_cache_t c, int32_t n_seq) {
  return !c || n_seq < 1 || n_seq > kMaxSeqs ? 0 : cache::compact_scratch(n_seq);
}

dkv_status_t dkv_cache_compact(dkv_cache_t c, int32_t* refs, const dkv_cache_table_t* from, const int32_t* keep, int32_t n_keep,
                               const int32_t* keep_start, const dkv_cache_table_t* to, void* scratch, size_t scratch_bytes,
                               void* stream) {
  Range range("dkv_cache_compact");
  if (!c || !refs || !aligned(refs, 16) || !keep_start || !aligned(keep_start, 4) || !scratch || !aligned(scratch, 256))
    return DKV_ERR_ARG;
  if (n_keep < 0 || n_keep > kMaxKeep) return DKV_ERR_SHAPE;
  if (n_keep > 0 && (!keep || !aligned(keep, 4))) return DKV_ERR_ARG;
  cache::Table a, z;
  dkv_status_t st = check_table(c->pool, from, &a);
  if (st == DKV_OK) st = check_table(c->pool, to, &z);
  if (st == DKV_OK && overlap(a, z)) st = DKV_ERR_ARG;
  if (st == DKV_OK && a.n != z.n) st = DKV_ERR_SHAPE;
  if (st != DKV_OK) return st;
  if (scratch_bytes < cache::compact_scratch(a.n)) return DKV_ERR_NOMEM;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_compact(c->pool, refs, a, keep, n_keep, keep_start, z, scratch, (cudaStream_t)stream));
}

// ------------------------------------------------------------------ chosen pages
dkv_status_t dkv_cache_summarise(dkv_cache_t c, const dkv_cache_seqs_t* seqs, const int32_t* first,
                                 const dkv_cache_summaries_t* sum, void* stream) {
  Range range("dkv_cache_summarise");
  if (!c || !aligned(first, 4)) return DKV_ERR_ARG;
  cache::Seqs s;
  dkv_status_t st = check_seqs(c->pool, seqs, kMaxRows, &s);
  if (st == DKV_OK) st = check_summaries(sum);
  if (st != DKV_OK) return st;
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_summarise(c->pool, s, first, sum->code, sum->scale, (cudaStream_t)stream));
}

dkv_status_t dkv_cache_choose(dkv_cache_t c, const dkv_cache_seqs_t* seqs, const dkv_cache_summaries_t* sum, const void* Q,
                              int32_t H_q, int32_t rows, int64_t q_head, int64_t q_row, const dkv_cache_choose_t* how,
                              int32_t* lists, void* stream) {
  Range range("dkv_cache_choose");
  if (!c || !how || !lists || !aligned(lists, 4)) return DKV_ERR_ARG;
  cache::Seqs s;
  cache::Packed q;
  dkv_status_t st = check_seqs(c->pool, seqs, rows, &s);
  if (st == DKV_OK) st = check_summaries(sum);
  if (st != DKV_OK) return st;
  if (H_q < c->pool.H || H_q % c->pool.H || H_q / c->pool.H > kMaxGroup) return DKV_ERR_SHAPE;
  if (how->tile < 1 || how->tile > kMaxTile || how->block < 0 || how->sink_pages < 0 || how->local_pages < 1 || how->top < 0)
    return DKV_ERR_ARG;
  if (how->width < 1 || how->width > kMaxWidth) return DKV_ERR_SHAPE;
  if ((int64_t)how->sink_pages + how->local_pages + (how->tile + c->pool.page_len - 2) / c->pool.page_len + how->top > how->width)
    return DKV_ERR_SHAPE;
  st = check_packed(Q, H_q, rows, q_head, q_row, 0, &q);
  if (st != DKV_OK) return st;
  const cache::Choose ch{how->tile, how->block, how->sink_pages, how->local_pages, how->top, how->width, cache::inverse_of(how->block)};
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  return status_of(cache::launch_choose(c->pool, s, sum->code, sum->scale, q, H_q, ch, lists, (cudaStream_t)stream));
}

dkv_status_t dkv_cache_attend_chosen(dkv_cache_t c, const dkv_cache_seqs_t* seqs, const void* Q, int32_t H_q, int32_t rows,
                                     int64_t q_head, int64_t q_row, void* O, int64_t o_head, int64_t o_row,
                                     const int32_t* lists, const dkv_cache_chosen_t* how, void* stream) {
  Range range("dkv_cache_attend_chosen");
  if (!c || !how || !lists || !aligned(lists, 4)) return DKV_ERR_ARG;
  cache::Seqs s;
  cache::Packed q, o;
  dkv_status_t st = check_seqs(c->pool, seqs, rows, &s);
  if (st != DKV_OK) return st;
  if (H_q < c->pool.H || H_q % c->pool.H || H_q / c->pool.H > kMaxGroup) return DKV_ERR_SHAPE;
  if (how->tile < 1 || how->tile > kMaxTile || how->block < 0 || !std::isfinite(how->scale)) return DKV_ERR_ARG;
  if (how->width < 1 || how->width > kMaxWidth) return DKV_ERR_SHAPE;
  st = check_packed(Q, H_q, rows, q_head, q_row, 8, &q);
  if (st == DKV_OK) st = check_packed(O, H_q, rows, o_head, o_row, c->pool.d, &o);
  if (st != DKV_OK) return st;
  const float scale = how->scale > 0.f ? how->scale : 1.0f / std::sqrt((float)c->pool.d);
  const cache::Mask m{scale * 1.4426950408889634f, 0, 0, how->block, cache::inverse_of(how->block)};
  const cache::Chosen ch{lists, how->tile, how->width, rows / how->tile + s.n, how->tile < rows ? how->tile : rows};
  OnDevice on(c->device);
  if (!on.ok) return DKV_ERR_CUDA;
  c->last = (cudaStream_t)stream;
  if (few_chosen_rows(c->pool, H_q, ch.tokens))
    return status_of(cache::launch_chosen_rows(c->pool, s, q, o, H_q, m, ch, (cudaStream_t)stream));
  return status_of(cache::launch_chosen_tc(c->pool, c->maps, s, q, o, H_q, m, ch, (cudaStream_t)stream));
}

}  // extern "C"
