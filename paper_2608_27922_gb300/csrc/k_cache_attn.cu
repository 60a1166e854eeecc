// Attention over the paged cache (include/dkv.h).  Simple form: one warp per query row.
#include "cache_internal.h"

#include <cuda_fp8.h>

namespace dkv {
namespace cache {

namespace {

constexpr int WARPS = 8;

template <int D, bool E4M3>
__device__ __forceinline__ void load_row(const void* pool, const uint8_t* sc, int64_t at, int lane, float (&x)[D / 32]) {
  constexpr int N = D / 32;
  if (E4M3) {
    const float s = scale_of(sc[at]);
    const uint8_t* p = static_cast<const uint8_t*>(pool) + at * D + lane * N;
#pragma unroll
    for (int k = 0; k < N; ++k)
      x[k] = __half2float(__half(__nv_cvt_fp8_to_halfraw(p[k], __NV_E4M3))) * s;
  } else {
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(pool) + at * D + lane * N;
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = __bfloat162float(p[k]);
  }
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(WARPS * 32) cache_attend_simple(Pool c, Seqs s, Packed q, Packed o, int G, int max_rows,
                                                                 Mask m) {
  constexpr int N = D / 32;
  const int row = blockIdx.x * WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31, hq = blockIdx.y, h = hq / G;
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = threadIdx.x; b < s.n; b += WARPS * 32) seq_at(c, s, b);
  if (row >= min(s.row_start[s.n], s.rows) || row < s.row_start[0]) return;
  const int b = seq_of_row(s, row);
  const Seq sq = seq_at(c, s, b);
  const int i = row - sq.r0, p = sq.len - sq.n + i;
  if (i < 0 || i >= sq.n) return;
  if (sq.n > max_rows) fail(c.status, DEV_INCONSISTENT, SITE_CHUNK);
  float qv[N], acc[N], mx = -INFINITY, l = 0.f;
  const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(q.p) + hq * q.head + row * q.row + lane * N;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    qv[k] = __bfloat162float(qp[k]);
    acc[k] = 0.f;
  }
  const int end = p >= 0 ? visible_end(m, p, sq.len) : 0, lo = window_first(m, end);
  for (int j = 0; j < end; ++j) {
    if (j >= m.sinks && j < lo) j = lo;
    const int64_t at = pool_row(c, s, b, h, j);
    if (at < 0) continue;
    float x[N], t = 0.f;
    load_row<D, E4M3>(c.k, c.ks, at, lane, x);
#pragma unroll
    for (int k = 0; k < N; ++k) t = fmaf(x[k], qv[k], t);
#pragma unroll
    for (int w = 16; w; w >>= 1) t += __shfl_xor_sync(0xffffffffu, t, w);
    t *= m.sl2;
    if (t == -INFINITY) continue;
    if (t > mx) {
      const float a = exp2f(mx - t);
      l *= a;
#pragma unroll
      for (int k = 0; k < N; ++k) acc[k] *= a;
      mx = t;
    }
    const float w = exp2f(t - mx);
    l += w;
    load_row<D, E4M3>(c.v, c.vs, at, lane, x);
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] = fmaf(w, x[k], acc[k]);
  }
  __nv_bfloat16* op = static_cast<__nv_bfloat16*>(o.p) + hq * o.head + row * o.row + lane * N;
#pragma unroll
  for (int k = 0; k < N; ++k) op[k] = __float2bfloat16_rn(l != 0.f ? acc[k] / l : 0.f);
}

}  // namespace

size_t attend_scratch(const Pool& c, int, int, int, int) { return attend_tc_scratch(c); }

cudaError_t launch_attend(const Pool& c, const Maps& maps, const Seqs& s, const Packed& q, const Packed& o, int Hq,
                          int max_rows, const Mask& m, void* scratch, cudaStream_t st) {
  if (max_rows * (Hq / c.H) > 16) return launch_attend_tc(c, maps, s, q, o, Hq, max_rows, m, scratch, st);
  const dim3 grid((s.rows + WARPS - 1) / WARPS, Hq);
  auto* f = c.d == 128 ? (c.e4m3 ? cache_attend_simple<128, true> : cache_attend_simple<128, false>)
                       : (c.e4m3 ? cache_attend_simple<64, true> : cache_attend_simple<64, false>);
  return launch_kernel(f, grid, WARPS * 32, 0, 1, false, st, c, s, q, o, Hq / c.H, max_rows, m);
}

}  // namespace cache
}  // namespace dkv
