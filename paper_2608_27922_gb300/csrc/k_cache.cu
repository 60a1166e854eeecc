// The paged cache's write and read (include/dkv.h): packed bf16 rows into pages, as they are or as
// e4m3 codes with a power-of-two scale a row, and back.
//
// Both move each byte once: bound by HBM (a stack's block of 160 heads x 4,680 rows quantised on its
// way in 85 us, 6.8 TB/s, and read back in 88, 6.6; as bf16 read in 114, 6.7).  A thread holds 16 values of a key row
// and of the value row beside it (four 16-byte loads in flight); d / 16 neighbouring threads hold a row, so
// that a row's largest magnitude is two or three shuffles away.  Consecutive rows of a head lie
// side by side in the packed tensor and, inside a page, in the pool.  (Two or four rows a thread read slower: 107
// and 121 us for 101.)
#include "cache_internal.h"
#include "cache_rows.cuh"

namespace dkv {
namespace cache {

namespace {

constexpr int THREADS = 256;

// One row's part into the pool.
template <int LANES>
__device__ __forceinline__ void store_e4m3(const Vals& x, uint8_t* codes, uint8_t* scale, int lane, bool on) {
  uint8_t byte;
  const uint4 c = codes_e4m3<LANES>(x, byte);
  if (!on) return;
  *reinterpret_cast<uint4*>(codes) = c;
  if (lane == 0) *scale = byte;
}

// Every sequence looked at once a call, also those that no row leads to.
__device__ __forceinline__ void check_seqs(const Pool& c, const Seqs& s) {
  for (int b = threadIdx.x; b < s.n; b += THREADS) seq_at(c, s, b);
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(THREADS) cache_write(Pool c, Seqs s, Packed k, Packed v) {
  constexpr int LANES = D / 16;
  const int lane = threadIdx.x % LANES;
  const int row = blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES;
  const int h = blockIdx.y;
  int64_t at = -1;
  if (row < min(s.row_start[s.n], s.rows) && row >= s.row_start[0]) {
    const int b = seq_of_row(s, row);
    const Seq q = seq_at(c, s, b);
    const int i = row - q.r0, pos = q.len - q.n + i;
    if (i >= 0 && i < q.n && pos >= 0) at = pool_row(c, s, b, h, pos);
  }
  if (blockIdx.x == 0 && h == 0) check_seqs(c, s);
  const bool on = at >= 0;
  if (!E4M3 && !on) return;
  Vals xk{}, xv{};
  if (on) {
    xk = load16(static_cast<const __nv_bfloat16*>(k.p) + h * k.head + row * k.row + lane * 16);
    xv = load16(static_cast<const __nv_bfloat16*>(v.p) + h * v.head + row * v.row + lane * 16);
  }
  const int64_t off = at * D + lane * 16;
  if (E4M3) {   // (a row's lanes are all on or all off, and all of a warp's take part in the shuffles)
    store_e4m3<LANES>(xk, static_cast<uint8_t*>(c.k) + off, c.ks + at, lane, on);
    store_e4m3<LANES>(xv, static_cast<uint8_t*>(c.v) + off, c.vs + at, lane, on);
  } else {
    store_wide(static_cast<__nv_bfloat16*>(c.k) + off, xk);   // (pages begin 128-byte aligned)
    store_wide(static_cast<__nv_bfloat16*>(c.v) + off, xv);
  }
}

__device__ __forceinline__ uint2 values4(uint32_t codes, float scale) {
  uint2 o;
  uint32_t* w = &o.x;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const __half2_raw hr = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> (16 * k)), __NV_E4M3);
    const float2 f = __half22float2(__half2(hr));
    const __nv_bfloat162 y = __floats2bfloat162_rn(f.x * scale, f.y * scale);
    w[k] = *reinterpret_cast<const uint32_t*>(&y);
  }
  return o;
}

__device__ __forceinline__ Vals decode16(uint4 c, float scale) {
  const uint2 a = values4(c.x, scale), b = values4(c.y, scale), d = values4(c.z, scale), e = values4(c.w, scale);
  return Vals{make_uint4(a.x, a.y, b.x, b.y), make_uint4(d.x, d.y, e.x, e.y)};
}

// 16 values, in one store where the tensor's rows are 32-byte aligned (a stack's quantised block read in 88 us; in
// two stores of half a sector each 103).
__device__ __forceinline__ void store16(const Packed& t, bool wide, int h, int row, int col, const Vals& x) {
  uint4* p = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(t.p) + h * t.head + row * t.row + col);
  if (wide) {
    store_wide(p, x);
  } else {
    p[0] = x.a;
    p[1] = x.b;
  }
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(THREADS) cache_read(Pool c, Seqs s, const int32_t* first, Packed k, Packed v, bool wide) {
  constexpr int LANES = D / 16;
  const int lane = threadIdx.x % LANES;
  const int row = blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES;
  const int h = blockIdx.y;
  if (blockIdx.x == 0 && h == 0) check_seqs(c, s);
  if (row >= min(s.row_start[s.n], s.rows) || row < s.row_start[0]) return;
  const int b = seq_of_row(s, row);
  const Seq q = seq_at(c, s, b);
  const int i = row - q.r0;
  if (i < 0 || i >= q.n) return;
  const int64_t pos = (int64_t)first[b] + i;
  const int64_t at = pos >= 0 && pos < q.len ? pool_row(c, s, b, h, (int)pos) : -1;
  Vals xk{}, xv{};
  if (at >= 0) {
    const int64_t off = at * D + lane * 16;
    if (E4M3) {
      const uint4 ck = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(c.k) + off));
      const uint4 cv = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(c.v) + off));
      const float sk = scale_of(c.ks[at]), sv = scale_of(c.vs[at]);
      xk = decode16(ck, sk);
      xv = decode16(cv, sv);
    } else {
      xk = load16(static_cast<const __nv_bfloat16*>(c.k) + off);
      xv = load16(static_cast<const __nv_bfloat16*>(c.v) + off);
    }
  }
  store16(k, wide, h, row, lane * 16, xk);
  store16(v, wide, h, row, lane * 16, xv);
}

}  // namespace

cudaError_t launch_write(const Pool& c, const Seqs& s, const Packed& k, const Packed& v, cudaStream_t st) {
  const int per = THREADS / (c.d / 16);
  const dim3 grid((s.rows + per - 1) / per, c.H);
  auto* f = c.d == 128 ? (c.e4m3 ? cache_write<128, true> : cache_write<128, false>)
                       : (c.e4m3 ? cache_write<64, true> : cache_write<64, false>);
  return launch_kernel(f, grid, THREADS, 0, 1, false, st, c, s, k, v);
}

cudaError_t launch_read(const Pool& c, const Seqs& s, const int32_t* first, const Packed& k, const Packed& v,
                        cudaStream_t st) {
  const int per = THREADS / (c.d / 16);
  const dim3 grid((s.rows + per - 1) / per, c.H);
  auto* f = c.d == 128 ? (c.e4m3 ? cache_read<128, true> : cache_read<128, false>)
                       : (c.e4m3 ? cache_read<64, true> : cache_read<64, false>);
  auto even = [](const Packed& t) { return (uintptr_t)t.p % 32 == 0 && t.head % 16 == 0 && t.row % 16 == 0; };
  return launch_kernel(f, grid, THREADS, 0, 1, false, st, c, s, first, k, v, even(k) && even(v));
}

}  // namespace cache
}  // namespace dkv
