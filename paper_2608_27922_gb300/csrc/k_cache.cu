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

#include <cuda_fp8.h>

namespace dkv {
namespace cache {

namespace {

constexpr int THREADS = 256;
constexpr int EMIN = -110;   // smallest scale exponent: every code times its scale is a normal bf16 number

struct Vals {
  uint4 a, b;   // 16 bf16
};

__device__ __forceinline__ Vals load16(const __nv_bfloat16* p) {
  const uint4* q = reinterpret_cast<const uint4*>(p);
  return Vals{__ldg(q), __ldg(q + 1)};
}

__device__ __forceinline__ void store_wide(void* p, const Vals& x) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x.a.x), "r"(x.a.y), "r"(x.a.z),
               "r"(x.a.w), "r"(x.b.x), "r"(x.b.y), "r"(x.b.z), "r"(x.b.w)
               : "memory");
}

// Larger of the magnitudes of the bf16 pairs of x, as bits (they order like the magnitudes; an
// infinity is 0x7f80, a NaN above it).
__device__ __forceinline__ uint32_t mag_max(uint32_t m, uint32_t x) {
  return __vmaxu2(m, x & 0x7fff7fffu);
}

__device__ __forceinline__ uint32_t codes4(uint32_t x, uint32_t y, float inv) {
  const float2 p = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&x));
  const float2 q = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&y));
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(p.x * inv, p.y * inv), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(q.x * inv, q.y * inv), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// One row's part: its largest magnitude over the row's LANES threads, the scale byte, the codes.
template <int LANES>
__device__ __forceinline__ void store_e4m3(const Vals& x, uint8_t* codes, uint8_t* scale, int lane, bool on) {
  uint32_t m = 0;
  m = mag_max(m, x.a.x); m = mag_max(m, x.a.y); m = mag_max(m, x.a.z); m = mag_max(m, x.a.w);
  m = mag_max(m, x.b.x); m = mag_max(m, x.b.y); m = mag_max(m, x.b.z); m = mag_max(m, x.b.w);
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
  const uint32_t a = max(m & 0xffffu, m >> 16);
  // a = (1 + f / 128) 2^(E - 127); 448 = 1.75 * 2^8, so the exponent is E - 135, one more above 1.75
  int e = max((int)(a >> 7) - 135 + ((a & 0x7fu) > 0x60u ? 1 : 0), EMIN);
  if (a == 0) e = 0;
  const bool bad = a >= 0x7f80u;
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  uint4 c;
  c.x = codes4(x.a.x, x.a.y, inv);
  c.y = codes4(x.a.z, x.a.w, inv);
  c.z = codes4(x.b.x, x.b.y, inv);
  c.w = codes4(x.b.z, x.b.w, inv);
  if (e == 120) {   // 256 2^120 is more than bf16 holds: 240 2^120
    c.x = __vminu4(c.x & 0x7f7f7f7fu, 0x77777777u) | (c.x & 0x80808080u);
    c.y = __vminu4(c.y & 0x7f7f7f7fu, 0x77777777u) | (c.y & 0x80808080u);
    c.z = __vminu4(c.z & 0x7f7f7f7fu, 0x77777777u) | (c.z & 0x80808080u);
    c.w = __vminu4(c.w & 0x7f7f7f7fu, 0x77777777u) | (c.w & 0x80808080u);
  }
  if (bad) c = make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
  if (!on) return;
  *reinterpret_cast<uint4*>(codes) = c;
  if (lane == 0) *scale = bad ? 255 : (uint8_t)(e + 127);
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
