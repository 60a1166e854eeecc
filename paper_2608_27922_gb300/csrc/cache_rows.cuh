// Rows of the paged cache in a thread's registers: 16 bf16 values each, and their e4m3 codes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace dkv {
namespace cache {

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

// One row's part of LANES threads' 16 values each: its codes, the row's scale byte.
template <int LANES>
__device__ __forceinline__ uint4 codes_e4m3(const Vals& x, uint8_t& scale) {
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
  scale = bad ? 255 : (uint8_t)(e + 127);
  return c;
}

}  // namespace cache
}  // namespace dkv
