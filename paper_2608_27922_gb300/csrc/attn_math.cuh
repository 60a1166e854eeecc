// Softmax arithmetic on a thread's row of scores, shared by the tensor-core attention kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

namespace dkv {
namespace tc {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// max(a, b, c) in one instruction (three-input form, sm_100 and later).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Row maximum accumulation over 32 scores (t: eight partial maxima).
__device__ __forceinline__ void max_acc(float (&t)[8], const float (&v)[32]) {
#pragma unroll
  for (int k = 0; k < 16; ++k) t[k & 7] = max3(t[k & 7], v[2 * k], v[2 * k + 1]);
}

// Scores of the columns at or past `lim` (keys past the end of the range) become -inf:
// they do not raise the maximum and their exponentials are exactly 0.
__device__ __forceinline__ void mask_tail(float (&v)[32], int lim) {
#pragma unroll
  for (int k = 0; k < 32; ++k)
    if (k >= lim) v[k] = -INFINITY;
}

// P = 2^(s sl2 - m) over 64 scores (a: the first 32, b: the next 32) as 32 packed bf16
// pairs; lab accumulates the even and the odd columns.
__device__ __forceinline__ void exp_pack(const float (&a)[32], const float (&b)[32], float sl2, float nm,
                                         float2& lab, uint32_t (&pk)[32]) {
  const float2 sl2x2 = make_float2(sl2, sl2), nmx2 = make_float2(nm, nm);
#pragma unroll
  for (int k = 0; k < 32; ++k) {
    const float s0 = k < 16 ? a[2 * k] : b[2 * k - 32];
    const float s1 = k < 16 ? a[2 * k + 1] : b[2 * k - 31];
    const float2 x = __ffma2_rn(make_float2(s0, s1), sl2x2, nmx2);
    const float2 pp = make_float2(ex2(x.x), ex2(x.y));
    lab = __fadd2_rn(lab, pp);
    pk[k] = pack_bf16(pp.x, pp.y);
  }
}

}  // namespace tc
}  // namespace dkv
