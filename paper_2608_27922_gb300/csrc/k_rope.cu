// Norm and rotation of queries and keys in one pass (include/dkv.h: dkv_norm_rope, dkv_cache_write_norm_rope).
//
// For a row x of d values: y = x w rsqrt(mean x^2 + eps), and each pair of y turned by its token's angle.  Every
// byte moves once, so HBM bounds large calls and the launch small ones.  A row lies with d / 16 neighbouring
// threads, thread l's 16 values being 8 l .. and d / 2 + 8 l ..: both elements of every pair, whichever the layout, and
// 16-byte accesses side by side.
// A thread keeps its token: the angles' sines and cosines are worked out once and serve all the heads that
// it walks over, whose rows come in one head ahead of their use.
//
// The angle c theta in turns, modulo 1: theta / 2 pi as a 64-bit fraction of a turn times the whole number c, modulo
// 2^64, which is exact but for the fraction's own rounding; the upper 32 bits, as a number in [-1, 1) half turns, go to
// sincospi.  The 64-bit fractions are a block's, made once (they need double precision).
//
// Measured: a block of 4,680 tokens, 40 heads of queries and of keys and values, into bf16 pages 55 us (47 us alone under the
// counters: 6.2 TB/s of the 6.8 that a copy reaches), into e4m3 pages 58; a frame of 1,561 tokens, 24 + 8 heads of 64, dense 8.3 us; 32 tokens of
// 40 + 8 heads 6.3 us, of which a launch is 4.
#include "cache_internal.h"
#include "cache_rows.cuh"

#include <algorithm>

namespace dkv {
namespace cache {

namespace {

constexpr int THREADS = 256;
constexpr int BLOCKS = 4;   // of an SM: 64 registers a thread (a block of 40 heads 55 us; with 3 of 80 registers 64)
enum { DENSE = 0, PAGES_BF16 = 1, PAGES_E4M3 = 2 };

struct Tensors {
  Packed q, qo, k, ko, v;
  int Hq, Hk;
  int per;         // heads of a block (queries, keys, then the values of a cache)
  int rows_log2;   // tokens of a block
};

__device__ __forceinline__ float2 pair_of(uint32_t x) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ Vals load_row(const Packed& t, int h, int row, int lane, int d) {
  // (ordinary loads: an output may be its input)
  const uint4* p = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(t.p) + h * t.head + row * t.row);
  return Vals{__ldcs(p + lane), __ldcs(p + d / 16 + lane)};
}

__device__ __forceinline__ void store_row(__nv_bfloat16* p, const Vals& x, int lane, int d) {
  reinterpret_cast<uint4*>(p)[lane] = x.a;
  reinterpret_cast<uint4*>(p)[d / 16 + lane] = x.b;
}

// Of thread l: the rotation pair of its values 2 i and 2 i + 1, and the element that value m is.
template <int D, bool HALF>
__device__ __forceinline__ int pair_index(int l, int i) {
  return HALF ? l * 8 + i : (i >> 2) * (D / 4) + l * 4 + (i & 3);
}
template <int D, bool HALF>
__device__ __forceinline__ int element(int l, int m) {
  return HALF ? (m & 1) * (D / 2) + l * 8 + (m >> 1) : (m >> 3) * (D / 2) + l * 8 + (m & 7);
}

// The 16 values normed (w: four of the thread's weights every D / 16 places, ones where there are none) and rotated.
template <int D, bool HALF>
__device__ __forceinline__ Vals turned(const Vals& x, const float4* w, bool norm, float eps, const float (&cs)[8],
                                       const float (&sn)[8]) {
  constexpr int LANES = D / 16;
  float v[16];   // pair i: v[2 i], v[2 i + 1]
  const uint32_t* xa = &x.a.x;
  const uint32_t* xb = &x.b.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 a = pair_of(xa[k]), b = pair_of(xb[k]);
    if (HALF) {
      v[4 * k] = a.x; v[4 * k + 2] = a.y;
      v[4 * k + 1] = b.x; v[4 * k + 3] = b.y;
    } else {
      v[2 * k] = a.x; v[2 * k + 1] = a.y;
      v[8 + 2 * k] = b.x; v[8 + 2 * k + 1] = b.y;
    }
  }
  if (norm) {
    auto squares = [&](float f) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float y = v[k] * f;
        s = fmaf(y, y, s);
      }
#pragma unroll
      for (int o = 1; o < LANES; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      return s;
    };
    float s = squares(1.0f), r = rsqrtf(fmaf(s, 1.0f / D, eps));
    if (__any_sync(0xffffffffu, !(s < INFINITY))) {   // 128 squares of 2^58 stay below 2^124
      const float z = squares(0x1p-70f);
      if (!(s < INFINITY)) r = z < INFINITY ? rsqrtf(fmaf(z, 1.0f / D, eps * 0x1p-70f * 0x1p-70f)) * 0x1p-70f : __int_as_float(0x7fffffff);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 f = w[k * LANES];
      v[4 * k] *= r * f.x; v[4 * k + 1] *= r * f.y; v[4 * k + 2] *= r * f.z; v[4 * k + 3] *= r * f.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = v[2 * i], b = v[2 * i + 1];
    v[2 * i] = fmaf(a, cs[i], -(b * sn[i]));
    v[2 * i + 1] = fmaf(a, sn[i], b * cs[i]);
  }
  Vals y;
  uint32_t* ya = &y.a.x;
  uint32_t* yb = &y.b.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    ya[k] = HALF ? pack(v[4 * k], v[4 * k + 2]) : pack(v[2 * k], v[2 * k + 1]);
    yb[k] = HALF ? pack(v[4 * k + 1], v[4 * k + 3]) : pack(v[8 + 2 * k], v[8 + 2 * k + 1]);
  }
  return y;
}

template <int D, bool HALF, int MODE>
__global__ void __launch_bounds__(THREADS, BLOCKS) norm_rope(Pool c, Seqs s, const __grid_constant__ RopeHow how,
                                                     const __grid_constant__ Tensors t) {
  constexpr int LANES = D / 16, SLOTS = THREADS / LANES;
  __shared__ int64_t turns[D / 2];
  __shared__ float4 weights[2][D / 4];   // four values of all threads, then the next four (side by side: no bank twice)
  if (threadIdx.x < D / 2) {
    double f = (double)how.theta[threadIdx.x] * 0.15915494309189533577;   // 1 / (2 pi)
    f -= rint(f);
    turns[threadIdx.x] = __double2ll_rn(f * 18446744073709551616.0);
  }
  for (int e = threadIdx.x; e < 2 * D; e += THREADS) {
    const int k = e % D, l = (k >> 2) % LANES, m = (k >> 2) / LANES * 4 + (k & 3);
    const float* w = e < D ? how.q_weight : how.k_weight;
    reinterpret_cast<float*>(weights[e / D])[k] = w ? w[element<D, HALF>(l, m)] : 1.0f;
  }
  if (MODE != DENSE && blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = threadIdx.x; b < s.n; b += THREADS) seq_at(c, s, b);
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const int row = (blockIdx.x << t.rows_log2) + (slot & ((1 << t.rows_log2) - 1));
  bool on = row < s.rows;
  int pos = 0;
  int64_t at = -1;   // of head 0
  if (MODE != DENSE) {
    on = on && row < s.row_start[s.n] && row >= s.row_start[0];
    if (on) {
      const int b = seq_of_row(s, row);
      const Seq q = seq_at(c, s, b);
      const int i = row - q.r0;
      on = i >= 0 && i < q.n;
      pos = q.len - q.n + i;
      if (on && pos >= 0) at = pool_row(c, s, b, 0, pos);
    }
  }
  __syncthreads();
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = pair_index<D, HALF>(lane, i);
    int a = 0;
    for (int k = 0; k < 3; ++k) a += j >= how.pair_end[k];   // (ends past the last axis' are d / 2)
    const int x = !on ? 0 : how.coord ? __ldg(how.coord + (int64_t)a * s.rows + row) : pos;
    const uint64_t turn = (uint64_t)(int64_t)x * (uint64_t)turns[j] + 0x80000000u;
    sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn[i], &cs[i]);
  }
  const int heads = t.Hq + t.Hk + (MODE == DENSE ? 0 : t.Hk), step = SLOTS >> t.rows_log2;
  const int end = min(heads, ((int)blockIdx.y + 1) * t.per);
  int h = blockIdx.y * t.per + (slot >> t.rows_log2);
  auto load = [&](int i) -> Vals {
    if (i < t.Hq) return load_row(t.q, i, row, lane, D);
    if (MODE == DENSE || i < t.Hq + t.Hk) return load_row(t.k, i - t.Hq, row, lane, D);
    return load_row(t.v, i - t.Hq - t.Hk, row, lane, D);
  };
  Vals next{};
  if (on && h < end) next = load(h);
  const int rounds = (t.per + step - 1) / step;   // the same for all threads (shuffles)
#pragma unroll 1
  for (int r = 0; r < rounds; ++r, h += step) {
    Vals x = next;
    const bool mine = on && h < end;
    if (on && h + step < end) next = load(h + step);
    const bool value = MODE != DENSE && h >= t.Hq + t.Hk, query = h < t.Hq;
    if (MODE == DENSE || !__all_sync(0xffffffffu, value)) {
      const Vals y = turned<D, HALF>(x, weights[query ? 0 : 1] + lane, how.norm != 0, how.eps, cs, sn);
      if (!value) x = y;
    }
    if (MODE == DENSE || query) {
      if (mine) {
        const Packed& o = query ? t.qo : t.ko;
        store_row(static_cast<__nv_bfloat16*>(o.p) + (query ? h : h - t.Hq) * o.head + row * o.row, x, lane, D);
      }
      if (MODE != PAGES_E4M3) continue;   // (whole warps stay together for the codes' shuffles)
    }
    if (MODE == DENSE) continue;
    const int hk = value ? h - t.Hq - t.Hk : h - t.Hq;
    const bool keep = mine && at >= 0 && !query;
    const int64_t to = at + ((int64_t)hk << c.page_log2);
    if (MODE == PAGES_BF16) {
      if (!keep) continue;
      store_row(static_cast<__nv_bfloat16*>(value ? c.v : c.k) + to * D, x, lane, D);
    } else {
      uint8_t byte;
      const uint4 codes = codes_e4m3<LANES>(x, byte);
      if (!keep) continue;
      uint8_t* p = static_cast<uint8_t*>(value ? c.v : c.k) + to * D;
      *reinterpret_cast<uint2*>(p + lane * 8) = make_uint2(codes.x, codes.y);
      *reinterpret_cast<uint2*>(p + D / 2 + lane * 8) = make_uint2(codes.z, codes.w);
      if (lane == 0) (value ? c.vs : c.ks)[to] = byte;
    }
  }
}

template <int D, bool HALF>
auto pick(int mode) {
  return mode == DENSE ? norm_rope<D, HALF, DENSE> : mode == PAGES_BF16 ? norm_rope<D, HALF, PAGES_BF16> : norm_rope<D, HALF, PAGES_E4M3>;
}

}  // namespace

cudaError_t launch_norm_rope(const Pool& c, const Seqs& s, bool dense, const RopeHow& how, int Hq, const Packed& q,
                             const Packed& qo, int Hk, const Packed& k, const Packed& ko, const Packed& v, cudaStream_t st) {
  const int n_sm = sm_count(), slots = THREADS / (c.d / 16);
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const int mode = dense ? DENSE : c.e4m3 ? PAGES_E4M3 : PAGES_BF16, heads = Hq + Hk * (dense ? 1 : 2);
  Tensors t{q, qo, k, ko, v, Hq, Hk, 0, 0};
  while ((1 << t.rows_log2) < std::min(s.rows, slots)) ++t.rows_log2;
  const int groups = (s.rows + (1 << t.rows_log2) - 1) >> t.rows_log2, step = slots >> t.rows_log2;
  // heads of a block: so many that all blocks run at once (a frame of 32 heads of 64: two heads a block 8.3 us, one 10.4)
  const int64_t room = (int64_t)BLOCKS * n_sm;
  t.per = (int)(((int64_t)heads * groups + room - 1) / room);
  t.per = (t.per + step - 1) / step * step;
  const dim3 grid(groups, (heads + t.per - 1) / t.per);
  auto* f = c.d == 128 ? (how.half ? pick<128, true>(mode) : pick<128, false>(mode))
                       : (how.half ? pick<64, true>(mode) : pick<64, false>(mode));
  return launch_kernel(f, grid, THREADS, 0, 1, false, st, c, s, how, t);
}

}  // namespace cache
}  // namespace dkv
