// Shared by the kernels of attention over an 8-bit cache.
//
// For row i of a sequence and query head h over KV head h / G:
//   s_j = scale 2^(ek_j) sum_d q_d k_jd,  o = sum_j softmax(s)_j 2^(ev_j) v_j
// over the tokens j that the row sees, in one pass with the running maximum and
// sum of the softmax. The 8-bit values are exact in f16, so both products run
// on the matrix cores in f16 with the scales outside of them: K's on the
// scores, V's on the probabilities. A probability goes into the second product
// as p 2^(ev - M) 2^u in f16, M the largest V exponent met so far in blocks of
// which the query sees a token (the accumulators are in units of 2^(M - u) and
// rescaled when M grows), so that what it loses is its rounding to 11 bits, or
// 2^-(25 + u) of the largest value (u is 15, or 7 where p may reach 2^8).
// bf16 queries enter as f16 times a power of two that puts a row's largest
// value in [2^14, 2^15): exact down to 2^-30 of it.
#pragma once

#include "qcache.h"

namespace jetk {

// Partial results of a split: o [split][row * Hq + head][hd] (not divided by
// l), then m and l [split][row * Hq + head].
struct Parts {
  float *o, *m, *l;
};
__device__ __host__ __forceinline__ Parts parts_of(void *ws, int64_t n, int nsplit, int hd) {
  float *o = (float *)ws;
  return {o, o + n * nsplit * hd, o + n * nsplit * (hd + 1)};
}

// A thread's index that the compiler takes for a new value at each place: what
// is computed from it stays inside the loop (moved out of it, the addresses of
// a whole tile took registers that the accumulators need).
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Query q as f16 fragments: fragment ks holds elements at + ks * step .. + 7,
// with the sign of scale2. Returns what scores are multiplied by, up to the
// scales of K (>= 0).
template <typename T, int NK>
__device__ __forceinline__ float load_query(Frag<f16> (&f)[NK], const T *q, int at, int step, bool vec, float scale2) {
  float x[NK][8];
  uint32_t top = 0;
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) {
    if (vec) {
      const uint4 u = ld16(q + at + ks * step);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[ks][2 * j] = to_f<T>(__builtin_bit_cast(T, (uint16_t)(w[j] & 0xffff)));
        x[ks][2 * j + 1] = to_f<T>(__builtin_bit_cast(T, (uint16_t)(w[j] >> 16)));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[ks][j] = to_f<T>(q[at + ks * step + j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[ks][j]) & 0x7fffffffu);
  }
  float up = scale2 < 0.0f ? -1.0f : 1.0f;
  scale2 = fabsf(scale2);
  if constexpr (__is_same(T, bf16)) {
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    // largest value 2^x f, f in [1, 2): times 2^(14 - x), and back on the scores
    const int e = min(max((int)(top >> 23) - 127, -112), 127);
    if (top) up *= pow2i(14 - e);
    if (top) scale2 *= pow2i(e - 14);
  }
#pragma unroll
  for (int ks = 0; ks < NK; ++ks)
#pragma unroll
    for (int j = 0; j < 8; ++j) f[ks].v[j] = (f16)(x[ks][j] * up);
  return scale2;
}

// Maximum over the four lanes that hold one query (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float query_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Scales of K and V blocks from their bytes (255: NaN), V's in units of
// 2^(M - 127).
__device__ __forceinline__ float k_scale(int e) {
  return e == kExpNaN ? __uint_as_float(0x7fc00000u) : pow2i(e - kExpBias);
}
__device__ __forceinline__ float v_scale(int e, int M) {
  return e == kExpNaN ? __uint_as_float(0x7fc00000u) : e - M < -126 ? 0.0f : pow2i(e - M);
}
__device__ __forceinline__ int v_top(int e) { return e == kExpNaN ? 0 : e; }

// The kernel of k_qattn_rows.hip on a batch, a row's keys in nsplit equal parts
// (no workspace where nsplit is 1).
hipError_t launch_qattn_rows(const QAttn &a, int nsplit, hipStream_t st);

}  // namespace jetk
