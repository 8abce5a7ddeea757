// Device-side view of an 8-bit attention cache (jet.h: jet_qcache), shared by
// the kernels that write, read and attend to it.
#pragma once

#include "device.h"
#include "kernels.h"

namespace jetk {

constexpr int kExpBias = 127, kExpMin = -60, kExpNaN = 255;

// Sequence s of a batch, checked against what the cache and the row arrays
// hold: its rows are row0 .. row0 + n - 1 at positions pos0 .. pos0 + n - 1 of
// which those in [lo, hi) exist (none when the sequence is left out).
struct QSeq {
  int64_t slot0;
  int len, n, row0, pos0, lo, hi;
};
// s is the same for every lane, and so is what belongs to it.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ QSeq qseq(const QBatch &b, const QCache &c, int s) {
  QSeq q;
  const int64_t slot0 = b.slot0[s];
  q.slot0 = (int64_t)((uint64_t)(uint32_t)uniform((int)(slot0 >> 32)) << 32 | (uint32_t)uniform((int)slot0));
  q.len = uniform(b.len[s]);
  q.row0 = uniform(b.rows ? b.rows[s] : s);
  const int end = uniform(b.rows ? b.rows[s + 1] : s + 1);
  q.n = end - q.row0;
  q.lo = q.hi = 0;
  // (slot0 = S: a sequence without tokens behind the last block of a full cache)
  const bool ok = c.S > 0 && q.slot0 >= 0 && q.slot0 <= c.S && (q.slot0 & ((1 << c.lb) - 1)) == 0 && q.row0 >= 0 &&
                  end >= q.row0 && end <= b.n_rows && q.len >= 0 && q.len <= (1 << 30) && q.len <= c.S - q.slot0;
  if (!ok) {
    q.slot0 = 0;
    q.len = q.n = q.row0 = q.pos0 = 0;
    return q;
  }
  q.pos0 = q.len - q.n;
  q.lo = max(q.pos0, 0);
  q.hi = q.len;
  return q;
}

// 2^e for e in [-126, 127]
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Scale byte of values whose largest magnitude has the float bits u.
template <int FMT> __device__ __forceinline__ int scale_byte(uint32_t u) {
  if (u >= 0x7f800000u) return kExpNaN;
  const int x = (int)(u >> 23) - 126;  // u = f 2^x, f in [1/2, 1) (a subnormal lies below any scale)
  const uint32_t m = u & 0x7fffffu;
  // int8: f <= 127 / 128, e4m3: f <= 448 / 512
  const int e = FMT == 0 ? (m <= 0x7e0000u ? x - 7 : x - 6) : (m <= 0x600000u ? x - 9 : x - 8);
  return max(e, kExpMin) + kExpBias;
}

// Four scaled values as bytes, rounded to nearest even, value 0 lowest.
template <int FMT> __device__ __forceinline__ uint32_t pack8x4(float a, float b, float c, float d) {
  if (FMT == 0) {
    const int i = (int)rintf(a), j = (int)rintf(b), k = (int)rintf(c), l = (int)rintf(d);
    return (uint32_t)(i & 255) | (uint32_t)(j & 255) << 8 | (uint32_t)(k & 255) << 16 | (uint32_t)l << 24;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Byte j of a word as the value that it stands for.
template <int FMT, int J> __device__ __forceinline__ float unpack8(uint32_t w) {
  if (FMT == 0) return (float)((int)(w << (24 - 8 * J)) >> 24);
  return __builtin_amdgcn_cvt_f32_fp8((int)w, J);
}

// Four bytes of the cache as f16 (exact: int8 has 7 bits and a sign, e4m3 4).
// int8: byte ^ 0x80 under the exponent of 1024 is 1024 + 128 + q.
template <int FMT> __device__ __forceinline__ uint2 f16x4_of(uint32_t w) {
  if (FMT == 0) {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t lo = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u), hi = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
    const f16x2_t c = {(f16)1152.0f, (f16)1152.0f};
    const f16x2_t a = __builtin_bit_cast(f16x2_t, lo) - c, b = __builtin_bit_cast(f16x2_t, hi) - c;
    return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
  }
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}

// Bytes of four words transposed: word b of the result holds byte b of each.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

}  // namespace jetk
