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
__device__ __forceinline__ QSeq qseq(const QBatch &b, const QCache &c, int s) {
  QSeq q;
  q.slot0 = b.slot0[s];
  q.len = b.len[s];
  q.row0 = b.rows ? b.rows[s] : s;
  const int end = b.rows ? b.rows[s + 1] : s + 1;
  q.n = end - q.row0;
  q.lo = q.hi = 0;
  const bool ok = q.slot0 >= 0 && q.slot0 < c.S && (q.slot0 & ((1 << c.lb) - 1)) == 0 && q.row0 >= 0 && end >= q.row0 &&
                  end <= b.n_rows && q.len >= 0 && q.len <= c.S - q.slot0;
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

}  // namespace jetk
