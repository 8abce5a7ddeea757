// Attention over a cache held in 8 bits (jet.h: jet_qcache_attention).
//
// For row i of a sequence and query head h over KV head h / G:
//   s_j = scale 2^(ek_j) sum_d q_d k_jd,  o = sum_j softmax(s)_j 2^(ev_j) v_j
// over the tokens j that the row sees, with the running maximum and sum of the
// softmax kept as the keys pass.
#include <algorithm>

#include "qcache.h"

namespace jetk {

int64_t qattn_workspace(const QCache &, const QBatch &, int) { return 0; }

// One wave per (row, query head); lane l holds dims l D .. l D + D - 1.
template <typename T, typename O, int FMT, int D>
__global__ __launch_bounds__(64) void qattn_row_kernel(QAttn a) {
  const int lane = threadIdx.x, hq = blockIdx.y, h = hq / (a.Hq / a.c.H);
  const QSeq s = qseq(a.b, a.c, blockIdx.z);
  const int hd = a.c.hd;
  const uint8_t *k = a.c.k + ((int64_t)h * a.c.S + s.slot0) * hd + lane * D;
  const uint8_t *v = a.c.v + ((int64_t)h * a.c.S + s.slot0) * hd + lane * D;
  const uint8_t *ke = a.c.ke + (int64_t)h * (a.c.S >> a.c.lb) + (s.slot0 >> a.c.lb);
  const uint8_t *ve = a.c.ve + (int64_t)h * (a.c.S >> a.c.lb) + (s.slot0 >> a.c.lb);
  auto scale_of = [](int e) { return e == kExpNaN ? __uint_as_float(0x7fc00000u) : pow2i(e - kExpBias); };
  for (int i = blockIdx.x; i < s.n; i += gridDim.x) {
    const int64_t row = s.row0 + i;
    const int pos = s.pos0 + i, end = pos < 0 ? 0 : a.causal ? pos + 1 : s.len;
    const T *q = (const T *)a.q.p + row * a.q.rs + (int64_t)hq * a.q.hs + lane * D;
    float x[D], o[D], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int d = 0; d < D; ++d) {
      x[d] = to_f<T>(q[d]);
      o[d] = 0.0f;
    }
    for (int j = 0; j < end; ++j) {
      float dot = 0.0f;
#pragma unroll
      for (int d = 0; d < D; ++d) dot += x[d] * unpack8<FMT, 0>(k[(int64_t)j * hd + d]);
      const float z = warp_sum(dot) * scale_of(ke[j >> a.c.lb]) * a.scale * kLog2e;
      const float top = fmaxf(m, z);
      const float base = top == -INFINITY ? 0.0f : top;
      const float f = __builtin_amdgcn_exp2f(m - base), p = __builtin_amdgcn_exp2f(z - base);
      l = l * f + p;
      const float pv = p * scale_of(ve[j >> a.c.lb]);
#pragma unroll
      for (int d = 0; d < D; ++d) o[d] = o[d] * f + pv * unpack8<FMT, 0>(v[(int64_t)j * hd + d]);
      m = top;
    }
    const float inv = end > 0 ? 1.0f / l : 0.0f;
    O *out = (O *)a.out.p + row * a.out.rs + (int64_t)hq * a.out.hs + lane * D;
#pragma unroll
    for (int d = 0; d < D; ++d) out[d] = from_f<O>(o[d] * inv);
    if (a.lse && lane == 0) a.lse[row * a.Hq + hq] = end > 0 ? m * kLn2 + logf(l) : -INFINITY;
  }
}

template <typename T, typename O, int FMT>
static hipError_t run_hd(const QAttn &a, hipStream_t st) {
  const dim3 grid((unsigned)std::min(std::max(a.b.max_rows, 1), 65536), (unsigned)a.Hq, (unsigned)a.b.n_seq);
  if (a.c.hd == 64) hipLaunchKernelGGL((qattn_row_kernel<T, O, FMT, 1>), grid, dim3(64), 0, st, a);
  else if (a.c.hd == 128) hipLaunchKernelGGL((qattn_row_kernel<T, O, FMT, 2>), grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL((qattn_row_kernel<T, O, FMT, 4>), grid, dim3(64), 0, st, a);
  return hipGetLastError();
}
template <typename T, typename O> static hipError_t run_fmt(const QAttn &a, hipStream_t st) {
  return a.c.fmt == 0 ? run_hd<T, O, 0>(a, st) : run_hd<T, O, 1>(a, st);
}

hipError_t launch_qattn(const QAttn &a, hipStream_t st) {
  if (a.b.n_seq <= 0 || a.b.n_rows <= 0) return hipSuccess;
  if (a.q.type == 1) return a.out.type == 0 ? run_fmt<f16, float>(a, st) : run_fmt<f16, f16>(a, st);
  return a.out.type == 0 ? run_fmt<bf16, float>(a, st) : run_fmt<bf16, bf16>(a, st);
}

}  // namespace jetk
