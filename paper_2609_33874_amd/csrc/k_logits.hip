// Penalties for repeated tokens, biases and masks on the logits of a decode
// step (jet.h: jet_logits_adjust).
//
// A workgroup takes a slice of one row's vocabulary: the row's history is
// counted into the slice's counters in LDS (whole numbers: the order of the
// additions does not matter), the row's biases are added up there in list
// order, and the slice's logits pass through registers once. Memory bound:
// every logit read and written once, the mask's bit and the history's ids
// besides; each slice reads the row's whole history (from L2 after the first).
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace jetk {

constexpr int kSlice = 4096, kLogitThreads = 256;

template <typename T>
__global__ __launch_bounds__(kLogitThreads) void logits_adjust_kernel(LogitsArgs a) {
  __shared__ uint32_t cnt[kSlice];  // bit 0: in the history; the rest: how often behind the prompt
  __shared__ float bias[kSlice];
  __shared__ int l_id[kLogitThreads];
  __shared__ float l_val[kLogitThreads];
  __shared__ int l_n[kLogitThreads / 64];
  const int tid = threadIdx.x, r = blockIdx.y, v0 = blockIdx.x * kSlice, nv = min(kSlice, a.V - v0);
  int h0 = 0, h1 = 0, b0 = 0, b1 = 0;
  if (a.h_off) {
    h0 = a.h_off[r];
    h1 = a.h_off[r + 1];
    if (h0 < 0 || h1 < h0 || h1 > a.n_hist) h0 = h1 = 0;
  }
  if (a.b_off) {
    b0 = a.b_off[r];
    b1 = a.b_off[r + 1];
    if (b0 < 0 || b1 < b0 || b1 > a.n_bias) b0 = b1 = 0;
  }
  if (h1 > h0) {
    for (int i = tid; i < kSlice; i += kLogitThreads) cnt[i] = 0;
    __syncthreads();
    const int made = a.h_prompt ? max(0, a.h_prompt[r]) : 0;
    for (int i = h0 + tid; i < h1; i += kLogitThreads) {
      const uint32_t v = (uint32_t)a.h_ids[i] - (uint32_t)v0;
      if (v < (uint32_t)nv) {
        atomicOr(&cnt[v], 1u);
        if (i - h0 >= made) atomicAdd(&cnt[v], 2u);
      }
    }
  }
  if (b1 > b0) {
    for (int i = tid; i < kSlice; i += kLogitThreads) bias[i] = 0.0f;
    // a run of the list at a time: its entries inside the slice are kept in
    // order, then every thread adds those of its own tokens
    for (int i0 = b0; i0 < b1; i0 += kLogitThreads) {
      const int i = i0 + tid;
      const uint32_t v = i < b1 ? (uint32_t)a.b_ids[i] - (uint32_t)v0 : 0xffffffffu;
      const bool in = v < (uint32_t)nv;
      const uint64_t m = __ballot(in);
      if ((tid & 63) == 0) l_n[tid >> 6] = __popcll(m);
      __syncthreads();
      int at = __popcll(m & ((1ull << (tid & 63)) - 1)), n = 0;
      for (int w = 0; w < kLogitThreads / 64; ++w) {
        if (w < tid >> 6) at += l_n[w];
        n += l_n[w];
      }
      if (in) {
        l_id[at] = (int)v;
        l_val[at] = a.b_val[i];
      }
      __syncthreads();
      for (int j = 0; j < n; ++j)
        if (l_id[j] % kLogitThreads == tid) bias[l_id[j]] += l_val[j];
      __syncthreads();
    }
  }
  __syncthreads();
  const int mi = !a.masks ? -1 : a.mask_index ? a.mask_index[r] : r;
  const uint32_t *mask = mi < 0 ? nullptr : a.masks + (int64_t)mi * a.mask_ld;
  const float rep = a.rep ? a.rep[r] : 1.0f, pres = a.pres ? a.pres[r] : 0.0f, freq = a.freq ? a.freq[r] : 0.0f;
  const T *in = (const T *)a.in + (int64_t)r * a.in_ld + v0;
  T *out = (T *)a.out + (int64_t)r * a.out_ld + v0;
  for (int i = tid; i < nv; i += kLogitThreads) {
    const int v = v0 + i;
    const bool allowed = !mask || (mi < a.n_masks && (mask[v >> 5] >> (v & 31) & 1));
    float z = to_f<T>(in[i]);
    if (h1 > h0) {
      const uint32_t c = cnt[i];
      if (c) z = z > 0.0f ? z / rep : z * rep;
      if (c > 1) z -= freq * (float)(c >> 1) + pres;
    }
    if (b1 > b0) z += bias[i];
    out[i] = from_f<T>(allowed ? z : -INFINITY);
  }
}

hipError_t launch_logits_adjust(const LogitsArgs &a, hipStream_t st) {
  if (a.R <= 0) return hipSuccess;
  for (int r0 = 0; r0 < a.R; r0 += 65535) {
    LogitsArgs b = a;
    b.R = std::min(a.R - r0, 65535);
    const int es = a.type == 0 ? 4 : 2;
    b.in = (const char *)a.in + (int64_t)r0 * a.in_ld * es;
    b.out = (char *)a.out + (int64_t)r0 * a.out_ld * es;
    if (b.h_off) b.h_off += r0;
    if (b.h_prompt) b.h_prompt += r0;
    if (b.rep) b.rep += r0;
    if (b.pres) b.pres += r0;
    if (b.freq) b.freq += r0;
    if (b.b_off) b.b_off += r0;
    if (b.mask_index) b.mask_index += r0;
    else if (b.masks) {
      b.masks += (int64_t)r0 * a.mask_ld;
      b.n_masks -= r0;
    }
    const dim3 grid((unsigned)((a.V + kSlice - 1) / kSlice), (unsigned)b.R);
    if (a.type == 0) hipLaunchKernelGGL(logits_adjust_kernel<float>, grid, dim3(kLogitThreads), 0, st, b);
    else if (a.type == 1) hipLaunchKernelGGL(logits_adjust_kernel<f16>, grid, dim3(kLogitThreads), 0, st, b);
    else hipLaunchKernelGGL(logits_adjust_kernel<bf16>, grid, dim3(kLogitThreads), 0, st, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace jetk
