// Penalties for repeated tokens, biases and masks on the logits of a decode
// step (jet.h: jet_logits_adjust).
//
// A workgroup takes a slice of one row's vocabulary: the row's history is
// counted into the slice's counters in LDS (whole numbers: the order of the
// additions does not matter), the row's biases are added up there in list
// order, and the slice's logits pass through registers once. What it cannot do
// without: every logit read and written once, the mask's bit and the history's
// ids besides; each slice reads the row's whole history (from L2 after the first).
// 256 rows of 151936 bf16 logits, histories of 200 .. 4096, 300 biases a row and
// masks: 51 us (3.1 TB/s) where a copy of the logits takes 31, the mask alone 30:
// the counting and the listed tokens are some 500 vector instructions a wave, in
// turn with the loads. Slices of 4096 because the work
// that every slice repeats (clearing, the lists) and the waves that wait at its
// barriers balance there: 8192 tokens 66 us, 16384 in eight waves 73, a
// workgroup that walks over several slices 88 (at 57 for this one then). Writing
// the slice by its mask alone and then only the listed tokens over it: 62
// (scattered 2-byte stores).
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace jetk {

constexpr int kSlice = 4096, kLogitThreads = 256;

// The rules of one token. c: bit 0, in the history; the rest, how often behind
// the prompt. Without branches: where a vector has any token of the lists, its
// tokens go through (a branch of each lane was slower), but for those that are of
// no list in any lane; those of no list come out as they went in. A product with
// 1 / repetition would save 4% of the time of 256 rows, but it rounds twice, and
// overflows where the quotient need not.
struct RowRules {
  float rep, pres, freq;
};
__device__ __forceinline__ float adjusted(float z, uint32_t c, float bias, const RowRules &w) {
  z = !c ? z : z > 0.0f ? z / w.rep : z * w.rep;
  z -= c > 1 ? w.freq * (float)(c >> 1) + w.pres : 0.0f;
  return z + bias;
}

__device__ const int32_t kNone[2] = {0, 0};
__device__ const float kOne = 1.0f, kZero = 0.0f;

// HIST, BIAS: whether any row may have a history or biases. VEC: rows of in and
// out start at 16-byte boundaries.
template <typename T, bool HIST, bool BIAS, bool VEC>
__global__ __launch_bounds__(kLogitThreads) void logits_adjust_kernel(LogitsArgs a) {
  // the slice's counters, then (in the same place: two arrays would halve the
  // workgroups a CU holds, 72 us against 57 for the rows above) its biases
  __shared__ __align__(16) uint32_t cnt[HIST || BIAS ? kSlice : 4];
  float *bias = reinterpret_cast<float *>(cnt);
  // Word of token v: of every second 8 groups of four the neighbours change
  // places, so that the lanes of a wave, each reading the first (or the second)
  // four of its eight tokens, meet every bank alike (54 us without, 50 with).
  auto at = [](int v) { return v ^ (v >> 3 & 4); };
  const int tid = threadIdx.x, r = blockIdx.y, v0 = blockIdx.x * kSlice, nv = min(kSlice, a.V - v0);
  const T *in = (const T *)a.in + (int64_t)r * a.in_ld + v0;
  T *out = (T *)a.out + (int64_t)r * a.out_ld + v0;
  const bool inplace = a.in == a.out;
  constexpr int N = VEC ? 16 / sizeof(T) : 1;  // tokens of a vector; they lie in one word of the mask
  constexpr int NV = kSlice / kLogitThreads / N;
  // The slice's logits are on their way while the lists are counted (unless
  // they are changed in place, where most need not be read at all).
  uint4 u[VEC ? NV : 1];
  uint32_t m[VEC ? NV : 1];
  if constexpr (VEC) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = (k * kLogitThreads + tid) * N;
      if (!inplace && i + N <= nv) u[k] = ld16(in + i);
    }
  }
  // what belongs to the row, in one round of loads: absent rules read a default
  const int32_t *hp = HIST ? a.h_off + r : kNone, *bp = BIAS ? a.b_off + r : kNone;
  const int32_t *pp = HIST && a.h_prompt ? a.h_prompt + r : kNone, *ip = a.mask_index ? a.mask_index + r : kNone;
  const float *rp = a.rep ? a.rep + r : &kOne, *sp = a.pres ? a.pres + r : &kZero, *fp = a.freq ? a.freq + r : &kZero;
  const int32_t *ep = HIST && a.h_end ? a.h_end + r : hp + 1;
  int h0 = hp[0], h1 = ep[0], b0 = bp[0], b1 = bp[1];
  const int prompt = pp[0], index = ip[0];
  const RowRules w = {*rp, *sp, *fp};
  if (h0 < 0 || h1 < h0 || h1 > a.n_hist) h0 = h1 = 0;
  if (b0 < 0 || b1 < b0 || b1 > a.n_bias) b0 = b1 = 0;
  const int mi = a.mask_index ? index : a.masks ? r : -1;  // (without masks n_masks is 0)
  const bool none = mi >= a.n_masks;  // a mask that does not exist allows nothing
  const uint32_t *mask = mi < 0 || none ? nullptr : a.masks + (int64_t)mi * a.mask_ld + v0 / 32;
  const bool hist = HIST && h1 > h0, biased = BIAS && b1 > b0;
  // A batch of the history is eight ids a thread, one of the biases four a lane
  // of the first wave; the first ones are on their way while LDS is cleared. An
  // id of -1 lies in no slice.
  const bool adds = biased && tid < 64;
  int hid[HIST ? 8 : 1], hnext[HIST ? 8 : 1], bid[BIAS ? 4 : 1];
  float bval[BIAS ? 4 : 1];
  auto load_hist = [&](int (&id)[HIST ? 8 : 1], int i0) {
#pragma unroll
    for (int j = 0; j < (HIST ? 8 : 1); ++j) {
      const int i = i0 + j * kLogitThreads + tid;
      id[j] = i < h1 ? a.h_ids[i] : -1;
    }
  };
  auto load_bias = [&](int i0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + j * 64 + tid;
      bid[j] = i < b1 ? a.b_ids[i] : -1;
      bval[j] = i < b1 ? a.b_val[i] : 0.0f;
    }
  };
  if constexpr (HIST)
    if (hist) load_hist(hid, h0);
  if constexpr (BIAS)
    if (adds) load_bias(b0);
  if constexpr (VEC) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = (k * kLogitThreads + tid) * N;
      m[k] = none ? 0u : 0xffffffffu;
      if (mask && i + N <= nv) m[k] = mask[i >> 5] >> (i & 31);
    }
  }
  // no bias is -0.0: added to any logit it leaves that logit, -0.0 too
  const uint32_t sign = __float_as_uint(-0.0f);
  const uint4 zero = {0, 0, 0, 0}, no_bias = {sign, sign, sign, sign};
  if (hist || biased) {
    const uint4 start = hist ? zero : no_bias;
    for (int i = tid; i < kSlice / 4; i += kLogitThreads) reinterpret_cast<uint4 *>(cnt)[i] = start;
    __syncthreads();
  }
  if constexpr (HIST) {
    const int made = h0 + max(0, min(prompt, h1 - h0));
    for (int i0 = h0; hist && i0 < h1; i0 += 8 * kLogitThreads) {
      if (i0 + 8 * kLogitThreads < h1) load_hist(hnext, i0 + 8 * kLogitThreads);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t v = (uint32_t)hid[j] - (uint32_t)v0;
        if (v < (uint32_t)nv) {
          if (i0 + j * kLogitThreads + tid >= made) atomicAdd(&cnt[at(v)], 2u);
          else atomicOr(&cnt[at(v)], 1u);
        }
        hid[j] = hnext[j];
      }
    }
  }
  // this thread's tokens: vector k's from (k kLogitThreads + tid) N, or those
  // from tid on, kLogitThreads apart
  constexpr int NT = kSlice / kLogitThreads;
  uint32_t c[HIST ? NT : 1];
  if constexpr (HIST) {
    if (hist) __syncthreads();
#pragma unroll
    for (int k = 0; k < NT; k += VEC ? 4 : 1) {
      const int i = VEC ? (k / N * kLogitThreads + tid) * N + k % N : k * kLogitThreads + tid;
      if constexpr (VEC) {
        const uint4 q = hist ? *reinterpret_cast<const uint4 *>(&cnt[at(i)]) : zero;
        c[k] = q.x; c[k + 1] = q.y; c[k + 2] = q.z; c[k + 3] = q.w;
        if (hist && biased) *reinterpret_cast<uint4 *>(&cnt[at(i)]) = no_bias;
      } else {
        c[k] = hist ? cnt[at(i)] : 0u;
        if (hist && biased) cnt[at(i)] = sign;
      }
    }
    if (hist && biased) __syncthreads();
  }
  if constexpr (BIAS) {
    // entry after entry: LDS operations of one wave are done in their order,
    // so equal ids add up in list order
    for (int i0 = b0; adds && i0 < b1; i0 += 256) {
      if (i0 > b0) load_bias(i0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t v = (uint32_t)bid[j] - (uint32_t)v0;
        for (uint64_t in_slice = __ballot(v < (uint32_t)nv); in_slice; in_slice &= in_slice - 1) {
          if (tid == __builtin_ctzll(in_slice)) atomicAdd(&bias[at(v)], bval[j]);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
    }
  }
  if (biased) __syncthreads();
  auto count_of = [&](int k) { return HIST ? c[k] : 0u; };
  if constexpr (VEC) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = (k * kLogitThreads + tid) * N;
      if (i + N > nv) {  // the row's end, inside a vector
        for (int j = 0; j < N && i + j < nv; ++j) {
          uint32_t q = 0;
#pragma unroll
          for (int e = 0; e < N; ++e) q = e == j ? count_of(k * N + e) : q;
          const float b = biased ? bias[at(i + j)] : -0.0f;
          T x = in[i + j];
          if (q || b != 0.0f) x = from_f<T>(adjusted(to_f<T>(x), q, b, w));
          const bool allowed = !none && (!mask || (mask[(i + j) >> 5] >> ((i + j) & 31) & 1));
          out[i + j] = allowed ? x : from_f<T>(-INFINITY);
        }
        continue;
      }
      uint32_t seen = 0;
      float b[N];
      bool off = false;  // any bias
#pragma unroll
      for (int j = 0; j < N; ++j) {
        seen |= count_of(k * N + j);
        b[j] = -0.0f;
      }
#pragma unroll
      for (int j = 0; j < N; j += 4) {
        if (biased) {
          const f32x4 q = *reinterpret_cast<const f32x4 *>(&bias[at(i + j)]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            b[j + e] = q[e];
            off |= q[e] != 0.0f;
          }
        }
      }
      const bool masked = ~m[k] & ((1u << N) - 1);
      if (!seen && !off && !masked) {  // these logits stay as they are
        if (!inplace) st16(out + i, u[k]);
        continue;
      }
      if (inplace) u[k] = ld16(in + i);
      T x[N];
      __builtin_memcpy(x, &u[k], 16);
      if (seen || off) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (__any(count_of(k * N + j) || b[j] != 0.0f))  // of any lane's vector
            x[j] = from_f<T>(adjusted(to_f<T>(x[j]), count_of(k * N + j), b[j], w));
      }
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (!(m[k] >> j & 1)) x[j] = from_f<T>(-INFINITY);
      __builtin_memcpy(&u[k], x, 16);
      st16(out + i, u[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      const int i = k * kLogitThreads + tid;
      if (i >= nv) break;
      const bool allowed = !none && (!mask || (mask[i >> 5] >> (i & 31) & 1));
      const float b = biased ? bias[at(i)] : -0.0f;
      T x = in[i];
      if (count_of(k) || b != 0.0f) x = from_f<T>(adjusted(to_f<T>(x), count_of(k), b, w));
      out[i] = allowed ? x : from_f<T>(-INFINITY);
    }
  }
}

template <typename T, bool HIST, bool BIAS> static void run_vec(const LogitsArgs &a, dim3 grid, hipStream_t st) {
  const int64_t es = sizeof(T);
  const bool vec = ((uintptr_t)a.in | (uintptr_t)a.out) % 16 == 0 && a.in_ld * es % 16 == 0 && a.out_ld * es % 16 == 0;
  if (vec) hipLaunchKernelGGL((logits_adjust_kernel<T, HIST, BIAS, true>), grid, dim3(kLogitThreads), 0, st, a);
  else hipLaunchKernelGGL((logits_adjust_kernel<T, HIST, BIAS, false>), grid, dim3(kLogitThreads), 0, st, a);
}
template <typename T> static void run_rules(const LogitsArgs &a, dim3 grid, hipStream_t st) {
  const bool hist = a.h_off && a.n_hist > 0, bias = a.b_off && a.n_bias > 0;
  if (hist && bias) run_vec<T, true, true>(a, grid, st);
  else if (hist) run_vec<T, true, false>(a, grid, st);
  else if (bias) run_vec<T, false, true>(a, grid, st);
  else run_vec<T, false, false>(a, grid, st);
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
    if (b.h_end) b.h_end += r0;
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
    if (a.type == 0) run_rules<float>(b, grid, st);
    else if (a.type == 1) run_rules<f16>(b, grid, st);
    else run_rules<bf16>(b, grid, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace jetk
