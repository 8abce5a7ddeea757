// Attention cache in 8 bits: rows of K and V quantised as they are written, and
// read back.
//
// A block of B tokens of one head has one scale 2^e (byte e + 127). Writing is
// a maximum over the block's new values and a rounding of each:
//   e = least (>= -60) with max|x| <= top 2^e, top = 127 (int8) or 448 (e4m3)
//   q = rne(x 2^-e); where earlier tokens of the sequence share the block,
//   e = max(e, e_old) and, if it grew, q_old = rne(q_old 2^(e_old - e)).
// 2^-e is exact, so every value is rounded once; an earlier value that goes
// through several growths is off by less than 2^e (1/2 + 1/4 + ... steps).
// Memory bound: rows read once, one byte written for each value, and the other
// way round to read. 36400 bf16 tokens of 8 heads of 128 in blocks of 64, K and V
// (224 MB either way): written in 57 us (3.9 TB/s), read back in 37 (6.0 TB/s, a
// part from the last-level cache, where the write left it). 164000 tokens read as
// f16 (1.0 GB): 183 us, 5.5 TB/s. A large copy moves 4.7 TB/s.
#include <algorithm>

#include "qcache.h"

namespace jetk {

// Eight consecutive values of a row as they lie in memory, and as floats.
template <typename T> struct Raw8 {
  uint4 u[sizeof(T) / 2];
};
template <typename T, bool VEC> __device__ __forceinline__ Raw8<T> load8(const T *p) {
  Raw8<T> r;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = ld16(p + i * 16 / sizeof(T));
  } else {
    T x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = p[j];
    __builtin_memcpy(&r, x, sizeof(r));
  }
  return r;
}
template <typename T> __device__ __forceinline__ void floats8(float (&x)[8], const Raw8<T> &r) {
  T t[8];
  __builtin_memcpy(t, &r, sizeof(r));
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = to_f<T>(t[j]);
}
template <typename T, bool VEC> __device__ __forceinline__ void store8(T *p, const float (&x)[8]) {
  if constexpr (VEC && sizeof(T) == 2) {
    st16(p, make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])));
  } else if constexpr (VEC) {
    st16(p, __builtin_bit_cast(uint4, f32x4{x[0], x[1], x[2], x[3]}));
    st16(p + 4, __builtin_bit_cast(uint4, f32x4{x[4], x[5], x[6], x[7]}));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = from_f<T>(x[j]);
  }
}
template <int FMT> __device__ __forceinline__ void unpack8x8(float (&x)[8], uint2 w) {
  x[0] = unpack8<FMT, 0>(w.x); x[1] = unpack8<FMT, 1>(w.x); x[2] = unpack8<FMT, 2>(w.x); x[3] = unpack8<FMT, 3>(w.x);
  x[4] = unpack8<FMT, 0>(w.y); x[5] = unpack8<FMT, 1>(w.y); x[6] = unpack8<FMT, 2>(w.y); x[7] = unpack8<FMT, 3>(w.y);
}

// One workgroup per (block that a sequence's rows touch, head of K or of V,
// sequence): it owns the block, so nothing is shared between workgroups. A
// thread holds NC pieces of eight values between the two passes over them
// (maximum, rounding); blocks of more values than that are read twice (the rows
// above: 62 us with every block read twice, from L2 the second time, 57 held).
template <typename T, int FMT, bool VEC, int NC>
__global__ __launch_bounds__(256) void qcache_write_kernel(QCache c, QBatch b, QRows rk, QRows rv) {
  __shared__ uint32_t wmax[4];
  const int tid = threadIdx.x, h = blockIdx.y >> 1;
  const bool isv = blockIdx.y & 1;
  const QSeq s = qseq(b, c, blockIdx.z);
  if (s.lo >= s.hi) return;
  const int B = 1 << c.lb, hd = c.hd, lc = __builtin_ctz(hd) - 3, cpr = 1 << lc;  // pieces per row
  const QRows &r = isv ? rv : rk;
  uint8_t *data = (isv ? c.v : c.k) + ((int64_t)h * c.S + s.slot0) * hd;
  uint8_t *exps = (isv ? c.ve : c.ke) + (int64_t)h * (c.S >> c.lb) + (s.slot0 >> c.lb);
  const int b0 = s.lo >> c.lb, b1 = (s.hi - 1) >> c.lb;
  for (int blk = b0 + blockIdx.x; blk <= b1; blk += gridDim.x) {
    const int first = blk << c.lb, lo = max(s.lo, first), hi = min(s.hi, first + B);  // the block's new tokens
    const T *src = (const T *)r.p + (int64_t)(s.row0 + lo - s.pos0) * r.rs + (int64_t)h * r.hs;
    const int n = (hi - lo) << lc;
    auto piece = [&](int i) { return load8<T, VEC>(src + (int64_t)(i >> lc) * r.rs + (i & (cpr - 1)) * 8); };
    uint32_t top = 0;  // float bits of |x| order like the values, NaN and infinity above all
    auto raise = [&](const Raw8<T> &p) {
      float x[8];
      floats8<T>(x, p);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    };
    const int old = lo > first ? exps[blk] : 0;  // scale byte of the block's earlier tokens
    Raw8<T> held[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k)
      if (k * 256 + tid < n) held[k] = piece(k * 256 + tid);
#pragma unroll
    for (int k = 0; k < NC; ++k)
      if (k * 256 + tid < n) raise(held[k]);
    for (int i = NC * 256 + tid; i < n; i += 256) raise(piece(i));
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) wmax[tid >> 6] = top;
    __syncthreads();
    top = max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3]));
    const int e = max(scale_byte<FMT>(top), old);
    const float down = e == kExpNaN ? 0.0f : pow2i(kExpBias - e);
    uint8_t *dst = data + (int64_t)lo * hd;
    auto put = [&](int i, const Raw8<T> &p) {
      float x[8];
      floats8<T>(x, p);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = e == kExpNaN ? 0.0f : x[j] * down;
      *reinterpret_cast<uint2 *>(dst + (int64_t)i * 8) =
          make_uint2(pack8x4<FMT>(x[0], x[1], x[2], x[3]), pack8x4<FMT>(x[4], x[5], x[6], x[7]));
    };
#pragma unroll
    for (int k = 0; k < NC; ++k)
      if (k * 256 + tid < n) put(k * 256 + tid, held[k]);
    for (int i = NC * 256 + tid; i < n; i += 256) put(i, piece(i));
    if (e > old && lo > first && e != kExpNaN) {  // the earlier tokens' scale grew
      for (int i = tid; i < (lo - first) * cpr; i += 256) {
        uint2 *p = reinterpret_cast<uint2 *>(data + (int64_t)first * hd + (int64_t)i * 8);
        float x[8];
        unpack8x8<FMT>(x, *p);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = ldexpf(x[j], old - e);
        *p = make_uint2(pack8x4<FMT>(x[0], x[1], x[2], x[3]), pack8x4<FMT>(x[4], x[5], x[6], x[7]));
      }
    }
    __syncthreads();  // wmax and the old scale have been read
    if (tid == 0) exps[blk] = (uint8_t)e;
  }
}

// One workgroup per (run of tokens, head of K or of V, sequence). (Sizes are
// powers of two: shifts. Divisions by them cost the read above 42 us for 37.)
constexpr int kReadTokens = 32;
template <typename T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void qcache_read_kernel(QCache c, QBatch b, QRows rk, QRows rv) {
  const int tid = threadIdx.x, h = blockIdx.y >> 1;
  const bool isv = blockIdx.y & 1;
  const QSeq s = qseq(b, c, blockIdx.z);
  const int hd = c.hd, lc = __builtin_ctz(hd) - 3;  // log2 of the pieces of eight values in a row
  const QRows &r = isv ? rv : rk;
  const uint8_t *data = (isv ? c.v : c.k) + ((int64_t)h * c.S + s.slot0) * hd;
  const uint8_t *exps = (isv ? c.ve : c.ke) + (int64_t)h * (c.S >> c.lb) + (s.slot0 >> c.lb);
  for (int64_t t0 = s.lo + (int64_t)blockIdx.x * kReadTokens; t0 < s.hi; t0 += (int64_t)gridDim.x * kReadTokens) {
    const int n = min(kReadTokens, s.hi - (int)t0) << lc;
    for (int i = tid; i < n; i += 256) {
      const int t = (int)t0 + (i >> lc), d = (i & ((1 << lc) - 1)) * 8;
      const int e = exps[t >> c.lb];
      float x[8];
      unpack8x8<FMT>(x, *reinterpret_cast<const uint2 *>(data + (int64_t)t * hd + d));
      const float up = e == kExpNaN ? __uint_as_float(0x7fc00000u) : pow2i(e - kExpBias);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= up;
      store8<T, VEC>((T *)r.p + (int64_t)(s.row0 + t - s.pos0) * r.rs + (int64_t)h * r.hs + d, x);
    }
  }
}

// Launch over (x, head of K or V, sequence); kernels walk on where a sequence
// has more rows than the grid was sized for. NC by the values of a whole block's
// new rows, so that appended tokens hold no idle pieces.
template <typename T, int NC>
static void write_nc(dim3 grid, const QCache &c, const QBatch &b, const QRows &k, const QRows &v, hipStream_t st) {
  const bool vec = k.vec && v.vec;
  if (c.fmt == 0 && vec) hipLaunchKernelGGL((qcache_write_kernel<T, 0, true, NC>), grid, dim3(256), 0, st, c, b, k, v);
  else if (c.fmt == 0) hipLaunchKernelGGL((qcache_write_kernel<T, 0, false, NC>), grid, dim3(256), 0, st, c, b, k, v);
  else if (vec) hipLaunchKernelGGL((qcache_write_kernel<T, 1, true, NC>), grid, dim3(256), 0, st, c, b, k, v);
  else hipLaunchKernelGGL((qcache_write_kernel<T, 1, false, NC>), grid, dim3(256), 0, st, c, b, k, v);
}
template <typename T>
static hipError_t write_t(const QCache &c, const QBatch &b, const QRows &k, const QRows &v, hipStream_t st) {
  const int64_t rows = std::max(b.max_rows, 1), blocks = (rows + (1 << c.lb) - 2) / (1 << c.lb) + 1;
  const dim3 grid((unsigned)std::min<int64_t>(blocks, 65536), (unsigned)(2 * c.H), (unsigned)b.n_seq);
  // pieces of eight values in a block's new rows
  const int64_t pieces = std::min<int64_t>(rows, 1 << c.lb) * c.hd / 8;
  if (pieces <= 256) write_nc<T, 1>(grid, c, b, k, v, st);
  else if (pieces <= 512) write_nc<T, 2>(grid, c, b, k, v, st);
  else write_nc<T, 4>(grid, c, b, k, v, st);
  return hipGetLastError();
}
template <typename T>
static hipError_t read_t(const QCache &c, const QBatch &b, const QRows &k, const QRows &v, hipStream_t st) {
  const int64_t runs = ((int64_t)std::max(b.max_rows, 1) + kReadTokens - 1) / kReadTokens;
  const dim3 grid((unsigned)std::min<int64_t>(runs, 65536), (unsigned)(2 * c.H), (unsigned)b.n_seq);
  const bool vec = k.vec && v.vec;
  if (c.fmt == 0 && vec) hipLaunchKernelGGL((qcache_read_kernel<T, 0, true>), grid, dim3(256), 0, st, c, b, k, v);
  else if (c.fmt == 0) hipLaunchKernelGGL((qcache_read_kernel<T, 0, false>), grid, dim3(256), 0, st, c, b, k, v);
  else if (vec) hipLaunchKernelGGL((qcache_read_kernel<T, 1, true>), grid, dim3(256), 0, st, c, b, k, v);
  else hipLaunchKernelGGL((qcache_read_kernel<T, 1, false>), grid, dim3(256), 0, st, c, b, k, v);
  return hipGetLastError();
}

hipError_t launch_qcache_write(const QCache &c, const QBatch &b, const QRows &k, const QRows &v, hipStream_t st) {
  if (b.n_seq <= 0 || b.n_rows <= 0 || c.S <= 0) return hipSuccess;
  if (k.type != v.type) return hipErrorInvalidValue;
  if (k.type == 0) return write_t<float>(c, b, k, v, st);
  if (k.type == 1) return write_t<f16>(c, b, k, v, st);
  return write_t<bf16>(c, b, k, v, st);
}

hipError_t launch_qcache_read(const QCache &c, const QBatch &b, const QRows &k, const QRows &v, hipStream_t st) {
  if (b.n_seq <= 0 || b.n_rows <= 0 || c.S <= 0) return hipSuccess;
  if (k.type != v.type) return hipErrorInvalidValue;
  if (k.type == 0) return read_t<float>(c, b, k, v, st);
  if (k.type == 1) return read_t<f16>(c, b, k, v, st);
  return read_t<bf16>(c, b, k, v, st);
}

// One workgroup per (block of a sequence, head of K or of V, sequence): 16-byte
// pieces of whole blocks and their scale bytes.
__global__ __launch_bounds__(256) void qcache_copy_kernel(QCache s, QCache d, const int64_t *__restrict__ s0,
                                                          const int64_t *__restrict__ d0, const int32_t *__restrict__ len) {
  const int h = blockIdx.y >> 1, q = blockIdx.z;
  const bool isv = blockIdx.y & 1;
  const int blocks = (len[q] + (1 << s.lb) - 1) >> s.lb, n = (s.hd << s.lb) / 16;
  const int64_t sb = s0[q] >> s.lb, db = d0[q] >> d.lb;
  for (int b = blockIdx.x; b < blocks; b += gridDim.x) {
    const uint4 *from = (const uint4 *)((isv ? s.v : s.k) + ((int64_t)h * s.S + ((sb + b) << s.lb)) * s.hd);
    uint4 *to = (uint4 *)((isv ? d.v : d.k) + ((int64_t)h * d.S + ((db + b) << d.lb)) * d.hd);
    for (int i = threadIdx.x; i < n; i += 256) to[i] = from[i];
    if (threadIdx.x == 0)
      (isv ? d.ve : d.ke)[(int64_t)h * (d.S >> d.lb) + db + b] = (isv ? s.ve : s.ke)[(int64_t)h * (s.S >> s.lb) + sb + b];
  }
}

hipError_t launch_qcache_copy(const QCache &src, const QCache &dst, const int64_t *src_slot0, const int64_t *dst_slot0,
                              const int32_t *len, int n_seq, hipStream_t st) {
  if (src.H != dst.H || src.hd != dst.hd || src.lb != dst.lb || src.fmt != dst.fmt) return hipErrorInvalidValue;
  for (int q = 0; q < n_seq; q += 65535) {
    const int n = std::min(n_seq - q, 65535);
    hipLaunchKernelGGL(qcache_copy_kernel, dim3(64, 2 * src.H, n), dim3(256), 0, st, src, dst, src_slot0 + q, dst_slot0 + q,
                       len + q);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace jetk
