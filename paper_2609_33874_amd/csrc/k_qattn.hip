// Attention over a cache held in 8 bits (jet.h: jet_qcache_attention).
// Few query slots: see qattn.h for the arithmetic, k_qattn_rows.hip for many.
//
// Bound by reading the cache once, 2 hd + a little bytes a key and KV head, while
// the matrix cores take at most 32 queries against each (a wave needs 16 at
// least: of one question's five or six heads of a group the rest are idle).
// 16 questions of 65536 .. 131072 keys, 8 KV heads of 128: 3.24 GB in 566 us, 5.7
// TB/s of the 6.4 that a kernel of plain reads reaches; 64 of 1024 .. 4096 keys 4.6
// TB/s in a single round of unequal workgroups; one question's 731 keys 10 us,
// which is latency (a tile's loads, products and softmax one after another, three
// tiles a wave, the joining in LDS).
#include <algorithm>

#include "qattn.h"

namespace jetk {

// ---------------------------------------------------------------------------
// Few query rows: keys split over waves and workgroups
// ---------------------------------------------------------------------------

constexpr int kTile = 32;    // keys of a wave's step
constexpr int kWaves = 8;    // waves of a workgroup, on neighbouring tiles
constexpr int kMaxSplit = 128;

template <int HD> struct QTile {
  static constexpr int KW = HD / 16;  // 32-bit words of K per lane and 16 keys
  static constexpr int VW = HD / 64;  // of V per lane and key
  uint32_t k[2][KW], v[8][VW];
  int ke[2], ve[2];
};

// Words of a row into registers: N words from p (aligned to their size).
template <int N> __device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t *p) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t *>(p);
  } else if constexpr (N == 2) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    w[0] = u.x; w[1] = u.y;
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 u = ld16(p + 16 * i);
      w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
    }
  }
}

// One workgroup per (block of 16 QB query slots and split of the keys, KV
// head, sequence); slot = row * G + head. Each wave takes every eighth tile of
// 32 keys of the split on its own (K and V go straight into registers as the
// matrix cores take them, the next tile's on their way meanwhile), and the
// waves' results are joined in LDS.
// A lane (g = lane / 16, c = lane % 16) holds of K dims HD/4 g .. of key c, as
// the A operand of S^T = K Q^T; then for query c the scores of keys 4 g .. + 3,
// as the B operand of O^T = V^T P^T; and of V the HD/16 dims from HD/16 c of
// those same keys: a transposition of bytes inside the lane makes the A
// operand, dim HD/16 c + i in product i.
template <typename T, typename O, int FMT, int HD, int QB>
__global__ __launch_bounds__(64 * kWaves, HD * QB == 256 ? 2 : 4) void qattn_split_kernel(QAttn a, int nsplit, int per) {
  constexpr int ND = HD / 16, NK = HD / 32, LD = HD + 4;
  typedef QTile<HD> Tile;
  __shared__ float s_o[kWaves][16 * QB][LD];
  __shared__ float s_m[kWaves][16 * QB], s_l[kWaves][16 * QB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.y, G = a.Hq / a.c.H, sp = blockIdx.x % nsplit;
  const QSeq sq = qseq(a.b, a.c, blockIdx.z);
  const int slots = sq.n * G;
  const int64_t base = ((int64_t)h * a.c.S + sq.slot0) * HD;
  const uint8_t *K = a.c.k + base, *V = a.c.v + base;
  const int64_t ebase = (int64_t)h * (a.c.S >> a.c.lb) + (sq.slot0 >> a.c.lb);
  const uint8_t *KE = a.c.ke + ebase, *VE = a.c.ve + ebase;

  for (int sb = blockIdx.x / nsplit * 16 * QB; sb < slots; sb += gridDim.x / nsplit * 16 * QB) {
    // keys of this block: up to the last one that its last row sees
    const int last_row = (min(sb + 16 * QB, slots) - 1) / G;
    const int kend = max(0, a.causal ? sq.pos0 + last_row + 1 : sq.len);
    const int ntile = (kend + kTile - 1) / kTile;
    const int t0 = (int)min((int64_t)sp * per, (int64_t)ntile);
    const int t1 = sp == nsplit - 1 ? ntile : (int)min((int64_t)(sp + 1) * per, (int64_t)ntile);
    int t = t0 + wave;

    // (a tile's rows lie one after another; past the sequence's end its last
    // row's bytes are loaded: those keys are masked)
    const int last = sq.len - 1;
    auto load_k = [&](Tile &x, int tile) {
      const int k0 = tile * kTile, lane = here(threadIdx.x) & 63, g = lane >> 4, c = lane & 15;
      const uint8_t *p = K + (int64_t)k0 * HD;
      const uint32_t end = (uint32_t)min(last - k0, kTile) * HD + (HD - HD / 4);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        load_words(x.k[kb], p + min((uint32_t)(c * HD + g * (HD / 4) + kb * 16 * HD), end));
        x.ke[kb] = KE[min(k0 + kb * 16, last) >> a.c.lb];
      }
    };
    auto load_v = [&](Tile &x, int tile) {
      const int k0 = tile * kTile, lane = here(threadIdx.x) & 63, g = lane >> 4, c = lane & 15;
      const uint8_t *p = V + (int64_t)k0 * HD;
      const uint32_t end = (uint32_t)min(last - k0, kTile) * HD + (HD - ND);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        load_words(x.v[i], p + min((uint32_t)(4 * g * HD + c * ND + ((i >> 2) * 16 + (i & 3)) * HD), end));
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) x.ve[kb] = VE[min(k0 + kb * 16, last) >> a.c.lb];
    };

    Tile cur;
    if (t < t1) load_k(cur, t), load_v(cur, t);  // (the queries' way here is as long)

    int vis[QB], vis_min = kend;  // keys that this lane's queries see
    Frag<f16> qf[QB][NK];
    float fq[QB];
    const int g = here(threadIdx.x) >> 4 & 3, c = here(threadIdx.x) & 15;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int slot = sb + qb * 16 + c, i = min(slot, slots - 1) / G, head = h * G + min(slot, slots - 1) % G;
      const int pos = sq.pos0 + i;
      vis[qb] = pos < 0 ? 0 : a.causal ? pos + 1 : sq.len;
      vis_min = min(vis_min, vis[qb]);
      const T *q = (const T *)a.q.p + (int64_t)(sq.row0 + i) * a.q.rs + (int64_t)head * a.q.hs;
      fq[qb] = load_query<T, NK>(qf[qb], q, g * (HD / 4), 8, a.q.vec, a.scale * kLog2e);
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) vis_min = min(vis_min, __shfl_xor(vis_min, o));

    float m[QB], l[QB];
    f32x4 acc[QB][ND];
    // V exponent byte of the accumulators' unit: M while every query sees all keys
    // of a tile, the larger of M and its query's Mq in the tiles after those
    int M = 0, Mq[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      Mq[qb] = 0;
      m[qb] = -INFINITY;
      l[qb] = 0.0f;
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[qb][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (; t < t1; t += kWaves) {
      const int k0 = t * kTile;
      f32x4 s[QB][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) s[qb][kb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const uint2 lo = f16x4_of<FMT>(cur.k[kb][2 * ks]), hi = f16x4_of<FMT>(cur.k[kb][2 * ks + 1]);
          Frag<f16> kf;
          kf.v = __builtin_bit_cast(f16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) mma16(s[qb][kb], kf, qf[qb][ks]);
        }
        if (ks & 1) __builtin_amdgcn_sched_barrier(0);  // (not all of K as f16 at once: registers)
      }
      // K's registers take the next tile's as soon as they are used, and V's
      // later: a second tile in registers would leave room for half the waves
      const int ke0 = __builtin_amdgcn_readfirstlane(cur.ke[0]), ke1 = __builtin_amdgcn_readfirstlane(cur.ke[1]);
      const int ve0 = __builtin_amdgcn_readfirstlane(cur.ve[0]), ve1 = __builtin_amdgcn_readfirstlane(cur.ve[1]);
      const float ks2[2] = {k_scale(ke0), k_scale(ke1)};
      __builtin_amdgcn_sched_barrier(0);
      load_k(cur, min(t + kWaves, t1 - 1));
      __builtin_amdgcn_sched_barrier(0);
      const bool all_seen = k0 + kTile <= vis_min;
      const int Mn = all_seen ? max(M, max(v_top(ve0), v_top(ve1))) : M;
      Frag<f16> pf[QB];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float z[2][4], mx = -INFINITY, vs[2] = {v_scale(ve0, Mn), v_scale(ve1, Mn)}, unit = v_scale(M, Mn);
        if (!all_seen) {  // a block that a query sees nothing of must not move its unit
          const int old = max(M, Mq[qb]);
          Mq[qb] = max(old, max(k0 < vis[qb] ? v_top(ve0) : 0, k0 + 16 < vis[qb] ? v_top(ve1) : 0));
          vs[0] = v_scale(ve0, Mq[qb]);
          vs[1] = v_scale(ve1, Mq[qb]);
          unit = v_scale(old, Mq[qb]);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[kb][e] = s[qb][kb][e] * ks2[kb] * fq[qb];
            if (!all_seen && k0 + kb * 16 + 4 * g + e >= vis[qb]) z[kb][e] = -INFINITY;
            mx = fmaxf(mx, z[kb][e]);
          }
        mx = query_max(mx);
        const float mn = fmaxf(m[qb], mx), ms = mn == -INFINITY ? 0.0f : mn;
        const float alpha = __builtin_amdgcn_exp2f(m[qb] - ms), ms15 = ms - 15.0f;
        m[qb] = mn;
        float p[2][4], sum = 0.0f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[kb][e] = __builtin_amdgcn_exp2f(z[kb][e] - ms15);  // 2^15 p, and l in that unit
            sum += p[kb][e];
            // (a masked key's 0 must stay 0 where the block's scale is NaN, or
            // larger than the unit)
            p[kb][e] = z[kb][e] == -INFINITY ? 0.0f : p[kb][e] * vs[kb];
          }
        l[qb] = l[qb] * alpha + sum;
        const float al = alpha * unit;
        if (__any(al != 1.0f)) {
#pragma unroll
          for (int d = 0; d < ND; ++d) acc[qb][d] *= al;
        }
        const uint4 u = make_uint4(f2h2(p[0][0], p[0][1]), f2h2(p[0][2], p[0][3]), f2h2(p[1][0], p[1][1]),
                                   f2h2(p[1][2], p[1][3]));
        pf[qb].v = __builtin_bit_cast(f16x8, u);
      }
      M = Mn;
#pragma unroll
      for (int w = 0; w < Tile::VW; ++w) {
        uint32_t a0[4] = {cur.v[0][w], cur.v[1][w], cur.v[2][w], cur.v[3][w]};
        uint32_t a1[4] = {cur.v[4][w], cur.v[5][w], cur.v[6][w], cur.v[7][w]};
        transpose4(a0);
        transpose4(a1);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const uint2 lo = f16x4_of<FMT>(a0[b]), hi = f16x4_of<FMT>(a1[b]);
          Frag<f16> vf;
          vf.v = __builtin_bit_cast(f16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) mma16(acc[qb][4 * w + b], vf, pf[qb]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      load_v(cur, min(t + kWaves, t1 - 1));
    }

    // the waves' results in LDS, in units of 1
    const int tid = here(threadIdx.x), go = tid >> 4 & 3, co = tid & 15;
    __syncthreads();  // the last block's have been read
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float up = pow2i(max(max(M, Mq[qb]) - kExpBias - 15, -126));
      float lt = l[qb] + __shfl_xor(l[qb], 16);
      lt += __shfl_xor(lt, 32);
      const int q = qb * 16 + co;
      if (go == 0) {
        s_m[wave][q] = m[qb];
        s_l[wave][q] = lt * 0x1p-15f;
      }
      // acc[i][e] is dim ND (4 g + e) + i
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < ND; i += 4) {
          const f32x4 o = {acc[qb][i][e] * up, acc[qb][i + 1][e] * up, acc[qb][i + 2][e] * up, acc[qb][i + 3][e] * up};
          *reinterpret_cast<f32x4 *>(&s_o[wave][q][ND * (4 * go + e) + i]) = o;
        }
    }
    __syncthreads();
    constexpr int CPQ = HD / 4;  // chunks of 4 dims per query
    const Parts parts = parts_of(a.ws, (int64_t)a.b.n_rows * a.Hq, nsplit, HD);
    for (int i = tid; i < 16 * QB * CPQ; i += 64 * kWaves) {
      const int q = i / CPQ, d = i % CPQ * 4, slot = sb + q;
      if (slot >= slots) break;
      float mm = s_m[0][q];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, s_m[w][q]);
      const float ms = mm == -INFINITY ? 0.0f : mm;
      float lt = 0.0f;
      f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_m[w][q] - ms);
        lt += s_l[w][q] * f;
        o += *reinterpret_cast<const f32x4 *>(&s_o[w][q][d]) * f;
      }
      const int64_t row = sq.row0 + slot / G, head = h * G + slot % G, at = row * a.Hq + head;
      if (nsplit > 1) {
        const int64_t n = (int64_t)a.b.n_rows * a.Hq;
        *reinterpret_cast<f32x4 *>(parts.o + (sp * n + at) * HD + d) = o;
        if (d == 0) {
          parts.m[sp * n + at] = mm;
          parts.l[sp * n + at] = lt;
        }
      } else {
        const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
        O *out = (O *)a.out.p + row * a.out.rs + head * a.out.hs + d;
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = from_f<O>(o[j] * inv);
        if (a.lse && d == 0) a.lse[at] = lt == 0.0f ? -INFINITY : mm * kLn2 + logf(lt);
      }
    }
  }
}

// The splits' results of a (row of a sequence, query head) joined, by W waves:
// every W-th split each, then added up in LDS. A workgroup takes NH heads.
// Rows of no sequence have no results and are left out.
template <typename O, int HD, int W, int NH>
__global__ __launch_bounds__(64 * W * NH) void qattn_join_kernel(QAttn a, int nsplit) {
  static_assert(W == 1 || NH == 1, "heads share no LDS");
  constexpr int D = HD / 64;
  __shared__ float s_o[W][HD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = wave % W;
  const int head = blockIdx.y * NH + wave / W;
  const QSeq sq = qseq(a.b, a.c, blockIdx.z);
  const int64_t n = (int64_t)a.b.n_rows * a.Hq;
  const Parts parts = parts_of(a.ws, n, nsplit, HD);
  for (int i = blockIdx.x; i < sq.n; i += gridDim.x) {
    const int64_t row = sq.row0 + i, at = row * a.Hq + head;
    float mm = -INFINITY, l = 0.0f, o[D] = {};
    if (head < a.Hq) {
      // every wave has all maxima and sums, one or two a lane (kMaxSplit 128)
      float ms[2], ls[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int s = lane + 64 * k;
        ms[k] = s < nsplit ? parts.m[s * n + at] : -INFINITY;
        ls[k] = s < nsplit ? parts.l[s * n + at] : 0.0f;
      }
      mm = warp_max(fmaxf(ms[0], ms[1]));
      const float base = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
      for (int k = 0; k < 2; ++k) ms[k] = __builtin_amdgcn_exp2f(ms[k] - base);  // the splits' weights
      l = warp_sum(ls[0] * ms[0] + ls[1] * ms[1]);
      for (int s0 = sub; s0 < nsplit; s0 += 8 * W) {  // eight splits' rows on their way at a time
        float x[8][D];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float *p = parts.o + (min(s0 + k * W, nsplit - 1) * n + at) * HD + lane * D;
#pragma unroll
          for (int d = 0; d < D; ++d) x[k][d] = p[d];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int s = min(s0 + k * W, nsplit - 1);
          const float f = s0 + k * W < nsplit ? __shfl(s < 64 ? ms[0] : ms[1], s & 63) : 0.0f;
#pragma unroll
          for (int d = 0; d < D; ++d) o[d] += f != 0.0f ? x[k][d] * f : 0.0f;
        }
      }
    }
    if constexpr (W > 1) {
      __syncthreads();
#pragma unroll
      for (int d = 0; d < D; ++d) s_o[wave][lane * D + d] = o[d];
      __syncthreads();
      if (sub) continue;
#pragma unroll
      for (int d = 0; d < D; ++d) {
        o[d] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) o[d] += s_o[w][lane * D + d];
      }
    }
    if (head >= a.Hq) continue;
    O *out = (O *)a.out.p + row * a.out.rs + head * a.out.hs + lane * D;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < D; ++d) out[d] = from_f<O>(o[d] * inv);
    if (a.lse && lane == 0) a.lse[at] = l == 0.0f ? -INFINITY : mm * kLn2 + logf(l);
  }
}

// The kernel and the splits of a launch. Query slots of a sequence and KV head
// (rows * heads of its group) up to kFewSlots take the kernel above, more take
// the one of k_qattn_rows.hip. Either wants about 512 workgroups, two on each of
// 256 CUs.
// Few slots: a split is so many keys of any sequence, so that workgroups are
// alike and a short sequence has fewer of them (3 sequences of 60000 .. 131072
// keys: 63 us, 70 with each sequence in 43 equal parts). 512 keys at least, two
// tiles a wave, and no split up to 1024 keys, where the joining costs more (one
// question's 731 keys 13.1 us with two splits, 10.9 with one). No more than 6144
// keys, or the longest sequences end alone: 16 of 65536 .. 131072 keys 633 us in 4
// splits, 584 in 16, 569 in 24; but 64 of 1024 .. 4096 keys 73 us in one, 81 in
// four.
// Many slots: a row's keys in equal parts, so many that they take the fewest
// rounds of 512 workgroups (of 256 where only one fits on a CU) over the keys of
// one, each workgroup counted as 512 keys longer than it is (its queries, its
// results and their joining): 4 x 256 rows of 40 heads over 4096 .. 8192 keys, 160
// workgroups of eight waves a split, take 302 us in one, 248 in 2 (two rounds, the
// second a quarter full), 203 in 3, 225 in 4; 16 x 64 slots over 8192 keys, 128
// workgroups of four waves, 113 in 2, 100 in 3, 82 in 4, 103 in 5.
constexpr int64_t kFewSlots = 32, kLeastKeys = 512, kMostKeys = 6144, kFill = 512;
struct Plan {
  bool few;
  int nsplit;
  int64_t keys;  // of a split (few slots)
};
// Query slots of a workgroup: 32 where a sequence has more than 16 (head_dim 256
// has no registers for them, and reads its keys again).
static int few_block(int hd, int64_t slots) { return slots > 16 && hd < 256 ? 32 : 16; }
static Plan plan_of(const QCache &c, const QBatch &b, int Hq) {
  const int64_t slots = (int64_t)std::max(b.max_rows, 1) * (Hq / c.H);
  const int64_t len = std::min(std::max<int64_t>(b.max_len, 1), (int64_t)1 << 30);
  const bool few = slots <= kFewSlots;
  const int64_t block = few ? few_block(c.hd, slots) : qattn_rows_block(c.hd, slots);
  const int64_t units = (int64_t)std::max(b.n_seq, 1) * c.H * ((slots + block - 1) / block);
  const int64_t most = std::min<int64_t>((len + kLeastKeys - 1) / kLeastKeys, kMaxSplit);
  if (few) {
    int64_t n = 1;
    if (len > 2 * kLeastKeys)
      n = std::min(most, std::max((kFill + units - 1) / units, (len + kMostKeys - 1) / kMostKeys));
    const int64_t step = kTile * kWaves, keys = ((len + n - 1) / n + step - 1) / step * step;
    return {few, (int)((len + keys - 1) / keys), keys};
  }
  // (of eight waves, or 128 KB of LDS: one workgroup a CU)
  const int64_t fill = block == 256 || c.hd == 256 ? kFill / 2 : kFill;
  double best = INFINITY;  // (whole numbers of 64 bits could overflow)
  int64_t at = 1;
  for (int64_t n = 1; n <= most; ++n) {
    const double cost = (double)((units * n + fill - 1) / fill) * (double)((len + n - 1) / n + kLeastKeys);
    if (cost < best) {
      best = cost;
      at = n;
    }
  }
  return {few, (int)at, 0};
}

int64_t qattn_workspace(const QCache &c, const QBatch &b, int Hq) {
  const int n = plan_of(c, b, Hq).nsplit;
  return n == 1 ? 0 : (int64_t)b.n_rows * Hq * n * (c.hd + 2) * 4;
}

// One wave for each (row, head) of few splits, four of them a workgroup (4 x 256
// rows of 40 heads, 3 splits: 27 us, 49 with four waves each); eight where there
// are many splits to read.
template <typename O, int HD> static hipError_t run_join(const QAttn &a, int nsplit, hipStream_t st) {
  const unsigned rows = (unsigned)std::min(std::max(a.b.max_rows, 1), 65536), n_seq = (unsigned)a.b.n_seq;
  if (nsplit <= 8)
    hipLaunchKernelGGL((qattn_join_kernel<O, HD, 1, 4>), dim3(rows, (a.Hq + 3) / 4, n_seq), dim3(256), 0, st, a, nsplit);
  else
    hipLaunchKernelGGL((qattn_join_kernel<O, HD, 8, 1>), dim3(rows, a.Hq, n_seq), dim3(512), 0, st, a, nsplit);
  return hipGetLastError();
}

template <typename T, typename O, int FMT, int HD, int QB>
static hipError_t run_few_qb(const QAttn &a, const Plan &p, hipStream_t st) {
  const int64_t slots = (int64_t)std::max(a.b.max_rows, 1) * (a.Hq / a.c.H), blocks = (slots + 16 * QB - 1) / (16 * QB);
  hipLaunchKernelGGL((qattn_split_kernel<T, O, FMT, HD, QB>), dim3((unsigned)(blocks * p.nsplit), a.c.H, a.b.n_seq),
                     dim3(64 * kWaves), 0, st, a, p.nsplit, (int)(p.keys / kTile));
  return hipGetLastError();
}
template <typename T, typename O, int FMT, int HD>
static hipError_t run_few(const QAttn &a, const Plan &p, hipStream_t st) {
  if constexpr (HD < 256) {
    if (few_block(HD, (int64_t)std::max(a.b.max_rows, 1) * (a.Hq / a.c.H)) == 32)
      return run_few_qb<T, O, FMT, HD, 2>(a, p, st);
  }
  return run_few_qb<T, O, FMT, HD, 1>(a, p, st);
}

template <typename T, typename O, int FMT, int HD> static hipError_t run_hd(const QAttn &a, hipStream_t st) {
  const Plan p = plan_of(a.c, a.b, a.Hq);
  const hipError_t e = p.few ? run_few<T, O, FMT, HD>(a, p, st) : launch_qattn_rows(a, p.nsplit, st);
  return e != hipSuccess || p.nsplit == 1 ? e : run_join<O, HD>(a, p.nsplit, st);
}
template <typename T, typename O, int FMT> static hipError_t run_fmt(const QAttn &a, hipStream_t st) {
  if (a.c.hd == 64) return run_hd<T, O, FMT, 64>(a, st);
  if (a.c.hd == 128) return run_hd<T, O, FMT, 128>(a, st);
  return run_hd<T, O, FMT, 256>(a, st);
}
template <typename T, typename O> static hipError_t run_types(const QAttn &a, hipStream_t st) {
  return a.c.fmt == 0 ? run_fmt<T, O, 0>(a, st) : run_fmt<T, O, 1>(a, st);
}

hipError_t launch_qattn(const QAttn &a, hipStream_t st) {
  if (a.b.n_seq <= 0 || a.b.n_rows <= 0) return hipSuccess;
  if (a.q.type == 1) return a.out.type == 0 ? run_types<f16, float>(a, st) : run_types<f16, f16>(a, st);
  return a.out.type == 0 ? run_types<bf16, float>(a, st) : run_types<bf16, bf16>(a, st);
}

}  // namespace jetk
