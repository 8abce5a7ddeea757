// Attention over a cache held in 8 bits, many query slots: see qattn.h for the
// arithmetic. A workgroup of four or eight waves takes 16 QB query slots a wave
// of one (sequence, KV head); tiles of 64 keys are turned into f16 once for all
// of them on their way into LDS (two stages: while one is computed the next one
// is converted and the one after it loaded into registers), so that per key
// tile and wave the conversion is a quarter or an eighth of what it would be in
// the waves' own registers, where it costs more than the products.
// What bounds it: 4 x 256 rows of 40 heads (8 KV heads of 128) over 4096 .. 8192
// keys take 204 us (0.59 PFLOP/s; a large library product of f16 reaches 1.15), of
// which the vector instructions of the softmax and the conversion (400 a tile and
// wave of 32 queries) are about 93 us, the matrix instructions 48 and the LDS
// reads of K and V 48: two waves a SIMD hide little of one behind the other.
// (Half of the waves converting after their products instead of before: 227 us;
// wave priorities for the products, or for the softmax: 204; 16 queries a wave and
// four waves a SIMD, which read K and V twice as often from LDS: 202.)
// With own rows (candidate scoring) the keys of a query's own candidate follow
// as 16-bit tiles of the same stream; there no split is made and every query
// runs the same operations in the same order whatever block it lies in. (28
// layers' scoring of 256 questions, 4 candidates each, 12 heads on 2 KV heads:
// 3.5 ms, where attention over f16 prefixes takes 3.0.)
#include <algorithm>
#include <type_traits>

#include "gemm_core.h"
#include "qattn.h"

namespace jetk {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

// A row's maximum is brought up to date when it lags by 2^8, and probabilities
// are kept as p 2^7 <= 2^15. The largest p of a row is then seldom a power of two
// and takes f16's rounding like the others: for 4 x 256 rows over 4096 .. 8192
// keys, outputs are off by 1.1e-4 (2-norm) before their own rounding, 2.3e-4 after
// it in f16. With every maximum taken at once: 3.4e-5 and 2.1e-4, in 2.5% more time.
constexpr float kLag = 8.0f;
constexpr int kUnit = 7;

// Work of a launch: units (sequence, KV head) of `per` workgroups each. The
// workgroups of a unit run on one XCD (they share its keys in that L2), which
// deals workgroup w to XCD w % 8.
struct Work {
  int64_t unit;
  int part;
};
__device__ __forceinline__ Work work_of(int64_t w, int64_t units, int per) {
  const int64_t even = units / 8 * 8 * per;
  if (w >= even) return {units / 8 * 8 + (w - even) / per, (int)((w - even) % per)};
  return {w / 8 / per * 8 + w % 8, (int)(w / 8 % per)};
}

template <typename T, typename O, int FMT, int HD, int QB, bool OWN, int NW>
__global__ __launch_bounds__(64 * NW, HD == 256 && NW == 4 ? 1 : 2) void qattn_rows_kernel(QAttn a, OwnRows own, int blocks,
                                                                           int nsplit) {
  constexpr int KT = 64, NT = 64 * NW, BLOCK = 16 * QB * NW, NK = HD / 32, ND = HD / 16;
  constexpr int RB = HD * 2, CPR = HD / 8;                // bytes and 16-byte chunks of an f16 row
  constexpr int PLANE = KT * RB, STAGE = 2 * PLANE;       // K, then V
  constexpr int RC = HD / 16, LD = KT * RC / NT;   // 16-byte chunks of an 8-bit row, and a thread's of a tile
  extern __shared__ __align__(1024) char smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
  const int G = a.Hq / a.c.H, lb = a.c.lb;
  const int64_t units = OWN ? own.n_items : (int64_t)a.b.n_seq * a.c.H;
  const int per = OWN ? 1 : blocks * nsplit;

  // chunk c of row r lies at c ^ kswz(r) (K: the 16 rows of a fragment read) or
  // c ^ vswz(r) (V: the rows of a transposed read)
  auto kswz = [](int r) { return r & (CPR < 16 ? CPR - 1 : 15); };
  auto vswz = [](int r) { return (r & (CPR < 16 ? 3 : 7)) << 1; };

  for (int64_t w = blockIdx.x; w < units * per; w += gridDim.x) {
    // this workgroup's sequence, KV head, rows and keys
    int h, sp = 0, sb0 = 0, row0, rows, pos0, len;
    int64_t slot0;
    int it_slots = 0, npre_item = 0;
    AttnItem it{};
    if constexpr (OWN) {
      it = own.items[w];
      h = it.kvh;
      row0 = own.qs.qrow0[it.q];
      rows = own.qs.nrows[it.q];
      slot0 = own.qs.pre_slot0[it.q];
      len = own.qs.pre_len[it.q];
      pos0 = len;  // (every row sees the whole prefix)
      sb0 = it.slot0;
      it_slots = it.slot0 + it.nslots;
    } else {
      const Work x = work_of(w, units, per);
      h = (int)(x.unit % a.c.H);
      sp = x.part % nsplit;
      sb0 = x.part / nsplit * BLOCK;
      const QSeq sq = qseq(a.b, a.c, (int)(x.unit / a.c.H));
      row0 = sq.row0;
      rows = sq.n;
      slot0 = sq.slot0;
      len = sq.len;
      pos0 = sq.pos0;
    }
    const int64_t base = ((int64_t)h * a.c.S + slot0) * HD, ebase = (int64_t)h * (a.c.S >> lb) + (slot0 >> lb);
    const uint8_t *K = a.c.k + base, *V = a.c.v + base, *KE = a.c.ke + ebase, *VE = a.c.ve + ebase;
    const int slots = OWN ? it_slots : rows * G;

    for (int sb = sb0; sb < slots; sb += OWN ? slots : blocks * BLOCK) {
      const int tid = here(threadIdx.x), lane = tid & 63, g = lane >> 4, l16 = lane & 15;
      const int r_last = (min(sb + BLOCK, slots) - 1) / G;  // last row of the block, in the sequence
      const int kend = OWN || !a.causal ? len : max(0, pos0 + r_last + 1);
      const int tps = ((kend + KT - 1) / KT + nsplit - 1) / nsplit;
      const int key0 = sp * tps * KT, key1 = min(kend, (sp + 1) * tps * KT);

      // The stream of key tiles: the cache's (cs < 0), then for every candidate
      // with rows in the block (first body row cs) its rows up to the block's
      // last one, in tiles that start at cs. nk = 0 past the end.
      struct Tile {
        int cs, t0, nk;
      };
      const int r_first = row0 + sb / G, r_end = row0 + r_last;
      int cs_first = 0, n_a = 1, n_b = 1;
      if constexpr (OWN) {
        cs_first = r_first - own.row_t[r_first] + 1;
        n_a = own.row_n[min(r_first + lane, r_end)];
        n_b = own.row_n[min(r_first + 64 + lane, r_end)];
      }
      auto own_n = [&](int cs) {  // body rows of the candidate that starts at row cs
        const int i = max(cs, r_first) - r_first;
        return i >= 64 ? __builtin_amdgcn_readlane(n_b, i - 64) : __builtin_amdgcn_readlane(n_a, i);
      };
      auto own_tile = [&](int cs, int ts) {
        if (cs > r_end) return Tile{0, 0, 0};
        return Tile{cs, ts, min(KT, min(cs + own_n(cs) - 1, r_end) - ts + 1)};
      };
      auto next_tile = [&](const Tile &t) {
        if (t.nk == 0) return t;
        if (!OWN || t.cs < 0) {
          const int kb = t.t0 + KT;
          if (kb < key1) return Tile{-1, kb, min(KT, key1 - kb)};
          if constexpr (OWN) return own_tile(cs_first, cs_first);
          return Tile{0, 0, 0};
        }
        const int n = own_n(t.cs);
        if (t.t0 + KT <= min(t.cs + n - 1, r_end)) return own_tile(t.cs, t.t0 + KT);
        return own_tile(t.cs + n, t.cs + n);
      };

      // 8-bit rows of a tile into registers, one after another as they lie (past
      // its end: its last 16 bytes), and the tile's scale bytes: lane l (mod 8)
      // the one of K (l < 4) or V of keys 16 (l mod 4) ..
      uint4 rk[LD], rv[LD];
      int re = 0;
      const uint8_t *scales = lane & 4 ? VE : KE;
      auto load = [&](const Tile &t) {
        const uint8_t *kt = K + (int64_t)t.t0 * HD, *vt = V + (int64_t)t.t0 * HD;
#pragma unroll
        for (int i = 0; i < LD; ++i) {
          const uint32_t at = min((i * NT + (int)threadIdx.x) * 16, t.nk * HD - 16);
          rk[i] = ld16(kt + at);
          rv[i] = ld16(vt + at);
        }
        re = scales[(t.t0 + min((here(threadIdx.x) & 3) * 16, t.nk - 1)) >> lb];
      };
      // ... and from there into a stage. (A thread's next chunk lies 16 NT / HD
      // rows on, where the swizzle is the same; chunks c and c + 1 of its 16
      // values are neighbours in the swizzle too.)
      auto store = [&](int stage) {
        const int tid = here(threadIdx.x), r = tid / RC, c = tid % RC * 2;
        const uint32_t at = lds0 + stage * STAGE + r * RB;
        const uint32_t ka = at + ((c ^ kswz(r)) << 4), va = at + PLANE + ((c ^ vswz(r)) << 4);
#pragma unroll
        for (int i = 0; i < LD; ++i) {
          auto put = [&](uint32_t to, const uint4 &u) {
            const uint2 p = f16x4_of<FMT>(u.x), q = f16x4_of<FMT>(u.y), s = f16x4_of<FMT>(u.z), t = f16x4_of<FMT>(u.w);
            *(lds_u32x4 *)(uintptr_t)(to + i * (NT * 16 / HD) * RB) = u32x4{p.x, p.y, q.x, q.y};
            *(lds_u32x4 *)(uintptr_t)((to ^ 16) + i * (NT * 16 / HD) * RB) = u32x4{s.x, s.y, t.x, t.y};
          };
          put(ka, rk[i]);
          put(va, rv[i]);
        }
      };
      // 16-bit rows of an own tile straight into a stage
      auto load_own = [&](const Tile &t, int stage) {
        constexpr int RPL = 64 / CPR;  // rows of a wave's load
        char *dst = smem + stage * STAGE;
        const f16 *Ko = (const f16 *)own.K + (int64_t)h * own.s_suf * HD, *Vo = (const f16 *)own.V + (int64_t)h * own.s_suf * HD;
#pragma unroll
        for (int i = 0; i < KT / RPL / NW; ++i) {
          const int blk = i * NW + wave, r = blk * RPL + lane / CPR, c = lane % CPR;
          const int64_t off = (int64_t)(t.t0 + min(r, t.nk - 1)) * HD;
          __builtin_amdgcn_global_load_lds((const void *)(Ko + off + (c ^ kswz(r)) * 8), (lds_void *)(dst + blk * 1024),
                                           16, 0, 0);
          __builtin_amdgcn_global_load_lds((const void *)(Vo + off + (c ^ vswz(r)) * 8),
                                           (lds_void *)(dst + PLANE + blk * 1024), 16, 0, 0);
        }
      };

      Tile cur = key0 < key1 ? Tile{-1, key0, min(KT, key1 - key0)} : Tile{0, 0, 0};
      if (OWN && cur.nk == 0) cur = own_tile(cs_first, cs_first);
      if (cur.nk > 0 && cur.cs < 0) load(cur);

      int row[QB], vis[QB], first[QB], vis_min = kend;
      Frag<f16> qf[QB][NK];
      float fq[QB], m[QB], l[QB];
      f32x4 acc[QB][ND];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int s = sb + (wave * QB + qb) * 16 + l16;
        const int i = (s < slots ? s : sb) / G, head = h * G + (s < slots ? s : sb) % G, pos = pos0 + i;
        row[qb] = row0 + i;
        vis[qb] = OWN ? len : pos < 0 ? 0 : a.causal ? pos + 1 : len;
        vis_min = min(vis_min, vis[qb]);
        first[qb] = OWN && s < slots ? row[qb] - own.row_t[row[qb]] + 1 : -1;
        const T *q = (const T *)a.q.p + (int64_t)row[qb] * a.q.rs + (int64_t)head * a.q.hs;
        fq[qb] = load_query<T, NK>(qf[qb], q, g * 8, 32, a.q.vec, a.scale * kLog2e);
        m[qb] = -INFINITY;
        l[qb] = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[qb][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) vis_min = min(vis_min, __shfl_xor(vis_min, o));
      const bool idle = sb + wave * QB * 16 >= slots;  // no query: loads and barriers only
      // V exponent byte of the accumulators' unit: M, the largest of the blocks so
      // far, while every query sees every block; where a query does not, 2^low less
      // (0 in all tiles but a causal call's last ones). udown = 2^-low.
      int M = 0;
      float low[QB], udown[QB];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) low[qb] = 0.0f, udown[qb] = 1.0f;

      int ec = re, stage = 0;  // the current tile's scale bytes
      __syncthreads();         // the block before is done with the stages
      if (cur.nk > 0) {
        if (!OWN || cur.cs < 0) store(0);
        else if constexpr (OWN) load_own(cur, 0);
      }
      Tile ahead = next_tile(cur);
      if (ahead.nk > 0 && ahead.cs < 0) load(ahead);
      // One tile. ALL: a whole one that every query of the workgroup sees all of
      // (with the other tiles' cases in the same code those cost 2 to 4%).
      auto step = [&](auto all) __attribute__((always_inline)) {
        constexpr bool ALL = decltype(all)::value;
        if constexpr (OWN) wait_vmcnt<0>();  // (own tiles are loaded into LDS directly)
        __syncthreads();                     // this tile is in place, and every wave is done with the other stage
        const int ea = re;
        Tile after = ahead;
        if (ahead.nk > 0) {
          if (!OWN || ahead.cs < 0) store(stage ^ 1);
          else if constexpr (OWN) load_own(ahead, stage ^ 1);
          after = next_tile(ahead);
          if constexpr (OWN) {
            if (after.nk > 0 && after.cs < 0) load(after);
          } else {
            load(after.nk > 0 ? after : ahead);  // (at the end the last tile again: no branch, no wait for it)
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (!idle) {
          const int lane = here(threadIdx.x) & 63, g = lane >> 4, l16 = lane & 15;
          // chunk 4 ks + g of key l16; the rest of a fragment's address is in its
          // offset (stages and rows are powers of two: bits of ks flip in place)
          const uint32_t ka = lds0 + stage * STAGE + l16 * RB + ((g ^ kswz(l16)) << 4);
          // V transposed on the way out of LDS: lane l supplies 4 elements of
          // key 4 g + (l % 16) / 4 and receives keys 4 g .. + 3 of dim l % 16
          const int vr = 4 * g + (l16 >> 2);  // (16 and 32 rows on have the same swizzle)
          const uint32_t va = lds0 + stage * STAGE + PLANE + vr * RB + (((l16 >> 1 & 1) ^ vswz(vr)) << 4) + (l16 & 1) * 8;
          const bool pre = !OWN || cur.cs < 0;
          f32x4 s[QB][4];
          auto read_k = [&](int ks, int kb) {
            return *(const lds_u32x4 *)(uintptr_t)((ka ^ (ks << 6)) + kb * 16 * RB);
          };
          auto score = [&](int ks, int kb, u32x4 u) {
            Frag<f16> f;
            f.v = __builtin_bit_cast(f16x8, u);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
              if (ks == 0) s[qb][kb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
              mma16(s[qb][kb], f, qf[qb][ks]);
            }
          };
          // fragments are read one group of products ahead, and no further (the
          // compiler would hold them all in registers)
          if (ALL || cur.nk > 48) {
            u32x4 f[2][4];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) f[0][kb] = read_k(0, kb);
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
              if (ks + 1 < NK) {
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) f[(ks + 1) & 1][kb] = read_k(ks + 1, kb);
              }
#pragma unroll
              for (int kb = 0; kb < 4; ++kb) score(ks, kb, f[ks & 1][kb]);
              __builtin_amdgcn_sched_barrier(0);
            }
          } else {
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
              if (kb < 3 && kb * 16 < cur.nk) {
#pragma unroll
                for (int ks = 0; ks < NK; ++ks) score(ks, kb, read_k(ks, kb));
              } else {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) s[qb][kb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
              }
            }
          }
          int ve[4], Mn = M;
          float ks2[4];
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) {
            // (own rows are as they are: scale 1)
            ks2[kb] = pre ? k_scale(__builtin_amdgcn_readlane(ec, kb)) : 1.0f;
            ve[kb] = pre ? __builtin_amdgcn_readlane(ec, 4 + kb) : kExpBias;
            Mn = max(Mn, v_top(ve[kb]));
          }
          // V's scales, in units of 2^(Mn - 127), and whether all lie so close
          // together that a probability may take them along (none NaN)
          float vs[4];
          bool near = true;
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) {
            vs[kb] = v_scale(ve[kb], Mn);
            near = near && vs[kb] >= 0x1p-60f;
          }
          const bool grown = Mn != M;
          const float unit = v_scale(M, Mn);
          const int M0 = M;
          M = Mn;
          const bool seen = ALL || (pre && cur.t0 + KT <= min(vis_min, key1));  // every key of the tile by every query
          Frag<f16> pf[QB][2];
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) {
            // z = s f, the largest z, and p = 2^(z - m): where all keys are
            // seen z itself is not needed (f >= 0: largest z from largest s)
            float f[4], mx = -INFINITY, un = unit;
            bool turn = false;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) f[kb] = ks2[kb] * fq[qb];
            if (seen) {
#pragma unroll
              for (int kb = 0; kb < 4; ++kb)
                mx = fmaxf(mx, f[kb] * fmaxf(fmaxf(s[qb][kb][0], s[qb][kb][1]), fmaxf(s[qb][kb][2], s[qb][kb][3])));
            } else {
              // last key of the tile that the query sees: the prefix's, or the
              // query's own row of its candidate's tile
              const int last = pre ? min(cur.nk, vis[qb] - cur.t0) - 1
                                   : (first[qb] == cur.cs ? min(cur.nk - 1, row[qb] - cur.t0) : -1);
#pragma unroll
              for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float z = kb * 16 + 4 * g + e <= last ? s[qb][kb][e] * f[kb] : -INFINITY;
                  s[qb][kb][e] = z;
                  mx = fmaxf(mx, z);
                }
                f[kb] = 1.0f;
              }
              // blocks that the query sees nothing of must not move its unit (with
              // own rows all see the same blocks)
              if constexpr (!OWN) {
                const int old = M0 - (int)low[qb];
                int top = old;
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
                  if (kb * 16 <= last) top = max(top, v_top(ve[kb]));
                un = v_scale(old, top);
                turn = top != old;
                low[qb] = (float)(M - top);
                udown[qb] = pow2i(max(top - M, -126));
              }
            }
            mx = query_max(mx);
            // the accumulators are rescaled when some query's maximum lags too
            // far behind (or their unit grew), not whenever one moves; each query
            // by its own maximum alone, whatever the others in its wave do
            const bool lags = mx > m[qb] + kLag;
            if (grown || __any(turn || lags)) {
              const float mn = lags ? mx : m[qb];
              const float al = lags ? __builtin_amdgcn_exp2f(m[qb] - mn) : 1.0f;
              m[qb] = mn;
              l[qb] *= al;
#pragma unroll
              for (int d = 0; d < ND; ++d) acc[qb][d] *= al * un;
            }
            const float m0 = m[qb] == -INFINITY ? 0.0f : m[qb];
            float p[4][4], sum = 0.0f;
            if (near) {
              // p' = 2^(z - m + log2 vs), and l adds it up in p's own unit (the
              // exponent's rounding, 2^-24 |m|, is in both alike)
              const float ms = m0 - ((ALL ? 0.0f : low[qb]) + (float)kUnit);
#pragma unroll
              for (int kb = 0; kb < 4; ++kb) {
                const float mk = ms - (float)(ve[kb] - Mn);
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  p[kb][e] = __builtin_amdgcn_exp2f(fmaf(s[qb][kb][e], f[kb], -mk));
                  part += p[kb][e];
                }
                sum = fmaf(part, pow2i(Mn - ve[kb]), sum);
              }
              l[qb] = ALL ? l[qb] + sum : fmaf(sum, udown[qb], l[qb]);
            } else {
              const float ms = m0 - (float)kUnit;
#pragma unroll
              for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float x = __builtin_amdgcn_exp2f(fmaf(s[qb][kb][e], f[kb], -ms));
                  sum += x;
                  // (a masked key's 0 must stay 0 where the scale is NaN, or
                  // larger than the unit)
                  p[kb][e] = !seen && s[qb][kb][e] == -INFINITY ? 0.0f : x * v_scale(ve[kb], ALL ? M : M - (int)low[qb]);
                }
              l[qb] += sum;
            }
#pragma unroll
            for (int mm = 0; mm < 2; ++mm) {
              const uint4 u = make_uint4(f2h2(p[2 * mm][0], p[2 * mm][1]), f2h2(p[2 * mm][2], p[2 * mm][3]),
                                         f2h2(p[2 * mm + 1][0], p[2 * mm + 1][1]), f2h2(p[2 * mm + 1][2], p[2 * mm + 1][3]));
              pf[qb][mm].v = __builtin_bit_cast(f16x8, u);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
          for (int mm = 0; mm < 2; ++mm) {
            if (!ALL && mm * 32 >= cur.nk) continue;
            auto read_v = [&](int d, int half) {
              return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (lds_s16x4 *)(uintptr_t)((va ^ (d << 5)) + (mm * 32 + half * 16) * RB));
            };
            constexpr int DB = 4;
            s16x4 f[2][DB][2];
#pragma unroll
            for (int d = 0; d < DB; ++d) f[0][d][0] = read_v(d, 0), f[0][d][1] = read_v(d, 1);
#pragma unroll
            for (int d0 = 0; d0 < ND; d0 += DB) {
              if (d0 + DB < ND) {
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                  f[(d0 / DB + 1) & 1][d][0] = read_v(d0 + DB + d, 0);
                  f[(d0 / DB + 1) & 1][d][1] = read_v(d0 + DB + d, 1);
                }
              }
#pragma unroll
              for (int d = 0; d < DB; ++d) {
                Frag<f16> v;
                v.v = __builtin_bit_cast(f16x8, __builtin_shufflevector(f[d0 / DB & 1][d][0], f[d0 / DB & 1][d][1], 0, 1,
                                                                        2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) mma16(acc[qb][d0 + d], v, pf[qb][mm]);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        }
        ec = ea;
        cur = ahead;
        ahead = after;
        stage ^= 1;
      };
      if constexpr (!OWN) {
        const int pos = pos0 + sb / G;  // of the block's first row
        const int seen_by_all = pos < 0 ? 0 : a.causal ? min(key1, pos + 1) : key1;
        while (cur.nk > 0 && cur.t0 + KT <= seen_by_all) step(std::true_type{});
      }
      while (cur.nk > 0) step(std::false_type{});

      {
      const int lane = here(threadIdx.x) & 63, g = lane >> 4, l16 = lane & 15;
      const int64_t n = (int64_t)a.b.n_rows * a.Hq;
      const Parts parts = parts_of(a.ws, n, nsplit, HD);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float lt = l[qb] + __shfl_xor(l[qb], 16);
        lt += __shfl_xor(lt, 32);
        lt *= pow2i(-kUnit);
        const float up = pow2i(max(M - (int)low[qb] - kExpBias - kUnit, -126));
        const int s = sb + (wave * QB + qb) * 16 + l16, head = h * G + s % G;
        if (s >= slots) continue;
        const int64_t row = row0 + s / G, at = row * a.Hq + head;
        if (!OWN && nsplit > 1) {
          float *o = parts.o + (sp * n + at) * HD + 4 * g;
#pragma unroll
          for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4 *>(o + 16 * d) = acc[qb][d] * up;
          if (g == 0) {
            parts.m[sp * n + at] = m[qb];
            parts.l[sp * n + at] = lt;
          }
          continue;
        }
        const float inv = lt == 0.0f ? 0.0f : up / lt;
        O *o = (O *)a.out.p + row * a.out.rs + (int64_t)head * a.out.hs + 4 * g;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const f32x4 x = acc[qb][d] * inv;
          if (a.out.vec) {
            if constexpr (sizeof(O) == 2)
              *reinterpret_cast<uint2 *>(o + 16 * d) = make_uint2(pack2<O>(x[0], x[1]), pack2<O>(x[2], x[3]));
            else *reinterpret_cast<f32x4 *>(o + 16 * d) = x;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[16 * d + e] = from_f<O>(x[e]);
          }
        }
        if (a.lse && g == 0) a.lse[at] = lt == 0.0f ? -INFINITY : m[qb] * kLn2 + logf(lt);
      }
      }
    }
  }
}

// Query slots of a workgroup: 64 where no sequence has more (all four waves have
// queries then: 8 KV heads, 16 sequences of 64 slots and 8192 keys, 113 us with
// blocks of 128, 91 with 64); from 256 on 256 in eight waves, which convert half
// as many keys each (4 x 256 rows of 40 heads over 4096 .. 8192 keys: 216 us, 203
// with 256). Of head_dim 256 half as many, a wave has registers for 16 queries; of
// head_dim 64 no more than 128, a tile is one load of four waves.
int qattn_rows_block(int hd, int64_t slots) {
  if (hd == 256) return slots < 128 ? 64 : 128;
  return slots <= 64 ? 64 : slots < 256 || hd == 64 ? 128 : 256;
}

template <typename T, typename O, int FMT, int HD, int QB, bool OWN, int NW>
static hipError_t run_rows(const QAttn &a, const OwnRows &own, int nsplit, hipStream_t st) {
  constexpr int lds = 2 * 2 * 64 * HD * 2, BLOCK = 16 * QB * NW;
  const auto kernel = qattn_rows_kernel<T, O, FMT, HD, QB, OWN, NW>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  const int64_t slots = (int64_t)std::max(a.b.max_rows, 1) * (a.Hq / a.c.H);
  const int blocks = (int)std::min<int64_t>((slots + BLOCK - 1) / BLOCK, 1 << 20);
  const int64_t total = OWN ? own.n_items : (int64_t)a.b.n_seq * a.c.H * blocks * nsplit;
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(total, 1 << 20)), dim3(64 * NW), lds, st, a, own, blocks,
                     nsplit);
  return hipGetLastError();
}

template <typename T, typename O, int FMT, int HD>
static hipError_t rows_block(const QAttn &a, int nsplit, hipStream_t st) {
  const int block = qattn_rows_block(HD, (int64_t)std::max(a.b.max_rows, 1) * (a.Hq / a.c.H));
  if constexpr (HD == 256) {
    return block == 64 ? run_rows<T, O, FMT, HD, 1, false, 4>(a, {}, nsplit, st)
                       : run_rows<T, O, FMT, HD, 1, false, 8>(a, {}, nsplit, st);
  } else {
    if (block == 64) return run_rows<T, O, FMT, HD, 1, false, 4>(a, {}, nsplit, st);
    if constexpr (HD == 128)
      if (block == 256) return run_rows<T, O, FMT, HD, 2, false, 8>(a, {}, nsplit, st);
    return run_rows<T, O, FMT, HD, 2, false, 4>(a, {}, nsplit, st);
  }
}
template <typename T, typename O, int FMT>
static hipError_t rows_hd(const QAttn &a, int nsplit, hipStream_t st) {
  if (a.c.hd == 64) return rows_block<T, O, FMT, 64>(a, nsplit, st);
  if (a.c.hd == 128) return rows_block<T, O, FMT, 128>(a, nsplit, st);
  return rows_block<T, O, FMT, 256>(a, nsplit, st);
}
template <typename T, typename O> static hipError_t rows_fmt(const QAttn &a, int nsplit, hipStream_t st) {
  return a.c.fmt == 0 ? rows_hd<T, O, 0>(a, nsplit, st) : rows_hd<T, O, 1>(a, nsplit, st);
}

hipError_t launch_qattn_rows(const QAttn &a, int nsplit, hipStream_t st) {
  if (a.q.type == 1) return a.out.type == 0 ? rows_fmt<f16, float>(a, nsplit, st) : rows_fmt<f16, f16>(a, nsplit, st);
  return a.out.type == 0 ? rows_fmt<bf16, float>(a, nsplit, st) : rows_fmt<bf16, bf16>(a, nsplit, st);
}

template <int FMT, int HD> static hipError_t run_own(const QAttn &a, const OwnRows &own, hipStream_t st) {
  if (own.block == 64) return run_rows<f16, f16, FMT, HD, 1, true, 4>(a, own, 1, st);
  if (own.block == 128) return run_rows<f16, f16, FMT, HD, 2, true, 4>(a, own, 1, st);
  return hipErrorInvalidValue;
}

hipError_t launch_qattn_own(const QAttn &a, const OwnRows &own, hipStream_t st) {
  if (own.n_items <= 0) return hipSuccess;
  if (a.q.type != 1 || a.out.type != 1) return hipErrorInvalidValue;
  if (a.c.hd == 64) return a.c.fmt == 0 ? run_own<0, 64>(a, own, st) : run_own<1, 64>(a, own, st);
  if (a.c.hd == 128) return a.c.fmt == 0 ? run_own<0, 128>(a, own, st) : run_own<1, 128>(a, own, st);
  return hipErrorInvalidValue;
}

}  // namespace jetk
