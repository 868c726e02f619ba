// Tree attention over a 4-bit prefix and the tree's bf16 rows, and the
// accumulated attention weights of the accepted nodes.
//
// Rows.  The heads that share a kv head read the same keys, so a kv head's
// rows are tree row x head, r = t G + a (a < G), in 16-row tiles.
//
// Products (v_mfma_f32_16x16x32_bf16; layouts as in the bf16 attention): S^T =
// K Q^T with the 32 keys of a block as two 16-row A operands, O^T += V^T P^T
// with 16 dims as the A operand.  A code word is one lane's 8 elements of an A
// operand; it enters as x = (16 + c) / 2, exact in bfloat16 (kvq_expand), and
// scale and zero are applied outside the products in float32:
//   S[k][q] = sum_g 2 s_kg (sum_d x_kd q_d) + (z_kg - 16 s_kg) (sum_d q_d)
//   O[d][q] = sum_k x_kd (2 s_kg P_kq) + sum_k (z_kg - 16 s_kg) P_kq
// over the 64-dim groups g, so a held value is never rounded.  A block's
// parameters go through a wave's own LDS, from which every lane reads those of
// its 8 keys.
//
// Work decomposition.  A workgroup takes a sequence, a kv head, up to 128 rows
// and one of KS key splits; its eight waves are QW side by side over tiles, NQ
// tiles each, and PARS over blocks, with no barrier in the loop: codes go
// straight into the registers of the wave that multiplies them, the next block
// requested while one is multiplied.  (NQ, QW, PARS) by the tiles of a kv head:
// (1, 1, 8) for one, (2, 1, 8) for two, (2, 2, 4) up to four, (2, 4, 2) beyond:
// two tiles share a block's expansion and parameters.  (The rule looks at tiles
// alone.  32 heads, 64 nodes, one tile a wave and two, both launches: 32768
// positions 110 and 89 us, 8192 36.2 and 33.8, but 4096 23.3 and 24.2, 2048 16.7
// and 19.6.)  Queries of two tiles a wave lie in
// LDS, their registers hold the sums.  Splits: as many as fill the compute
// units; a second launch adds them in order.
//
// Bounds.  A block takes 345 vector instructions for one tile (112 of them the
// expansion), about 280 a tile for two, 24 or 32 matrix instructions: with small
// trees that and the stream are near each other, with large ones the vector unit
// is the bound.  us a launch under the profiler (+ the launch that adds splits): 32
// heads, 16 nodes, 32768 positions 33 (4.5 TB/s) + 5; 64 nodes, 2048 positions 17
// + 4, of which 9 stay at 32 positions (tree rows, meeting of the waves, launch);
// 16 heads, one node, 200 positions 6.  Not kept: four waves a SIMD (128
// registers, nothing requested ahead; 16 nodes 46 us against 45 then), two blocks
// ahead (40.0 against 38.6), loads past the caches (38.8 against 35.5).
#include <algorithm>

#include "ppd_kvq.h"

namespace {

constexpr int NT = 512;              // eight waves
constexpr int OROW = PPD_ATTN_OROW;  // partial row: 128 dims, m, l, padding (floats)
constexpr int kGroupRows = 128;      // rows of a workgroup at most
constexpr float kLn2 = 0.69314718055994531f;

// what a wave keeps of one 16-row tile (its queries apart)
struct RTile {
  float qs[2];    // sums of q over the two groups' dims
  uint64_t mk0, mk1;
  floatx4 o[8];   // O^T: dims 16 dt + 4 (lane / 16) + e, row lane % 16
  float pz[2];    // sums of P (z - 16 s), this lane's keys
  float m_run, l_run;
};

__device__ __forceinline__ float sum8(u32x4 v) {
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) s += __uint_as_float(v[w] << 16) + __uint_as_float(v[w] & 0xffff0000u);
  return s;
}

// Probabilities as two bf16 parts: the matrix cores take bf16, one part would
// leave 2^-9 of a probability, the size of the output's own rounding; two leave
// 2^-17, and a third would be half as many products with the values again.  (The
// outputs differ by 2e-4 to 3e-4 of their norm from those with float32
// probabilities, single bf16 steps; from 64 bits both differ by 0.0016 to 0.0017.)
__device__ __forceinline__ void split8(const float (&v)[8], u32x4 &hi, u32x4 &lo) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = v[e] - bf16_to_f32(f32_to_bf16(v[e]));
  hi = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  lo = u32x4{pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7])};
}

// One block's scores (unscaled, hidden keys at -inf) into the running softmax:
// the reference moves only when a maximum passes it by 8 (log2), P in pv.
__device__ __forceinline__ void softmax_step(RTile &R, const float (&sv)[8], float c, float (&pv)[8]) {
  const float lmax = c * fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])),
                               fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
  if (__ballot(lmax > R.m_run + 8.f)) {
    const float bmax = quad_max(lmax);
    const bool need = bmax > R.m_run + 8.f;
    const float alpha = need ? __builtin_amdgcn_exp2f(R.m_run - bmax) : 1.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) R.o[dt] *= alpha;
    R.pz[0] *= alpha;
    R.pz[1] *= alpha;
    R.l_run *= alpha;
    R.m_run = need ? bmax : R.m_run;
  }
  const float m_eff = R.m_run == -INFINITY ? 0.f : R.m_run;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    pv[e] = __builtin_amdgcn_exp2f(fmaf(sv[e], c, -m_eff));
    R.l_run += pv[e];
  }
}

// NQ tiles a wave, QW waves side by side over tiles, PARS over blocks
template <int NQ, int QW, int PARS, bool PLANES>
__global__ __launch_bounds__(NT, 1) void kvq_attention_kernel(KvqAttnLaunch p) {
  static_assert(QW * PARS * 64 == NT && QW * NQ * 16 <= kGroupRows, "eight waves");
  constexpr int RW = QW * NQ * 16;  // rows of the workgroup
  constexpr int PARTS = PLANES ? 2 : 1;
  // the waves' rows, after the main loop; before, with several tiles a wave,
  // their queries (64 registers would not be left for them)
  __shared__ __attribute__((aligned(16))) float rows_s[PARS][RW][OROW];
  u32x4 *q_s = (u32x4 *)rows_s;  // [tile][ds][part][lane]
  static_assert((size_t)QW * NQ * 4 * PARTS * 1024 <= sizeof(rows_s), "queries fit");
  __shared__ __attribute__((aligned(16))) floatx4 par_s[8][2 * kQB];  // per wave: affine pairs of 32 keys, 32 values

  __shared__ float fac_s[RW][PARS];  // what a row's waves are added with
  __shared__ int at_s[RW];           // its place, token x heads + head

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qw = wave % QW, par = wave / QW;
  const int lr = lane & 15, lg = lane >> 4;
  // slot -> sequence, kv head, row group, split
  int sq = 0;
  for (int j = 1; j < p.sb.B; ++j) sq = (int)blockIdx.x >= p.slot0[j] ? j : sq;
  const int t0 = p.sb.t0[sq], T = p.sb.t0[sq + 1] - t0, L = p.sb.L[sq];
  const int G = p.nh / p.nkv, R = T * G, n_grp = (R + RW - 1) / RW;
  const int KS = p.splits[sq];
  int local = blockIdx.x - p.slot0[sq];
  const int ks = local % KS;
  local /= KS;
  const int grp = local % n_grp, kvh = local / n_grp;
  const int n4 = (L + kQB - 1) / kQB, nblk = n4 + (T + kQB - 1) / kQB;
  const int b0 = min(nblk, ks * p.chunk[sq]), b1 = min(nblk, b0 + p.chunk[sq]);
  const unsigned char *blocks = p.sb.blocks[sq] + (size_t)kvh * p.sb.nb[sq] * kQBytes;
  const int tcap = p.sb.tcap[sq];
  const bf16_t *tk = p.sb.tk[sq] + (size_t)kvh * tcap * 128, *tv = p.sb.tv[sq] + (size_t)kvh * 128 * tcap;
  const int row0 = grp * RW;
  const int MT = p.T_pad >> 4;

  // a block's codes and parameters; past the wave's blocks the first one again
  // (the same loads on every path, so that the wait for them is a counted one)
  u32x4 kw[2], vw[2];
  u32x2 pr;
  auto request = [&](int blk) {
    const unsigned char *src = blocks + (size_t)(blk < b1 && blk < n4 ? blk : 0) * kQBytes;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      kw[t] = *(const u32x4 *)(src + (t * 64 + lane) * 16);
      vw[t] = *(const u32x4 *)(src + kQV + (t * 64 + lane) * 16);
    }
    pr = *(const u32x2 *)(src + kQP + lane * 8);
  };
  if (n4 > 0) request(b0 + par);
  __builtin_amdgcn_sched_barrier(0);

  RTile rt[NQ];
  u32x4 qr[4][PARTS];  // the queries, with one tile a wave
  const int n_live = min(NQ, ((min(R - row0, RW) + 15) / 16 - qw + QW - 1) / QW);
  // queries and masks, all requested before the first is used
  u32x4 qa[NQ][4][PARTS];  // B operand, dims 32 ds + 8 (lane / 16) .. + 7, parts hi, lo
  int tok_of[NQ], head_of[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int r = row0 + (qw + QW * i) * 16 + lr, rc = min(r, R - 1);
    const int tok = tok_of[i] = t0 + rc / G, head = head_of[i] = kvh * G + rc % G;
#pragma unroll
    for (int ds = 0; ds < 4; ++ds) {
      if constexpr (PLANES) {
        const unsigned char *src = (const unsigned char *)p.q + plane_off(MT, tok, head * 128 + ds * 32 + lg * 8);
        qa[i][ds][0] = *(const u32x4 *)src;
        qa[i][ds][1] = *(const u32x4 *)(src + kPlaneLo);
      } else {
        qa[i][ds][0] = *(const u32x4 *)((const bf16_t *)p.q + ((size_t)tok * p.nh + head) * 128 + ds * 32 + lg * 8);
      }
    }
    rt[i].mk0 = p.mask[2 * (size_t)tok];
    rt[i].mk1 = p.mask[2 * (size_t)tok + 1];
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const bool live = row0 + (qw + QW * i) * 16 + lr < R;
    const int tok = tok_of[i], head = head_of[i];
    const u32x4 (&q)[4][PARTS] = qa[i];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int part = PARTS - 1; part >= 0; --part) sum += sum8(q[2 * g][part]) + sum8(q[2 * g + 1][part]);
      rt[i].qs[g] = quad_sum(sum);
    }
    if constexpr (PLANES) {
      if (p.q_out && ks == 0 && par == 0 && live) {
        float *dst = p.q_out + ((size_t)tok * p.nh + head) * 128 + lg * 8;
#pragma unroll
        for (int ds = 0; ds < 4; ++ds)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t a = q[ds][0][w], b = q[ds][1][w];
            *(float2 *)(dst + ds * 32 + 2 * w) =
                float2{__uint_as_float(a << 16) + __uint_as_float(b << 16),
                       __uint_as_float(a & 0xffff0000u) + __uint_as_float(b & 0xffff0000u)};
          }
      }
    }
#pragma unroll
    for (int ds = 0; ds < 4; ++ds)
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        if constexpr (NQ == 1)
          qr[ds][part] = q[ds][part];
        else if (par == 0)
          q_s[(((qw + QW * i) * 4 + ds) * PARTS + part) * 64 + lane] = q[ds][part];
      }
    rt[i].mk0 = live ? rt[i].mk0 : 0ull;
    rt[i].mk1 = live ? rt[i].mk1 : 0ull;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) rt[i].o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    rt[i].pz[0] = rt[i].pz[1] = 0.f;
    rt[i].m_run = -INFINITY;
    rt[i].l_run = 0.f;
  }
  if constexpr (NQ > 1) __syncthreads();  // the queries are in LDS
  auto query = [&](int i, int ds, int part) {
    if constexpr (NQ == 1)
      return as_bf16x8(qr[ds][part]);
    else
      return as_bf16x8(q_s[(((qw + QW * i) * 4 + ds) * PARTS + part) * 64 + lane]);
  };
  const float c = p.scale_log2;
  const KvqBits bits;

  int blk = b0 + par;
  if (n_live > 0) {
    for (; blk < min(b1, n4); blk += PARS) {
      const u32x4 kc[2] = {kw[0], kw[1]}, vc[2] = {vw[0], vw[1]};
      const u32x2 pc = pr;
      request(blk + PARS);
      const bool valid = blk * kQB + (lane & 31) < L;
      const float2 a0 = kvq_affine(pc[0]), a1 = kvq_affine(pc[1]);
      par_s[wave][lane] = valid ? floatx4{a0.x, a0.y, a1.x, a1.y} : floatx4{0.f, 0.f, 0.f, 0.f};
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      float sv[NQ][8];
      floatx4 acc[NQ][2][2];  // [tile][group][key tile]: a query fragment is read once for both key tiles
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) acc[i][g][0] = acc[i][g][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const bf16x8 x0 = as_bf16x8(kvq_expand(kc[0][2 * g + d], bits)), x1 = as_bf16x8(kvq_expand(kc[1][2 * g + d], bits));
#pragma unroll
          for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
              const bf16x8 q = query(i, 2 * g + d, part);
              acc[i][g][0] = mfma16x16x32(x0, q, acc[i][g][0]);
              acc[i][g][1] = mfma16x16x32(x1, q, acc[i][g][1]);
            }
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const floatx4 a = par_s[wave][8 * lg + 4 * t + e];
#pragma unroll
          for (int i = 0; i < NQ; ++i) {
            const float x = fmaf(a[0], acc[i][0][t][e], a[1] * rt[i].qs[0]);
            sv[i][4 * t + e] = fmaf(a[2], acc[i][1][t][e], fmaf(a[3], rt[i].qs[1], x));
          }
        }
      if (blk * kQB + kQB > L) {  // the prefix ends in this block
        const int vis = L - blk * kQB - 8 * lg;
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
          for (int u = 0; u < 8; ++u) sv[i][u] = u < vis ? sv[i][u] : -INFINITY;
      }
      float pv[NQ][8];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NQ; ++i) softmax_step(rt[i], sv[i], c, pv[i]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        u32x4 ph[NQ], pl[NQ];
        float ps[NQ][8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float2 a = *((const float2 *)&par_s[wave][kQB + 8 * lg + u] + g);
#pragma unroll
          for (int i = 0; i < NQ; ++i) {
            ps[i][u] = pv[i][u] * a.x;
            rt[i].pz[g] = fmaf(pv[i][u], a.y, rt[i].pz[g]);
          }
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) split8(ps[i], ph[i], pl[i]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const bf16x8 x = as_bf16x8(kvq_expand(vc[g][w], bits));
#pragma unroll
          for (int i = 0; i < NQ; ++i) rt[i].o[4 * g + w] = mfma16x16x32(x, as_bf16x8(pl[i]), rt[i].o[4 * g + w]);
#pragma unroll
          for (int i = 0; i < NQ; ++i) rt[i].o[4 * g + w] = mfma16x16x32(x, as_bf16x8(ph[i]), rt[i].o[4 * g + w]);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the parameters' LDS is written next
    }
    for (; blk < b1; blk += PARS) {
      // tree rows: keys and values straight from the tail, all requested at once
      const int k0 = (blk - n4) * kQB;
      const int j0 = k0 + 8 * lg, keep_n = max(0, min(8, T - j0));  // keys of the lane that exist
      u32x4 kf[2][4], vf[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16_t *row = tk + (size_t)min(k0 + kvq_key_of(t, lr), tcap - 1) * 128 + lg * 8;
#pragma unroll
        for (int ds = 0; ds < 4; ++ds) kf[t][ds] = *(const u32x4 *)(row + ds * 32);
      }
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) vf[dt] = *(const u32x4 *)(tv + (size_t)(16 * dt + lr) * tcap + min(j0, tcap - 8));
      __builtin_amdgcn_sched_barrier(0);
      float sv[NQ][8];
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          floatx4 acc = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
            for (int ds = 0; ds < 4; ++ds) acc = mfma16x16x32(as_bf16x8(kf[t][ds]), query(i, ds, part), acc);
#pragma unroll
          for (int e = 0; e < 4; ++e) sv[i][4 * t + e] = acc[e];
        }
      __builtin_amdgcn_sched_barrier(0);
      u32x4 ph[NQ], pl[NQ];
      uint32_t seen[NQ];
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const uint64_t win = j0 >= 128 ? 0ull : j0 >= 64 ? rt[i].mk1 >> (j0 - 64) : rt[i].mk0 >> j0;
        seen[i] = (uint32_t)win & ((1u << keep_n) - 1u);
#pragma unroll
        for (int u = 0; u < 8; ++u) sv[i][u] = (seen[i] >> u) & 1u ? sv[i][u] : -INFINITY;
        float pv[8];
        softmax_step(rt[i], sv[i], c, pv);
        split8(pv, ph[i], pl[i]);
      }
      __builtin_amdgcn_sched_barrier(0);
      uint32_t end = 0;  // bit 15 of a half: an exponent of all ones
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          vf[dt][w] &= (2 * w < keep_n ? 0xffffu : 0u) | (2 * w + 1 < keep_n ? 0xffff0000u : 0u);
          end |= (vf[dt][w] & 0x7fff7fffu) + 0x00800080u;
        }
      if (__ballot(end & 0x80008000u)) {
        // infinities and NaN must not reach the rows that do not see them (0
        // times them is NaN): they are taken out, and the rows that see one
        // get NaN
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          u32x4 odd;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            odd[w] = ((((vf[dt][w] & 0x7fff7fffu) + 0x00800080u) >> 15) & 0x00010001u) * 0x3f80u;  // 1.0 where one is
            vf[dt][w] &= ~(odd[w] / 0x3f80u * 0xffffu);
          }
#pragma unroll
          for (int i = 0; i < NQ; ++i) {
            u32x4 on;
#pragma unroll
            for (int w = 0; w < 4; ++w)
              on[w] = (seen[i] >> (2 * w) & 1u ? 0x3f80u : 0u) | (seen[i] >> (2 * w + 1) & 1u ? 0x3f800000u : 0u);
            const floatx4 n = mfma16x16x32(as_bf16x8(odd), as_bf16x8(on), floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) rt[i].o[dt][e] = n[e] > 0.f ? NAN : rt[i].o[dt][e];
          }
        }
      }
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) rt[i].o[dt] = mfma16x16x32(as_bf16x8(vf[dt]), as_bf16x8(pl[i]), rt[i].o[dt]);
#pragma unroll
        for (int i = 0; i < NQ; ++i) rt[i].o[dt] = mfma16x16x32(as_bf16x8(vf[dt]), as_bf16x8(ph[i]), rt[i].o[dt]);
      }
    }
  }

  if constexpr (NQ > 1) __syncthreads();  // the queries' LDS is free
  // ---- the waves meet in LDS: thread -> row tid / 32 + 16 n, dims 4 (tid % 32) .. + 3
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const float l = quad_sum(rt[i].l_run), z0 = quad_sum(rt[i].pz[0]), z1 = quad_sum(rt[i].pz[1]);
    if (i < n_live) {
      float *row = rows_s[par][(qw + QW * i) * 16 + lr];
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *(floatx4 *)(row + dt * 16 + lg * 4) = rt[i].o[dt] + (dt < 4 ? z0 : z1);
      if (lg == 0) *(float2 *)(row + 128) = float2{rt[i].m_run, l};
    }
  }
  __syncthreads();
  // a row's factors of the waves' sums, its place, maximum and sum: a thread a row
  const int n_rows = min(R - row0, RW);
  const size_t part0 = (size_t)ks * p.sb.t0[p.sb.B] * p.nh;
  if (tid < n_rows) {
    const int r = row0 + tid, at = (t0 + r / G) * p.nh + kvh * G + r % G;
    float2 ml[PARS];
    float M = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < PARS; ++w) {
      ml[w] = *(const float2 *)(rows_s[w][tid] + 128);
      M = fmaxf(M, ml[w].x);
    }
    float f[PARS];
#pragma unroll
    for (int w = 0; w < PARS; ++w) {
      f[w] = ml[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w].x - M);
      l += f[w] * ml[w].y;
    }
    const float inv = KS > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int w = 0; w < PARS; ++w) fac_s[tid][w] = f[w] * inv;
    at_s[tid] = at;
    if (KS > 1)
      *(float2 *)(p.part + (part0 + at) * OROW + 128) = float2{M, l};
    else if (p.lse)
      p.lse[at] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
  }
  __syncthreads();
  const int d4 = (tid & 31) * 4;
#pragma unroll 2
  for (int rl = tid >> 5; rl < n_rows; rl += NT / 32) {
    const int at = at_s[rl];
    floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < PARS; ++w) o += fac_s[rl][w] * *(const floatx4 *)(rows_s[w][rl] + d4);
    if (KS > 1) {
      *(floatx4 *)(p.part + (part0 + at) * OROW + d4) = o;
    } else if constexpr (PLANES) {
      const int tok = at / p.nh;
      store_plane4((unsigned char *)p.out, MT, tok, (at - tok * p.nh) * 128 + d4, {o[0], o[1], o[2], o[3]});
    } else {
      *(u32x2 *)((bf16_t *)p.out + (size_t)at * 128 + d4) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
    }
  }
}

// the splits of a row, added in order; 32 threads a row
template <bool PLANES>
__global__ __launch_bounds__(NT) void kvq_merge_kernel(KvqAttnLaunch p) {
  const int n_rows = p.sb.t0[p.sb.B] * p.nh;
  const int at = blockIdx.x * (NT / 32) + (threadIdx.x >> 5), d4 = (threadIdx.x & 31) * 4;
  if (at >= n_rows) return;
  const int tok = at / p.nh, head = at % p.nh;
  int sq = 0;
  for (int j = 1; j < p.sb.B; ++j) sq = tok >= p.sb.t0[j] ? j : sq;
  const int KS = p.splits[sq];
  if (KS == 1) return;  // already final
  constexpr int N = 8;  // rows in flight: one round trip for all of them
  float M = -INFINITY, l = 0.f;
  floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < KS; s0 += N) {
    float2 ml[N];
    floatx4 x[N];
#pragma unroll
    for (int v = 0; v < N; ++v) {
      const float *row = p.part + ((size_t)min(s0 + v, KS - 1) * n_rows + at) * OROW;
      ml[v] = *(const float2 *)(row + 128);
      x[v] = *(const floatx4 *)(row + d4);
    }
    __builtin_amdgcn_sched_barrier(0);
    float m = M;
#pragma unroll
    for (int v = 0; v < N; ++v) m = fmaxf(m, ml[v].x);  // (the last row repeats)
    const float keep = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - m);
    o *= keep;
    l *= keep;
    M = m;
#pragma unroll
    for (int v = 0; v < N; ++v) {
      const float f = s0 + v >= KS || ml[v].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[v].x - M);
      // (a split that sees NaN alone has no maximum: 0 times its sum keeps it)
      l += s0 + v < KS ? f * ml[v].y : 0.f;
      if (s0 + v < KS) o += f * x[v];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (PLANES)
    store_plane4((unsigned char *)p.out, p.T_pad >> 4, tok, head * 128 + d4, {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv});
  else
    *(u32x2 *)((bf16_t *)p.out + (size_t)at * 128 + d4) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
  if (p.lse && d4 == 0) p.lse[at] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
}

// ---------------------------------------------------------------------------
// Accumulated weights.  Here the rows are the A operand and the keys the B
// operand, S = Q K^T: a lane then holds one key and four rows, and the sum over
// rows is over its registers and four lane groups.  Rows: path node x head, r =
// i G + a, in passes of TILES tiles, whose queries stay in registers as bf16
// parts: three of a float32 (its last bits too, so that a weight is exact to
// float32's own rounding of its exponent), one of a bfloat16.  A wave takes every
// step-th block of a (layer, kv head), the next one requested ahead.
//
// Three nodes, 32 layers of 32 heads, 2048 positions 43 us (3.9 TB/s of a copy's
// 4.8); five nodes, 32 heads on 8 kv heads, 8191 positions 50 (3.4 TB/s; two
// tiles a key).  Bounds on registers: a tile of queries fits four waves a SIMD
// (45 us with two; float32's spills 14 registers, outside the loops over blocks),
// two tiles three with bfloat16 queries (56 with two), two with float32's three
// parts.  With queries in LDS instead, 24 KB read for every block and tile, 62
// and 89.
struct ScoreRow {
  float qs0, qs1, lse2;  // sums of q over the groups, ln sum exp in log2
};
constexpr int kScoreWaves = 4;

template <int TILES, int PARTS>
__global__ __launch_bounds__(64 * kScoreWaves, TILES > 1 ? PARTS > 1 ? 2 : 3 : 4) void kvq_score_kernel(KvqScoreLaunch p) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int lh = blockIdx.x / p.runs, layer = lh / p.nkv, kvh = lh % p.nkv;
  const int first = (blockIdx.x % p.runs) * kScoreWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int step = p.runs * kScoreWaves;
  const unsigned char *blocks = p.blocks + (size_t)lh * p.nb * kQBytes;
  const float *in = p.in ? p.in + (size_t)lh * p.cap : nullptr;
  float *out = p.out + (size_t)lh * p.cap;
  const int n4 = (p.L + kQB - 1) / kQB;
  const float c = p.scale_log2;
  const KvqBits bits;
  // a block's keys: codes, this lane's keys' parameters, their sums so far
  u32x4 kw[2];
  u32x2 pr[2];
  float base[2];
  auto request = [&](int blk, bool more) {
    blk = blk < n4 ? blk : 0;  // past the last one: the first again
    const unsigned char *src = blocks + (size_t)blk * kQBytes;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = kvq_key_of(t, lr);
      kw[t] = *(const u32x4 *)(src + (t * 64 + lane) * 16);
      pr[t] = *(const u32x2 *)(src + kQP + j * 8);
      const float *from = more ? out : in;
      base[t] = from ? from[min(blk * kQB + j, p.L - 1)] : 0.f;
    }
  };
  if (n4 > 0) request(first, false);
  const int n = max(0, min(*p.n_path, min(p.path_len, p.cap - p.L)));
  const int G = p.nh / p.nkv, R = n * G, nblk = n4 + (n + kQB - 1) / kQB;

  for (int r0 = 0; r0 == 0 || r0 < R; r0 += TILES * 16) {
    const bool more = r0 > 0;  // a further pass adds to the sums of the last
    if (more && n4 > 0) request(first, true);
    // ---- the pass's rows: lane lr loads row r0 + 16 m + lr; the products' rows
    // are 4 lg + e
    u32x4 q[TILES][4][PARTS];
    ScoreRow row[TILES][4];
#pragma unroll
    for (int m = 0; m < TILES; ++m) {
      const int r = r0 + 16 * m + lr;
      const bool live = r < R;
      const int i = live ? r / G : 0, head = kvh * G + (live ? r - i * G : 0);
      const int node = n > 0 ? max(0, min(p.path[i], p.T - 1)) : 0;
      const size_t at = ((size_t)layer * p.rows + node) * p.nh + head;
      const float lse = p.lse[at];
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int ds = 0; ds < 4; ++ds) {
        float v[8];
        if constexpr (PARTS == 1) {
          const u32x4 w = *(const u32x4 *)((const bf16_t *)p.q + at * 128 + ds * 32 + lg * 8);
          q[m][ds][0] = w;
          sum[ds >> 1] += live ? sum8(w) : 0.f;
        } else {
          const floatx4 x = *(const floatx4 *)((const float *)p.q + at * 128 + ds * 32 + lg * 8);
          const floatx4 y = *(const floatx4 *)((const float *)p.q + at * 128 + ds * 32 + lg * 8 + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = x[e], v[4 + e] = y[e];
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[ds >> 1] += live ? v[e] : 0.f;
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t w = q[m][ds][part][e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
              v[2 * e] -= __uint_as_float(w << 16);
              v[2 * e + 1] -= __uint_as_float(w & 0xffff0000u);
            }
        }
      }
      sum[0] = quad_sum(sum[0]);
      sum[1] = quad_sum(sum[1]);
      const float l2 = lse * 1.4426950408889634f;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        row[m][e] = ScoreRow{__shfl(sum[0], 4 * lg + e, 64), __shfl(sum[1], 4 * lg + e, 64), __shfl(l2, 4 * lg + e, 64)};
    }
    // weights of this lane's key: a its affine pairs, only rows r0 + from .. R - 1
    const int rows = R - r0;
    auto weigh = [&](const u32x4 (&b)[4], float4 a, int from) {
      float w = 0.f;
#pragma unroll
      for (int m = 0; m < TILES; ++m) {
        if (m > 0 && 16 * m >= rows) break;
        floatx4 acc[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          acc[g] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
            for (int d = 0; d < 2; ++d)
              acc[g] = mfma16x16x32(as_bf16x8(q[m][2 * g + d][part]), as_bf16x8(b[2 * g + d]), acc[g]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const ScoreRow &x = row[m][e];
          const float s = fmaf(a.x, acc[0][e], a.y * x.qs0) + fmaf(a.z, acc[1][e], a.w * x.qs1);
          const int r = 16 * m + 4 * lg + e;
          w += r >= from && r < rows ? __builtin_amdgcn_exp2f(fmaf(s, c, -x.lse2)) : 0.f;
        }
      }
      return quad_sum(w);
    };
    // ---- the prefix
    int blk = first;
    for (; blk < n4; blk += step) {
      const u32x4 kc[2] = {kw[0], kw[1]};
      const u32x2 pc[2] = {pr[0], pr[1]};
      const float bc[2] = {base[0], base[1]};
      request(blk + step, more);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 b[4];
#pragma unroll
        for (int ds = 0; ds < 4; ++ds) b[ds] = kvq_expand(kc[t][ds], bits);
        const float2 a0 = kvq_affine(pc[t][0]), a1 = kvq_affine(pc[t][1]);
        const float w = weigh(b, float4{a0.x, a0.y, a1.x, a1.y}, 0);
        const int pos = blk * kQB + kvq_key_of(t, lr);
        if (lg == 0 && pos < p.L) out[pos] = bc[t] + w;
      }
    }
    // ---- the accepted nodes' own keys, from the tail
    const bf16_t *tk = p.tk + (size_t)lh * p.tcap * 128;
    for (; blk < nblk; blk += step)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int k = (blk - n4) * kQB + kvq_key_of(t, lr);
        const int node = max(0, min(p.path[min(k, n - 1)], min(p.T, p.tcap) - 1));
        u32x4 b[4];
#pragma unroll
        for (int ds = 0; ds < 4; ++ds) b[ds] = *(const u32x4 *)(tk + (size_t)node * 128 + ds * 32 + lg * 8);
        const float w = weigh(b, float4{1.f, 0.f, 1.f, 0.f}, k * G - r0);  // the nodes from its own on
        if (lg == 0 && k < n) out[p.L + k] = (more ? out[p.L + k] : 0.f) + w;
      }
  }
}

}  // namespace

// 16-row tiles a wave holds and waves side by side, by the most tiles a kv head has
static void kvq_shape(int tiles, int *nq, int *qw) {
  *nq = tiles <= 1 ? 1 : 2;
  *qw = tiles <= 2 ? 1 : tiles <= 4 ? 2 : 4;
}

// a workgroup a compute unit: the kernels' registers and LDS leave room for one
constexpr long kSlots = 256;

// (64: of one or two kv heads 128 splits were slower, what they save lost in
// adding them: 2 kv heads, 65536 positions 27.3 us against 31.4, one head, 128 rows,
// 8192 positions 21.8 against 24.7)
int kvq_attn_max_splits(int nkv) { return (int)std::max<long>(1, std::min<long>(64, kSlots / nkv)); }

size_t kvq_attn_part_bytes(int nh, int nkv, int T) {
  return (size_t)kvq_attn_max_splits(nkv) * T * nh * OROW * sizeof(float);
}

void kvq_attn_plan(KvqAttnLaunch &a) {
  const int B = a.sb.B, G = a.nh / a.nkv, cap = kvq_attn_max_splits(a.nkv);
  a.tiles = 1;
  for (int j = 0; j < B; ++j) a.tiles = std::max(a.tiles, ((a.sb.t0[j + 1] - a.sb.t0[j]) * G + 15) / 16);
  int nq, qw;
  kvq_shape(a.tiles, &nq, &qw);
  const int rw = 16 * nq * qw, pars = 8 / qw;
  long total = 0;
  int nblk[PPD_BATCH_MAX], units[PPD_BATCH_MAX];
  for (int j = 0; j < B; ++j) {
    const int T = a.sb.t0[j + 1] - a.sb.t0[j];
    nblk[j] = (a.sb.L[j] + kQB - 1) / kQB + (T + kQB - 1) / kQB;
    units[j] = a.nkv * ((T * G + rw - 1) / rw);
    total += (long)units[j] * nblk[j];
  }
  a.n_slots = 0;
  for (int j = 0; j < B; ++j) {
    // the sequence's share of kSlots workgroups, a block a wave at least
    const long want = std::max<long>(1, kSlots * (long)nblk[j] / std::max<long>(1, total));
    a.splits[j] = (int)std::max<long>(1, std::min<long>(std::min<long>(cap, want), nblk[j] / pars));
    a.chunk[j] = (nblk[j] + a.splits[j] - 1) / a.splits[j];
    a.splits[j] = (nblk[j] + a.chunk[j] - 1) / a.chunk[j];
    a.slot0[j] = a.n_slots;
    a.n_slots += units[j] * a.splits[j];
  }
}

template <bool PLANES>
static hipError_t launch_attn(const KvqAttnLaunch &a, hipStream_t s) {
  auto kernel = a.tiles <= 1   ? kvq_attention_kernel<1, 1, 8, PLANES>
                : a.tiles <= 2 ? kvq_attention_kernel<2, 1, 8, PLANES>
                : a.tiles <= 4 ? kvq_attention_kernel<2, 2, 4, PLANES>
                               : kvq_attention_kernel<2, 4, 2, PLANES>;
  const bool merge = *std::max_element(a.splits, a.splits + a.sb.B) > 1;
  const hipEvent_t ev0 = (hipEvent_t)a.ev_start, ev1 = (hipEvent_t)a.ev_stop;
  if (ev0)
    hipExtLaunchKernelGGL(kernel, dim3(a.n_slots), dim3(NT), 0, s, ev0, merge ? (hipEvent_t) nullptr : ev1, 0, a);
  else
    hipLaunchKernelGGL(kernel, dim3(a.n_slots), dim3(NT), 0, s, a);
  if (merge) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((a.sb.t0[a.sb.B] * a.nh + NT / 32 - 1) / (NT / 32));
    if (ev1)
      hipExtLaunchKernelGGL(kvq_merge_kernel<PLANES>, grid, dim3(NT), 0, s, (hipEvent_t) nullptr, ev1, 0, a);
    else
      hipLaunchKernelGGL(kvq_merge_kernel<PLANES>, grid, dim3(NT), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_kvq_attn(const KvqAttnLaunch &a, hipStream_t s) {
  return a.planes ? launch_attn<true>(a, s) : launch_attn<false>(a, s);
}

hipError_t launch_kvq_score(KvqScoreLaunch p, hipStream_t s) {
  // As many workgroups as are resident at once, eight blocks a wave or more where
  // there are.  How many rows there are is only known on the device: an accepted
  // path is a few nodes, so a tile holds those of one or two heads, two tiles
  // those of four.
  const int heads = p.layers * p.nkv, nblk = (p.L + p.path_len + 2 * kQB - 2) / kQB;
  const bool two = p.nh / p.nkv > 2;
  const int resident = 256 * (!two ? 4 : p.q_bf16 ? 3 : 2);
  p.runs = std::max(1, std::min(resident / heads, nblk / (8 * kScoreWaves)));
  auto kernel = p.q_bf16 ? (two ? kvq_score_kernel<2, 1> : kvq_score_kernel<1, 1>)
                         : (two ? kvq_score_kernel<2, 3> : kvq_score_kernel<1, 3>);
  hipLaunchKernelGGL(kernel, dim3(heads * p.runs), dim3(64 * kScoreWaves), 0, s, p);
  return hipGetLastError();
}
