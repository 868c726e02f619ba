// Attention over a paged prefix and the new rows, lengths on the device.
//
// Rows.  The heads that share a kv head read the same keys, so a kv head's rows
// are new row x head, r = t G + a (a < G), in 16-row tiles.
//
// Products (v_mfma_f32_16x16x32_bf16): S^T = K Q^T with the 32 keys of a block as
// two 16-row A operands, O^T += V^T P^T with 16 dims as the A operand.  Pages hold
// blocks in the order of these operands: 16 loads of 1 KB, straight into the
// registers of the wave that multiplies them, the next block's keys requested
// when a block's are multiplied, its values when its values are.  A wave's rows of
// S^T are the keys that its lanes hold as the B operand of the second product.
//
// Work decomposition.  A workgroup takes a sequence, a kv head, up to RW rows and
// one of KS key splits; its waves are QW side by side over tiles, NQ tiles each,
// and PARS over blocks, with no barrier in the loop: (NQ, QW, PARS) = (1, 1, 4),
// (2, 1, 4), (2, 2, 4) or (2, 4, 2), by paged_width.  The grid is fixed by what the
// host knows (sequences, rows, the tables' width); which part a workgroup takes
// every wave finds for itself from the lengths, so a captured call follows them.
// Splits are such that a compute unit has one workgroup, of one sequence exactly as
// many for every row group: where 9 splits of 32 groups put two workgroups on 32
// units, 16 rows over 2048 positions took 20.1 us, with 8 16.5; twice as many
// workgroups throughout, 131072 positions 93 us, 88 as it is.  Row groups of the
// same keys are workgroups of one XCD; started at places of their own instead of
// side by side they took 29 us for 20 (64 rows, 2048 positions).  Splits of one
// or two tiles are added by the last of them to arrive, through memory past
// the caches; wider ones by a second launch, since their rows are too many for
// one compute unit.
//
// Bounds.  A compute unit has at most 32 KB of loads in flight (its L1), and four
// waves keep it there: with eight a workgroup 32 heads over 2000 positions took 17.3 us
// for 15.6 and 64 sequences 104 for 101, with two blocks requested ahead 64
// sequences 101 for 96 (each beside the kernel of its time).  131072 positions 88 us (6.1
// TB/s of reads; a copy 5.0), 64 sequences of up to 8192 positions 89 (5.6 TB/s, by
// uneven shares), 128 of 2000 positions 168 (6.0).  64 rows over
// 2048 positions 19.4: a unit loads 540 KB, each block for four tiles.  200 positions
// 6.0: launch, lengths, table, keys, waves' meeting, one after another; splits
// add about 4 (rows out, arrival, rows in).  Streaming (non-temporal) loads of pages
// that one wave alone reads: 131072 positions 108 -> 97 us then.
#include <algorithm>

#include "ppd_paged.h"

namespace {

constexpr int NT = 512;              // threads of the second launch
constexpr int kLeast = 2;            // blocks of a wave, at least, where a prefix is split
constexpr int OROW = PPD_ATTN_OROW;  // partial row: 128 dims, m, l, padding (floats)
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kNoSplit = PPD_CAPACITY_MAX;  // more blocks than a sequence has

// parts of a query and of a probability on the matrix cores: a bfloat16 output is
// rounded by up to 2^-8 of itself, a probability of two parts by 2^-16 (one would
// double the output's error); float32 calls carry three parts of both, 2^-24
__host__ __device__ constexpr int q_parts(int qt) { return qt == PAGED_Q_BF16 ? 1 : qt == PAGED_Q_F32 ? 3 : 2; }
__host__ __device__ constexpr int p_parts(int qt) { return qt == PAGED_Q_F32 ? 3 : 2; }

struct PTile {
  uint64_t mk0, mk1;
  floatx4 o[8];  // O^T: dims 16 dt + 4 (lane / 16) + e, row lane % 16
  float m_run, l_run;
};

// v in PARTS bf16 parts, the largest first
template <int PARTS>
__device__ __forceinline__ void split8(const float (&v)[8], u32x4 (&out)[PARTS]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
    out[part] = u32x4{pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7])};
    if (part + 1 < PARTS)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        r[e] -= __uint_as_float(e & 1 ? out[part][e >> 1] & 0xffff0000u : out[part][e >> 1] << 16);
  }
}

// One block's scores (unscaled, hidden keys at -inf) into the running softmax:
// the reference moves only when a maximum passes it by 8 (log2), P in pv.  Scaled
// scores are rounded before the reference is taken off: a fused product would
// leave the reference's own rounding, past 128 (and infinity) from scores of 2^31 on.
__device__ __forceinline__ void softmax_step(PTile &R, const float (&sv)[8], float c, float (&pv)[8]) {
#pragma clang fp contract(off)
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = sv[e] * c;
  const float lmax = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  if (__ballot(lmax > R.m_run + 8.f)) {
    const float bmax = quad_max(lmax);
    const bool need = bmax > R.m_run + 8.f;
    const float alpha = need ? __builtin_amdgcn_exp2f(R.m_run - bmax) : 1.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) R.o[dt] *= alpha;
    R.l_run *= alpha;
    R.m_run = need ? bmax : R.m_run;
  }
  const float m_eff = R.m_run == -INFINITY ? 0.f : R.m_run;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    pv[e] = __builtin_amdgcn_exp2f(x[e] - m_eff);
    R.l_run += pv[e];
  }
}

// a sequence's work: blocks of the prefix and of its rows, row groups
struct Load {
  int n4, nblk, grps, units;
};
__device__ __forceinline__ Load load_of(const PagedAttnLaunch &p, int s, const PagedSeq &q, int RW, bool *bad) {
  Load w;
  const int lb = p.sq.lp - 5, pages = (q.L + (1 << p.sq.lp) - 1) >> p.sq.lp;
  int n = (q.L + kPB - 1) / kPB;
  if (p.sel) {
    const int m = p.n_sel[s], most = min(pages, p.budget);
    *bad |= m < 0 || m > most;
    n = max(0, min(m, most)) << lb;
  }
  w.n4 = n;
  w.nblk = n + (q.T + kPB - 1) / kPB;
  w.grps = (q.T * (p.nh / p.nkv) + RW - 1) / RW;
  w.units = w.grps * p.nkv;
  return w;
}
// Blocks of a workgroup at most, LEAST at least.  With c of them a row group of n
// blocks is cut into ceil(n / c) splits.  Where c is not below total / (S slots),
// there are at most units + S workgroups, at most 2 S of them in groups of several
// splits and less than S such groups (each holds more than c blocks); S is
// 1.5 kPagedSlots at most below.
template <int LEAST>
__device__ __forceinline__ int blocks_each(int64_t total, int slots) {
  return (int)min(max((total + slots - 1) / slots, (int64_t)LEAST), (int64_t)kNoSplit);
}
__device__ __forceinline__ int splits_of(int units, int nblk, int c) {
  if (nblk <= c) return units ? 1 : 0;
  c = max(c, (nblk + kPagedSplits - 1) / kPagedSplits);
  return units ? (nblk + c - 1) / c : 0;
}
__device__ __forceinline__ int splits_of(const Load &w, int c) { return splits_of(w.units, w.nblk, c); }

struct Place {
  int sq, local, KS, part0;
  int bits;  // of a place's share of the counters
  PagedSeq q;
  Load w;
};
// Where workgroups of several sequences start: those of groups that are cut first (so
// a partial row's place is its workgroup's), and where not all start at once
// the others by their length, in three classes, so that the last to start are short.
// us in this order and in the sequences': 64 of up to 8192 positions 92 and 97, 200 of up
// to 4000 147 and 169, 32 of up to 3000 with four rows 46 and 49, 128 of 2000 174 both
constexpr int kClasses = 4;
__device__ __forceinline__ int class_of(int nblk, int KS, int c, bool at_once) {
  return KS > 1 ? 0 : at_once || nblk > c >> 1 ? 1 : nblk > c >> 2 ? 2 : 3;
}
// More than 64 sequences: a thread takes every NT-th, the workgroup adds.  Every wave
// by itself, 64 at a time, took 113 us for 81 with 1000 sequences of up to 1000
// positions, 524 for 195 with 3000 of up to 300 (192 since one workgroup alone looks
// for bad numbers); with the lengths read again for the second sum in place of LDS 94
// and 280.
template <int RW, int LEAST, int NT>
__device__ __forceinline__ bool find_place_of_many(const PagedAttnLaunch &p, int slot, int2 *list, Place *out, bool *bad) {
  constexpr int NW = NT / 64;
  __shared__ int64_t total_s[NW];
  __shared__ int count_s[NW][kClasses];
  __shared__ Place place_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t total = 0;
  int low = 0;
  if (blockIdx.x == 0)  // (3000 sequences on 8 kv heads 728 us, looked for in all workgroups 754)
    for (int s = tid; s < p.sq.B; s += NT) load_of(p, s, paged_seq(p.sq, s, bad), RW, bad);
  bool unused = false;
  for (int s0 = tid; s0 < p.sq.B; s0 += 4 * NT) {  // (past the last: the last again)
    PagedSeq q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = paged_seq(p.sq, min(s0 + i * NT, p.sq.B - 1), &unused, &low);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (s0 + i * NT < p.sq.B) {
        const Load w = load_of(p, s0 + i * NT, q[i], RW, &unused);
        list[s0 + i * NT] = int2{w.units, w.nblk};
        total += (int64_t)w.units * w.nblk;
      }
  }
  total = wave_total(total);
  if (__ballot(low < 0)) total = -1;  // (offsets fall)
  if (lane == 0) total_s[wave] = total;
  if (tid == 0) place_s.sq = -1;
  __syncthreads();
  total = 0;
  bool falls = false;
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    falls |= total_s[v] < 0;
    total += total_s[v];
  }
  if (falls) return false;
  const int c = blocks_each<2 * LEAST>(total, kPagedSlots * 3 / 2);
  int n[kClasses] = {}, upto[kClasses];
#pragma unroll 4
  for (int s = tid; s < p.sq.B; s += NT) {
    const int2 w = list[s];
    const int KS = splits_of(w.x, w.y, c), cls = class_of(w.y, KS, c, false);
#pragma unroll
    for (int k = 0; k < kClasses; ++k) n[k] += cls == k ? w.x * KS : 0;
  }
#pragma unroll
  for (int k = 0; k < kClasses; ++k) {
    upto[k] = wave_incl(n[k]);
    if (lane == 63) count_s[wave][k] = upto[k];
  }
  __syncthreads();
  int base = 0;
  for (int k = 0; k < kClasses; ++k) {
    int at = base + upto[k] - n[k];
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      at += v < wave ? count_s[v][k] : 0;
      base += count_s[v][k];
    }
    if (slot < at || slot >= at + n[k]) continue;
    for (int s = tid; s < p.sq.B; s += NT) {  // one of this thread's
      const int2 w = list[s];
      const int KS = splits_of(w.x, w.y, c), m = class_of(w.y, KS, c, false) == k ? w.x * KS : 0;
      if (slot < at + m) {
        const PagedSeq q = paged_seq(p.sq, s, &unused);
        place_s = Place{s, slot - at, KS, at, 2, q, load_of(p, s, q, RW, &unused)};
        break;
      }
      at += m;
    }
  }
  __syncthreads();
  *out = place_s;
  return out->sq >= 0;
}
// the workgroup's sequence and place in it; false: it has no part.  Offsets that fall
// give no workgroup one: the rows could ask for more workgroups than the grid has,
// and a split that is never run leaves the others' arrivals in the counters, where
// the workspace's next call would find them.  list: LDS for all sequences' work
template <int RW, int LEAST, int NT>
__device__ __forceinline__ bool find_place(const PagedAttnLaunch &p, int slot, int2 *list, Place *out, bool *bad) {
  if (p.sq.B == 1) {  // alike in all lanes
    out->sq = out->part0 = 0;
    out->bits = 6;
    out->q = paged_seq(p.sq, 0, bad);
    out->w = load_of(p, 0, out->q, RW, bad);
    // (as many for each row group: no compute unit gets one workgroup more than the others)
    const int even = max(1, kPagedSlots / max(1, out->w.units));
    out->KS = splits_of(out->w, max((out->w.nblk + even - 1) / even, LEAST));
    out->local = slot;
    return slot < out->w.units * out->KS;
  }
  if (p.sq.B > 64) return find_place_of_many<RW, LEAST, NT>(p, slot, list, out, bad);
  // a wave's lanes take a sequence each
  const int lane = threadIdx.x & 63;
  PagedSeq q{};
  Load w{};
  int low = 0;
  if (lane < p.sq.B) {
    q = paged_seq(p.sq, lane, bad, &low);
    w = load_of(p, lane, q, RW, bad);
  }
  if (__ballot(low < 0)) return false;
  const int64_t total = wave_total((int64_t)w.units * w.nblk);
  const int units = (int)wave_total((int64_t)w.units);
  const bool at_once = units <= kPagedSlots;
  int c;
  out->bits = at_once ? 3 : 2;
  if (!at_once) {  // several rounds of workgroups: only long groups are cut
    c = blocks_each<2 * LEAST>(total, kPagedSlots * 3 / 2);
  } else {  // one round: each is rounded up, so fewer until they fit
    c = blocks_each<LEAST>(total, kPagedSlots);
    for (int i = 0; i < 4; ++i) {
      const int n = (int)wave_total((int64_t)w.units * splits_of(w, c));
      if (n <= kPagedSlots) {
        out->bits = 6;
        break;
      }
      c = (int)min(((int64_t)c * n + kPagedSlots - 1) / kPagedSlots, (int64_t)kNoSplit);
    }
  }
  const int KS = splits_of(w, c), cls = class_of(w.nblk, KS, c, at_once);
  int base = 0;
  for (int k = 0; k < (at_once ? 2 : kClasses); ++k) {
    const int mine = cls == k ? w.units * KS : 0, upto = base + wave_incl(mine);
    const uint64_t hit = __ballot(slot < upto);
    if (hit) {
      const int at = __builtin_ctzll(hit);
      out->sq = at;
      out->part0 = lane_of(upto - mine, at);
      out->local = slot - out->part0;
      out->KS = lane_of(KS, at);
      out->q = PagedSeq{lane_of(q.t0, at), lane_of(q.T, at), lane_of(q.L, at)};
      out->w = Load{lane_of(w.n4, at), lane_of(w.nblk, at), lane_of(w.grps, at), lane_of(w.units, at)};
      return true;
    }
    base = lane_of(upto, 63);
  }
  return false;
}

template <int QT>
__device__ __forceinline__ void load_query(const PagedAttnLaunch &p, int tok, int head, int lg, u32x4 (&q)[4][q_parts(QT)]) {
#pragma unroll
  for (int ds = 0; ds < 4; ++ds) {
    if constexpr (QT == PAGED_Q_PLANES) {
      const unsigned char *src = (const unsigned char *)p.q + plane_off(p.T_pad >> 4, tok, head * 128 + ds * 32 + lg * 8);
      q[ds][0] = *(const u32x4 *)src;
      q[ds][1] = *(const u32x4 *)(src + kPlaneLo);
    } else if constexpr (QT == PAGED_Q_BF16) {
      q[ds][0] = *(const u32x4 *)((const bf16_t *)p.q + ((size_t)tok * p.nh + head) * 128 + ds * 32 + lg * 8);
    } else {
      const float *src = (const float *)p.q + ((size_t)tok * p.nh + head) * 128 + ds * 32 + lg * 8;
      const floatx4 a = *(const floatx4 *)src, b = *(const floatx4 *)(src + 4);
      split8<3>({a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}, q[ds]);
    }
  }
}

template <int QT>
__device__ __forceinline__ void store_out4(const PagedAttnLaunch &p, int tok, int head, int d4, floatx4 o) {
  if constexpr (QT == PAGED_Q_PLANES)
    store_plane4((unsigned char *)p.out, p.T_pad >> 4, tok, head * 128 + d4, {o[0], o[1], o[2], o[3]});
  else if constexpr (QT == PAGED_Q_BF16)
    *(u32x2 *)((bf16_t *)p.out + ((size_t)tok * p.nh + head) * 128 + d4) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
  else
    *(floatx4 *)((float *)p.out + ((size_t)tok * p.nh + head) * 128 + d4) = o;
}

// what a split's row is added with, M the largest maximum (a split that sees NaN
// alone has none: its sum is kept as it is)
__device__ __forceinline__ float factor_of(float2 ml, float M) {
  return ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(ml.x - M);
}

// Partial rows that another workgroup adds are written and read past this XCD's
// caches (sc1, the cache policy of agent scope), so no cache has to be written
// back or dropped for them.
constexpr int kFar = 16;
__device__ __forceinline__ void put_far(__amdgpu_buffer_rsrc_t r, size_t at, floatx4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, (int)(at * sizeof(float)), 0, kFar);
}
__device__ __forceinline__ floatx4 get_far(__amdgpu_buffer_rsrc_t r, size_t at) {
  return __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(at * sizeof(float)), 0, kFar));
}

// STREAM: past the caches (non-temporal), in workgroups of one tile or two.  Pages that
// one row group reads gain by it (131072 positions, one row 91 us for 101); where
// row groups share them neither is better throughout: 64 rows over 1024, 2048, 4096 and
// 8192 positions 16.1, 20.8, 26.7, 39.0 us, through the caches 15.4, 21.2, 27.1, 38.6.
template <bool STREAM>
__device__ __forceinline__ u32x4 load_page(const unsigned char *p) {
  if constexpr (STREAM) return __builtin_nontemporal_load((const u32x4 *)p);
  return *(const u32x4 *)p;
}

// table entries are read through the scalar cache: they are alike in a wave
__device__ __forceinline__ int uniform_load(const int32_t *p, int64_t i) {
  typedef const __attribute__((address_space(4))) int32_t cint;
  return ((cint *)(uintptr_t)p)[i];
}

// NQ tiles a wave, QW waves side by side over tiles, PARS over blocks
template <int NQ, int QW, int PARS, int QT>
__global__ __launch_bounds__(64 * QW * PARS, 2) void paged_attention_kernel(PagedAttnLaunch p) {
  constexpr int NT = 64 * QW * PARS;
  constexpr bool JOIN = QW == 1;  // the last of a row group's splits adds them
  constexpr int RW = QW * NQ * 16;  // rows of the workgroup
  constexpr int QP = q_parts(QT), PP = p_parts(QT);
  constexpr bool QLDS = NQ > 1 || QP > 2;  // no registers left for the queries
  // the waves' rows, after the main loop; before, the queries that lie in LDS
  __shared__ __attribute__((aligned(16))) float rows_s[PARS][RW][OROW];
  u32x4 *q_s = (u32x4 *)rows_s;  // [tile][ds][part][lane]
  static_assert((size_t)QW * NQ * 4 * QP * 1024 <= sizeof(rows_s), "queries fit");
  static_assert(PPD_PAGED_SEQS_MAX * sizeof(int2) <= sizeof(rows_s), "the sequences' work fits");
  __shared__ float fac_s[RW][PARS];  // what a row's waves are added with

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qw = wave % QW, par = wave / QW;
  const int lr = lane & 15, lg = lane >> 4;
  Place pl;
  bool bad = false;
  const bool mine = find_place<RW, kLeast * PARS, NT>(p, blockIdx.x, (int2 *)rows_s, &pl, &bad);
  if (bad && blockIdx.x == 0) atomicOr(p.status, PPD_DEV_BAD_LENGTH);
  if (!mine) {
    // (of a call without work: what the second launch reads of each sequence)
    if (!JOIN && blockIdx.x == 0)
      for (int s = tid; s < p.sq.B; s += NT) p.rec[s] = int2{0, 0};
    return;
  }
  const int sq = __builtin_amdgcn_readfirstlane(pl.sq), KS = __builtin_amdgcn_readfirstlane(pl.KS);
  const int t0 = __builtin_amdgcn_readfirstlane(pl.q.t0), T = __builtin_amdgcn_readfirstlane(pl.q.T);
  const int L = __builtin_amdgcn_readfirstlane(pl.q.L);
  const int n4 = __builtin_amdgcn_readfirstlane(pl.w.n4), nblk = __builtin_amdgcn_readfirstlane(pl.w.nblk);
  const int n_grp = __builtin_amdgcn_readfirstlane(pl.w.grps);
  const int part0 = __builtin_amdgcn_readfirstlane(pl.part0);
  const int local = __builtin_amdgcn_readfirstlane(pl.local);
  const int bits = __builtin_amdgcn_readfirstlane(pl.bits);
  if (!JOIN && local == 0 && tid == 0) p.rec[sq] = int2{KS, part0};
  const int G = p.nh / p.nkv, R = T * G;
  // row groups that read the same keys are nkv KS workgroups apart: mostly on one
  // XCD, whose cache then holds them
  const int ranges = p.nkv * KS, grp = local / ranges, kvh = local % ranges / KS, ks = local % KS;
  const int my_part = part0 + (kvh * n_grp + grp) * KS + ks;  // its place among those that leave partial rows
  const int chunk = (nblk + KS - 1) / KS;  // (the last splits may be left without blocks)
  const int b0 = min(nblk, ks * chunk), b1 = min(nblk, b0 + chunk);
  const int row0 = grp * RW;
  const int lb = p.sq.lp - 5, n_pages = p.sq.n_pages;
  const int last_page = max(0, ((L + (1 << p.sq.lp) - 1) >> p.sq.lp) - 1);
  const int32_t *table = p.sq.table + (size_t)sq * p.sq.max_pages;
  const int32_t *sel = p.sel ? p.sel + ((size_t)sq * p.nkv + kvh) * p.budget : nullptr;
  const unsigned char *pages = p.pages + (size_t)kvh * ((size_t)kPBytes << lb);
  const size_t page_bytes = (size_t)p.nkv * ((size_t)kPBytes << lb);

  // the workgroup's blocks: n_pre of the prefix, from b0 on, then n_new of new rows
  const int n_pre = max(0, min(b1, n4) - b0), n_new = b1 - b0 - n_pre, first_new = max(0, b0 - n4);
  auto block_at = [&](int j) {  // past the last: the first again (the same loads on every path)
    return min(b0, max(0, n4 - 1)) + (j < n_pre ? j : 0);
  };
  // a block's page by its place in the table, then the block's address
  auto place_of = [&](int blk) {
    const int i = blk >> lb;
    return sel ? max(0, min(uniform_load(sel, i), last_page)) : i;
  };
  auto address_of = [&](int blk, int place) {
    const int page = paged_clamp(uniform_load(table, place), n_pages);
    return pages + (size_t)page * page_bytes + (size_t)(blk & ((1 << lb) - 1)) * kPBytes;
  };
  u32x4 kf[2][4], vf[8];
  auto load_keys = [&](const unsigned char *src) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int ds = 0; ds < 4; ++ds) kf[t][ds] = load_page<QW == 1>(src + (t * 4 + ds) * 1024 + lane * 16);
  };
  auto load_values = [&](const unsigned char *src) {
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) vf[dt] = load_page<QW == 1>(src + 2 * kPElems + dt * 1024 + lane * 16);
  };
  int j = par;  // of the workgroup's blocks
  int blk = block_at(j), next = block_at(j + PARS), place = 0, next_place = 0;
  if (n4 > 0) {
    place = place_of(blk);
    next_place = place_of(next);
    const unsigned char *addr = address_of(blk, place);
    load_keys(addr);
    load_values(addr);
  }
  __builtin_amdgcn_sched_barrier(0);

  PTile rt[NQ];
  u32x4 qr[4][QP];  // the queries, where registers hold them
  const int n_live = min(NQ, ((min(R - row0, RW) + 15) / 16 - qw + QW - 1) / QW);
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int r = row0 + (qw + QW * i) * 16 + lr, rc = min(r, R - 1);
    const int t = rc / G, tok = t0 + t, head = kvh * G + rc % G;
    const bool live = r < R;
    u32x4 q[4][QP];
    load_query<QT>(p, tok, head, lg, q);
    uint64_t m0, m1;
    if (p.mask) {
      m0 = p.mask[2 * (size_t)tok];
      m1 = p.mask[2 * (size_t)tok + 1];
    } else {  // its sequence's rows up to itself
      m0 = t >= 63 ? ~0ull : (2ull << t) - 1;
      m1 = t < 64 ? 0ull : t >= 127 ? ~0ull : (2ull << (t - 64)) - 1;
    }
    rt[i].mk0 = live ? m0 : 0ull;
    rt[i].mk1 = live ? m1 : 0ull;
#pragma unroll
    for (int ds = 0; ds < 4; ++ds)
#pragma unroll
      for (int part = 0; part < QP; ++part) {
        if constexpr (!QLDS)
          qr[ds][part] = q[ds][part];
        else if (par == 0)
          q_s[(((qw + QW * i) * 4 + ds) * QP + part) * 64 + lane] = q[ds][part];
      }
    if constexpr (QLDS) __builtin_amdgcn_sched_barrier(0);  // (registers: a tile's queries at a time)
  }
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) rt[i].o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    rt[i].m_run = -INFINITY;
    rt[i].l_run = 0.f;
  }
  if constexpr (QLDS) __syncthreads();  // the queries are in LDS
  auto query = [&](int i, int ds, int part) {
    if constexpr (!QLDS)
      return as_bf16x8(qr[ds][part]);
    else
      return as_bf16x8(q_s[(((qw + QW * i) * 4 + ds) * QP + part) * 64 + lane]);
  };
  const float c = p.scale_log2;
  // S^T of a block's keys, smallest parts first
  auto scores = [&](float (&sv)[NQ][8]) {
    floatx4 acc[NQ][2];
#pragma unroll
    for (int i = 0; i < NQ; ++i) acc[i][0] = acc[i][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int part = QP - 1; part >= 0; --part) {
#pragma unroll
      for (int ds = 0; ds < 4; ++ds)
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          const bf16x8 q = query(i, ds, part);
          acc[i][0] = mfma16x16x32(as_bf16x8(kf[0][ds]), q, acc[i][0]);
          acc[i][1] = mfma16x16x32(as_bf16x8(kf[1][ds]), q, acc[i][1]);
        }
      if constexpr (QLDS && QP > 1) __builtin_amdgcn_sched_barrier(0);  // (registers: one part's queries at a time)
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) sv[i][u] = acc[i][u >> 2][u & 3];
  };
  // O^T += V^T P^T of its values
  auto products = [&](const u32x4 (&pf)[NQ][PP]) {
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
      for (int part = PP - 1; part >= 0; --part)
#pragma unroll
        for (int i = 0; i < NQ; ++i)
          rt[i].o[dt] = mfma16x16x32(as_bf16x8(vf[dt]), as_bf16x8(pf[i][part]), rt[i].o[dt]);
  };

  if (n_live > 0) {
    for (; j < n_pre; j += PARS) {
      // the next block's address, the place of the one after it
      const unsigned char *addr = address_of(next, next_place);
      const int after = block_at(j + 2 * PARS), after_place = place_of(after);
      float sv[NQ][8];
      scores(sv);
      __builtin_amdgcn_sched_barrier(0);
      load_keys(addr);
      __builtin_amdgcn_sched_barrier(0);
      const int pos = (place << p.sq.lp) + (blk & ((1 << lb) - 1)) * kPB;
      const int vis = L - pos - 8 * lg;  // the lane's keys below the length
      if (pos + kPB > L) {  // the prefix ends in this block, or before it
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
          for (int u = 0; u < 8; ++u) sv[i][u] = u < vis ? sv[i][u] : -INFINITY;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)  // (0 times what lies there may be NaN)
#pragma unroll
          for (int w = 0; w < 4; ++w) vf[dt][w] &= (2 * w < vis ? 0xffffu : 0u) | (2 * w + 1 < vis ? 0xffff0000u : 0u);
      }
      u32x4 pf[NQ][PP];
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        float pv[8];
        softmax_step(rt[i], sv[i], c, pv);
        split8<PP>(pv, pf[i]);
      }
      __builtin_amdgcn_sched_barrier(0);
      products(pf);
      __builtin_amdgcn_sched_barrier(0);
      load_values(addr);
      __builtin_amdgcn_sched_barrier(0);
      blk = next;
      next = after;
      place = next_place;
      next_place = after_place;
    }
    // the new rows, straight from the tail
    const bf16_t *tk = p.tk + (size_t)kvh * p.tcap * 128, *tv = p.tv + (size_t)kvh * 128 * p.tcap;
    for (; j < n_pre + n_new; j += PARS) {
      const int k0 = (first_new + j - n_pre) * kPB;
      const int j0 = k0 + 8 * lg, keep_n = max(0, min(8, T - j0));  // keys of the lane that exist
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16_t *row = tk + (size_t)min(t0 + k0 + paged_key_of(t, lr), p.tcap - 1) * 128 + lg * 8;
#pragma unroll
        for (int ds = 0; ds < 4; ++ds) kf[t][ds] = *(const u32x4 *)(row + ds * 32);
      }
      // (a sequence's rows start anywhere: elements one by one where not by eights)
      const int c0 = t0 + j0;
      if (t0 % 8 == 0) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
          vf[dt] = *(const u32x4 *)(tv + (size_t)(16 * dt + lr) * p.tcap + min(c0, p.tcap - 8));
      } else {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          const bf16_t *row = tv + (size_t)(16 * dt + lr) * p.tcap;
#pragma unroll
          for (int w = 0; w < 4; ++w)
            vf[dt][w] = row[min(c0 + 2 * w, p.tcap - 1)] | (uint32_t)row[min(c0 + 2 * w + 1, p.tcap - 1)] << 16;
          if (dt & 1) __builtin_amdgcn_sched_barrier(0);  // (registers: 16 elements at a time)
        }
      }
      float sv[NQ][8];
      scores(sv);
      u32x4 pf[NQ][PP];
      uint32_t seen[NQ];
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const uint64_t win = j0 >= 128 ? 0ull : j0 >= 64 ? rt[i].mk1 >> (j0 - 64) : rt[i].mk0 >> j0;
        seen[i] = (uint32_t)win & ((1u << keep_n) - 1u);
#pragma unroll
        for (int u = 0; u < 8; ++u) sv[i][u] = (seen[i] >> u) & 1u ? sv[i][u] : -INFINITY;
        float pv[8];
        softmax_step(rt[i], sv[i], c, pv);
        split8<PP>(pv, pf[i]);
      }
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
      products(pf);
    }
  }

  if constexpr (QLDS) __syncthreads();  // the queries' LDS is free
  // ---- the waves meet in LDS: thread -> row tid / 32 + 16 n, dims 4 (tid % 32) .. + 3
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const float l = quad_sum(rt[i].l_run);
    if (i < n_live) {
      float *row = rows_s[par][(qw + QW * i) * 16 + lr];
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *(floatx4 *)(row + dt * 16 + lg * 4) = rt[i].o[dt];
      if (lg == 0) *(float2 *)(row + 128) = float2{rt[i].m_run, l};
    }
  }
  __syncthreads();
  const int n_rows = min(R - row0, RW);
  const size_t part0_at = (size_t)my_part * RW * OROW;  // (only with several splits)
  const __amdgpu_buffer_rsrc_t far = rsrc_of(p.part, JOIN ? kPagedParts * RW * OROW * (uint32_t)sizeof(float) : 0);
  if (tid < n_rows) {
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
      f[w] = factor_of(ml[w], M);
      l += f[w] * ml[w].y;
    }
    const float inv = KS > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int w = 0; w < PARS; ++w) fac_s[tid][w] = f[w] * inv;
    if (KS > 1) {
      if constexpr (JOIN)
        put_far(far, part0_at + (size_t)tid * OROW + 128, floatx4{M, l, 0.f, 0.f});
      else
        *(float2 *)(p.part + part0_at + (size_t)tid * OROW + 128) = float2{M, l};
    } else if (p.lse) {
      const int r = row0 + tid;
      p.lse[(size_t)(t0 + r / G) * p.nh + kvh * G + r % G] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
    }
  }
  __syncthreads();
  const int d4 = (tid & 31) * 4;
#pragma unroll 2
  for (int rl = tid >> 5; rl < n_rows; rl += NT / 32) {
    floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < PARS; ++w) o += fac_s[rl][w] * *(const floatx4 *)(rows_s[w][rl] + d4);
    if (KS > 1) {
      if constexpr (JOIN)
        put_far(far, part0_at + (size_t)rl * OROW + d4, o);
      else
        *(floatx4 *)(p.part + part0_at + (size_t)rl * OROW + d4) = o;
    } else {
      const int r = row0 + rl;
      store_out4<QT>(p, t0 + r / G, kvh * G + r % G, d4, o);
    }
  }
  if constexpr (JOIN) {
    if (KS == 1) return;
    // ---- the last of the splits to arrive adds them all, in a fixed order
    __shared__ int last_s;
    __builtin_amdgcn_s_waitcnt(0);  // this thread's rows are in memory
    __syncthreads();
    if (tid == 0) {
      const SplitCounter c = split_counter(my_part - ks, KS, bits);
      uint32_t *ctr = p.ctr + c.word;
      const uint32_t n = __hip_atomic_fetch_add(ctr, 1u << c.shift, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) >> c.shift & c.mask;
      last_s = n + 1 == (uint32_t)KS;
      if (last_s) __hip_atomic_fetch_sub(ctr, (uint32_t)KS << c.shift, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last_s) return;
    const size_t first_at = (size_t)(my_part - ks) * RW * OROW;
    constexpr size_t stride = (size_t)RW * OROW;
    // 32 threads a row; of few rows several such groups share one (ways), of more
    // than eight a group takes two at a time.  A round of splits is requested for
    // both, and beside the first the splits' maxima and sums, of which LDS gets the
    // factors
    constexpr int GR = NT / 32, N = 8;
    const int ways = n_rows >= 5 ? 1 : n_rows >= 3 ? GR / 4 : n_rows == 2 ? GR / 2 : GR;
    const int group = tid >> 5, sub = group % ways;
    int rl = group / ways;
    floatx4 x[N], y[N];
    auto two = [&] { return ways == 1 && rl + GR < n_rows; };
    auto request = [&](int s0) {
#pragma unroll
      for (int v = 0; v < N; ++v)
        x[v] = get_far(far, first_at + min(s0 + v * ways, KS - 1) * stride + (size_t)min(rl, n_rows - 1) * OROW + d4);
      if (two())
#pragma unroll
        for (int v = 0; v < N; ++v) y[v] = get_far(far, first_at + min(s0 + v, KS - 1) * stride + (size_t)(rl + GR) * OROW + d4);
    };
    float(*wt_s)[kPagedSplits] = (float(*)[kPagedSplits])rows_s;
    floatx4 *sum_s = (floatx4 *)((char *)rows_s + sizeof(float) * RW * kPagedSplits);  // [GR][32]
    constexpr int TR = NT / RW;  // threads a row
    static_assert(TR <= 64 && kPagedSplits % TR == 0 && sizeof(float) * RW * kPagedSplits + GR * 512 <= sizeof(rows_s), "they fit");
    {
      const int row = tid / TR, j0 = tid % TR;
      floatx4 ml[kPagedSplits / TR];
      float M = -INFINITY, l = 0.f;
#pragma unroll
      for (int j = 0; j < kPagedSplits / TR; ++j)
        ml[j] = row < n_rows && j0 + TR * j < KS ? get_far(far, first_at + (j0 + TR * j) * stride + (size_t)row * OROW + 128)
                                                : floatx4{-INFINITY, 0.f, 0.f, 0.f};
      request(sub);
#pragma unroll
      for (int j = 0; j < kPagedSplits / TR; ++j) M = fmaxf(M, ml[j][0]);
#pragma unroll
      for (int o = TR / 2; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
#pragma unroll
      for (int j = 0; j < kPagedSplits / TR; ++j) {
        const float f = factor_of(float2{ml[j][0], ml[j][1]}, M);
        l += f * ml[j][1];
        if (j0 + TR * j < KS) wt_s[row][j0 + TR * j] = f;
      }
#pragma unroll
      for (int o = TR / 2; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
      if (j0 == 0 && row < n_rows) {
        fac_s[row][0] = l == 0.f ? 0.f : 1.f / l;
        const int r = row0 + row;
        if (p.lse) p.lse[(size_t)(t0 + r / G) * p.nh + kvh * G + r % G] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
      }
    }
    __syncthreads();
    auto store = [&](int row, floatx4 v) {
      const int r = row0 + row;
      store_out4<QT>(p, t0 + r / G, kvh * G + r % G, d4, v * fac_s[row][0]);
    };
    for (bool first = true; first || rl < n_rows; first = false, rl += 2 * GR) {
      floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f}, o2 = o;
      const int row = min(rl, n_rows - 1);
      for (int s0 = sub; s0 < KS; s0 += N * ways) {
        if (!first || s0 != sub) request(s0);
#pragma unroll
        for (int v = 0; v < N; ++v)
          if (s0 + v * ways < KS) o += wt_s[row][s0 + v * ways] * x[v];
        if (two())
#pragma unroll
          for (int v = 0; v < N; ++v)
            if (s0 + v < KS) o2 += wt_s[rl + GR][s0 + v] * y[v];
      }
      if (ways == 1) {
        if (rl < n_rows) store(rl, o);
        if (two()) store(rl + GR, o2);
        continue;
      }
      sum_s[group * 32 + (tid & 31)] = o;  // (a single round: few rows)
      __syncthreads();
      if (sub == 0 && rl < n_rows) {
        for (int w = 1; w < ways; ++w) o += sum_s[(group + w) * 32 + (tid & 31)];
        store(rl, o);
      }
      return;
    }
  }
}

// the splits of a row, added in order; 32 threads a row
template <int QT>
__global__ __launch_bounds__(NT) void paged_merge_kernel(PagedAttnLaunch p, int RW) {
  const int64_t first = (int64_t)blockIdx.x * (NT / 32) + 2 * (threadIdx.x >> 6);  // the wave's first row
  const int64_t n_rows = (int64_t)p.sq.n_rows * p.nh;
  const int d4 = (threadIdx.x & 31) * 4;
  int sq = -1, tok = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t at = first + h;
    if (at >= n_rows) break;
    const int t = (int)(at / p.nh), s = paged_seq_of(p.sq.row_start, p.sq.B, t);
    if ((int)(threadIdx.x >> 5 & 1) == h) sq = s, tok = t;
  }
  if (sq < 0) return;
  bool bad = false;
  const PagedSeq q = paged_seq(p.sq, sq, &bad);
  const int2 rec = p.rec[sq];
  const int head = (int)(first + (threadIdx.x >> 5 & 1) - (int64_t)tok * p.nh), t = tok - q.t0;
  const int KS = rec.x, G = p.nh / p.nkv;
  if (t < 0 || t >= q.T || KS <= 1) return;  // no sequence's row, or already final
  const int kvh = head / G, r = t * G + head % G, grps = (q.T * G + RW - 1) / RW;
  const int slot0 = rec.y + (kvh * grps + r / RW) * KS;
  const float *part = p.part + ((size_t)slot0 * RW + r % RW) * OROW;
  const size_t stride = (size_t)RW * OROW;
  constexpr int N = 8;  // rows in flight: one round trip for all of them
  float M = -INFINITY, l = 0.f;
  floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < KS; s0 += N) {
    float2 ml[N];
    floatx4 x[N];
#pragma unroll
    for (int v = 0; v < N; ++v) {
      const float *row = part + min(s0 + v, KS - 1) * stride;
      ml[v] = *(const float2 *)(row + 128);
      x[v] = *(const floatx4 *)(row + d4);
    }
    __builtin_amdgcn_sched_barrier(0);
    float m = M;
#pragma unroll
    for (int v = 0; v < N; ++v) m = fmaxf(m, ml[v].x);  // (the last row repeats)
    const float keep = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - m);
    o *= keep;
    l *= keep;
    M = m;
#pragma unroll
    for (int v = 0; v < N; ++v) {
      const float f = factor_of(ml[v], M);
      l += s0 + v < KS ? f * ml[v].y : 0.f;
      if (s0 + v < KS) o += f * x[v];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store_out4<QT>(p, tok, head, d4, o * inv);
  if (p.lse && d4 == 0) p.lse[(size_t)tok * p.nh + head] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
}

}  // namespace

// tiles a wave holds, waves side by side and over blocks, by the tiles of a workgroup
struct Shape {
  int nq, qw, pars;
  int rows() const { return 16 * nq * qw; }
};
static Shape paged_shape(int tiles) {
  return tiles == 1 ? Shape{1, 1, 4} : tiles == 2 ? Shape{2, 1, 4} : tiles == 4 ? Shape{2, 2, 4} : Shape{2, 4, 2};
}
// 16-row tiles of a kv head's rows (of an average sequence: how many a single one
// has is only known on the device, and any shape serves any number)
static int paged_tiles(int nh, int nkv, int B, int n_rows) {
  const int64_t rows = std::min<int64_t>((n_rows + B - 1) / B, PPD_T_MAX) * (nh / nkv);
  return (int)std::min<int64_t>(64, (rows + 15) / 16);
}
// Tiles of a workgroup, by the blocks that one would read with a tile or two of its
// own.  While they are few the tiles of a kv head read its keys from the XCD's
// cache beside one another, which is less than what more tiles in a workgroup cost
// in registers, LDS and meeting; with many a compute unit's load path (it holds 32
// KB of loads, some 50 GB/s) is the bound, and wide workgroups read every block once.
// us, by tiles of a workgroup 1, 2, 4 or 8: 32 heads of 64 nodes, 1024 positions 16.0,
// 18.1, 19.9; 4096 29.3, 26.1, 29.5; 32768 166, 121, 111; of 128 nodes 2048 25.3, 24.8,
// 28.9; 8192 74, 60, 52; of 32 nodes 2000 16.3, 20.9; 4096 22.4, 26.3; 8192 34.3, 36.3;
// 16384 58.3, 57.0.  The limits are alike for all numbers of tiles, so that 32 nodes get
// two from 6100 positions on, where they lose 6 %: 64 nodes over 4096, which are as many
// blocks, gain 10.  Blocks are those of the tables' width: short prefixes in wide tables
// are read in the shape of long ones (32 nodes over 2048 positions 15.8 us, from a table of
// 8192 on 20.4; 64 over 1024 15.6, from 4096 on 18.0, from 32768 on 18.9)
constexpr int64_t kOwnTileBlocks = 48, kTwoTileBlocks = 96;
static int paged_width(int tiles, int64_t blocks_of_a_tile) {
  const int64_t two = blocks_of_a_tile * ((tiles + 1) / 2), one = blocks_of_a_tile * tiles;
  if (tiles == 1 || one <= kOwnTileBlocks * kPagedSlots) return 1;
  return tiles == 2 || two <= kTwoTileBlocks * kPagedSlots ? 2 : tiles <= 4 ? 4 : 8;
}

size_t paged_attn_part_bytes(int nh, int nkv, int B, int n_rows) {
  const int tiles = paged_tiles(nh, nkv, B, n_rows);  // (of the widest workgroup it may become)
  const Shape sh = paged_shape(tiles <= 2 ? tiles : tiles <= 4 ? 4 : 8);
  return (size_t)kPagedParts * sh.rows() * OROW * sizeof(float);
}

void paged_attn_shape(PagedAttnLaunch &a) {
  const int most = a.sel ? std::min(a.budget, a.sq.max_pages) : a.sq.max_pages;
  const int64_t blocks = ((int64_t)most << (a.sq.lp - 5)) + 1;
  a.tiles = paged_width(paged_tiles(a.nh, a.nkv, a.sq.B, a.sq.n_rows), blocks * a.nkv * std::min(a.sq.B, a.sq.n_rows));
  a.may_split = blocks + PPD_T_MAX / kPB > kLeast * paged_shape(a.tiles).pars;
}

template <int QT>
static hipError_t launch_attn(const PagedAttnLaunch &a, hipStream_t s) {
  auto kernel = a.tiles == 1   ? paged_attention_kernel<1, 1, 4, QT>
                : a.tiles == 2 ? paged_attention_kernel<2, 1, 4, QT>
                : a.tiles == 4 ? paged_attention_kernel<2, 2, 4, QT>
                               : paged_attention_kernel<2, 4, 2, QT>;
  const Shape sh = paged_shape(a.tiles);
  const int rw = sh.rows();
  // row groups of all sequences at most, and the splits of those that have several
  const int64_t rows = (int64_t)a.sq.n_rows * (a.nh / a.nkv);
  const int64_t units = a.nkv * (std::min<int64_t>(a.sq.B, a.sq.n_rows) + rows / rw);
  const dim3 grid((unsigned)(units + (a.may_split ? 3 * kPagedSlots / 2 : 0))), block(64 * sh.qw * sh.pars);
  const bool merge = a.may_split && sh.qw > 1;
  const hipEvent_t ev0 = (hipEvent_t)a.ev_start, ev1 = (hipEvent_t)a.ev_stop;
  if (ev0)
    hipExtLaunchKernelGGL(kernel, grid, block, 0, s, ev0, merge ? (hipEvent_t) nullptr : ev1, 0, a);
  else
    hipLaunchKernelGGL(kernel, grid, block, 0, s, a);
  if (merge) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 rows16((unsigned)(((int64_t)a.sq.n_rows * a.nh + NT / 32 - 1) / (NT / 32)));
    if (ev1)
      hipExtLaunchKernelGGL(paged_merge_kernel<QT>, rows16, dim3(NT), 0, s, (hipEvent_t) nullptr, ev1, 0, a, rw);
    else
      hipLaunchKernelGGL(paged_merge_kernel<QT>, rows16, dim3(NT), 0, s, a, rw);
  }
  return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnLaunch &a, hipStream_t s) {
  return a.q_type == PAGED_Q_PLANES ? launch_attn<PAGED_Q_PLANES>(a, s)
         : a.q_type == PAGED_Q_F32  ? launch_attn<PAGED_Q_F32>(a, s)
                                    : launch_attn<PAGED_Q_BF16>(a, s);
}
