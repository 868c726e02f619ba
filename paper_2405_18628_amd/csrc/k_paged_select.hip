// Pages of a long prefix by a score of their key bounds.
//
// A page's keys k of a head lie between its bounds, so a query's product with any
// of them is at most sum_d max(q_d, 0) largest_d + min(q_d, 0) smallest_d; summed
// over the rows and heads that share the choice, with Qp and Qm the sums of their
// positive and negative parts, it is one product of 256 elements a page whatever
// the number of rows.  Its sums are float64: pages' scores lie close together,
// and whole numbers hang on their order (scores that differ by their roundings alone may
// rank either way).
//
// Scores: a wave takes 16 pages, two at a time (512 bytes of bounds a page, 16
// bytes a lane), the rows of queries and then the bounds requested before either is
// used; every workgroup sums the queries for itself, which takes a third of the
// time with 64 rows of them.  4096 pages of 8 heads, 64 rows 10.5 us, 8 sequences
// of up to 512 pages, 32 heads 8.1 (27 MB in pieces of 512 bytes, one row each).
// With 32 pages a wave 3 us slower.
// Selection: a workgroup for each (sequence, kv head) narrows the threshold among
// the scores' ordered 64-bit keys 8 bits at a time, from the first bit in which
// any two differ on (scores share sign and most of the exponent), and compares the
// last 64 or fewer with each other.  4097 pages 7.0 us, 513 or 125 pages 5.0, half
// of it launch and first loads.  One launch for both, the last workgroup of a head
// selecting, took 27.7 us for 17.6 (4096 pages): its 256 threads hold 16 keys each.
#include <algorithm>

#include "ppd_paged.h"

namespace {

typedef unsigned long long u64;

constexpr int ST = 256;    // threads of the scores' workgroup
constexpr int PAGES = 16;  // pages of a wave
constexpr int CH = PAGES * (ST / 64);

constexpr u64 kKept = ~0ull;  // the key of a page that is always taken: no number's

// the order of numbers as unsigned keys; NaN below every number
__device__ __forceinline__ u64 key_of(double v) {
  if (v != v) return 0;
  const u64 b = __builtin_bit_cast(u64, v + 0.0);  // -0 as 0
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

// elements d, d + 1 of a query row
template <int QT>
__device__ __forceinline__ float2 query2(const PagedSelectLaunch &p, int tok, int head, int d) {
  auto pair = [](uint32_t w) { return float2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)}; };
  if constexpr (QT == PAGED_Q_F32) return *(const float2 *)((const float *)p.q + ((size_t)tok * p.nh + head) * 128 + d);
  if constexpr (QT == PAGED_Q_BF16) return pair(*(const uint32_t *)((const bf16_t *)p.q + ((size_t)tok * p.nh + head) * 128 + d));
  const unsigned char *src = (const unsigned char *)p.q + plane_off(p.T_pad >> 4, tok, head * 128 + d);
  const float2 hi = pair(*(const uint32_t *)src), lo = pair(*(const uint32_t *)(src + kPlaneLo));
  return float2{hi.x + lo.x, hi.y + lo.y};
}

template <int QT>
__global__ __launch_bounds__(ST) void paged_score_kernel(PagedSelectLaunch p, int chunks) {
  __shared__ double sum_s[ST / 64][2][128];
  __shared__ double q_s[2][128];  // Qm, Qp
  const int tid = threadIdx.x, lane = tid & 63;
  const int c = blockIdx.x % chunks, kvh = blockIdx.x / chunks % p.nkv, sq = blockIdx.x / chunks / p.nkv;
  const int page0 = c * CH + (tid >> 6) * PAGES;
  // (the table's entries are requested beside the length)
  const int32_t *table = p.sq.table + (size_t)sq * p.sq.max_pages;
  const int entry = table[min(page0 + (lane & (PAGES - 1)), p.sq.max_pages - 1)];
  bool bad = false;  // (the selection, which every call launches, reports it)
  const PagedSeq s = paged_seq(p.sq, sq, &bad);
  const int n = (s.L + (1 << p.sq.lp) - 1) >> p.sq.lp;
  if (n <= p.budget || c * CH >= n) return;  // all are taken
  // ---- sums of the queries' positive and negative parts; the first rows and then the
  // bounds are requested before either is used
  const int G = p.nh / p.nkv, R = s.T * G, wave = tid >> 6;
  const uint32_t inv = G > 1 ? 0xffffffffu / G + 1 : 0;
  constexpr int QB = 16;  // rows of a wave in flight
  float2 x[QB];
  auto request = [&](int r0) {
#pragma unroll
    for (int u = 0; u < QB; ++u) {
      const int r = r0 + u * (ST / 64);
      if (r >= R) break;
      int t = G > 1 ? (int)__umulhi((uint32_t)r, inv) : r;  // r / G
      t -= t * G > r;
      x[u] = query2<QT>(p, s.t0 + t, kvh * G + r - t * G, 2 * lane);
    }
  };
  request(wave);
  __builtin_amdgcn_sched_barrier(0);
  const int phys = paged_clamp(entry, p.sq.n_pages);
  u32x4 w[PAGES / 2];
#pragma unroll
  for (int i = 0; i < PAGES / 2; ++i) {
    const int page = __shfl(phys, 2 * i + (lane >> 5), 64);
    w[i] = *(const u32x4 *)(p.bounds + ((size_t)page * p.nkv + kvh) * 256 + (lane & 31) * 8);
  }
  __builtin_amdgcn_sched_barrier(0);
  double qp[2] = {0.0, 0.0}, qm[2] = {0.0, 0.0};
  for (int r0 = wave; r0 < R; r0 += QB * (ST / 64)) {
    if (r0 != wave) request(r0);
#pragma unroll
    for (int u = 0; u < QB; ++u) {
      if (r0 + u * (ST / 64) >= R) break;
      qp[0] += (double)(x[u].x <= 0.f ? 0.f : x[u].x);  // (a NaN stays one)
      qp[1] += (double)(x[u].y <= 0.f ? 0.f : x[u].y);
      qm[0] += (double)(x[u].x >= 0.f ? 0.f : x[u].x);
      qm[1] += (double)(x[u].y >= 0.f ? 0.f : x[u].y);
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    sum_s[wave][0][2 * lane + e] = qm[e];
    sum_s[wave][1][2 * lane + e] = qp[e];
  }
  __syncthreads();
  {
    double x = 0.0;
#pragma unroll
    for (int i = 0; i < ST / 64; ++i) x += sum_s[i][tid >> 7][tid & 127];
    q_s[tid >> 7][tid & 127] = x;
  }
  __syncthreads();
  double q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = q_s[lane >> 4 & 1][(lane & 15) * 8 + e];
  // ---- products, summed over a page's 32 lanes
  double v[PAGES / 2];
#pragma unroll
  for (int i = 0; i < PAGES / 2; ++i) {
    double x = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      x = fma(q[e], (double)__uint_as_float(e & 1 ? w[i][e >> 1] & 0xffff0000u : w[i][e >> 1] << 16), x);
    v[i] = x;
  }
  // each step halves the pages a lane holds; which it is left with, its bits say
  constexpr int NV = PAGES / 2;
  int i = 0;
#pragma unroll
  for (int half = NV / 2, o = 16; half > 0; half /= 2, o /= 2) {
    const bool up = lane & o;
#pragma unroll
    for (int j = 0; j < half; ++j) {
      const double mine = up ? v[j + half] : v[j], other = up ? v[j] : v[j + half];
      v[j] = mine + __shfl_xor(other, o, 64);
    }
    i = 2 * i + up;
  }
  double score = v[0];
#pragma unroll
  for (int o = 16 / NV; o > 0; o /= 2) score += __shfl_xor(score, o, 64);
  const int page = page0 + 2 * i + (lane >> 5);
  if (lane % (32 / NV) == 0 && page < n) {
    const bool kept = page < p.n_first || page >= n - p.n_last;
    p.keys[((size_t)sq * p.nkv + kvh) * p.sq.max_pages + page] = kept ? kKept : key_of(score);
  }
}

// KT threads, REG keys of each in registers; of more, the passes read them again
template <int KT, int REG>
__global__ __launch_bounds__(KT) void paged_pick_kernel(PagedSelectLaunch p) {
  constexpr int KW = KT / 64;
  __shared__ uint32_t red_s[2][KW];
  __shared__ u64 list_s[64], pick_s;
  __shared__ unsigned hist_s[256];
  __shared__ int cnt_s[2][REG][KW], bin_s, above_s, in_s, n_list;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kvh = blockIdx.x % p.nkv, sq = blockIdx.x / p.nkv;
  const u64 *keys = p.keys + ((size_t)sq * p.nkv + kvh) * p.sq.max_pages;
  u64 kr[REG];  // (requested before the length is known: of this head's keys, or its last one)
#pragma unroll
  for (int j = 0; j < REG; ++j) kr[j] = keys[min(j * KT + tid, p.sq.max_pages - 1)];
  bool bad = false;
  const PagedSeq s = paged_seq(p.sq, sq, &bad);
  const int n = (s.L + (1 << p.sq.lp) - 1) >> p.sq.lp;
  int32_t *sel = p.sel + ((size_t)sq * p.nkv + kvh) * p.budget;
  if (kvh == 0 && tid == 0) {
    p.n_sel[sq] = min(n, p.budget);
    if (bad) atomicOr(p.status, PPD_DEV_BAD_LENGTH);
  }
  if (n <= p.budget) {
    for (int i = tid; i < n; i += KT) sel[i] = i;
    return;
  }
  const int rounds = (n + KT - 1) / KT;
  // f(key, index) of this thread's pages that are ranked
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < REG; ++j)
      if (j * KT + tid < n && kr[j] != kKept) f(kr[j]);
    for (int j = REG; j < rounds; ++j) {
      const int i = j * KT + tid;
      const u64 k = keys[min(i, n - 1)];
      if (i < n && k != kKept) f(k);
    }
  };
  // ---- the bits in which ranked keys' upper halves differ
  uint32_t all = ~0u, any = 0;
  each([&](u64 k) { all &= (uint32_t)(k >> 32), any |= (uint32_t)(k >> 32); });
  all = wave_all(all, [](uint32_t a, uint32_t b) { return a & b; });
  any = wave_all(any, [](uint32_t a, uint32_t b) { return a | b; });
  if (lane == 0) red_s[0][wave] = all, red_s[1][wave] = any;
  if (KT == 256 || tid < 256) hist_s[tid] = 0;
  if (tid == 0) n_list = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < KW; ++i) all &= red_s[0][i], any |= red_s[1][i];
  // ---- the threshold: keys whose bits from `shift` up are above `prefix` are taken,
  // of those that equal it `left` (from the smallest index on)
  const int kept = min(n, p.n_first) + min(max(0, n - p.n_first), p.n_last);
  int shift = 64 - __builtin_clz((all ^ any) | 1), left = p.budget - kept;
  u64 prefix = shift == 64 ? 0 : (u64)all << 32 >> shift;
  bool split = left > 0;  // of the keys at the threshold some are taken, or none at all
  while (split && shift > 0) {
    const int bits = min(8, shift), low = shift - bits;
    each([&](u64 k) {
      if (shift == 64 || k >> shift == prefix) atomicAdd(&hist_s[(k >> low) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    if (wave == 0) {  // lane: bins 255 - 4 lane .. 252 - 4 lane, the largest first
      int h[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += h[j] = (int)hist_s[255 - 4 * lane - j];
      int before = wave_incl(sum) - sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < left && before + h[j] >= left) {
          bin_s = 255 - 4 * lane - j;
          above_s = before;
          in_s = h[j];
        }
        before += h[j];
        hist_s[255 - 4 * lane - j] = 0;
      }
    }
    __syncthreads();
    left -= above_s;
    split = in_s != left;
    prefix = (shift == 64 ? 0 : prefix << bits) | (u64)bin_s;
    shift = low;
    if (split && shift > 0 && in_s <= 64) {
      // a wave's worth of keys at the threshold: the left-th largest of them
      each([&](u64 k) {
        if (k >> shift == prefix) list_s[atomicAdd(&n_list, 1)] = k;
      });
      __syncthreads();
      if (wave == 0) {
        const u64 mine = list_s[min(lane, in_s - 1)];
        int above = 0, same = 0;
        for (int i = 0; i < in_s; ++i) {
          const u64 k = list_s[i];
          above += k > mine;
          same += k == mine;
        }
        if (lane < in_s && above < left && above + same >= left) {  // (alike in all lanes that hold it)
          pick_s = mine;
          above_s = above;
        }
      }
      __syncthreads();
      prefix = pick_s;
      left -= above_s;
      shift = 0;
    }
  }
  // ---- the taken pages in order, REG rounds of them at a time
  int done = 0, ties = 0;  // written, and met at the threshold, before
  for (int r0 = 0; r0 < rounds; r0 += REG) {
    if (r0 > 0) {
#pragma unroll
      for (int j = 0; j < REG; ++j) kr[j] = keys[min((r0 + j) * KT + tid, n - 1)];
      __syncthreads();  // the counts of the rounds before are read
    }
    u64 tb[REG], ab[REG];  // the wave's pages at and above the threshold
#pragma unroll
    for (int j = 0; j < REG; ++j) {
      const bool on = (r0 + j) * KT + tid < n;
      const u64 top = shift == 64 ? 0 : kr[j] >> shift;
      tb[j] = __ballot(on && kr[j] != kKept && top == prefix);
      ab[j] = __ballot(on && (kr[j] == kKept || top > prefix));
      if (lane == 0) cnt_s[0][j][wave] = __popcll(tb[j]), cnt_s[1][j][wave] = __popcll(ab[j]);
    }
    __syncthreads();
    // counts before each (round, wave): lane: entries lane and 64 + lane
    constexpr int E = REG * KW;
    static_assert(E <= 128 && (E < 64 || E % 64 == 0), "two counts a lane");
    const int *tie_n = &cnt_s[0][0][0], *over_n = &cnt_s[1][0][0];
    const int t0 = lane < E ? tie_n[min(lane, E - 1)] : 0, t1 = E > 64 ? tie_n[64 % E + lane % (E / 2)] : 0;
    const int a0 = lane < E ? over_n[min(lane, E - 1)] : 0, a1 = E > 64 ? over_n[64 % E + lane % (E / 2)] : 0;
    const int ti0 = wave_incl(t0), ti1 = wave_incl(t1) + lane_of(ti0, 63);
    // of a group of ties, those below `left` are taken
    auto taken = [&](int upto, int n_ties) { return max(0, min(n_ties, left - (ties + upto - n_ties))); };
    const int b0 = a0 + taken(ti0, t0), b1 = a1 + taken(ti1, t1);
    const int bi0 = wave_incl(b0), bi1 = wave_incl(b1) + lane_of(bi0, 63);
#pragma unroll
    for (int j = 0; j < REG; ++j) {
      if (r0 + j >= rounds) break;
      const int from = j * KW % 64 + __builtin_amdgcn_readfirstlane(wave);
      const int t_before = ties + lane_of(j * KW < 64 ? ti0 - t0 : ti1 - t1, from);
      int at = done + lane_of(j * KW < 64 ? bi0 - b0 : bi1 - b1, from);
      const u64 below = (1ull << lane) - 1;
      const int my_ties = __popcll(tb[j] & below);
      const bool tie = tb[j] >> lane & 1, take = (ab[j] >> lane & 1) || (tie && t_before + my_ties < left);
      at += __popcll(ab[j] & below) + max(0, min(my_ties, left - t_before));
      if (take) sel[at] = (r0 + j) * KT + tid;
    }
    ties += lane_of(ti1, 63);
    done += lane_of(bi1, 63);
  }
}

}  // namespace

size_t paged_select_key_bytes(int nkv, int B, int max_pages) { return (size_t)B * nkv * max_pages * sizeof(u64); }

hipError_t launch_paged_select(const PagedSelectLaunch &p, hipStream_t s) {
  if (p.sq.max_pages > p.budget) {
    const int chunks = (p.sq.max_pages + CH - 1) / CH;
    const dim3 grid((unsigned)((int64_t)chunks * p.nkv * p.sq.B));
    auto kernel = p.q_type == PAGED_Q_PLANES ? paged_score_kernel<PAGED_Q_PLANES>
                  : p.q_type == PAGED_Q_F32  ? paged_score_kernel<PAGED_Q_F32>
                                             : paged_score_kernel<PAGED_Q_BF16>;
    hipLaunchKernelGGL(kernel, grid, dim3(ST), 0, s, p, chunks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // (fewer threads start and meet sooner: 125 pages 4.9 us with 256, 6.3 with 1024;
  // of more than a few keys each they take longer: 4097 pages 8.5 us with 512, 7.0 with 1024)
  const bool few = p.sq.max_pages <= 4 * 256;
  hipLaunchKernelGGL((few ? paged_pick_kernel<256, 8> : paged_pick_kernel<1024, 8>), dim3(p.nkv * p.sq.B), dim3(few ? 256 : 1024), 0, s, p);
  return hipGetLastError();
}
