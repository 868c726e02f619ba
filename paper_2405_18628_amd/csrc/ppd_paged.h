// The paged cache (ppd_paged, ppd_page_tables): layout, the division of an
// attention call's work from lengths on the device, and launchers.
#pragma once

#include "ppd_internal.h"

constexpr int kPB = PPD_PAGED_BLOCK;              // positions of a block
constexpr int kPElems = kPB * 128;                // elements of a block's keys (or values)
constexpr int kPBytes = 2 * kPElems * 2;          // bytes of a block: keys, then values

// element of a block's keys, and of its values, at position u (of the block), dim d
__host__ __device__ __forceinline__ int paged_key_at(int u, int d) {
  return ((((u >> 2) & 1) * 4 + (d >> 5)) * 64 + 16 * ((d >> 3) & 3) + 4 * (u >> 3) + (u & 3)) * 8 + (d & 7);
}
__host__ __device__ __forceinline__ int paged_value_at(int u, int d) {
  return ((d >> 4) * 64 + 16 * (u >> 3) + (d & 15)) * 8 + (u & 7);
}
// position (of its block) that row m of key tile t holds
__host__ __device__ __forceinline__ int paged_key_of(int t, int m) { return 8 * (m >> 2) + 4 * t + (m & 3); }

// the sequences as the device sees them
struct PagedSeqs {
  const int32_t *table, *len, *row_start;
  int B, max_pages, n_pages;
  int lp;      // log2 of the page's positions
  int n_rows;  // rows that the call's buffers hold
};

// A sequence's own numbers, clamped so that no index that follows from them
// leaves its buffer; *bad where one had to be.  Where clamped offsets fall (*low below
// zero) rows can be several sequences', and more than n_rows altogether: a call that
// divides work among all of them has to leave it.
struct PagedSeq {
  int t0, T, L;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedSeqs &p, int s, bool *bad, int *low) {
  const int n = p.len[s], a = p.row_start[s], b = p.row_start[s + 1];
  PagedSeq q;
  q.L = max(0, min((int64_t)n, (int64_t)p.max_pages << p.lp));
  q.t0 = max(0, min(a, p.n_rows));
  const int end = max(0, min(b, p.n_rows)), rows = end - q.t0;  // (clamped first: no difference of offsets overflows)
  q.T = max(0, min(rows, PPD_T_MAX));
  *low = min(*low, rows);
  *bad |= n != q.L || a != q.t0 || b != end || rows != q.T;
  return q;
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedSeqs &p, int s, bool *bad) {
  int low = 0;
  return paged_seq(p, s, bad, &low);
}
__device__ __forceinline__ int paged_clamp(int page, int n_pages) { return max(0, min(page, n_pages - 1)); }

// ---- over a wave with cross-lane moves (no LDS round trips): inclusive sums, and
// sums, ands and ors that every lane gets
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int lane_move(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_incl(int v) {
  v += lane_move<0x111>(v);       // row_shr:1, 2, 4, 8
  v += lane_move<0x112>(v);
  v += lane_move<0x114>(v);
  v += lane_move<0x118>(v);
  v += lane_move<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
  v += lane_move<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
  return v;
}
template <typename F>
__device__ __forceinline__ uint32_t wave_all(uint32_t v, F f) {
  v = f(v, (uint32_t)lane_move<0xb1>((int)v));   // quad_perm: pairs, then pairs of pairs
  v = f(v, (uint32_t)lane_move<0x4e>((int)v));
  v = f(v, (uint32_t)lane_move<0x141>((int)v));  // row_half_mirror
  v = f(v, (uint32_t)lane_move<0x140>((int)v));  // row_mirror
  auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(a[0], a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(b[0], b[1]);
}
// (whole numbers below 2^48; 24 bits at a time, so that 64 of them fit)
__device__ __forceinline__ int64_t wave_total(int64_t v) {
  auto add = [](uint32_t a, uint32_t b) { return a + b; };
  int64_t sum = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) sum += (int64_t)wave_all((uint32_t)(v >> 24 * i) & 0xffffffu, add) << 24 * i;
  return sum;
}
__device__ __forceinline__ int64_t wave_incl64(int64_t v) {
  auto step = [&](auto move) {
    const uint32_t lo = (uint32_t)move((int)v), hi = (uint32_t)move((int)(v >> 32));
    v += (int64_t)((uint64_t)hi << 32 | lo);
  };
  step([](int x) { return lane_move<0x111>(x); });
  step([](int x) { return lane_move<0x112>(x); });
  step([](int x) { return lane_move<0x114>(x); });
  step([](int x) { return lane_move<0x118>(x); });
  step([](int x) { return lane_move<0x142, 0xa>(x); });
  step([](int x) { return lane_move<0x143, 0xc>(x); });
  return v;
}
__device__ __forceinline__ int64_t lane_of64(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}
__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// The sequence of a row: the last one whose rows start at or before it.  Called
// by a whole wave, `tok` alike in its lanes.
__device__ __forceinline__ int paged_seq_of(const int32_t *row_start, int B, int tok) {
  int n = 0;
  for (int base = 0; base < B; base += 64) {
    const int s = base + (int)(threadIdx.x & 63);
    n += __popcll(__ballot(s < B && row_start[min(s, B - 1)] <= tok));
  }
  return n - 1;
}

struct PagedTablesLaunch {
  int32_t *table, *free_pages;
  const int32_t *len, *free_state, *add;
  int32_t *len_out, *free_state_out, *start, *slots;
  int B, max_pages, n_pages, lp, n_slots;
  uint32_t *ctr;  // workgroups that have read their inputs; zero between launches
  uint32_t *status;
};
hipError_t launch_paged_tables(const PagedTablesLaunch &p, hipStream_t s);

struct PagedStoreLaunch {
  unsigned char *pages;
  bf16_t *bounds;       // or null
  const bf16_t *k, *v;  // [heads][scap][128], [heads][128][scap]
  int layers, nkv, n_pages, lp, scap;
  int B, n_rows;
  int n_path;
  int rows_each, chunks;  // rows of a part, parts that are workgroups of a head (the launcher's)
  const int32_t *start, *row_start, *path, *slots;
};
hipError_t launch_paged_store(PagedStoreLaunch p, hipStream_t s);

enum { PAGED_Q_BF16 = 0, PAGED_Q_F32 = 1, PAGED_Q_PLANES = 2 };

struct PagedAttnLaunch {
  PagedSeqs sq;
  const unsigned char *pages;  // this layer's
  const bf16_t *tk, *tv;       // this layer's new rows, row i at position i
  int tcap;
  const void *q;               // rows [n_rows][nh][128] of a type, or operand planes
  void *out;                   // likewise
  int q_type, T_pad;
  const uint64_t *mask;        // [n_rows][2], or null: a row sees its sequence's rows up to itself
  float *lse;                  // [n_rows][nh], or null
  const int32_t *sel, *n_sel;  // [B][nkv][budget], [B], or null
  int budget;
  int nh, nkv;
  float *part;                 // [kPagedParts][rows of a workgroup][PPD_ATTN_OROW]
  int2 *rec;                   // [B]: splits, first of the partial rows' workgroups
  uint32_t *ctr;               // arrivals of row groups' splits (SplitCounter): zero between launches
  uint32_t *status;
  float scale_log2;
  int tiles;                   // 16-row tiles of a workgroup: 1, 2, 4 or 8
  int may_split;               // a sequence can be long enough for more than one workgroup
  void *ev_start, *ev_stop;
};
// Workgroups that a call's keys are divided among: one a compute unit
constexpr int kPagedSlots = 256;
constexpr int kPagedSplits = 128;  // most splits of a row group
constexpr int kPagedParts = 3 * kPagedSlots;  // workgroups of row groups with several, at most
constexpr size_t kPagedCounters = 2 * kPagedParts / 8;  // bytes of their counters
// Where the splits of a row group, KS of them from place `first` on, count their
// arrivals: `bits` of the workspace's header for each place (6 of up to kPagedSlots
// places, 3 of twice and 2 of three times as many), which no call's scratch covers.
// The group's counter holds up to KS and lies in one word, in the next where it would
// cross into it.  Few groups share a word: arrivals at one are served one after
// another (with 2 bits throughout, 16 rows over 2000 positions took 17.0 us for 15.9).
struct SplitCounter {
  int word, shift;
  uint32_t mask;
};
__host__ __device__ constexpr SplitCounter split_counter(int first, int KS, int bits) {
  const int need = 32 - __builtin_clz((unsigned)KS), at = bits * first;
  const int from = at % 32 + need > 32 ? (at + 31) / 32 * 32 : at;
  return SplitCounter{from / 32, from % 32, (1u << need) - 1};
}
constexpr bool split_counters_fit(int bits) {
  for (int first = 0; first < 32; ++first)  // (later places: the same, whole words on)
    for (int KS = 2; KS <= kPagedSplits; ++KS) {
      const SplitCounter c = split_counter(first, KS, bits);
      const int from = 32 * c.word + c.shift, need = 32 - __builtin_clz(c.mask);
      if (from < bits * first || from + need > bits * (first + KS) || c.shift + need > 32 || (unsigned)KS > c.mask) return false;
    }
  return true;
}
static_assert(split_counters_fit(2) && split_counters_fit(3) && split_counters_fit(6), "in the group's own bits and one word, and hold KS");
size_t paged_attn_part_bytes(int nh, int nkv, int B, int n_rows);
void paged_attn_shape(PagedAttnLaunch &a);  // fills tiles, may_split
hipError_t launch_paged_attn(const PagedAttnLaunch &a, hipStream_t s);

struct PagedSelectLaunch {
  PagedSeqs sq;
  const bf16_t *bounds;  // this layer's [n_pages][nkv][2][128]
  const void *q;
  int q_type, T_pad, nh, nkv;
  int budget, n_first, n_last;
  unsigned long long *keys;  // [B][nkv][max_pages]
  int32_t *sel, *n_sel;
  uint32_t *status;
};
hipError_t launch_paged_select(const PagedSelectLaunch &p, hipStream_t s);

// The step of ppd_api.cpp on pages
struct PagedStep {
  const ppd_paged *kv;
  const ppd_page_tables *pt;
  const int32_t *row_start;
  int budget, n_first, n_last;  // budget 0: every page
};
PagedSeqs paged_seqs(const ppd_page_tables *pt, const int32_t *row_start, int n_rows);
// the arguments that the calls on pages share (ppd_paged.cpp)
ppd_status paged_check(const ppd_paged *kv, const ppd_page_tables *pt, bool tail);
ppd_status paged_check_rows(const ppd_paged *kv, const int32_t *row_start, int n_rows);
ppd_status paged_check_select(const ppd_paged *kv, int budget, int n_first, int n_last);
size_t paged_select_key_bytes(int nkv, int B, int max_pages);
