// Page tables and slot maps from lengths on the device, and rows into pages.
#include <algorithm>

#include "ppd_paged.h"

namespace {

// ---------------------------------------------------------------------------
// Tables.  With old = ceil(len / P), new = ceil((len + add) / P) pages, what each
// sequence gets follows from three running sums over the sequences: of added
// rows (where its rows start), of new - old over those that fit the table and the
// slot buffer (its first entry of the ring, and whether the ring suffices) and of
// pages given back.  Every workgroup forms them for itself, a thread a sequence
// (from 1025 sequences on several), in LDS: that takes less than another
// launch.  Rows are then independent: a thread takes four, finds their sequence by
// bisection of the starts, and the first row of a new page writes the table's
// entry, so every new page is written by exactly one row.  Lengths and the ring's
// state may be written where they are read: the last workgroup to have read
// them does it.  16 sequences with 60 rows 5.5 us, 512 with 0.8 million rows 10.6 (two
// launches, the sums in the first: 17.0): launch, counts, two sums, bisection, ring and
// slots one after another, a few KB to 3 MB.

enum { kEnded = -1, kRefused = 0, kServed = 1 };

struct TablesPlan {
  int start[PPD_PAGED_SEQS_MAX + 1];
  int len[PPD_PAGED_SEQS_MAX];
  int at[PPD_PAGED_SEQS_MAX];  // ring index of the first new page, or place of the first given back; ~: refused
  uint32_t ended[PPD_PAGED_SEQS_MAX / 32];
};

// inclusive sums over the workgroup's threads; all: of all of them
template <int TT, int N>
__device__ __forceinline__ void block_scan(int64_t (&v)[N], int64_t (&all)[N], int64_t (*waves)[N]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = wave_incl64(v[i]);
    if (lane == 63) waves[w][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // lanes 0 .. 15: the waves' sums
    const int64_t s = wave_incl64(lane < TT / 64 ? waves[min(lane, TT / 64 - 1)][i] : 0);
    v[i] += w ? lane_of64(s, w - 1) : 0;
    all[i] = lane_of64(s, TT / 64 - 1);
  }
}
__device__ __forceinline__ int64_t pages_of(int64_t n, int lp) { return (n + (1 << lp) - 1) >> lp; }
// i of a ring of n, i < 2 n
__device__ __forceinline__ int in_ring(int64_t i, int n) { return (int)(i >= n ? i - n : i); }

template <int TT, int PER>  // threads, sequences of a thread
__global__ __launch_bounds__(TT) void paged_tables_kernel(PagedTablesLaunch p) {
  __shared__ TablesPlan plan;
  __shared__ int64_t sums_s[2][TT / 64][2];
  __shared__ int taken_s, last_s;
  const int tid = threadIdx.x, P = 1 << p.lp;
  const int s0 = tid * PER, n_mine = max(0, min(PER, p.B - s0));
  int len[PER], grow[PER], old[PER];
  bool ended[PER];
  bool bad = false;
  int first = p.free_state[0], count = p.free_state[1];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int n = i < n_mine ? p.len[s0 + i] : 0, a = i < n_mine ? p.add[s0 + i] : 0;
    len[i] = (int)max((int64_t)0, min((int64_t)n, (int64_t)p.max_pages << p.lp));
    bad |= n != len[i];
    ended[i] = a < 0;
    grow[i] = max(a, 0);
    old[i] = (int)pages_of(len[i], p.lp);
  }
  if (first < 0 || first >= p.n_pages || count < 0 || count > p.n_pages) {
    bad = true;
    first = max(0, min(first, p.n_pages - 1));
    count = max(0, min(count, p.n_pages));
  }
  if (tid == 0) taken_s = 0;
  for (int i = tid; i < PPD_PAGED_SEQS_MAX / 32; i += TT) plan.ended[i] = 0;
  int64_t v[2] = {0, 0}, all[2];
#pragma unroll
  for (int i = 0; i < PER; ++i) v[0] += grow[i], v[1] += ended[i] ? old[i] : 0;
  const int64_t rows = v[0], back = v[1];
  block_scan<TT, 2>(v, all, sums_s[0]);
  int64_t start = v[0] - rows, given = v[1] - back;
  const int64_t all_back = all[1];
  // new pages of those that fit
  int need[PER];
  bool fits[PER];
  int64_t at = start, mine[1] = {0}, all_need[1];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int64_t now = pages_of((int64_t)len[i] + grow[i], p.lp);
    fits[i] = !ended[i] && now <= p.max_pages && at + grow[i] <= p.n_slots;
    need[i] = fits[i] ? (int)(now - old[i]) : 0;
    mine[0] += need[i];
    at += grow[i];
  }
  const int64_t wanted = mine[0];
  block_scan<TT, 1>(mine, all_need, (int64_t(*)[1])sums_s[1]);
  int64_t asked = mine[0] - wanted;
  bool refused = false;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i < n_mine) {
      asked += need[i];
      const bool ok = ended[i] || (fits[i] && (need[i] == 0 || asked <= count));
      plan.start[s0 + i] = (int)min(start, (int64_t)INT32_MAX);
      plan.len[s0 + i] = len[i];
      // (asked - need < count <= n_pages, given <= n_pages: below 3 rings)
      const int64_t a = ended[i] ? (int64_t)in_ring((int64_t)first + count, p.n_pages) + given : (int64_t)first + asked - need[i];
      plan.at[s0 + i] = ok ? (int)(a % p.n_pages) : ~0;
      if (ended[i]) atomicOr(&plan.ended[(s0 + i) >> 5], 1u << ((s0 + i) & 31));
      // the last sequence served a page has the largest sum that the ring suffices for
      if (ok && need[i]) atomicMax(&taken_s, (int)asked);
      refused |= !ok;
      given += ended[i] ? old[i] : 0;
      start += grow[i];
      if (!ok) grow[i] = 0;  // (it keeps its length)
    }
  if (n_mine && s0 + n_mine == p.B) plan.start[p.B] = (int)min(start, (int64_t)INT32_MAX);
  __syncthreads();
  const int taken = taken_s;
  if (tid == 0)
    last_s = gridDim.x == 1 || __hip_atomic_fetch_add(p.ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  // ---- slots, four rows a thread
  const int n = min(plan.start[p.B], p.n_slots);
  const bool wide = ((uintptr_t)p.slots & 15) == 0;
  for (int64_t i0 = 4 * ((int64_t)blockIdx.x * TT + tid); i0 < n; i0 += 4 * (int64_t)gridDim.x * TT) {
    int lo = 0, hi = p.B - 1;  // the last sequence that starts at or before i0
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (plan.start[mid] <= i0)
        lo = mid;
      else
        hi = mid - 1;
    }
    int s = -1, j = -1, page = 0, x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = (int)i0 + e;
      while (lo < p.B - 1 && plan.start[lo + 1] <= i) ++lo;
      x[e] = -1;
      if (i < n && plan.at[lo] >= 0) {
        const int pos = plan.len[lo] + (i - plan.start[lo]), q = pos >> p.lp;  // below max_pages pages
        if (lo != s || q != j) {
          s = lo, j = q;
          const int before = (int)pages_of(plan.len[lo], p.lp);
          int32_t *row = p.table + (size_t)lo * p.max_pages;
          page = q < before ? row[q] : p.free_pages[in_ring((int64_t)plan.at[lo] + (q - before), p.n_pages)];
          if (q >= before && (pos & (P - 1)) == 0) row[q] = page;
        }
        x[e] = page * P + (pos & (P - 1));
      }
    }
    if (wide && i0 + 4 <= n) {
      *(int4 *)(p.slots + i0) = int4{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i0 + e < n) p.slots[i0 + e] = x[e];
    }
  }
  // ---- pages given back, a wave a sequence
  if (all_back)
    for (int s = (blockIdx.x * TT + tid) >> 6; s < p.B; s += gridDim.x * (TT / 64)) {
      if (!(plan.ended[s >> 5] >> (s & 31) & 1)) continue;
      const int m = (int)pages_of(plan.len[s], p.lp);
      for (int j = tid & 63; j < m; j += 64)
        // (a length of more pages than there are is bad, but goes round the ring)
        p.free_pages[(uint32_t)(plan.at[s] + j) % (uint32_t)p.n_pages] = p.table[(size_t)s * p.max_pages + j];
    }
  if (blockIdx.x == 0) {
    for (int s = tid; s <= p.B; s += TT) p.start[s] = plan.start[s];
    if (refused) atomicOr(p.status, PPD_DEV_NO_PAGES);
    if (bad || (tid == 0 && count + all_back > p.n_pages)) atomicOr(p.status, PPD_DEV_BAD_LENGTH);
  }
  __syncthreads();
  if (!last_s) return;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i < n_mine) p.len_out[s0 + i] = ended[i] ? 0 : len[i] + grow[i];
  if (tid == 0) {
    p.free_state_out[0] = in_ring((int64_t)first + taken, p.n_pages);
    p.free_state_out[1] = (int)min(count - taken + all_back, (int64_t)p.n_pages);
    __hip_atomic_store(p.ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// ---------------------------------------------------------------------------
// Rows into pages.  A run is the rows of one sequence that fall into one page; it
// is one workgroup's for each (layer, kv head), so a page's bounds have one
// writer and no atomics.  Keys move as 16-byte pieces (8 dims of a position, 16
// lanes a row), values are turned: 8 positions of a dim are 16 bytes of a block.
//
// Accepted rows and single tokens (paged_put_kernel): a wave a run, eight rows at
// a time, values element by element, a lane two dims; keys, values and bounds
// requested together, since a call takes round trips and the lines it touches
// in part rather than bytes.  Prompts (paged_fill_rows_kernel): up to four waves a run,
// a block of 32 positions each, values 16 bytes at a time -- of a source that is
// not aligned by eights two neighbouring pieces shifted into one -- and the waves'
// bounds joined in LDS.
//
// Prompts of four sequences, 24 layers of 8 heads 206 to 212 us (4.7 TB/s of rows in and
// out; a copy 5.0), in pages of 256 positions 234, from a source off by three rows 183
// (700 of 904 MB).  Accepted rows of four sequences, 32 layers of 32 heads 15 us: 22 MB
// in and 22 MB out, in lines touched in part, for 18 MB.  One kernel for both took
// 250 and 27.

constexpr int SW = 4;     // waves of a workgroup
constexpr int SB = 255;   // sequences whose offsets fit its LDS
constexpr int FEW = 8;    // rows that a wave has in flight

__device__ __forceinline__ float lo_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// smallest and largest of a lane's 8 dims (what is left of NaN alone: infinities)
struct Bounds8 {
  float mn[8], mx[8];
  __device__ __forceinline__ Bounds8() {
#pragma unroll
    for (int e = 0; e < 8; ++e) mn[e] = INFINITY, mx[e] = -INFINITY;
  }
  __device__ __forceinline__ void add(u32x4 lo, u32x4 hi) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mn[e] = fminf(mn[e], e & 1 ? hi_of(lo[e >> 1]) : lo_of(lo[e >> 1]));
      mx[e] = fmaxf(mx[e], e & 1 ? hi_of(hi[e >> 1]) : lo_of(hi[e >> 1]));
    }
  }
  // over the wave's four rows of 16 lanes
  __device__ __forceinline__ void join() {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mn[e] = -quad_max(-mn[e]);
      mx[e] = quad_max(mx[e]);
    }
  }
  __device__ __forceinline__ void store(u32x4 *smallest, u32x4 *largest) const {
    u32x4 lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = pack_bf16x2(mn[2 * e], mn[2 * e + 1]);
      hi[e] = pack_bf16x2(mx[2 * e], mx[2 * e + 1]);
    }
    *smallest = lo;
    *largest = hi;
  }
};

// The runs that start among `rows` rows (SR at most), from row `at` on, in LDS;
// false: there are no rows from there on.
template <int SR>
struct Runs {
  int4 run[SR];  // first row, rows, sequence, slot
  int start[SB + 1], rows[SB + 1];
  int n;
};
template <int SR>
__device__ __forceinline__ void load_offsets(Runs<SR> &s, const PagedStoreLaunch &p) {
  const int tid = threadIdx.x;
  if (p.B <= SB && tid <= p.B) {
    s.start[tid] = p.start[tid];
    s.rows[tid] = tid < p.B ? p.row_start[tid] : 0;
  }
}
template <int SR>
__device__ __forceinline__ bool find_runs(Runs<SR> &s, const PagedStoreLaunch &p, int64_t at, int rows) {
  const int tid = threadIdx.x, P = 1 << p.lp;
  const int32_t *start = p.B <= SB ? s.start : p.start;
  const int i = (int)at + tid;
  const int slot = tid < rows && i < p.n_rows ? p.slots[i] : -1;
  __syncthreads();  // the offsets are there, the last rows' runs done
  if (tid == 0) s.n = 0;
  __syncthreads();
  const int n = min(start[p.B], p.n_rows);
  if (at >= n) return false;
  if (tid < rows && i < n) {
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (start[mid] <= i)
        lo = mid;
      else
        hi = mid - 1;
    }
    const int first = start[lo];
    if (i >= first && slot >= 0 && (slot >> p.lp) < p.n_pages && (i == first || (slot & (P - 1)) == 0)) {
      const int m = min(P - (slot & (P - 1)), min(start[lo + 1], n) - i);
      s.run[atomicAdd(&s.n, 1)] = int4{i, m, lo, slot};  // (runs are independent of one another)
    }
  }
  __syncthreads();
  return true;
}

// a run as a wave takes it
struct Run {
  int m, off;         // rows, position of the first in its page
  int base, k0;       // the sequence's first row of the source, the run's first of its rows
  unsigned char *dst;
  bf16_t *bounds;
};
template <int SR>
__device__ __forceinline__ Run take_run(const Runs<SR> &s, const PagedStoreLaunch &p, int r, int layer, int kvh) {
  const int4 run = s.run[r];
  const int sq = __builtin_amdgcn_readfirstlane(run.z), page = __builtin_amdgcn_readfirstlane(run.w >> p.lp);
  Run x;
  x.m = __builtin_amdgcn_readfirstlane(run.y);
  x.off = __builtin_amdgcn_readfirstlane(run.w & ((1 << p.lp) - 1));
  const bool near = p.B <= SB;
  x.base = __builtin_amdgcn_readfirstlane(near ? s.rows[sq] : p.row_start[sq]);
  x.k0 = __builtin_amdgcn_readfirstlane(run.x - (near ? s.start[sq] : p.start[sq]));
  const size_t head = ((size_t)layer * p.n_pages + page) * p.nkv + kvh;
  x.dst = p.pages + head * ((size_t)kPBytes << (p.lp - 5));
  x.bounds = p.bounds ? p.bounds + head * 256 : nullptr;
  return x;
}

constexpr int PUT_ROWS = 128;

__global__ __launch_bounds__(64 * SW) void paged_put_kernel(PagedStoreLaunch p) {
  __shared__ Runs<PUT_ROWS> runs;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  load_offsets(runs, p);
  const int lh = blockIdx.x / p.chunks, layer = lh / p.nkv, kvh = lh % p.nkv;
  const bf16_t *k = p.k + (size_t)lh * p.scap * 128, *v = p.v + (size_t)lh * 128 * p.scap;
  const int piece = lane & 15;
  for (int64_t at = (int64_t)(blockIdx.x % p.chunks) * PUT_ROWS; at < p.n_rows; at += (int64_t)p.chunks * PUT_ROWS) {
    if (!find_runs(runs, p, at, PUT_ROWS)) return;
    for (int r = wave; r < runs.n; r += SW) {
      const Run run = take_run(runs, p, r, layer, kvh);
      u32x4 was[2] = {};
      if (run.bounds && run.off && lane < 16) {
        was[0] = *((const u32x4 *)run.bounds + piece);
        was[1] = *((const u32x4 *)run.bounds + 16 + piece);
      }
      Bounds8 bd;
      for (int j0 = 0; j0 < run.m; j0 += FEW) {
        const int m = min(FEW, run.m - j0);
        // lane j: the source's row of row j0 + j (past the last: the last again)
        int64_t row = (int64_t)run.base + run.k0 + j0 + min(lane, m - 1);
        if (p.path) row = (int64_t)run.base + p.path[max((int64_t)0, min(row, (int64_t)p.n_path - 1))];
        const int mine = (int)max((int64_t)0, min(row, (int64_t)p.scap - 1));
        u32x4 kw[FEW / 4];
        bf16_t vw[FEW][2];
#pragma unroll
        for (int j = 0; j < FEW / 4; ++j)
          kw[j] = *(const u32x4 *)(k + (size_t)__shfl(mine, min(4 * j + (lane >> 4), m - 1), 64) * 128 + piece * 8);
#pragma unroll
        for (int j = 0; j < FEW; ++j) {
          const int from = lane_of(mine, j);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (j < m) vw[j][h] = v[(size_t)(lane + 64 * h) * p.scap + from];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < FEW / 4; ++j) {
          const int pos = run.off + j0 + 4 * j + (lane >> 4);
          if (4 * j + (lane >> 4) < m) {
            *(u32x4 *)(run.dst + (size_t)(pos >> 5) * kPBytes + 2 * paged_key_at(pos & 31, piece * 8)) = kw[j];
            bd.add(kw[j], kw[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < FEW; ++j) {
          const int pos = run.off + j0 + j;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (j < m) ((bf16_t *)(run.dst + (size_t)(pos >> 5) * kPBytes))[kPElems + paged_value_at(pos & 31, lane + 64 * h)] = vw[j][h];
        }
      }
      if (run.bounds) {
        bd.join();
        if (lane < 16) {
          if (run.off) bd.add(was[0], was[1]);
          bd.store((u32x4 *)run.bounds + piece, (u32x4 *)run.bounds + 16 + piece);
        }
      }
    }
  }
}

constexpr int FILL_ROWS = 256;

__global__ __launch_bounds__(64 * SW) void paged_fill_rows_kernel(PagedStoreLaunch p) {
  __shared__ Runs<FILL_ROWS> runs;
  __shared__ __attribute__((aligned(16))) u32x4 join_s[SW][2][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int piece = lane & 15, lg = lane >> 4;
  load_offsets(runs, p);
  const int lh = blockIdx.x / p.chunks, layer = lh / p.nkv, kvh = lh % p.nkv;
  const bf16_t *k = p.k + (size_t)lh * p.scap * 128, *v = p.v + (size_t)lh * 128 * p.scap;
  const int each = min(SW, 1 << (p.lp - 5)), sub = wave % each;  // waves of a run, this one among them
  const int rows = p.rows_each;
  for (int64_t at = (int64_t)(blockIdx.x % p.chunks) * rows; at < p.n_rows; at += (int64_t)p.chunks * rows) {
    if (!find_runs(runs, p, at, rows)) return;
    for (int r0 = 0; r0 < runs.n; r0 += SW / each) {  // (alike in all waves: they meet below)
      const bool on = r0 + wave / each < runs.n;
      const Run run = take_run(runs, p, on ? r0 + wave / each : r0, layer, kvh);
      Bounds8 bd;
      u32x4 was[2] = {};
      if (run.bounds && run.off && lane < 16) {
        was[0] = *((const u32x4 *)run.bounds + piece);
        was[1] = *((const u32x4 *)run.bounds + 16 + piece);
      }
      const int first = run.off >> 5, last = on ? (run.off + run.m - 1) >> 5 : -1;
      const int64_t src = (int64_t)run.base + run.k0 - run.off;  // the source's row of the page's position 0
      for (int blk = first + sub; blk <= last; blk += each) {
        const int p0 = max(run.off, blk * 32), p1 = min(run.off + run.m, blk * 32 + 32);  // its positions
        u32x4 kw[8], vw[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int64_t row = src + max(p0, min(blk * 32 + 4 * j + lg, p1 - 1));
          kw[j] = *(const u32x4 *)(k + (size_t)max((int64_t)0, min(row, (int64_t)p.scap - 1)) * 128 + piece * 8);
        }
        // values: dim 16 t + lane % 16, positions 8 lg .. + 7 of the block
        const int64_t s0 = src + blk * 32 + 8 * lg;
        const int part = (int)(s0 & 7);  // alike in the wave
        const int64_t most = p.scap - 8, a0 = max((int64_t)0, min(s0 - part, most));
#pragma unroll
        for (int t = 0; t < 8; ++t) vw[t] = *(const u32x4 *)(v + (size_t)(16 * t + piece) * p.scap + a0);
        if (part) {
          const int64_t a1 = max((int64_t)0, min(s0 - part + 8, most));
          const int q = part >> 1, odd = 16 * (part & 1);
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const u32x4 more = *(const u32x4 *)(v + (size_t)(16 * t + piece) * p.scap + a1);
            const uint32_t w[9] = {vw[t][0], vw[t][1], vw[t][2], vw[t][3], more[0], more[1], more[2], more[3], 0u};
            uint32_t x[5];
#pragma unroll
            for (int e = 0; e < 5; ++e) x[e] = q == 0 ? w[e] : q == 1 ? w[e + 1] : q == 2 ? w[e + 2] : w[e + 3];
#pragma unroll
            for (int e = 0; e < 4; ++e) vw[t][e] = __builtin_amdgcn_alignbit(x[e + 1], x[e], odd);
          }
        }
        unsigned char *d = run.dst + (size_t)blk * kPBytes;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int pos = blk * 32 + 4 * j + lg;
          if (pos >= p0 && pos < p1) {
            *(u32x4 *)(d + 2 * paged_key_at(pos & 31, piece * 8)) = kw[j];
            bd.add(kw[j], kw[j]);
          }
        }
        const int from = max(0, p0 - (blk * 32 + 8 * lg)), to = min(8, p1 - (blk * 32 + 8 * lg));
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          unsigned char *dv = d + 2 * kPElems + t * 1024 + lane * 16;
          if (from == 0 && to == 8) {
            *(u32x4 *)dv = vw[t];
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e >= from && e < to) ((bf16_t *)dv)[e] = (bf16_t)(vw[t][e >> 1] >> 16 * (e & 1));
          }
        }
      }
      if (p.bounds) {  // (alike in all waves)
        bd.join();
        if (each > 1) {
          if (lane < 16) bd.store(&join_s[wave][0][lane], &join_s[wave][1][lane]);
          __syncthreads();
          if (sub == 0 && lane < 16)
            for (int w = 1; w < each; ++w) bd.add(join_s[wave + w][0][lane], join_s[wave + w][1][lane]);
          __syncthreads();
        }
        if (on && sub == 0 && lane < 16) {
          if (run.off) bd.add(was[0], was[1]);
          bd.store((u32x4 *)run.bounds + piece, (u32x4 *)run.bounds + 16 + piece);
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_paged_tables(const PagedTablesLaunch &p, hipStream_t s) {
  // four rows a thread, a sequence a wave (for pages given back)
  auto parts = [&](int threads) {
    const int64_t rows = ((int64_t)p.n_slots + 4 * threads - 1) / (4 * threads), seqs = (p.B + threads / 64 - 1) / (threads / 64);
    return (int)std::min<int64_t>(256, std::max(rows, seqs));
  };
  if (p.B <= 256 && p.n_slots <= 4096)  // (few threads start and meet sooner)
    hipLaunchKernelGGL((paged_tables_kernel<256, 1>), dim3(parts(256)), dim3(256), 0, s, p);
  else if (p.B <= 1024)
    hipLaunchKernelGGL((paged_tables_kernel<1024, 1>), dim3(parts(1024)), dim3(1024), 0, s, p);
  else
    hipLaunchKernelGGL((paged_tables_kernel<1024, PPD_PAGED_SEQS_MAX / 1024>), dim3(parts(1024)), dim3(1024), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_paged_store(PagedStoreLaunch p, hipStream_t s) {
  // (a launch's threads are counted in 32 bits: of very many rows a workgroup takes several parts)
  const int heads = p.layers * p.nkv;
  const bool put = p.path || p.n_rows <= FEW * (int64_t)p.B;
  p.rows_each = put ? PUT_ROWS : std::max(128, 1 << p.lp);
  p.chunks = std::min((p.n_rows - 1) / p.rows_each + 1, std::max(1, (1 << 22) / heads));
  hipLaunchKernelGGL(put ? paged_put_kernel : paged_fill_rows_kernel, dim3(heads * p.chunks), dim3(64 * SW), 0, s, p);
  return hipGetLastError();
}
