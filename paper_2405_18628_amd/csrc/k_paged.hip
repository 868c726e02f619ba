// Page tables and slot maps from lengths on the device, and rows into pages.
#include <algorithm>

#include "ppd_paged.h"

namespace {

// ---------------------------------------------------------------------------
// Tables.  With old = ceil(len / P), new = ceil((len + add) / P) pages, what each
// sequence gets follows from three running sums over the sequences: of added
// rows (where its rows start), of new - old over those that fit the table and the
// slot buffer (its first entry of the ring, and whether the ring suffices) and of
// pages given back.  One workgroup forms them, a run of sequences a thread
// (tables_plan); rows are then independent: a row finds its sequence by
// bisection of the starts, and the first row of a new page writes the
// table's entry, so every new page is written by exactly one row.

constexpr int TT = 1024;
enum { kEnded = -1, kRefused = 0, kServed = 1 };

// inclusive sum over the workgroup's threads; *all: of all of them
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *waves, int64_t *all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(v, o, 64);
    v += lane >= o ? u : 0;
  }
  if (lane == 63) waves[w] = v;
  __syncthreads();
  int64_t before = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < TT / 64; ++i) {
    before += i < w ? waves[i] : 0;
    sum += waves[i];
  }
  __syncthreads();
  *all = sum;
  return v + before;
}

// a sequence's numbers as read, clamped
struct TSeq {
  int len, old, grow;
  bool ended, bad;
};
__device__ __forceinline__ TSeq tables_seq(const PagedTablesLaunch &p, int s) {
  TSeq q;
  const int64_t most = (int64_t)p.max_pages << p.lp;
  const int n = p.len[s], a = p.add[s];
  q.len = (int)max((int64_t)0, min((int64_t)n, most));
  q.bad = n != q.len;
  q.old = (int)(((int64_t)q.len + (1 << p.lp) - 1) >> p.lp);
  q.ended = a < 0;
  q.grow = q.ended ? 0 : a;
  return q;
}
__device__ __forceinline__ int64_t pages_of(int64_t n, int lp) { return (n + (1 << lp) - 1) >> lp; }

// start, lengths, ring state and the plan [B] of {length, old pages, ring index of
// the first new page or place of the first page given back, kServed ..}
__device__ void tables_plan(const PagedTablesLaunch &p) {
  __shared__ int64_t waves[TT / 64];
  __shared__ int64_t taken_s;
  const int tid = threadIdx.x;
  const int per = (p.B + TT - 1) / TT, s0 = tid * per, s1 = min(p.B, s0 + per);
  int first = p.free_state[0], count = p.free_state[1];
  if (tid == 0) taken_s = 0;
  bool bad = false;
  if (first < 0 || first >= p.n_pages || count < 0 || count > p.n_pages) {
    bad = true;
    first = max(0, min(first, p.n_pages - 1));
    count = max(0, min(count, p.n_pages));
  }
  int64_t rows = 0, back = 0;
  for (int s = s0; s < s1; ++s) {
    const TSeq q = tables_seq(p, s);
    rows += q.grow;
    back += q.ended ? q.old : 0;
    bad |= q.bad;
  }
  int64_t all_rows, all_back, all_need;
  int64_t start = block_scan(rows, waves, &all_rows) - rows;
  int64_t given = block_scan(back, waves, &all_back) - back;
  const int64_t start0 = start;
  auto fits = [&](const TSeq &q, int64_t from, int64_t *need) {
    const int64_t now = pages_of((int64_t)q.len + q.grow, p.lp);
    const bool ok = now <= p.max_pages && from + q.grow <= p.n_slots;
    *need = ok ? now - q.old : 0;
    return ok;
  };
  int64_t need = 0;
  for (int s = s0; s < s1; ++s) {
    const TSeq q = tables_seq(p, s);
    int64_t n;
    fits(q, start, &n);
    need += n;
    start += q.grow;
  }
  int64_t asked = block_scan(need, waves, &all_need) - need;
  start = start0;
  bool refused = false;
  for (int s = s0; s < s1; ++s) {
    const TSeq q = tables_seq(p, s);
    int64_t n;
    bool ok = fits(q, start, &n);
    asked += n;
    ok = ok && (n == 0 || asked <= count);
    const int64_t at = q.ended ? first + (int64_t)count + given : first + asked - n;
    p.plan[s] = int4{q.len, q.old, (int)(at % p.n_pages), q.ended ? kEnded : ok ? kServed : kRefused};
    p.start[s] = (int)min(start, (int64_t)INT32_MAX);
    p.len_out[s] = q.ended ? 0 : q.len + (ok ? q.grow : 0);
    // the last sequence served a page has the largest sum that the ring suffices for
    if (ok && n) atomicMax((unsigned long long *)&taken_s, (unsigned long long)asked);
    refused |= !ok;
    given += q.ended ? q.old : 0;
    start += q.grow;
  }
  if (s0 < p.B && s1 == p.B) p.start[p.B] = (int)min(start, (int64_t)INT32_MAX);
  __syncthreads();
  if (tid == 0) {
    const int64_t taken = taken_s;
    p.free_state_out[0] = (int)((first + taken) % p.n_pages);
    p.free_state_out[1] = (int)min(count - taken + all_back, (int64_t)p.n_pages);
  }
  if (refused) atomicOr(p.status, PPD_DEV_NO_PAGES);
  if (bad || (tid == 0 && count + all_back > p.n_pages)) atomicOr(p.status, PPD_DEV_BAD_LENGTH);
}

// slots of rows [i0, n) by steps of `step`, and the new pages' table entries;
// pages given back, a wave a sequence
__device__ void tables_fill(const PagedTablesLaunch &p, const int *start, int i0, int step, int w0, int w_step) {
  const int n = min(start[p.B], p.n_slots), P = 1 << p.lp;
  for (int i = i0; i < n; i += step) {
    int lo = 0, hi = p.B - 1;  // the last sequence that starts at or before i
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (start[mid] <= i)
        lo = mid;
      else
        hi = mid - 1;
    }
    const int4 q = p.plan[lo];
    if (q.w != kServed) {
      p.slots[i] = -1;
      continue;
    }
    const int pos = q.x + (i - start[lo]), j = pos >> p.lp;  // below max_pages pages
    int32_t *row = p.table + (size_t)lo * p.max_pages;
    int page;
    if (j < q.y) {
      page = row[j];
    } else {
      page = p.free_pages[((int64_t)q.z + (j - q.y)) % p.n_pages];
      if ((pos & (P - 1)) == 0) row[j] = page;
    }
    p.slots[i] = page * P + (pos & (P - 1));
  }
  for (int s = w0; s < p.B; s += w_step) {
    const int4 q = p.plan[s];
    if (q.w != kEnded) continue;
    for (int j = threadIdx.x & 63; j < q.y; j += 64)
      p.free_pages[((int64_t)q.z + j) % p.n_pages] = p.table[(size_t)s * p.max_pages + j];
  }
}

// everything in one workgroup
__global__ __launch_bounds__(TT) void paged_tables_kernel(PagedTablesLaunch p) {
  __shared__ int start_s[PPD_PAGED_SEQS_MAX + 1];
  tables_plan(p);
  __threadfence_block();
  __syncthreads();
  for (int s = threadIdx.x; s <= p.B; s += TT) start_s[s] = p.start[s];
  __syncthreads();
  tables_fill(p, start_s, threadIdx.x, TT, threadIdx.x >> 6, TT / 64);
}

__global__ __launch_bounds__(TT) void paged_plan_kernel(PagedTablesLaunch p) { tables_plan(p); }

__global__ __launch_bounds__(256) void paged_fill_kernel(PagedTablesLaunch p) {
  __shared__ int start_s[PPD_PAGED_SEQS_MAX + 1];
  for (int s = threadIdx.x; s <= p.B; s += 256) start_s[s] = p.start[s];
  __syncthreads();
  const int i = blockIdx.x * 256 + threadIdx.x;
  tables_fill(p, start_s, i, gridDim.x * 256, i >> 6, gridDim.x * 4);
}

// ---------------------------------------------------------------------------
// Rows into pages.  A run is the rows of one sequence that fall into one page; a
// wave takes a run of one (layer, kv head), so a page's bounds have one writer
// and no atomics.  Keys move as 16-byte pieces (8 dims of a position), values
// are turned: 8 positions of a dim are 16 bytes of a block, read at once where the
// source holds them side by side.

constexpr int SW = 4;    // waves of a workgroup
constexpr int SR = 128;  // rows of a workgroup

__device__ __forceinline__ float lo_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__global__ __launch_bounds__(64 * SW) void paged_store_kernel(PagedStoreLaunch p) {
  __shared__ int4 run_s[SR];  // first row, rows, sequence
  __shared__ int n_run;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int P = 1 << p.lp;
  const int n = max(0, min(p.start[p.B], p.n_rows));
  const int lh = blockIdx.x / p.chunks, layer = lh / p.nkv, kvh = lh % p.nkv;
  const bf16_t *k = p.k + (size_t)lh * p.scap * 128, *v = p.v + (size_t)lh * 128 * p.scap;
  for (int64_t at = (int64_t)(blockIdx.x % p.chunks) * SR; at < n; at += (int64_t)p.chunks * SR) {
    const int i0 = (int)at;
    __syncthreads();  // the last rows' runs are done
    if (tid == 0) n_run = 0;
    __syncthreads();
    const int i = i0 + tid;
    if (tid < SR && i < n) {
      int lo = 0, hi = p.B - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.start[mid] <= i)
          lo = mid;
        else
          hi = mid - 1;
      }
      const int first = p.start[lo], slot = p.slots[i];
      if (i >= first && slot >= 0 && (slot >> p.lp) < p.n_pages && (i == first || (slot & (P - 1)) == 0)) {
        const int m = min(P - (slot & (P - 1)), min(p.start[lo + 1], n) - i);
        run_s[atomicAdd(&n_run, 1)] = int4{i, m, lo, slot};  // (runs are independent of one another)
      }
    }
    __syncthreads();
    for (int r = wave; r < n_run; r += SW) {
      const int4 run = run_s[r];
      const int m = run.y, page = run.w >> p.lp, off = run.w & (P - 1);
      const int first = p.start[run.z], base = p.row_start[run.z], k0 = run.x - first;
      auto source = [&](int j) {  // the source's row of the run's row j
        int row = base + k0 + j;
        if (p.path) row = base + p.path[max(0, min(row, p.n_path - 1))];
        return max(0, min(row, p.scap - 1));
      };
      unsigned char *dst = p.pages + (((size_t)layer * p.n_pages + page) * p.nkv + kvh) * ((size_t)kPBytes << (p.lp - 5));
      // ---- keys: 16 lanes a row
      const int piece = lane & 15;
      float mn[8], mx[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) mn[e] = INFINITY, mx[e] = -INFINITY;  // (what is left of NaN alone)
      constexpr int U = 4;  // rows of a lane in flight
      for (int j0 = lane >> 4; j0 < m; j0 += 4 * U) {
        u32x4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = *(const u32x4 *)(k + (size_t)source(min(j0 + 4 * u, m - 1)) * 128 + piece * 8);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int j = j0 + 4 * u;
          if (j >= m) break;
          const int pos = off + j;
          *(u32x4 *)(dst + (size_t)(pos >> 5) * kPBytes + 2 * paged_key_at(pos & 31, piece * 8)) = w[u];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = e & 1 ? hi_of(w[u][e >> 1]) : lo_of(w[u][e >> 1]);
            mn[e] = fminf(mn[e], x);
            mx[e] = fmaxf(mx[e], x);
          }
        }
      }
      if (p.bounds) {
        bf16_t *b = p.bounds + (((size_t)layer * p.n_pages + page) * p.nkv + kvh) * 256 + piece * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
          for (int o = 16; o < 64; o <<= 1) {
            mn[e] = fminf(mn[e], __shfl_xor(mn[e], o, 64));
            mx[e] = fmaxf(mx[e], __shfl_xor(mx[e], o, 64));
          }
        }
        if (lane < 16) {
          if (off) {
            const u32x4 a = *(const u32x4 *)b, c = *(const u32x4 *)(b + 128);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              mn[e] = fminf(mn[e], e & 1 ? hi_of(a[e >> 1]) : lo_of(a[e >> 1]));
              mx[e] = fmaxf(mx[e], e & 1 ? hi_of(c[e >> 1]) : lo_of(c[e >> 1]));
            }
          }
          u32x4 a, c;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a[e] = pack_bf16x2(mn[2 * e], mn[2 * e + 1]);
            c[e] = pack_bf16x2(mx[2 * e], mx[2 * e + 1]);
          }
          *(u32x4 *)b = a;
          *(u32x4 *)(b + 128) = c;
        }
      }
      // ---- values: blocks of 32 positions, lane: dim 16 w + lane % 16, positions 8 (lane / 16) ..
      for (int blk = off >> 5; blk <= (off + m - 1) >> 5; ++blk) {
        const int u0 = blk * 32 + 8 * (lane >> 4) - off;       // the run's row of the lane's first position
        const int from = max(0, -u0), to = min(8, m - u0);     // its positions that are of the run
        if (from >= to) continue;
        const int s0 = p.path ? 0 : base + k0 + u0;
        const bool whole = from == 0 && to == 8;
        unsigned char *d = dst + (size_t)blk * kPBytes + 2 * kPElems + lane * 16;
        if (whole && !p.path && s0 % 8 == 0 && s0 >= 0 && s0 + 8 <= p.scap) {
          u32x4 w[8];
#pragma unroll
          for (int t = 0; t < 8; ++t) w[t] = *(const u32x4 *)(v + (size_t)(16 * t + (lane & 15)) * p.scap + s0);
#pragma unroll
          for (int t = 0; t < 8; ++t) *(u32x4 *)(d + t * 1024) = w[t];
        } else {
          int src[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) src[e] = source(max(0, min(u0 + e, m - 1)));
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const bf16_t *row = v + (size_t)(16 * t + (lane & 15)) * p.scap;
            uint32_t x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = row[src[e]];
            if (whole) {
              *(u32x4 *)(d + t * 1024) = u32x4{x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e >= from && e < to) ((bf16_t *)(d + t * 1024))[e] = (bf16_t)x[e];
            }
          }
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_paged_tables(const PagedTablesLaunch &p, hipStream_t s) {
  // one workgroup while a thread of it has a few rows; else its sums first, the
  // rows over the device
  if (p.n_slots <= 8 * TT) {
    hipLaunchKernelGGL(paged_tables_kernel, dim3(1), dim3(TT), 0, s, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(TT), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int grid = (int)std::min<int64_t>(1024, ((int64_t)p.n_slots + 1023) / 1024);
  hipLaunchKernelGGL(paged_fill_kernel, dim3(grid), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_paged_store(PagedStoreLaunch p, hipStream_t s) {
  // (a launch's threads are counted in 32 bits: of very many rows a workgroup takes several parts)
  const int heads = p.layers * p.nkv;
  p.chunks = std::min((p.n_rows - 1) / SR + 1, std::max(1, (1 << 22) / heads));
  hipLaunchKernelGGL(paged_store_kernel, dim3(heads * p.chunks), dim3(64 * SW), 0, s, p);
  return hipGetLastError();
}
