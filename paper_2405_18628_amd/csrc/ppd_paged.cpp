// Host side of the paged cache: argument checks and launches (the step on it is
// ppd_api.cpp's).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ppd_paged.h"

namespace {

#define PPD_TRY_HIP(call)                                                                   \
  do {                                                                                      \
    hipError_t e_ = (call);                                                                 \
    if (e_ != hipSuccess) return ppd_fail(PPD_EDEVICE, "%s: %s", #call, hipGetErrorString(e_)); \
  } while (0)

constexpr int kMaxHeads = 1 << 20;   // layers x kv heads
constexpr int kMaxRows = 1 << 22;    // new rows x heads: workgroups and threads are counted in 32 bits
constexpr int64_t kMaxKeys = 1 << 29;  // sequences x kv heads x pages that are ranked
// the header of a workspace: the status word, from byte 16 on the counter of the tables,
// from kCounters on those of the attention's splits
constexpr size_t kHeader = 256, kCounters = 64;
static_assert(kCounters + kPagedCounters <= kHeader, "the counters fit the header");

int log2_of(int page) {
  int lp = 5;
  while (1 << lp < page) ++lp;
  return lp;
}

ppd_status check_sizes(int n_layers, int n_kv_heads, int n_pages, int page) {
  if (n_layers < 1 || n_kv_heads < 1 || n_pages < 1) return ppd_fail(PPD_EINVAL, "a cache needs layers, heads and pages");
  if (page < PPD_PAGED_BLOCK || page > PPD_PAGED_PAGE_MAX || (page & (page - 1)))
    return ppd_fail(PPD_EUNSUPPORTED, "pages hold 32, 64, 128 or 256 positions, not %d", page);
  if ((int64_t)n_layers * n_kv_heads > kMaxHeads)
    return ppd_fail(PPD_EUNSUPPORTED, "%lld layers x heads > %d", (long long)n_layers * n_kv_heads, kMaxHeads);
  if ((int64_t)n_pages * page > INT32_MAX)  // slots are 32-bit
    return ppd_fail(PPD_EUNSUPPORTED, "%d pages of %d positions pass 2^31 slots", n_pages, page);
  return PPD_OK;
}

ppd_status check_cache(const ppd_paged *kv) {
  if (!kv || !kv->pages) return ppd_fail(PPD_EINVAL, "page pointer must be set");
  if ((uintptr_t)kv->pages % 16 || (uintptr_t)kv->bounds % 16)
    return ppd_fail(PPD_EINVAL, "pages and bounds must be 16-byte aligned");
  return check_sizes(kv->n_layers, kv->n_kv_heads, kv->n_pages, kv->page);
}

ppd_status check_kv(const ppd_kv *kv, const char *what) {
  if (!kv || !kv->k || !kv->v) return ppd_fail(PPD_EINVAL, "%s: cache pointers must be set", what);
  if ((uintptr_t)kv->k % 16 || (uintptr_t)kv->v % 16) return ppd_fail(PPD_EINVAL, "%s: 16-byte alignment", what);
  if (kv->capacity < 1) return ppd_fail(PPD_EINVAL, "%s: capacity must be positive", what);
  if (kv->capacity % 8) return ppd_fail(PPD_EUNSUPPORTED, "%s: capacity %% 8 must be 0", what);
  if (kv->capacity > PPD_CAPACITY_MAX)
    return ppd_fail(PPD_EUNSUPPORTED, "%s: capacity %d > %d", what, kv->capacity, PPD_CAPACITY_MAX);
  return PPD_OK;
}

ppd_status check_tables(const ppd_page_tables *pt) {
  if (!pt || !pt->table || !pt->len) return ppd_fail(PPD_EINVAL, "page tables and lengths must be set");
  if (pt->n_seqs < 1 || pt->n_seqs > PPD_PAGED_SEQS_MAX)
    return ppd_fail(PPD_EINVAL, "n_seqs=%d outside [1, %d]", pt->n_seqs, PPD_PAGED_SEQS_MAX);
  if (pt->max_pages < 1) return ppd_fail(PPD_EINVAL, "max_pages must be positive");
  const ppd_status st = check_sizes(1, 1, pt->n_pages, pt->page);
  if (st != PPD_OK) return st;
  if ((int64_t)pt->max_pages * pt->page > PPD_CAPACITY_MAX)
    return ppd_fail(PPD_EUNSUPPORTED, "%d pages of %d positions a sequence > %d", pt->max_pages, pt->page, PPD_CAPACITY_MAX);
  return PPD_OK;
}

bool heads_ok(int n_heads, int n_kv_heads) {
  return n_kv_heads >= 1 && n_heads >= 1 && n_heads <= 1 << 16 && n_heads % n_kv_heads == 0;
}

ppd_status check_work(const void *ws, size_t ws_bytes, size_t need) {
  if (!ws || ws_bytes < need)
    return ppd_fail(PPD_EWORKSPACE, "workspace of %zu bytes is smaller than the %zu required", ws_bytes, need);
  if ((uintptr_t)ws % 16) return ppd_fail(PPD_EINVAL, "ws must be 16-byte aligned");
  return PPD_OK;
}

// what attention and selection share
ppd_status check_call(int n_heads, const ppd_paged *kv, int layer, const ppd_page_tables *pt, const int32_t *row_start,
                      int n_rows, const void *q, int dtype) {
  ppd_status st = paged_check(kv, pt, false);
  if (st != PPD_OK) return st;
  if (!heads_ok(n_heads, kv->n_kv_heads)) return ppd_fail(PPD_EINVAL, "n_kv_heads must divide n_heads <= %d", 1 << 16);
  if (layer < 0 || layer >= kv->n_layers) return ppd_fail(PPD_EINVAL, "layer %d outside [0, %d)", layer, kv->n_layers);
  if (n_rows < 1 || (int64_t)n_rows * n_heads > kMaxRows)
    return ppd_fail(PPD_EINVAL, "n_rows=%d must be positive, with heads at most %d rows", n_rows, kMaxRows);
  if (!row_start || !q) return ppd_fail(PPD_EINVAL, "NULL argument");
  if (dtype != PPD_F32 && dtype != PPD_BF16) return ppd_fail(PPD_EINVAL, "unknown dtype");
  if ((uintptr_t)q % 16) return ppd_fail(PPD_EINVAL, "q must be 16-byte aligned");
  return PPD_OK;
}

}  // namespace

ppd_status paged_check(const ppd_paged *kv, const ppd_page_tables *pt, bool tail) {
  ppd_status st = check_cache(kv);
  if (st != PPD_OK) return st;
  if ((st = check_tables(pt)) != PPD_OK) return st;
  if (pt->page != kv->page || pt->n_pages != kv->n_pages)
    return ppd_fail(PPD_EINVAL, "tables of %d pages of %d positions, a cache of %d of %d", pt->n_pages, pt->page, kv->n_pages,
                    kv->page);
  return tail ? check_kv(&kv->tail, "tail") : PPD_OK;
}

ppd_status paged_check_rows(const ppd_paged *kv, const int32_t *row_start, int n_rows) {
  if (!row_start) return ppd_fail(PPD_EINVAL, "NULL row offsets");
  if (n_rows > kv->tail.capacity)
    return ppd_fail(PPD_ECAPACITY, "%d new rows exceed the tail's capacity %d", n_rows, kv->tail.capacity);
  return PPD_OK;
}

ppd_status paged_check_select(const ppd_paged *kv, int budget, int n_first, int n_last) {
  if (!kv->bounds) return ppd_fail(PPD_EINVAL, "selecting pages needs a cache with bounds");
  if (budget < 1 || n_first < 0 || n_last < 0 || (int64_t)n_first + n_last > budget)
    return ppd_fail(PPD_EINVAL, "budget=%d must be positive and hold n_first=%d and n_last=%d", budget, n_first, n_last);
  return PPD_OK;
}

PagedSeqs paged_seqs(const ppd_page_tables *pt, const int32_t *row_start, int n_rows) {
  PagedSeqs s{};
  s.table = pt->table;
  s.len = pt->len;
  s.row_start = row_start;
  s.B = pt->n_seqs;
  s.max_pages = pt->max_pages;
  s.n_pages = pt->n_pages;
  s.lp = log2_of(pt->page);
  s.n_rows = n_rows;
  return s;
}

extern "C" {

size_t ppd_paged_bytes(int32_t n_layers, int32_t n_kv_heads, int32_t n_pages, int32_t page) {
  if (check_sizes(n_layers, n_kv_heads, n_pages, page) != PPD_OK) return 0;
  return (size_t)n_layers * n_pages * n_kv_heads * (page / kPB) * kPBytes;
}

size_t ppd_paged_bounds_bytes(int32_t n_layers, int32_t n_kv_heads, int32_t n_pages) {
  if (check_sizes(n_layers, n_kv_heads, n_pages, kPB) != PPD_OK) return 0;
  return (size_t)n_layers * n_pages * n_kv_heads * 256 * sizeof(bf16_t);
}

size_t ppd_paged_tables_workspace_bytes(int32_t n_seqs) {
  if (n_seqs < 1 || n_seqs > PPD_PAGED_SEQS_MAX) {
    ppd_fail(PPD_EINVAL, "n_seqs=%d outside [1, %d]", n_seqs, PPD_PAGED_SEQS_MAX);
    return 0;
  }
  return kHeader;
}

ppd_status ppd_paged_tables(const ppd_page_tables *pt, const int32_t *add, int32_t *len_out, int32_t *free_state_out,
                            int32_t *start, int32_t *slots, int32_t n_slots, void *ws, size_t ws_bytes, void *stream) {
  ppd_status st = check_tables(pt);
  if (st != PPD_OK) return st;
  if (!pt->free_pages || !pt->free_state) return ppd_fail(PPD_EINVAL, "the ring of free pages must be set");
  if (!add || !len_out || !free_state_out || !start || !slots) return ppd_fail(PPD_EINVAL, "NULL argument");
  if (n_slots < 1) return ppd_fail(PPD_EINVAL, "n_slots must be positive");
  if ((st = check_work(ws, ws_bytes, ppd_paged_tables_workspace_bytes(pt->n_seqs))) != PPD_OK) return st;
  PagedTablesLaunch p{};
  p.table = pt->table;
  p.free_pages = pt->free_pages;
  p.len = pt->len;
  p.free_state = pt->free_state;
  p.add = add;
  p.len_out = len_out;
  p.free_state_out = free_state_out;
  p.start = start;
  p.slots = slots;
  p.B = pt->n_seqs;
  p.max_pages = pt->max_pages;
  p.n_pages = pt->n_pages;
  p.lp = log2_of(pt->page);
  p.n_slots = n_slots;
  p.ctr = (uint32_t *)ws + 4;
  p.status = (uint32_t *)ws;
  PPD_TRY_HIP(launch_paged_tables(p, (hipStream_t)stream));
  return PPD_OK;
}

ppd_status ppd_paged_store(const ppd_paged *kv, const ppd_kv *src, int32_t n_seqs, const int32_t *start,
                           const int32_t *row_start, const int32_t *path, int32_t n_path, const int32_t *slots,
                           int32_t n_rows, void *stream) {
  ppd_status st = check_cache(kv);
  if (st != PPD_OK) return st;
  if ((st = check_kv(src, "src")) != PPD_OK) return st;
  if (n_seqs < 1 || n_seqs > PPD_PAGED_SEQS_MAX)
    return ppd_fail(PPD_EINVAL, "n_seqs=%d outside [1, %d]", n_seqs, PPD_PAGED_SEQS_MAX);
  if (!start || !row_start || !slots) return ppd_fail(PPD_EINVAL, "NULL argument");
  if (path && n_path < 1) return ppd_fail(PPD_EINVAL, "path must have entries");
  if (n_rows < 1 || n_rows > INT32_MAX / 2) return ppd_fail(PPD_EINVAL, "n_rows must be positive, at most %d", INT32_MAX / 2);
  PagedStoreLaunch p{};
  p.pages = (unsigned char *)kv->pages;
  p.bounds = (bf16_t *)kv->bounds;
  p.k = (const bf16_t *)src->k;
  p.v = (const bf16_t *)src->v;
  p.layers = kv->n_layers;
  p.nkv = kv->n_kv_heads;
  p.n_pages = kv->n_pages;
  p.lp = log2_of(kv->page);
  p.scap = src->capacity;
  p.B = n_seqs;
  p.n_rows = n_rows;
  p.n_path = n_path;
  p.start = start;
  p.row_start = row_start;
  p.path = path;
  p.slots = slots;
  PPD_TRY_HIP(launch_paged_store(p, (hipStream_t)stream));
  return PPD_OK;
}

size_t ppd_paged_attention_workspace_bytes(int32_t n_heads, int32_t n_kv_heads, int32_t n_seqs, int32_t n_rows) {
  if (!heads_ok(n_heads, n_kv_heads) || n_seqs < 1 || n_seqs > PPD_PAGED_SEQS_MAX || n_rows < 1 ||
      (int64_t)n_rows * n_heads > kMaxRows) {
    ppd_fail(PPD_EINVAL, "n_kv_heads must divide n_heads, n_seqs be in [1, %d], n_rows x n_heads in [1, %d]",
             PPD_PAGED_SEQS_MAX, kMaxRows);
    return 0;
  }
  return kHeader + (size_t)PPD_PAGED_SEQS_MAX * sizeof(int2) + paged_attn_part_bytes(n_heads, n_kv_heads, n_seqs, n_rows);
}

ppd_status ppd_paged_attention(int32_t n_heads, const ppd_paged *kv, int32_t layer, const ppd_page_tables *pt,
                               const int32_t *row_start, int32_t n_rows, const void *q, int32_t dtype,
                               const uint64_t *mask, void *out, float *lse, const int32_t *sel, const int32_t *n_sel,
                               int32_t budget, void *ws, size_t ws_bytes, void *stream) {
  ppd_status st = check_call(n_heads, kv, layer, pt, row_start, n_rows, q, dtype);
  if (st != PPD_OK) return st;
  if ((st = check_kv(&kv->tail, "tail")) != PPD_OK) return st;
  if ((st = paged_check_rows(kv, row_start, n_rows)) != PPD_OK) return st;
  if (!out || (sel != nullptr) != (n_sel != nullptr)) return ppd_fail(PPD_EINVAL, "NULL argument");
  if ((uintptr_t)out % 16) return ppd_fail(PPD_EINVAL, "out must be 16-byte aligned");
  const uintptr_t span = (uintptr_t)n_rows * n_heads * 128 * (dtype == PPD_F32 ? 4 : 2);
  if ((uintptr_t)out - (uintptr_t)q < span || (uintptr_t)q - (uintptr_t)out < span)
    return ppd_fail(PPD_EINVAL, "q and out must not overlap");
  if (sel && budget < 1) return ppd_fail(PPD_EINVAL, "budget=%d must be positive", budget);
  if ((st = check_work(ws, ws_bytes, ppd_paged_attention_workspace_bytes(n_heads, kv->n_kv_heads, pt->n_seqs, n_rows))) != PPD_OK)
    return st;
  PagedAttnLaunch a{};
  a.sq = paged_seqs(pt, row_start, n_rows);
  a.pages = (const unsigned char *)kv->pages + (size_t)layer * kv->n_pages * kv->n_kv_heads * (kv->page / kPB) * kPBytes;
  const size_t per_layer = (size_t)kv->n_kv_heads * kv->tail.capacity * 128;
  a.tk = (const bf16_t *)kv->tail.k + layer * per_layer;
  a.tv = (const bf16_t *)kv->tail.v + layer * per_layer;
  a.tcap = kv->tail.capacity;
  a.q = q;
  a.out = out;
  a.q_type = dtype == PPD_F32 ? PAGED_Q_F32 : PAGED_Q_BF16;
  a.mask = mask;
  a.lse = lse;
  a.sel = sel;
  a.n_sel = n_sel;
  a.budget = budget;
  a.nh = n_heads;
  a.nkv = kv->n_kv_heads;
  a.status = (uint32_t *)ws;
  a.ctr = (uint32_t *)((char *)ws + kCounters);  // (zeroed by ppd_workspace_init)
  a.rec = (int2 *)((char *)ws + kHeader);
  a.part = (float *)(a.rec + PPD_PAGED_SEQS_MAX);
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt(128.0));
  paged_attn_shape(a);
  PPD_TRY_HIP(launch_paged_attn(a, (hipStream_t)stream));
  return PPD_OK;
}

size_t ppd_paged_select_workspace_bytes(int32_t n_kv_heads, int32_t n_seqs, int32_t max_pages) {
  if (n_kv_heads < 1 || n_kv_heads > 1 << 16 || n_seqs < 1 || n_seqs > PPD_PAGED_SEQS_MAX || max_pages < 1 ||
      max_pages > PPD_CAPACITY_MAX / PPD_PAGED_BLOCK || (int64_t)n_kv_heads * n_seqs > kMaxRows / 2 ||
      (int64_t)n_kv_heads * n_seqs * max_pages > kMaxKeys) {
    ppd_fail(PPD_EINVAL, "n_kv_heads, n_seqs=%d or max_pages=%d out of range", n_seqs, max_pages);
    return 0;
  }
  return kHeader + paged_select_key_bytes(n_kv_heads, n_seqs, max_pages);
}

ppd_status ppd_paged_select(int32_t n_heads, const ppd_paged *kv, int32_t layer, const ppd_page_tables *pt,
                            const int32_t *row_start, int32_t n_rows, const void *q, int32_t dtype, int32_t budget,
                            int32_t n_first, int32_t n_last, int32_t *sel, int32_t *n_sel, void *ws, size_t ws_bytes,
                            void *stream) {
  ppd_status st = check_call(n_heads, kv, layer, pt, row_start, n_rows, q, dtype);
  if (st != PPD_OK) return st;
  if ((st = paged_check_select(kv, budget, n_first, n_last)) != PPD_OK) return st;
  if (!sel || !n_sel) return ppd_fail(PPD_EINVAL, "NULL argument");
  const size_t need = ppd_paged_select_workspace_bytes(kv->n_kv_heads, pt->n_seqs, pt->max_pages);
  if (!need) return PPD_EINVAL;
  if ((st = check_work(ws, ws_bytes, need)) != PPD_OK) return st;
  PagedSelectLaunch p{};
  p.sq = paged_seqs(pt, row_start, n_rows);
  p.bounds = (const bf16_t *)kv->bounds + (size_t)layer * kv->n_pages * kv->n_kv_heads * 256;
  p.q = q;
  p.q_type = dtype == PPD_F32 ? PAGED_Q_F32 : PAGED_Q_BF16;
  p.nh = n_heads;
  p.nkv = kv->n_kv_heads;
  p.budget = budget;
  p.n_first = n_first;
  p.n_last = n_last;
  p.keys = (unsigned long long *)((char *)ws + kHeader);
  p.sel = sel;
  p.n_sel = n_sel;
  p.status = (uint32_t *)ws;
  PPD_TRY_HIP(launch_paged_select(p, (hipStream_t)stream));
  return PPD_OK;
}

}  // extern "C"
