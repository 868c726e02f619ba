// Host side of the 4-bit cache: argument checks and launches (the step on it is
// ppd_api.cpp's).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ppd_kvq.h"

namespace {

#define PPD_TRY_HIP(call)                                                                   \
  do {                                                                                      \
    hipError_t e_ = (call);                                                                 \
    if (e_ != hipSuccess) return ppd_fail(PPD_EDEVICE, "%s: %s", #call, hipGetErrorString(e_)); \
  } while (0)

constexpr int kMaxHeads = 1 << 20, kMaxQueryHeads = 1 << 16;

// row and head indices are 32-bit in the kernels
bool heads_ok(int n_heads, int n_kv_heads) {
  return n_kv_heads >= 1 && n_heads >= 1 && n_heads <= kMaxQueryHeads && n_heads % n_kv_heads == 0;
}

ppd_status check_sizes(int n_layers, int n_kv_heads, int capacity) {
  if (n_layers < 1 || n_kv_heads < 1) return ppd_fail(PPD_EINVAL, "a cache needs layers and heads");
  if ((int64_t)n_layers * n_kv_heads > kMaxHeads)  // a launch's threads are counted in 32 bits
    return ppd_fail(PPD_EUNSUPPORTED, "%lld layers x heads > %d", (long long)n_layers * n_kv_heads, kMaxHeads);
  if (capacity < kQB || capacity % kQB)
    return ppd_fail(PPD_EUNSUPPORTED, "4-bit caches need a capacity that is a multiple of %d, got %d", kQB, capacity);
  if (capacity > PPD_CAPACITY_MAX)
    return ppd_fail(PPD_EUNSUPPORTED, "capacity %d > %d", capacity, PPD_CAPACITY_MAX);
  return PPD_OK;
}

ppd_status check_kvq(const ppd_kvq *kv) {
  if (!kv || !kv->blocks) return ppd_fail(PPD_EINVAL, "4-bit cache pointer must be set");
  if ((uintptr_t)kv->blocks % 16) return ppd_fail(PPD_EINVAL, "blocks must be 16-byte aligned");
  return check_sizes(kv->n_layers, kv->n_kv_heads, kv->capacity);
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

ppd_status check_range(int pos, int n, int capacity, const char *what) {
  if (pos < 0 || n < 0) return ppd_fail(PPD_EINVAL, "%s: positions must be >= 0", what);
  if ((int64_t)pos + n > capacity)
    return ppd_fail(PPD_ECAPACITY, "%s: positions [%d, %lld) of %d", what, pos, (long long)pos + n, capacity);
  return PPD_OK;
}

ppd_status check_path(const int32_t *path, int path_len, const int32_t *n_path) {
  if (!path || !n_path) return ppd_fail(PPD_EINVAL, "NULL path");
  if (path_len < 1 || path_len > PPD_T_MAX)
    return ppd_fail(PPD_EINVAL, "path_len=%d outside [1, %d]", path_len, PPD_T_MAX);
  return PPD_OK;
}

}  // namespace

ppd_status kvq_check_seqs(int B, const ppd_kvq *kvs, const int32_t *L, const int32_t *T, int *total) {
  if (B < 1 || B > PPD_BATCH_MAX) return ppd_fail(PPD_EINVAL, "B=%d outside [1, %d]", B, PPD_BATCH_MAX);
  if (!kvs || !L || !T) return ppd_fail(PPD_EINVAL, "NULL sequence arrays");
  int64_t all = 0;
  for (int j = 0; j < B; ++j) {
    ppd_status st = check_kvq(&kvs[j]);
    if (st != PPD_OK) return st;
    if ((st = check_kv(&kvs[j].tail, "tail")) != PPD_OK) return st;
    if (T[j] < 1) return ppd_fail(PPD_EINVAL, "T[%d]=%d must be >= 1", j, T[j]);
    if (L[j] < 0) return ppd_fail(PPD_EINVAL, "L[%d] must be >= 0", j);
    if (L[j] > kvs[j].capacity)
      return ppd_fail(PPD_ECAPACITY, "sequence %d: L = %d exceeds capacity %d", j, L[j], kvs[j].capacity);
    if (T[j] > kvs[j].tail.capacity)
      return ppd_fail(PPD_ECAPACITY, "sequence %d: %d tree rows exceed the tail's capacity %d", j, T[j],
                      kvs[j].tail.capacity);
    all += T[j];
  }
  if (all > PPD_T_MAX) return ppd_fail(PPD_EINVAL, "%lld tree tokens in all > %d", (long long)all, PPD_T_MAX);
  *total = (int)all;
  return PPD_OK;
}

KvqSeqs kvq_seqs(int B, const ppd_kvq *kvs, const int32_t *L, const int32_t *T, int layer) {
  KvqSeqs sb{};
  sb.B = B;
  for (int j = 0; j < B; ++j) {
    const ppd_kvq &kv = kvs[j];
    sb.t0[j + 1] = sb.t0[j] + T[j];
    sb.L[j] = L[j];
    sb.nb[j] = kv.capacity / kQB;
    sb.tcap[j] = kv.tail.capacity;
    sb.blocks[j] = (const unsigned char *)kv.blocks + (size_t)layer * kv.n_kv_heads * sb.nb[j] * kQBytes;
    const size_t per_layer = (size_t)kv.n_kv_heads * kv.tail.capacity * 128;
    sb.tk[j] = (const bf16_t *)kv.tail.k + layer * per_layer;
    sb.tv[j] = (const bf16_t *)kv.tail.v + layer * per_layer;
  }
  return sb;
}

extern "C" {

size_t ppd_kvq_bytes(int32_t n_layers, int32_t n_kv_heads, int32_t capacity) {
  if (check_sizes(n_layers, n_kv_heads, capacity) != PPD_OK) return 0;
  return (size_t)n_layers * n_kv_heads * (capacity / kQB) * kQBytes;
}

ppd_status ppd_kvq_quantize(const ppd_kvq *dst, int32_t dst_pos, const ppd_kv *src, int32_t src_pos, int32_t n,
                            void *stream) {
  ppd_status st = check_kvq(dst);
  if (st != PPD_OK) return st;
  if ((st = check_kv(src, "src")) != PPD_OK) return st;
  if ((st = check_range(dst_pos, n, dst->capacity, "dst")) != PPD_OK) return st;
  if ((st = check_range(src_pos, n, src->capacity, "src")) != PPD_OK) return st;
  if (n == 0) return PPD_OK;
  KvqStore p{};
  p.blocks = (unsigned char *)dst->blocks;
  p.k = (const bf16_t *)src->k;
  p.v = (const bf16_t *)src->v;
  p.heads = dst->n_layers * dst->n_kv_heads;
  p.nb = dst->capacity / kQB;
  p.scap = src->capacity;
  p.pos0 = dst_pos;
  p.n = n;
  p.src0 = src_pos;
  PPD_TRY_HIP(launch_kvq_store(p, (hipStream_t)stream));
  return PPD_OK;
}

ppd_status ppd_kvq_dequantize(const ppd_kvq *src, int32_t src_pos, const ppd_kv *dst, int32_t dst_pos, int32_t n,
                              void *stream) {
  ppd_status st = check_kvq(src);
  if (st != PPD_OK) return st;
  if ((st = check_kv(dst, "dst")) != PPD_OK) return st;
  if ((st = check_range(src_pos, n, src->capacity, "src")) != PPD_OK) return st;
  if ((st = check_range(dst_pos, n, dst->capacity, "dst")) != PPD_OK) return st;
  if (n == 0) return PPD_OK;
  KvqLoad p{};
  p.blocks = (const unsigned char *)src->blocks;
  p.k = (bf16_t *)dst->k;
  p.v = (bf16_t *)dst->v;
  p.heads = src->n_layers * src->n_kv_heads;
  p.nb = src->capacity / kQB;
  p.dcap = dst->capacity;
  p.pos0 = src_pos;
  p.n = n;
  p.dst0 = dst_pos;
  PPD_TRY_HIP(launch_kvq_load(p, (hipStream_t)stream));
  return PPD_OK;
}

ppd_status ppd_kvq_commit(const ppd_kvq *kv, int32_t L, const int32_t *path, int32_t path_len,
                          const int32_t *n_path, void *stream) {
  ppd_status st = check_kvq(kv);
  if (st != PPD_OK) return st;
  if ((st = check_kv(&kv->tail, "tail")) != PPD_OK) return st;
  if (L < 0 || L >= kv->capacity)
    return ppd_fail(PPD_ECAPACITY, "L=%d must be in [0, capacity=%d)", L, kv->capacity);
  if ((st = check_path(path, path_len, n_path)) != PPD_OK) return st;
  KvqStore p{};
  p.blocks = (unsigned char *)kv->blocks;
  p.k = (const bf16_t *)kv->tail.k;
  p.v = (const bf16_t *)kv->tail.v;
  p.heads = kv->n_layers * kv->n_kv_heads;
  p.nb = kv->capacity / kQB;
  p.scap = kv->tail.capacity;
  p.pos0 = L;
  p.n = path_len;
  p.path = path;
  p.n_path = n_path;
  p.room = kv->capacity - L;
  p.len_dev = kv->tail.len_dev;
  PPD_TRY_HIP(launch_kvq_store(p, (hipStream_t)stream));
  return PPD_OK;
}

size_t ppd_kvq_attention_workspace_bytes(int32_t n_heads, int32_t n_kv_heads, int32_t t_max) {
  if (!heads_ok(n_heads, n_kv_heads) || t_max < 1 || t_max > PPD_T_MAX) {
    ppd_fail(PPD_EINVAL, "n_kv_heads must divide n_heads <= %d, t_max be in [1, %d]", kMaxQueryHeads, PPD_T_MAX);
    return 0;
  }
  return 256 + kvq_attn_part_bytes(n_heads, n_kv_heads, t_max);
}

ppd_status ppd_kvq_attention(int32_t n_heads, int32_t B, const ppd_kvq *kvs, int32_t layer, const int32_t *L,
                             const int32_t *T, const void *q, const uint64_t *mask, void *out, float *lse, void *ws,
                             size_t ws_bytes, void *stream) {
  int total = 0;
  const ppd_status st = kvq_check_seqs(B, kvs, L, T, &total);
  if (st != PPD_OK) return st;
  const int nkv = kvs[0].n_kv_heads;
  if (!heads_ok(n_heads, nkv)) return ppd_fail(PPD_EINVAL, "n_kv_heads must divide n_heads <= %d", kMaxQueryHeads);
  for (int j = 0; j < B; ++j) {
    if (kvs[j].n_kv_heads != nkv) return ppd_fail(PPD_EINVAL, "sequence %d has %d kv heads, not %d", j, kvs[j].n_kv_heads, nkv);
    if (layer < 0 || layer >= kvs[j].n_layers)
      return ppd_fail(PPD_EINVAL, "layer %d outside [0, %d)", layer, kvs[j].n_layers);
  }
  if (!q || !mask || !out) return ppd_fail(PPD_EINVAL, "NULL argument");
  if ((uintptr_t)q % 16 || (uintptr_t)out % 16) return ppd_fail(PPD_EINVAL, "q and out must be 16-byte aligned");
  const size_t need = ppd_kvq_attention_workspace_bytes(n_heads, nkv, total);
  if (!ws || ws_bytes < need)
    return ppd_fail(PPD_EWORKSPACE, "workspace of %zu bytes is smaller than the %zu required", ws_bytes, need);
  if ((uintptr_t)ws % 16) return ppd_fail(PPD_EINVAL, "ws must be 16-byte aligned");
  KvqAttnLaunch a{};
  a.q = q;
  a.out = out;
  a.mask = mask;
  a.lse = lse;
  a.part = (float *)((char *)ws + 256);
  a.nh = n_heads;
  a.nkv = nkv;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt(128.0));
  a.sb = kvq_seqs(B, kvs, L, T, layer);
  kvq_attn_plan(a);
  PPD_TRY_HIP(launch_kvq_attn(a, (hipStream_t)stream));
  return PPD_OK;
}

ppd_status ppd_kvq_score(const ppd_kvq *kv, int32_t L, int32_t n_heads, int32_t T, const void *q, int32_t q_dtype,
                         const float *lse, int32_t rows, const int32_t *path, int32_t path_len,
                         const int32_t *n_path, const float *score_in, float *score_out, void *stream) {
  ppd_status st = check_kvq(kv);
  if (st != PPD_OK) return st;
  if ((st = check_kv(&kv->tail, "tail")) != PPD_OK) return st;
  if (L < 0 || L > kv->capacity) return ppd_fail(PPD_ECAPACITY, "L=%d must be in [0, capacity=%d]", L, kv->capacity);
  if (!heads_ok(n_heads, kv->n_kv_heads))
    return ppd_fail(PPD_EINVAL, "n_kv_heads must divide n_heads <= %d", kMaxQueryHeads);
  if (T < 1 || T > PPD_T_MAX || rows < T) return ppd_fail(PPD_EINVAL, "T must be in [1, %d], rows at least T", PPD_T_MAX);
  if (T > kv->tail.capacity)
    return ppd_fail(PPD_ECAPACITY, "%d tree rows exceed the tail's capacity %d", T, kv->tail.capacity);
  if (q_dtype != PPD_F32 && q_dtype != PPD_BF16) return ppd_fail(PPD_EINVAL, "unknown dtype");
  if (!q || !lse || !score_out) return ppd_fail(PPD_EINVAL, "NULL argument");
  if ((uintptr_t)q % 16) return ppd_fail(PPD_EINVAL, "q must be 16-byte aligned");
  if ((st = check_path(path, path_len, n_path)) != PPD_OK) return st;
  KvqScoreLaunch p{};
  p.blocks = (const unsigned char *)kv->blocks;
  p.tk = (const bf16_t *)kv->tail.k;
  p.layers = kv->n_layers;
  p.nkv = kv->n_kv_heads;
  p.nh = n_heads;
  p.nb = kv->capacity / kQB;
  p.tcap = kv->tail.capacity;
  p.L = L;
  p.cap = kv->capacity;
  p.q = q;
  p.q_bf16 = q_dtype == PPD_BF16;
  p.rows = rows;
  p.T = T;
  p.lse = lse;
  p.path = path;
  p.n_path = n_path;
  p.path_len = path_len;
  p.in = score_in;
  p.out = score_out;
  p.scale_log2 = (float)(1.4426950408889634 / std::sqrt(128.0));
  PPD_TRY_HIP(launch_kvq_score(p, (hipStream_t)stream));
  return PPD_OK;
}

ppd_status ppd_kvq_evict(const ppd_kvq *src, const ppd_kvq *dst, int32_t L, int32_t budget, int32_t n_sink,
                         int32_t n_recent, const float *score, float *score_out, int32_t *kept, void *stream) {
  ppd_status st = check_kvq(src);
  if (st != PPD_OK) return st;
  if ((st = check_kvq(dst)) != PPD_OK) return st;
  if (src->n_layers != dst->n_layers || src->n_kv_heads != dst->n_kv_heads)
    return ppd_fail(PPD_EINVAL, "src and dst differ in layers or heads");
  if (L < 0 || L > src->capacity) return ppd_fail(PPD_ECAPACITY, "L=%d must be in [0, capacity=%d]", L, src->capacity);
  if (n_sink < 0 || n_recent < 0 || budget < 1 || (int64_t)n_sink + n_recent > budget)
    return ppd_fail(PPD_EINVAL, "budget=%d must be positive and hold n_sink=%d and n_recent=%d", budget, n_sink, n_recent);
  if (budget > dst->capacity) return ppd_fail(PPD_ECAPACITY, "budget=%d exceeds capacity %d", budget, dst->capacity);
  if (!score || !score_out || !kept) return ppd_fail(PPD_EINVAL, "NULL argument");
  const size_t sb = ppd_kvq_bytes(src->n_layers, src->n_kv_heads, src->capacity);
  const size_t db = ppd_kvq_bytes(dst->n_layers, dst->n_kv_heads, dst->capacity);
  const bool same = src->blocks == dst->blocks && src->capacity == dst->capacity;
  const char *s0 = (const char *)src->blocks, *d0 = (const char *)dst->blocks;
  if (!same && s0 < d0 + db && d0 < s0 + sb) return ppd_fail(PPD_EINVAL, "src and dst overlap");
  const size_t heads = (size_t)src->n_layers * src->n_kv_heads;
  const char *si = (const char *)score, *so = (const char *)score_out;
  if (!(si == so && same) && si < so + heads * dst->capacity * 4 && so < si + heads * src->capacity * 4)
    return ppd_fail(PPD_EINVAL, "score and score_out overlap");
  if (L == 0) return PPD_OK;
  KvqEvict p{};
  p.src = (const unsigned char *)src->blocks;
  p.dst = (unsigned char *)dst->blocks;
  p.heads = (int)heads;
  p.src_nb = src->capacity / kQB;
  p.dst_nb = dst->capacity / kQB;
  p.L = L;
  p.n = std::min(L, budget);
  p.n_sink = n_sink;
  p.n_recent = n_recent;
  p.budget = budget;
  p.score = score;
  p.score_out = score_out;
  p.kept = kept;
  PPD_TRY_HIP(launch_kvq_evict(p, (hipStream_t)stream));
  return PPD_OK;
}

}  // extern "C"
