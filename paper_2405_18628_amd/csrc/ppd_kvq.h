// The 4-bit cache (ppd_kvq): block layout, code conversions and launchers.
#pragma once

#include "ppd_internal.h"

constexpr int kQB = PPD_KVQ_BLOCK;             // positions of a block
constexpr int kQBytes = PPD_KVQ_BLOCK_BYTES;   // keys' codes, values' codes, parameters
constexpr int kQV = 2048, kQP = 4096;          // the values' codes, the parameters
constexpr int kGroups = 2;                     // 64-dim groups of a row

// position (of its block) that row m of key tile t holds
__host__ __device__ __forceinline__ int kvq_key_of(int t, int m) { return 8 * (m >> 2) + 4 * t + (m & 3); }

// Operand fragment of a code word: elements e of the word as bfloat16 pairs
// (2 j, 2 j + 1), each (16 + c) / 2 -- the code in the upper mantissa bits of
// 8.0, so a pair costs a shift and an and-or.  With it a row's value s c + z is
// (2 s) x + (z - 16 s) of the operand element x: exact products on the matrix
// cores, the scale and the zero applied to their float32 sums.
// (The mask and the magic bits are kept in registers: as literals they take an
// instruction each.)
struct KvqBits {
  uint32_t mask = 0x00780078u, magic = 0x41004100u;
  __device__ __forceinline__ KvqBits() { asm("" : "+v"(mask), "+v"(magic)); }
};
__device__ __forceinline__ u32x4 kvq_expand(uint32_t w, const KvqBits &k) {
  return u32x4{((w << 3) & k.mask) | k.magic, ((w >> 1) & k.mask) | k.magic, ((w >> 5) & k.mask) | k.magic,
               ((w >> 9) & k.mask) | k.magic};
}
// a (scale, zero) pair as (2 s, z - 16 s).  With rows of magnitude M both times
// x or 1 stay below 4.2 M and 3.2 M (s < 2.01 M / 15), so with 2^24 keys and
// probabilities of up to 2^8 a sum stays below 2^35 M, a score's below 2^10 M |q|:
// M = 2^90 and M |q| = 2^116 are the documented limits (float32 ends at 2^128;
// z - 16 s itself from M = 2^126 on).
__device__ __forceinline__ float2 kvq_affine(uint32_t sz) {
  const float s = __uint_as_float(sz << 16), z = __uint_as_float(sz & 0xffff0000u);
  return float2{2.f * s, fmaf(-16.f, s, z)};
}
// element e's bit position in its word
__host__ __device__ __forceinline__ int kvq_shift(int e) { return 4 * (e >> 1) + 16 * (e & 1); }

// ---- bf16 rows into blocks: positions [pos0, pos0 + n) of every head from
// source rows (path null) src0 + i or path[i]
struct KvqStore {
  unsigned char *blocks;
  const bf16_t *k, *v;  // [heads][scap][128], [heads][128][scap]
  int heads, nb, scap;  // heads: layers x kv heads; nb: blocks a head
  int pos0, n;          // path: n = its length
  int src0;
  const int32_t *path, *n_path;
  int room;             // path: positions of the cache from pos0 on
  int32_t *len_dev;
  int runs;             // workgroups a head (the launcher's)
};
hipError_t launch_kvq_store(KvqStore p, hipStream_t s);

struct KvqLoad {
  const unsigned char *blocks;
  bf16_t *k, *v;
  int heads, nb, dcap;
  int pos0, n, dst0;
  int runs;
};
hipError_t launch_kvq_load(KvqLoad p, hipStream_t s);

struct KvqEvict {
  const unsigned char *src;
  unsigned char *dst;
  int heads, src_nb, dst_nb;
  int L, n, n_sink, n_recent, budget;
  const float *score;
  float *score_out;
  int32_t *kept;
  int runs;
};
hipError_t launch_kvq_evict(KvqEvict p, hipStream_t s);

// ---- attention over 4-bit prefixes and bf16 tree rows
struct KvqSeqs {
  int B;
  int t0[PPD_BATCH_MAX + 1];  // t0[B]: all tokens
  int L[PPD_BATCH_MAX];
  int nb[PPD_BATCH_MAX];      // blocks a head
  int tcap[PPD_BATCH_MAX];    // tail capacity
  const unsigned char *blocks[PPD_BATCH_MAX];       // this layer's
  const bf16_t *tk[PPD_BATCH_MAX], *tv[PPD_BATCH_MAX];  // this layer's tree rows
};

struct KvqAttnLaunch {
  const void *q;        // operand planes [T_pad][nh 128], or bfloat16 rows [T][nh][128]
  void *out;            // likewise
  int planes, T_pad;
  const uint64_t *mask; // [T][2]
  float *lse;           // [T][nh] or null
  float *q_out;         // planes: float32 rows [T][nh][128], or null
  float *part;          // [splits][T][nh][PPD_ATTN_OROW]
  int nh, nkv;
  int tiles;            // most 16-row tiles of a kv head's rows (tree rows x heads that share it)
  KvqSeqs sb;
  // sequence s: slots slot0[s] + ((kv head x row groups + row group) x splits[s] + split), a split
  // holding chunk[s] 32-key blocks
  int slot0[PPD_BATCH_MAX], splits[PPD_BATCH_MAX], chunk[PPD_BATCH_MAX];
  int n_slots;
  float scale_log2;
  void *ev_start, *ev_stop;
};
// most splits a (kv head, row group) is cut into, and the bytes of `part`
int kvq_attn_max_splits(int nkv);
size_t kvq_attn_part_bytes(int nh, int nkv, int T);
// splits of the sequences (fills tiles, slot0, splits, chunk, n_slots)
void kvq_attn_plan(KvqAttnLaunch &a);
hipError_t launch_kvq_attn(const KvqAttnLaunch &a, hipStream_t s);

struct KvqScoreLaunch {
  const unsigned char *blocks;
  const bf16_t *tk;
  int layers, nkv, nh, nb, tcap, L, cap;
  const void *q;
  int q_bf16, rows, T;
  const float *lse;
  const int32_t *path, *n_path;
  int path_len;
  const float *in;
  float *out;
  float scale_log2;
  int runs;  // workgroups a (layer, kv head) (the launcher's)
};
hipError_t launch_kvq_score(KvqScoreLaunch p, hipStream_t s);

// The step of ppd_api.cpp on 4-bit caches
struct KvqStep {
  const ppd_kvq *kvs;
  const int32_t *L, *pos;
  float *q_out, *lse_out;
};
// the arguments of a batch (ppd_kvq.cpp); *total: all tree tokens
ppd_status kvq_check_seqs(int B, const ppd_kvq *kvs, const int32_t *L, const int32_t *T, int *total);
KvqSeqs kvq_seqs(int B, const ppd_kvq *kvs, const int32_t *L, const int32_t *T, int layer);
