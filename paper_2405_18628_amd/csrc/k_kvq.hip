// The 4-bit cache's own kernels: bf16 rows into blocks and back, and eviction.
//
// A 4-bit block (32 positions of one head) lies in the operand order of the
// attention's matrix instructions (see ppd_kvq in ppd.h), so storing rows is a
// transposition of codes, and a block is the unit of work here: nibbles of
// different positions share the words of the value codes, and a block has one
// writer.
#include <algorithm>

#include "ppd_kvq.h"

#pragma clang fp contract(off)  // codes are defined by separate float32 operations

namespace {

constexpr int kRow = 132;  // LDS row of 128 elements, padded

// codes' group of 64 in a row: (scale, zero) pair of n finite elements
struct Range {
  float lo, hi;
  bool bad;
};

// ---- bf16 rows -> block.  Workgroup: (head, block); 256 threads.
__global__ __launch_bounds__(256) void kvq_store_kernel(KvqStore p) {
  __shared__ float x[2][kQB][kRow];          // keys, values [position][dim]
  __shared__ uint32_t sz[2][kQB][kGroups];
  const int tid = threadIdx.x;
  int n = p.n;
  if (p.path) n = max(0, min(*p.n_path, min(p.n, p.room)));
  if (p.len_dev && blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) *p.len_dev = p.pos0 + n;
  const size_t head = blockIdx.x;
  for (int blk = p.pos0 / kQB + blockIdx.y; blk * kQB < p.pos0 + n; blk += gridDim.y) {
  const int i0 = blk * kQB - p.pos0;             // index of the block's first position in the run
  const int a = max(0, -i0), b = min(kQB, n - i0);  // the block's positions [a, b) are written
  const bf16_t *ks = p.k + head * p.scap * 128, *vs = p.v + head * 128 * (size_t)p.scap;
  auto source = [&](int j) { return p.path ? max(0, min(p.path[i0 + j], p.scap - 1)) : p.src0 + i0 + j; };
  for (int e = tid; e < kQB * 128; e += 256) {
    const int j = e >> 7, d = e & 127;
    if (j >= a && j < b) x[0][j][d] = bf16_to_f32(ks[(size_t)source(j) * 128 + d]);
  }
  for (int e = tid; e < kQB * 128; e += 256) {
    const int j = e & 31, d = e >> 5;
    if (j >= a && j < b) x[1][j][d] = bf16_to_f32(vs[(size_t)d * p.scap + source(j)]);
  }
  __syncthreads();
  if (tid < 2 * kQB * kGroups) {
    const int w = tid / (kQB * kGroups), j = tid / kGroups % kQB, g = tid % kGroups;
    if (j >= a && j < b) {
      float lo = INFINITY, hi = -INFINITY;
      bool bad = false;
      for (int d = 0; d < 64; ++d) {
        const float v = x[w][j][64 * g + d];
        bad |= !(fabsf(v) < INFINITY);
        lo = fminf(lo, v);
        hi = fmaxf(hi, v);
      }
      const float r = hi - lo;
      bad |= !(r < INFINITY);
      const uint32_t s = bad ? 0x7fc0u : f32_to_bf16(r / 15.f);
      sz[w][j][g] = s | (bad ? 0u : (__float_as_uint(lo) & 0xffff0000u));
    }
  }
  __syncthreads();
  auto code = [&](int w, int j, int d) -> uint32_t {
    const uint32_t q = sz[w][j][d >> 6];
    const float s = __uint_as_float(q << 16), z = __uint_as_float(q & 0xffff0000u);
    if (!(s > 0.f)) return 0u;  // an even group, or one without a value
    return (uint32_t)fminf(15.f, rintf((x[w][j][d] - z) / s));
  };
  unsigned char *out = p.blocks + (head * p.nb + blk) * (size_t)kQBytes;
  for (int e = tid; e < 512; e += 256) {  // key words: the position's own
    const int t = e >> 8, lane = (e >> 2) & 63, w = e & 3;
    const int j = kvq_key_of(t, lane & 15), d = 32 * w + 8 * (lane >> 4);
    if (j < a || j >= b) continue;
    uint32_t v = 0;
    for (int i = 0; i < 8; ++i) v |= code(0, j, d + i) << kvq_shift(i);
    ((uint32_t *)out)[e] = v;
  }
  for (int e = tid; e < 512; e += 256) {  // value words: eight positions of a dim
    const int h = e >> 8, lane = (e >> 2) & 63, w = e & 3;
    const int d = 64 * h + 16 * w + (lane & 15), j0 = 8 * (lane >> 4);
    if (j0 >= b || j0 + 8 <= a) continue;
    uint32_t v = 0, keep = 0;
    for (int i = 0; i < 8; ++i) {
      if (j0 + i >= a && j0 + i < b)
        v |= code(1, j0 + i, d) << kvq_shift(i);
      else
        keep |= 15u << kvq_shift(i);
    }
    uint32_t *o = (uint32_t *)(out + kQV) + e;
    *o = keep ? v | (*o & keep) : v;
  }
  if (tid < 2 * kQB * kGroups) {
    const int w = tid / (kQB * kGroups), j = tid / kGroups % kQB, g = tid % kGroups;
    if (j >= a && j < b) ((uint32_t *)(out + kQP))[(w * kQB + j) * kGroups + g] = sz[w][j][g];
  }
  __syncthreads();
  }
}

// held value of code c
__device__ __forceinline__ float held(uint32_t sz, uint32_t c) {
  return (float)c * __uint_as_float(sz << 16) + __uint_as_float(sz & 0xffff0000u);
}

// ---- block -> bf16 rows.  Workgroup: (head, block); 256 threads.
__global__ __launch_bounds__(256) void kvq_load_kernel(KvqLoad p) {
  __shared__ uint32_t blk_s[kQBytes / 4];
  const int tid = threadIdx.x;
  const size_t head = blockIdx.x;
  for (int blk = p.pos0 / kQB + blockIdx.y; blk * kQB < p.pos0 + p.n; blk += gridDim.y) {
  const int i0 = blk * kQB - p.pos0;
  const int a = max(0, -i0), b = min(kQB, p.n - i0);
  const u32x4 *in = (const u32x4 *)(p.blocks + (head * p.nb + blk) * (size_t)kQBytes);
  for (int e = tid; e < kQBytes / 16; e += 256) ((u32x4 *)blk_s)[e] = in[e];
  __syncthreads();
  const uint32_t *par = blk_s + kQP / 4;
  bf16_t *ks = p.k + head * p.dcap * 128, *vs = p.v + head * 128 * (size_t)p.dcap;
  for (int e = tid; e < kQB * 128; e += 256) {
    const int j = e >> 7, d = e & 127;
    if (j < a || j >= b) continue;
    const int m = 4 * (j >> 3) + (j & 3), t = (j >> 2) & 1;
    const uint32_t w = blk_s[(t * 64 + m + 16 * ((d >> 3) & 3)) * 4 + (d >> 5)];
    ks[(size_t)(p.dst0 + i0 + j) * 128 + d] =
        f32_to_bf16(held(par[j * kGroups + (d >> 6)], (w >> kvq_shift(d & 7)) & 15u));
  }
  for (int e = tid; e < kQB * 128; e += 256) {
    const int j = e & 31, d = e >> 5;
    if (j < a || j >= b) continue;
    const uint32_t w = blk_s[kQV / 4 + ((d >> 6) * 64 + (d & 15) + 16 * (j >> 3)) * 4 + ((d >> 4) & 3)];
    vs[(size_t)d * p.dcap + p.dst0 + i0 + j] =
        f32_to_bf16(held(par[(kQB + j) * kGroups + (d >> 6)], (w >> kvq_shift(j & 7)) & 15u));
  }
  __syncthreads();
  }
}

// ---- eviction, first launch: a head's kept positions.  The scores' order
// words (a float's bits mapped onto unsigned order, -0 as +0, NaN as 0) are
// searched for the last one that is kept, eight bits at a time; then the
// positions are written in order.
constexpr int kSel = 1024;

__device__ __forceinline__ uint32_t order_word(float v) {
  uint32_t b = __float_as_uint(v);
  const uint32_t mag = b & 0x7fffffffu;
  b = mag == 0 ? 0u : b;
  const uint32_t k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return mag > 0x7f800000u ? 0u : k;
}

// sum of v over the threads before this one (and over all of them in *total)
__device__ __forceinline__ int block_prefix(int v, int *wave_s, int *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();  // wave_s is free
  if (lane == 63) wave_s[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kSel / 64; ++w) {
    if (w < wave) before += wave_s[w];
    all += wave_s[w];
  }
  *total = all;
  return before + x - v;
}

__global__ __launch_bounds__(kSel) void kvq_select_kernel(KvqEvict p) {
  __shared__ int hist[256];
  __shared__ int wave_s[kSel / 64];
  __shared__ uint32_t pick_s;
  __shared__ int rest_s;
  const int tid = threadIdx.x;
  const size_t head = blockIdx.x;
  const float *sc = p.score + head * (size_t)p.src_nb * kQB;
  const int m0 = p.n_sink, m1 = p.L - p.n_recent;  // ranked positions
  const int k = p.n - p.n_sink - p.n_recent;       // of which so many are kept
  uint32_t top = 0;   // the last kept order word's upper bits found so far
  int rest = k;       // kept positions among those that share these bits
  if (k > 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = m0 + tid; i < m1; i += kSel) {
        const uint32_t w = order_word(sc[i]);
        if (shift == 24 || (w >> (shift + 8)) == (top >> (shift + 8))) atomicAdd(&hist[(w >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int b = 255, left = rest;
        while (b > 0 && hist[b] < left) left -= hist[b--];
        pick_s = (uint32_t)b;
        rest_s = left;
      }
      __syncthreads();
      top |= pick_s << shift;
      rest = rest_s;
    }
  int n_kept = 0, n_eq = 0;
  int32_t *kept = p.kept + head * (size_t)p.budget;
  float *so = p.score_out + head * (size_t)p.dst_nb * kQB;
  for (int c = 0; c < p.L; c += kSel) {
    const int i = c + tid;
    float v = 0.f;
    bool keep = false, eq = false;
    if (i < p.L) {
      v = sc[i];
      if (i < m0 || i >= m1) {
        keep = true;
      } else if (k > 0) {
        const uint32_t w = order_word(v);
        keep = w > top;
        eq = w == top;
      }
    }
    int all;
    const int before = block_prefix(eq, wave_s, &all);
    keep |= eq && n_eq + before < rest;
    n_eq += all;
    const int at = n_kept + block_prefix(keep, wave_s, &all);
    // (the barrier in between: score and score_out may be the same, and a
    // position is only moved to one that has been read)
    if (keep) {
      kept[at] = i;
      so[at] = v;
    }
    n_kept += all;
  }
}

// ---- eviction, second launch: the kept rows.  256 threads a block; a
// workgroup moves every step-th block of a head's destination from `first` on,
// each read in whole before it is written (where src is dst one workgroup
// moves all of them in order: a kept position never lies before its place).
__global__ __launch_bounds__(256) void kvq_gather_kernel(KvqEvict p) {
  __shared__ int at_s[kQB];
  const int tid = threadIdx.x;
  const size_t head = blockIdx.x;
  const unsigned char *src = p.src + head * (size_t)p.src_nb * kQBytes;
  const int32_t *kept = p.kept + head * (size_t)p.budget;
  for (int blk = blockIdx.y; blk * kQB < p.n; blk += gridDim.y) {
    const int b = min(kQB, p.n - blk * kQB);
    __syncthreads();
    if (tid < kQB) at_s[tid] = tid < b ? max(0, min(kept[blk * kQB + tid], p.L - 1)) : -1;
    __syncthreads();
    unsigned char *out = p.dst + (head * p.dst_nb + blk) * (size_t)kQBytes;
    auto block_of = [&](int at) { return src + (size_t)(at / kQB) * kQBytes; };
    uint32_t kw[2] = {0, 0}, vw[2], pw = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = tid + 256 * i;
      {
        const int t = e >> 8, lane = (e >> 2) & 63, w = e & 3;
        const int at = at_s[kvq_key_of(t, lane & 15)];
        if (at >= 0) {
          const int j = at & 31, m = 4 * (j >> 3) + (j & 3), ts = (j >> 2) & 1;
          kw[i] = ((const uint32_t *)block_of(at))[(ts * 64 + m + (lane & 48)) * 4 + w];
        }
      }
      {
        const int lane = (e >> 2) & 63, j0 = 8 * (lane >> 4);
        uint32_t v = 0, keep = 0;
        for (int u = 0; u < 8; ++u) {
          const int at = at_s[j0 + u];
          if (at >= 0) {
            const int j = at & 31;
            const uint32_t w = ((const uint32_t *)(block_of(at) + kQV))[(e & ~(48 << 2)) | ((j >> 3) << 6)];
            v |= ((w >> kvq_shift(j & 7)) & 15u) << kvq_shift(u);
          } else {
            keep |= 15u << kvq_shift(u);
          }
        }
        if (keep && keep != ~0u) v |= ((const uint32_t *)(out + kQV))[e] & keep;
        vw[i] = v;
      }
    }
    if (tid < 2 * kQB * kGroups) {
      const int w = tid / (kQB * kGroups), j = tid / kGroups % kQB, g = tid % kGroups;
      const int at = at_s[j];
      if (at >= 0) pw = ((const uint32_t *)(block_of(at) + kQP))[(w * kQB + (at & 31)) * kGroups + g];
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);  // every load has returned before the workgroup stores
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = tid + 256 * i, lane = (e >> 2) & 63;
      if (at_s[kvq_key_of(e >> 8, lane & 15)] >= 0) ((uint32_t *)out)[e] = kw[i];
      if (at_s[8 * (lane >> 4)] >= 0) ((uint32_t *)(out + kQV))[e] = vw[i];
    }
    if (tid < 2 * kQB * kGroups && at_s[tid / kGroups % kQB] >= 0) ((uint32_t *)(out + kQP))[tid] = pw;
  }
}

}  // namespace

hipError_t launch_kvq_store(const KvqStore &p, hipStream_t s) {
  const int blocks = (p.pos0 % kQB + p.n + kQB - 1) / kQB;
  hipLaunchKernelGGL(kvq_store_kernel, dim3(p.heads, std::min(blocks, 65535)), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kvq_load(const KvqLoad &p, hipStream_t s) {
  const int blocks = (p.pos0 % kQB + p.n + kQB - 1) / kQB;
  hipLaunchKernelGGL(kvq_load_kernel, dim3(p.heads, std::min(blocks, 65535)), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kvq_evict(const KvqEvict &p, hipStream_t s) {
  hipLaunchKernelGGL(kvq_select_kernel, dim3(p.heads), dim3(kSel), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = (p.n + kQB - 1) / kQB;
  const bool same = p.src == p.dst;
  hipLaunchKernelGGL(kvq_gather_kernel, dim3(p.heads, same ? 1 : std::min(blocks, 65535)), dim3(256), 0, s, p);
  return hipGetLastError();
}
