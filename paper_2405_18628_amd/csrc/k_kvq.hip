// The 4-bit cache's own kernels: bf16 rows into blocks and back, and eviction.
//
// A 4-bit block (32 positions of one head) lies in the operand order of the
// attention's matrix instructions (see ppd_kvq in ppd.h).  A wave takes a block
// at a time, lane l = 16 g + r holding what it holds there: of the keys the
// words of position 8 (r / 4) + 4 t + r % 4 (t < 2), dims 32 w + 8 g + e (w < 4);
// of the values those of dims 64 h + 16 w + r (h < 2), positions 8 g + e.  So
// codes are stored and loaded 1 KB a wave, a lane's bf16 pieces are 16 bytes of
// a key's row or of a dim's positions, and nothing passes between waves.
// Nibbles of eight positions share a word of the value codes: a block has one
// writer.
//
// All of them are bound by memory.  (us; 8 layers of 32 heads, 2048 positions)
#include <algorithm>

#include "ppd_kvq.h"

#pragma clang fp contract(off)  // codes are defined by separate float32 operations

namespace {

constexpr int kWaves = 4;  // blocks a workgroup works on together
// 16 bytes at any 2-byte border
typedef unsigned int Piece __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float piece_elem(u32x4 v, int e) {  // e a constant
  return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
}
__device__ __forceinline__ float low16(uint32_t sz) { return __uint_as_float(sz << 16); }
__device__ __forceinline__ float high16(uint32_t sz) { return __uint_as_float(sz & 0xffff0000u); }

// running range of a group
struct Range {
  float lo = INFINITY, hi = -INFINITY;
  uint32_t bad = 0;  // it holds a NaN or an infinity
  __device__ __forceinline__ void add(float v) {
    lo = fminf(lo, v);
    hi = fmaxf(hi, v);
    bad |= (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
  }
  // (scale, zero) of the group
  __device__ __forceinline__ uint32_t pair() const {
    const float r = hi - lo;
    return bad || !(r < INFINITY) ? 0x7fc0u : f32_to_bf16(r / 15.f) | (__float_as_uint(lo) & 0xffff0000u);
  }
};
// over the lanes of a position's key: l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ void join_groups(Range &r) {
  r.lo = -quad_max(-r.lo);
  r.hi = quad_max(r.hi);
  r.bad = quad_max((float)r.bad) > 0.f;
}
// over the 16 lanes of a row
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ void join_step(Range &r) {
  r.lo = fminf(r.lo, dpp<CTRL>(r.lo));
  r.hi = fmaxf(r.hi, dpp<CTRL>(r.hi));
  r.bad |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)r.bad, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ void join_row(Range &r) {
  join_step<0xb1>(r);   // quad_perm [1,0,3,2]
  join_step<0x4e>(r);   // quad_perm [2,3,0,1]
  join_step<0x141>(r);  // row_half_mirror
  join_step<0x140>(r);  // row_mirror
}

// Codes of eight elements (element e with its group's s[e], z[e] and inv[e], about
// 1 / s[e]) as a word.  rint((x - z) / s) is that of the product with inv unless
// that lies within 2^-10 of a half (both quotients are within 2^-16 of each
// other) or is no number; then the division itself decides.
template <typename F>
__device__ __forceinline__ uint32_t code_word(F elem, const float (&s)[8], const float (&z)[8], const float (&inv)[8]) {
  float c[8];
  bool close = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = (elem(e) - z[e]) * inv[e];
    c[e] = rintf(q);
    close |= !(fabsf(fabsf(q - c[e]) - 0.5f) > 0x1p-10f);
  }
  if (close)
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = s[e] > 0.f ? rintf((elem(e) - z[e]) / s[e]) : 0.f;  // 0: an even group, or one without a value
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) w |= (uint32_t)fminf(c[e], 15.f) << kvq_shift(e);
  return w;
}

// ---- bf16 rows -> blocks.  Workgroup (head, run of blocks), a block a wave.
template <bool PATH>
__global__ __launch_bounds__(64 * kWaves) void kvq_store_kernel(KvqStore p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  int n = p.n;
  if constexpr (PATH) {
    n = max(0, min(*p.n_path, min(p.n, p.room)));
    if (p.len_dev && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.len_dev = p.pos0 + n;
  }
  const size_t head = blockIdx.x;
  const bf16_t *ks = p.k + head * p.scap * 128, *vs = p.v + head * 128 * (size_t)p.scap;
  for (int blk = p.pos0 / kQB + blockIdx.y * kWaves + wave; blk * kQB < p.pos0 + n; blk += gridDim.y * kWaves) {
    const int i0 = blk * kQB - p.pos0;                // index of the block's first position in the run
    const int a = max(0, -i0), b = min(kQB, n - i0);  // the block's positions [a, b) are written
    if (a >= b) break;  // an empty path
    auto source = [&](int j) {                        // source row of the block's position j, kept in [a, b)
      const int i = i0 + max(a, min(j, b - 1));
      return PATH ? max(0, min(p.path[i], p.scap - 1)) : p.src0 + i;
    };
    unsigned char *out = p.blocks + (head * p.nb + blk) * (size_t)kQBytes;
    u32x4 kx[2][4], vx[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16_t *row = ks + (size_t)source(kvq_key_of(t, r)) * 128 + 8 * g;
#pragma unroll
      for (int w = 0; w < 4; ++w) kx[t][w] = *(const u32x4 *)(row + 32 * w);
    }
    const bf16_t *col = vs + (size_t)r * p.scap;
    if (!PATH && a == 0 && b == kQB) {
      const bf16_t *at = col + p.src0 + i0 + 8 * g;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int w = 0; w < 4; ++w) vx[h][w] = *(const Piece *)(at + (size_t)(64 * h + 16 * w) * p.scap);
    } else {
      int from[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) from[e] = source(8 * g + e);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bf16_t *at = col + (size_t)(64 * h + 16 * w) * p.scap;
            vx[h][w][e] = at[from[2 * e]] | (uint32_t)at[from[2 * e + 1]] << 16;
          }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = kvq_key_of(t, r);
      u32x4 words;
      uint32_t sz[kGroups];
#pragma unroll
      for (int q = 0; q < kGroups; ++q) {
        Range range;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int e = 0; e < 8; ++e) range.add(piece_elem(kx[t][2 * q + w], e));
        join_groups(range);
        sz[q] = range.pair();
        float s[8], z[8], inv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = low16(sz[q]), z[e] = high16(sz[q]), inv[e] = __builtin_amdgcn_rcpf(s[e]);
#pragma unroll
        for (int w = 0; w < 2; ++w)
          words[2 * q + w] = code_word([&](int e) { return piece_elem(kx[t][2 * q + w], e); }, s, z, inv);
      }
      if (j >= a && j < b) {
        *(u32x4 *)(out + (t * 64 + lane) * 16) = words;
        if (g == 0) *(u32x2 *)(out + kQP + j * 8) = u32x2{sz[0], sz[1]};
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float s[8], z[8], inv[8];
      uint32_t mine = 0;  // position 8 g + r % 8's pair
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        Range range;
#pragma unroll
        for (int w = 0; w < 4; ++w) range.add(piece_elem(vx[h][w], e));
        join_row(range);
        const uint32_t sz = range.pair();
        s[e] = low16(sz), z[e] = high16(sz), inv[e] = __builtin_amdgcn_rcpf(s[e]);
        if ((r & 7) == e) mine = sz;
      }
      u32x4 words;
#pragma unroll
      for (int w = 0; w < 4; ++w) words[w] = code_word([&](int e) { return piece_elem(vx[h][w], e); }, s, z, inv);
      u32x4 *o = (u32x4 *)(out + kQV + (h * 64 + lane) * 16);
      if (8 * g >= a && 8 * g + 8 <= b) {
        *o = words;
      } else if (8 * g < b && 8 * g + 8 > a) {
        uint32_t put = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) put |= 8 * g + e >= a && 8 * g + e < b ? 15u << kvq_shift(e) : 0u;
        const u32x4 old = *o;
        *o = (words & put) | (old & ~put);
      }
      const int j = 8 * g + (r & 7);
      if (r < 8 && j >= a && j < b) *(uint32_t *)(out + kQP + (kQB + j) * 8 + 4 * h) = mine;
    }
  }
}

// a held value: c s is exact (4 and 8 bits), so one rounding
__device__ __forceinline__ float held(float s, float z, uint32_t c) { return (float)c * s + z; }

// ---- blocks -> bf16 rows.  Workgroup (head, run of blocks), a block a wave.
__global__ __launch_bounds__(64 * kWaves) void kvq_load_kernel(KvqLoad p) {
  __shared__ u32x2 par_s[kWaves][2 * kQB];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const size_t head = blockIdx.x;
  bf16_t *ks = p.k + head * p.dcap * 128, *vs = p.v + head * 128 * (size_t)p.dcap;
  for (int blk = p.pos0 / kQB + blockIdx.y * kWaves + wave; blk * kQB < p.pos0 + p.n; blk += gridDim.y * kWaves) {
    const int i0 = blk * kQB - p.pos0;
    const int a = max(0, -i0), b = min(kQB, p.n - i0);
    const unsigned char *in = p.blocks + (head * p.nb + blk) * (size_t)kQBytes;
    u32x4 kw[2], vw[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      kw[t] = __builtin_nontemporal_load((const u32x4 *)(in + (t * 64 + lane) * 16));
      vw[t] = __builtin_nontemporal_load((const u32x4 *)(in + kQV + (t * 64 + lane) * 16));
    }
    par_s[wave][lane] = *(const u32x2 *)(in + kQP + lane * 8);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = kvq_key_of(t, r);
      const u32x2 sz = par_s[wave][j];
      if (j < a || j >= b) continue;
      bf16_t *row = ks + (size_t)(p.dst0 + i0 + j) * 128 + 8 * g;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float s = low16(sz[w >> 1]), z = high16(sz[w >> 1]);
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[e] = pack_bf16x2(held(s, z, (kw[t][w] >> kvq_shift(2 * e)) & 15u), held(s, z, (kw[t][w] >> kvq_shift(2 * e + 1)) & 15u));
        *(u32x4 *)(row + 32 * w) = o;
      }
    }
    bf16_t *at = vs + (size_t)r * p.dcap + p.dst0 + i0 + 8 * g;
    const bool whole = 8 * g >= a && 8 * g + 8 <= b;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float s[8], z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t sz = par_s[wave][kQB + 8 * g + e][h];
        s[e] = low16(sz), z[e] = high16(sz);
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        bf16_t *dst = at + (size_t)(64 * h + 16 * w) * p.dcap;
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[e] = pack_bf16x2(held(s[2 * e], z[2 * e], (vw[h][w] >> kvq_shift(2 * e)) & 15u),
                             held(s[2 * e + 1], z[2 * e + 1], (vw[h][w] >> kvq_shift(2 * e + 1)) & 15u));
        if (whole) {
          *(Piece *)dst = o;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (8 * g + e >= a && 8 * g + e < b) dst[e] = (bf16_t)(o[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the parameters' LDS is written next
  }
}

// ---- eviction, first launch: a head's kept positions.  The scores' order
// words (a float's bits mapped onto unsigned order, -0 as +0, NaN as 0) are
// searched for the last one that is kept, eleven bits at a time by counting;
// then the positions are written in order.
constexpr int kSel = 1024, kBins = 2048, kSelRun = 4;

__device__ __forceinline__ uint32_t order_word(float v) {
  uint32_t b = __float_as_uint(v);
  const uint32_t mag = b & 0x7fffffffu;
  b = mag == 0 ? 0u : b;
  const uint32_t k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return mag > 0x7f800000u ? 0u : k;
}

// sums of two counts over the threads before this one, and over all of them
__device__ __forceinline__ int2 block_before(int2 v, int2 *wave_s, int2 *all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int2 x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int a = __shfl_up(x.x, o, 64), b = __shfl_up(x.y, o, 64);
    if (lane >= o) x.x += a, x.y += b;
  }
  __syncthreads();  // wave_s is free
  if (lane == 63) wave_s[wave] = x;
  __syncthreads();
  int2 before = int2{0, 0}, sum = int2{0, 0};
#pragma unroll
  for (int w = 0; w < kSel / 64; ++w) {
    const int2 s = wave_s[w];
    if (w < wave) before.x += s.x, before.y += s.y;
    sum.x += s.x, sum.y += s.y;
  }
  *all = sum;
  return int2{before.x + x.x - v.x, before.y + x.y - v.y};
}

__global__ __launch_bounds__(kSel) void kvq_select_kernel(KvqEvict p) {
  __shared__ int hist[kBins];
  __shared__ int2 wave_s[kSel / 64];
  __shared__ uint32_t pick_s;
  __shared__ int rest_s;
  const int tid = threadIdx.x;
  const size_t head = blockIdx.x;
  const float *sc = p.score + head * (size_t)p.src_nb * kQB;
  const int m0 = p.n_sink, m1 = p.L - p.n_recent;  // ranked positions
  const int k = p.n - p.n_sink - p.n_recent;       // of which so many are kept
  uint32_t top = 0;  // the last kept order word's upper bits found so far
  int rest = k;      // kept positions among those that share these bits
  if (k > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : kBins;
      hist[tid] = hist[tid + kSel] = 0;
      __syncthreads();
#pragma unroll 4
      for (int i = m0 + tid; i < m1; i += kSel) {
        const uint32_t w = order_word(sc[i]);
        if (pass == 0 || w >> (pass == 1 ? 21 : 10) == top >> (pass == 1 ? 21 : 10))
          atomicAdd(&hist[(w >> shift) & (bins - 1)], 1);
      }
      __syncthreads();
      // bins from the largest on, two a thread: the one that holds the rest-th
      const int b1 = kBins - 1 - 2 * tid;
      const int c1 = hist[b1], c0 = hist[b1 - 1];
      int2 all;
      const int before = block_before(int2{c1 + c0, 0}, wave_s, &all).x;
      if (before < rest && before + c1 >= rest) pick_s = (uint32_t)b1, rest_s = rest - before;
      if (before + c1 < rest && before + c1 + c0 >= rest) pick_s = (uint32_t)(b1 - 1), rest_s = rest - before - c1;
      __syncthreads();
      top |= pick_s << shift;
      rest = rest_s;
      __syncthreads();
    }
  }
  int n_sure = 0, n_eq = 0;
  int32_t *kept = p.kept + head * (size_t)p.budget;
  float *so = p.score_out + head * (size_t)p.dst_nb * kQB;
  for (int c = 0; c < p.L; c += kSel * kSelRun) {
    const int i0 = c + kSelRun * tid;
    float v[kSelRun];
    bool sure[kSelRun], eq[kSelRun];
    int2 mine = int2{0, 0};
#pragma unroll
    for (int e = 0; e < kSelRun; ++e) v[e] = sc[min(i0 + e, p.L - 1)];
#pragma unroll
    for (int e = 0; e < kSelRun; ++e) {
      const int i = i0 + e;
      const uint32_t w = order_word(v[e]);
      const bool ranked = i >= m0 && i < m1;
      sure[e] = i < p.L && (!ranked || (k > 0 && w > top));
      eq[e] = i < p.L && ranked && k > 0 && w == top;
      mine.x += sure[e], mine.y += eq[e];
    }
    int2 all;
    int2 before = block_before(mine, wave_s, &all);
    // (every score of the chunk has been read: score and score_out may be the
    // same, and a position only moves to one that has been read)
    before.x += n_sure, before.y += n_eq;
#pragma unroll
    for (int e = 0; e < kSelRun; ++e) {
      const int at = before.x + min(before.y, max(0, rest));  // equal ones: the first `rest` stay
      if (sure[e] || (eq[e] && before.y < rest)) {
        kept[at] = i0 + e;
        so[at] = v[e];
      }
      before.x += sure[e], before.y += eq[e];
    }
    n_sure += all.x, n_eq += all.y;
  }
}

// ---- eviction, second launch: the kept rows, a destination block a wave.
// WAIT (src is dst, one workgroup a head): a workgroup's blocks are read whole
// before any is written, and the runs follow in order, so that no row is
// overwritten before it was read (a kept position never lies before its place).
template <int W, bool WAIT>
__global__ __launch_bounds__(64 * W) void kvq_gather_kernel(KvqEvict p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const size_t head = blockIdx.x;
  const unsigned char *src = p.src + head * (size_t)p.src_nb * kQBytes;
  const int32_t *kept = p.kept + head * (size_t)p.budget;
  const int nblk = (p.n + kQB - 1) / kQB;
  for (int run = blockIdx.y * W; run < nblk; run += gridDim.y * W) {
    const int blk = run + wave, b = min(kQB, p.n - blk * kQB);  // b <= 0: no block
    unsigned char *out = p.dst + (head * p.dst_nb + blk) * (size_t)kQBytes;
    u32x4 kw[2], vw[2];
    u32x2 par;
    if (b > 0) {
      // this lane's sources: position l % 32's, its keys', its eight positions' (kept once more below the last)
      auto from = [&](int j) { return max(0, min(kept[blk * kQB + min(j, b - 1)], p.L - 1)); };
      const int own = from(lane & 31);
      int at[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int s = __shfl(own, kvq_key_of(t, r), 64), j = s & 31;
        const int m = 4 * (j >> 3) + (j & 3), ts = (j >> 2) & 1;
        kw[t] = *(const u32x4 *)(src + (size_t)(s / kQB) * kQBytes + (ts * 64 + m + 16 * g) * 16);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) at[u] = __shfl(own, 8 * g + u, 64);
      par = *(const u32x2 *)(src + (size_t)(own / kQB) * kQBytes + kQP + ((lane & 32) + (own & 31)) * 8);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
          x[u] = *(const u32x4 *)(src + (size_t)(at[u] / kQB) * kQBytes + kQV + (h * 64 + r + 16 * ((at[u] & 31) >> 3)) * 16);
        vw[h] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int sh = kvq_shift(at[u] & 7);
#pragma unroll
          for (int w = 0; w < 4; ++w) vw[h][w] |= ((x[u][w] >> sh) & 15u) << kvq_shift(u);
        }
        if (8 * g < b && 8 * g + 8 > b) {  // the last positions' word: what lies behind stays
          uint32_t put = 0;
#pragma unroll
          for (int u = 0; u < 8; ++u) put |= 8 * g + u < b ? 15u << kvq_shift(u) : 0u;
          const u32x4 old = *(const u32x4 *)(out + kQV + (h * 64 + lane) * 16);
          vw[h] = (vw[h] & put) | (old & ~put);
        }
      }
    }
    if constexpr (WAIT) {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0);  // every load has returned before the workgroup stores
      __syncthreads();
    }
    if (b > 0) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (kvq_key_of(t, r) < b) *(u32x4 *)(out + (t * 64 + lane) * 16) = kw[t];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (8 * g < b) *(u32x4 *)(out + kQV + (h * 64 + lane) * 16) = vw[h];
      if ((lane & 31) < b) *(u32x2 *)(out + kQP + lane * 8) = par;
    }
    if constexpr (WAIT) __syncthreads();
  }
}

int runs_of(int pos0, int n, int waves) {
  return std::min(65535, ((pos0 % kQB + n + kQB - 1) / kQB + waves - 1) / waves);
}

}  // namespace

hipError_t launch_kvq_store(const KvqStore &p, hipStream_t s) {
  const dim3 grid(p.heads, runs_of(p.pos0, p.n, kWaves)), block(64 * kWaves);
  if (p.path)
    hipLaunchKernelGGL(kvq_store_kernel<true>, grid, block, 0, s, p);
  else
    hipLaunchKernelGGL(kvq_store_kernel<false>, grid, block, 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kvq_load(const KvqLoad &p, hipStream_t s) {
  hipLaunchKernelGGL(kvq_load_kernel, dim3(p.heads, runs_of(p.pos0, p.n, kWaves)), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kvq_evict(const KvqEvict &p, hipStream_t s) {
  hipLaunchKernelGGL(kvq_select_kernel, dim3(p.heads), dim3(kSel), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.src == p.dst)
    hipLaunchKernelGGL((kvq_gather_kernel<16, true>), dim3(p.heads, 1), dim3(64 * 16), 0, s, p);
  else
    hipLaunchKernelGGL((kvq_gather_kernel<kWaves, false>), dim3(p.heads, runs_of(0, p.n, kWaves)), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}
