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
// All of them are bound by memory (a large copy runs at 4.8 TB/s here).  8 layers
// of 32 heads: 2048 positions to 4 bits 73 us (4.7 TB/s; 1730 vector
// instructions a block, 50 us of them, behind the loads), back 66 us (5.2 TB/s);
// of 4096 positions 2048 kept 13.8 + 44 us (5.2 TB/s counting the lines of rows
// that go, in place 12.5 + 35).  A path's rows: 1024 heads, five rows, 12.8 us, a
// chain of three round trips (path, rows, the words that neighbours share) and 3
// us of codes.  Bf16 key rows bypass the caches (with them to 4 bits 92 us, back
// 77); codes do not, they are read again soon.
#include <algorithm>
#include <type_traits>

#include "ppd_kvq.h"

#pragma clang fp contract(off)  // codes are defined by separate float32 operations

namespace {

template <int N>
using Const = std::integral_constant<int, N>;

constexpr int kWaves = 4;  // blocks a workgroup works on together
// 16 bytes at any 2-byte border
typedef unsigned int Piece __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float piece_elem(u32x4 v, int e) {  // e a constant
  return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
}
__device__ __forceinline__ float low16(uint32_t sz) { return __uint_as_float(sz << 16); }
__device__ __forceinline__ float high16(uint32_t sz) { return __uint_as_float(sz & 0xffff0000u); }

// ---- ranges, on bfloat16 pairs as they are loaded: the bits of a number with
// those of a negative one flipped order as 16-bit integers do, infinities and
// NaN at the ends
typedef short Pair __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pmin(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(Pair, a), __builtin_bit_cast(Pair, b)));
}
__device__ __forceinline__ uint32_t pmax(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Pair, a), __builtin_bit_cast(Pair, b)));
}
// to the order and back
__device__ __forceinline__ uint32_t ordered(uint32_t x) {
  const Pair sign = __builtin_bit_cast(Pair, x) >> (Pair){15, 15};
  return x ^ (__builtin_bit_cast(uint32_t, sign) & 0x7fff7fffu);
}
struct Range {  // of the pair's two numbers, in the order
  uint32_t lo = 0x7fff7fffu, hi = 0x80008000u;
  __device__ __forceinline__ void add(uint32_t pair) {
    const uint32_t x = ordered(pair);
    lo = pmin(lo, x);
    hi = pmax(hi, x);
  }
  __device__ __forceinline__ void join(uint32_t l, uint32_t h) {
    lo = pmin(lo, l);
    hi = pmax(hi, h);
  }
};
// over both halves and the lanes of a position's key: l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ void join_groups(Range &r) {
  r.join(r.lo >> 16 | r.lo << 16, r.hi >> 16 | r.hi << 16);
  auto l16 = __builtin_amdgcn_permlane16_swap(r.lo, r.lo, false, false);
  auto h16 = __builtin_amdgcn_permlane16_swap(r.hi, r.hi, false, false);
  r.lo = pmin(l16[0], l16[1]);
  r.hi = pmax(h16[0], h16[1]);
  auto l32 = __builtin_amdgcn_permlane32_swap(r.lo, r.lo, false, false);
  auto h32 = __builtin_amdgcn_permlane32_swap(r.hi, r.hi, false, false);
  r.lo = pmin(l32[0], l32[1]);
  r.hi = pmax(h32[0], h32[1]);
}
// over the 16 lanes of a row
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ void join_row(Range &r) {
  r.join(dpp<0xb1>(r.lo), dpp<0xb1>(r.hi));    // quad_perm [1,0,3,2]
  r.join(dpp<0x4e>(r.lo), dpp<0x4e>(r.hi));    // quad_perm [2,3,0,1]
  r.join(dpp<0x141>(r.lo), dpp<0x141>(r.hi));  // row_half_mirror
  r.join(dpp<0x140>(r.lo), dpp<0x140>(r.hi));  // row_mirror
}

// A group's (scale, zero) pair and the reciprocal that its codes are taken with
// (0 for an even group); `odd`: a group without a value, or a scale so small
// that remainders underflow.
struct Affine {
  uint32_t pair;
  float inv;
  bool odd;
  // lo, hi: the range in the order, in the low halves
  __device__ __forceinline__ Affine(uint32_t lo, uint32_t hi) {
    const float l = __uint_as_float(ordered(lo) << 16), h = __uint_as_float(ordered(hi) << 16);
    const bool end = (int16_t)hi >= 0x7f80 || (int16_t)lo <= (int16_t)0x807f;
    const float r = h - l;
    // r / 15, correctly rounded: the remainder of the product with RN(1 / 15)
    // corrects it (checked for every mantissa; subnormal quotients are divided)
    const float q0 = r * (1.f / 15.f);
    float q = fmaf(fmaf(-15.f, q0, r), 1.f / 15.f, q0);
    const bool tiny = r < 0x1p-90f;
    if (__ballot(tiny)) q = tiny ? r / 15.f : q;
    const bool none = end || !(r < INFINITY);
    pair = none ? 0x7fc0u : f32_to_bf16(q) | (__float_as_uint(l) & 0xffff0000u);
    const float s = low16(pair), y = __builtin_amdgcn_rcpf(s);
    inv = s > 0.f ? fmaf(fmaf(-s, y, 1.f), y, y) : 0.f;
    odd = none || tiny;
  }
  __device__ __forceinline__ Affine(uint32_t pair_, float inv_) : pair(pair_), inv(inv_), odd(false) {}
  // rint of the float32 quotient (x - z) / s: a product with the reciprocal and
  // one correction by its remainder give it to the last bit, so that a quotient
  // that is exactly a half is one here (with bfloat16 rows these are common)
  __device__ __forceinline__ float code(float x) const {
    const float s = low16(pair), d = x - high16(pair), q0 = d * inv;
    return rintf(fmaf(fmaf(-q0, s, d), inv, q0));
  }
  __device__ __forceinline__ float divide(float x) const {
    const float s = low16(pair), z = high16(pair);
    return s > 0.f ? fminf(rintf((x - z) / s), 15.f) : 0.f;
  }
};

// Codes of eight elements as a word, its two halves put together in float32
// (16 bits, exact).
template <typename X, typename A>
__device__ __forceinline__ uint32_t code_word(X x, A affine, bool odd) {
  float lo = 0.f, hi = 0.f;
#pragma unroll
  for (int e = 7; e >= 0; --e) {
    const float c = affine(e).code(x(e));
    if (e & 1)
      hi = fmaf(hi, 16.f, c);
    else
      lo = fmaf(lo, 16.f, c);
  }
  uint32_t w = (uint32_t)lo | (uint32_t)hi << 16;
  if (odd) {
    w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= (uint32_t)affine(e).divide(x(e)) << kvq_shift(e);
  }
  return w;
}

// ---- bf16 rows -> blocks.  Workgroup (head, run of W blocks), a block a wave.
template <int W, bool PATH>
__global__ __launch_bounds__(64 * W, 2) void kvq_store_kernel(KvqStore p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  // (most runs behind a path's first are empty: the heads' first ones come first)
  const size_t head = PATH ? blockIdx.x % p.heads : blockIdx.x / p.runs;
  const int run0 = PATH ? blockIdx.x / p.heads : blockIdx.x % p.runs;
  const bf16_t *ks = p.k + head * p.scap * 128, *vs = p.v + head * 128 * (size_t)p.scap;
  for (int blk = p.pos0 / kQB + run0 * W + wave; blk * kQB < p.pos0 + p.n; blk += p.runs * W) {
    const int i0 = blk * kQB - p.pos0;  // index of the block's first position in the run
    int n = p.n, own = 0;
    if constexpr (PATH) {
      // the path is read beside its length
      own = max(0, min(p.path[max(0, min(i0 + (lane & 31), p.n - 1))], p.scap - 1));
      n = max(0, min(*p.n_path, min(p.n, p.room)));
      if (p.len_dev && blockIdx.x == 0 && threadIdx.x == 0) *p.len_dev = p.pos0 + n;
    }
    const int a = max(0, -i0), b = min(kQB, n - i0);  // the block's positions [a, b) are written
    if (a >= b) return;                               // a shorter path: no later block either
    auto source = [&](int j) {                        // source row of the block's position j, kept in [a, b)
      j = max(a, min(j, b - 1));
      return PATH ? __shfl(own, j, 64) : p.src0 + i0 + j;
    };
    const bool all = !PATH && a == 0 && b == kQB;
    unsigned char *out = p.blocks + (head * p.nb + blk) * (size_t)kQBytes;
    u32x4 kx[2][4], vx[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16_t *row = ks + (size_t)source(kvq_key_of(t, r)) * 128 + 8 * g;
#pragma unroll
      for (int w = 0; w < 4; ++w) kx[t][w] = __builtin_nontemporal_load((const u32x4 *)(row + 32 * w));
    }
    const bf16_t *col = vs + (size_t)r * p.scap;
    const bool some = 8 * g < b && 8 * g + 8 > a;  // the lane has a value to write
    if (all) {
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
        for (int w = 0; w < 4; ++w) vx[h][w] = u32x4{0u, 0u, 0u, 0u};
      if (some) {
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
    }
    __builtin_amdgcn_sched_barrier(0);  // every load in flight
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
          for (int e = 0; e < 4; ++e) range.add(kx[t][2 * q + w][e]);
        join_groups(range);
        const Affine f(range.lo, range.hi);
        sz[q] = f.pair;
#pragma unroll
        for (int w = 0; w < 2; ++w)
          words[2 * q + w] = code_word([&](int e) { return piece_elem(kx[t][2 * q + w], e); }, [&](int) { return f; }, f.odd);
      }
      if (j >= a && j < b) {
        *(u32x4 *)(out + (t * 64 + lane) * 16) = words;
        if (g == 0) *(u32x2 *)(out + kQP + j * 8) = u32x2{sz[0], sz[1]};
      }
    }
    // the values' 16 groups of eight positions: all lanes of a row take part in
    // each range, lane r then settles group r / 8 of position 8 g + r % 8
    Range range[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int w = 0; w < 4; ++w) range[h][e].add(vx[h][w][e]);
        join_row(range[h][e]);
      }
    // (bits, not selections: those of array elements become memory accesses)
    const uint32_t m8 = 0u - (r >> 3), m4 = 0u - (r >> 2 & 1), m2 = 0u - (r >> 1 & 1);
    auto either = [](uint32_t m, uint32_t one, uint32_t zero) { return (one & m) | (zero & ~m); };
    auto own_group = [&](auto part) {  // of the 8 pairs of groups, the lane's
      const uint32_t p0 = either(m8, part(1, 0), part(0, 0)), p1 = either(m8, part(1, 1), part(0, 1));
      const uint32_t p2 = either(m8, part(1, 2), part(0, 2)), p3 = either(m8, part(1, 3), part(0, 3));
      return either(m2, either(m4, p3, p1), either(m4, p2, p0)) >> (16 * (r & 1));
    };
    const Affine mine(own_group([&](int h, int e) { return range[h][e].lo; }),
                      own_group([&](int h, int e) { return range[h][e].hi; }));
    const bool odd = __ballot(mine.odd) != 0;
    {
      const int j = 8 * g + (r & 7);
      if (j >= a && j < b) *(uint32_t *)(out + kQP + (kQB + j) * 8 + 4 * (r >> 3)) = mine.pair;
    }
    auto share = [&](auto tag) {  // lane k's
      constexpr int CTRL = 0x150 + decltype(tag)::value;  // row_newbcast:k
      return Affine(dpp<CTRL>(mine.pair), __uint_as_float(dpp<CTRL>(__float_as_uint(mine.inv))));
    };
    auto store_half = [&](auto tag) {
      constexpr int h = decltype(tag)::value;
      const Affine f[8] = {share(Const<8 * h>()),     share(Const<8 * h + 1>()), share(Const<8 * h + 2>()),
                           share(Const<8 * h + 3>()), share(Const<8 * h + 4>()), share(Const<8 * h + 5>()),
                           share(Const<8 * h + 6>()), share(Const<8 * h + 7>())};
      u32x4 words;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        words[w] = code_word([&](int e) { return piece_elem(vx[h][w], e); }, [&](int e) -> const Affine & { return f[e]; }, odd);
      u32x4 *o = (u32x4 *)(out + kQV + (h * 64 + lane) * 16);
      if (8 * g >= a && 8 * g + 8 <= b) {
        *o = words;
      } else if (some) {
        uint32_t put = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) put |= 8 * g + e >= a && 8 * g + e < b ? 15u << kvq_shift(e) : 0u;
        const u32x4 old = *o;
        *o = (words & put) | (old & ~put);
      }
    };
    store_half(Const<0>());
    store_half(Const<1>());
  }
}

// a held value: c s is exact (4 and 8 bits), so one rounding
__device__ __forceinline__ float held(float s, float z, uint32_t c) { return (float)c * s + z; }

// ---- blocks -> bf16 rows.  Workgroup (head, run of blocks), a block a wave.
__global__ __launch_bounds__(64 * kWaves) void kvq_load_kernel(KvqLoad p) {
  __shared__ u32x2 par_s[kWaves][2 * kQB];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const size_t head = blockIdx.x / p.runs;
  const int run0 = blockIdx.x % p.runs;
  bf16_t *ks = p.k + head * p.dcap * 128, *vs = p.v + head * 128 * (size_t)p.dcap;
  for (int blk = p.pos0 / kQB + run0 * kWaves + wave; blk * kQB < p.pos0 + p.n; blk += p.runs * kWaves) {
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
        __builtin_nontemporal_store(o, (u32x4 *)(row + 32 * w));
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
// searched for the last one that is kept, eleven bits at a time by counting (a
// thread's scan of 256 counts in four passes took half of 26 us); then the
// positions are written in order.  One workgroup a head, 4096 positions 13.8 us:
// three passes of an L2 round trip and four barriers, and one to write.  (Few
// heads leave compute units idle: with the move 2 heads, 524288 positions 670 us.)
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
// That is one compute unit's stream: 2 heads, 524288 positions 2.7 ms in place,
// 0.67 into another cache; with 256 heads the two are alike.
template <int W, bool WAIT>
__global__ __launch_bounds__(64 * W) void kvq_gather_kernel(KvqEvict p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const size_t head = blockIdx.x / p.runs;
  const unsigned char *src = p.src + head * (size_t)p.src_nb * kQBytes;
  const int32_t *kept = p.kept + head * (size_t)p.budget;
  const int nblk = (p.n + kQB - 1) / kQB;
  for (int run = blockIdx.x % p.runs * W; run < nblk; run += p.runs * W) {
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

// Workgroups of a head, which follow one another in the grid: neighbours then
// work on neighbouring positions.  (With the heads first, all workgroups under
// way touch the same positions of their heads; where a dim's row of positions is
// a multiple of 4 KB they meet in the same memory channels.)
int runs_of(int heads, int pos0, int n, int waves) {
  constexpr int kMostWorkgroups = 1 << 22;  // a launch's threads are counted in 32 bits (heads <= 2^20)
  return std::min(kMostWorkgroups / heads, ((pos0 % kQB + n + kQB - 1) / kQB + waves - 1) / waves);
}

}  // namespace

hipError_t launch_kvq_store(KvqStore p, hipStream_t s) {
  // a path is short: a wave a workgroup, so that a head's blocks spread
  p.runs = runs_of(p.heads, p.pos0, p.n, p.path ? 1 : kWaves);
  if (p.path)
    hipLaunchKernelGGL((kvq_store_kernel<1, true>), dim3(p.heads * p.runs), dim3(64), 0, s, p);
  else
    hipLaunchKernelGGL((kvq_store_kernel<kWaves, false>), dim3(p.heads * p.runs), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kvq_load(KvqLoad p, hipStream_t s) {
  p.runs = runs_of(p.heads, p.pos0, p.n, kWaves);
  hipLaunchKernelGGL(kvq_load_kernel, dim3(p.heads * p.runs), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kvq_evict(KvqEvict p, hipStream_t s) {
  hipLaunchKernelGGL(kvq_select_kernel, dim3(p.heads), dim3(kSel), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.src == p.dst) {
    p.runs = 1;
    hipLaunchKernelGGL((kvq_gather_kernel<16, true>), dim3(p.heads), dim3(64 * 16), 0, s, p);
  } else {
    p.runs = runs_of(p.heads, 0, p.n, kWaves);
    hipLaunchKernelGGL((kvq_gather_kernel<kWaves, false>), dim3(p.heads * p.runs), dim3(64 * kWaves), 0, s, p);
  }
  return hipGetLastError();
}
