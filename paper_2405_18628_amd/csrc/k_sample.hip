// Verification of drafted tokens against the target's probabilities from given
// random numbers (ppd_accept_sample).
//
// What happens at a node -- which of its children is accepted, or which bonus
// token it gives -- depends on its own logits row and the random numbers
// alone, so all nodes are settled side by side and a walk from the root reads
// the answers off: two launches, whatever the tree.
//
// Weights and sums are float64: with V tokens V borders compete for one draw,
// and float32's rounding moves each by about 1e-7 of the whole.  exp is
// table-driven (Tang, 1989): e^x = 2^(k / 64) e^r, |r| <= ln 2 / 128, from 64
// table entries and five terms of e^r's series (4e-14 of a weight), eleven
// float64 operations.
//
// Without draft probabilities a rejected token leaves the residual whole, so a
// node needs one sum over its row, that of the tokens none of its children
// holds (`rest`); everything else is arithmetic on the children's own weights.
// Rows are cut into parts of 4096 tokens, a workgroup each, which puts the
// loads and exponentials of a few rows on many compute units; the walk, one
// workgroup, combines the parts, decides all nodes at once and reads one part
// of one row again for the bonus token.
//
// With draft probabilities the residual after rejections with sums Z_1 .. Z_j
// is max(w - C q, 0), C = Z_1 + .. + Z_j, since max(max(w - a, 0) - b, 0) =
// max(w - a - b, 0): one row of weights, one of probabilities and a number, but
// a sum over the row for each rejection, the next depending on it.  A workgroup
// settles a node alone: probabilities in LDS, weights in registers (128 a thread:
// two of eight chunks' weights lie in scratch and come back in each sum).
//
// Bounds: latency.  64 nodes, V = 32000, no drafts 4.9 + 9.8 us (parts and walk:
// each a chain of two or three memory round trips and a few barriers); 25 nodes
// with drafts, V = 32001, 29.4 + 5.1: 256 KB a compute unit and float64 sums and
// exponentials of a row (with the library's exp 36 + 5), while as many compute
// units work as there are nodes.  One node, both launches: V = 4000 15.8, 32000
// 23.6, 50257, whose rows do not fit the registers, 40.6.  Several workgroups a
// node (a wait among them for each rejection) have not been measured.

#include "ppd_sample.h"

namespace {

constexpr int kPart = 4096;        // tokens of a part
constexpr int kPartThreads = 512;
constexpr int kThreads = 1024;

__device__ __forceinline__ bool candidate(int id, int vocab) { return id >= 0 && id < vocab; }

// parent[t] with anything that is not an earlier node as 0
__device__ __forceinline__ int parent_of(const SampleLaunch &p, int t) {
  const int up = p.parent[t];
  return t == 0 ? -1 : up >= 0 && up < t ? up : 0;
}

// sum over the wave in every lane, by lane permutations in the vector unit
// (pairs, quads, halves of 16, 16, then the row and half swaps)
template <int CTRL>
__device__ __forceinline__ double dpp64(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double join64(uint32_t lo, uint32_t hi) {
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum64(double v) {
  v += dpp64<0xb1>(v);   // quad_perm [1,0,3,2]
  v += dpp64<0x4e>(v);   // quad_perm [2,3,0,1]
  v += dpp64<0x141>(v);  // row_half_mirror
  v += dpp64<0x140>(v);  // row_mirror
  uint64_t b = __builtin_bit_cast(uint64_t, v);
  auto l16 = __builtin_amdgcn_permlane16_swap((uint32_t)b, (uint32_t)b, false, false);
  auto h16 = __builtin_amdgcn_permlane16_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
  v = join64(l16[0], h16[0]) + join64(l16[1], h16[1]);
  b = __builtin_bit_cast(uint64_t, v);
  auto l32 = __builtin_amdgcn_permlane32_swap((uint32_t)b, (uint32_t)b, false, false);
  auto h32 = __builtin_amdgcn_permlane32_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
  return join64(l32[0], h32[0]) + join64(l32[1], h32[1]);
}

// sum over the workgroup, the same value in every thread
template <int N>
__device__ __forceinline__ double block_sum64(double v, double *wave_s) {
  v = wave_sum64(v);
  __syncthreads();  // wave_s is free
  if ((threadIdx.x & 63) == 0) wave_s[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.;
#pragma unroll
  for (int w = 0; w < N / 64; ++w) s += wave_s[w];
  return s;
}
template <int N>
__device__ __forceinline__ float block_max(float v, float *wave_s) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) wave_s[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < N / 64; ++w) v = fmaxf(v, wave_s[w]);
  return v;
}
// of two numbers at once
template <int N>
__device__ __forceinline__ void block_max(float &a, float &b, float2 *wave_s) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor(a, o, 64)), b = fmaxf(b, __shfl_xor(b, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) wave_s[threadIdx.x >> 6] = float2{a, b};
  __syncthreads();
#pragma unroll
  for (int w = 0; w < N / 64; ++w) a = fmaxf(a, wave_s[w].x), b = fmaxf(b, wave_s[w].y);
}
// sum over the threads before this one; the whole in *all
__device__ __forceinline__ double block_before64(double v, double *wave_s, double *all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) wave_s[wave] = x;
  __syncthreads();
  double before = 0., sum = 0.;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += wave_s[w];
    sum += wave_s[w];
  }
  *all = sum;
  return before + (x - v);
}

// What the running sum has to pass.  A draw of 1 or more takes the last token
// that has weight: nothing passes its goal (the whole and the running sum are
// rounded apart, so the whole may be passed before the last token).
__device__ __forceinline__ double goal_of(float u, double whole) { return u < 1.f ? (double)u * whole : INFINITY; }

// The first token of a thread's four whose running sum passes the goal goes to
// *pick (the least), the last that has weight to *last (the greatest); runs rise
// with the thread, so a wave's first and last lane stand for it (an LDS atomic
// of every thread on one word took 14 us a chunk).
__device__ __forceinline__ void note_pick(const double (&r)[4], double run, double goal, int i0, int *pick, int *last) {
  int first = -1, end = -1;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    run += r[e];
    if (r[e] > 0.) {
      if (first < 0 && run > goal) first = i0 + e;
      end = i0 + e;
    }
  }
  const uint64_t hit = __ballot(first >= 0), any = __ballot(end >= 0);
  const int lane = threadIdx.x & 63;
  if (hit && lane == __ffsll((unsigned long long)hit) - 1) atomicMin(pick, first);
  if (any && lane == 63 - __clzll((long long)any)) atomicMax(last, end);
}

// The weights of a row whose largest logit is m (not -inf): e^((l - m) / t).
// e^x = 2^(k / 64) e^r: k comes from adding 1.5 2^52, which leaves it in the low
// bits, and its multiple of 64 goes straight into the table entry's exponent.
// Weights under e^-700 and those of NaN are 0; of an infinite m only its like
// have weight.
struct Weights {
  double m, inv_t, scale, cut;  // scale: 64 / (t ln 2), cut: -700 t
  bool endless;                 // m is infinite
  const double *table;          // 2^(j / 64)
  __device__ __forceinline__ Weights(float m_, float t, const double *tab)
      : m(m_), inv_t(1. / (double)t), scale(92.332482616893656768 / (double)t), cut(-700. * (double)t),
        endless(m_ == INFINITY), table(tab) {}
  __device__ __forceinline__ double operator()(float l) const {
    // (float64: the difference of two floats has no rounding that could pass the cut)
    const double d = endless ? (l == INFINITY ? 0. : -INFINITY) : (double)l - m;
    const double y = fma(d, scale, 6755399441055744.);
    const uint32_t k = (uint32_t)__builtin_bit_cast(uint64_t, y);
    const double r = fma(y - 6755399441055744., -1.0830424696249145e-02, d * inv_t);  // |r| <= ln 2 / 128
    const double q = fma(r, fma(r, fma(r, 1. / 24., 1. / 6.), 0.5), 1.);
    const double t = table[k & 63];
    const uint64_t w = __builtin_bit_cast(uint64_t, fma(t * r, q, t)) + ((uint64_t)((k & ~63u) << 14) << 32);
    return d >= cut ? __builtin_bit_cast(double, w) : 0.;
  }
};
__device__ __forceinline__ void fill_table(double *table) {
  if (threadIdx.x < 64) table[threadIdx.x] = exp2((double)threadIdx.x * (1. / 64.));
}

// ---------------------------------------------------------------------------
// without draft probabilities

// Workgroup (node, part): the part's largest logit and, the children's tokens
// left out, the largest one and the sum of weights against it.
__global__ __launch_bounds__(kPartThreads) void sample_part_kernel(SampleLaunch p) {
  constexpr int E = kPart / kPartThreads;
  __shared__ double wave_s[kPartThreads / 64];
  __shared__ float2 max_s[kPartThreads / 64];
  __shared__ double table[64];
  __shared__ int tok_s[PPD_T_MAX];
  __shared__ int n_s, nan_s;
  const int tid = threadIdx.x, a = blockIdx.y, V = p.vocab;
  if (a > 0 && !candidate(p.ids[a], V)) return;  // never reached
  const float *row = p.logits + (size_t)a * V;
  const int i0 = blockIdx.x * kPart;
  float x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = row[min(i0 + tid + kPartThreads * e, V - 1)];
  __builtin_amdgcn_sched_barrier(0);  // all loads in flight (a conditional load would be waited for by itself)
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = i0 + tid + kPartThreads * e < V ? x[e] : -INFINITY;
  if (tid == 0) n_s = nan_s = 0;
  fill_table(table);
  __syncthreads();
  if (tid < p.T && tid > a && parent_of(p, tid) == a) {
    const int id = p.ids[tid];
    if (id >= i0 && id < min(V, i0 + kPart)) tok_s[atomicAdd(&n_s, 1)] = id;
  }
  float m = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    nan |= x[e] != x[e];
    m = fmaxf(m, x[e]);
  }
  if (nan) nan_s = 1;
  __syncthreads();
  const int n = n_s;
  for (int c = 0; c < n; ++c) {
    const int at = tok_s[c] - i0;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (at == tid + kPartThreads * e) x[e] = NAN;  // no weight
  }
  // the sum is taken against the largest logit of what it sums, so that a part
  // has weight in the row exactly where its largest token has
  float top = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) top = fmaxf(top, x[e]);
  block_max<kPartThreads>(m, top, max_s);
  double s = 0.;
  if (top > -INFINITY) {
    const Weights weight(top, p.temperature, table);
#pragma unroll
    for (int e = 0; e < E; ++e) s += weight(x[e]);
  }
  s = block_sum64<kPartThreads>(s, wave_s);
  if (tid == 0) p.part[(size_t)a * gridDim.x + blockIdx.x] = SamplePart{s, top, m, (uint32_t)nan_s, 0u};
}

// One workgroup: all nodes decided, the walk, the bonus token.
__global__ __launch_bounds__(kThreads) void sample_walk_kernel(SampleLaunch p, int parts) {
  __shared__ double wave_s[kThreads / 64];
  __shared__ double table[64];
  __shared__ int up_s[PPD_T_MAX], id_s[PPD_T_MAX], go_s[PPD_T_MAX], path_s[PPD_T_MAX];
  __shared__ float m_s[PPD_T_MAX], u_s[PPD_T_MAX];
  __shared__ double rest_s[PPD_T_MAX], w_s[PPD_T_MAX];  // a node's rest; a child's weight in its parent's row
  __shared__ int nan_s[PPD_T_MAX];
  __shared__ uint32_t out_s[kPart / 32];  // tokens of the chosen part that children hold
  __shared__ double base_s;
  __shared__ int n_s, pick_s, last_s, first_s, final_s, n_part_s;
  const int tid = threadIdx.x, T = p.T, V = p.vocab;
  fill_table(table);
  if (tid < T) {
    const int up = p.parent[tid];
    const int at = parent_of(p, tid), id = p.ids[tid];
    if (tid == 0 ? up != -1 : at != up) atomicOr(p.status, PPD_DEV_BAD_PARENT);
    up_s[tid] = at;
    id_s[tid] = id;
    go_s[tid] = INT_MAX;
    path_s[tid] = -1;
  }
  if (tid == 0) pick_s = first_s = INT_MAX, last_s = final_s = -1;
  if (tid < kPart / 32) out_s[tid] = 0u;
  __syncthreads();
  // a child's logit in its parent's row (requested before the parts are combined)
  const bool child = tid > 0 && tid < T && candidate(id_s[tid], V);
  float lc = 0.f;
  if (child) lc = p.logits[(size_t)up_s[tid] * V + id_s[tid]];
  if (tid < T) u_s[tid] = p.u[tid];
  // the parts of a node: eight threads
  {
    const int a = tid >> 3;
    const bool on = a < T && (a == 0 || candidate(id_s[a], V));
    const SamplePart *part = p.part + (size_t)a * parts;
    float m = -INFINITY;
    int nan = 0;
    for (int s = tid & 7; on && s < parts; s += 8) {
      m = fmaxf(m, part[s].m);
      nan |= part[s].nan;
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      m = fmaxf(m, __shfl_xor(m, o, 64));
      nan |= __shfl_xor(nan, o, 64);
    }
    const Weights weight(m, p.temperature, table);
    double rest = 0.;
    for (int s = tid & 7; on && s < parts; s += 8) {
      const double r = part[s].rest;
      if (r > 0.) rest += r * weight(part[s].top);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) rest += __shfl_xor(rest, o, 64);
    if (on && (tid & 7) == 0) {
      m_s[a] = m;
      nan_s[a] = nan;
      rest_s[a] = rest;
    }
  }
  __syncthreads();
  if (tid < T) w_s[tid] = child && m_s[up_s[tid]] > -INFINITY ? Weights(m_s[up_s[tid]], p.temperature, table)(lc) : 0.;
  __syncthreads();
  // a child's weight in the residual when its turn comes: 0 where an earlier
  // sibling holds its token (that one was rejected).  Eight threads a child look
  // through the others.
  const int t = tid >> 3;
  const bool mine = t > 0 && t < T && candidate(id_s[min(t, T - 1)], V);
  const int up = mine ? up_s[t] : -1, id = mine ? id_s[t] : -1;
  bool again = false;
#pragma unroll 4
  for (int j = tid & 7; j < T; j += 8) again |= mine && j < t && up_s[j] == up && id_s[j] == id;
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) again |= __shfl_xor((int)again, o, 64) != 0;
  __syncthreads();
  if (again && (tid & 7) == 0) w_s[t] = 0.;
  __syncthreads();
  // what is left then: the rest, itself and its later siblings
  double Z = 0.;
#pragma unroll 4
  for (int j = tid & 7; j < T; j += 8) Z += mine && j >= t && up_s[j] == up ? w_s[j] : 0.;
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) Z += __shfl_xor(Z, o, 64);
  if (mine && (tid & 7) == 0 && (double)u_s[t] * (Z + rest_s[up]) < w_s[t]) atomicMin(&go_s[up], t);
  __syncthreads();
  if (tid == 0) {
    int u = 0, n = 0;
    bool bad = false;
    for (;;) {  // children follow their parents: it ends
      path_s[n++] = u;
      bad |= nan_s[u] || m_s[u] == -INFINITY;
      if (go_s[u] == INT_MAX) break;
      u = go_s[u];
    }
    n_s = n;
    if (bad) atomicOr(p.status, PPD_DEV_NAN_LOGIT);
  }
  __syncthreads();
  const int a = path_s[n_s - 1];
  const float m = m_s[a];
  const double rest = rest_s[a];
  if (tid < T) p.path[tid] = path_s[tid];
  if (rest > 0.) {
    // the part that the draw falls into (a draw of 1 or more: the last that has
    // weight), then the token: a part's tokens in runs of four a thread
    const SamplePart *part = p.part + (size_t)a * parts;
    const Weights weight(m, p.temperature, table);
    const double goal = goal_of(u_s[0], rest);
    const int per = (parts + kThreads - 1) / kThreads;
    auto part_sum = [&](int s) {
      const SamplePart x = part[min(s, parts - 1)];
      return s < parts && x.rest > 0. ? x.rest * weight(x.top) : 0.;
    };
    double sum = 0., all;
    for (int s = 0; s < per; ++s) sum += part_sum(tid * per + s);
    const double before = block_before64(sum, wave_s, &all);
    if (sum > 0.) {  // (as many as there are parts)
      if (before + sum > goal) atomicMin(&first_s, tid);
      atomicMax(&final_s, tid);
    }
    __syncthreads();
    if (tid == (first_s != INT_MAX ? first_s : final_s)) {
      double b = before;
      int at = tid * per;
      for (int s = 0; s < per; ++s) {
        const double x = part_sum(tid * per + s);
        if (x > 0.) {
          at = tid * per + s;
          base_s = b;
          if (b + x > goal) break;
        }
        b += x;
      }
      n_part_s = at;
    }
    __syncthreads();
    const int at = n_part_s;
    if (child && up_s[tid] == a && id_s[tid] / kPart == at) atomicOr(&out_s[id_s[tid] % kPart >> 5], 1u << (id_s[tid] & 31));
    const double base = base_s;
    const float *row = p.logits + (size_t)a * V;
    const int i0 = at * kPart + 4 * tid;
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = row[min(i0 + e, V - 1)];
    __syncthreads();
    const uint32_t out = out_s[tid >> 3] >> (4 * (tid & 7));
    double r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = i0 + e < V && !(out >> e & 1u) ? weight(x[e]) : 0.;
    sum = (r[0] + r[1]) + (r[2] + r[3]);
    note_pick(r, base + block_before64(sum, wave_s, &all), goal, i0, &pick_s, &last_s);
  } else if (m > -INFINITY) {
    // all weight lies on the children's tokens, of which none was accepted: the
    // bonus token is drawn from them
    double whole = 0., run = 0.;
    for (int j = a + 1; j < T; ++j)
      if (up_s[j] == a) whole += w_s[j];
    const double goal = goal_of(u_s[0], whole);
    if (child && up_s[tid] == a && w_s[tid] > 0.) {
      for (int j = a + 1; j < T; ++j)
        if (up_s[j] == a && id_s[j] <= id_s[tid]) run += w_s[j];
      if (run > goal) atomicMin(&pick_s, id_s[tid]);
      atomicMax(&last_s, id_s[tid]);
    }
  }
  __syncthreads();
  if (tid == 0) {
    *p.n_path = n_s;
    *p.next_tok = pick_s != INT_MAX ? pick_s : max(0, last_s);
  }
}

// ---------------------------------------------------------------------------
// with draft probabilities

// One node's row, its tokens dealt to the threads in runs of four, kThreads
// runs a chunk.  RES: up to kResChunks chunks, whose weights stay in registers
// and whose probabilities in LDS; else a pass over the row forms them again.
constexpr int kRun = 4, kChunk = kThreads * kRun;
constexpr int kResChunks = 8;
constexpr int kChunkSums = 32;

template <bool RES>
__global__ __launch_bounds__(kThreads) void sample_node_kernel(SampleLaunch p) {
  __shared__ double wave_s[kThreads / 64];
  __shared__ float max_s[kThreads / 64];
  __shared__ double table[64];
  __shared__ int par_s[PPD_T_MAX], id_s[PPD_T_MAX];
  __shared__ double cw_s[PPD_T_MAX], cq_s[PPD_T_MAX];  // a child's weight and probability in the node's row
  __shared__ double sums_s[kChunkSums][kThreads / 64], before_s[kChunkSums];
  __shared__ int nan_s, pick_s, last_s, first_s, final_s;
  __shared__ __attribute__((aligned(16))) float4 q_s[RES ? kResChunks : 1][kThreads];
  const int tid = threadIdx.x, a = blockIdx.x, V = p.vocab;
  if (a > 0 && !candidate(p.ids[a], V)) return;  // never reached
  const float *row = p.logits + (size_t)a * V;
  const float *draft = p.draft + (size_t)a * V;
  const int n_chunks = (V + kChunk - 1) / kChunk;
  // four tokens from i on (past the row: `past`), one 16-byte load wherever the
  // row starts (4-byte alignment is enough for it).  The last run is loaded as
  // the row's last four tokens and moved up; a conditional load would be waited
  // for by itself.
  typedef float Run __attribute__((ext_vector_type(4), aligned(4)));
  auto get4 = [&](const float *from, int i) {
    if (V < 4) return float4{from[min(i, V - 1)], from[min(i + 1, V - 1)], from[min(i + 2, V - 1)], 0.f};
    const Run v = *(const Run *)(from + min(i, V - 4));
    return float4{v[0], v[1], v[2], v[3]};
  };
  auto up4 = [&](float4 v, int i) {
    const int d = V < 4 ? 0 : i - min(i, V - 4);
    return float4{d == 0 ? v.x : d == 1 ? v.y : d == 2 ? v.z : v.w, d == 0 ? v.y : d == 1 ? v.z : v.w,
                  d == 0 ? v.z : v.w, v.w};
  };
  auto cut4 = [&](float4 v, int i, float past) {
    v = up4(v, i);
    return float4{i < V ? v.x : past, i + 1 < V ? v.y : past, i + 2 < V ? v.z : past, i + 3 < V ? v.w : past};
  };
  auto load4 = [&](const float *from, int i, float past) { return cut4(get4(from, i), i, past); };
  auto prob = [](float q) { return q > 0.f ? q : 0.f; };
  float4 x[RES ? kResChunks : 1];
  if constexpr (RES) {
#pragma unroll
    for (int k = 0; k < kResChunks; ++k) x[k] = get4(row, k * kChunk + kRun * tid);
    float4 q[kResChunks];
#pragma unroll
    for (int k = 0; k < kResChunks; ++k) q[k] = get4(draft, k * kChunk + kRun * tid);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kResChunks; ++k) {
      const int i = k * kChunk + kRun * tid;
      x[k] = cut4(x[k], i, -INFINITY);
      q[k] = cut4(q[k], i, 0.f);
      q_s[k][tid] = float4{prob(q[k].x), prob(q[k].y), prob(q[k].z), prob(q[k].w)};
    }
  }
  if (tid == 0) nan_s = 0, pick_s = first_s = INT_MAX, last_s = final_s = -1;
  fill_table(table);
  if (tid < p.T) {
    const int up = p.parent[tid];
    par_s[tid] = parent_of(p, tid);
    id_s[tid] = p.ids[tid];
    if (a == 0 && (tid == 0 ? up != -1 : par_s[tid] != up)) atomicOr(p.status, PPD_DEV_BAD_PARENT);
  }
  __syncthreads();
  float m = -INFINITY;
  bool nan = false;
  auto look = [&](float4 v) {
    m = fmaxf(fmaxf(m, fmaxf(v.x, v.y)), fmaxf(v.z, v.w));
    nan |= v.x != v.x || v.y != v.y || v.z != v.z || v.w != v.w;
  };
  if constexpr (RES) {
#pragma unroll
    for (int k = 0; k < kResChunks; ++k) look(x[k]);
  } else {
#pragma unroll 4
    for (int k = 0; k < n_chunks; ++k) look(load4(row, k * kChunk + kRun * tid, -INFINITY));
  }
  if (nan) nan_s = 1;
  m = block_max<kThreads>(m, max_s);
  const Weights weight(m, p.temperature, table);
  if (tid > a && tid < p.T && par_s[tid] == a && candidate(id_s[tid], V)) {
    cw_s[tid] = weight(row[id_s[tid]]);
    cq_s[tid] = prob(draft[id_s[tid]]);
  }
  double w[RES ? kResChunks : 1][kRun];
  if constexpr (RES) {
#pragma unroll
    for (int k = 0; k < kResChunks; ++k) {
      const float v[kRun] = {x[k].x, x[k].y, x[k].z, x[k].w};
      if (k < n_chunks)
#pragma unroll
        for (int e = 0; e < kRun; ++e) w[k][e] = weight(v[e]);
    }
  }
  // the residuals of this thread's run of chunk k
  auto residual4 = [&](int k, double C, double (&r)[kRun]) {
    float4 q;
    if constexpr (RES) {
      q = q_s[k][tid];
#pragma unroll
      for (int e = 0; e < kRun; ++e) r[e] = w[k][e];
    } else {
      const float4 v = load4(row, k * kChunk + kRun * tid, -INFINITY);
      q = load4(draft, k * kChunk + kRun * tid, 0.f);
      q = float4{prob(q.x), prob(q.y), prob(q.z), prob(q.w)};
      const float l[kRun] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < kRun; ++e) r[e] = weight(l[e]);
    }
    const float qe[kRun] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < kRun; ++e)  // (an infinite probability times C = 0 takes nothing)
      r[e] = C > 0. ? fmax(fma(-C, (double)qe[e], r[e]), 0.) : r[e];
  };
  auto chunk_sum = [&](int k, double C) {
    double r[kRun];
    residual4(k, C, r);
    return (r[0] + r[1]) + (r[2] + r[3]);
  };
  auto total = [&](double C) {
    double s = 0.;
    if constexpr (RES) {
#pragma unroll
      for (int k = 0; k < kResChunks; ++k)
        if (k < n_chunks) s += chunk_sum(k, C);
    } else {
#pragma unroll 2
      for (int k = 0; k < n_chunks; ++k) s += chunk_sum(k, C);
    }
    return block_sum64<kThreads>(s, wave_s);
  };
  int taken = -1, bonus = 0;
  if (m > -INFINITY) {
    double C = 0., Z = total(0.);
    for (int c = a + 1; c < p.T; ++c) {  // the same in every thread
      if (par_s[c] != a || !candidate(id_s[c], V)) continue;
      const double q = cq_s[c], r = C > 0. ? fmax(fma(-C, q, cw_s[c]), 0.) : cw_s[c];
      if ((double)p.u[c] * q * Z < r) {
        taken = c;
        break;
      }
      C += Z;
      Z = total(C);
    }
    if (taken < 0) {
      if (!(Z > 0.)) C = 0., Z = total(0.);  // nothing is left: the bonus token is drawn from the weights
      // the chunk that the draw falls into, then the token (a draw of 1 or
      // more: the last token that has weight).  The chunks' sums come from one
      // pass, kChunkSums of them at a time.
      const double goal = goal_of(p.u[0], Z);
      const int lane = tid & 63, wave = tid >> 6;
      double base = 0.;
      for (int k0 = 0; k0 < n_chunks; k0 += kChunkSums) {
        const int nk = min(kChunkSums, n_chunks - k0);
        auto note_sum = [&](int k, double v) {
          v = wave_sum64(v);
          if (lane == 0) sums_s[k][wave] = v;
        };
        if constexpr (RES) {
#pragma unroll
          for (int k = 0; k < kResChunks; ++k)
            if (k < n_chunks) note_sum(k, chunk_sum(k, C));
        } else {
#pragma unroll 2
          for (int k = 0; k < nk; ++k) note_sum(k, chunk_sum(k0 + k, C));
        }
        __syncthreads();
        double sum = 0., all;
        if (tid < nk)
#pragma unroll
          for (int w = 0; w < kThreads / 64; ++w) sum += sums_s[tid][w];
        const double before = base + block_before64(sum, wave_s, &all);
        if (sum > 0.) {  // (one thread a chunk)
          if (before + sum > goal) atomicMin(&first_s, k0 + tid);
          atomicMax(&final_s, k0 + tid);
        }
        if (tid < nk) before_s[tid] = before;
        __syncthreads();
        if (first_s != INT_MAX || k0 + kChunkSums >= n_chunks) {
          const int k = first_s != INT_MAX ? first_s : max(0, final_s);
          double r[kRun];
          if constexpr (RES) {
#pragma unroll
            for (int j = 0; j < kResChunks; ++j)
              if (j == k) residual4(j, C, r);
          } else {
            residual4(k, C, r);
          }
          // (no first_s: a draw of 1 or more, whose goal nothing passes; then k may lie before k0)
          const double at = (k >= k0 ? before_s[k - k0] : base) + block_before64((r[0] + r[1]) + (r[2] + r[3]), wave_s, &all);
          note_pick(r, at, goal, k * kChunk + kRun * tid, &pick_s, &last_s);
          break;
        }
        base += all;
        __syncthreads();  // the sums' LDS is written next
      }
      __syncthreads();
      bonus = pick_s != INT_MAX ? pick_s : max(0, last_s);
    }
  }
  if (tid == 0) p.node[a] = SampleNode{taken, bonus, nan_s || m == -INFINITY, 0};
}

__global__ __launch_bounds__(PPD_T_MAX) void sample_path_kernel(SampleLaunch p) {
  __shared__ SampleNode node_s[PPD_T_MAX];
  __shared__ int path_s[PPD_T_MAX];
  const int tid = threadIdx.x;
  if (tid < p.T) {
    if (tid == 0 || candidate(p.ids[tid], p.vocab)) node_s[tid] = p.node[tid];
    path_s[tid] = -1;
  }
  __syncthreads();
  if (tid == 0) {
    int u = 0, n = 0;
    bool bad = false;
    for (;;) {  // children follow their parents: it ends
      path_s[n++] = u;
      bad |= node_s[u].bad;
      if (node_s[u].taken < 0) break;
      u = node_s[u].taken;
    }
    *p.n_path = n;
    *p.next_tok = node_s[u].bonus;
    if (bad) atomicOr(p.status, PPD_DEV_NAN_LOGIT);
  }
  __syncthreads();
  if (tid < p.T) p.path[tid] = path_s[tid];
}

int parts_of(int vocab) { return (vocab + kPart - 1) / kPart; }

}  // namespace

size_t sample_workspace_bytes(int T, int vocab) {
  return 256 + sizeof(SamplePart) * (size_t)T * parts_of(vocab);  // at least a SampleNode a node
}

hipError_t launch_sample(const SampleLaunch &p, hipStream_t s) {
  static_assert(sizeof(SampleNode) <= sizeof(SamplePart), "they share the workspace");
  if (!p.draft) {
    const int parts = parts_of(p.vocab);
    hipLaunchKernelGGL(sample_part_kernel, dim3(parts, p.T), dim3(kPartThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(sample_walk_kernel, dim3(1), dim3(kThreads), 0, s, p, parts);
  } else {
    if (p.vocab <= kResChunks * kChunk)
      hipLaunchKernelGGL(sample_node_kernel<true>, dim3(p.T), dim3(kThreads), 0, s, p);
    else
      hipLaunchKernelGGL(sample_node_kernel<false>, dim3(p.T), dim3(kThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(sample_path_kernel, dim3(1), dim3(PPD_T_MAX), 0, s, p);
  }
  return hipGetLastError();
}
