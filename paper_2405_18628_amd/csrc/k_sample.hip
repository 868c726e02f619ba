// Verification of drafted tokens against the target's probabilities from given
// random numbers (ppd_accept_sample).
//
// What happens at a node -- which of its children is accepted, or which bonus
// token it gives -- depends on its own logits row and the random numbers
// alone, so every node is settled at once, a workgroup each, and a second
// launch walks from the root.
//
// Residuals.  After rejections with sums Z_1 .. Z_j the residual is max(w - C q,
// 0), C = Z_1 + .. + Z_j, since max(max(w - a, 0) - b, 0) = max(w - a - b, 0):
// one row of weights and one number.  Weights and sums are float64: with V
// tokens V borders compete for one draw, and float32's rounding moves each by
// about 1e-7 of the whole.
#include "ppd_internal.h"
#include "ppd_sample.h"

namespace {

constexpr int kThreads = 1024;

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// sum over the workgroup, the same value in every thread
__device__ __forceinline__ double block_sum64(double v, double *wave_s) {
  v = wave_sum64(v);
  __syncthreads();  // wave_s is free
  if ((threadIdx.x & 63) == 0) wave_s[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.;
  for (int w = 0; w < kThreads / 64; ++w) s += wave_s[w];
  return s;
}

__device__ __forceinline__ bool candidate(int id, int vocab) { return id >= 0 && id < vocab; }

// One node's row: thread t owns the run [t per, (t + 1) per) of the vocabulary.
__global__ __launch_bounds__(kThreads) void sample_node_kernel(SampleLaunch p) {
  __shared__ double wave_s[kThreads / 64];
  __shared__ int par_s[PPD_T_MAX], id_s[PPD_T_MAX];
  __shared__ int nan_s, pick_s, last_s;
  const int tid = threadIdx.x, a = blockIdx.x, V = p.vocab;
  if (tid == 0) nan_s = 0, pick_s = -1, last_s = 0;
  if (tid < p.T) {
    const int up = p.parent[tid];
    par_s[tid] = tid == 0 ? -1 : up >= 0 && up < tid ? up : 0;
    id_s[tid] = p.ids[tid];
    if (a == 0 && (tid == 0 ? up != -1 : up < 0 || up >= tid)) atomicOr(p.status, PPD_DEV_BAD_PARENT);
  }
  __syncthreads();
  if (a > 0 && !candidate(id_s[a], V)) return;  // never reached
  const float *row = p.logits + (size_t)a * V;
  const float *draft = p.draft ? p.draft + (size_t)a * V : nullptr;
  const int per = (V + kThreads - 1) / kThreads;
  const int i0 = min(V, tid * per), i1 = min(V, i0 + per);
  float m = -INFINITY;
  bool nan = false;
  for (int i = i0; i < i1; ++i) {
    nan |= row[i] != row[i];
    m = fmaxf(m, row[i]);
  }
  if (nan) nan_s = 1;
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  __shared__ float max_s[kThreads / 64];
  if ((tid & 63) == 0) max_s[tid >> 6] = m;
  __syncthreads();
  for (int w = 0; w < kThreads / 64; ++w) m = fmaxf(m, max_s[w]);
  const double inv_t = 1.0 / (double)p.temperature;
  auto weight = [&](int i) {
    const float x = row[i];
    return x == m ? 1.0 : x < m ? exp(((double)x - (double)m) * inv_t) : 0.0;
  };
  auto prob = [&](int i) { const float q = draft[i]; return q > 0.f ? (double)q : 0.0; };

  int taken = -1;
  double C = 0.;  // what the rejections have taken, in draft probabilities
  int first = a + 1, lo = 0;  // without draft: the rejected children are those of [first, lo)
  auto rejected = [&](int i) {
    for (int c = first; c < lo; ++c)
      if (par_s[c] == a && id_s[c] == i) return true;
    return false;
  };
  auto residual = [&](int i) {
    const double w = weight(i);
    if (draft) return C > 0. ? fmax(w - C * prob(i), 0.) : w;
    return rejected(i) ? 0. : w;
  };
  auto total = [&]() {
    double s = 0.;
    for (int i = i0; i < i1; ++i) s += residual(i);
    return block_sum64(s, wave_s);
  };
  double Z = m == -INFINITY ? 0. : total();
  if (m != -INFINITY)
    for (int c = a + 1; c < p.T; ++c) {  // the same in every thread
      if (par_s[c] != a || !candidate(id_s[c], V)) continue;
      const int x = id_s[c];
      if ((double)p.u[c] * (draft ? prob(x) : 1.0) * Z < residual(x)) {
        taken = c;
        break;
      }
      if (draft) C += Z;
      lo = c + 1;
      Z = total();
      if (!(Z > 0.)) C = 0., first = lo, Z = total();  // nothing left: from the start
    }
  int bonus = 0;
  if (taken < 0 && m != -INFINITY) {
    // the run whose border the draw falls before, then the token in it
    double s = 0.;
    for (int i = i0; i < i1; ++i) s += residual(i);
    double x = s;
    const int lane = tid & 63, wave = tid >> 6;
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) wave_s[wave] = x;
    __syncthreads();
    double before = 0., all = 0.;
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < wave) before += wave_s[w];
      all += wave_s[w];
    }
    const double goal = (double)p.u[0] * all;
    const double from = before + (x - s);
    if (s > 0.) atomicMax(&last_s, i1 - 1);
    // runs are few: the first whose end passes the goal
    __shared__ int first_s;
    if (tid == 0) first_s = kThreads;
    __syncthreads();
    if (from + s > goal && s > 0.) atomicMin(&first_s, tid);
    __syncthreads();
    if (tid == first_s) {
      double run = from;
      int pick = -1, last = i0;
      for (int i = i0; i < i1 && pick < 0; ++i) {
        const double r = residual(i);
        run += r;
        if (r > 0.) last = i;
        if (run > goal) pick = i;
      }
      pick_s = pick < 0 ? last : pick;
    }
    __syncthreads();
    if (pick_s < 0 && i0 <= last_s && last_s < i1) {  // a draw of 1 or more: the last token that has weight
      for (int i = i0; i < i1; ++i)
        if (residual(i) > 0.) pick_s = i;
    }
    __syncthreads();
    bonus = max(0, pick_s);
  }
  if (tid == 0) p.node[a] = SampleNode{taken, bonus, nan_s || m == -INFINITY};
}

__global__ __launch_bounds__(PPD_T_MAX) void sample_walk_kernel(SampleLaunch p) {
  __shared__ SampleNode node_s[PPD_T_MAX];
  __shared__ int path_s[PPD_T_MAX];
  const int tid = threadIdx.x;
  if (tid < p.T) {
    const int id = p.ids[tid];
    if (tid == 0 || candidate(id, p.vocab)) node_s[tid] = p.node[tid];
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

}  // namespace

size_t sample_workspace_bytes(int T, int vocab) { return 256 + (size_t)T * 16; }

hipError_t launch_sample(const SampleLaunch &p, hipStream_t s) {
  hipLaunchKernelGGL(sample_node_kernel, dim3(p.T), dim3(kThreads), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(sample_walk_kernel, dim3(1), dim3(PPD_T_MAX), 0, s, p);
  return hipGetLastError();
}
