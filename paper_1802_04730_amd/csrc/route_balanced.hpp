// A router that keeps its experts' load even: scores of their own, a bias that only the choice sees, groups of experts.
//   S(t,e) = 1 / (1 + exp(-L(t,e))), or softmax(L(t,:));   C(t,e) = S(t,e) + Bias(e), -inf where L is
//   groups of E/groups neighbours: a group's score is the sum of its two best C (of one, where there is no other); the `keep` best groups stay
//   the k largest C of those, largest first, equal ones by the lower number;  w = scale S, or (norm) scale S / sum of the k S
//   dS(t,e_i) = scale g_i, or (norm) scale (g_i - sum_j g_j S_j / s) / s, s = sum_j S_j;   dL = dS S (1 - S), or S (dS - sum_j dS_j S_j)
// Off, Row and Place as in route.hpp, whose counting and placing follow the selection.
//
// Scores lie next to each other -- 256 of them in (0, 1) are 1/256 apart, and in some tens of thousands of tokens several pairs at the border of the choice agree
// in 24 bits --, so they are computed, biased and compared in 64 bits: which experts a token gets does not hang on a rounding to 32.
//
// A group of 16 lanes (64 for more than 256 experts or 16 chosen) takes a token, each lane a few neighbouring logits.  With groups of experts the biased scores
// go through LDS once: lane g finds the two best of group g, and ranks it by counting the better ones.  Then k rounds find the largest of what is left,
// by the upper halves of keys that order as the scores do and, only where several lanes agree in those, by the lower ones.  The scores of the k
// chosen are computed again by the lanes that write them, all at once.  What bounds it is the rounds' latency and the exponentials of 64 bits.
#pragma once
#include "expert_types.hpp"
#include "lanes.hpp"
#include "route.hpp"

namespace tc355 {

constexpr int ROUTE_MOST_GROUPS = 64;

struct RouteBalancedArgs {
  RouteArgs r;
  const float* Bias;  // [E] or nullptr
  float scale;
  int groups, keep, sigmoid;
};

__device__ __forceinline__ unsigned long long score_order(double x) {  // orders as the scores do; 0: -inf
  if (x != x) return ~0ull;
  const unsigned long long b = __builtin_bit_cast(unsigned long long, x + 0.0);
  const unsigned long long o = b >> 63 ? ~b : b | 1ull << 63;
  return o - 0x000fffffffffffffull;  // (-inf is the lowest: 0x000fffffffffffff)
}
__device__ __forceinline__ double sigmoid64(double x) { return 1.0 / (1.0 + exp(-x)); }

template <typename T, int G, int V>
__global__ __launch_bounds__(WG_THREADS) void route_balanced_kernel(RouteBalancedArgs a) {
  const RouteArgs& p = a.r;
  extern __shared__ __align__(8) int mem[];  // as route_kernel's; behind it, with groups, [WG_THREADS / G][E + groups] scores
  __shared__ int part[WAVES_PER_WG];
  const int bins = 1 << p.bits;
  for (int b = threadIdx.x; b < bins; b += WG_THREADS) mem[b] = 0;
  __syncthreads();
  const int lane = threadIdx.x & (G - 1), group = threadIdx.x / G;
  const T* L = static_cast<const T*>(p.L);
  double* const scores = reinterpret_cast<double*>(mem + (p.count ? bins : bins * (1 + WAVES_PER_WG))) + group * (p.E + a.groups);
  const bool grouped = a.keep < a.groups;
  const int size = p.E / a.groups;
  float bias[V];
#pragma unroll
  for (int v = 0; v < V; v++) bias[v] = a.Bias && lane * V + v < p.E ? a.Bias[lane * V + v] : 0.0f;
  for (int r = group; r < p.tokens; r += WG_THREADS / G) {
    const int64_t t = (int64_t)blockIdx.x * p.tokens + r;
    if (t >= p.T) break;  // (the whole group, and all groups behind it)
    float x[V];
    load_logits<T, V>(L + t * p.E, lane * V, p.E, x);
    double s[V];
    double most = 0, sum = 1;
    if (a.sigmoid) {
#pragma unroll
      for (int v = 0; v < V; v++) s[v] = sigmoid64(x[v]);
    } else {
      float m = -__builtin_inff();
#pragma unroll
      for (int v = 0; v < V; v++) m = fmaxf(m, x[v]);
      m = group_all<G>(m, most_of);
      if (m == -__builtin_inff()) m = 0.0f;  // (nothing to choose: every exp is 0, or NaN)
      most = m;
      sum = 0;
#pragma unroll
      for (int v = 0; v < V; v++) {
        s[v] = exp((double)x[v] - most);
        sum += s[v];
      }
      sum = group_all<G>(sum, [](double p, double q) { return p + q; });
#pragma unroll
      for (int v = 0; v < V; v++) s[v] = s[v] / sum;  // (0 / 0: nothing to choose, and never chosen)
    }
    unsigned long long key[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
      s[v] = x[v] == -__builtin_inff() ? -__builtin_inf() : s[v] + (double)bias[v];
      key[v] = score_order(s[v]);
    }
    if (grouped) {
      double* const best = scores + p.E;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int v = 0; v < V; v++)
        if (lane * V + v < p.E) scores[lane * V + v] = s[v];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      for (int g = lane; g < a.groups; g += G) {
        unsigned long long one = 0, two = 0;
        double first = -__builtin_inf(), second = -__builtin_inf();
        for (int j = 0; j < size; j++) {
          const double c = scores[g * size + j];
          const unsigned long long o = score_order(c);
          if (o > one) {
            two = one;
            second = first;
            one = o;
            first = c;
          } else if (o > two) {
            two = o;
            second = c;
          }
        }
        best[g] = __builtin_bit_cast(double, score_order(two ? first + second : first));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      for (int g = lane; g < a.groups; g += G) {
        const unsigned long long mine = __builtin_bit_cast(unsigned long long, best[g]);
        int better = 0;
        for (int h = 0; h < a.groups; h++) {
          const unsigned long long other = __builtin_bit_cast(unsigned long long, best[h]);
          better += other > mine || (other == mine && h < g) ? 1 : 0;
        }
        scores[g] = better < a.keep ? 1.0 : 0.0;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int v = 0; v < V; v++) {
        const int e = lane * V + v;
        if (e < p.E && scores[e / size] == 0.0) key[v] = 0;
      }
    }
    int id = -1;
    float logit = 0;
    for (int i = 0; i < p.k; i++) {
      unsigned long long mine = 0;
      int at = 0;
#pragma unroll
      for (int v = V - 1; v >= 0; v--)
        if (key[v] >= mine) {
          mine = key[v];
          at = v;
        }
      const unsigned upper = (unsigned)(mine >> 32), best = group_all<G>(upper, larger);
      const unsigned long long agree = __ballot(upper == best);
      const unsigned within = (threadIdx.x & 63) & ~(G - 1);
      const unsigned long long members = agree >> within & (~0ull >> (64 - G));
      bool winner = upper == best;
      if (members & (members - 1)) {  // (several: by the lower halves, then by the lane, whose experts come first)
        const unsigned lower = winner ? (unsigned)mine : 0, low = group_all<G>(lower, larger);
        winner = winner && lower == low;
      }
      const unsigned long long last = __ballot(winner);
      const int src = __ffsll((long long)(last >> within & (~0ull >> (64 - G)))) - 1;
      float chosen = 0;
#pragma unroll
      for (int v = 0; v < V; v++)
        if (at == v) chosen = x[v];
      const bool none = __shfl(mine == 0 ? 1 : 0, src, G) != 0;
      const int e = __shfl(lane * V + at, src, G);
      chosen = __shfl(chosen, src, G);
      if (lane == src) {
#pragma unroll
        for (int v = 0; v < V; v++)
          if (at == v) key[v] = 0;
      }
      if (lane == i) {  // (k <= G, by the host's choice of G)
        id = none ? -1 : e;
        logit = chosen;
      }
    }
    double w = 0;
    if (id >= 0) w = a.sigmoid ? sigmoid64(logit) : exp((double)logit - most) / sum;
    double total = 1;
    if (p.norm) {
      total = group_all<G>(w, [](double p, double q) { return p + q; });
      if (total < 1e-300) total = 1e-300;  // (scores of nothing have weights of nothing)
    }
    if (lane < p.k) {
      p.Wt[t * p.k + lane] = id < 0 ? 0.0f : (float)((double)a.scale * w / total);
      p.Id[t * p.k + lane] = id;
      atomicAdd(&mem[id < 0 ? p.E : id], 1);
    }
  }
  route_counted(p, mem, part);
}

struct RouteBalancedGradArgs {
  RouteGradArgs r;
  float scale;
  int sigmoid;
};

// The chosen experts' part in 64 bits, by the lanes that hold the slots: their scores may be far below the others'.
template <typename T, int G, int V>
__global__ __launch_bounds__(WG_THREADS) void route_balanced_grad_kernel(RouteBalancedGradArgs a, int64_t first) {
  const RouteGradArgs& p = a.r;
  const int lane = threadIdx.x & (G - 1);
  const int64_t t = (first + blockIdx.x) * (WG_THREADS / G) + threadIdx.x / G;
  if (t >= p.T) return;
  const auto add = [](double x, double y) { return x + y; };
  const T* L = static_cast<const T*>(p.L) + t * p.E;
  float x[V], grad[V];
  bool free[V];
  if (!a.sigmoid) {
    load_logits<T, V>(L, lane * V, p.E, x);
  } else {  // (of the chosen alone, below)
#pragma unroll
    for (int v = 0; v < V; v++) x[v] = 0.0f;
  }
  double most = 0, sum = 1;
  if (!a.sigmoid) {
    float m = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < V; v++) m = fmaxf(m, x[v]);
    m = group_all<G>(m, most_of);
    if (m == -__builtin_inff()) m = 0.0f;
    most = m;
    float part = 0;
#pragma unroll
    for (int v = 0; v < V; v++) part += expf(x[v] - m);
    sum = group_all<G>((double)part, add);
    if (sum == 0) sum = 1;  // (a row of nothing)
  }
  // a slot a lane, G slots at a time: scores and sums over all slots first
  const auto slot = [&](int i, int* id, double* g, double* s) {
    *id = i < p.k ? p.Id[t * p.k + i] : -1;
    if (*id >= p.E) *id = -1;
    *g = *id >= 0 ? (double)p.dWt[t * p.k + i] : 0.0;
    const double l = *id >= 0 ? (double)(float)L[*id] : 0.0;
    *s = *id < 0 || l == -__builtin_inf() ? 0.0 : a.sigmoid ? sigmoid64(l) : exp(l - most) / sum;
  };
  double total = 0, mean = 0;
  for (int i0 = 0; i0 < p.k; i0 += G) {
    int id;
    double g, s;
    slot(i0 + lane, &id, &g, &s);
    total += s;
    mean += s == 0 ? 0.0 : g * s;
  }
  total = group_all<G>(total, add);
  mean = group_all<G>(mean, add);
  if (total < 1e-300) total = 1e-300;
  const double each = p.norm ? a.scale / total : a.scale, less = p.norm ? mean / total : 0.0;  // dS_i = each (g_i - less)
  const double inner = a.sigmoid || p.norm ? 0.0 : each * mean;  // sum_j dS_j S_j, of which norm leaves nothing
#pragma unroll
  for (int v = 0; v < V; v++) {
    free[v] = x[v] != -__builtin_inff();
    grad[v] = a.sigmoid || !free[v] ? 0.0f : -(expf(x[v] - (float)most) / (float)sum) * (float)inner;
  }
  for (int i0 = 0; i0 < p.k; i0 += G) {
    int id;
    double g, s;
    slot(i0 + lane, &id, &g, &s);
    const double l = id >= 0 ? (double)(float)L[id] : 0.0;
    const double ds = each * (g - less);
    const float mine = s == 0 ? 0.0f : (float)(a.sigmoid ? ds * s * sigmoid64(-l) : s * (ds - inner));
    const int n = min(G, p.k - i0);
    for (int j = 0; j < n; j++) {
      const int e = __shfl(id, j, G);
      const float d = __shfl(mine, j, G);
#pragma unroll
      for (int v = 0; v < V; v++)
        if (e == lane * V + v && free[v]) grad[v] = d;
    }
  }
  T* const out = static_cast<T*>(p.dL) + t * p.E;
  const int c = lane * V;
  if (c + V <= p.E) {
    constexpr int P = V < Elem<T>::PER16 ? V : Elem<T>::PER16;
#pragma unroll
    for (int h = 0; h < V; h += P) {
      Pack<T, P> v;
#pragma unroll
      for (int i = 0; i < P; i++) v.e[i] = narrow<T>(grad[h + i]);
      *reinterpret_cast<Pack<T, P>*>(out + c + h) = v;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; v++)
      if (c + v < p.E) out[c + v] = narrow<T>(grad[v]);
  }
}

}  // namespace tc355
