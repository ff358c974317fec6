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
// go through LDS once: lane g finds the two best of group g, and ranks it by counting the better ones.  Then k rounds find the largest of what is left, by keys of 32 bits
// made of the score and the expert's number; where these do not tell two scores apart that differ, the wavefront chooses again by 64 bits.  The scores of the k
// chosen are computed again by the lanes that write them, all at once.  What bounds it is the rounds' latency and the exponentials of 64 bits.
//
// Measured: 16384 tokens of 256 experts, 16 groups of which 5, 8 chosen, 28-32 us for the selection (43 with k rounds over keys of 64 bits, library exponentials and scores at a stride of
// 128 bytes in LDS; of it 8 for the rounds, 3 for the groups), 12 for sums and places, 7-8 for the gradient.  All but the gradient 37, by softmax without groups 31; tc_route, which gives as many
// experts 64 lanes a token, 44.
// 16 tokens of 128, 8 groups of which 3, 6 chosen, 9.7 in one launch (7.4 with one chosen and no groups).
#pragma once
#include "expert_types.hpp"
#include "lanes.hpp"
#include "route.hpp"

namespace tc355 {

constexpr int ROUTE_MOST_GROUPS = 64;

// The scores of a token in LDS: one place in 17 stays empty, so that lanes that take V neighbours each, or a group of experts each, meet in few banks; the tokens of a wavefront
// lie half the banks apart.
__host__ __device__ constexpr int score_place(int e) { return e + (e >> 4); }
__host__ __device__ constexpr int score_places(int E, int groups) {
  const int n = score_place(E - 1) + 1 + groups;
  return n + (48 - n % 32) % 32;  // (16 of every 32)
}

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
// exp(y) for y <= 0 to about one part in 2^52: y = n ln 2 + r with |r| <= ln 2 / 2, ln 2 in two parts so that n times the first is exact, and the series up to r^12 / 12!
// (the next term is below 2^-52).  A third of the instructions of the function for any argument.
__device__ __forceinline__ double exp64(double y) {
  y = y < -1100.0 ? -1100.0 : y;  // (0; NaN stays)
  const double n = __builtin_rint(y * 1.4426950408889634);
  const double r = __builtin_fma(-n, 0x1.a39ef35793c76p-33, __builtin_fma(-n, 0x1.62e42fee00000p-1, y));
  double p = 1.0 / 479001600;
  p = __builtin_fma(p, r, 1.0 / 39916800);
  p = __builtin_fma(p, r, 1.0 / 3628800);
  p = __builtin_fma(p, r, 1.0 / 362880);
  p = __builtin_fma(p, r, 1.0 / 40320);
  p = __builtin_fma(p, r, 1.0 / 5040);
  p = __builtin_fma(p, r, 1.0 / 720);
  p = __builtin_fma(p, r, 1.0 / 120);
  p = __builtin_fma(p, r, 1.0 / 24);
  p = __builtin_fma(p, r, 1.0 / 6);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_amdgcn_ldexp(p, (int)n);
}
// 1 / d for finite d >= 1, by two of Newton's steps.
__device__ __forceinline__ double inverse64(double d) {
  double r = __builtin_amdgcn_rcp(d);
  r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
  return __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
}
__device__ __forceinline__ double sigmoid64(double x) {
  const double t = exp64(-__builtin_fabs(x)), r = inverse64(1.0 + t);
  return x < 0 ? t * r : r;
}
__device__ __forceinline__ double add64(double x, double y) { return x + y; }
__device__ __forceinline__ double most64(double x, double y) { return __builtin_fmax(x, y); }

// The lane of the group's best key of 64 bits, `mine` each lane's own best: by the upper halves and, where several lanes agree in those, by the lower ones, then by the lane.
template <int G>
__device__ __forceinline__ int best_lane(unsigned long long mine) {
  const unsigned upper = (unsigned)(mine >> 32), within = (threadIdx.x & 63) & ~(G - 1);
  bool winner = upper == group_all<G>(upper, larger);
  const unsigned long long members = __ballot(winner) >> within & (~0ull >> (64 - G));
  if (members & (members - 1)) {
    const unsigned lower = winner ? (unsigned)mine : 0;
    winner = lower == group_all<G>(lower, larger) && winner;
  }
  return __ffsll((long long)(__ballot(winner) >> within & (~0ull >> (64 - G)))) - 1;
}

template <typename T, int G, int V>
__global__ __launch_bounds__(WG_THREADS) void route_balanced_kernel(RouteBalancedArgs a) {
  const RouteArgs& p = a.r;
  extern __shared__ __align__(8) int mem[];  // as route_kernel's; behind it, with groups, [WG_THREADS / G][score_places] scores
  __shared__ int part[WAVES_PER_WG];
  const int bins = 1 << p.bits;
  for (int b = threadIdx.x; b < bins; b += WG_THREADS) mem[b] = 0;
  __syncthreads();
  const int lane = threadIdx.x & (G - 1), group = threadIdx.x / G;
  const T* L = static_cast<const T*>(p.L);
  double* const scores = reinterpret_cast<double*>(mem + (p.count ? bins : bins * (1 + WAVES_PER_WG))) + group * score_places(p.E, a.groups);
  const bool grouped = a.keep < a.groups;
  const int size = p.E / a.groups;
  float bias[V];
#pragma unroll
  for (int v = 0; v < V; v++) bias[v] = a.Bias && lane * V + v < p.E ? a.Bias[lane * V + v] : 0.0f;
  // how far biases lie apart, 1 at most: what the window of softmax scores takes beside them
  float low = 0.0f, high = 0.0f;
#pragma unroll
  for (int v = 0; v < V; v++) {
    low = fminf(low, bias[v]);
    high = fmaxf(high, bias[v]);
  }
  const double spread = fminf(1.0f, group_all<G>(high, most_of) + group_all<G>(-low, most_of));
  const int number_bits = 32 - __builtin_clz(max(1, p.E - 1));
  for (int r = group; r < p.tokens; r += WG_THREADS / G) {
    const int64_t t = (int64_t)blockIdx.x * p.tokens + r;
    if (t >= p.T) break;  // (the whole group, and all groups behind it)
    float x[V];
    load_logits<T, V>(L + t * p.E, lane * V, p.E, x);
    double c[V];
    double most = 0, share = 1, window = 2;
    if (a.sigmoid) {
#pragma unroll
      for (int v = 0; v < V; v++) c[v] = sigmoid64(x[v]);
    } else {
      float m = -__builtin_inff();
#pragma unroll
      for (int v = 0; v < V; v++) m = fmaxf(m, x[v]);
      m = group_all<G>(m, most_of);
      if (m == -__builtin_inff()) m = 0.0f;  // (nothing to choose: every exp is 0, or NaN)
      most = m;
      double sum = 0;
#pragma unroll
      for (int v = 0; v < V; v++) {
        c[v] = exp64((double)x[v] - most);
        sum += c[v];
      }
      sum = group_all<G>(sum, add64);
      share = sum == 0 ? 1.0 : inverse64(sum);
#pragma unroll
      for (int v = 0; v < V; v++) c[v] *= share;
      window = share + spread;  // (the largest score is `share`)
    }
    bool odd = false;  // NaN or +inf among the scores
#pragma unroll
    for (int v = 0; v < V; v++) {
      c[v] = x[v] == -__builtin_inff() ? -__builtin_inf() : c[v] + (double)bias[v];
      odd |= !(c[v] < __builtin_inf());
    }
    bool exact = __ballot(odd) != 0;  // (of the wavefront)
    if (grouped) {
      unsigned long long* const best = reinterpret_cast<unsigned long long*>(scores + score_place(p.E - 1) + 1);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int v = 0; v < V; v++)
        if (lane * V + v < p.E) scores[score_place(lane * V + v)] = c[v];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      for (int g = lane; g < a.groups; g += G) {
        double first = -__builtin_inf(), second = -__builtin_inf();
        if (exact) {  // NaN before every number
          unsigned long long one = 0, two = 0;
          for (int j = 0; j < size; j++) {
            const double s = scores[score_place(g * size + j)];
            const unsigned long long o = score_order(s);
            if (o > one) {
              two = one;
              second = first;
              one = o;
              first = s;
            } else if (o > two) {
              two = o;
              second = s;
            }
          }
        } else {
#pragma unroll 4
          for (int j = 0; j < size; j++) {
            const double s = scores[score_place(g * size + j)];
            second = most64(second, __builtin_fmin(first, s));
            first = most64(first, s);
          }
        }
        best[g] = score_order(second == -__builtin_inf() ? first : first + second);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      for (int g = lane; g < a.groups; g += G) {
        const unsigned long long mine = best[g];
        int better = 0;
#pragma unroll 4
        for (int h = 0; h < a.groups; h++) {
          const unsigned long long other = best[h];
          better += other > mine || (other == mine && h < g) ? 1 : 0;
        }
        scores[g] = better < a.keep ? 1.0 : 0.0;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      int g = lane * V / size, end = (g + 1) * size;
#pragma unroll
      for (int v = 0; v < V; v++) {
        const int e = lane * V + v;
        if (e >= end) {
          g++;
          end += size;
        }
        if (e < p.E && scores[g] == 0.0) c[v] = -__builtin_inf();
      }
    }
    int id = -1;
    if (!exact) {
      // Keys of 32 bits: where the score lies in a window below the largest one, in steps, then the expert, lower numbers first: a maximum names its expert.  Chosen ones that follow each
      // other in one step are told apart by the scores themselves, and so are the last chosen and all that are left in its step; where these differ, the wavefront chooses again, by them.
      double top = c[0];
#pragma unroll
      for (int v = 1; v < V; v++) top = most64(top, c[v]);
      top = group_all<G>(top, most64);
      const unsigned last = (1u << number_bits) - 1, steps = 0xffffffffu >> number_bits;
      const double per = (double)(steps - 1) / window, from = (double)steps - top * per;
      unsigned key[V];
#pragma unroll
      for (int v = 0; v < V; v++) {
        // (1 .. steps: below the window, and beyond `steps` where a bias takes the bits that `from` has, one step holds many)
        const double at = __builtin_fmin(most64(__builtin_fma(c[v], per, from), 1.0), (double)steps);
        key[v] = c[v] == -__builtin_inf() ? 0 : (unsigned)at << number_bits | (last - (lane * V + v));
      }
      const auto score = [&](unsigned of) {  // of the expert that a key names, in all lanes
        double c_ = -__builtin_inf();
        const int e = (int)(last - (of & last));
#pragma unroll
        for (int v = 0; v < V; v++) c_ = lane * V + v == e ? c[v] : c_;
        return group_all<G>(c_, most64);
      };
      unsigned before = 0;
      for (int i = 0; i < p.k; i++) {
        unsigned best = key[0];
#pragma unroll
        for (int v = 1; v < V; v++) best = larger(best, key[v]);
        best = group_all<G>(best, larger);
        if (best >> number_bits == before >> number_bits && best) exact |= score(best) != score(before);
        if (lane == i && best) id = (int)(last - (best & last));
        before = best;
#pragma unroll
        for (int v = 0; v < V; v++) key[v] = key[v] == best ? 0 : key[v];
      }
      bool near = false;
#pragma unroll
      for (int v = 0; v < V; v++) near |= key[v] && key[v] >> number_bits == before >> number_bits;
      if (__ballot(near)) {
        const double border = score(before);
#pragma unroll
        for (int v = 0; v < V; v++) exact |= key[v] && key[v] >> number_bits == before >> number_bits && c[v] != border;
      }
      exact = __ballot(exact) != 0;
    }
    if (exact) {
      unsigned long long key[V];
#pragma unroll
      for (int v = 0; v < V; v++) key[v] = score_order(c[v]);
      id = -1;
      for (int i = 0; i < p.k; i++) {
        unsigned long long mine = 0;
        int at = 0;
#pragma unroll
        for (int v = V - 1; v >= 0; v--)
          if (key[v] >= mine) {
            mine = key[v];
            at = v;
          }
        const int src = best_lane<G>(mine);
        const bool none = __shfl(mine == 0 ? 1 : 0, src, G) != 0;
        const int e = __shfl(lane * V + at, src, G);
#pragma unroll
        for (int v = 0; v < V; v++)
          if (lane == src && at == v) key[v] = 0;
        if (lane == i) id = none ? -1 : e;  // (k <= G, by the host's choice of G)
      }
    }
    const float logit = id >= 0 ? (float)L[t * p.E + id] : 0.0f;
    double w = 0;
    if (id >= 0) w = a.sigmoid ? sigmoid64(logit) : exp64((double)logit - most) * share;
    double total = 1;
    if (p.norm) {
      total = group_all<G>(w, add64);
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

// The chosen experts' part in 64 bits, by the lanes that hold the slots: their scores may be far below the others'.  softmax's other columns and its sum take
// exponentials in 32 bits (the sum joins lanes in 64): such a column is off by some 2^-18 of itself, in float too, which a gradient bears; in 64 bits they would cost what they cost the selection.
template <typename T, int G, int V>
__global__ __launch_bounds__(WG_THREADS) void route_balanced_grad_kernel(RouteBalancedGradArgs a, int64_t first) {
  const RouteGradArgs& p = a.r;
  const int lane = threadIdx.x & (G - 1);
  const int64_t t = (first + blockIdx.x) * (WG_THREADS / G) + threadIdx.x / G;
  if (t >= p.T) return;
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
    sum = group_all<G>((double)part, add64);
    if (sum == 0) sum = 1;  // (a row of nothing)
  }
  // a slot a lane, G slots at a time: scores and sums over all slots first
  int id = -1;
  double g = 0, s = 0, slope = 0;  // slope: dS / dL of a sigmoid
  const auto slot = [&](int i) {
    id = i < p.k ? p.Id[t * p.k + i] : -1;
    if (id >= p.E) id = -1;
    g = s = slope = 0;
    if (id < 0) return;
    g = p.dWt[t * p.k + i];
    const double l = (float)L[id];
    if (l == -__builtin_inf()) return;
    if (a.sigmoid) {
      const double e = exp64(-__builtin_fabs(l)), r = inverse64(1.0 + e);
      s = l < 0 ? e * r : r;
      slope = e * r * r;
    } else {
      s = exp64(l - most) / sum;
    }
  };
  double total = 0, mean = 0;
  for (int i0 = 0; i0 < p.k; i0 += G) {
    slot(i0 + lane);
    total += s;
    mean += s == 0 ? 0.0 : g * s;
  }
  total = group_all<G>(total, add64);
  mean = group_all<G>(mean, add64);
  if (total < 1e-300) total = 1e-300;
  const double each = p.norm ? a.scale / total : a.scale, less = p.norm ? mean / total : 0.0;  // dS_i = each (g_i - less)
  const double inner = a.sigmoid || p.norm ? 0.0 : each * mean;  // sum_j dS_j S_j, of which norm leaves nothing
#pragma unroll
  for (int v = 0; v < V; v++) {
    free[v] = x[v] != -__builtin_inff();
    grad[v] = a.sigmoid || !free[v] ? 0.0f : -(expf(x[v] - (float)most) / (float)sum) * (float)inner;
  }
  for (int i0 = 0; i0 < p.k; i0 += G) {
    if (p.k > G) slot(i0 + lane);
    const double ds = each * (g - less);
    const float mine = s == 0 ? 0.0f : (float)(a.sigmoid ? ds * slope : s * (ds - inner));
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
