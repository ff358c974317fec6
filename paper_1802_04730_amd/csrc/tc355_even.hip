// Host side of the operators around experts whose load is kept even and whose weights are in 8 bits: layer norm, the balanced router, blocks of 8 bits, products
// of them, and the gradients (include/tc355.h).  Argument validation, kernel selection and launches.
#include <cmath>
#include <type_traits>

#include "expert_host.hpp"
#include "expert_mm_q8.hpp"
#include "expert_mm_q8_plan.hpp"
#include "layer_norm.hpp"
#include "quantize8.hpp"
#include "route_balanced.hpp"

using namespace tc355;

namespace {

template <int I>
using Int = std::integral_constant<int, I>;

// True if one of the outputs is an input or another output (NULL ones aside).
bool aliased(std::initializer_list<const void*> out, std::initializer_list<const void*> in) {
  for (auto o = out.begin(); o != out.end(); ++o) {
    if (!*o) continue;
    for (const void* i : in)
      if (*o == i) return true;
    for (auto q = out.begin(); q != o; ++q)
      if (*o == *q) return true;
  }
  return false;
}
bool misaligned_any(std::initializer_list<const void*> all) {
  for (const void* p : all)
    if (misaligned(p)) return true;
  return false;
}

// ---- layer norm -------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostNorm = (int64_t)1 << 26;  // columns
constexpr int NORM_MOST_PARTS = 512;             // workgroups of the gradient
constexpr int NORM_WORKGROUPS = 2048;            // of the norm itself

// f(lanes, units a lane) for rows of N columns in units of V, or false: they do not fit into registers.
template <int V, typename F>
bool by_row(int64_t N, F f) {
  const int64_t units = ceil_div(N, V);
  if constexpr (V == 1) {
    f(Int<16>{}, Int<1>{});
    return true;
  } else {
    if (units <= 32) f(Int<16>{}, Int<2>{});
    else if (units <= 128) f(Int<64>{}, Int<2>{});
    else if (units <= 256) f(Int<64>{}, Int<4>{});
    else if (units <= 512) f(Int<256>{}, Int<2>{});
    else if (units <= 1024) f(Int<256>{}, Int<4>{});
    else return false;
    return true;
  }
}
template <typename F>
tc_status by_norm_types(tc_type type, tc_type weight, F f) {
  return by_type(type, [&](auto t) { return weight == TC_F32 ? f(t, float{}) : f(t, t); });
}

// Parts of the sums for dW and dB: a row each while there are few, so that as many compute units work on them, though each part's sums are written and read again (N of 4 or 8 bytes for dW, as many for dB).  Measured, the
// gradient with its join, us, a row a part / 16 rows: bfloat16 (T,N) = (128,4096) 12 / 31, (512,2048) 20 / 24, (512,4096) 26 / 31, (512,8192) 44 / 51, (2048,4096) 29 / 34; float (300,1000) 13 / 17, (1500,333) 13 / 13.  The other
// way round where a part has the most to write beside its rows: bfloat16 (2048,2048) 39 / 28, (2048,8192) 58 / 54, float beyond registers (512,8192) 61 / 37.  From 8192 rows on both are 512.
int64_t norm_parts(int64_t T) { return std::min<int64_t>(T, NORM_MOST_PARTS); }
struct NormPlan {
  int64_t parts, stat, bytes;
};
NormPlan norm_plan(int64_t T, int64_t N) {
  NormPlan p{};
  p.parts = norm_parts(T);
  p.stat = round256(p.parts * 2 * N * 8);
  p.bytes = p.stat + round256(T * 2 * 8);
  return p;
}

// ---- router -----------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostTokens = (int64_t)ROUTE_TOKENS << 23;

template <typename F>
tc_status by_lanes(int64_t E, int64_t k, F f) {
  if (k <= 16 && E <= 256) {
    if (E <= 16) return f(Int<16>{}, Int<1>{});
    if (E <= 32) return f(Int<16>{}, Int<2>{});
    if (E <= 64) return f(Int<16>{}, Int<4>{});
    if (E <= 128) return f(Int<16>{}, Int<8>{});
    return f(Int<16>{}, Int<16>{});
  }
  if (E <= 128) return f(Int<64>{}, Int<2>{});
  if (E <= 256) return f(Int<64>{}, Int<4>{});
  if (E <= 512) return f(Int<64>{}, Int<8>{});
  return f(Int<64>{}, Int<16>{});
}
int64_t route_ws(int64_t T, int64_t E) {
  const int64_t tiles = ceil_div(T, ROUTE_TOKENS);
  return T <= ROUTE_ALONE ? 0 : (tiles + 1) * ((int64_t)4 << bits_of(E));
}

// ---- products -----------------------------------------------------------------------------------------------------------------

int64_t q8_blocks(int64_t n) { return ceil_div(n, Q8_BLOCK); }

struct Q8Plan {
  int64_t scales, bytes;  // of the rows in 8 bits, in the workspace
};
Q8Plan q8_plan(int64_t T, int64_t K) {
  const int64_t n = T * q8_blocks(K);
  return {round256(n * Q8_BLOCK), round256(n * Q8_BLOCK) + round256(n)};
}

tc_status quantize_rows(const void* X, void* Q, void* S, int64_t R, int64_t K, tc_type type, hipStream_t s) {
  const QuantizeRowsArgs a{X, static_cast<unsigned char*>(Q), static_cast<unsigned char*>(S), R * q8_blocks(K), (int)K, (int)q8_blocks(K)};
  return by_type(type, [&](auto t) {
    constexpr int U = 4;
    return in_launches(ceil_div(a.all, WG_THREADS / 16 * U), [&](dim3 n, int64_t at) { quantize_rows_kernel<decltype(t), U><<<n, dim3(WG_THREADS), 0, s>>>(a, at); });
  });
}

template <typename T, int BM, int WM, int WN>
tc_status launch_q8_tile(Q8Args a, hipStream_t s) {
  a.nt = (int)ceil_div(a.NO, BM);
  const int64_t grid = (most_row_tiles(a.R, a.E, BM) * a.nt + 7) / 8 * 8 + (BM == 256 ? 8 : 0);  // (two sets of tiles, each in whole eights)
  if (grid > kMostIndex / (64 * WM * WN) * 2) return TC_ERR_UNSUPPORTED;
  expert_mm_q8_kernel<T, BM, BM, WM, WN><<<dim3((unsigned)grid), dim3(64 * WM * WN), 0, s>>>(a);
  return launched();
}
template <typename T, int CT, int WK>
tc_status launch_q8_few(Q8Args a, hipStream_t s) {
  a.nt = (int)ceil_div(a.NO, 16 * CT);
  const int64_t grid = (most_row_tiles(a.R, a.E, 16) * a.nt + 7) / 8 * 8;
  if (grid > kMostIndex / (64 * WK) * 2) return TC_ERR_UNSUPPORTED;
  expert_few_rows_q8_kernel<T, CT, WK><<<dim3((unsigned)grid), dim3(64 * WK), 0, s>>>(a);
  return launched();
}

bool q8_extents(int64_t T, int64_t R, int64_t E, int64_t N, int64_t K) {
  return T >= 0 && R >= 0 && E > 0 && N > 0 && K > 0 && T < kMostRows && R < kMostRows && E < kMostRows && N < kMostWidth && K < kMostWidth;
}

}  // namespace

extern "C" {

tc_status tc_layer_norm(const void* X, const void* W, const void* B, void* O, int64_t T, int64_t N, float eps, tc_type type, tc_type weight_type,
                        void* hip_stream) {
  if (!known(type) || (weight_type != type && weight_type != TC_F32) || T < 0 || N <= 0 || !(eps >= 0.0f)) return TC_ERR_SHAPE;
  if (!W || (T && (!X || !O))) return TC_ERR_NULL;
  if (T && aliased({O}, {X, W, B})) return TC_ERR_ALIAS;
  if (misaligned_any({X, W, B, O})) return TC_ERR_ALIGN;
  if (T > kMostRows || N >= kMostNorm) return TC_ERR_UNSUPPORTED;
  if (T == 0) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  NormArgs a{};
  a.X = X; a.W = W; a.B = B; a.O = O; a.T = T; a.N = (int)N; a.eps = eps;
  return by_norm_types(type, weight_type, [&](auto t, auto w) {
    typedef decltype(t) X_;
    typedef decltype(w) W_;
    const auto run = [&](auto v) {
      constexpr int V = decltype(v)::value;
      const bool fits = by_row<V>(N, [&](auto g, auto c) {
        const int64_t grid = std::min<int64_t>(ceil_div(T, WG_THREADS / g.value), NORM_WORKGROUPS);
        norm_rows_kernel<X_, W_, V, g.value, c.value><<<dim3((unsigned)grid), dim3(WG_THREADS), 0, s>>>(a);
      });
      if (!fits) norm_long_kernel<X_, W_, V><<<dim3((unsigned)std::min<int64_t>(T, NORM_WORKGROUPS)), dim3(WG_THREADS), 0, s>>>(a);
      return took(fits ? "layer_norm:rows" : "layer_norm:long", launched());
    };
    constexpr int V = Elem<X_>::PER16;
    return N < V ? run(Int<1>{}) : run(Int<V>{});
  });
}

size_t tc_layer_norm_grad_workspace_bytes(int64_t T, int64_t N) {
  if (T <= 0 || N <= 0 || T > kMostRows || N >= kMostNorm) return 0;
  return (size_t)norm_plan(T, N).bytes;
}

tc_status tc_layer_norm_grad(const void* dO, const void* X, const void* W, void* dX, void* dW, void* dB, int64_t T, int64_t N, float eps, int32_t add,
                             tc_type type, tc_type weight_type, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!known(type) || (weight_type != type && weight_type != TC_F32) || T < 0 || N <= 0 || !(eps >= 0.0f)) return TC_ERR_SHAPE;
  if (!W || (dB && !dW) || (T && (!dO || !X || !dX))) return TC_ERR_NULL;
  if (aliased({dX, dW, dB, workspace}, {dO, X, W})) return TC_ERR_ALIAS;
  if (misaligned_any({dO, X, W, dX, dW, dB})) return TC_ERR_ALIGN;
  if (T > kMostRows || N >= kMostNorm) return TC_ERR_UNSUPPORTED;
  const NormPlan pl = norm_plan(T, N);
  if (T && dW && (!workspace || misaligned(workspace) || workspace_bytes < (size_t)pl.bytes)) return TC_ERR_WORKSPACE;
  if (T == 0 && (add || !dW)) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  NormArgs a{};
  a.X = X; a.W = W; a.dO = dO; a.dX = dX; a.T = T; a.N = (int)N; a.eps = eps;
  a.part = dW ? workspace : nullptr;
  a.stat = dW ? static_cast<char*>(workspace) + pl.stat : nullptr;
  return by_norm_types(type, weight_type, [&](auto t, auto w) {
    typedef decltype(t) X_;
    typedef decltype(w) W_;
    typedef typename Wide<X_>::type S;
    int64_t parts = 0;
    const auto run = [&](auto v) {
      constexpr int V = decltype(v)::value;
      const bool fits = by_row<V>(N, [&](auto g, auto c) {
        constexpr int SLOTS = WG_THREADS / g.value;
        parts = std::min<int64_t>(norm_parts(T), ceil_div(T, SLOTS));
        norm_rows_grad_kernel<X_, W_, V, g.value, c.value><<<dim3((unsigned)parts), dim3(WG_THREADS), SLOTS > 1 && dW ? 2 * N * sizeof(S) : 0, s>>>(a);
      });
      if (!fits) {
        norm_long_grad_kernel<X_, W_, V><<<dim3((unsigned)std::min<int64_t>(T, NORM_WORKGROUPS)), dim3(WG_THREADS), 0, s>>>(a);
        if (dW) {
          parts = norm_parts(T);
          norm_columns_kernel<X_, V><<<dim3((unsigned)ceil_div(ceil_div(N, V), WG_THREADS), (unsigned)parts), dim3(WG_THREADS), 0, s>>>(a);
        }
      }
      return fits;
    };
    constexpr int V = Elem<X_>::PER16;
    const bool fits = T == 0 || (N < V ? run(Int<1>{}) : run(Int<V>{}));
    if (dW)
      norm_join_kernel<S, W_><<<dim3((unsigned)ceil_div((dB ? 2 : 1) * N, 16)), dim3(WG_THREADS), 0, s>>>(static_cast<const S*>(workspace), (int)parts, (int)N, dW, dB, add != 0);
    return took(fits ? "layer_norm_grad:rows" : "layer_norm_grad:long", launched());
  });
}

size_t tc_route_balanced_workspace_bytes(int64_t T, int64_t E, int64_t k) {
  if (T <= 0 || E <= 0 || k <= 0 || k > E || E > ROUTE_MOST_E || k > ROUTE_MOST_K || T >= kMostTokens || prod_reaches({T, k}, kMostRows)) return 0;
  return (size_t)route_ws(T, E);
}

tc_status tc_route_balanced(const void* L, const float* Bias, float* Wt, int32_t* Id, int32_t* Off, int32_t* Row, int32_t* Place, int64_t T, int64_t E,
                            int64_t k, int64_t groups, int64_t keep, int32_t sigmoid, int32_t norm, float scale, tc_type type, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  if (!known(type) || T < 0 || E <= 0 || k <= 0 || k > E || groups <= 0 || E % groups || keep <= 0 || keep > groups) return TC_ERR_SHAPE;
  if (!Off || (T && (!L || !Wt || !Id || !Row || !Place))) return TC_ERR_NULL;
  if (aliased({Wt, Id, Off, Row, Place, workspace}, {L, Bias})) return TC_ERR_ALIAS;
  if (misaligned_any({L, Bias, Wt, Id, Off, Row, Place})) return TC_ERR_ALIGN;
  if (E > ROUTE_MOST_E || k > ROUTE_MOST_K || prod_reaches({std::max<int64_t>(T, 1), k}, kMostRows) || T >= kMostTokens) return TC_ERR_UNSUPPORTED;
  if (keep < groups && groups > ROUTE_MOST_GROUPS) return TC_ERR_UNSUPPORTED;
  const int64_t need = route_ws(T, E);
  const bool tiles = need && workspace && !misaligned(workspace) && workspace_bytes >= (size_t)need;
  if (!tiles && T > ROUTE_MOST_ALONE) return TC_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  RouteBalancedArgs a{};
  a.r = RouteArgs{L, Wt, Id, Off, Row, Place, tiles ? static_cast<int*>(workspace) : nullptr, (int)T, (int)E, (int)k, norm != 0, bits_of(E),
                  tiles ? (int)ceil_div(T, ROUTE_TOKENS) : 1, 0, tiles ? ROUTE_TOKENS : ROUTE_MOST_ALONE};
  a.r.summed = a.r.tiles > ROUTE_DIRECT_TILES;
  a.Bias = Bias; a.scale = scale; a.groups = (int)groups; a.keep = (int)keep; a.sigmoid = sigmoid != 0;
  const size_t bins = (size_t)4 << a.r.bits;
  return by_type(type, [&](auto x) {
    return by_lanes(E, k, [&](auto g, auto v) {
      typedef decltype(x) X;
      const size_t scores = keep < groups ? (size_t)(WG_THREADS / g.value) * score_places((int)E, (int)groups) * 8 : 0;
      route_balanced_kernel<X, g.value, v.value><<<dim3((unsigned)a.r.tiles), dim3(WG_THREADS), (a.r.count ? bins : bins * (1 + WAVES_PER_WG)) + scores, s>>>(a);
      if (!a.r.count) return took("route_balanced:one", launched());
      if (a.r.summed) sort_sum_kernel<<<dim3(1u << a.r.bits), dim3(WG_THREADS), 0, s>>>(a.r.count, a.r.tiles);
      route_place_kernel<<<dim3((unsigned)a.r.tiles), dim3(WG_THREADS), bins * (1 + WAVES_PER_WG), s>>>(a.r);
      return took("route_balanced:tiles", launched());
    });
  });
}

tc_status tc_route_balanced_grad(const void* L, const int32_t* Id, const float* dWt, void* dL, int64_t T, int64_t E, int64_t k, int32_t sigmoid, int32_t norm,
                                 float scale, tc_type type, void* hip_stream) {
  if (!known(type) || T < 0 || E <= 0 || k <= 0 || k > E) return TC_ERR_SHAPE;
  if (T && (!L || !Id || !dWt || !dL)) return TC_ERR_NULL;
  if (T && aliased({dL}, {L, Id, dWt})) return TC_ERR_ALIAS;
  if (misaligned_any({L, Id, dWt, dL})) return TC_ERR_ALIGN;
  if (E > ROUTE_MOST_E || k > ROUTE_MOST_K || prod_reaches({std::max<int64_t>(T, 1), k}, kMostRows)) return TC_ERR_UNSUPPORTED;
  if (T == 0) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const RouteBalancedGradArgs a{RouteGradArgs{L, Id, dWt, dL, (int)T, (int)E, (int)k, norm != 0}, scale, sigmoid != 0};
  return by_type(type, [&](auto x) {
    return by_lanes(E, 1, [&](auto g, auto v) {
      typedef decltype(x) X;
      return took("route_balanced_grad:rows", in_launches(ceil_div(T, WG_THREADS / g.value), [&](dim3 n, int64_t at) {
                    route_balanced_grad_kernel<X, g.value, v.value><<<n, dim3(WG_THREADS), 0, s>>>(a, at);
                  }));
    });
  });
}

tc_status tc_quantize_rows(const void* X, void* Q, void* S, int64_t R, int64_t K, tc_type type, void* hip_stream) {
  if (!known(type) || R < 0 || K <= 0) return TC_ERR_SHAPE;
  if (R && (!X || !Q || !S)) return TC_ERR_NULL;
  if (R && aliased({Q, S}, {X})) return TC_ERR_ALIAS;
  if (misaligned_any({X, Q, S})) return TC_ERR_ALIGN;
  if (R > kMostRows || K > kMostRows) return TC_ERR_UNSUPPORTED;
  if (R == 0) return TC_OK;
  return took("quantize_rows:blocks", quantize_rows(X, Q, S, R, K, type, static_cast<hipStream_t>(hip_stream)));
}

tc_status tc_quantize_weights(const void* W, void* Q, void* S, void* Qt, void* St, int64_t E, int64_t N, int64_t K, tc_type type, void* hip_stream) {
  if (!known(type) || E <= 0 || N <= 0 || K <= 0) return TC_ERR_SHAPE;
  if (!W || !Q || !S || !Qt != !St) return TC_ERR_NULL;
  if (aliased({Q, S, Qt, St}, {W})) return TC_ERR_ALIAS;
  if (misaligned_any({W, Q, S, Qt, St})) return TC_ERR_ALIGN;
  if (E >= kMostRows || N > kMostRows || K > kMostRows || prod_reaches({E, q8_blocks(N), q8_blocks(K)}, (int64_t)1 << 45)) return TC_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const auto bytes = [](void* p) { return static_cast<unsigned char*>(p); };
  const QuantizeWeightsArgs a{W, bytes(Q), bytes(S), bytes(Qt), bytes(St), E, (int)N, (int)K, (int)q8_blocks(N), (int)q8_blocks(K)};
  return took("quantize_weights:blocks", by_type(type, [&](auto t) {
                return in_launches(E * a.nb * a.kb, [&](dim3 n, int64_t at) { quantize_weights_kernel<decltype(t)><<<n, dim3(WG_THREADS), 0, s>>>(a, at); });
              }));
}

size_t tc_expert_mm_q8_workspace_bytes(int64_t T, int64_t R, int64_t E, int64_t N, int64_t K) {
  if (!q8_extents(T, R, E, N, K) || T == 0 || R == 0) return 0;
  return (size_t)q8_plan(T, K).bytes;
}

tc_status tc_expert_mm_q8(const void* X, const void* SX, const void* W, const void* SW, const int32_t* Off, const int32_t* Row, const void* gate, void* Y,
                          int64_t T, int64_t R, int64_t E, int64_t N, int64_t K, int32_t relu, tc_type type, void* workspace, size_t workspace_bytes,
                          void* hip_stream) {
  if (!known(type) || T < 0 || R < 0 || E <= 0 || N <= 0 || K <= 0 || (R && !Row && T != R) || (!Off && E != 1)) return TC_ERR_SHAPE;
  if (!W || !SW || (R && (!Y || (T && !X)))) return TC_ERR_NULL;
  if (R && aliased({Y}, {X, SX, W, SW, Off, Row, gate, workspace})) return TC_ERR_ALIAS;
  if (workspace && aliased({workspace}, {X, SX, W, SW, Off, Row, gate})) return TC_ERR_ALIAS;
  if (misaligned_any({X, SX, W, SW, Off, Row, gate, Y})) return TC_ERR_ALIGN;
  if (!q8_extents(T, R, E, N, K)) return TC_ERR_UNSUPPORTED;
  const Q8Plan pl = q8_plan(T, K);
  if (R && T && !SX && (!workspace || misaligned(workspace) || workspace_bytes < (size_t)pl.bytes)) return TC_ERR_WORKSPACE;
  if (R == 0) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const auto bytes = [](const void* p) { return static_cast<const unsigned char*>(p); };
  Q8Args a{bytes(X), bytes(SX), bytes(W), bytes(SW), Y, gate, Off, Row, (int)R, (int)T, (int)E, (int)q8_blocks(K), (int)N, 0, relu != 0};
  if (!SX && T) {
    a.A = bytes(workspace);
    a.SA = bytes(workspace) + pl.scales;
    if (const tc_status st = quantize_rows(X, workspace, static_cast<char*>(workspace) + pl.scales, T, K, type, s); st != TC_OK) return st;
  }
  const bool few = q8_few_rows(type == TC_F32, compute_units(), R, E, N);
  return took(few ? "expert_mm_q8:rows" : "expert_mm_q8:tile", by_type(type, [&](auto t) {
                typedef decltype(t) X_;
                if (few) return launch_q8_few<X_, 2, 4>(a, s);
                const int side = q8_tile_side(type == TC_F32, compute_units(), R, E, N, a.stages);
                if constexpr (sizeof(X_) == 2)
                  if (side == 256) return launch_q8_tile<X_, 256, 2, 2>(a, s);
                return side == 64 ? launch_q8_tile<X_, 64, 2, 2>(a, s) : launch_q8_tile<X_, 128, 2, 2>(a, s);
              }));
}

}  // extern "C"
