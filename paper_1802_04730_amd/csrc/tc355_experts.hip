// Host side of the operators around experts: token tables, router, products grouped by expert, weighted sums, and their gradients
// (include/tc355.h).  Argument validation, kernel selection and launches.
#include <type_traits>

#include "embed.hpp"
#include "expert_host.hpp"
#include "expert_mm.hpp"
#include "expert_mm_plan.hpp"
#include "expert_rows.hpp"
#include "expert_sum.hpp"
#include "key_sort.hpp"
#include "route.hpp"

using namespace tc355;

namespace {

constexpr int64_t kMostTokens = (int64_t)ROUTE_TOKENS << 23;  // of the router: fewer than 2^32 threads

// Lanes that share a row of `units` 16-byte units, and groups of them that a row takes.
struct RowLanes {
  int lpr, cols;
};
RowLanes row_lanes(int64_t width, int per16) {
  const int64_t units = ceil_div(width, per16);
  int lpr = 1;
  while (lpr < units && lpr < 64) lpr *= 2;
  return {lpr, (int)ceil_div(units, lpr)};
}

// ---- token tables -----------------------------------------------------------------------------------------------------------

struct EmbedGradPlan {
  int key_bits, passes, bits;
  int64_t tiles;
  int64_t key_a, order_a, key_b, order_b, count, part, bytes;  // offsets into the workspace
};

EmbedGradPlan embed_grad_plan(int64_t E, int64_t D, int64_t T) {
  EmbedGradPlan p{};
  p.key_bits = bits_of(E);
  p.passes = (int)ceil_div(p.key_bits, SORT_MOST_BITS);
  p.bits = (int)ceil_div(p.key_bits, p.passes);
  p.tiles = ceil_div(T, SORT_TILE);
  // (as many as short chunks make; never fewer than fewer tokens have: a workspace for more tokens serves fewer)
  const int64_t chunks = std::max(ceil_div(T, EMBED_CHUNK), ceil_div(std::min<int64_t>(T, EMBED_FEW), EMBED_SMALL_CHUNK));
  int64_t at = 0;
  const auto take = [&](int64_t n) {
    const int64_t o = at;
    at += round256(n);
    return o;
  };
  p.key_a = take(T * 4);
  p.order_a = take(T * 4);
  if (T > SORT_SMALL) {
    p.key_b = take(T * 4);
    p.order_b = take(T * 4);
    p.count = take((p.tiles + 1) * ((int64_t)4 << p.bits));
  }
  p.part = take(chunks * 2 * D * 8);
  p.bytes = at;
  return p;
}

// The tokens sorted by number, for embed_grad; *key and *order: where they are.
tc_status sort_tokens(const EmbedGradPlan& pl, const int32_t* Idx, int64_t T, int64_t E, int64_t pad, char* ws, const int** key, const int** order,
                      hipStream_t s) {
  int* keys[2] = {reinterpret_cast<int*>(ws + pl.key_a), reinterpret_cast<int*>(ws + pl.key_b)};
  int* orders[2] = {reinterpret_cast<int*>(ws + pl.order_a), reinterpret_cast<int*>(ws + pl.order_b)};
  SortPass a{};
  a.n = (int)T;
  a.E = (int)E;
  a.bits = pl.bits;
  a.pad = pad;
  a.tiles = (int)pl.tiles;
  a.key = Idx;
  if (T <= SORT_SMALL) {
    a.key_out = keys[0];
    a.order_out = orders[0];
    sort_rank_kernel<<<(unsigned)ceil_div(T, 32), WG_THREADS, (size_t)ceil_div(T, 32) * 32 * 4, s>>>(a);
    *key = keys[0];
    *order = orders[0];
    return launched();
  }
  a.count = reinterpret_cast<int*>(ws + pl.count);
  a.summed = pl.tiles > SORT_DIRECT_TILES;
  const unsigned tiles = (unsigned)pl.tiles, bins = 1u << pl.bits;
  for (int i = 0; i < pl.passes; i++) {
    a.shift = i * pl.bits;
    a.key_out = keys[i & 1];
    a.order_out = orders[i & 1];
    sort_count_kernel<<<tiles, SORT_THREADS, 0, s>>>(a);
    if (a.summed) sort_sum_kernel<<<bins, WG_THREADS, 0, s>>>(a.count, (int)tiles);
    sort_scatter_kernel<<<tiles, SORT_THREADS, 0, s>>>(a);
    if (const tc_status st = launched(); st != TC_OK) return st;
    a.key = keys[i & 1];
    a.order = orders[i & 1];
  }
  *key = a.key;
  *order = a.order;
  return TC_OK;
}

// ---- router -----------------------------------------------------------------------------------------------------------------

template <typename F>
tc_status by_lanes(int64_t E, int64_t k, F f) {
  typedef std::integral_constant<int, 16> G16;
  typedef std::integral_constant<int, 64> G64;
  if (k <= 16 && E <= 128) {
    if (E <= 16) return f(G16{}, std::integral_constant<int, 1>{});
    if (E <= 32) return f(G16{}, std::integral_constant<int, 2>{});
    if (E <= 64) return f(G16{}, std::integral_constant<int, 4>{});
    return f(G16{}, std::integral_constant<int, 8>{});
  }
  if (E <= 128) return f(G64{}, std::integral_constant<int, 2>{});
  if (E <= 256) return f(G64{}, std::integral_constant<int, 4>{});
  if (E <= 512) return f(G64{}, std::integral_constant<int, 8>{});
  return f(G64{}, std::integral_constant<int, 16>{});
}

int64_t route_ws(int64_t T, int64_t E) {
  const int64_t tiles = ceil_div(T, ROUTE_TOKENS);
  return T <= ROUTE_ALONE ? 0 : (tiles + 1) * ((int64_t)4 << bits_of(E));
}

// ---- products grouped by expert -----------------------------------------------------------------------------------------------

template <typename T, bool ACROSS, int MODE, int BM, int BN, int WM, int WN, int D>
tc_status launch_rows_tile(ExpertRowsArgs a, hipStream_t s) {
  a.nt = (int)ceil_div(a.NO, BN);
  const int64_t grid = (most_row_tiles(a.R, a.E, BM) * a.nt + 7) / 8 * 8;
  if (grid > kMostIndex / (64 * WM * WN) * 2) return TC_ERR_UNSUPPORTED;
  expert_rows_tile_kernel<T, ACROSS, MODE, BM, BN, WM, WN, D><<<dim3((unsigned)grid), dim3(64 * WM * WN), 0, s>>>(a);
  return launched();
}

template <typename T, int CT, int WK>
tc_status launch_few_rows(ExpertRowsArgs a, hipStream_t s) {
  a.nt = (int)ceil_div(a.NO, 16 * CT);
  const int64_t grid = (most_row_tiles(a.R, a.E, 16) * a.nt + 7) / 8 * 8;
  if (grid > kMostIndex / (64 * WK) * 2) return TC_ERR_UNSUPPORTED;
  expert_few_rows_kernel<T, CT, WK><<<dim3((unsigned)grid), dim3(64 * WK), 0, s>>>(a);
  return launched();
}

template <bool ACROSS>
tc_status run_rows(const ExpertRowsArgs& a, tc_type type, hipStream_t s) {
  return by_type(type, [&](auto t) {
    typedef decltype(t) T;
    constexpr int PER = Elem<T>::PER16;
    const bool whole = a.Q % PER == 0 && (!ACROSS || a.NO % PER == 0), thin = a.Q < PER || (ACROSS && a.NO < PER);
    const bool near = !prod_reaches({std::max(a.T, 1), a.Q, (int64_t)sizeof(T)}, (int64_t)1 << 32);
    const int most = sizeof(T) == 4 || thin ? 64 : whole && near && !ACROSS ? 256 : 128;
    const int side = expert_tile_side(most, compute_units(), [&](int b) { return expected_row_tiles(a.R, a.E, b) * (double)ceil_div(a.NO, b); });
    if constexpr (sizeof(T) == 2) {
      if constexpr (!ACROSS)
        if (side == 256) return launch_rows_tile<T, ACROSS, EMM_WHOLE, 256, 256, 2, 4, 2>(a, s);
      if (side == 128) return whole ? launch_rows_tile<T, ACROSS, EMM_WHOLE, 128, 128, 2, 4, 2>(a, s) : launch_rows_tile<T, ACROSS, EMM_ANY, 128, 128, 2, 4, 2>(a, s);
    }
    if (thin) return launch_rows_tile<T, ACROSS, EMM_NARROW, 64, 64, 2, 2, 2>(a, s);
    return whole ? launch_rows_tile<T, ACROSS, EMM_WHOLE, 64, 64, 2, 2, 2>(a, s) : launch_rows_tile<T, ACROSS, EMM_ANY, 64, 64, 2, 2, 2>(a, s);
  });
}

// The tile's side for the gradient of the weights.
int weights_side(bool f32, int64_t E, int64_t N, int64_t K) {
  const int per = f32 ? 4 : 8;
  return expert_tile_side(f32 || N < per || K < per ? 64 : 128, compute_units(), [&](int b) { return (double)E * (double)ceil_div(N, b) * (double)ceil_div(K, b); });
}
int64_t weights_ws(bool f32, int64_t R, int64_t E, int64_t N, int64_t K, int* parts) {
  *parts = R ? expert_weights_parts(f32, compute_units(), R, E, N, K, weights_side(f32, E, N, K)) : 1;
  return *parts > 1 ? *parts * E * N * K * 4 : 0;
}

template <typename T, typename TO, int MODE, bool LIST, int BM, int BN, int WM, int WN, int D>
tc_status launch_weights_list(ExpertWeightsArgs a, hipStream_t s) {
  a.mt = (int)ceil_div(a.N, BM);
  a.nt = (int)ceil_div(a.K, BN);
  const int64_t share = ceil_div((int64_t)a.mt * a.nt, 8);
  if (prod_reaches({share, 8, a.E}, kMostIndex / (64 * WM * WN) * 2)) return TC_ERR_UNSUPPORTED;
  const int64_t grid = 8 * share * a.E;
  expert_weights_kernel<T, TO, MODE, LIST, BM, BN, WM, WN, D><<<dim3((unsigned)grid, (unsigned)a.parts), dim3(64 * WM * WN), 0, s>>>(a);
  return launched();
}
template <typename T, typename TO, int MODE, int B, int WM, int WN, int D>
tc_status launch_weights(const ExpertWeightsArgs& a, hipStream_t s) {
  return a.row ? launch_weights_list<T, TO, MODE, true, B, B, WM, WN, D>(a, s) : launch_weights_list<T, TO, MODE, false, B, B, WM, WN, D>(a, s);
}
template <typename T, typename TO>
tc_status run_weights(const ExpertWeightsArgs& a, hipStream_t s) {
  constexpr int PER = Elem<T>::PER16;
  const bool whole = a.N % PER == 0 && a.K % PER == 0, thin = a.N < PER || a.K < PER;
  const int side = weights_side(sizeof(T) == 4, a.E, a.N, a.K);
  if constexpr (sizeof(T) == 2)
    if (side == 128) return whole ? launch_weights<T, TO, EMM_WHOLE, 128, 2, 4, 2>(a, s) : launch_weights<T, TO, EMM_ANY, 128, 2, 4, 2>(a, s);
  if (thin) return launch_weights<T, TO, EMM_NARROW, 64, 2, 2, 2>(a, s);
  return whole ? launch_weights<T, TO, EMM_WHOLE, 64, 2, 2, 2>(a, s) : launch_weights<T, TO, EMM_ANY, 64, 2, 2, 2>(a, s);
}

}  // namespace

extern "C" {

tc_status tc_embed(const void* LUT, const int32_t* Idx, void* O, int64_t E, int64_t D, int64_t T, float scale, tc_type type, void* hip_stream) {
  if (!known(type) || E <= 0 || D <= 0 || T < 0) return TC_ERR_SHAPE;
  if (!LUT || (T && (!Idx || !O))) return TC_ERR_NULL;
  if (T && (O == LUT || O == static_cast<const void*>(Idx))) return TC_ERR_ALIAS;
  if (misaligned(LUT) || misaligned(Idx) || misaligned(O)) return TC_ERR_ALIGN;
  if (E > kMostIndex + 1 || D > kMostRows || T > kMostIndex) return TC_ERR_UNSUPPORTED;
  if (T == 0) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  return took("embed:rows", by_type(type, [&](auto x) {
                typedef decltype(x) X;
                constexpr int V = Elem<X>::PER16;
                const int v = D < V ? 1 : V;
                const RowLanes rl = row_lanes(D, v);
                const EmbedArgs a{LUT, Idx, O, E, T, (int)D, rl.lpr, rl.cols, scale};
                return in_launches(ceil_div(T * a.cols, WG_THREADS / a.lpr), [&](dim3 n, int64_t at) {
                  if (v == V) embed_kernel<X, V><<<n, dim3(WG_THREADS), 0, s>>>(a, at);
                  else embed_kernel<X, 1><<<n, dim3(WG_THREADS), 0, s>>>(a, at);
                });
              }));
}

size_t tc_embed_grad_workspace_bytes(int64_t E, int64_t D, int64_t T) {
  if (E <= 0 || D <= 0 || T <= 0 || E >= kMostIndex || D > kMostRows || T > kMostRows || prod_reaches({T, D}, (int64_t)1 << 59)) return 0;
  return (size_t)embed_grad_plan(E, D, T).bytes;
}

tc_status tc_embed_grad(const void* dO, const int32_t* Idx, void* dLUT, int64_t E, int64_t D, int64_t T, float scale, int64_t pad, int32_t add, tc_type type,
                        tc_type grad_type, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!known(type) || (grad_type != type && grad_type != TC_F32) || E <= 0 || D <= 0 || T < 0) return TC_ERR_SHAPE;
  if (!dLUT || (T && (!dO || !Idx))) return TC_ERR_NULL;
  if (T && (dLUT == dO || dLUT == static_cast<const void*>(Idx))) return TC_ERR_ALIAS;
  if (workspace && (workspace == dO || workspace == static_cast<const void*>(Idx) || workspace == dLUT)) return TC_ERR_ALIAS;
  if (misaligned(dO) || misaligned(Idx) || misaligned(dLUT)) return TC_ERR_ALIGN;
  if (E >= kMostIndex || D > kMostRows || T > kMostRows || prod_reaches({std::max<int64_t>(T, 1), D}, (int64_t)1 << 59)) return TC_ERR_UNSUPPORTED;
  const EmbedGradPlan pl = embed_grad_plan(E, D, T);
  if (T && (!workspace || misaligned(workspace) || workspace_bytes < (size_t)pl.bytes)) return TC_ERR_WORKSPACE;
  if (T == 0 && add) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char* ws = static_cast<char*>(workspace);
  const auto run_by = [&](auto x, auto y, auto v) {
    typedef decltype(x) X;
    typedef decltype(y) Y;
    constexpr int V = decltype(v)::value;
    EmbedGradArgs a{};
    a.dO = dO; a.dLUT = dLUT; a.part = T ? ws + pl.part : nullptr;
    a.T = (int)T; a.E = (int)E; a.D = (int)D; a.scale = scale; a.add = add != 0;
    a.chunk = T < (add || D < EMBED_WIDE ? EMBED_FEW : EMBED_FEW_WRITTEN) ? EMBED_SMALL_CHUNK : EMBED_CHUNK;
    const int64_t chunks = ceil_div(T, a.chunk);
    a.lpr = 1;
    while (a.lpr < ceil_div(D, V) && a.lpr < WG_THREADS) a.lpr *= 2;
    a.token_wgs = (unsigned)ceil_div(chunks, WG_THREADS / a.lpr);
    int64_t rows = EMBED_FILL_ROWS;
    while (ceil_div(E, rows) > (int64_t)1 << 22) rows *= 2;  // (fewer than 2^32 threads)
    a.rows = (int)rows;
    const int64_t grid = a.token_wgs + (add ? 0 : ceil_div(E, rows));
    if (grid > kMostIndex / WG_THREADS * 2) return TC_ERR_UNSUPPORTED;
    if (T) {
      const tc_status st = sort_tokens(pl, Idx, T, E, pad, ws, &a.key, &a.order, s);
      if (st != TC_OK) return st;
    }
    const size_t lds = (size_t)(WG_THREADS / a.lpr) * (2 * a.chunk + 4) * 4;
    embed_grad_kernel<X, Y, V><<<dim3((unsigned)grid), dim3(WG_THREADS), lds, s>>>(a);
    if (chunks > 1) {
      const dim3 join((unsigned)ceil_div(chunks, WAVES_PER_WG), (unsigned)std::min<int64_t>(64, ceil_div(ceil_div(D, V), 64)));
      embed_join_kernel<X, Y, V><<<join, dim3(WG_THREADS), 0, s>>>(a);
    }
    return took(T <= SORT_SMALL ? "embed_grad:ranks" : "embed_grad:sort", launched());
  };
  const auto run = [&](auto x, auto y) {
    constexpr int V = std::min(Elem<decltype(x)>::PER16, Elem<decltype(y)>::PER16);
    return D < V ? run_by(x, y, std::integral_constant<int, 1>{}) : run_by(x, y, std::integral_constant<int, V>{});
  };
  return by_type(type, [&](auto x) { return grad_type == TC_F32 ? run(x, float{}) : run(x, x); });
}

size_t tc_route_workspace_bytes(int64_t T, int64_t E, int64_t k) {
  if (T <= 0 || E <= 0 || k <= 0 || k > E || E > ROUTE_MOST_E || k > ROUTE_MOST_K || T >= kMostTokens || prod_reaches({T, k}, kMostRows)) return 0;
  return (size_t)route_ws(T, E);
}

tc_status tc_route(const void* L, float* Wt, int32_t* Id, int32_t* Off, int32_t* Row, int32_t* Place, int64_t T, int64_t E, int64_t k, int32_t norm,
                   tc_type type, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!known(type) || T < 0 || E <= 0 || k <= 0 || k > E) return TC_ERR_SHAPE;
  if (!Off || (T && (!L || !Wt || !Id || !Row || !Place))) return TC_ERR_NULL;
  const void* out[] = {Wt, Id, Off, Row, Place, workspace};
  for (int i = 0; i < 6; i++) {
    if (out[i] && out[i] == L) return TC_ERR_ALIAS;
    for (int j = 0; j < i; j++)
      if (out[i] && out[i] == out[j]) return TC_ERR_ALIAS;
    if (i < 5 && misaligned(out[i])) return TC_ERR_ALIGN;
  }
  if (misaligned(L)) return TC_ERR_ALIGN;
  if (E > ROUTE_MOST_E || k > ROUTE_MOST_K || prod_reaches({std::max<int64_t>(T, 1), k}, kMostRows) || T >= kMostTokens) return TC_ERR_UNSUPPORTED;
  const int64_t need = route_ws(T, E);
  const bool tiles = need && workspace && !misaligned(workspace) && workspace_bytes >= (size_t)need;
  if (!tiles && T > ROUTE_MOST_ALONE) return TC_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  RouteArgs a{L, Wt, Id, Off, Row, Place, tiles ? static_cast<int*>(workspace) : nullptr, (int)T, (int)E, (int)k, norm != 0, bits_of(E),
              tiles ? (int)ceil_div(T, ROUTE_TOKENS) : 1, 0, tiles ? ROUTE_TOKENS : ROUTE_MOST_ALONE};
  a.summed = a.tiles > ROUTE_DIRECT_TILES;
  const size_t bins = (size_t)4 << a.bits;
  return by_type(type, [&](auto x) {
    return by_lanes(E, k, [&](auto g, auto v) {
      typedef decltype(x) X;
      route_kernel<X, g.value, v.value><<<dim3((unsigned)a.tiles), dim3(WG_THREADS), a.count ? bins : bins * (1 + WAVES_PER_WG), s>>>(a);
      if (!a.count) return took("route:one", launched());
      if (a.summed) sort_sum_kernel<<<dim3(1u << a.bits), dim3(WG_THREADS), 0, s>>>(a.count, a.tiles);
      route_place_kernel<<<dim3((unsigned)a.tiles), dim3(WG_THREADS), bins * (1 + WAVES_PER_WG), s>>>(a);
      return took("route:tiles", launched());
    });
  });
}

tc_status tc_route_grad(const void* L, const int32_t* Id, const float* dWt, void* dL, int64_t T, int64_t E, int64_t k, int32_t norm, tc_type type,
                        void* hip_stream) {
  if (!known(type) || T < 0 || E <= 0 || k <= 0 || k > E) return TC_ERR_SHAPE;
  if (T && (!L || !Id || !dWt || !dL)) return TC_ERR_NULL;
  if (T && (dL == L || dL == static_cast<const void*>(Id) || dL == static_cast<const void*>(dWt))) return TC_ERR_ALIAS;
  if (misaligned(L) || misaligned(Id) || misaligned(dWt) || misaligned(dL)) return TC_ERR_ALIGN;
  if (E > ROUTE_MOST_E || k > ROUTE_MOST_K || prod_reaches({std::max<int64_t>(T, 1), k}, kMostRows)) return TC_ERR_UNSUPPORTED;
  if (T == 0) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const RouteGradArgs a{L, Id, dWt, dL, (int)T, (int)E, (int)k, norm != 0};
  return by_type(type, [&](auto x) {
    return by_lanes(E, 1, [&](auto g, auto v) {
      typedef decltype(x) X;
      return took("route_grad:rows", in_launches(ceil_div(T, WG_THREADS / g.value), [&](dim3 n, int64_t at) {
                    route_grad_kernel<X, g.value, v.value><<<n, dim3(WG_THREADS), 0, s>>>(a, at);
                  }));
    });
  });
}

tc_status tc_expert_mm(const void* X, const void* W, const int32_t* Off, const int32_t* Row, void* Y, int64_t T, int64_t R, int64_t E, int64_t N, int64_t K,
                       int32_t relu, tc_type type, void* hip_stream) {
  if (!known(type) || T < 0 || R < 0 || E <= 0 || N <= 0 || K <= 0 || (R && !Row && T != R)) return TC_ERR_SHAPE;
  if (!W || !Off || (R && (!Y || (T && !X)))) return TC_ERR_NULL;
  if (R && (Y == X || Y == W || Y == static_cast<const void*>(Off) || Y == static_cast<const void*>(Row))) return TC_ERR_ALIAS;
  if (misaligned(X) || misaligned(W) || misaligned(Off) || misaligned(Row) || misaligned(Y)) return TC_ERR_ALIGN;
  if (T >= kMostRows || R >= kMostRows || E >= kMostRows || N >= kMostWidth || K >= kMostWidth) return TC_ERR_UNSUPPORTED;
  if (R == 0) return TC_OK;
  const ExpertRowsArgs a{X, W, Y, nullptr, Off, Row, (int)R, (int)T, (int)E, (int)K, (int)N, 0, relu != 0};
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (expert_few_rows(type == TC_F32, K % (type == TC_F32 ? 4 : 8) == 0, compute_units(), R, E, N))
    return took("expert_mm:rows", by_type(type, [&](auto t) { return launch_few_rows<decltype(t), 2, 4>(a, s); }));
  return took("expert_mm:tile", run_rows<false>(a, type, s));
}

tc_status tc_expert_mm_grad_x(const void* dY, const void* W, const int32_t* Off, const void* gate, void* dX, int64_t R, int64_t E, int64_t N, int64_t K,
                              tc_type type, void* hip_stream) {
  if (!known(type) || R < 0 || E <= 0 || N <= 0 || K <= 0) return TC_ERR_SHAPE;
  if (!W || !Off || (R && (!dY || !dX))) return TC_ERR_NULL;
  if (R && (dX == dY || dX == W || dX == static_cast<const void*>(Off) || dX == gate)) return TC_ERR_ALIAS;
  if (misaligned(dY) || misaligned(W) || misaligned(Off) || misaligned(gate) || misaligned(dX)) return TC_ERR_ALIGN;
  if (R >= kMostRows || E >= kMostRows || N >= kMostWidth || K >= kMostWidth) return TC_ERR_UNSUPPORTED;
  if (R == 0) return TC_OK;
  const ExpertRowsArgs a{dY, W, dX, gate, Off, nullptr, (int)R, (int)R, (int)E, (int)N, (int)K, 0, 0};
  return took("expert_mm_grad_x:tile", run_rows<true>(a, type, static_cast<hipStream_t>(hip_stream)));
}

size_t tc_expert_mm_grad_w_workspace_bytes(int64_t R, int64_t E, int64_t N, int64_t K) {
  if (R <= 0 || E <= 0 || N <= 0 || K <= 0 || R >= kMostRows || E >= kMostRows || N >= kMostWidth || K >= kMostWidth || prod_reaches({E, N, K}, (int64_t)1 << 50)) return 0;
  int parts;
  return (size_t)std::max(weights_ws(true, R, E, N, K, &parts), weights_ws(false, R, E, N, K, &parts));
}

tc_status tc_expert_mm_grad_w(const void* dY, const void* X, const int32_t* Off, const int32_t* Row, void* dW, int64_t T, int64_t R, int64_t E, int64_t N,
                              int64_t K, int32_t add, tc_type type, tc_type grad_type, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!known(type) || (grad_type != type && grad_type != TC_F32) || T < 0 || R < 0 || E <= 0 || N <= 0 || K <= 0 || (R && !Row && T != R)) return TC_ERR_SHAPE;
  if (!Off || !dW || (R && (!dY || (T && !X)))) return TC_ERR_NULL;
  if (dW == dY || dW == X || dW == static_cast<const void*>(Off) || dW == static_cast<const void*>(Row)) return TC_ERR_ALIAS;
  if (workspace && (workspace == dY || workspace == X || workspace == dW || workspace == static_cast<const void*>(Off) || workspace == static_cast<const void*>(Row)))
    return TC_ERR_ALIAS;
  if (misaligned(dY) || misaligned(X) || misaligned(Off) || misaligned(Row) || misaligned(dW) || misaligned(workspace)) return TC_ERR_ALIGN;
  if (T >= kMostRows || R >= kMostRows || E >= kMostRows || N >= kMostWidth || K >= kMostWidth) return TC_ERR_UNSUPPORTED;
  if (prod_reaches({E, N, K}, (int64_t)1 << 50)) return TC_ERR_UNSUPPORTED;
  if (R == 0 && add) return TC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  ExpertWeightsArgs a{dY, X, dW, Off, Row, (int)R, (int)T, (int)E, (int)N, (int)K, 0, 0, add != 0, 1};
  int parts;
  const int64_t need = weights_ws(type == TC_F32, R, E, N, K, &parts);
  return by_type(type, [&](auto t) {
    typedef decltype(t) T_;
    const auto join_to = [&](auto o) {
      a.dW = workspace;
      a.parts = parts;
      a.add = 0;
      const tc_status st = run_weights<T_, float>(a, s);
      if (st != TC_OK) return st;
      const int64_t n = E * N * K, grid = ceil_div(n, 4 * WG_THREADS);
      expert_weights_join_kernel<decltype(o)><<<dim3((unsigned)grid), dim3(WG_THREADS), 0, s>>>(static_cast<const float*>(workspace), dW, n, parts, add != 0);
      return took("expert_mm_grad_w:parts", launched());
    };
    if (need && workspace && workspace_bytes >= (size_t)need && ceil_div(E * N * K, 4 * WG_THREADS) <= kMostIndex / WG_THREADS * 2)
      return grad_type == TC_F32 ? join_to(float{}) : join_to(t);
    return took("expert_mm_grad_w:tile", grad_type == TC_F32 ? run_weights<T_, float>(a, s) : run_weights<T_, T_>(a, s));
  });
}

tc_status tc_expert_sum(const void* Y, const float* Wt, const int32_t* Place, void* O, int64_t T, int64_t R, int64_t k, int64_t N, tc_type type,
                        void* hip_stream) {
  if (!known(type) || T < 0 || R < 0 || k <= 0 || N <= 0) return TC_ERR_SHAPE;
  if (T && (!Place || !O || (R && !Y))) return TC_ERR_NULL;
  if (T && (O == Y || O == static_cast<const void*>(Wt) || O == static_cast<const void*>(Place))) return TC_ERR_ALIAS;
  if (misaligned(Y) || misaligned(Wt) || misaligned(Place) || misaligned(O)) return TC_ERR_ALIGN;
  if (T > kMostRows || R > kMostRows || N > kMostRows || k > kMostRows) return TC_ERR_UNSUPPORTED;
  if (T == 0) return TC_OK;
  return took("expert_sum:rows", by_type(type, [&](auto x) {
                typedef decltype(x) X;
                constexpr int V = Elem<X>::PER16;
                const RowLanes rl = row_lanes(N, N < V ? 1 : V);
                const ExpertSumArgs a{Y, Wt, Place, O, T, R, (int)N, (int)k, rl.lpr, rl.cols};
                hipStream_t s = static_cast<hipStream_t>(hip_stream);
                return in_launches(ceil_div(T * a.cols, WG_THREADS / a.lpr), [&](dim3 n, int64_t at) {
                  const dim3 b(WG_THREADS);
                  if (N < V) expert_sum_kernel<X, 1, 4><<<n, b, 0, s>>>(a, at);
                  else if (k == 1) expert_sum_kernel<X, V, 1><<<n, b, 0, s>>>(a, at);
                  else if (k == 2) expert_sum_kernel<X, V, 2><<<n, b, 0, s>>>(a, at);
                  else if (k <= 4) expert_sum_kernel<X, V, 4><<<n, b, 0, s>>>(a, at);
                  else expert_sum_kernel<X, V, 8><<<n, b, 0, s>>>(a, at);
                });
              }));
}

tc_status tc_expert_sum_grad(const void* dO, const void* Y, const float* Wt, const int32_t* Place, void* dY, float* dWt, int64_t T, int64_t R, int64_t k,
                             int64_t N, tc_type type, void* hip_stream) {
  if (!known(type) || T < 0 || R < 0 || k <= 0 || N <= 0) return TC_ERR_SHAPE;
  if (T && (!dO || !Wt || !Place || !dWt || (R && (!Y || !dY)))) return TC_ERR_NULL;
  const void* in[] = {dO, Y, Wt, Place};
  for (const void* i : in) {
    if (i && (dY == i || dWt == i)) return TC_ERR_ALIAS;
    if (misaligned(i)) return TC_ERR_ALIGN;
  }
  if (dY && dY == static_cast<const void*>(dWt)) return TC_ERR_ALIAS;
  if (misaligned(dY) || misaligned(dWt)) return TC_ERR_ALIGN;
  if (T > kMostRows || R > kMostRows || N > kMostRows || k > kMostRows) return TC_ERR_UNSUPPORTED;
  if (T == 0) return TC_OK;
  return took("expert_sum_grad:rows", by_type(type, [&](auto x) {
                typedef decltype(x) X;
                const ExpertSumGradArgs a{dO, Y, Wt, Place, dY, dWt, T, R, (int)N, (int)k};
                hipStream_t s = static_cast<hipStream_t>(hip_stream);
                constexpr int V = Elem<X>::PER16;
                return in_launches(ceil_div(T, WAVES_PER_WG), [&](dim3 n, int64_t at) {
                  const dim3 b(WG_THREADS);
                  if (N < V) expert_sum_grad_kernel<X, 1, 4><<<n, b, 0, s>>>(a, at);
                  else if (k <= 2) expert_sum_grad_kernel<X, V, 2><<<n, b, 0, s>>>(a, at);
                  else if (k <= 4) expert_sum_grad_kernel<X, V, 4><<<n, b, 0, s>>>(a, at);
                  else expert_sum_grad_kernel<X, V, 8><<<n, b, 0, s>>>(a, at);
                });
              }));
}

}  // extern "C"
