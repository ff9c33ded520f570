// Dispatch of the product of 8-bit codes: the choice of tile and K split, the sum of the pieces.
#include <algorithm>

#include "gemm_i8.hpp"

namespace hxf {

namespace {

// The pieces' sums and the epilogue, four columns a thread.  Sums of whole numbers: exact in any order.
template <int EPI>
__global__ __launch_bounds__(256) void gemm_i8_join_kernel(GemmI8Args a, int S) {
  constexpr bool SW = EPI == EPI_SWIGLU;
  const int quads = (a.N + 3) / 4, n_all = SW ? 2 * a.N : a.N;
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= (int64_t)a.M * quads) return;
  const int row = (int)(idx / quads), col = (int)(idx % quads) * 4;
  const size_t MN = (size_t)a.M * n_all;
  const bool whole = col + 3 < a.N;
  auto sum = [&](int c) {
    const int32_t* p = a.partial + (size_t)row * n_all + c;
    i32x4 s = {0, 0, 0, 0};
    if (whole) {
      for (int z = 0; z < S; ++z) s += load4<i32x4>(p + z * MN);
    } else {
      for (int z = 0; z < S; ++z)
        for (int e = 0; e < 4 && col + e < a.N; ++e) s[e] += p[z * MN + e];
    }
    return s;
  };
  const float sa = a.sa[row];
  f32x4 y = scaled(sum(col), sa, load_scales(a.sb, col, a.N));
  if constexpr (SW) {
    const f32x4 u = scaled(sum(a.N + col), sa, load_scales(a.sb2, col, a.N));
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = swiglu(y[e], u[e]);
  }
  store4<EPI>(a, row, col, y);
}

template <int EPI>
hipError_t join(const GemmI8Args& a, int S, hipStream_t st) {
  const int64_t n = (int64_t)a.M * ((a.N + 3) / 4);
  hipLaunchKernelGGL(gemm_i8_join_kernel<EPI>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, S);
  return hipGetLastError();
}

}  // namespace

hipError_t gemm_i8_run(GemmI8Args a, int epi, const GemmI8Plan& p, hipStream_t st) {
  a.piece = p.piece;
  if (p.thin) return gemm_i8_thin(a, epi, p, st);
  if (p.splits > 1) {
    if (hipError_t e = epi == EPI_SWIGLU ? gemm_i8_split_swiglu(a, p, st) : gemm_i8_split(a, p, st)) return e;
    switch (epi) {
      case EPI_BF16: return join<EPI_BF16>(a, p.splits, st);
      case EPI_RESID: return join<EPI_RESID>(a, p.splits, st);
      case EPI_SWIGLU: return join<EPI_SWIGLU>(a, p.splits, st);
      default: return join<EPI_F32>(a, p.splits, st);
    }
  }
  switch (epi) {
    case EPI_BF16: return gemm_i8_bf16(a, p, st);
    case EPI_RESID: return gemm_i8_resid(a, p, st);
    case EPI_SWIGLU: return gemm_i8_swiglu(a, p, st);
    default: return gemm_i8_f32(a, p, st);
  }
}

namespace {

// Estimated time (us) of a plan.  A step of 64 of K takes a CU the longer of its matrix instructions' time (i0 + i1 per
// 16 tiles) and its codes' way into the CU (fetch, by rows of tiles, per 16 KB of weights and, times a_share, of
// activations); a workgroup then stores its outputs (store us per KB; SwiGLU as if of `gated` bytes a value).  A CU runs
// `resident` workgroups at once, which share its time but wait each by itself (start).  The weights come at tb_s at best.
//
// Fitted to 140,000 launches of 3,400 shapes (1 to 3,000 rows, half of them projections of d 4096-8192), weights not
// in the caches, in graphs: the choice is 2.4% slower than the best plan on average, 27% at the worst hundredth.
struct WideCost {
  float t0, start, store, i0, i1, fetch[3], a_share, tb_s, gated;
  int resident;
};
constexpr WideCost kNarrowOnce{2.22f, 0.724f, 0.034f, 0.0347f, 0.0734f, {0.373f, 0.33f, 0.3f}, 0.782f, 5.95f, 6.53f, 1};   // 32 columns a wavefront, one row of tiles
constexpr WideCost kNarrowLow{3.15f, 0.f, 0.0436f, 0.11f, 0.0208f, {0.35f, 0.282f, 0.224f}, 0.599f, 6.f, 5.43f, 3};   // 32 columns, up to 4 row tiles a workgroup
constexpr WideCost kNarrow{3.39f, 0.f, 0.0422f, 0.0287f, 0.0515f, {0.209f, 0.203f, 0.173f}, 1.57f, 4.22f, 6.3f, 2};   // 32 columns, more
constexpr WideCost kCols64Once{2.97f, 0.f, 0.0286f, 0.f, 0.047f, {0.333f, 0.33f, 0.3f}, 0.838f, 6.11f, 9.58f, 1};   // 64 columns, one row of tiles
constexpr WideCost kCols64Low{3.22f, 0.f, 0.0389f, 0.053f, 0.044f, {0.35f, 0.151f, 0.13f}, 3.89f, 4.12f, 4.95f, 2};   // 64 columns, up to 7 row tiles: two workgroups a CU
constexpr WideCost kCols64{0.f, 3.87f, 0.031f, 0.0211f, 0.0435f, {0.35f, 0.304f, 0.277f}, 0.747f, 6.f, 6.02f, 1};   // 64 columns, more
constexpr WideCost kEight{0.f, 3.08f, 0.0239f, 0.267f, 0.0276f, {0.266f, 0.254f, 0.23f}, 1.07f, 3.71f, 5.94f, 1};   // eight wavefronts of 64 columns
// Pieces of K are joined by a launch of its own; a plan with one is only taken where it saves a twentieth
constexpr float kJoin = 2.77f, kJoinGated = 1.7f, kJoinMb = 0.302f, kSplitBias = 1.06f;

// The kernel that joins K inside the workgroup: the wait for a first step, a step, a CU's 100 KB of codes, the weights,
// a workgroup's rest
struct ThinCost {
  int tm, nw, wv;
  float t0, first, step, kb, tb_s, rest;
};
constexpr ThinCost kThin[] = {{1, 1, 4, 2.7f, 0.785f, 0.139f, 2.31f, 5.96f, 0.926f}, {1, 2, 16, 1.78f, 4.47f, 0.0909f, 2.35f, 5.81f, 2.89f}, {2, 1, 16, 2.87f, 3.14f, 0.f, 2.53f, 5.44f, 1.95f},
                              {2, 2, 8, 1.86f, 0.39f, 0.627f, 2.16f, 5.57f, 2.63f}, {4, 1, 8, 1.82f, 3.37f, 0.176f, 2.36f, 7.08f, 2.62f}, {4, 2, 8, 0.f, 6.04f, 0.247f, 2.57f, 5.67f, 4.08f}};

struct Choice {
  int M, N, kt, row_tiles, bytes;   // bytes: of an output value, its old one read included
  bool gated;
  float mb;   // of codes of the weights
  float best;
  GemmI8Plan p;

  void wide(const WideCost& c, int tm, int nw, int wv, bool once) {
    const int tiles_m = (row_tiles + tm - 1) / tm, cols = 16 * (gated ? nw / 2 : nw) * wv;
    const int64_t tiles = (int64_t)tiles_m * ((N + cols - 1) / cols);
    const float unit = tm * nw * wv / 16.f, ways = (nw * wv + c.a_share * tm) / 16.f;
    const float step = std::max(c.i0 + c.i1 * unit, c.fetch[tiles_m == 1 ? 0 : tiles_m <= 3 ? 1 : 2] * ways);
    for (int s = 1; s <= 8 && (s == 1 || (kt >= 12 * s && tiles * s <= 256)); ++s) {
      const int piece = ((kt + s - 1) / s + 1) / 2 * 2;
      if (s > 1 && (kt + piece - 1) / piece != s) continue;
      const float a_value = s > 1 ? (gated ? 8.f : 4.f) : gated ? c.gated : bytes;
      const float one = std::min(piece, kt) * step + c.store * 0.256f * tm * cols / 16 * a_value;
      const int64_t per_cu = (tiles * s + 255) / 256;
      float t = std::max(per_cu * one, ((per_cu + c.resident - 1) / c.resident) * (one + c.start));
      t = c.t0 + std::max(t, mb / c.tb_s);
      if (s > 1)
        t = kSplitBias * (t + kJoin + (gated ? kJoinGated : 0.f) + kJoinMb * s * 4e-6f * M * (gated ? 2.f : 1.f) * N);
      take(t, tm, nw, wv, once, false, s, piece);
    }
  }
  void thin(const ThinCost& c) {
    const int tiles = (N + 16 * c.nw - 1) / (16 * c.nw);
    const float kb = kt * (c.nw * (gated ? 2 : 1) + 0.5f * c.tm);
    const float t = c.t0 + std::max({c.first + c.step * ((kt + c.wv - 1) / c.wv),
                                     (tiles + 255) / 256 * (kb * 0.01f * c.kb + c.rest), mb / c.tb_s});
    take(t, c.tm, c.nw, c.wv, false, true, 1, (kt + 1) / 2 * 2);
  }
  void take(float t, int tm, int nw, int wv, bool once, bool thin, int splits, int piece) {
    if (best != 0 && t >= best) return;
    best = t;
    p.tm = tm;
    p.nw = nw;
    p.wv = wv;
    p.once = once;
    p.thin = thin;
    p.splits = splits;
    p.piece = piece;
  }
};

}  // namespace

// All plans that can be the best for their rows: heights that leave fewer rows of tiles than the next lower one.
GemmI8Plan gemm_i8_plan(int M, int N, int kt, int epi) {
  Choice c{};
  c.M = M;
  c.N = N;
  c.kt = kt;
  c.row_tiles = (M + 15) / 16;
  c.bytes = epi == EPI_RESID ? 8 : epi == EPI_F32 ? 4 : 2;
  c.gated = epi == EPI_SWIGLU;
  c.mb = (c.gated ? 2e-6f : 1e-6f) * N * kt * 64;
  const int rt = c.row_tiles;
  if (rt <= 4)
    for (const ThinCost& t : kThin)
      if (t.tm == (rt <= 2 ? rt : 4)) c.thin(t);
  if (rt <= 8) {
    const int tm = rt <= 2 ? rt : rt <= 4 ? 4 : 8;
    c.wide(kNarrowOnce, tm, 2, 4, true);
    c.wide(kCols64Once, rt > 4 && rt <= 6 ? 6 : tm, 4, 4, true);
  }
  auto fewer = [&](int tm, int first) { return tm == first || (rt + tm - 1) / tm < (rt + tm - 2) / (tm - 1); };
  for (int tm = 3; tm <= 12; ++tm)
    if (rt > tm ? fewer(tm, 3) : rt > 8 && rt == tm) c.wide(tm <= 4 ? kNarrowLow : kNarrow, tm, 2, 4, false);
  for (int tm = 4; tm <= 16; ++tm) {
    if (rt > tm && fewer(tm, 4)) c.wide(tm <= 7 ? kCols64Low : kCols64, tm, 4, 4, false);
    if (rt <= tm && rt > 8 && tm % 2 == 0 && rt + 2 > tm) c.wide(kCols64Once, tm, 4, 4, true);
  }
  if (rt > 8)
    for (int tm = 5; tm <= 9; ++tm)
      if (fewer(tm, 5)) c.wide(kEight, tm, 4, 8, false);
  return c.p;
}

namespace {

int64_t partial_bytes(const GemmI8Plan& p, int M, int N, int epi) {
  return p.splits > 1 ? (int64_t)p.splits * M * N * (epi == EPI_SWIGLU ? 8 : 4) : 0;
}

}  // namespace

int64_t gemm_i8_ws_bytes(int M, int N, int K) {
  if (M == 0) return 0;
  int64_t need = 0;
  for (int epi : {EPI_BF16, EPI_RESID, EPI_F32, EPI_SWIGLU}) {
    if (epi == EPI_SWIGLU && N % 2) continue;
    const int n = epi == EPI_SWIGLU ? N / 2 : N;
    need = std::max(need, partial_bytes(gemm_i8_plan(M, n, (K + 63) / 64, epi), M, n, epi));
  }
  return need;
}

hipError_t gemm_i8_launch(const GemmI8Args& a, int epi, int64_t ws_bytes, hipStream_t st) {
  const GemmI8Plan p = gemm_i8_plan(a.M, a.N, a.kt, epi);
  if (ws_bytes < partial_bytes(p, a.M, a.N, epi)) return hipErrorOutOfMemory;
  return gemm_i8_run(a, epi, p, st);
}

}  // namespace hxf
