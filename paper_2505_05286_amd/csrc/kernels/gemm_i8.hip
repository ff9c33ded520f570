// Dispatch of the product of 8-bit codes: the choice of tile and K split, the sum of the pieces.
#include <algorithm>

#include "gemm_i8.hpp"

namespace hxf {

namespace {

// The pieces' sums and the epilogue, four columns a thread: memory is the bound (256 x 8192 of four pieces into the
// residual 10 us, 5 TB/s).  Sums of whole numbers: exact in any order.
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
    y = swiglu(y, scaled(sum(a.N + col), sa, load_scales(a.sb2, col, a.N)));
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
// Fitted to 190,000 launches of 4,900 shapes (1 to 3,000 rows, half of them projections of d 4096-8192), weights not
// in the caches, in graphs: the choice is 2.2% slower than the best plan on average, 28% at the worst hundredth.  Among the
// worst are some batches of model shapes, where two estimates lie closer than the times (us, the choice and the best plan):
// 1-16 rows of 28672 x 4096 SwiGLU 25.7 / 20.8, 17-32 of 8192 x 28672 45 / 39, 82 68 / 48, 130 of 4096 x 4096 15.0 / 11.5,
// 192 14.0 / 11.7, 440 of 5120 x 27648 108 / 72.
struct WideCost {
  float t0, start, store, i0, i1, fetch[3], a_share, tb_s, gated;
  int resident;
};
// 32 columns a wavefront, one row of tiles
constexpr WideCost kNarrowOnce{2.17f, 0.753f, 0.0348f, 0.192f, 0.033f, {0.37f, 0.33f, 0.3f}, 0.792f, 5.95f, 6.74f, 1};
// 32 columns, up to 4 row tiles a workgroup
constexpr WideCost kNarrowLow{3.22f, 0.f, 0.0426f, 0.112f, 0.0194f, {0.35f, 0.278f, 0.226f}, 0.64f, 6.f, 5.37f, 3};
// 32 columns, more
constexpr WideCost kNarrow{3.4f, 0.f, 0.0425f, 0.0314f, 0.0505f, {0.209f, 0.204f, 0.173f}, 1.55f, 4.24f, 6.25f, 2};
// 64 columns, one row of tiles
constexpr WideCost kCols64Once{2.94f, 0.f, 0.0299f, 0.f, 0.0449f, {0.335f, 0.33f, 0.3f}, 0.781f, 6.08f, 9.39f, 1};
// 64 columns, up to 7 row tiles: two workgroups a CU
constexpr WideCost kCols64Low{3.27f, 0.f, 0.0392f, 0.12f, 0.0335f, {0.35f, 0.135f, 0.115f}, 4.7f, 4.1f, 4.94f, 2};
// 64 columns, 8 to 10
constexpr WideCost kCols64{0.f, 4.11f, 0.0292f, 0.0925f, 0.036f, {0.35f, 0.133f, 0.115f}, 2.19f, 6.f, 5.68f, 1};
// 64 columns, more
constexpr WideCost kCols64High{2.27f, 2.77f, 0.0301f, 0.f, 0.0413f, {0.35f, 0.33f, 0.3f}, 0.5f, 6.f, 4.42f, 1};
// eight wavefronts of 64 columns
constexpr WideCost kEight{0.f, 3.16f, 0.0241f, 0.263f, 0.0276f, {0.275f, 0.255f, 0.237f}, 0.795f, 3.68f, 5.79f, 1};
// Pieces of K are joined by a launch of its own; a plan with one is only taken where it saves a twentieth
constexpr float kJoin = 2.71f, kJoinGated = 1.66f, kJoinMb = 0.308f, kSplitBias = 1.06f;
// and only where all pieces of all tiles run at once, one a CU
constexpr int kMaxPieces = 8, kPieceSteps = 12;
constexpr int kMaxTile = 9 * 4 * 8 * 256;   // the most sums a workgroup holds, both halves of a gated one counted

// The kernel that joins K inside the workgroup: the wait for a first step, a step, a CU's 100 KB of codes, the weights,
// a workgroup's rest
struct ThinCost {
  int tm, nw, wv;
  float t0, first, step, kb, tb_s, rest;
};
constexpr ThinCost kThin[] = {
    {1, 1, 4, 2.66f, 0.615f, 0.0423f, 2.32f, 5.96f, 0.94f},
    {1, 2, 16, 1.74f, 4.44f, 0.129f, 2.38f, 5.86f, 2.9f},
    {2, 1, 16, 2.8f, 3.19f, 0.f, 2.54f, 5.44f, 2.01f},
    {2, 2, 8, 1.74f, 2.58f, 0.44f, 2.35f, 5.58f, 2.39f},
    {4, 1, 8, 1.95f, 3.18f, 0.203f, 2.36f, 7.28f, 2.52f},
    {4, 2, 8, 0.f, 5.55f, 0.56f, 2.58f, 5.68f, 3.97f}};

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
    for (int s = 1; s <= kMaxPieces && (s == 1 || (kt >= kPieceSteps * s && tiles * s <= kCus)); ++s) {
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
    if (rt > tm && fewer(tm, 4)) c.wide(tm <= 7 ? kCols64Low : tm <= 10 ? kCols64 : kCols64High, tm, 4, 4, false);
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

// For every plan of at most these sizes.  What one plan needs goes up and down with its rows (4096 x 14336: 14.7 MB at 448
// rows, 8.4 at 256, none at 2080), and a caller keeps one buffer for batches of any size up to its largest.
int64_t gemm_i8_ws_bytes(int M, int N, int K) {
  const int pieces = std::min(kMaxPieces, (K + 63) / 64 / kPieceSteps);
  return pieces < 2 ? 0 : std::min((int64_t)pieces * M * N * 4, (int64_t)kCus * kMaxTile * 4);
}

hipError_t gemm_i8_launch(const GemmI8Args& a, int epi, int64_t ws_bytes, hipStream_t st) {
  const GemmI8Plan p = gemm_i8_plan(a.M, a.N, a.kt, epi);
  if (ws_bytes < partial_bytes(p, a.M, a.N, epi)) return hipErrorOutOfMemory;
  return gemm_i8_run(a, epi, p, st);
}

}  // namespace hxf
