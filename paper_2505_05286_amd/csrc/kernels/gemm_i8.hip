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

// A step of 64 codes moves and multiplies the bytes of a step of 32 bf16 values in as many cycles, so a plan is that of
// the bf16 product of half the K.
GemmI8Plan gemm_i8_plan(int M, int N, int kt, bool swiglu) {
  const GemmPlan b = gemm_plan(M, swiglu ? 2 * N : N, kt * 32, 8, swiglu, true);
  GemmI8Plan p;
  p.tm = b.tm;
  p.nw = b.nw;
  p.wv = b.wv;
  p.once = b.once;
  p.splits = b.splits;
  p.piece = b.k_chunk / 32;
  return p;
}

int64_t gemm_i8_ws_bytes(int M, int N, int K) {
  int64_t need = 0;
  for (bool sw : {false, true}) {
    if (M == 0 || (sw && N % 2)) continue;
    const GemmI8Plan p = gemm_i8_plan(M, sw ? N / 2 : N, (K + 63) / 64, sw);
    if (p.splits > 1) need = std::max(need, (int64_t)p.splits * M * N * 4);
  }
  return need;
}

hipError_t gemm_i8_launch(const GemmI8Args& a, int epi, hipStream_t st) {
  return gemm_i8_run(a, epi, gemm_i8_plan(a.M, a.N, a.kt, epi == EPI_SWIGLU), st);
}

}  // namespace hxf
