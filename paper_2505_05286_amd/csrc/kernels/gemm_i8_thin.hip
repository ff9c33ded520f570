// The product of 8-bit codes for one to four row tiles (a decode step of a few sequences) in one launch: the wavefronts
// of a workgroup share out K and join their sums in LDS.
//
// The weights' bytes are the bound, and below some tens of MB the latency of the first loads and of a second launch.
// With 16 or 32 columns a workgroup an output of a few thousand fills the chip without cutting K across workgroups,
// whose partials take a launch of their own to join (a call in a graph, us, this kernel and the other's best plan, with cut
// K: 1 x 6144 x 4096 8.0 / 10.0, 64 rows 10.8 / 13.8; 1 x 4096 x 14336 13.5 / 15.5; 1 x 8192 x 28672 39 / 38.2, 6.0 TB/s).
// But every workgroup reads all activations itself, and with a gate twice the weights wait in two rounds of workgroups: there
// the other kernel is ahead, while the plan's estimate, a few percent off, still takes this one (17 and 32 rows of 8192 x 28672
// 45 / 39; 1 to 16 rows of 28672 x 4096 SwiGLU 25.7 / 20.8, whole K; from 33 rows of 8192 x 28672 on it takes the other).
#include "gemm_i8.hpp"

namespace hxf {

namespace {

// A workgroup owns 16 HALF output columns and all rows (TM tiles of 16); wavefront w multiplies the steps (64 of K)
// w, w + WV, .. of both operands, which go straight to registers, R steps ahead.  Steps past the end are zeros that
// no memory is read for.
template <int TM, int HALF, int R, int EPI, int WV>
__global__ __launch_bounds__(64 * WV) void gemm_i8_thin_kernel(GemmI8Args a) {
  constexpr bool SW = EPI == EPI_SWIGLU;
  constexpr int NW = SW ? 2 * HALF : HALF;
  __shared__ __attribute__((aligned(16))) i32x4 part[WV][TM * NW][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = blockIdx.x * 16 * HALF, b_tiles = (a.N + 15) / 16, bt = c0 / 16;
  const uint32_t b_bytes = (uint32_t)min(HALF, b_tiles - bt) * a.kt * 1024;
  const rsrc_t ra = make_rsrc(a.A, (uint32_t)((a.M + 15) / 16) * a.kt * 1024);
  const rsrc_t rb0 = make_rsrc(a.B + (size_t)bt * a.kt * 1024, b_bytes);
  const rsrc_t rb1 = SW ? make_rsrc(a.B2 + (size_t)bt * a.kt * 1024, b_bytes) : rb0;
  uint4 fa[R][TM], fb[R][NW];
  auto load = [&](auto rc, int s) __attribute__((always_inline)) {
    constexpr int r = decltype(rc)::value;
    const int k = w + s * WV, past = k < a.kt ? 0 : kOutOfRange, at = min(k, a.kt - 1) * 1024;
#pragma unroll
    for (int j = 0; j < NW; ++j)
      fb[r][j] = buf_load16<2>(j < HALF ? rb0 : rb1, (lane * 16 + (j % HALF) * a.kt * 1024) | past, at);
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[r][i] = buf_load16(ra, (lane * 16 + i * a.kt * 1024) | past, at);
  };
  i32x4 acc[TM][NW];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < NW; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const int n = (a.kt + WV - 1) / WV;
  static_for<R>([&](auto rc) { load(rc, decltype(rc)::value); });
  for (int s = 0; s < n; s += R) {
    static_for<R>([&](auto rc) {
      constexpr int r = decltype(rc)::value;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < NW; ++j) acc[i][j] = mfma16x16x64(fb[r][j], fa[r][i], acc[i][j]);
      load(rc, s + R + r);
    });
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < NW; ++j) part[w][i * NW + j][lane] = acc[i][j];
  __syncthreads();
  // reads in flight: with all sixteen parts of two gate and two up tiles the kernel would need scratch memory
  // (1 x 28672 x 4096 27.8 us instead of 25.9)
  constexpr int AHEAD = NW * WV > 32 ? 8 : WV;
  for (int t = w; t < TM * HALF; t += WV) {
    const int i = t / HALF, j = t % HALF;
    const int row = i * 16 + (lane & 15), col = c0 + j * 16 + (lane >> 4) * 4;
    if (row >= a.M || col >= a.N) continue;
    auto sum = [&](int tile) {
      i32x4 s = {0, 0, 0, 0};
#pragma unroll AHEAD
      for (int v = 0; v < WV; ++v) s += part[v][tile][lane];
      return s;
    };
    const float sa = a.sa[row];
    f32x4 y = scaled(sum(i * NW + j), sa, load_scales(a.sb, col, a.N));
    if constexpr (SW) {
      y = swiglu(y, scaled(sum(i * NW + HALF + j), sa, load_scales(a.sb2, col, a.N)));
    }
    store4<EPI>(a, row, col, y);
  }
}

template <int TM, int HALF, int R, int WV>
hipError_t launch_thin(const GemmI8Args& a, int epi, hipStream_t st) {
  const dim3 grid((a.N + 16 * HALF - 1) / (16 * HALF)), block(64 * WV);
  switch (epi) {
    case EPI_BF16: hipLaunchKernelGGL((gemm_i8_thin_kernel<TM, HALF, R, EPI_BF16, WV>), grid, block, 0, st, a); break;
    case EPI_RESID: hipLaunchKernelGGL((gemm_i8_thin_kernel<TM, HALF, R, EPI_RESID, WV>), grid, block, 0, st, a); break;
    case EPI_SWIGLU: hipLaunchKernelGGL((gemm_i8_thin_kernel<TM, HALF, R, EPI_SWIGLU, WV>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((gemm_i8_thin_kernel<TM, HALF, R, EPI_F32, WV>), grid, block, 0, st, a); break;
  }
  return hipGetLastError();
}

}  // namespace

// plan: tm row tiles, nw columns tiles, wv wavefronts
hipError_t gemm_i8_thin(const GemmI8Args& a, int epi, const GemmI8Plan& p, hipStream_t st) {
#define HXF_THIN(T, N, R, W) \
  if (p.tm == T && p.nw == N && p.wv == W) return launch_thin<T, N, R, W>(a, epi, st);
  HXF_THIN(1, 1, 8, 4) HXF_THIN(1, 2, 4, 16) HXF_THIN(2, 1, 4, 16) HXF_THIN(2, 2, 4, 8) HXF_THIN(4, 1, 4, 8) HXF_THIN(4, 2, 4, 8)
#undef HXF_THIN
  return hipErrorInvalidValue;
}

}  // namespace hxf
