// C = A[M,K] * B[N,K]^T of 8-bit codes, exact in 32-bit integers, scaled back by row and column.
#include "common.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mfma16x16x64(u32x4_t a, u32x4_t b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// A wavefront owns a tile of 16 x 16 outputs and reads both operands from memory.
template <int EPI>
__global__ __launch_bounds__(256) void gemm_i8_kernel(GemmI8Args a) {
  const int lane = threadIdx.x & 63, c0 = ((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)) * 16;
  if (c0 >= a.N) return;
  const u32x4_t* ap = reinterpret_cast<const u32x4_t*>(a.A + (size_t)blockIdx.y * a.kt * 1024) + lane;
  const u32x4_t* bp = reinterpret_cast<const u32x4_t*>(a.B + (size_t)(c0 / 16) * a.kt * 1024) + lane;
  const u32x4_t* up = EPI == EPI_SWIGLU ? reinterpret_cast<const u32x4_t*>(a.B2 + (size_t)(c0 / 16) * a.kt * 1024) + lane : bp;
  i32x4 acc = {0, 0, 0, 0}, acc2 = acc;
  for (int k = 0; k < a.kt; ++k) {
    const u32x4_t x = ap[k * 64];
    acc = mfma16x16x64(bp[k * 64], x, acc);
    if (EPI == EPI_SWIGLU) acc2 = mfma16x16x64(up[k * 64], x, acc2);
  }
  // lane holds row l % 16 and columns 4 (l / 16) .. + 3
  const int row = (int)blockIdx.y * 16 + (lane & 15);
  if (row >= a.M) return;
  const float sa = a.sa[row];
  for (int e = 0; e < 4; ++e) {
    const int col = c0 + (lane >> 4) * 4 + e;
    if (col >= a.N) continue;
    const size_t o = (size_t)row * a.ldc + col;
    const float y = (float)acc[e] * sa * a.sb[col];
    if (EPI == EPI_SWIGLU)
      reinterpret_cast<bf16_t*>(a.C)[o] = f2bf(y / (1.f + __expf(-y)) * ((float)acc2[e] * sa * a.sb2[col]));
    else if (EPI == EPI_BF16)
      reinterpret_cast<bf16_t*>(a.C)[o] = f2bf(y);
    else if (EPI == EPI_RESID)
      reinterpret_cast<float*>(a.C)[o] += y;
    else
      reinterpret_cast<float*>(a.C)[o] = y;
  }
}

}  // namespace

int64_t gemm_i8_ws_bytes(int, int, int) { return 0; }

hipError_t gemm_i8_launch(const GemmI8Args& a, int epi, hipStream_t st) {
  const dim3 grid((a.N + 63) / 64, (a.M + 15) / 16);
  switch (epi) {
    case EPI_BF16: hipLaunchKernelGGL(gemm_i8_kernel<EPI_BF16>, grid, dim3(256), 0, st, a); break;
    case EPI_RESID: hipLaunchKernelGGL(gemm_i8_kernel<EPI_RESID>, grid, dim3(256), 0, st, a); break;
    case EPI_SWIGLU: hipLaunchKernelGGL(gemm_i8_kernel<EPI_SWIGLU>, grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL(gemm_i8_kernel<EPI_F32>, grid, dim3(256), 0, st, a); break;
  }
  return hipGetLastError();
}

}  // namespace hxf
