// Rows into 8-bit codes with a scale each: bf16 rows, and RMSNorm of fp32 rows.
//
// With t the row's values (bf16 as fp32, or x * g) and m = max|t|: code = rint(t * (127 / m)), scale = m / 127 times
// what the norm divides by, which cancels in the codes.  Every step of a code is one correctly rounded fp32
// operation, so the codes do not depend on how a row is shared out.
#include "common.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

constexpr float kTiny = 0x1p-119f;   // below it 127 / m may be no fp32 number

struct RowMax {
  float inv, unit;   // 127 / m and m / 127
};
// m: NaN or infinite where the row holds one
__device__ __forceinline__ RowMax row_max(float m) {
  if (!(m < __builtin_inff())) return {0.f, __builtin_nanf("")};
  if (m < kTiny) return {0.f, 0.f};
  return {127.f / m, m / 127.f};
}

// |x| for a maximum over the bits of magnitudes: NaN above infinity above every number
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  const int i = (int)rintf(a * inv), j = (int)rintf(b * inv), k = (int)rintf(c * inv), l = (int)rintf(d * inv);
  return (uint32_t)(i & 255) | (uint32_t)(j & 255) << 8 | (uint32_t)(k & 255) << 16 | (uint32_t)l << 24;
}

__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, kWave));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return max(max(red[0], red[1]), max(red[2], red[3]));
}

// a workgroup per row of the padded matrix
__global__ __launch_bounds__(256) void quant_i8_kernel(const uint16_t* x, int64_t stride, int R, int K, int8_t* codes,
                                                       float* scale) {
  __shared__ uint32_t red[4];
  const int r = blockIdx.x, kt = (K + 63) / 64;
  const uint16_t* row = x + (int64_t)r * stride;
  uint32_t m = 0;
  if (r < R)
    for (int k = threadIdx.x; k < K; k += 256) m = max(m, mag(bf2f(row[k])));
  const RowMax q = row_max(__uint_as_float(block_max(m, red)));
  for (int k = threadIdx.x; k < kt * 64; k += 256) {
    const bool in = r < R && k < K && q.inv != 0.f;   // 0 times an infinity would be NaN
    codes[i8_elem(r, k, kt)] = in ? (int8_t)rintf(bf2f(row[k]) * q.inv) : 0;
  }
  if (r < R && threadIdx.x == 0) scale[r] = q.unit;
}

__global__ __launch_bounds__(256) void rmsnorm_i8_kernel(const float* x, const int32_t* rows, int x_rows,
                                                         const uint16_t* g, int8_t* codes, float* scale, int n_rows,
                                                         int d, float eps) {
  __shared__ uint32_t red[4];
  __shared__ float sums[4];
  const int r = blockIdx.x, kt = (d + 63) / 64;
  int src = r < n_rows ? r : -1;
  if (rows && r < n_rows) src = rows[r];
  const bool live = src >= 0 && src < x_rows;
  const float* row = x + (size_t)(live ? src : 0) * d;
  uint32_t m = 0;
  float ss = 0.f;
  if (live)
    for (int k = threadIdx.x; k < d; k += 256) {
      m = max(m, mag(row[k] * bf2f(g[k])));
      ss += row[k] * row[k];
    }
  ss = wave_sum(ss);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
  const RowMax q = row_max(__uint_as_float(block_max(m, red)));
  for (int k = threadIdx.x; k < kt * 64; k += 256) {
    const bool in = live && k < d && q.inv != 0.f;
    codes[i8_elem(r, k, kt)] = in ? (int8_t)rintf(row[k] * bf2f(g[k]) * q.inv) : 0;
  }
  if (r < n_rows && threadIdx.x == 0)
    scale[r] = live ? q.unit * rsqrtf((sums[0] + sums[1] + sums[2] + sums[3]) / (float)d + eps) : 0.f;
}

}  // namespace

hipError_t quant_i8_launch(const uint16_t* x, int64_t stride, int R, int K, int8_t* codes, float* scale,
                           hipStream_t st) {
  const int padded = (R + 15) / 16 * 16;
  hipLaunchKernelGGL(quant_i8_kernel, dim3(padded), dim3(256), 0, st, x, stride, R, K, codes, scale);
  return hipGetLastError();
}

hipError_t rmsnorm_i8_launch(const float* x, const int32_t* rows, int x_rows, const uint16_t* g, int8_t* codes,
                             float* scale, int n_rows, int d, float eps, hipStream_t st) {
  const int padded = (n_rows + 15) / 16 * 16;
  hipLaunchKernelGGL(rmsnorm_i8_kernel, dim3(padded), dim3(256), 0, st, x, rows, x_rows, g, codes, scale, n_rows, d, eps);
  return hipGetLastError();
}

}  // namespace hxf
