// Rows into 8-bit codes with a scale each: bf16 rows, and RMSNorm of fp32 rows.
//
// With t the row's values (bf16 as fp32, or x * g) and m = max|t|: code = rint(t * (127 / m)), scale = m / 127 times
// what the norm divides by, which cancels in the codes.  Every step of a code is one correctly rounded fp32
// operation, so the codes do not depend on how a row is shared out.
//
// Memory is the bound (3 bytes a value, 5 with the norm).  A workgroup takes four rows; a wavefront's unit is four
// rows x 256 columns, a lane's 16 successive values of one row: they are one 16-byte piece of a tile, and the four
// rows' pieces are neighbours there.  A row's values stay in registers between the maximum and the codes.
#include "common.hpp"
#include "gemm_util.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

constexpr float kTiny = 0x1p-119f;   // below it 127 / m may be no fp32 number
constexpr int kRows = 4, kUnit = 256;

struct RowMax {
  float inv, unit;   // 127 / m and m / 127
};
// bits of m, the largest of the magnitudes' bits: NaN above infinity above every number
__device__ __forceinline__ RowMax row_max(uint32_t bits) {
  const float m = __uint_as_float(bits);
  if (bits >= 0x7F800000u) return {0.f, __builtin_nanf("")};
  if (m < kTiny) return {0.f, 0.f};
  return {127.f / m, m / 127.f};
}

__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Four codes.  t * inv is rounded to fp32 first (no fused multiply-add); adding 1.5 * 2^23 then rounds it to a whole
// number, ties to even, which stands in the low bits of the sum.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
#pragma clang fp contract(off)
  constexpr float kMagic = 12582912.f;
  const float p = a * inv, q = b * inv, r = c * inv, s = d * inv;
  const uint32_t i = __float_as_uint(p + kMagic), j = __float_as_uint(q + kMagic), k = __float_as_uint(r + kMagic),
                 l = __float_as_uint(s + kMagic);
  const uint32_t lo = __builtin_amdgcn_perm(j, i, 0x0c0c0400), hi = __builtin_amdgcn_perm(l, k, 0x04000c0c);
  return lo | hi;
}

// Maximum of a row over the workgroup (NWV wavefronts; a lane's row is lane % 4), and the sum of s
template <int NWV, bool SUM>
__device__ __forceinline__ uint32_t rows_reduce(uint32_t m, float& s, uint32_t* red, float* sums) {
  const int lane = threadIdx.x & 63, row = lane & (kRows - 1);
#pragma unroll
  for (int o = 32; o >= kRows; o >>= 1) {
    m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
    if constexpr (SUM) s += __shfl_xor(s, o, kWave);
  }
  if (lane < kRows) {
    red[(threadIdx.x >> 6) * kRows + lane] = m;
    if constexpr (SUM) sums[(threadIdx.x >> 6) * kRows + lane] = s;
  }
  __syncthreads();
  m = red[row];
#pragma unroll
  for (int w = 1; w < NWV; ++w) m = max(m, red[w * kRows + row]);
  if constexpr (SUM) {
    s = sums[row];
#pragma unroll
    for (int w = 1; w < NWV; ++w) s += sums[w * kRows + row];
  }
  return m;
}

__device__ __forceinline__ uint4 load16(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }

// V: units of a wavefront held in registers; 0: any number of them, read twice.
template <int NWV, int V>
__global__ __launch_bounds__(64 * NWV) void quant_i8_kernel(const uint16_t* x, int64_t stride, int R, int K,
                                                            int8_t* codes, float* scale) {
  __shared__ uint32_t red[NWV * kRows];
  const int kt = (K + 63) / 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = xcd_remap(blockIdx.x, gridDim.x) * kRows + (lane & (kRows - 1));
  const int c0 = w * kUnit + (lane / kRows) * 16;   // the lane's first column of the wavefront's first unit
  const bool live = r < R;
  const uint16_t* row = x + (int64_t)min(r, R - 1) * stride;
  struct Vals {
    uint32_t v[8];
  };
  auto load = [&](int k) {   // what is outside the matrix is zero
    const bool in0 = live && k < K, in1 = live && k + 8 < K;
    const uint4 p = load16(row + (in0 ? k : 0)), q = load16(row + (in1 ? k + 8 : 0));
    return Vals{{in0 ? p.x : 0, in0 ? p.y : 0, in0 ? p.z : 0, in0 ? p.w : 0, in1 ? q.x : 0, in1 ? q.y : 0,
                 in1 ? q.z : 0, in1 ? q.w : 0}};
  };
  auto largest = [&](const Vals& a, uint32_t m) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max_halves(m, a.v[e] & 0x7FFF7FFFu);
    return m;
  };
  Vals held[V ? V : 1];
  uint32_t m = 0;
  if constexpr (V > 0) {
#pragma unroll
    for (int u = 0; u < V; ++u) held[u] = load(c0 + u * NWV * kUnit);
#pragma unroll
    for (int u = 0; u < V; ++u) m = largest(held[u], m);
  } else {
    for (int k = c0; k < K; k += NWV * kUnit) m = largest(load(k), m);
  }
  float none = 0.f;
  const RowMax q = row_max(rows_reduce<NWV, false>(max(m << 16, m & 0xFFFF0000u), none, red, nullptr));
  const uint32_t keep = q.inv != 0.f ? ~0u : 0u;   // 0 times an infinity is none
  int8_t* out = codes + i8_elem(r, 0, kt);
  auto store = [&](const Vals& a, int k) {
    if (k >= kt * 64) return;
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t p = a.v[2 * e], s = a.v[2 * e + 1];
      o[e] = codes4(__uint_as_float(p << 16), __uint_as_float(p & 0xFFFF0000u), __uint_as_float(s << 16),
                    __uint_as_float(s & 0xFFFF0000u), q.inv) & keep;
    }
    *reinterpret_cast<uint4*>(out + (k >> 6) * 1024 + ((k >> 4) & 3) * 256) = make_uint4(o[0], o[1], o[2], o[3]);
  };
  if constexpr (V > 0) {
#pragma unroll
    for (int u = 0; u < V; ++u) store(held[u], c0 + u * NWV * kUnit);
  } else {
    for (int k = c0; k < kt * 64; k += NWV * kUnit) store(load(k), k);
  }
  if (live && threadIdx.x < kRows) scale[r] = q.unit;
}

template <int NWV, int V>
__global__ __launch_bounds__(64 * NWV) void rmsnorm_i8_kernel(const float* x, const int32_t* rows, int x_rows,
                                                              const uint16_t* g, int8_t* codes, float* scale,
                                                              int n_rows, int d, float eps) {
  __shared__ uint32_t red[NWV * kRows];
  __shared__ float sums[NWV * kRows];
  const int kt = (d + 63) / 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = xcd_remap(blockIdx.x, gridDim.x) * kRows + (lane & (kRows - 1));
  const int c0 = w * kUnit + (lane / kRows) * 16;
  int src = r < n_rows ? r : -1;
  if (rows && r < n_rows) src = rows[r];
  const bool live = src >= 0 && src < x_rows;
  const float* row = x + (size_t)(live ? src : 0) * d;
  struct Vals {
    float v[16];
  };
  float ss = 0.f;
  uint32_t m = 0;
  auto load = [&](int k) {   // x
    Vals a;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const bool in = live && k + 4 * h < d;
      float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
      if (in) p = *reinterpret_cast<const float4*>(row + k + 4 * h);
      a.v[4 * h] = p.x, a.v[4 * h + 1] = p.y, a.v[4 * h + 2] = p.z, a.v[4 * h + 3] = p.w;
    }
    return a;
  };
  auto gain = [&](Vals& a, int k) {   // x * g
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const uint2 p = *reinterpret_cast<const uint2*>(g + (k + 4 * h < d ? k + 4 * h : 0));
      a.v[4 * h] *= __uint_as_float(p.x << 16);
      a.v[4 * h + 1] *= __uint_as_float(p.x & 0xFFFF0000u);
      a.v[4 * h + 2] *= __uint_as_float(p.y << 16);
      a.v[4 * h + 3] *= __uint_as_float(p.y & 0xFFFF0000u);
    }
  };
  auto take = [&](Vals& a, int k) {
#pragma unroll
    for (int e = 0; e < 16; ++e) ss += a.v[e] * a.v[e];
    gain(a, k);
#pragma unroll
    for (int e = 0; e < 16; ++e) m = max(m, mag(a.v[e]));
  };
  Vals held[V ? V : 1];
  if constexpr (V > 0) {
#pragma unroll
    for (int u = 0; u < V; ++u) held[u] = load(c0 + u * NWV * kUnit);
#pragma unroll
    for (int u = 0; u < V; ++u) take(held[u], c0 + u * NWV * kUnit);
  } else {
    for (int k = c0; k < d; k += NWV * kUnit) {
      Vals a = load(k);
      take(a, k);
    }
  }
  const RowMax q = row_max(rows_reduce<NWV, true>(m, ss, red, sums));
  const uint32_t keep = q.inv != 0.f ? ~0u : 0u;
  int8_t* out = codes + i8_elem(r, 0, kt);
  auto store = [&](const Vals& a, int k) {
    if (k >= kt * 64) return;
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o[e] = codes4(a.v[4 * e], a.v[4 * e + 1], a.v[4 * e + 2], a.v[4 * e + 3], q.inv) & keep;
    *reinterpret_cast<uint4*>(out + (k >> 6) * 1024 + ((k >> 4) & 3) * 256) = make_uint4(o[0], o[1], o[2], o[3]);
  };
  if constexpr (V > 0) {
#pragma unroll
    for (int u = 0; u < V; ++u) store(held[u], c0 + u * NWV * kUnit);
  } else {
    for (int k = c0; k < kt * 64; k += NWV * kUnit) {
      Vals a = load(k);
      gain(a, k);
      store(a, k);
    }
  }
  if (r < n_rows && threadIdx.x < kRows) scale[r] = live ? q.unit * rsqrtf(ss / (float)d + eps) : 0.f;
}

}  // namespace

hipError_t quant_i8_launch(const uint16_t* x, int64_t stride, int R, int K, int8_t* codes, float* scale,
                           hipStream_t st) {
  const dim3 grid((R + 15) / 16 * (16 / kRows));
#define HXF_Q(W, V)                                                                                            \
  do {                                                                                                         \
    hipLaunchKernelGGL((quant_i8_kernel<W, V>), grid, dim3(64 * W), 0, st, x, stride, R, K, codes, scale);     \
    return hipGetLastError();                                                                                  \
  } while (0)
  const int units = (K + kUnit - 1) / kUnit;
  if (units <= 4) HXF_Q(4, 1);
  if (units <= 8) HXF_Q(4, 2);
  if (units <= 16) HXF_Q(4, 4);
  if (units <= 32) HXF_Q(8, 4);
  if (units <= 56) HXF_Q(8, 7);
  if (units <= 80) HXF_Q(8, 10);
  if (units <= 112) HXF_Q(8, 14);
  HXF_Q(8, 0);
#undef HXF_Q
}

hipError_t rmsnorm_i8_launch(const float* x, const int32_t* rows, int x_rows, const uint16_t* g, int8_t* codes,
                             float* scale, int n_rows, int d, float eps, hipStream_t st) {
  const dim3 grid((n_rows + 15) / 16 * (16 / kRows));
#define HXF_N(W, V)                                                                                                 \
  do {                                                                                                              \
    hipLaunchKernelGGL((rmsnorm_i8_kernel<W, V>), grid, dim3(64 * W), 0, st, x, rows, x_rows, g, codes, scale, n_rows, \
                       d, eps);                                                                                     \
    return hipGetLastError();                                                                                       \
  } while (0)
  const int units = (d + kUnit - 1) / kUnit;
  if (units <= 4) HXF_N(4, 1);
  if (units <= 8) HXF_N(4, 2);
  if (units <= 16) HXF_N(8, 2);
  if (units <= 24) HXF_N(8, 3);
  if (units <= 32) HXF_N(8, 4);
  if (units <= 56) HXF_N(8, 7);
  HXF_N(8, 0);
#undef HXF_N
}

}  // namespace hxf
