// Rows into 8-bit codes with a scale each: bf16 rows, and RMSNorm of fp32 rows.
//
// With t the row's values (bf16 as fp32, or x * g) and m = max|t|: code = rint(t * (127 / m)), scale = m / 127 times
// what the norm divides by, which cancels in the codes.  Every step of a code is one correctly rounded fp32
// operation, so the codes do not depend on how a row is shared out.
//
// Memory is the bound (3 bytes a value, 5 with the norm).  A workgroup takes ROWS rows, 64 / ROWS lanes of a wavefront
// each: successive lanes load successive 16 bytes of a row (sixteen values of one row a lane, in whole pieces of a
// tile, stored 16 bytes at once but loaded from four rows' lines by every four lanes, took 20.4 us instead of 16.3 for
// the norm of 2080 x 5120), and the rows' pieces are neighbours in the tile.  A row's values stay in registers between
// the maximum and the codes (read twice instead: 2080 x 28672 in 57 us where two rows in registers take 46).
//
// ROWS = 4 up to K of 8192, 2048 with the norm, where a workgroup is small; 2 up to 16384, 4096 with the norm, and 1
// above, where more rows would fill a CU's registers and none is loaded while another is written (us with 4, 2 and 1 rows,
// wavefronts chosen for each: 2080 x 28672 48.5 / 46.1 / 40.8, 64 x 28672 9.9 / 6.5 / 5.6, 2080 x 14336 25.8 / 22.8 /
// 23.4; the norm of 2080 x 14336 45.2 / 41.0 / 35.1, of 2080 x 5120 16.3 / 15.7 / 14.9, of 256 x 8192 8.1 / 6.1 / 6.0;
// but 16000 x 512 7.5 / 9.9, 28672 x 8192 124 / 135 and 2080 x 8192 15.1 / 15.4 / 15.6).  Rows above 32768 fit no workgroup's
// registers and are read twice, two a workgroup (us with 4, 2 and 1 rows: 2080 x 40000 85 / 82 / 75, 64 x 40000 14.2 / 8.7 /
// 6.1, 2080 x 131064 353 / 366 / 348, 300 x 131064 67 / 48 / 54; the norm of them 160 / 144 / 132, 28 / 16 / 10, 609 / 640 /
// 628, 131 / 92 / 101): the longest rows of few take least with two, the rest with one.
#include "common.hpp"
#include "gemm_util.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

constexpr float kTiny = 0x1p-119f;   // below it 127 / m may be no fp32 number

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

// Maximum of a row over the workgroup (NWV wavefronts; a lane's row is lane / (64 / ROWS)), and the sum of s
template <int ROWS, int NWV, bool SUM>
__device__ __forceinline__ uint32_t rows_reduce(uint32_t m, float& s, uint32_t* red, float* sums) {
  const int lane = threadIdx.x & 63, row = lane / (64 / ROWS);
#pragma unroll
  for (int o = 32 / ROWS; o >= 1; o >>= 1) {
    m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
    if constexpr (SUM) s += __shfl_xor(s, o, kWave);
  }
  if ((lane & (64 / ROWS - 1)) == 0) {
    red[(threadIdx.x >> 6) * ROWS + row] = m;
    if constexpr (SUM) sums[(threadIdx.x >> 6) * ROWS + row] = s;
  }
  __syncthreads();
  m = red[row];
#pragma unroll
  for (int w = 1; w < NWV; ++w) m = max(m, red[w * ROWS + row]);
  if constexpr (SUM) {
    s = sums[row];
#pragma unroll
    for (int w = 1; w < NWV; ++w) s += sums[w * ROWS + row];
  }
  return m;
}

__device__ __forceinline__ uint4 load16(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }

// V: units (ROWS rows x 1024 / ROWS columns) of a wavefront held in registers; 0: any number of them, read twice.
template <int ROWS, int NWV, int V>
__global__ __launch_bounds__(64 * NWV) void quant_i8_kernel(const uint16_t* x, int64_t stride, int R, int K,
                                                            int8_t* codes, float* scale) {
  __shared__ uint32_t red[NWV * ROWS];
  constexpr int LPR = 64 / ROWS, UNIT = 16 * LPR;
  const int kt = (K + 63) / 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = xcd_remap(blockIdx.x, gridDim.x) * ROWS + lane / LPR;
  const int c0 = w * UNIT + (lane & (LPR - 1)) * 8;
  const bool live = r < R;
  const uint16_t* row = x + (int64_t)min(r, R - 1) * stride;
  struct Vals {
    uint32_t v[8];
  };
  auto load = [&](int k) {   // what is outside the matrix is zero
    const bool in0 = live && k < K, in1 = live && k + LPR * 8 < K;
    const uint4 p = load16(row + (in0 ? k : 0)), q = load16(row + (in1 ? k + LPR * 8 : 0));
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
    for (int u = 0; u < V; ++u) held[u] = load(c0 + u * NWV * UNIT);
#pragma unroll
    for (int u = 0; u < V; ++u) m = largest(held[u], m);
  } else {
    for (int k = c0; k < K; k += NWV * UNIT) m = largest(load(k), m);
  }
  float none = 0.f;
  const RowMax q = row_max(rows_reduce<ROWS, NWV, false>(max(m << 16, m & 0xFFFF0000u), none, red, nullptr));
  const uint32_t keep = q.inv != 0.f ? ~0u : 0u;   // 0 times an infinity is none
  int8_t* out = codes + i8_elem(r, 0, kt);
  auto store = [&](const Vals& a, int k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int kk = k + LPR * 8 * h;
      if (kk >= kt * 64) return;
      uint32_t o[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t p = a.v[4 * h + 2 * e], s = a.v[4 * h + 2 * e + 1];
        o[e] = codes4(__uint_as_float(p << 16), __uint_as_float(p & 0xFFFF0000u), __uint_as_float(s << 16),
                      __uint_as_float(s & 0xFFFF0000u), q.inv) & keep;
      }
      *reinterpret_cast<uint2*>(out + (kk >> 6) * 1024 + ((kk >> 4) & 3) * 256 + (kk & 15)) = make_uint2(o[0], o[1]);
    }
  };
  if constexpr (V > 0) {
#pragma unroll
    for (int u = 0; u < V; ++u) store(held[u], c0 + u * NWV * UNIT);
  } else {
    for (int k = c0; k < kt * 64; k += NWV * UNIT) store(load(k), k);
  }
  if (live && w == 0 && (lane & (LPR - 1)) == 0) scale[r] = q.unit;
}

template <int ROWS, int NWV, int V>
__global__ __launch_bounds__(64 * NWV) void rmsnorm_i8_kernel(const float* x, const int32_t* rows, int x_rows,
                                                              const uint16_t* g, int8_t* codes, float* scale,
                                                              int n_rows, int d, float eps) {
  __shared__ uint32_t red[NWV * ROWS];
  __shared__ float sums[NWV * ROWS];
  constexpr int LPR = 64 / ROWS, UNIT = 16 * LPR;
  const int kt = (d + 63) / 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = xcd_remap(blockIdx.x, gridDim.x) * ROWS + lane / LPR;
  const int c0 = w * UNIT + (lane & (LPR - 1)) * 4;
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
      const bool in = live && k + LPR * 4 * h < d;
      float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
      if (in) p = *reinterpret_cast<const float4*>(row + k + LPR * 4 * h);
      a.v[4 * h] = p.x, a.v[4 * h + 1] = p.y, a.v[4 * h + 2] = p.z, a.v[4 * h + 3] = p.w;
    }
    return a;
  };
  auto gain = [&](Vals& a, int k) {   // x * g
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const uint2 p = *reinterpret_cast<const uint2*>(g + (k + LPR * 4 * h < d ? k + LPR * 4 * h : 0));
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
    for (int u = 0; u < V; ++u) held[u] = load(c0 + u * NWV * UNIT);
#pragma unroll
    for (int u = 0; u < V; ++u) take(held[u], c0 + u * NWV * UNIT);
  } else {
    for (int k = c0; k < d; k += NWV * UNIT) {
      Vals a = load(k);
      take(a, k);
    }
  }
  const RowMax q = row_max(rows_reduce<ROWS, NWV, true>(m, ss, red, sums));
  const uint32_t keep = q.inv != 0.f ? ~0u : 0u;
  int8_t* out = codes + i8_elem(r, 0, kt);
  auto store = [&](const Vals& a, int k) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int kk = k + LPR * 4 * e;
      if (kk >= kt * 64) return;
      *reinterpret_cast<uint32_t*>(out + (kk >> 6) * 1024 + ((kk >> 4) & 3) * 256 + (kk & 15)) =
          codes4(a.v[4 * e], a.v[4 * e + 1], a.v[4 * e + 2], a.v[4 * e + 3], q.inv) & keep;
    }
  };
  if constexpr (V > 0) {
#pragma unroll
    for (int u = 0; u < V; ++u) store(held[u], c0 + u * NWV * UNIT);
  } else {
    for (int k = c0; k < kt * 64; k += NWV * UNIT) {
      Vals a = load(k);
      gain(a, k);
      store(a, k);
    }
  }
  if (r < n_rows && w == 0 && (lane & (LPR - 1)) == 0)
    scale[r] = q.unit == 0.f ? 0.f : q.unit * rsqrtf(ss / (float)d + eps);   // (a row of zeros may be divided by zero)
}

}  // namespace

hipError_t quant_i8_launch(const uint16_t* x, int64_t stride, int R, int K, int8_t* codes, float* scale,
                           hipStream_t st) {
#define HXF_Q(ROWS, W, V)                                                                                           \
  if (K <= ROWS_K(ROWS, W, V)) {                                                                                    \
    hipLaunchKernelGGL((quant_i8_kernel<ROWS, W, V>), dim3((R + 15) / 16 * (16 / ROWS)), dim3(64 * W), 0, st, x,    \
                       stride, R, K, codes, scale);                                                                 \
    return hipGetLastError();                                                                                       \
  }
#define ROWS_K(ROWS, W, V) (V ? W * V * 1024 / ROWS : INT32_MAX)
  HXF_Q(4, 4, 1) HXF_Q(4, 8, 1) HXF_Q(4, 8, 2) HXF_Q(4, 8, 4) HXF_Q(2, 16, 2) HXF_Q(1, 16, 2) HXF_Q(2, 16, 0)
  return hipErrorInvalidValue;
#undef HXF_Q
}

hipError_t rmsnorm_i8_launch(const float* x, const int32_t* rows, int x_rows, const uint16_t* g, int8_t* codes,
                             float* scale, int n_rows, int d, float eps, hipStream_t st) {
#define HXF_N(ROWS, W, V)                                                                                           \
  if (d <= ROWS_K(ROWS, W, V)) {                                                                                    \
    hipLaunchKernelGGL((rmsnorm_i8_kernel<ROWS, W, V>), dim3((n_rows + 15) / 16 * (16 / ROWS)), dim3(64 * W), 0, st, \
                       x, rows, x_rows, g, codes, scale, n_rows, d, eps);                                           \
    return hipGetLastError();                                                                                       \
  }
  HXF_N(4, 4, 1) HXF_N(4, 8, 1) HXF_N(2, 8, 1) HXF_N(1, 8, 1) HXF_N(1, 16, 1) HXF_N(1, 16, 2) HXF_N(2, 16, 0)
  return hipErrorInvalidValue;
#undef HXF_N
#undef ROWS_K
}

}  // namespace hxf
