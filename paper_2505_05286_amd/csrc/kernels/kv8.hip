// The 8-bit KV cache: tables of a batch from its lengths, and the quantised write.
#include "common.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

// Exclusive sum over the workgroup's 1024 threads of v; *total gets the whole sum.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* part, int64_t* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  __syncthreads();   // (part may still be read from the scan before)
  if (lane == 63) part[w] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int i = 0; i < 16; ++i) {
    if (i < w) before += part[i];
    all += part[i];
  }
  *total = all;
  return before + x - v;
}

// One workgroup: totals and checks, then the scans, then the rows.
__global__ __launch_bounds__(1024) void slot_map_kernel(SlotMapArgs a) {
  __shared__ int64_t part[16];
  __shared__ int32_t row0[kSlotMapMaxSeqs + 1], page0[kSlotMapMaxSeqs];
  int64_t rows = 0, pages = 0;
  bool bad = false;
  for (int s0 = 0; s0 < a.S; s0 += 1024) {
    const int s = s0 + threadIdx.x;
    const int64_t st = s < a.S ? a.start[s] : 0, n = s < a.S ? a.n_new[s] : 0;
    const int64_t have = (st + kPage - 1) / kPage, end = (st + n + kPage - 1) / kPage;
    bad |= st < 0 || n < 0 || (s < a.S && end > a.bt_stride);
    int64_t t_rows, t_pages;
    const int64_t r = block_scan(n, part, &t_rows), p = block_scan(end - have, part, &t_pages);
    if (s < a.S) {
      row0[s] = (int32_t)(rows + r);
      page0[s] = (int32_t)(pages + p);
    }
    rows += t_rows;
    pages += t_pages;
  }
  const int n_free = min(max(a.n_free[0], 0), a.free_cap);
  const bool ok = !__syncthreads_or(bad) && rows <= a.T && pages <= n_free;
  if (threadIdx.x == 0) {
    a.status[0] = ok ? (int32_t)pages : -1;
    a.status[1] = ok ? (int32_t)rows : 0;
    a.row0[a.S] = ok ? (int32_t)rows : 0;
    row0[a.S] = (int32_t)rows;
  }
  for (int s = threadIdx.x; s < a.S; s += 1024) {
    const int st = a.start[s];
    a.row0[s] = ok ? row0[s] : 0;
    a.ctx[s] = ok ? st + a.n_new[s] : max(st, 0);
    if (!ok) continue;
    const int have = (st + kPage - 1) / kPage, end = (st + a.n_new[s] + kPage - 1) / kPage;
    for (int p = have; p < end; ++p) a.bt[(size_t)s * a.bt_stride + p] = a.free_pages[page0[s] + p - have];
  }
  __syncthreads();
  for (int t = threadIdx.x; t < a.T; t += 1024) {
    int ps = 0, sl = -1;
    if (ok && t < rows) {
      int lo = 0, hi = a.S;   // the last s with row0[s] <= t (row0[S] = rows > t)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row0[mid] <= t) lo = mid;
        else hi = mid;
      }
      const int st = a.start[lo], have = (st + kPage - 1) / kPage;
      ps = st + t - row0[lo];
      const int p = ps / kPage;
      const int page = p < have ? a.bt[(size_t)lo * a.bt_stride + p] : a.free_pages[page0[lo] + p - have];
      sl = (uint32_t)page < (1u << 27) ? page * kPage + ps % kPage : -1;
    }
    a.pos[t] = ps;
    a.slot[t] = sl;
  }
}

// Scale exponent of a page whose largest finite magnitude is amax: the least e with
// amax <= 448 * 2^e, no less than -100 (448 = 1.75 * 2^8, so e is amax's exponent minus 8, plus one
// where the significand exceeds 1.75).  Returned as the power of two.
__device__ __forceinline__ float scale_of(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u);   // biased; an fp32 subnormal has exponent 0
  return __uint_as_float((uint32_t)max(e, 27) << 23);
}
// 1 / s of a power of two in the range that scale_of makes
__device__ __forceinline__ float inverse(float s) { return __uint_as_float((254u << 23) - (__float_as_uint(s) & 0x7F800000u)); }

__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}
__device__ __forceinline__ uint8_t e4m3(float a) { return (uint8_t)e4m3x2(a, 0.f); }
__device__ __forceinline__ float from_e4m3(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8(c, 0); }

// |x|, or 0 where x is not finite
__device__ __forceinline__ float finite_abs(float x) {
  const float m = fabsf(x);
  return m < __builtin_huge_valf() ? m : 0.f;
}

struct Rows {
  const Kv8WriteArgs& a;
  __device__ bool live(int t) const {
    const int s = a.slot[t];
    if (s < 0 || s >= a.pool.n_blocks * kPage) return false;
    return !a.cs || (a.pos[t] >= 0 && a.pos[t] < a.max_pos);
  }
  // Value (dimension d) of a head of row t, rotated where wanted: products and their sum each rounded to
  // fp32, so that the codes do not depend on how a compiler contracts them.
  __device__ float value(int t, int head, int d, bool rotate) const {
#pragma clang fp contract(off)
    const uint16_t* x = a.qkv + t * a.qkv_stride + head * a.dh;
    if (!rotate || !a.cs) return bf2f(x[d]);
    const int half = a.dh >> 1, i = d < half ? d : d - half;
    const float2 cs = a.cs[(size_t)a.pos[t] * half + i];
    const float u = bf2f(x[i]), w = bf2f(x[i + half]);
    return d < half ? u * cs.x - w * cs.y : w * cs.x + u * cs.y;
  }
};

// One wavefront per (row, kv-head) or (row, q-head); a kv wavefront works where its row begins a run.
__global__ __launch_bounds__(64) void kv8_write_kernel(Kv8WriteArgs a) {
  const Rows rows{a};
  const int t = blockIdx.x, lane = threadIdx.x;
  if (!rows.live(t)) return;
  const int dh = a.dh;
  if (blockIdx.y >= (unsigned)a.Hkv) {
    const int h = blockIdx.y - a.Hkv;
    for (int d = lane; d < dh; d += 64) a.q_out[t * a.q_stride + h * dh + d] = f2bf(rows.value(t, h, d, true));
    return;
  }
  const int slot = a.slot[t], o = slot % kPage;
  if (o && t && a.slot[t - 1] == slot - 1 && rows.live(t - 1)) return;
  int n = 1;
  while (o + n < kPage && t + n < a.T && a.slot[t + n] == slot + n && rows.live(t + n)) ++n;
  const int h = blockIdx.y;
  for (int kind = 0; kind < 2; ++kind) {
    const bool is_k = kind == 0;
    const int head = a.Hq + (is_k ? 0 : a.Hkv) + h;
    uint8_t* tile = (is_k ? a.pool.k : a.pool.v) + kv_tile(h, a.pool.n_blocks, slot / kPage, dh);
    float* scale = (is_k ? a.pool.ks : a.pool.vs) + h * a.pool.n_blocks + slot / kPage;
    float amax = 0.f;
    for (int r = 0; r < n; ++r)
      for (int d = lane; d < dh; d += 64) amax = fmaxf(amax, finite_abs(rows.value(t + r, head, d, is_k)));
    float s = scale_of(wave_max(amax));
    if (o) {
      const float before = *scale;
      s = fmaxf(s, before);
      if (s != before) {
        const float f = before * inverse(s);
        for (int p = 0; p < o; ++p)
          for (int d = lane; d < dh; d += 64) {
            uint8_t* c = tile + (is_k ? k8_offset(d, p) : v8_offset(d, p, dh));
            *c = e4m3(from_e4m3(*c) * f);
          }
      }
    }
    const float inv = inverse(s);
    for (int r = 0; r < n; ++r)
      for (int d = lane; d < dh; d += 64)
        tile[is_k ? k8_offset(d, o + r) : v8_offset(d, o + r, dh)] = e4m3(rows.value(t + r, head, d, is_k) * inv);
    if (lane == 0) *scale = s;
  }
}

}  // namespace

hipError_t slot_map_launch(const SlotMapArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(slot_map_kernel, dim3(1), dim3(1024), 0, st, a);
  return hipGetLastError();
}

hipError_t kv8_write_launch(const Kv8WriteArgs& a, hipStream_t st) {
  if (a.T <= 0) return hipSuccess;
  hipLaunchKernelGGL(kv8_write_kernel, dim3(a.T, a.Hkv + (a.q_out ? a.Hq : 0)), dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace hxf
