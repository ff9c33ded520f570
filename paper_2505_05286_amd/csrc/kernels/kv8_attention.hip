// Attention over the 8-bit KV cache, lengths on the device.
#include "common.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

// One wavefront per (query row, head): 64 tokens at a time, a lane scoring one of them, then
// each lane summing its dimensions over the 64 weights.
template <int DH>
__device__ void attend(const Kv8AttnArgs& a, int seq, int row, int head, int n, float* qs) {
  const int lane = threadIdx.x;
  const int kvh = head / (a.Hq / a.Hkv);
  const uint16_t* q = a.q + row * a.q_stride + head * DH;
  for (int d = lane; d < DH; d += 64) qs[d] = bf2f(q[d]);
  __syncthreads();
  const int32_t* bt = a.bt + (size_t)seq * a.bt_stride;
  float m = -1e30f, l = 0.f, acc[DH / 64] = {};
  for (int t0 = 0; t0 < n; t0 += 64) {
    const int t = t0 + lane;
    const int blk = t < n ? bt[t / kPage] : -1;
    const bool ok = blk >= 0 && blk < a.pool.n_blocks;
    float x = -__builtin_huge_valf(), vs = 0.f;
    if (ok) {
      const uint8_t* k = a.pool.k + kv_tile(kvh, a.pool.n_blocks, blk, DH);
      float s = 0.f;
      for (int d = 0; d < DH; ++d) s += qs[d] * __builtin_amdgcn_cvt_f32_fp8(k[k8_offset(d, t % kPage)], 0);
      x = s * a.pool.ks[kvh * a.pool.n_blocks + blk] * a.scale_log2;
      vs = a.pool.vs[kvh * a.pool.n_blocks + blk];
    }
    const float m_new = fmaxf(m, wave_max(x));
    const float alpha = exp2f(m - m_new), p = exp2f(x - m_new);
    l = l * alpha + wave_sum(p);
    m = m_new;
    for (int j = 0; j < DH / 64; ++j) acc[j] *= alpha;
    for (int u = 0; u < 64; ++u) {
      const int b = __shfl(ok ? blk : -1, u, kWave);
      const float w = __shfl(p, u, kWave), sc = __shfl(vs, u, kWave);
      if (b < 0) continue;
      const uint8_t* v = a.pool.v + kv_tile(kvh, a.pool.n_blocks, b, DH);
      for (int j = 0; j < DH / 64; ++j)
        acc[j] += w * sc * __builtin_amdgcn_cvt_f32_fp8(v[v8_offset(j * 64 + lane, (t0 + u) % kPage, DH)], 0);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int j = 0; j < DH / 64; ++j) a.out[row * a.out_stride + head * DH + j * 64 + lane] = f2bf(acc[j] * inv);
}

template <int DH>
__global__ __launch_bounds__(64) void kv8_decode_kernel(Kv8AttnArgs a) {
  __shared__ float qs[DH];
  const int n = min(max(a.ctx[blockIdx.x], 0), a.bt_stride * kPage);
  attend<DH>(a, blockIdx.x, blockIdx.x, blockIdx.y, n, qs);
}

template <int DH>
__global__ __launch_bounds__(64) void kv8_prefill_kernel(Kv8AttnArgs a) {
  __shared__ float qs[DH];
  const int row = blockIdx.x;
  for (int s = 0; s < a.S; ++s) {
    const int r0 = max(a.row0[s], 0), r1 = min(a.row0[s + 1], a.T);
    if (row < r0 || row >= r1) continue;
    const int64_t n = (int64_t)a.pos0[s] + (row - a.row0[s]) + 1;
    attend<DH>(a, s, row, blockIdx.y, (int)min(max(n, (int64_t)0), (int64_t)a.bt_stride * kPage), qs);
    return;
  }
}

}  // namespace

int64_t kv8_decode_ws_bytes(int, int, int, int) { return 256; }
int64_t kv8_prefill_ws_bytes(int, int, int, int, int) { return 256; }

hipError_t kv8_decode_launch(const Kv8AttnArgs& a, hipStream_t st) {
  const dim3 grid(a.S, a.Hq);
  if (a.dh == 128) hipLaunchKernelGGL(kv8_decode_kernel<128>, grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL(kv8_decode_kernel<64>, grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

hipError_t kv8_prefill_launch(const Kv8AttnArgs& a, hipStream_t st) {
  const dim3 grid(a.T, a.Hq);
  if (a.dh == 128) hipLaunchKernelGGL(kv8_prefill_kernel<128>, grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL(kv8_prefill_kernel<64>, grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace hxf
