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

constexpr float kNegInf = -__builtin_huge_valf();

// Pages of sequence b that its context reaches, and its tokens
__device__ __forceinline__ int ctx_of(const Kv8AttnArgs& a, int b) { return min(max(a.ctx[b], 0), a.bt_stride * kPage); }
__device__ __forceinline__ int pages_of(int n) { return (n + kPage - 1) / kPage; }

// The longest part of this batch (kv8_target_pages), found by every wavefront for itself from the contexts:
// one load and a scan for up to 64 sequences, against a launch and a round trip of a list through memory.
__device__ __forceinline__ int decode_target(const Kv8AttnArgs& a, int lane) {
  int64_t total = 0;
  for (int i0 = 0; i0 < a.S; i0 += kWave) {
    const int p = i0 + lane < a.S ? pages_of(ctx_of(a, i0 + lane)) : 0;
    // (64 counts of up to 2^27 pages: low and high halves apart)
    total += __builtin_amdgcn_readlane(wave_scan(p & 0xFFFFF), 63);
    total += (int64_t)__builtin_amdgcn_readlane(wave_scan(p >> 20), 63) << 20;
  }
  return (int)min(kv8_target_pages(total, a.S, a.Hkv), (int64_t)1 << 27);
}

// K and V bytes of a pair of pages: a lane's 16 dimensions of a token for K; for V four dimensions of the
// four tokens whose scores the lane holds
template <int DH>
struct Kv8Pair {
  uint4 k[2][DH / 64], v[2][DH / 64];
};

template <int DH>
__device__ __forceinline__ void kv8_load_page(Kv8Pair<DH>& R, int h, const Kv8AttnArgs& a, int kvh, int blk, int lane) {
  const size_t tile = kv_tile(kvh, a.pool.n_blocks, blk, DH);
  const uint8_t* k = a.pool.k + tile;
  const uint8_t* v = a.pool.v + tile;
  const int vo = (lane >> 4) * DH * 4 + (lane & 15) * 16;
#pragma unroll
  for (int u = 0; u < DH / 64; ++u) R.k[h][u] = load_stream16(k + u * 1024 + lane * 16);
#pragma unroll
  for (int u = 0; u < DH / 64; ++u) R.v[h][u] = load_stream16(v + u * 256 + vo);
}

// Mask keeping the first n (0..4) of four bytes
__device__ __forceinline__ uint32_t keep_bytes(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1; }

template <int DH>
struct Kv8State {
  f32x4 acc[DH / 16];   // tile (u, n): row r of the lane's column is dimension u*64 + r*4 + n
  float m, l;           // reference maximum of the column (log2 units); the lane's part of the denominator
};

// Scores, online softmax and PV product of one pair.  ks, vs: the pages' scales; cnt: their tokens that count.
template <int DH>
__device__ __forceinline__ void kv8_pair(Kv8State<DH>& S, const Kv8Pair<DH>& R, const bf16x8 (&qf)[DH / 32],
                                         const float (&ks)[2], const float (&vs)[2], const int (&cnt)[2],
                                         float scale_log2, int lane) {
  const int t0 = (lane >> 4) * 4;
  const bool full = cnt[0] + cnt[1] == 2 * kPage;   // wavefront-uniform
  float x[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < DH / 64; ++u) {
      const uint4 c = R.k[h][u];
      const uint2 w0 = e4m3x4_to_bf16(c.x, ks[h]), w1 = e4m3x4_to_bf16(c.y, ks[h]);
      const uint2 w2 = e4m3x4_to_bf16(c.z, ks[h]), w3 = e4m3x4_to_bf16(c.w, ks[h]);
      s = mfma16x16x32(as_bf16x8(make_uint4(w0.x, w0.y, w1.x, w1.y)), qf[2 * u], s);
      s = mfma16x16x32(as_bf16x8(make_uint4(w2.x, w2.y, w3.x, w3.y)), qf[2 * u + 1], s);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * h + e] = full || t0 + e < cnt[h] ? s[e] * scale_log2 : kNegInf;
  }
  float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  mx = half_swap_max(row_swap_max(mx));
  // the reference moves only where a score exceeds it by more than 2^8: the weights stay below 256
  if (__any(mx > S.m + 8.f)) {
    const float m_new = fmaxf(S.m, mx);
    const float alpha = __builtin_amdgcn_exp2f(S.m - m_new);
    S.m = m_new;
    S.l *= alpha;
#pragma unroll
    for (int n = 0; n < DH / 16; ++n) S.acc[n] *= alpha;
  }
  float p[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = __builtin_amdgcn_exp2f(x[e] - S.m);
    S.l += p[e];
  }
  // the weights of the product with V are rounded to bf16, the type of the matrix operand; the denominator is not
  const bf16x8 pf =
      as_bf16x8(make_uint4(pack_bf2(p[0], p[1]), pack_bf2(p[2], p[3]), pack_bf2(p[4], p[5]), pack_bf2(p[6], p[7])));
  // places that do not count may hold NaN codes, and zero times NaN is NaN
  const uint32_t keep[2] = {full ? ~0u : keep_bytes(cnt[0] - t0), full ? ~0u : keep_bytes(cnt[1] - t0)};
#pragma unroll
  for (int u = 0; u < DH / 64; ++u) {
    const uint32_t ca[4] = {R.v[0][u].x, R.v[0][u].y, R.v[0][u].z, R.v[0][u].w};
    const uint32_t cb[4] = {R.v[1][u].x, R.v[1][u].y, R.v[1][u].z, R.v[1][u].w};
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint2 va = e4m3x4_to_bf16(ca[n] & keep[0], vs[0]), vb = e4m3x4_to_bf16(cb[n] & keep[1], vs[1]);
      S.acc[4 * u + n] = mfma16x16x32(as_bf16x8(make_uint4(va.x, va.y, vb.x, vb.y)), pf, S.acc[4 * u + n]);
    }
  }
}

// Split-K decode: one wavefront per part of a (sequence, kv-head) stream, its 16 columns the heads of the group.
template <int DH>
__global__ __launch_bounds__(64) void kv8_decode_kernel(Kv8AttnArgs a) {
  const int lane = threadIdx.x;
  const int target = decode_target(a, lane);
  // this wavefront's sequence: parts come sequence by sequence, then head by head
  int item = blockIdx.x, b = -1, n_parts = 0;
  for (int i0 = 0; i0 < a.S; i0 += kWave) {
    const int mine = i0 + lane < a.S ? kv8_parts(pages_of(ctx_of(a, i0 + lane)), target) : 0;
    const int upto = wave_scan(mine);
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (item < all * a.Hkv) {
      const int at = __builtin_ctzll(__ballot(item < upto * a.Hkv));
      n_parts = __builtin_amdgcn_readlane(mine, at);
      item -= (__builtin_amdgcn_readlane(upto, at) - n_parts) * a.Hkv;
      b = i0 + at;
      break;
    }
    item -= all * a.Hkv;
  }
  if (b < 0) return;
  const int kvh = item / n_parts, part = item - kvh * n_parts;
  const int n = ctx_of(a, b), n_pages = pages_of(n);
  const int len = kv8_part_pages(n_pages, target);
  const int p0 = part * len, np = min(len, n_pages - p0);   // pages [p0, p0 + np)
  const int G = a.Hq / a.Hkv;
  const int col = lane & 15, rq = lane >> 4;
  const bool ok = col < G;
  bf16x8 qf[DH / 32];
  {
    const uint16_t* q = a.q + b * a.q_stride + (kvh * G + (ok ? col : 0)) * DH + rq * 16;
#pragma unroll
    for (int s = 0; s < DH / 32; ++s)
      qf[s] = ok ? as_bf16x8(*reinterpret_cast<const uint4*>(q + (s >> 1) * 64 + (s & 1) * 8)) : as_bf16x8(make_uint4(0, 0, 0, 0));
  }
  const int32_t* bt = a.bt + (size_t)b * a.bt_stride + p0;
  const float* ksp = a.pool.ks + kvh * a.pool.n_blocks;
  const float* vsp = a.pool.vs + kvh * a.pool.n_blocks;
  // Tables of 64 pages, one page a lane: the numbers of the pages being loaded and of the 64 after them, and the
  // scales of the pages being loaded and of those being multiplied.  A scale of 0 marks an entry that is no page.
  auto entries = [&](int r0) { return r0 + lane < np ? bt[r0 + lane] : 0; };
  int blk = entries(0), blk_next = entries(kWave);
  float ks_next, vs_next;
  auto scales = [&]() {
    const bool there = (uint32_t)blk < (uint64_t)a.pool.n_blocks;
    if (!there) blk = 0;
    ks_next = there ? ksp[blk] : 0.f;
    vs_next = there ? vsp[blk] : 0.f;
  };
  scales();
  float ks_now = ks_next, vs_now = vs_next;
  Kv8State<DH> S;
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) S.acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  S.m = -1e30f;   // finite, so that a column without keys keeps zero weights
  S.l = 0.f;
  constexpr int NB = 3;   // pairs of pages in registers: one multiplied, two on their way
  Kv8Pair<DH> R[NB];
  auto issue = [&](Kv8Pair<DH>& P, int r) __attribute__((always_inline)) {
    if (r && r % kWave == 0) {
      blk = blk_next;
      blk_next = entries(r + kWave);
      scales();
    }
    const int ba = __builtin_amdgcn_readlane(blk, r % kWave);
    const int bb = r + 1 < np ? __builtin_amdgcn_readlane(blk, r % kWave + 1) : ba;
    kv8_load_page<DH>(P, 0, a, kvh, ba, lane);
    kv8_load_page<DH>(P, 1, a, kvh, bb, lane);
  };
  auto multiply = [&](const Kv8Pair<DH>& P, int r) __attribute__((always_inline)) {
    if (r && r % kWave == 0) {
      ks_now = ks_next;
      vs_now = vs_next;
    }
    float ks[2], vs[2];
    int cnt[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s = __builtin_amdgcn_readlane(__float_as_int(ks_now), r % kWave + h);
      const bool there = s != 0 && r + h < np;
      ks[h] = there ? __int_as_float(s) : 1.f;
      vs[h] = there ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vs_now), r % kWave + h)) : 1.f;
      cnt[h] = there ? min(kPage, n - (p0 + r + h) * kPage) : 0;
    }
    kv8_pair<DH>(S, P, qf, ks, vs, cnt, a.scale_log2, lane);
  };
  static_for<NB - 1>([&](auto ic) {
    constexpr int J = decltype(ic)::value;
    if (2 * J < np) issue(R[J], 2 * J);
  });
  for (int r = 0; r < np; r += 2 * NB) {
    static_for<NB>([&](auto ic) {
      constexpr int J = decltype(ic)::value;
      const int rj = r + 2 * J;
      if (rj < np) {
        if (rj + 2 * (NB - 1) < np) issue(R[(J + NB - 1) % NB], rj + 2 * (NB - 1));
        multiply(R[J], rj);
      }
    });
  }
  S.l += __shfl_xor(S.l, 16, kWave);
  S.l += __shfl_xor(S.l, 32, kWave);
  if (!ok) return;
  // the lane's dimensions are u*64 + 16*rq + 4e + n: 16 successive ones for each u
  if (n_parts == 1) {
    const float inv = S.l == 0.f ? 0.f : 1.f / S.l;
    uint16_t* o = a.out + b * a.out_stride + (kvh * G + col) * DH + rq * 16;
#pragma unroll
    for (int u = 0; u < DH / 64; ++u) {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[2 * e] = pack_bf2(S.acc[4 * u][e] * inv, S.acc[4 * u + 1][e] * inv);
        w[2 * e + 1] = pack_bf2(S.acc[4 * u + 2][e] * inv, S.acc[4 * u + 3][e] * inv);
      }
      *reinterpret_cast<uint4*>(o + u * 64) = make_uint4(w[0], w[1], w[2], w[3]);
      *reinterpret_cast<uint4*>(o + u * 64 + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
    return;
  }
  const size_t slot = (size_t)blockIdx.x * G + col;
  float* o = reinterpret_cast<float*>(a.ws) + slot * DH + rq * 16;
#pragma unroll
  for (int u = 0; u < DH / 64; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<float4*>(o + u * 64 + 4 * e) =
          make_float4(S.acc[4 * u][e], S.acc[4 * u + 1][e], S.acc[4 * u + 2][e], S.acc[4 * u + 3][e]);
  if (rq == 0) reinterpret_cast<float2*>(a.ws + a.ws_ml)[slot] = make_float2(S.m, S.l);
}

// Joins the parts of one (sequence, head) per wavefront; zeros for an empty context.
template <int DH>
__global__ __launch_bounds__(256) void kv8_merge_kernel(Kv8AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int job = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (job >= a.S * a.Hq) return;
  const int b = job / a.Hq, head = job - b * a.Hq;
  constexpr int PER = DH / 64;   // dimensions a lane
  uint16_t* out = a.out + b * a.out_stride + head * DH + lane * PER;
  const int n_pages = pages_of(ctx_of(a, b));
  if (n_pages == 0) {
#pragma unroll
    for (int k = 0; k < PER; ++k) out[k] = 0;
    return;
  }
  const int target = decode_target(a, lane);
  const int n = kv8_parts(n_pages, target);
  if (n == 1) return;
  int before = 0;
  for (int i0 = 0; i0 < b; i0 += kWave)
    before += __builtin_amdgcn_readlane(
        wave_scan(i0 + lane < b ? kv8_parts(pages_of(ctx_of(a, i0 + lane)), target) : 0), 63);
  const int G = a.Hq / a.Hkv, kvh = head / G;
  const size_t first = ((size_t)before * a.Hkv + (size_t)kvh * n) * G + head - kvh * G;
  const float2* ml = reinterpret_cast<const float2*>(a.ws + a.ws_ml) + first;
  const float* o = reinterpret_cast<const float*>(a.ws) + first * DH + lane * PER;
  float M = -1e30f;
  for (int j = lane; j < n; j += kWave) M = fmaxf(M, ml[(size_t)j * G].x);
  M = wave_max(M);
  float L = 0.f, acc[PER] = {};
  for (int j = 0; j < n; ++j) {
    const float2 v = ml[(size_t)j * G];
    const float w = __builtin_amdgcn_exp2f(v.x - M);
    L += w * v.y;
#pragma unroll
    for (int k = 0; k < PER; ++k) acc[k] += w * o[(size_t)j * G * DH + k];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  if constexpr (PER == 2) *reinterpret_cast<uint32_t*>(out) = pack_bf2(acc[0] * inv, acc[1] * inv);
  else out[0] = f2bf(acc[0] * inv);
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

// Partial outputs [items][G][dh], then their (maximum, sum) pairs
static int64_t decode_ml_offset(int B, int Hq, int Hkv, int dh) { return kv8_decode_items(B, Hkv) * (Hq / Hkv) * dh * 4; }
int64_t kv8_decode_ws_bytes(int B, int Hq, int Hkv, int dh) {
  return decode_ml_offset(B, Hq, Hkv, dh) + kv8_decode_items(B, Hkv) * (Hq / Hkv) * 8;
}
int64_t kv8_prefill_ws_bytes(int, int, int, int, int) { return 256; }

hipError_t kv8_decode_launch(const Kv8AttnArgs& args, hipStream_t st) {
  Kv8AttnArgs a = args;
  a.ws_ml = decode_ml_offset(a.S, a.Hq, a.Hkv, a.dh);
  const dim3 grid((unsigned)kv8_decode_items(a.S, a.Hkv)), merge((unsigned)(((int64_t)a.S * a.Hq + 3) / 4));
  if (a.dh == 128) hipLaunchKernelGGL(kv8_decode_kernel<128>, grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL(kv8_decode_kernel<64>, grid, dim3(64), 0, st, a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (a.dh == 128) hipLaunchKernelGGL(kv8_merge_kernel<128>, merge, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(kv8_merge_kernel<64>, merge, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t kv8_prefill_launch(const Kv8AttnArgs& a, hipStream_t st) {
  const dim3 grid(a.T, a.Hq);
  if (a.dh == 128) hipLaunchKernelGGL(kv8_prefill_kernel<128>, grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL(kv8_prefill_kernel<64>, grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace hxf
