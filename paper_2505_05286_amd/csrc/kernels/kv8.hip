// The 8-bit KV cache: tables of a batch from its lengths, and the quantised write.
#include "common.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

// Every workgroup scans the lengths of all sequences (a few KB from L2) into LDS for itself and then fills a slice of
// the rows, of the new pages and of the sequences, each by a search for its sequence: no second launch and no
// traffic between workgroups.  Bound by the latency of the loads that depend on each other (lengths, page
// numbers) and of the scan: 3.5 us for 64 rows; 96k rows of 1000 sequences take 7.4 us against 112 with one workgroup.
__global__ __launch_bounds__(1024) void slot_map_kernel(SlotMapArgs a) {
  __shared__ int32_t row0[kSlotMapMaxSeqs], page0[kSlotMapMaxSeqs], first[kSlotMapMaxSeqs];
  __shared__ int64_t sums[2][16];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int waves = blockDim.x >> 6;
  const int n_free = min(max(a.n_free[0], 0), a.free_cap);
  int64_t rows = 0, pages = 0;
  bool bad = false;
  for (int s0 = 0; s0 < a.S; s0 += blockDim.x) {
    const int s = s0 + tid;
    const int st = s < a.S ? a.start[s] : 0, n = s < a.S ? a.n_new[s] : 0;
    const int have = (int)(((int64_t)st + kPage - 1) / kPage);
    const int64_t end = ((int64_t)st + n + kPage - 1) / kPage;
    bad |= st < 0 || n < 0 || (s < a.S && end > a.bt_stride);
    const int need = bad ? 0 : (int)end - have, m = bad ? 0 : n;
    // sums over a wavefront in 32 bits, low and high halves apart; the others in 64
    const int rl = wave_scan(m & 0xFFFF), rh = wave_scan(m >> 16);
    const int pl = wave_scan(need & 0xFFFF), ph = wave_scan(need >> 16);
    const int64_t r = ((int64_t)rh << 16) + rl, p = ((int64_t)ph << 16) + pl;
    __syncthreads();   // (the sums of the round before are read)
    if (lane == 63) {
      sums[0][w] = r;
      sums[1][w] = p;
    }
    __syncthreads();
    int64_t rb = rows, pb = pages;
    for (int i = 0; i < waves; ++i) {
      if (i < w) {
        rb += sums[0][i];
        pb += sums[1][i];
      }
      rows += sums[0][i];
      pages += sums[1][i];
    }
    if (s < a.S) {
      row0[s] = (int32_t)(rb + r - m);
      page0[s] = (int32_t)(pb + p - need);
      first[s] = st;
    }
  }
  const bool ok = !__syncthreads_or(bad) && rows <= a.T && pages <= n_free;   // (also orders the LDS writes)
  const int at = blockIdx.x * blockDim.x + tid, step = gridDim.x * blockDim.x;
  // the last sequence whose rows, or pages, begin at or before i: it is the one that has any
  auto find = [&](const int32_t* begin, int i) {
    int lo = 0, hi = a.S;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (begin[mid] <= i) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  for (int t = at; t < a.T; t += step) {
    int ps = 0, sl = -1;
    if (ok && t < rows) {
      const int s = find(row0, t);
      const int st = first[s], have = (st + kPage - 1) / kPage;
      ps = st + t - row0[s];
      const int p = ps / kPage;
      const int page = p < have ? a.bt[(size_t)s * a.bt_stride + p] : a.free_pages[page0[s] + p - have];
      sl = (uint32_t)page < (1u << 27) ? page * kPage + ps % kPage : -1;
    }
    a.pos[t] = ps;
    a.slot[t] = sl;
  }
  for (int s = at; s < a.S; s += step) {
    a.row0[s] = ok ? row0[s] : 0;
    a.ctx[s] = ok ? first[s] + ((s + 1 < a.S ? row0[s + 1] : (int)rows) - row0[s]) : max(first[s], 0);
  }
  if (at == 0) {
    a.status[0] = ok ? (int32_t)pages : -1;
    a.status[1] = ok ? (int32_t)rows : 0;
    a.row0[a.S] = ok ? (int32_t)rows : 0;
  }
  if (!ok) return;
  for (int i = at; i < pages; i += step) {
    const int s = find(page0, i);
    a.bt[(size_t)s * a.bt_stride + (first[s] + kPage - 1) / kPage + i - page0[s]] = a.free_pages[i];
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

// Four values as e4m3 codes, nearest even; the first in the low byte
__device__ __forceinline__ uint32_t to_e4m3x4(float x0, float x1, float x2, float x3) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, lo, true);
}
// Four codes moved to a scale 1 / f times theirs
__device__ __forceinline__ uint32_t requantise(uint32_t c, float f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  return to_e4m3x4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// max(m, |x|) where x is finite
__device__ __forceinline__ float finite_max(float m, float x) {
  const float v = fabsf(x);
  return v < __builtin_huge_valf() ? fmaxf(m, v) : m;
}

__device__ __forceinline__ void unpack8(uint4 v, float x[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// Rotates the pairs (u, w) of dimensions i .. i + 7 and i + dh/2 ..; each product and their sum is rounded to fp32,
// so that the codes do not depend on how a compiler contracts them.
__device__ __forceinline__ void rotate8(float u[8], float w[8], const float2* cs) {
#pragma clang fp contract(off)
  const float4* c4 = reinterpret_cast<const float4*>(cs);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 c = c4[i];   // (cos, sin) of two pairs
    const float u0 = u[2 * i], w0 = w[2 * i], u1 = u[2 * i + 1], w1 = w[2 * i + 1];
    u[2 * i] = u0 * c.x - w0 * c.y;
    w[2 * i] = w0 * c.x + u0 * c.y;
    u[2 * i + 1] = u1 * c.z - w1 * c.w;
    w[2 * i + 1] = w1 * c.z + u1 * c.w;
  }
}

// The page's scale with amax of the new rows; the old one counts where the page has tokens before them
__device__ __forceinline__ float page_scale(float amax, const float* scale, bool begun, float& before) {
  const float s = scale_of(wave_max(amax));
  before = begun ? *scale : s;
  return begun ? fmaxf(s, before) : s;
}

// K (blockIdx.y < Hkv) or V of one kv-head of the run of n rows from row t on, which go to the places of `slot` on; lane
// b + r of pos_i holds the position of row r.
template <int DH>
__device__ __forceinline__ void kv8_write_run(const Kv8WriteArgs& a, int slot, int t, int n, int b, int pos_i, int lane) {
  constexpr int HALF = DH / 2, LT = DH / 16, NJ = DH / 64;   // lanes a token, tokens a lane (K)
  const int o = slot % kPage, blk = slot / kPage;
  const bool is_k = blockIdx.y < a.Hkv;
  const int h = is_k ? blockIdx.y : blockIdx.y - a.Hkv;
  const uint16_t* rows = a.qkv + (int64_t)t * a.qkv_stride + (a.Hq + (int)blockIdx.y) * DH;
  const size_t tile_at = kv_tile(h, a.pool.n_blocks, blk, DH);
  float* scale = (is_k ? a.pool.ks : a.pool.vs) + h * a.pool.n_blocks + blk;
  float before, amax = 0.f;
  if (is_k) {
    uint8_t* tile = a.pool.k + tile_at;
    const int c = lane % LT;   // dimensions 8 c .. and HALF + 8 c ..
    float u[NJ][8], w[NJ][8];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int p = lane / LT + j * (64 / LT), r = p - o;   // place in the page, row of the run
      const int ps = __shfl(pos_i, b + (r & 15), kWave);
      if (r < 0 || r >= n) continue;
      const uint16_t* x = rows + r * a.qkv_stride + c * 8;
      unpack8(*reinterpret_cast<const uint4*>(x), u[j]);
      unpack8(*reinterpret_cast<const uint4*>(x + HALF), w[j]);
      if (a.cs) rotate8(u[j], w[j], a.cs + (size_t)ps * HALF + c * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = finite_max(finite_max(amax, u[j][i]), w[j][i]);
    }
    const float s = page_scale(amax, scale, o > 0, before), inv = inverse(s);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int p = lane / LT + j * (64 / LT), r = p - o;
      uint2* lo = reinterpret_cast<uint2*>(tile + k8_offset(c * 8, p));
      uint2* hi = reinterpret_cast<uint2*>(tile + k8_offset(HALF + c * 8, p));
      if (r >= 0 && r < n) {
        const float *x = u[j], *y = w[j];
        *lo = make_uint2(to_e4m3x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                         to_e4m3x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
        *hi = make_uint2(to_e4m3x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                         to_e4m3x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
      } else if (r < 0 && s != before) {
        const float f = before * inv;
        *lo = make_uint2(requantise(lo->x, f), requantise(lo->y, f));
        *hi = make_uint2(requantise(hi->x, f), requantise(hi->y, f));
      }
    }
    if (lane == 0) *scale = s;
    return;
  }
  constexpr int VD = DH / 16;
  const int g = lane >> 4, d0 = (lane & 15) * VD;
  const int r0 = g * 4 - o;   // row of the group's first token
  uint32_t* words = reinterpret_cast<uint32_t*>(a.pool.v + tile_at) + g * DH + d0;
  const bool some = r0 + 3 >= 0 && r0 < n, all = r0 >= 0 && r0 + 3 < n;
  uint32_t old[VD];
  if (some && !all) {   // (asked for early: a decode row's word has old bytes beside the new one)
#pragma unroll
    for (int i = 0; i < VD; i += 4) *reinterpret_cast<uint4*>(old + i) = *reinterpret_cast<const uint4*>(words + i);
  }
  float x[4][VD] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (r0 + j < 0 || r0 + j >= n) continue;
    const uint16_t* v = rows + (r0 + j) * a.qkv_stride + d0;
    if constexpr (VD == 8) {
      unpack8(*reinterpret_cast<const uint4*>(v), x[j]);
    } else {
      const uint2 b = *reinterpret_cast<const uint2*>(v);
      x[j][0] = __uint_as_float(b.x << 16);
      x[j][1] = __uint_as_float(b.x & 0xFFFF0000u);
      x[j][2] = __uint_as_float(b.y << 16);
      x[j][3] = __uint_as_float(b.y & 0xFFFF0000u);
    }
#pragma unroll
    for (int i = 0; i < VD; ++i) amax = finite_max(amax, x[j][i]);
  }
  const float s = page_scale(amax, scale, o > 0, before), inv = inverse(s);
  const bool grown = o > 0 && s != before;
  if (!some && !(grown && r0 < 0)) {
    if (lane == 0) *scale = s;
    return;
  }
  if (!some) {
#pragma unroll
    for (int i = 0; i < VD; i += 4) *reinterpret_cast<uint4*>(old + i) = *reinterpret_cast<const uint4*>(words + i);
  }
  const float f = before * inv;
  // bytes of the word that are new, and that are tokens before them
  uint32_t fresh = 0, held = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    fresh |= r0 + j >= 0 && r0 + j < n ? 0xFFu << (8 * j) : 0u;
    held |= r0 + j < 0 ? 0xFFu << (8 * j) : 0u;
  }
  uint32_t out[VD];
#pragma unroll
  for (int i = 0; i < VD; ++i) {
    out[i] = to_e4m3x4(x[0][i] * inv, x[1][i] * inv, x[2][i] * inv, x[3][i] * inv);
    if (!all) {
      const uint32_t moved = grown ? requantise(old[i], f) : old[i];
      out[i] = (out[i] & fresh) | (moved & held) | (old[i] & ~(fresh | held));
    }
  }
#pragma unroll
  for (int i = 0; i < VD; i += 4) *reinterpret_cast<uint4*>(words + i) = *reinterpret_cast<const uint4*>(out + i);
  if (lane == 0) *scale = s;
}

// The same for up to four runs of one row each (decode rows), side by side in the wavefront: K takes dh/16 lanes a row, V
// 16.  mine: this lane has a row; slot, t, ps: its place, row and position.
template <int DH>
__device__ __forceinline__ void kv8_write_rows(const Kv8WriteArgs& a, bool mine, int slot, int t, int ps, int lane) {
  constexpr int HALF = DH / 2, LT = DH / 16;
  const int o = slot % kPage, blk = slot / kPage;
  const bool is_k = blockIdx.y < a.Hkv;
  const int h = is_k ? blockIdx.y : blockIdx.y - a.Hkv;
  const uint16_t* row = a.qkv + (int64_t)t * a.qkv_stride + (a.Hq + (int)blockIdx.y) * DH;
  const size_t tile_at = kv_tile(h, a.pool.n_blocks, blk, DH);
  float* scale = (is_k ? a.pool.ks : a.pool.vs) + h * a.pool.n_blocks + blk;
  const float held = mine && o > 0 ? *scale : 0.f;   // (0: the page starts afresh, and any scale is larger)
  float amax = 0.f;
  if (is_k) {
    uint8_t* tile = a.pool.k + tile_at;
    const int c = lane % LT;
    float u[8] = {}, w[8] = {};
    if (mine) {
      unpack8(*reinterpret_cast<const uint4*>(row + c * 8), u);
      unpack8(*reinterpret_cast<const uint4*>(row + HALF + c * 8), w);
      if (a.cs) rotate8(u, w, a.cs + (size_t)ps * HALF + c * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = finite_max(finite_max(amax, u[i]), w[i]);
    }
#pragma unroll
    for (int x = 1; x < LT; x *= 2) amax = fmaxf(amax, __shfl_xor(amax, x, kWave));
    if (!mine) return;
    const float s = fmaxf(scale_of(amax), held), inv = inverse(s);
    auto lo = [&](int p) { return reinterpret_cast<uint2*>(tile + k8_offset(c * 8, p)); };
    auto hi = [&](int p) { return reinterpret_cast<uint2*>(tile + k8_offset(HALF + c * 8, p)); };
    *lo(o) = make_uint2(to_e4m3x4(u[0] * inv, u[1] * inv, u[2] * inv, u[3] * inv),
                        to_e4m3x4(u[4] * inv, u[5] * inv, u[6] * inv, u[7] * inv));
    *hi(o) = make_uint2(to_e4m3x4(w[0] * inv, w[1] * inv, w[2] * inv, w[3] * inv),
                        to_e4m3x4(w[4] * inv, w[5] * inv, w[6] * inv, w[7] * inv));
    if (s != held) {
      const float f = held * inv;
      for (int p = 0; p < o; ++p) {
        const uint2 x = *lo(p), y = *hi(p);
        *lo(p) = make_uint2(requantise(x.x, f), requantise(x.y, f));
        *hi(p) = make_uint2(requantise(y.x, f), requantise(y.y, f));
      }
      if (c == 0) *scale = s;
    }
    return;
  }
  constexpr int VD = DH / 16;
  const int d0 = (lane & 15) * VD, g = o >> 2, sh = (o & 3) * 8;
  uint32_t* words = reinterpret_cast<uint32_t*>(a.pool.v + tile_at) + d0;
  float x[VD] = {};
  uint32_t old[VD] = {};
  if (mine) {
#pragma unroll
    for (int i = 0; i < VD; i += 4) *reinterpret_cast<uint4*>(old + i) = *reinterpret_cast<const uint4*>(words + g * DH + i);
#pragma unroll
    for (int i = 0; i < VD; i += 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(row + d0 + i);
      x[i] = __uint_as_float(v.x << 16);
      x[i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
      x[i + 2] = __uint_as_float(v.y << 16);
      x[i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
#pragma unroll
    for (int i = 0; i < VD; ++i) amax = finite_max(amax, x[i]);
  }
#pragma unroll
  for (int y = 1; y < 16; y *= 2) amax = fmaxf(amax, __shfl_xor(amax, y, kWave));
  if (!mine) return;
  const float s = fmaxf(scale_of(amax), held), inv = inverse(s);
  const bool grown = s != held;
  const float f = held * inv;
  const uint32_t before = (1u << sh) - 1;   // bytes of the word's earlier tokens
#pragma unroll
  for (int i = 0; i < VD; ++i) {
    const uint32_t code = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[i] * inv, 0.f, 0, false) & 0xFFu;
    const uint32_t moved = grown ? requantise(old[i], f) : old[i];
    old[i] = (moved & before) | code << sh | (old[i] & ~(before | 0xFFu << sh));
  }
#pragma unroll
  for (int i = 0; i < VD; i += 4) *reinterpret_cast<uint4*>(words + g * DH + i) = *reinterpret_cast<const uint4*>(old + i);
  if (grown) {
    for (int q = 0; q < g; ++q)
#pragma unroll
      for (int i = 0; i < VD; ++i) words[q * DH + i] = requantise(words[q * DH + i], f);
    if ((lane & 15) == 0) *scale = s;
  }
}

// A workgroup takes 16 rows and one job: K of a kv-head, V of a kv-head, or some q heads.  For K and V its wavefronts take
// the runs that begin in those rows, at most a page each, so that no two write one page and its scale is known before a
// code is: a longer run by a whole wavefront (K: a lane holds 8 rotated pairs of a token, of two tokens at dh 128; V: a
// lane holds dh/16 dimensions of four tokens, the words of the page), runs of one row up to four side by side.  Of the q
// heads a wavefront takes four rows.  Bound by latency for decode rows (a slot, then the row, scale and page, a
// reduction), by memory for prompts.  32 + 8 heads of 128, us: 64 decode rows 4.2, 1024 of them 8.5, a prompt of 1024
// rows 6.1, of 2048 and 32 decode rows 12.1 (4.0 TB/s), of 8192 42 (4.5).  A wavefront for each row instead: 4.1, 12.4,
// 10.0, 16.4, 44; runs of one row after each other: 8.6, 13.7, 6.1, 14.1, 41.
template <int DH>
__global__ __launch_bounds__(256) void kv8_write_kernel(Kv8WriteArgs a) {
  constexpr int HALF = DH / 2, LT = DH / 16, R = kWriteRows, W = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x * R;
  // lane i: row t0 - 1 + i, as far as a run that begins in this group can reach
  const int ti = t0 - 1 + lane;
  const bool in = lane <= R + 15 && ti >= 0 && ti < a.T;
  const int slot_i = in ? a.slot[ti] : -1, pos_i = in && a.cs ? a.pos[ti] : 0;
  const bool live = slot_i >= 0 && slot_i < a.pool.n_blocks * kPage && (!a.cs || (pos_i >= 0 && pos_i < a.max_pos));
  const uint64_t live_rows = __ballot(live);
  if (blockIdx.y >= 2 * a.Hkv) {
    const int head = (blockIdx.y - 2 * a.Hkv) * (64 / LT) + lane / LT, i = (lane % LT) * 8;
    if (head >= a.Hq) return;
    constexpr int N = R / W;   // rows of this wavefront
    const int b0 = 1 + wave * N;
    uint4 lo[N], hi[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (!(live_rows >> (b0 + j) & 1)) continue;
      const uint16_t* x = a.qkv + (int64_t)(t0 - 1 + b0 + j) * a.qkv_stride + head * DH + i;
      lo[j] = *reinterpret_cast<const uint4*>(x);
      hi[j] = *reinterpret_cast<const uint4*>(x + HALF);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (!(live_rows >> (b0 + j) & 1)) continue;
      if (a.cs) {
        float u[8], w[8];
        unpack8(lo[j], u);
        unpack8(hi[j], w);
        rotate8(u, w, a.cs + (size_t)__builtin_amdgcn_readlane(pos_i, b0 + j) * HALF + i);
        lo[j] = make_uint4(pack_bf2(u[0], u[1]), pack_bf2(u[2], u[3]), pack_bf2(u[4], u[5]), pack_bf2(u[6], u[7]));
        hi[j] = make_uint4(pack_bf2(w[0], w[1]), pack_bf2(w[2], w[3]), pack_bf2(w[4], w[5]), pack_bf2(w[6], w[7]));
      }
      uint16_t* q = a.q_out + (int64_t)(t0 - 1 + b0 + j) * a.q_stride + head * DH + i;
      *reinterpret_cast<uint4*>(q) = lo[j];
      *reinterpret_cast<uint4*>(q + HALF) = hi[j];
    }
    return;
  }
  // rows that continue the run of the row before them: the next place of the same page
  const int slot_b = __shfl_up(slot_i, 1, kWave);
  const bool goes_on = live && lane > 0 && (live_rows << 1 >> lane & 1) && slot_b == slot_i - 1 && slot_i % kPage;
  const uint64_t on = __ballot(goes_on);
  uint64_t leads = live_rows & ~on & (((1ull << R) - 1) << 1);
  // this wavefront's runs: every fourth; those of one row are left for the end
  int one[4] = {0, 0, 0, 0}, ones = 0;
  for (int k = 0; leads; ++k, leads &= leads - 1) {
    if (k % W != wave) continue;
    const int b = __builtin_ctzll(leads);
    const int n = 1 + __builtin_ctzll(~(on >> (b + 1)));
    if (n == 1) {
      one[3] = one[2];
      one[2] = one[1];
      one[1] = one[0];
      one[0] = b;
      ++ones;
    } else {
      kv8_write_run<DH>(a, __builtin_amdgcn_readlane(slot_i, b), t0 - 1 + b, n, b, pos_i, lane);
    }
  }
  if (!ones) return;
  const int i = lane / (blockIdx.y < a.Hkv ? LT : 16);   // (R / W = 4 runs at most)
  const int b = i == 0 ? one[0] : i == 1 ? one[1] : i == 2 ? one[2] : one[3];
  kv8_write_rows<DH>(a, i < ones, __shfl(slot_i, b, kWave), t0 - 1 + b, __shfl(pos_i, b, kWave), lane);
}

}  // namespace

hipError_t slot_map_launch(const SlotMapArgs& a, hipStream_t st) {
  // small batches in a workgroup of four wavefronts (its barriers cost less); otherwise a thread a row, and
  // no more workgroups than CUs
  const int threads = a.S <= 256 && a.T <= 256 ? 256 : 1024;
  const int64_t groups = std::min<int64_t>(std::max<int64_t>((std::max(a.S, a.T) + (int64_t)threads - 1) / threads, 1), 256);
  hipLaunchKernelGGL(slot_map_kernel, dim3((unsigned)groups), dim3(threads), 0, st, a);
  return hipGetLastError();
}

hipError_t kv8_write_launch(const Kv8WriteArgs& a, hipStream_t st) {
  if (a.T <= 0) return hipSuccess;
  const int q_heads = 64 / (a.dh / 16);   // of a wavefront
  const dim3 grid((a.T + kWriteRows - 1) / kWriteRows, 2 * a.Hkv + (a.q_out ? (a.Hq + q_heads - 1) / q_heads : 0));
  if (a.dh == 128) hipLaunchKernelGGL(kv8_write_kernel<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(kv8_write_kernel<64>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace hxf
