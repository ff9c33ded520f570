// Attention over the 8-bit KV cache, lengths on the device.
#include "common.hpp"
#include "kernels.hpp"

namespace hxf {

namespace {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLowest = -3.0e38f;   // a reference before any score: finite, so that a column without keys keeps zero weights

constexpr int kKv8DecodeScan = 128;

// Pages of sequence b that its context reaches, and its tokens
__device__ __forceinline__ int ctx_of(const Kv8AttnArgs& a, int b) { return min(max(a.ctx[b], 0), a.bt_stride * kPage); }
__device__ __forceinline__ int pages_of(int n) { return (n + kPage - 1) / kPage; }

// The longest part of this batch (kv8_target_pages), found by every wavefront for itself from the contexts: with few
// sequences a load and a scan or two, against a launch and a round trip through memory.  Above kKv8DecodeScan
// sequences a launch of its own does it once (a.starts); us for contexts of 64 to 128 tokens, 32 + 8 heads, every
// wavefront / one launch: 64 sequences 9.5 / 12.1, 128 14.1 / 16.0, 256 16.0 / 16.8, 1024 87 / 48.5, 4096 615 / 184.
__device__ __forceinline__ int decode_target(const Kv8AttnArgs& a, int lane) {
  int64_t total = 0;
  for (int i0 = 0; i0 < a.S; i0 += kWave) {
    const int p = i0 + lane < a.S ? pages_of(ctx_of(a, i0 + lane)) : 0;
    // (64 counts of up to 2^27 pages: low and high halves apart)
    total += __builtin_amdgcn_readlane(wave_scan(p & 0xFFFFF), 63);
    total += (int64_t)__builtin_amdgcn_readlane(wave_scan(p >> 20), 63) << 20;
  }
  return (int)min(kv8_target_pages(total, a.S, a.Hkv, a.bt_stride), (int64_t)1 << 27);
}

// starts[b]: parts of a kv-head's streams before sequence b, for b = 0 .. S.  By one wavefront:
__device__ __forceinline__ void decode_starts(const Kv8AttnArgs& a, int lane) {
  const int target = decode_target(a, lane);
  int before = 0;
  for (int i0 = 0; i0 < a.S; i0 += kWave) {
    const int n = i0 + lane < a.S ? kv8_parts(pages_of(ctx_of(a, i0 + lane)), target) : 0;
    const int upto = wave_scan(n);
    if (i0 + lane < a.S) a.starts[i0 + lane] = before + upto - n;
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  if (lane == 0) a.starts[a.S] = before;
}
// ... and by a workgroup:
__global__ __launch_bounds__(1024) void kv8_decode_plan_kernel(Kv8AttnArgs a) {
  __shared__ int64_t sums[16];
  __shared__ int32_t waves[16];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t mine = 0;
  for (int b = threadIdx.x; b < a.S; b += 1024) mine += pages_of(ctx_of(a, b));
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) mine += __shfl_xor(mine, x, kWave);
  if (lane == 0) sums[w] = mine;
  __syncthreads();
  int64_t total = 0;
  for (int i = 0; i < 16; ++i) total += sums[i];
  const int target = (int)min(kv8_target_pages(total, a.S, a.Hkv, a.bt_stride), (int64_t)1 << 27);
  int base = 0;
  for (int b0 = 0; b0 < a.S; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    const int n = b < a.S ? kv8_parts(pages_of(ctx_of(a, b)), target) : 0;
    const int upto = wave_scan(n);
    __syncthreads();
    if (lane == 63) waves[w] = upto;
    __syncthreads();
    int before = base;
    for (int i = 0; i < 16; ++i) {
      if (i < w) before += waves[i];
      base += waves[i];
    }
    if (b < a.S) a.starts[b] = before + upto - n;
  }
  if (threadIdx.x == 0) a.starts[a.S] = base;
}

// The sequence whose parts, Hkv times each, hold `item` (the last whose parts begin at or before it), or -1 past the
// last one: 64 entries at a time.
__device__ __forceinline__ int seq_of_item(const Kv8AttnArgs& a, int item, int lane) {
  const int part = item / a.Hkv;   // (streams of a sequence are cut alike: Hkv times as many items as parts)
  int lo = 0, n = a.S + 1;         // entries [lo, lo + n); the answer is in them
  if (part >= a.starts[a.S]) return -1;
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave, i = lane * step;
    const uint64_t below = __ballot(i < n && a.starts[lo + (i < n ? i : 0)] <= part);
    const int k = 63 - __builtin_clzll(below);   // (entry 0 is 0: never empty at the first level, nor below it)
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
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

// The product with V runs in fp16, whose weights are rounded to 2^-11 where bf16's are to 2^-8, and V's codes are exact in
// it: with E the largest exponent of the pages' scales so far, V enters as code * 2^(its exponent - E) and the outputs are
// in units of 2^E, which moves (upwards) with the tables of 64 pages.  Codes of a page under 2^-15 of the largest scale
// become fp16 subnormals, off by up to 2^-25 of 2^E.  The weights are 2^(x - m): the reference m is set kRefBelow under
// the largest score so far and moves only when one exceeds it by kRefRange, so that they stay under 2^15, the largest is
// 2^7 or more, and one is rounded to 2^-11 of itself or to 2^-32 of the largest, whichever is more.  (Far scores count in
// coarse steps: mx - m is exact where it decides, m + kRefRange would be rounded.  Prefill's exponents, whose x is not rounded
// to fp32 as mx is, stay under 16 for scores up to 2^28.)
constexpr float kRefBelow = 7.f, kRefRange = 15.f;
constexpr int kNoExp = -127;   // exponent of an entry that is no page
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23 & 255) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return e < -126 ? 0.f : __int_as_float((127 + e) << 23); }

// A part of a stream, or of a block, leaves its outputs as the averages that they would be alone: no larger than V's values,
// where its sums may pass fp32 (weights up to 2^15, any number of them, V scales up to 2^120).  Its share (m, l) goes with
// them, l brought into [2^-13, 2^-12) by the power of two that m takes up: a join's sums, over fewer than 2^12 parts,
// stay under the largest average then.  unit_share: what turns sums in units of 2^e into averages
// (l is 1 or more).
static_assert(kKv8Resident + 1 < 1 << 12 && kPrefillResident + 1 < 1 << 12, "parts of a stream, and of a block");
__device__ __forceinline__ float unit_share(float l, int e) { return l == 0.f ? 0.f : __builtin_amdgcn_ldexpf(1.f, e) / l; }
__device__ __forceinline__ float2 part_share(float m, float l) {
  return make_float2(m + (float)__builtin_amdgcn_frexp_expf(l), __builtin_amdgcn_frexp_mantf(l) * 0x1p-12f);
}

template <int DH>
struct Kv8State {
  f32x4 acc[DH / 16];   // tile (u, n): row r of the lane's column is dimension u*64 + r*4 + n
  float m, l;           // reference of the column's scores (log2 units); the lane's part of the denominator
};

// Scores, online softmax and PV product of one pair.  ks: the pages' K scales; vs: what their V codes are
// multiplied by; cnt: their tokens that count.
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
  if (__any(mx - S.m > kRefRange)) {
    const float m_new = fmaxf(S.m, mx - kRefBelow);
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
  // the weights of the product with V are rounded to fp16, the denominator's are not
  const f16x8 pf =
      as_f16x8(make_uint4(pack_h2(p[0], p[1]), pack_h2(p[2], p[3]), pack_h2(p[4], p[5]), pack_h2(p[6], p[7])));
  // places that do not count may hold NaN codes, and zero times NaN is NaN
  const uint32_t keep[2] = {full ? ~0u : keep_bytes(cnt[0] - t0), full ? ~0u : keep_bytes(cnt[1] - t0)};
#pragma unroll
  for (int u = 0; u < DH / 64; ++u) {
    const uint32_t ca[4] = {R.v[0][u].x, R.v[0][u].y, R.v[0][u].z, R.v[0][u].w};
    const uint32_t cb[4] = {R.v[1][u].x, R.v[1][u].y, R.v[1][u].z, R.v[1][u].w};
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint2 va = e4m3x4_to_f16(ca[n] & keep[0], vs[0]), vb = e4m3x4_to_f16(cb[n] & keep[1], vs[1]);
      S.acc[4 * u + n] = mfma16x16x32(as_f16x8(make_uint4(va.x, va.y, vb.x, vb.y)), pf, S.acc[4 * u + n]);
    }
  }
}

// Split-K decode: one wavefront per part of a (sequence, kv-head) stream, its 16 columns the heads of the group.  Bound by
// HBM: 64 contexts of 1-8k tokens (451 MB) in 78 us, 5.8 of the 6.0 TB/s that a plain read reaches.
template <int DH, bool PLANNED>
__device__ __forceinline__ void decode_part(const Kv8AttnArgs& a, int lane) {
  // this wavefront's sequence: parts come sequence by sequence, then head by head
  int item = blockIdx.x, b = -1, n_parts = 0;
  if (PLANNED) {
    b = seq_of_item(a, item, lane);
    if (b < 0) return;
    const int first = a.starts[b];
    n_parts = a.starts[b + 1] - first;
    item -= first * a.Hkv;
  } else {
    const int target = decode_target(a, lane);
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
  }
  const int kvh = item / n_parts, part = item - kvh * n_parts;
  const int n = ctx_of(a, b), n_pages = pages_of(n);
  const int len = (n_pages + n_parts - 1) / n_parts;   // (what kv8_part_pages made the parts of)
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
  // scales of the pages being loaded and of those being multiplied.  An entry that is no page reads page 0, whose tokens do
  // not count.
  auto entries = [&](int r0) { return r0 + lane < np ? bt[r0 + lane] : -1; };
  int blk = entries(0), blk_next = entries(kWave);
  float ks_next, vs_next;
  uint64_t gone_next;    // the entries that are no page
  int e_next = kNoExp;   // E of the tables being loaded; of those multiplied: e_now
  auto scales = [&]() {
    const bool there = (uint32_t)blk < (uint64_t)a.pool.n_blocks;
    gone_next = __ballot(!there);
    if (!there) blk = 0;
    ks_next = ksp[blk];
    const int e = there ? exponent_of(vsp[blk]) : kNoExp;
    e_next = max(e_next, wave_max(e));
    vs_next = power_of_two(e - e_next);
  };
  scales();
  float ks_now = ks_next, vs_now = vs_next;
  uint64_t gone_now = gone_next;
  int e_now = e_next;
  Kv8State<DH> S;
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) S.acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  S.m = kLowest;
  S.l = 0.f;
  // Pairs of pages in registers: one multiplied, one asked for.  The loads stand under a branch, so the compiler counts them
  // as if they had not been issued: of the two pairs of a turn the first waits for both, and it is the other wavefronts of
  // the SIMD that hide this.  (So does the first pair for the scales.)  A third pair takes the registers of a third wavefront,
  // which hides more: 128 contexts of 1.5-3k tokens, 32 + 8 heads, 109 us against 118, 97 of 4.5-9k 226 against 238.
  constexpr int NB = 2;
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
      gone_now = gone_next;
      if (e_now != e_next) {
        const float f = power_of_two(e_now - e_next);
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) S.acc[i] *= f;
        e_now = e_next;
      }
    }
    float ks[2], vs[2];
    int cnt[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = r % kWave + h;   // (past the part's last page: an entry that is none)
      ks[h] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ks_now), i));
      vs[h] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vs_now), i));
      cnt[h] = gone_now >> i & 1 ? 0 : min(kPage, n - (p0 + r + h) * kPage);
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
  const float inv = unit_share(S.l, e_now);
  if (n_parts == 1) {
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
          make_float4(S.acc[4 * u][e] * inv, S.acc[4 * u + 1][e] * inv, S.acc[4 * u + 2][e] * inv,
                      S.acc[4 * u + 3][e] * inv);
  if (rq == 0) reinterpret_cast<float2*>(a.ws + a.ws_ml)[slot] = part_share(S.m, S.l);
}

template <int DH, bool PLANNED>
__global__ __launch_bounds__(64) void kv8_decode_kernel(Kv8AttnArgs a) {
  const int lane = threadIdx.x, b = blockIdx.x;
  const int n = b < a.S ? a.ctx[b] : 1;   // (looked at when the work is done)
  if (!PLANNED && blockIdx.x == gridDim.x - 1) decode_starts(a, lane);   // for the join: the last seldom has a part
  decode_part<DH, PLANNED>(a, lane);
  if (n > 0) return;
  // sequence b is empty: zeros
  uint16_t* out = a.out + b * a.out_stride;
  for (int i = lane * 8; i < a.Hq * DH; i += 64 * 8) *reinterpret_cast<uint4*>(out + i) = make_uint4(0, 0, 0, 0);
}

// Joins the parts of a sequence's heads.  A thread owns four dimensions and every R-th part, four of them in flight, with a
// running maximum; the streams of a wavefront meet by exchanges between lanes, those of wavefronts in LDS.  A wavefront
// takes a head, unless that would leave CUs without a workgroup and the tables are long enough for more than kMergeAlone
// parts: then a workgroup takes a head, or, with up to kMergeWide such workgroups, a quarter of its dimensions.
// Both launches, 32 + 8 heads, us: 64 sequences of up to 12 parts, a wavefront a head 83.0, a workgroup 83.3; a context of
// 30000 tokens (125 parts), quarters 17.9, whole heads 20.2, a wavefront 29.7; 64000 (182 parts) 30.1 / 33.2 / 46.1; 8191 (64
// parts) 11.3 / 12.0 / 16.5; 16 contexts of 100 to 1500, a workgroup a head 10.2, a wavefront 11.3.
constexpr int kMergeAlone = 16;
constexpr int kMergeWide = 1024;
template <int DH>
struct MergeState {
  float M = kLowest, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  // x: averages of a part, or (sums) what another stream summed up
  template <bool SUMS>
  __device__ __forceinline__ void fold(float2 v, float4 x) {
    const float m = fmaxf(M, v.x);
    const float sc = __builtin_amdgcn_exp2f(M - m), at_m = __builtin_amdgcn_exp2f(v.x - m);
    const float l = at_m * v.y, w = SUMS ? at_m : l;
    M = m;
    L = L * sc + l;
    acc.x = acc.x * sc + w * x.x;
    acc.y = acc.y * sc + w * x.y;
    acc.z = acc.z * sc + w * x.z;
    acc.w = acc.w * sc + w * x.w;
  }
  // parts r, r + R, ... of n; part j at ml[j * G] and o + j * G * DH
  __device__ __forceinline__ void take(const float2* ml, const float* o, int G, int n, int r, int R) {
    for (int j0 = r; j0 < n; j0 += 4 * R) {
      float2 v[4];
      float4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const size_t j = (size_t)min(j0 + u * R, n - 1) * G;
        v[u] = ml[j];
        x[u] = *reinterpret_cast<const float4*>(o + j * DH);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (j0 + u * R < n) fold<false>(v[u], x[u]);
    }
  }
  __device__ __forceinline__ void write(uint16_t* out) const {
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf2(acc.x * inv, acc.y * inv), pack_bf2(acc.z * inv, acc.w * inv));
  }
  // streams of lanes X, 2 X, ... apart, into each of them
  template <int X>
  __device__ __forceinline__ void fold_lanes() {
#pragma unroll
    for (int x = X; x < kWave; x *= 2) {
      const float2 v = make_float2(__shfl_xor(M, x, kWave), __shfl_xor(L, x, kWave));
      const float4 y = make_float4(__shfl_xor(acc.x, x, kWave), __shfl_xor(acc.y, x, kWave), __shfl_xor(acc.z, x, kWave),
                                   __shfl_xor(acc.w, x, kWave));
      fold<true>(v, y);
    }
  }
};

// The parts of `head` of sequence b: their number, and the first one's place
__device__ __forceinline__ int merge_parts(const Kv8AttnArgs& a, int b, int head, size_t& first) {
  const int before = a.starts[b], n = a.starts[b + 1] - before, G = a.Hq / a.Hkv;
  first = ((size_t)before * a.Hkv + (size_t)(head / G) * n) * G + head % G;
  return n;
}

// A head a wavefront
template <int DH>
__global__ __launch_bounds__(256) void kv8_merge_kernel(Kv8AttnArgs a) {
  constexpr int C = DH / 4;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (a.Hq + 3) / 4, b = blockIdx.x / groups, head = (blockIdx.x - b * groups) * 4 + w;
  if (head >= a.Hq) return;
  size_t f;
  const int n = merge_parts(a, b, head, f);
  if (n <= 1) return;
  const int c = lane % C;
  MergeState<DH> S;
  S.take(reinterpret_cast<const float2*>(a.ws + a.ws_ml) + f, reinterpret_cast<const float*>(a.ws) + f * DH + c * 4,
         a.Hq / a.Hkv, n, lane / C, kWave / C);
  S.template fold_lanes<C>();
  if (lane < C) S.write(a.out + b * a.out_stride + head * DH + c * 4);
}

// DH / Q dimensions of a head a workgroup
template <int DH, int Q>
__global__ __launch_bounds__(256) void kv8_merge_wide_kernel(Kv8AttnArgs a) {
  constexpr int C = DH / 4 / Q;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = blockIdx.x / Q, b = i / a.Hq, head = i - b * a.Hq;
  size_t f;
  const int n = merge_parts(a, b, head, f);
  if (n <= 1) return;
  const int c = lane % C, d = (blockIdx.x % Q * C + c) * 4;
  __shared__ float2 s_ml[4];
  __shared__ float4 s_acc[4][C];
  MergeState<DH> S;
  S.take(reinterpret_cast<const float2*>(a.ws + a.ws_ml) + f, reinterpret_cast<const float*>(a.ws) + f * DH + d,
         a.Hq / a.Hkv, n, threadIdx.x / C, 256 / C);
  S.template fold_lanes<C>();
  if (lane < C) {
    if (lane == 0) s_ml[w] = make_float2(S.M, S.L);
    s_acc[w][lane] = S.acc;
  }
  __syncthreads();
  if (w > 0 || lane >= C) return;
  for (int j = 1; j < 4; ++j) S.template fold<true>(s_ml[j], s_acc[j][lane]);
  S.write(a.out + b * a.out_stride + head * DH + d);
}

// ------------------------------------------------------------------ prefill
// One block of queries of a sequence (up to 128 / G of them), or one part of its keys: rows [row, row + nq) at positions
// pos .. over the key tiles [t0, t1) of 32 positions, an even number of them.  slot < 0: the whole block, whose output it
// writes; otherwise the partial slot.  Every kv-head runs the same units.
struct PrefillUnit {
  int32_t seq, row, nq, pos;
  int32_t t0, t1, slot, pad;
};
// Partial slots [slot0, slot0 + n_part) of a block that was cut
struct PrefillJob {
  int32_t row, nq, slot0, n_part;
};
struct PrefillHead {
  int32_t n_units, n_jobs, pad[14];
};
struct PrefillWs {
  int64_t units, jobs, part_o, part_ml, total;   // byte offsets
  int32_t unit_cap, slots;                       // units; partial slots of a kv-head
};
PrefillWs prefill_ws(int S, int T, int Hq, int Hkv, int dh) {
  PrefillWs w;
  const int queries = prefill_queries_per_item(Hq / Hkv);
  w.unit_cap = (int32_t)kv8_prefill_unit_cap(S, T, queries, Hkv);
  w.slots = (int32_t)kv8_prefill_slots(S, T, queries, Hkv);
  auto al = [](int64_t x) { return (x + 255) & ~int64_t(255); };
  w.units = sizeof(PrefillHead);
  w.jobs = al(w.units + w.unit_cap * (int64_t)sizeof(PrefillUnit));
  w.part_o = al(w.jobs + (kCus + 1) * (int64_t)sizeof(PrefillJob));
  const int64_t rows = (int64_t)w.slots * Hkv * kPrefillPairs;
  w.part_ml = al(w.part_o + rows * dh * 4);
  w.total = w.part_ml + rows * 8;
  return w;
}

struct Kv8PrefillArgs {
  Kv8AttnArgs a;
  PrefillHead* head;
  PrefillUnit* units;
  PrefillJob* jobs;
  float* part_o;    // [Hkv][slots][128 pairs][dh]: averages (part_share)
  float* part_ml;   // [Hkv][slots][128 pairs][2]: their shares
  int unit_cap, slots, qpi;
  bool cuts;        // whether blocks may be cut
};

// What the planning kernels share.  kPlanThreads threads, a thread for each block of a batch that is cut.
constexpr int kPlanThreads = 256;
static_assert(kPlanThreads == kCus, "a thread for each block of a batch that is cut");

struct PlanLds {
  int32_t sums[kPlanThreads / kWave], pre[kPlanThreads];
};

// Exclusive sum over the workgroup
__device__ __forceinline__ int plan_scan(PlanLds& lds, int v, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int x = wave_scan(v);
  __syncthreads();
  if (lane == 63) lds.sums[w] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kPlanThreads / kWave; ++i) {
    if (i < w) before += lds.sums[i];
    all += lds.sums[i];
  }
  total = all;
  return before + x - v;
}
// The last of the entries begin[0 .. n), ascending from begin[0] <= i, that is at or before i
__device__ __forceinline__ int last_at(const int32_t* begin, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ int plan_rows(const Kv8AttnArgs& a, int s, int& r0) {
  r0 = min(max(a.row0[s], 0), a.T);
  return max(min(a.row0[s + 1], a.T) - r0, 0);
}
// Block j of a sequence whose rows are r0 .. r0 + n - 1, whole
__device__ __forceinline__ PrefillUnit plan_block(const Kv8AttnArgs& a, int queries, int s, int r0, int n, int j) {
  const int kcap = a.bt_stride * kPage;
  PrefillUnit u;
  u.seq = s;
  u.row = r0 + j * queries;
  u.nq = min(queries, n - j * queries);
  u.pos = min(max(a.pos0[s], -(1 << 30)), kcap) + j * queries;
  u.t0 = 0;
  u.t1 = (max(min(u.pos + u.nq, kcap), 0) + 63) / 64 * 2;
  u.slot = -1;
  u.pad = 0;
  return u;
}
// The cut of a batch of few blocks, thread b's being u (past the blocks: with t1 0)
struct PlanCut {
  uint32_t at, share;             // this thread's block: the sizes before it
  int parts, first, job;          // its parts, their first unit (and partial slot), its job
  int n_units, n_jobs;
};
__device__ __forceinline__ PlanCut plan_cut(PlanLds& lds, const Kv8AttnArgs& a, int n_blocks, const PrefillUnit& u) {
  const uint32_t size = kv8_prefill_size(u.t1, kv8_prefill_shift(a.bt_stride));
  int total, all;
  PlanCut c;
  c.at = (uint32_t)plan_scan(lds, (int)size, total);
  c.share = kv8_prefill_share((uint32_t)total, a.Hkv);
  c.parts = (int)threadIdx.x < n_blocks ? kv8_prefill_cut(c.at, size, c.share).parts : 0;
  // units and jobs number under 2^12 each: one scan
  const int n = plan_scan(lds, c.parts | (c.parts > 1) << 16, all);
  c.first = n & 0xFFFF;
  c.job = n >> 16;
  c.n_units = all & 0xFFFF;
  c.n_jobs = all >> 16;
  return c;
}
// Part k of a cut block, whose sizes begin at `at`, as unit i.  (Partial slots number under `slots` where row0 ascends.)
__device__ __forceinline__ void plan_part(PrefillUnit& u, const Kv8AttnArgs& a, uint32_t at, uint32_t share, int k, int i,
                                          int slots) {
  const int shift = kv8_prefill_shift(a.bt_stride), tiles = u.t1;
  const Kv8Cut cut = kv8_prefill_cut(at, kv8_prefill_size(tiles, shift), share);
  u.t0 = kv8_prefill_part_tile(cut, at, share, shift, tiles, k);
  u.t1 = kv8_prefill_part_tile(cut, at, share, shift, tiles, k + 1);
  u.slot = cut.parts > 1 ? min(i, slots - 1) : -1;
}
// The blocks of a batch that is cut, and the tiles of its units
struct CutLds {
  PrefillUnit whole[kCus];
  uint32_t at[kCus];
  int32_t first[kCus];
  int32_t tiles[kCus + kPrefillResident + 4] __attribute__((aligned(16)));
};
// f(unit, its place) for every unit of that batch, in the order in which they are to run: the longest first where not all
// are resident at once.
template <typename F>
__device__ __forceinline__ void plan_units(CutLds& lds, const Kv8AttnArgs& a, int n_blocks, const PrefillUnit& u,
                                           const PlanCut& c, int slots, F&& f) {
  const int tid = threadIdx.x;
  lds.whole[tid] = u;
  lds.at[tid] = c.at;
  lds.first[tid] = c.first;
  __syncthreads();
  auto unit = [&](int i) {
    const int b = last_at(lds.first, n_blocks, i);
    PrefillUnit x = lds.whole[b];
    plan_part(x, a, lds.at[b], c.share, i - lds.first[b], i, slots);
    return x;
  };
  if (c.n_units <= kv8_prefill_streams(a.Hkv)) {
    for (int i = tid; i < c.n_units; i += kPlanThreads) f(unit(i), i);
    return;
  }
  for (int i = tid; i < c.n_units + 4; i += kPlanThreads) {
    int n = -1;
    if (i < c.n_units) {
      const PrefillUnit x = unit(i);
      n = x.t1 - x.t0;
    }
    lds.tiles[i] = n;
  }
  __syncthreads();
  for (int i = tid; i < c.n_units; i += kPlanThreads) {
    const int mine = lds.tiles[i];
    int rank = 0;   // units that come before this one
#pragma unroll 4
    for (int j = 0; j < c.n_units; j += 4) {
      const int4 t = *reinterpret_cast<const int4*>(lds.tiles + j);
      rank += (t.x > mine || (t.x == mine && j < i)) + (t.y > mine || (t.y == mine && j + 1 < i)) +
              (t.z > mine || (t.z == mine && j + 2 < i)) + (t.w > mine || (t.w == mine && j + 3 < i));
    }
    f(unit(i), rank);
  }
}

// A batch of up to kPlanThreads sequences and blocks is planned by every workgroup for itself, in the time that a list
// made by a launch of its own would take to read: this makes unit `want` and returns the units' number.  The first
// workgroup leaves the jobs for the launch that joins them.  Units come longest first; and among the first resident
// workgroups the second half in reverse, so that a CU gets a long one and a short one.
struct SmallPlan {
  PlanLds scan;
  PrefillUnit unit;
  union {
    int32_t tiles[kPlanThreads];
    CutLds cut;
  };
};
__device__ __forceinline__ int plan_small(SmallPlan& lds, const Kv8PrefillArgs& p, int want) {
  const Kv8AttnArgs& a = p.a;
  const int tid = threadIdx.x, queries = p.qpi;
  int r0 = 0, total;
  const int rows = tid < a.S ? plan_rows(a, tid, r0) : 0;
  const int before = plan_scan(lds.scan, (rows + queries - 1) / queries, total);
  lds.scan.pre[tid] = before;
  __syncthreads();
  const int n = min(total, kPlanThreads);   // (more only where row0 does not ascend)
  PrefillUnit u;
  u.t1 = 0;
  if (tid < n) {
    const int s = last_at(lds.scan.pre, a.S, tid);
    const int m = plan_rows(a, s, r0);
    u = plan_block(a, queries, s, r0, m, tid - lds.scan.pre[s]);
  }
  if (!p.cuts || !kv8_prefill_cuts(n, a.Hkv)) {
    if (blockIdx.x == 0 && tid == 0) p.head->n_jobs = 0;
    if (n * a.Hkv <= kCus) {   // a CU each, in any order
      if (tid == want) lds.unit = u;
      __syncthreads();
      return n;
    }
    const int half = kPrefillResident / 2 / a.Hkv, window = min(n, kPrefillResident / a.Hkv);
    if (want >= half && want < window) want = half + window - 1 - want;
    lds.tiles[tid] = u.t1;
    __syncthreads();
    int rank = 0;   // blocks that come before this one
    for (int i = 0; i < n; ++i) {
      const int t = lds.tiles[i];
      rank += t > u.t1 || (t == u.t1 && i < tid);
    }
    if (tid < n && rank == want) lds.unit = u;
    __syncthreads();
    return n;
  }
  const PlanCut c = plan_cut(lds.scan, a, n, u);
  if (blockIdx.x == 0) {
    if (c.parts > 1) p.jobs[c.job] = PrefillJob{u.row, u.nq, c.first, c.parts};
    if (tid == 0) p.head->n_jobs = c.n_jobs;
  }
  if (c.n_units <= kv8_prefill_streams(a.Hkv)) {
    if (want >= c.first && want < c.first + c.parts) {
      plan_part(u, a, c.at, c.share, want - c.first, want, p.slots);
      lds.unit = u;
    }
  } else {
    plan_units(lds.cut, a, n, u, c, p.slots, [&](const PrefillUnit& x, int place) {
      if (place == want) lds.unit = x;
    });
  }
  __syncthreads();
  return c.n_units;
}

// The units of a larger batch, in the order above, and the jobs; one workgroup, of four wavefronts because most of its
// time is barriers (with 16 wavefronts 4.9 us for one cut chunk against 4.0).
__global__ __launch_bounds__(kPlanThreads) void kv8_prefill_plan_kernel(Kv8PrefillArgs p) {
  constexpr int kBins = 1024, kPer = kBins / kPlanThreads;
  __shared__ PlanLds lds;
  __shared__ int32_t bins[kBins];
  const Kv8AttnArgs& a = p.a;
  const int tid = threadIdx.x;
  // f(whole block, its number) for every block; the number of blocks
  auto blocks = [&](auto&& f) {
    int base = 0;
    for (int s0 = 0; s0 < a.S; s0 += kPlanThreads) {
      int r0, total;
      const int n = s0 + tid < a.S ? plan_rows(a, s0 + tid, r0) : 0;
      const int before = plan_scan(lds, (n + p.qpi - 1) / p.qpi, total);
      lds.pre[tid] = before;
      __syncthreads();
      total = kv8_prefill_take(base, total, p.unit_cap);
      for (int i = tid; i < total; i += kPlanThreads) {
        const int s = last_at(lds.pre, min(kPlanThreads, a.S - s0), i);
        const int m = plan_rows(a, s0 + s, r0);
        f(plan_block(a, p.qpi, s0 + s, r0, m, i - lds.pre[s]), base + i);
      }
      base += total;
    }
    return base;
  };
  for (int i = tid; i < kBins; i += kPlanThreads) bins[i] = 0;
  __syncthreads();
  // bin of a tile count, so that longer units come first (with under kBins tiles: in exact order)
  const int shift = max(0, 32 - __clz((a.bt_stride * kPage + 31) / 32) - 10);
  auto bin_of = [&](int tiles) { return kBins - 1 - min(tiles >> shift, kBins - 1); };
  const int n_blocks = blocks([&](const PrefillUnit& u, int) { atomicAdd(&bins[bin_of(u.t1)], 1); });
  __syncthreads();
  if (!p.cuts || !kv8_prefill_cuts(n_blocks, a.Hkv)) {
    int all, sum = 0;
    for (int k = 0; k < kPer; ++k) sum += bins[tid * kPer + k];
    int at = plan_scan(lds, sum, all);
    for (int k = 0; k < kPer; ++k) {
      const int n = bins[tid * kPer + k];
      bins[tid * kPer + k] = at;
      at += n;
    }
    __syncthreads();
    const int half = kPrefillResident / 2 / a.Hkv, window = min(n_blocks, kPrefillResident / a.Hkv);
    blocks([&](const PrefillUnit& u, int) {
      int i = atomicAdd(&bins[bin_of(u.t1)], 1);
      if (i >= half && i < window) i = half + window - 1 - i;
      p.units[i] = u;
    });
    if (tid == 0) {
      p.head->n_units = n_blocks;
      p.head->n_jobs = 0;
    }
    return;
  }
  __shared__ CutLds cut;
  blocks([&](const PrefillUnit& u, int i) { cut.whole[i] = u; });
  __syncthreads();
  PrefillUnit u;
  u.t1 = 0;
  if (tid < n_blocks) u = cut.whole[tid];
  const PlanCut c = plan_cut(lds, a, n_blocks, u);
  if (c.parts > 1) p.jobs[c.job] = PrefillJob{u.row, u.nq, c.first, c.parts};
  plan_units(cut, a, n_blocks, u, c, p.slots, [&](const PrefillUnit& x, int place) { p.units[place] = x; });
  if (tid == 0) {
    p.head->n_units = c.n_units;
    p.head->n_jobs = c.n_jobs;
  }
}

// Causal attention of a unit and kv-head, as the bf16 cache's prefill kernel computes it: the (query, head) pairs
// of the block are the columns of
//   S^T[32 keys x 32 pairs] = K[32 x dh] . Q^T[dh x 32]       (v_mfma_f32_32x32x16_bf16)
//   O^T[32 dims x 32 pairs] += V^T[32 x 32 keys] . P^T[32 x 32]   (in fp16)
// with 32 pairs per wavefront.  Every wavefront multiplies every key, so a tile of 32 keys is converted once for the
// workgroup, on its way into LDS: a thread loads DH/8 bytes of K and of V, up to two tiles ahead, into registers, and writes
// them, K as exact bf16 (the page's power of two is applied by the conversion), V's codes as fp16, in the order of the
// matrix operands.  A step multiplies K of tile t + 1 and V of tile t, so that the scores of the next tile and the
// exponentials of this one run side by side; the conversions run beside the product with V.
//
// What bounds it: at 6144 + 2048 the wavefronts' waits (28% of their cycles, MFMA busy 46%, LDS ports 35%), of which one is
// for all loads in flight, every second step (see the loop); how much of it that makes, and how much the power limit, was not
// taken apart.  2048 queries there 239-252 us by card, 0.95-1.0 PFLOP/s, where the bf16 cache's kernel takes 257.  17
// queries over 30k keys: 28 us, 2.2 TB/s, of which four are the plan and the first loads, and the steps' latency the rest.
template <int DH, bool SMALL>
__global__ __launch_bounds__(256, 2) void kv8_prefill_kernel(Kv8PrefillArgs p) {
  constexpr int KS = DH / 16;      // 16-dim steps of QK^T
  constexpr int DT = DH / 32;      // 32-dim tiles of O^T
  constexpr int KT = 32 * DH;      // elements of a K (or V) tile of 32 keys
  __shared__ __attribute__((aligned(1024))) bf16_t K0[KT], K1[KT], V0[KT], V1[KT];
  const Kv8AttnArgs& a = p.a;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroup -> (unit, head): heads innermost, so that with 8 of them an XCD works on one head's keys
  const int ui = blockIdx.x / a.Hkv, kvh = blockIdx.x - ui * a.Hkv;
  PrefillUnit it;
  if constexpr (SMALL) {
    __shared__ SmallPlan plan;
    if (ui >= plan_small(plan, p, ui)) return;
    // (what came through LDS is wavefront-uniform)
    const int32_t* u = reinterpret_cast<const int32_t*>(&plan.unit);
    int32_t* v = reinterpret_cast<int32_t*>(&it);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(PrefillUnit) / 4); ++i) v[i] = __builtin_amdgcn_readfirstlane(u[i]);
  } else {
    it = p.units[ui];   // (asked for together with the number of units; the array holds one for each workgroup)
    if (ui >= p.head->n_units) return;
  }
  const int G = a.Hq / a.Hkv;
  const int npairs = it.nq * G;
  const int kend = min(it.pos + it.nq, a.bt_stride * kPage);   // keys [0, kend) are visible to some pair
  const int tbase = it.t0, ntiles = it.t1 - it.t0;
  const int last_page = max(kend - 1, 0) / kPage;
  const int32_t* bt = a.bt + (size_t)it.seq * a.bt_stride;
  const float* ksp = a.pool.ks + kvh * a.pool.n_blocks;
  const float* vsp = a.pool.vs + kvh * a.pool.n_blocks;
  const int h = lane >> 5;

  const int pair = w * 32 + (lane & 31);
  const bool pair_ok = pair < npairs;
  const int qi = pair_ok ? pair / G : 0, hj = pair_ok ? pair % G : 0;
  const int qpos = pair_ok ? it.pos + qi : -1;   // -1: every key masked
  const int64_t row = it.row + qi;
  const int col0 = (kvh * G + hj) * DH;
  bf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)   // (a column past the pairs computes with row 0, fully masked)
    qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(a.q + row * a.q_stride + col0 + ks * 16 + h * 8));

  // What this thread moves of a tile: page pg of its two, half hw of the page's K chunks, and of V the groups of four
  // tokens hw and hw + 2 (the order in which the keys of the P^T operand lie) of DH/64 dimensions.
  const int pg = w >> 1, hw = w & 1;
  const int k_src = hw * (DH * 8) + (DH == 128 ? lane * 16 : (lane >> 5) * 256 + (lane & 15) * 16 + (lane >> 4 & 1) * 8);
  const int v_src = (hw * DH + lane * (DH / 64)) * 4;
  // Tables of 64 pages (32 tiles), one page a lane: the pages being loaded and the 64 after them, and the scales of the
  // pages being loaded and of those being stored.  (Scalar loads of each tile's entries would leave no LDS read's wait
  // without theirs.)  An entry that is no page reads page 0, whose keys `settle` masks.
  auto entries = [&](int r0) { return bt[min(tbase * 2 + r0 + lane, last_page)]; };
  int blk = 0, blk_next = 0;
  float ks_next = 0.f, vs_next = 0.f, ks_now = 0.f, vs_now = 0.f;
  // E, and the entries that are no page, of the tables being loaded, and of the tiles being multiplied
  int e_next = kNoExp, e_now = kNoExp;
  uint64_t gone_next = 0, gone_now = 0;
  auto scales = [&]() {
    const bool there = (uint32_t)blk < (uint32_t)a.pool.n_blocks;
    gone_next = __ballot(!there);
    blk = there ? blk : 0;
    const float vs = vsp[blk];
    ks_next = ksp[blk];
    const int e = there ? exponent_of(vs) : kNoExp;
    e_next = max(e_next, wave_max(e));
    vs_next = power_of_two(e - e_next);
  };
  // before K of tile t, a multiple of 32, is loaded; before K of any tile t is stored
  auto turn_loads = [&](int t) __attribute__((always_inline)) {
    blk = blk_next;
    blk_next = entries(t * 2 + kWave);
    scales();
  };
  auto turn_stores = [&](int t) __attribute__((always_inline)) {
    if ((t & 31) == 0) {
      ks_now = ks_next;
      vs_now = vs_next;
    }
  };
  // V of a tile is loaded and stored a step after its K, with the page and the scale that K looked up
  typedef uint32_t words_t[DH / 32];
  uint64_t at_last = 0;
  float vs_last = 1.f;
  // (one buffer descriptor for each page: scalar work only, and the pools may exceed 4 GiB)
  const uint8_t* k_head = a.pool.k + kv_tile(kvh, a.pool.n_blocks, 0, DH);
  const uint8_t* v_head = a.pool.v + kv_tile(kvh, a.pool.n_blocks, 0, DH);
  float scale_log2 = a.scale_log2;
  // (what the steps use, apart from the arguments' registers: those are spilled and fetched back sixteen at a time)
  asm volatile("" : "+s"(k_head), "+s"(v_head), "+s"(scale_log2));
  auto load_k = [&](words_t& R, int t) __attribute__((always_inline)) {
    at_last = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(blk, (t & 31) * 2 + pg) * (kPage * DH);
    const rsrc_t rs = make_rsrc(k_head + at_last, kPage * DH);
    if constexpr (DH == 128) {
      const uint4 x = buf_load16(rs, k_src, 0);
      R[0] = x.x; R[1] = x.y; R[2] = x.z; R[3] = x.w;
    } else {
      const uint2 x = buf_load8(rs, k_src, 0);
      R[0] = x.x; R[1] = x.y;
    }
  };
  auto load_v = [&](words_t& R) __attribute__((always_inline)) {
    const rsrc_t rs = make_rsrc(v_head + at_last, kPage * DH);
    if constexpr (DH == 128) {
      const uint2 y = buf_load8(rs, v_src, 0), z = buf_load8(rs, v_src, 8 * DH);
      R[0] = y.x; R[1] = y.y; R[2] = z.x; R[3] = z.y;
    } else {
      R[0] = buf_load4(rs, v_src, 0);
      R[1] = buf_load4(rs, v_src, 8 * DH);
    }
  };
  // K: DH/64 chunks of 8 dimensions of one token; V: 8 positions of DH/64 dimensions.  Among 32 dimensions of V the even
  // ones come first, and the halves of rows change places by bits 2 and 4 of the row, so that the 16 lanes of a read
  // (successive dimensions, 64 banks) and the 8 of a write (every second one at dh 128, 32 banks) hit distinct banks.
  auto v_row = [](int d) { return (d & ~31) | (d >> 1 & 15) | (d & 1) << 4; };
  auto v_half = [](int row, int half) { return half ^ (row >> 2 & 1) ^ (row >> 4 & 1); };
  const int k_dst = pg * (KT / 2) + (DH == 128 ? ((hw * 8 + (lane >> 4) * 2) * 16 + (lane & 15)) * 8
                                               : ((hw * 4 + (lane >> 4)) * 16 + (lane & 15)) * 8);
  auto store_v = [&](const words_t& R, bf16_t* base) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < DH / 64; ++c) {
      const int row = v_row(lane * (DH / 64) + c);
      const uint2 lo = e4m3x4_to_f16(R[c], vs_last), hi = e4m3x4_to_f16(R[DH / 64 + c], vs_last);
      *reinterpret_cast<uint4*>(base + (pg * DH + row) * 16 + v_half(row, hw) * 8) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  };
  // scales of tile t, before its K is stored (in a step: ahead of the matrix work, which waits for nothing scalar then)
  float ks_here = 1.f, vs_here = 1.f;
  auto look_up = [&](int t) __attribute__((always_inline)) {
    const int r = (t & 31) * 2 + pg;
    ks_here = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ks_now), r));
    vs_here = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vs_now), r));
  };
  auto store_k = [&](const words_t& R, bf16_t* base) __attribute__((always_inline)) {
    vs_last = vs_here;
#pragma unroll
    for (int c = 0; c < DH / 64; ++c) {
      const uint2 lo = e4m3x4_to_bf16(R[2 * c], ks_here), hi = e4m3x4_to_bf16(R[2 * c + 1], ks_here);
      *reinterpret_cast<uint4*>(base + k_dst + c * 128) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  };

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  float m = kLowest, l = 0.f;
  const int k_off = ((lane & 31) >> 4) * (KT / 2) + (lane & 15) * 8 + h * 128;
  const int v_off = v_row(lane & 31) * 16 + v_half(v_row(lane & 31), h) * 8;
  bf16x8 kf[KS];
  auto read_k = [&](const bf16_t* base) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(base + k_off + ks * 256));
  };
  auto scores = [&]() __attribute__((always_inline)) {
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) x = mfma32x32x16(kf[ks], qf[ks], x);
    return x;
  };
  // largest scaled score of the pair (the scale is positive)
  auto score_max = [&](const f32x16& x) __attribute__((always_inline)) {
    float v = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) v = fmaxf(v, x[r]);
    return half_swap_max(v) * scale_log2;
  };
  // NaN in V of a tile with masked keys (one that some pairs see and others do not, or a place past the context, which
  // may hold anything): a weight of zero would spread it to pairs that do not see its key.  So the tile's NaN become
  // zeros in LDS, and infinities are added where a pair sees one, as
  //   (2 where V is NaN)^T . (2^127 where the key is seen),
  // which the end turns into NaN: nothing else in the outputs is infinite.
  // Every wavefront looks at the whole tile, so all of them take the branch with the barriers, or none.  (V's codes are
  // at most 448 in fp16, whose two highest exponent bits are set together in NaN alone.)  The look costs 1% of the time
  // at 6144 + 2048, 2% for chunks of 5 to 256 queries over 4000 keys; one at the codes on their way into LDS, a step
  // ahead, cost 3% and 6%.
  auto nan_bits = [](uint32_t x) { return x & x << 1 & 0x40004000u; };   // (as bf16: 2)
  auto spread_nan = [&](bf16_t* base, int k0, uint32_t miss) __attribute__((always_inline)) {
    uint32_t any = 0;
    const uint4* words = reinterpret_cast<const uint4*>(base) + lane;
#pragma unroll 2
    for (int i = 0; i < KT / 8; i += kWave)
      any |= nan_bits(words[i].x) | nan_bits(words[i].y) | nan_bits(words[i].z) | nan_bits(words[i].w);
    if (!__any(any != 0)) return;
    bf16x8 seen[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = k0 + (r >> 2) * 8 + h * 4 + (r & 3);
      seen[r >> 3][r & 7] = key > qpos || key >= kend || (miss >> (r >> 3) & 1) ? (__bf16)0.f : (__bf16)0x1p127f;
    }
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint4 v = *reinterpret_cast<const uint4*>(base + v_off + (st * DH + dt * 32) * 16);
        const uint4 n = make_uint4(nan_bits(v.x), nan_bits(v.y), nan_bits(v.z), nan_bits(v.w));
        o[dt] = mfma32x32x16(as_bf16x8(n), seen[st], o[dt]);
      }
    __syncthreads();
    for (int i = threadIdx.x; i < KT / 2; i += 256) {
      const uint32_t x = reinterpret_cast<uint32_t*>(base)[i];
      reinterpret_cast<uint32_t*>(base)[i] = x & ~((nan_bits(x) >> 14) * 0xFFFFu);
    }
    __syncthreads();
  };
  // the mask of a tile that needs one, then the reference
  auto settle = [&](f32x16& x, float& mx, bf16_t* v_now, int t) __attribute__((always_inline)) {
    const int k0 = (tbase + t) * 32;
    const uint32_t miss = (uint32_t)(gone_now >> ((t & 31) * 2)) & 3;
    if (k0 + 32 > kend || k0 + 31 > it.pos || miss) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = k0 + (r >> 2) * 8 + h * 4 + (r & 3);
        if (key > qpos || key >= kend || (miss >> (r >> 3) & 1)) x[r] = kNegInf;
      }
      mx = score_max(x);
      spread_nan(v_now, k0, miss);
    }
    if (__any(mx - m > kRefRange)) {
      const float m_new = fmaxf(m, mx - kRefBelow);
      const float alpha = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
    }
  };
  uint4 vv[2][DT];
  auto read_v = [&](const bf16_t* base) __attribute__((always_inline)) {
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vv[st][dt] = *reinterpret_cast<const uint4*>(base + v_off + (st * DH + dt * 32) * 16);
  };
  f16x8 pf[2];
  auto probs = [&](const f32x16& x) __attribute__((always_inline)) {
    float ps = 0.f;
    float pv[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      pv[r] = __builtin_amdgcn_exp2f(fmaf(x[r], scale_log2, -m));
      ps += pv[r];
    }
    l += ps;
    // the weights of the product with V are rounded to fp16, the denominator's are not
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      f16x8 v;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (_Float16)pv[st * 8 + j];
      pf[st] = v;
    }
  };
  auto accumulate = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32x32x16(as_f16x8(vv[st][dt]), pf[st], o[dt]);
  };

  // order of a step's matrix work: the K reads, then QK^T of the next tile one MFMA at a time with a V read and the
  // exponentials between, then V^T . P^T with the conversions of the tiles to come, their LDS writes and the sums
  auto interleave = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_group_barrier(0x100, KS, 0);   // LDS reads
    __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);    // VALU
    __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);    // exponentials
    static_for<KS>([&](auto) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 16 * 3 / KS / 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x400, 16 / KS, 0);
    });
    static_for<2 * DT>([&](auto ic) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
      if (decltype(ic)::value % 2) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);   // LDS write
    });
  };

  if (ntiles > 0) {
    words_t RK0, RK1, RV0, RV1;   // tiles on their way: K of two, V of two
    blk_next = entries(0);
    turn_loads(0);
    turn_stores(0);
    auto in_order = [] { __builtin_amdgcn_sched_barrier(0); };   // (the loads' order is what the waits count)
    load_k(RK0, 0);
    load_v(RV0);
    load_k(RK1, 1);
    in_order();
    load_v(RV1);
    in_order();
    look_up(0);
    store_k(RK0, K0);
    load_k(RK0, 2);
    in_order();
    store_v(RV0, V0);
    load_v(RV0);
    in_order();
    look_up(1);
    store_k(RK1, K1);
    load_k(RK1, 3);
    in_order();
    __syncthreads();
    read_k(K0);
    f32x16 s = scores();
    float mx = score_max(s);
    __syncthreads();
    // a step: V of tile t + 1 and K of t + 2 into LDS, V of t + 3 and K of t + 4 on their way, scores of t + 1, output of t.
    // Past the last tile it moves and scores the last page again, which nothing uses: no step has a branch around
    // its loads, so that the second of a turn's two steps counts those in flight.  The first begins with a wait for all of
    // them: turn_stores chooses among scales whose loads may be the newest, from between two rounds of the loop.
    auto step = [&](words_t& rk, words_t& rv, bf16_t* k_now, bf16_t* k_next, bf16_t* v_now, bf16_t* v_next, int t)
        __attribute__((always_inline)) {
      turn_stores(t + 2);
      look_up(t + 2);
      if ((t & 31) == 0) {   // (t + 4 is no multiple of 32: e_next is that of tile t's table)
        gone_now = gone_next;
        if (e_now != e_next) {
          const float f = power_of_two(e_now - e_next);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[dt][e] *= f;
          e_now = e_next;
        }
      }
      settle(s, mx, v_now, t);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);   // over the other workgroup's wavefront while that moves tiles
      read_k(k_next);
      read_v(v_now);
      probs(s);
      const f32x16 next = scores();
      accumulate();
      store_v(rv, v_next);
      store_k(rk, k_now);
      mx = score_max(next);
      s = next;
      interleave();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      load_v(rv);
      load_k(rk, t + 4);
      __syncthreads();
    };
    // (the tables turn outside of the loop over steps; ntiles is even)
    for (int t = 0;;) {
      const int stop = min(ntiles, ((t + 4) | 31) - 3);   // the next t with t + 4 a multiple of 32
      do {
        step(RK0, RV1, K0, K1, V0, V1, t);
        step(RK1, RV0, K1, K0, V1, V0, t + 1);
        t += 2;
      } while (t < stop);
      if (t >= ntiles) break;
      turn_loads(t + 4);
    }
  }

#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = fmaf(o[dt][e], 0.f, o[dt][e]);   // infinity to NaN (see spread_nan)
  const float lt = l + __shfl_xor(l, 32, kWave);
  if (!pair_ok) return;
  const float inv = unit_share(lt, e_now);
  if (it.slot >= 0) {
    const size_t slot = ((size_t)kvh * p.slots + it.slot) * kPrefillPairs + pair;
    float* po = p.part_o + slot * DH;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<float4*>(po + dt * 32 + g4 * 8 + h * 4) =
            make_float4(o[dt][g4 * 4] * inv, o[dt][g4 * 4 + 1] * inv, o[dt][g4 * 4 + 2] * inv, o[dt][g4 * 4 + 3] * inv);
    if (h == 0) *reinterpret_cast<float2*>(p.part_ml + slot * 2) = part_share(m, lt);
    return;
  }
  uint16_t* out = a.out + row * a.out_stride + col0;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      *reinterpret_cast<uint2*>(out + dt * 32 + g4 * 8 + h * 4) =
          make_uint2(pack_bf2(o[dt][g4 * 4] * inv, o[dt][g4 * 4 + 1] * inv),
                     pack_bf2(o[dt][g4 * 4 + 2] * inv, o[dt][g4 * 4 + 3] * inv));
}

// Joins the parts of cut blocks: DH/4 threads a (query, head) pair; the workgroups walk the pairs of all jobs, so that a
// launch with nothing to join (the host does not know) is short.  With few jobs, of many parts then, R streams of parts
// share a pair (17 queries over 30k keys 33 us; with one 41); with more than kMergeWalk rounds of that, a pair has one
// (512 queries at 8192 107 us; with R 120).
constexpr int kMergeWalk = 2;
template <int DH>
__global__ __launch_bounds__(256) void kv8_prefill_merge_kernel(Kv8PrefillArgs p) {
  constexpr int C = DH / 4, N = 256 / C, R = 4;
  const Kv8AttnArgs& a = p.a;
  const int G = a.Hq / a.Hkv;
  const int c = threadIdx.x % C, row = threadIdx.x / C;
  __shared__ float2 s_ml[N];
  __shared__ float4 s_acc[N][C];
  const int n_jobs = p.head->n_jobs;
  // f(job, head, pair of this thread) for every R-th row, or every row
  auto walk = [&](int streams, auto&& f) {
    const int groups = kPrefillPairs / N * streams;
    for (int i = blockIdx.x; i < n_jobs * a.Hkv * groups; i += gridDim.x) {
      const int job = i / groups, jb = job / a.Hkv, kvh = job - jb * a.Hkv;
      const PrefillJob mg = p.jobs[jb];
      const int pair0 = (i - job * groups) * (N / streams);
      if (pair0 >= mg.nq * G || mg.slot0 + mg.n_part > p.slots) continue;   // (uniform over the workgroup)
      const int pair = pair0 + row / streams;   // a pair past the block's: its slot exists, its row is not written
      const size_t slot = ((size_t)kvh * p.slots + mg.slot0) * kPrefillPairs + pair;
      MergeState<DH> S;
      S.take(reinterpret_cast<const float2*>(p.part_ml) + slot, p.part_o + slot * DH + c * 4, kPrefillPairs, mg.n_part,
             row % streams, streams);
      f(S);
      if (row % streams == 0 && pair < mg.nq * G) {
        const int qi = pair / G, hj = pair - qi * G;
        S.write(a.out + (int64_t)(mg.row + qi) * a.out_stride + (kvh * G + hj) * DH + c * 4);
      }
    }
  };
  if (n_jobs * a.Hkv * (kPrefillPairs * R / N) > kMergeWalk * (int)gridDim.x) {
    walk(1, [](MergeState<DH>&) {});
    return;
  }
  walk(R, [&](MergeState<DH>& S) {
    __syncthreads();
    if (c == 0) s_ml[row] = make_float2(S.M, S.L);
    s_acc[row][c] = S.acc;
    __syncthreads();
    if (row % R == 0)
      for (int j = 1; j < R; ++j) S.template fold<true>(s_ml[row + j], s_acc[row + j][c]);
  });
}

}  // namespace

// Partial outputs [items][G][dh], then their shares (part_share), then the starts of the sequences
static int64_t decode_ml_offset(int B, int Hq, int Hkv, int dh) { return kv8_decode_items(B, Hkv) * (Hq / Hkv) * dh * 4; }
static int64_t decode_starts_offset(int B, int Hq, int Hkv, int dh) {
  return decode_ml_offset(B, Hq, Hkv, dh) + kv8_decode_items(B, Hkv) * (Hq / Hkv) * 8;
}
int64_t kv8_decode_ws_bytes(int B, int Hq, int Hkv, int dh) {
  return decode_starts_offset(B, Hq, Hkv, dh) + ((int64_t)B + 1) * 4;
}
int64_t kv8_prefill_ws_bytes(int S, int T, int Hq, int Hkv, int dh) { return prefill_ws(S, T, Hq, Hkv, dh).total; }

template <int DH, bool PLANNED>
static hipError_t decode_launch(const Kv8AttnArgs& a, hipStream_t st) {
  if (PLANNED) {
    hipLaunchKernelGGL(kv8_decode_plan_kernel, dim3(1), dim3(1024), 0, st, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((kv8_decode_kernel<DH, PLANNED>), dim3((unsigned)kv8_decode_items(a.S, a.Hkv)), dim3(64), 0, st, a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (a.bt_stride <= kKv8WholePages) return hipSuccess;   // no context is cut
  const int64_t quads = (int64_t)a.S * ((a.Hq + 3) / 4), heads = (int64_t)a.S * a.Hq;
  if (quads >= kCus || kv8_parts(a.bt_stride, kKv8MinPages) <= kMergeAlone)
    hipLaunchKernelGGL((kv8_merge_kernel<DH>), dim3((unsigned)quads), dim3(256), 0, st, a);
  else if (heads * 4 > kMergeWide)
    hipLaunchKernelGGL((kv8_merge_wide_kernel<DH, 1>), dim3((unsigned)heads), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((kv8_merge_wide_kernel<DH, 4>), dim3((unsigned)heads * 4), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t kv8_decode_launch(const Kv8AttnArgs& args, hipStream_t st) {
  Kv8AttnArgs a = args;
  a.ws_ml = decode_ml_offset(a.S, a.Hq, a.Hkv, a.dh);
  a.starts = reinterpret_cast<int32_t*>(a.ws + decode_starts_offset(a.S, a.Hq, a.Hkv, a.dh));
  if (a.S > kKv8DecodeScan) return a.dh == 128 ? decode_launch<128, true>(a, st) : decode_launch<64, true>(a, st);
  return a.dh == 128 ? decode_launch<128, false>(a, st) : decode_launch<64, false>(a, st);
}

// whole: blocks at most
template <int DH, bool SMALL>
static hipError_t prefill_launch(const Kv8PrefillArgs& p, int64_t whole, hipStream_t st) {
  const int hkv = p.a.Hkv;
  const int64_t units = p.cuts ? p.unit_cap : std::min<int64_t>(whole, p.unit_cap);
  hipLaunchKernelGGL((kv8_prefill_kernel<DH, SMALL>), dim3((unsigned)(units * hkv)), dim3(256), 0, st, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !p.cuts) return e;
  // cut blocks, over all heads, number under kPrefillCutUnits; 256 / (dh / 4) / 4 pairs a workgroup
  const int64_t jobs = std::min<int64_t>(whole * hkv, kPrefillCutUnits);
  const int64_t groups = std::min<int64_t>(jobs * kPrefillPairs / (256 / DH), 4 * kCus);
  hipLaunchKernelGGL((kv8_prefill_merge_kernel<DH>), dim3((unsigned)groups), dim3(256), 0, st, p);
  return hipGetLastError();
}

hipError_t kv8_prefill_launch(const Kv8AttnArgs& a, hipStream_t st) {
  const PrefillWs w = prefill_ws(a.S, a.T, a.Hq, a.Hkv, a.dh);
  Kv8PrefillArgs p{};
  p.a = a;
  p.head = reinterpret_cast<PrefillHead*>(a.ws);
  p.units = reinterpret_cast<PrefillUnit*>(a.ws + w.units);
  p.jobs = reinterpret_cast<PrefillJob*>(a.ws + w.jobs);
  p.part_o = reinterpret_cast<float*>(a.ws + w.part_o);
  p.part_ml = reinterpret_cast<float*>(a.ws + w.part_ml);
  p.unit_cap = w.unit_cap;
  p.slots = w.slots;
  p.qpi = prefill_queries_per_item(a.Hq / a.Hkv);
  // A block of up to 3 kPrefillMinTiles tiles is never cut: with short tables there is nothing to join
  const int64_t whole = std::min<int64_t>((int64_t)a.T / p.qpi + a.S, INT32_MAX);
  const int most = (a.bt_stride * kPage + 63) / 64 * 2;   // tiles of the longest block there can be
  p.cuts = most > 3 * kPrefillMinTiles;
  if (a.S <= kPlanThreads && whole <= kPlanThreads)
    return a.dh == 128 ? prefill_launch<128, true>(p, whole, st) : prefill_launch<64, true>(p, whole, st);
  hipLaunchKernelGGL(kv8_prefill_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  return a.dh == 128 ? prefill_launch<128, false>(p, whole, st) : prefill_launch<64, false>(p, whole, st);
}

}  // namespace hxf
