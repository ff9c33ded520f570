// The product of 8-bit codes C[M,N] = A[M,K] * B[N,K]^T with the weights read straight into registers.
// Instantiated by gemm_i8_*.hip, one epilogue each.
#pragma once

#include "gemm_util.hpp"

namespace hxf {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mfma16x16x64(uint4 a, uint4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Four values at an address aligned to one of them: global memory takes 8 and 16 bytes at any address.
template <typename V, typename T>
__device__ __forceinline__ V load4(const T* p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <typename V, typename T>
__device__ __forceinline__ void put4(T* p, V v) {
  __builtin_memcpy(p, &v, sizeof(V));
}

// Epilogues of four columns of one row from col on; y = float(acc) * sa * sb, in this order: the first product has
// the size of a sum of activations, while that of the two scales may pass below fp32's range.
__device__ __forceinline__ float4 load_scales(const float* s, int col, int n) {
  if (col + 3 < n) return load4<float4>(s + col);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = s[min(col + e, n - 1)];
  return make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ f32x4 scaled(i32x4 acc, float sa, float4 sb) {
  return f32x4{(float)acc[0] * sa * sb.x, (float)acc[1] * sa * sb.y, (float)acc[2] * sa * sb.z,
               (float)acc[3] * sa * sb.w};
}
// silu(g) u = g / (1 + e^-g) u of four columns.  (The reciprocal's last place is far below bf16's: a division takes ten
// instructions more.)  From -87.3 down the sum passes 2^126, where its reciprocal is subnormal (v_rcp_f32 makes it 0), and
// from -88.7 fp32's end, while silu itself is a normal number down to -91.9 and times a large u much further.  There the
// sum is e^-g to fp32's last place, and e^(g/2) on each factor keeps both in range.  Such gates are rare: a branch around
// them, its code out of the way, takes less than selects in every value (without it, with the
// branch and with selects, us: 1870 x 60000 x 256 83.1, 84.7 and 88.6; 2080 x 57344 x 8192 692, 0.5% and 1.2% more).
__device__ __forceinline__ f32x4 swiglu(f32x4 g, f32x4 u) {
  constexpr float kFar = -87.f;
  f32x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = g[e] * __builtin_amdgcn_rcpf(1.f + __expf(-g[e])) * u[e];
  if (__builtin_expect(__any(fminf(fminf(g[0], g[1]), fminf(g[2], g[3])) < kFar), 0)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float h = __expf(0.5f * g[e]);
      y[e] = g[e] < kFar ? (g[e] * h) * (h * u[e]) : y[e];
    }
  }
  return y;
}

template <int EPI>
__device__ __forceinline__ void store4(const GemmI8Args& a, int row, int col, f32x4 y) {
  const size_t o = (size_t)row * a.ldc + col;
  const bool whole = col + 3 < a.N;
  if constexpr (EPI == EPI_BF16 || EPI == EPI_SWIGLU) {
    bf16_t* c = reinterpret_cast<bf16_t*>(a.C) + o;
    if (whole) {
      put4(c, make_uint2(pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])));
    } else {
      for (int e = 0; e < 4 && col + e < a.N; ++e) c[e] = f2bf(y[e]);
    }
  } else {
    float* c = reinterpret_cast<float*>(a.C) + o;
    constexpr bool ADD = EPI == EPI_RESID;
    if (whole) {
      put4(c, ADD ? load4<f32x4>(c) + y : y);
    } else {
      for (int e = 0; e < 4 && col + e < a.N; ++e) c[e] = ADD ? c[e] + y[e] : y[e];
    }
  }
}

// Macro tiles of 16 TM rows x 16 NW WV columns on the 16x16x64 i8 MFMA: WV wavefronts, each owning all the tile's
// rows and 16 NW of its columns.  A tile of codes is a kilobyte in operand order like a packed bf16 tile, but of 64 of
// K: the weights go straight from memory to registers, R steps of 64 of K ahead, and only the activations pass
// through LDS, stages of 128 of K by buffer DMA, NS in flight.  Steps past the end of K multiply weights of zero, so
// what the activations hold there does not matter.
// Up to ~128 rows the weights' bytes are the bound (64 rows of 28672 x 4096 SwiGLU 21.3 us, 5.6 TB/s; weights that one row
// of tiles reads are fetched with the non-temporal hint); with 2080 rows the power (57344 x 8192 709 us, 2.76 P/s at
// 1.7 GHz, MFMAs busy 73% of the time; 692 to 735 us from run to run) and, in products of one round of tiles, the
// instructions between the MFMAs of a wavefront that is alone on its SIMD (4096 x 14336 112 us, 2.18 P/s, MFMAs busy 50%).
// 32x32x32 MFMAs in this scheme were 7% slower (831 us against 774, before loads were spread as below), eight stages of
// activations or weights eight steps ahead gained nothing (0-2%).
// SwiGLU: half of a wavefront's column tiles are gate and half the same columns of up, so one lane holds both.
// Weights are the first MFMA operand: a lane ends up with 4 consecutive columns of one row.
// SPLIT: grid.y cuts K into pieces of a.piece steps (even); each writes its int32 partial [M][N] (SwiGLU: gate, then
// up columns) to slot blockIdx.y of a.partial.
template <int TM, int NW, int R, int EPI, bool SPLIT, int WV, int OCC, int CACHE>
__global__ __launch_bounds__(64 * WV, OCC) void gemm_i8_kernel(GemmI8Args a) {
  constexpr bool SW = EPI == EPI_SWIGLU;
  constexpr int HALF = SW ? NW / 2 : NW;                         // column tiles of the output per wavefront
  constexpr int BM = 16 * TM, BN = 16 * HALF * WV, NS = 4;
  // Whether the loads of a step are spread over its matrix instructions.  A wavefront that is alone on its SIMD hides an
  // instruction or two behind each matrix instruction but not a row of them; spread, loads come later, which costs
  // tiles with shorter steps more than it gains (us, spread and not: 2080 x 57344 x 8192 SwiGLU in 192-row tiles
  // 724 / 768, 2080 x 10240 x 8192 in 176 137 / 150; 2080 x 4096 x 14336 in 160 122 / 109, in 144 108 / 104).
  constexpr bool SPREAD = WV == 4 && NW == 4 && TM >= 11;
  constexpr int A_BLK = TM * 2, A_PW = (A_BLK + WV - 1) / WV, STAGE = A_BLK * 1024;   // 1 KB blocks per stage, per wavefront
  // outstanding loads allowed when stage s + 1 must have landed: the younger stages' DMAs and the weight loads
  // issued since its own DMAs (without the first step's of the same pass, which may stand before the last of those)
  constexpr int WAIT = (NS - 3) * A_PW + 2 * NW * (NS - 2) - NW;
  static_assert((2 * NS) % R == 0 && WAIT < 64 && NW * R + (NS - 2) * A_PW < 64, "pipeline");
  static_assert(!SW || NW % 2 == 0, "a wavefront holds as many up columns as gate columns");
  static_assert(NS * STAGE + WV * 16 * (16 * HALF * 4 + 16) <= 160 * 1024, "stage layout");
  __shared__ __attribute__((aligned(1024))) uint8_t L0[STAGE], L1[STAGE], L2[STAGE], L3[STAGE];
  auto slot = [&](auto ic) -> uint8_t* {
    constexpr int I = decltype(ic)::value % NS;
    if constexpr (I == 0) return L0; else if constexpr (I == 1) return L1; else if constexpr (I == 2) return L2;
    else return L3;
  };
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int L = xcd_remap(blockIdx.x, tiles_m * tiles_n);
  const int tn = L / tiles_m, tm = L % tiles_m, m0 = tm * BM;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kb = SPLIT ? blockIdx.y * a.piece : 0;                 // first step
  const int kt = (SPLIT ? min(a.kt, kb + a.piece) : a.kt) - kb;    // steps
  const int nst = (kt + 1) / 2;                                    // stages

  // activation DMA: block (row tile, half) of the stage; row tiles past M repeat the last one (never stored)
  const int last_tile = (a.M - m0 - 1) / 16;
  const rsrc_t ra = make_rsrc(a.A + (size_t)(m0 / 16) * a.kt * 1024, (uint32_t)min(TM, last_tile + 1) * a.kt * 1024);
  int a_off[A_PW], a_dst[A_PW];
#pragma unroll
  for (int u = 0; u < A_PW; ++u) {
    const int b = min(w * A_PW + u, A_BLK - 1), rt = b >> 1, kk = b & 1;
    a_dst[u] = b * 1024;
    a_off[u] = (min(rt, last_tile) * a.kt + kk) * 1024 + lane * 16;
  }
  // one block of stage s; `check`: past the last stage nothing is read (by or-ing, without a branch)
  auto issue_a1 = [&](auto check, int u, int s, uint8_t* base) __attribute__((always_inline)) {
    if constexpr (decltype(check)::value)
      buf_dma16(ra, a_off[u] | (s >= nst ? kOutOfRange : 0), (kb + 2 * min(s, nst - 1)) * 1024, base + a_dst[u]);
    else
      buf_dma16(ra, a_off[u], (kb + 2 * s) * 1024, base + a_dst[u]);
  };
  auto issue_a = [&](int s, uint8_t* base) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < A_PW; ++u) issue_a1(std::true_type{}, u, s, base);
  };
  const int c0 = tn * BN + w * 16 * HALF;                          // the wavefront's first output column
  const int b_tiles = (a.N + 15) / 16, bt = min(c0 / 16, b_tiles - 1);
  const uint32_t b_bytes = (uint32_t)min(HALF, b_tiles - bt) * a.kt * 1024;
  const rsrc_t rb0 = make_rsrc(a.B + (size_t)bt * a.kt * 1024, b_bytes);
  const rsrc_t rb1 = SW ? make_rsrc(a.B2 + (size_t)bt * a.kt * 1024, b_bytes) : rb0;
  int b_off[HALF];
#pragma unroll
  for (int j = 0; j < HALF; ++j) b_off[j] = lane * 16 + j * a.kt * 1024;
  uint4 fb[R][NW];
  // `check`: past the last step zeros
  auto load_b1 = [&](auto check, auto rc, int j, int k) __attribute__((always_inline)) {
    constexpr int r = decltype(rc)::value % R;
    if constexpr (decltype(check)::value)
      fb[r][j] = buf_load16<CACHE>(j < HALF ? rb0 : rb1, b_off[j % HALF] | (k < kt ? 0 : kOutOfRange),
                                   (kb + min(k, kt - 1)) * 1024);
    else
      fb[r][j] = buf_load16<CACHE>(j < HALF ? rb0 : rb1, b_off[j % HALF], (kb + k) * 1024);
  };
  auto load_b = [&](auto rc, int k) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NW; ++j) load_b1(std::true_type{}, rc, j, k);
  };
  i32x4 acc[TM][NW];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < NW; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  uint4 fa[TM];
  auto read_a = [&](const uint8_t* base, int i, int h) __attribute__((always_inline)) {
    return *reinterpret_cast<const uint4*>(base + i * 2048 + h * 1024 + lane * 16);
  };
  // One step with the weights of ring slot r; reads the next step's fragments as it goes.  SPREAD: one at a time between
  // its matrix instructions, and with them n loads or DMAs, mem(0) .. mem(n - 1).
  auto step = [&](auto rc, const uint8_t* next, int h, auto nc, auto&& mem) __attribute__((always_inline)) {
    constexpr int r = decltype(rc)::value % R, n = decltype(nc)::value, PLACES = TM * (NW / 2);
    if constexpr (SPREAD) {
      static_for<TM * NW>([&](auto tc) {
        constexpr int i = decltype(tc)::value / NW, j = decltype(tc)::value % NW;
        acc[i][j] = mfma16x16x64(fb[r][j], fa[i], acc[i][j]);
        if constexpr (j == 0 && i > 0) fa[i - 1] = read_a(next, i - 1, h);
        if constexpr (j % 2 == 1) {
          constexpr int q = i * (NW / 2) + j / 2;
          static_for<(q + 1) * n / PLACES - q * n / PLACES>([&](auto oc) {
            mem(std::integral_constant<int, q * n / PLACES + decltype(oc)::value>{});
          });
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      fa[TM - 1] = read_a(next, TM - 1, h);
      __builtin_amdgcn_sched_barrier(0);
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < NW; ++j) acc[i][j] = mfma16x16x64(fb[r][j], fa[i], acc[i][j]);
        fa[i] = read_a(next, i, h);
      }
      static_for<TM>([&](auto) {
        __builtin_amdgcn_sched_group_barrier(0x008, NW, 0);   // MFMAs
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);    // one LDS read
      });
    }
  };
  auto nothing = [](auto) {};
  constexpr std::integral_constant<int, 0> none{};
  static_for<NS - 1>([&](auto ic) {
    issue_a(decltype(ic)::value, slot(ic));
    __builtin_amdgcn_sched_barrier(0);   // the waits below count in this order
  });
  static_for<R>([&](auto ic) { load_b(ic, decltype(ic)::value); });
  __builtin_amdgcn_sched_barrier(0);
  wait_vmcnt<NW * R + (NS - 2) * A_PW>();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int i = 0; i < TM; ++i) fa[i] = read_a(L0, i, 0);
  step(none, L0, 1, none, nothing);
  if constexpr (!SPREAD) load_b(none, R);
  __builtin_amdgcn_sched_barrier(0);
  // Pass s: the second step of stage s (it reads stage s + 1's first fragments) and the first of stage s + 1; with SPREAD
  // each loads the weights of the ring slot that the step before it used, otherwise its own.
  // Every LDS read follows, without a branch, the wait for its stage's DMA, and a loop has one exit: otherwise
  // the compiler adds waits for everything in flight.  Whole trips of 2 NS steps (with SPREAD first those that load nothing
  // past the end); a last trip that has at least three steps of its own runs on over zeros, which costs less than so
  // many single steps.
  const int s_end = (kt - 1 + 2 * NS - 3) / (2 * NS) * NS;
  int s0 = 0;
  auto trip = [&](auto check) __attribute__((always_inline)) {
    static_for<NS>([&](auto ic) {
      constexpr int J = decltype(ic)::value;
      constexpr std::integral_constant<int, 2 * J + 1> first{};
      constexpr std::integral_constant<int, 2 * J + 2> second{};
      wait_vmcnt<WAIT>();
      __builtin_amdgcn_s_barrier();
      uint8_t* fill = slot(std::integral_constant<int, J + NS - 1>{});
      const uint8_t* next = slot(std::integral_constant<int, J + 1>{});
      if constexpr (SPREAD) {
        __builtin_amdgcn_sched_barrier(0);
        step(first, next, 0, std::integral_constant<int, A_PW + NW>{}, [&](auto oc) {
          constexpr int o = decltype(oc)::value;
          if constexpr (o < A_PW) issue_a1(check, o, s0 + J + NS - 1, fill);
          else load_b1(check, std::integral_constant<int, 2 * J>{}, o - A_PW, (s0 + J) * 2 + R);
        });
        step(second, next, 1, std::integral_constant<int, NW>{}, [&](auto oc) {
          load_b1(check, first, decltype(oc)::value, (s0 + J) * 2 + 1 + R);
        });
      } else {
        issue_a(s0 + J + NS - 1, fill);
        step(first, next, 0, none, nothing);
        load_b(first, (s0 + J) * 2 + 1 + R);
        __builtin_amdgcn_sched_barrier(0);
        step(second, next, 1, none, nothing);
        load_b(second, (s0 + J) * 2 + 2 + R);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
  };
  if constexpr (SPREAD) {
    const int inside = max(0, min(kt - R - 2 * NS + 1, 2 * nst - 4 * NS + 4) + 2 * NS - 1) / (2 * NS) * NS;
    for (; s0 < inside; s0 += NS) trip(std::false_type{});
  }
  for (; s0 < s_end; s0 += NS) trip(std::true_type{});
  if constexpr (SPREAD) load_b(none, 2 * s0 + R);
  // one or two remaining steps singly, the ring shifted by copies
  auto dyn_slot = [&](int i) -> uint8_t* {
    i %= NS;
    return i == 0 ? L0 : i == 1 ? L1 : i == 2 ? L2 : L3;
  };
  for (int k = 2 * s0 + 1; k < kt; ++k) {
    if (k & 1) {
      wait_vmcnt<0>();
      __builtin_amdgcn_s_barrier();
      issue_a((k >> 1) + NS - 1, dyn_slot((k >> 1) + NS - 1));
    }
    step(std::integral_constant<int, 1>{}, dyn_slot((k >> 1) + (k & 1)), (k & 1) ^ 1, none, nothing);
#pragma unroll
    for (int j = 0; j < NW; ++j) {
#pragma unroll
      for (int r = 1; r < R; ++r) fb[r][j] = fb[(r + 1) % R][j];
    }
    load_b(std::integral_constant<int, 0>{}, k + R);
  }
  wait_vmcnt<0>();

  // A lane holds row l % 16 and columns 4 (l / 16) .. + 3 of each 16 x 16 tile.  A row tile's values pass through LDS
  // (the wavefront's own part of it), so that a store covers whole rows of the wavefront's columns instead of 16 rows'
  // pieces of 8 or 16 bytes.
  constexpr bool WIDE = SPLIT || EPI == EPI_RESID || EPI == EPI_F32;       // 4 bytes a value, or 2
  constexpr int COLS = 16 * HALF, SIZE = WIDE ? 4 : 2, PER = 16 / SIZE;    // columns, bytes a value, values per 16 bytes
  constexpr int LPR = COLS / PER, RPI = 64 / LPR < 16 ? 64 / LPR : 16;      // lanes per row, rows per store
  constexpr int INSTS = 16 / RPI;                                           // stores per row tile
  constexpr int PITCH = COLS * SIZE + 16;                                  // bytes: rows start in different banks
  __shared__ __attribute__((aligned(16))) uint8_t stage[WV][16 * PITCH];
  uint8_t* mine = stage[w];
  const int in_row = (lane & 15) * PITCH + (lane >> 4) * 4 * SIZE;          // where the lane writes, tile 0
  const int out_row = lane / LPR % RPI, out_col = lane % LPR * PER, col0 = c0 + out_col;
  const int n_all = SPLIT && SW ? 2 * a.N : a.N;
  const size_t ld = SPLIT ? n_all : a.ldc;
  uint8_t* const C = SPLIT ? reinterpret_cast<uint8_t*>(a.partial + (size_t)blockIdx.y * a.M * n_all)
                           : reinterpret_cast<uint8_t*>(a.C);
  const bool whole = col0 + PER <= a.N;
  // put(i, shift): row tile i from LDS to its rows, `shift` columns to the right (up columns of a partial)
  constexpr bool ADD = !SPLIT && EPI == EPI_RESID;
  f32x4 old[ADD ? INSTS : 1];
  auto place = [&](int i, int h, int shift) {
    return C + ((size_t)(m0 + i * 16 + h * RPI + out_row) * ld + col0 + shift) * SIZE;
  };
  auto in_rows = [&](int i, int h) { return lane < RPI * LPR && m0 + i * 16 + h * RPI + out_row < a.M; };
  auto fetch = [&](int i) {   // what the residual holds, one row tile ahead of its use
    if constexpr (ADD) {
#pragma unroll
      for (int h = 0; h < INSTS; ++h)
        if (in_rows(i, h) && whole) old[h] = load4<f32x4>(reinterpret_cast<const float*>(place(i, h, 0)));
    }
  };
  // Other lanes of the wavefront read what a lane has written: without this the compiler takes a value that its own
  // lane does not read as never read, and leaves it out
  auto exchange = [] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  auto put = [&](int i, int shift) {
    exchange();
    uint4 v[INSTS];
#pragma unroll
    for (int h = 0; h < INSTS; ++h)
      v[h] = *reinterpret_cast<const uint4*>(mine + (h * RPI + out_row) * PITCH + out_col * SIZE);
    exchange();
    f32x4 was[ADD ? INSTS : 1];
    if constexpr (ADD) {
#pragma unroll
      for (int h = 0; h < INSTS; ++h) was[h] = old[h];
      if (i + 1 < TM) fetch(i + 1);
    }
#pragma unroll
    for (int h = 0; h < INSTS; ++h) {
      if (!in_rows(i, h)) continue;
      uint8_t* c = place(i, h, shift);
      if constexpr (WIDE) {
        const f32x4 y = __builtin_bit_cast(f32x4, v[h]);
        float* f = reinterpret_cast<float*>(c);
        if (whole) {
          if constexpr (ADD) put4(f, was[h] + y); else put4(f, v[h]);
        } else {
          for (int e = 0; e < 4 && col0 + e < a.N; ++e) f[e] = ADD ? f[e] + y[e] : y[e];
        }
      } else {
        bf16_t* f = reinterpret_cast<bf16_t*>(c);
        const uint32_t u[4] = {v[h].x, v[h].y, v[h].z, v[h].w};
        if (whole) put4(f, v[h]);
        else for (int e = 0; e < 8 && col0 + e < a.N; ++e) f[e] = (bf16_t)(u[e >> 1] >> (16 * (e & 1)));
      }
    }
  };
  if constexpr (SPLIT) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int g = 0; g < NW / HALF; ++g) {
#pragma unroll
        for (int j = 0; j < HALF; ++j)
          *reinterpret_cast<i32x4*>(mine + in_row + j * 64) = acc[i][g * HALF + j];
        put(i, g * a.N);
      }
  } else {
    fetch(0);
    float4 sb[NW];
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const int col = min(c0 + (j % HALF) * 16 + (lane >> 4) * 4, a.N - 1);
      sb[j] = load_scales(j < HALF ? a.sb : a.sb2, col, a.N);
    }
    float sa[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = a.sa[min(m0 + i * 16 + (lane & 15), a.M - 1)];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < HALF; ++j) {
        f32x4 y = scaled(acc[i][j], sa[i], sb[j]);
        if constexpr (SW) {
          y = swiglu(y, scaled(acc[i][j + HALF], sa[i], sb[j + HALF]));
        }
        if constexpr (WIDE) *reinterpret_cast<f32x4*>(mine + in_row + j * 64) = y;
        else *reinterpret_cast<uint2*>(mine + in_row + j * 32) = make_uint2(pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3]));
      }
      put(i, 0);
    }
  }
}

template <int TM, int NW, int WV, int CACHE, int EPI, bool SPLIT>
hipError_t launch_i8(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
  constexpr int BM = 16 * TM, BN = 16 * (EPI == EPI_SWIGLU ? NW / 2 : NW) * WV, R = WV == 8 ? 2 : NW == 2 ? 8 : 4;
  constexpr int OCC = WV == 8 || TM <= 7 ? 2 : 1;   // wavefronts a SIMD that the registers are to leave room for
  const unsigned nb = (unsigned)((a.M + BM - 1) / BM) * (unsigned)((a.N + BN - 1) / BN);
  hipLaunchKernelGGL((gemm_i8_kernel<TM, NW, R, EPI, SPLIT, WV, OCC, CACHE>), dim3(nb, p.splits), dim3(64 * WV), 0,
                     st, a);
  return hipGetLastError();
}

template <int EPI, bool SPLIT>
hipError_t launch_i8_cfg(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
#define HXF_I8(T, NW, WV, CACHE) \
  case T: return launch_i8<T, NW, WV, CACHE, EPI, SPLIT>(a, p, st);
  if (p.nw == 2 && p.once) switch (p.tm) {
      HXF_I8(1, 2, 4, 2) HXF_I8(2, 2, 4, 2) HXF_I8(4, 2, 4, 2) HXF_I8(8, 2, 4, 2)
    }
  else if (p.nw == 2) switch (p.tm) {
      HXF_I8(3, 2, 4, 0) HXF_I8(4, 2, 4, 0) HXF_I8(5, 2, 4, 0) HXF_I8(6, 2, 4, 0) HXF_I8(7, 2, 4, 0)
      HXF_I8(8, 2, 4, 0) HXF_I8(9, 2, 4, 0) HXF_I8(10, 2, 4, 0) HXF_I8(11, 2, 4, 0) HXF_I8(12, 2, 4, 0)
    }
  else if (p.wv == 4 && p.once) switch (p.tm) {
      HXF_I8(1, 4, 4, 2) HXF_I8(2, 4, 4, 2) HXF_I8(4, 4, 4, 2) HXF_I8(6, 4, 4, 2) HXF_I8(8, 4, 4, 2)
      HXF_I8(10, 4, 4, 2) HXF_I8(12, 4, 4, 2) HXF_I8(14, 4, 4, 2) HXF_I8(16, 4, 4, 2)
    }
  else if (p.wv == 4) switch (p.tm) {
      HXF_I8(4, 4, 4, 0) HXF_I8(5, 4, 4, 0) HXF_I8(6, 4, 4, 0) HXF_I8(7, 4, 4, 0) HXF_I8(8, 4, 4, 0)
      HXF_I8(9, 4, 4, 0) HXF_I8(10, 4, 4, 0) HXF_I8(11, 4, 4, 0) HXF_I8(12, 4, 4, 0) HXF_I8(13, 4, 4, 0)
      HXF_I8(14, 4, 4, 0) HXF_I8(15, 4, 4, 0) HXF_I8(16, 4, 4, 0)
    }
  else switch (p.tm) {
      HXF_I8(5, 4, 8, 0) HXF_I8(6, 4, 8, 0) HXF_I8(7, 4, 8, 0) HXF_I8(8, 4, 8, 0) HXF_I8(9, 4, 8, 0)
    }
#undef HXF_I8
  return hipErrorInvalidValue;
}

}  // namespace

}  // namespace hxf
