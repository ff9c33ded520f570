// Host-side launchers of the gfx950 kernels (one translation unit each).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

namespace hxf {

// Physical KV layout (per layer; K pool then V pool), kv-head major:
//   K: [Hkv][n_blocks][dh/8][16 tokens][8]  (8-dimension chunks of the 16 tokens
//      side by side: the order in which a wavefront feeds them to the MFMA)
//   V: [Hkv][n_blocks][dh][16 positions]    (a dimension's 16 tokens contiguous, token t
//      at position v_pos(t): groups of four tokens in the order 0-3, 8-11, 4-7, 12-15,
//      the key order of the 32x32x16 MFMA's P operand in the prefill kernel)
// so one (page, kv-head) is one contiguous 16*dh*2-byte tile in each pool, and
// the pages of one kv-head of a sequence allocated together are contiguous.
constexpr int kPage = 16;
__host__ __device__ inline size_t kv_tile(int kvh, int64_t n_blocks, int blk, int dh) {
  return ((size_t)kvh * n_blocks + blk) * kPage * dh;
}
// Position of token t (0..15) inside a V page row: bits 2 and 3 swapped.
__host__ __device__ inline int v_pos(int t) { return (t & 3) | ((t >> 1) & 4) | ((t << 1) & 8); }

// ------------------------------------------------------------------ GEMM
enum { EPI_BF16 = 0, EPI_RESID = 1, EPI_SWIGLU = 2, EPI_F32 = 3 };

// Packed tile layout of a bf16 [rows, K] matrix (the weights', also used for the
// activations the prefill GEMMs read): 16-row x 32-column tiles of 1 KB, row tiles
// outermost, kt = ceil(K / 32) tiles per row tile, inside a tile [k%32 / 8][r%16][k%8].
// A DMA of one 16 x 32 block is then one contiguous kilobyte instead of 16 row pieces.
__host__ __device__ inline size_t packed_elem(int r, int k, int kt) {
  return ((size_t)(r >> 4) * kt + (k >> 5)) * 512 + ((k >> 3) & 3) * 128 + (r & 15) * 8 + (k & 7);
}

struct GemmArgs {
  const uint16_t* A;   // bf16 [M, lda]
  const uint16_t* B;   // bf16 [N, K] (SwiGLU: gate rows [F, K])
  const uint16_t* B2;  // SwiGLU: up rows [F, K]
  void* C;             // bf16 / fp32 output or fp32 residual, row stride ldc
  float* partial;      // split-K partials [splits][M][N] fp32
  int M, N, K;         // N is logical (2F for SwiGLU); K % 8 == 0
  int lda, ldc;
  int k_chunk;
  int kt;              // K tiles of the packed weights, ceil(K / 32)
  int a_packed;        // A is in the packed tile layout (lda unused)
  int c_kt;            // SwiGLU: > 0 writes C in the packed tile layout with c_kt tiles per row tile
};

// Bytes of the split-K partials array behind hxf_op_gemm_noalloc
constexpr int64_t kNoallocPartials = int64_t(16) << 20;

struct GemmPlan {
  int tm = 4, nw = 4, wv = 4;   // a workgroup's row tiles, column tiles per wavefront, wavefronts
  bool once = false;            // one row of tiles: the weights are read once (non-temporal loads)
  int splits = 1;
  int k_chunk = 0;
};

// swiglu: the plan is for the SwiGLU epilogue (N = 2F logical columns); own_partials: the caller has
// its own array for them, so nothing hangs on the size of the allocation-free one
GemmPlan gemm_plan(int M, int N, int K, int max_splits, bool swiglu = false, bool own_partials = false);
// With reduce == false a split-K plan leaves its fp32 partials [splits][M][N] in
// a.partial for the consumer to sum (no reduction launch).  e0 / e1 (may be null):
// events recorded at the first kernel's start and the last kernel's end.
hipError_t gemm_launch(const GemmArgs& a, int epi, const GemmPlan& p, hipStream_t st, bool reduce = true,
                       hipEvent_t e0 = nullptr, hipEvent_t e1 = nullptr);
// The wide kernel with one epilogue each (gemm_wide_*.hip); a.k_chunk set, no reduction.
hipError_t gemm_wide_bf16(const GemmArgs& a, const GemmPlan& p, hipStream_t st, hipEvent_t e0, hipEvent_t e1);
hipError_t gemm_wide_resid(const GemmArgs& a, const GemmPlan& p, hipStream_t st, hipEvent_t e0, hipEvent_t e1);
hipError_t gemm_wide_swiglu(const GemmArgs& a, const GemmPlan& p, hipStream_t st, hipEvent_t e0, hipEvent_t e1);
hipError_t gemm_wide_f32(const GemmArgs& a, const GemmPlan& p, hipStream_t st, hipEvent_t e0, hipEvent_t e1);
hipError_t gemm_wide_split(const GemmArgs& a, const GemmPlan& p, hipStream_t st, hipEvent_t e0, hipEvent_t e1);
// Weight packing: W bf16 [N, K] row-major -> tiles of 16 rows x 32 columns in MFMA
// operand order, zero padded to ceil(N/16)*16 rows and ceil(K/32)*32 columns.
size_t packed_weight_elems(int N, int K);
hipError_t pack_weight_launch(const uint16_t* W, int N, int K, uint16_t* out, hipStream_t st);

// ------------------------------------------------------------------ 8-bit linear layers
// Codes of an int8 matrix [R, K] in tiles of 16 rows x 64 columns (1 KB), kt = ceil(K / 64) tiles per row tile,
// inside a tile [k%64 / 16][r%16][k%16]: the operand order of the 16x16x64 i8 MFMA, the same bytes as a bf16 tile.
__host__ __device__ inline size_t i8_elem(int r, int k, int kt) {
  return ((size_t)(r >> 4) * kt + (k >> 6)) * 1024 + ((k >> 4) & 3) * 256 + (r & 15) * 16 + (k & 15);
}
inline size_t i8_codes_bytes(int R, int K) { return (size_t)((R + 15) / 16) * ((K + 63) / 64) * 1024; }

// codes and scales of bf16 rows x [R, K], row stride in elements
hipError_t quant_i8_launch(const uint16_t* x, int64_t stride, int R, int K, int8_t* codes, float* scale, hipStream_t st);
// codes and scales of rmsnorm(x[rows ? rows[r] : r]) * g; x fp32 [x_rows, d]; zeros where rows[r] is none of them
hipError_t rmsnorm_i8_launch(const float* x, const int32_t* rows, int x_rows, const uint16_t* g, int8_t* codes,
                             float* scale, int n_rows, int d, float eps, hipStream_t st);

struct GemmI8Args {
  const int8_t *A, *B, *B2;        // codes of A [M, K], B [N, K] (SwiGLU: gate) and the up weight
  const float *sa, *sb, *sb2;      // scales of their rows
  void* C;                         // bf16 or fp32, row stride ldc
  int32_t* partial;                // split-K partials
  int M, N, ldc;                   // N: output columns
  int kt;                          // K tiles, ceil(K / 64)
  int piece;                       // K tiles of a piece (even)
};
struct GemmI8Plan {
  int tm = 4, nw = 4, wv = 4;   // a workgroup's row tiles, column tiles per wavefront, wavefronts
  bool once = false;            // one row of tiles: the weights are read once (non-temporal loads)
  int splits = 1;
  int piece = 0;                // K tiles of a piece (even)
  bool thin = false;            // gemm_i8_thin: wavefronts share K, nw column tiles a workgroup
};
GemmI8Plan gemm_i8_plan(int M, int N, int kt, int epi);   // N output columns
hipError_t gemm_i8_run(GemmI8Args a, int epi, const GemmI8Plan& p, hipStream_t st);
// The kernel with one epilogue each (gemm_i8_*.hip)
hipError_t gemm_i8_bf16(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st);
hipError_t gemm_i8_resid(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st);
hipError_t gemm_i8_swiglu(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st);
hipError_t gemm_i8_f32(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st);
hipError_t gemm_i8_split(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st);
hipError_t gemm_i8_thin(const GemmI8Args& a, int epi, const GemmI8Plan& p, hipStream_t st);
hipError_t gemm_i8_split_swiglu(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st);
int64_t gemm_i8_ws_bytes(int M, int N, int K);   // up to these sizes; N as the caller counts it (SwiGLU: 2F)
// hipErrorOutOfMemory (nothing enqueued) where the plan's partials need more than ws_bytes
hipError_t gemm_i8_launch(const GemmI8Args& a, int epi, int64_t ws_bytes, hipStream_t st);

// ------------------------------------------------------------------ norms / embedding
// out[r] = bf16(rmsnorm(x[rows ? rows[r] : r]) * g); x fp32 [*, d]
hipError_t rmsnorm_launch(const float* x, const int32_t* rows, const uint16_t* g, uint16_t* out,
                          int n_rows, int d, float eps, hipStream_t st);
// x[rows[r]] += sum over z < S of part[z][rows[r]] (split-K partials [S][part_rows][d] of a
// residual GEMM, in split order), then out[r] = bf16(rmsnorm(x[rows[r]]) * g); out_kt > 0
// writes out in the packed tile layout (d / 32 tiles per row tile, d % 32 == 0)
hipError_t resid_rmsnorm_launch(float* x, const float* part, int S, int part_rows, const int32_t* rows,
                                const uint16_t* g, uint16_t* out, int n_rows, int d, float eps, hipStream_t st,
                                int out_kt = 0);
// resid[t] = E[ids[t]] (fp32); out[t] = bf16(rmsnorm(resid[t]) * g) (packed as above with out_kt)
hipError_t embed_rmsnorm_launch(const int32_t* ids, const uint16_t* E, const uint16_t* g, float* resid,
                                uint16_t* out, int T, int d, float eps, hipStream_t st, int out_kt = 0);

// ------------------------------------------------------------------ RoPE + KV write
// qkv bf16 [T, (Hq+2Hkv)*dh]: rotates q (in place) and k at pos[t] with the
// table cs[pos][i] = (cos, sin) of pos * base^(-2i/dh); writes k and v to slot[t].
hipError_t rope_kv_launch(uint16_t* qkv, const int32_t* pos, const int32_t* slot, const float2* cs,
                          uint16_t* k_pool, uint16_t* v_pool, int64_t n_blocks, int T, int Hq, int Hkv, int dh,
                          hipStream_t st);
// The same with the projection given as S split-K partials part [S][T][(Hq+2Hkv)*dh]
// (each value = bf16 of their sum in split order); rotated q goes to qkv.
hipError_t rope_kv_partials_launch(uint16_t* qkv, const float* part, int S, const int32_t* pos, const int32_t* slot,
                                   const float2* cs, uint16_t* k_pool, uint16_t* v_pool, int64_t n_blocks, int T,
                                   int Hq, int Hkv, int dh, hipStream_t st);
// Write k, v bf16 [T, Hkv, dh] to slot[t] (no rotation).
hipError_t kv_scatter_launch(const uint16_t* k, const uint16_t* v, const int32_t* slot, uint16_t* k_pool,
                             uint16_t* v_pool, int64_t n_blocks, int T, int Hkv, int dh, hipStream_t st);

// ------------------------------------------------------------------ attention
// One decode work item: tokens [t0, t1) of kv-head `kvh`, read through the block
// table of entry[0], attended by the queries of entries entry[0 .. n_rows) (more
// than one when they share those pages: forks of one parent); row r's partial
// result goes to slot part[r].  The query columns of a wavefront are (row, head)
// pairs: one tile of 16 (at most 16 / G rows) or, for a wide item, two tiles of 16
// (at most min(kDecodeRows, 32 / G) rows) that share every K/V read.
constexpr int kDecodeRows = 8;
struct DecodeItem {
  int32_t kvh, t0, t1, n_rows;
  int32_t entry[kDecodeRows];
  int32_t part[kDecodeRows];
  int32_t pad[4];
};
// Rows one 16-column tile holds, and the rows a wide (two-tile) item holds, for GQA group G.
inline int decode_rows_narrow(int G) { return std::max(1, std::min(kDecodeRows, 16 / G)); }
inline int decode_rows_wide(int G) { return std::max(1, std::min(kDecodeRows, 32 / G)); }
// Decode work split.  Each (sequence, kv-head) context is cut into equal, page-aligned
// partitions no longer than a per-launch target.  With fewer (stream, kv-head) pairs than
// the wavefronts the chip holds at once (two per SIMD at the one-tile kernel's register
// count, 2 x 4 x 256), the target makes the items just fill them.  With more pairs each
// already has an item, and the target is an even share of all the tokens over the
// resident wavefronts: a stream much longer than the others (the shared prefix of a fork
// group next to the forks' short own tails) is cut instead of running alone after the
// rest have drained.  A partition is never shorter than kDecodeMinPartition tokens
// unless its whole context is.
constexpr int kDecodeResident = 2048;
constexpr int kDecodeMinPartition = 256;
inline int64_t decode_target_tokens(int64_t sum_ctx, int64_t n_seqs, int64_t hkv) {
  const int64_t pairs = n_seqs * hkv;
  const int64_t slots = pairs < kDecodeResident ? kDecodeResident - pairs : kDecodeResident;
  return std::max<int64_t>((sum_ctx * hkv + slots - 1) / slots, kDecodeMinPartition);
}
// Partition length (a whole number of pages) for a context of ctx tokens; its
// ceil(ctx / length) parts number at most ceil(ctx / target).
inline int decode_part_len(int ctx, int64_t target) {
  const int64_t n = ((int64_t)ctx + target - 1) / target;
  const int64_t len = ((int64_t)ctx + n - 1) / n;
  return (int)((len + kPage - 1) / kPage * kPage);
}
// One merge job per (entry, kv-head): partials [part0, part0 + n_part).
struct MergeItem {
  int32_t entry, kvh, part0, n_part;
};
struct DecodeAttnArgs {
  const uint16_t* q;       // bf16, q of entry e at q + q_row[e]*q_stride (+ head*dh)
  const int32_t* q_row;    // [entries]
  int q_stride;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  int64_t n_blocks;
  const int32_t* bt;       // [entries][bt_stride]
  int bt_stride;
  const DecodeItem* items;     // n_items one-tile items, then n_wide two-tile items
  int n_items;                 // one-tile items, or that launch's capacity when n_items_dev is set
  int n_wide;                  // two-tile items, or that launch's capacity when n_items_dev is set
  const int32_t* n_items_dev;  // may be null: both counts in device memory (captured launches)
  const MergeItem* merges;
  int n_merges;
  float* part_o;           // [parts][G][dh]
  float* part_ml;          // [parts][G][2]  (max in log2 units, sum)
  uint16_t* out;           // bf16, row q_row[e]*out_stride + head*dh
  int out_stride;
  int out_kt;              // > 0: out in the packed tile layout with out_kt tiles per row tile
  int Hq, Hkv, dh;
  float scale_log2;        // log2(e) / sqrt(dh)
};
// Split-K partials of every work item, then the log-sum-exp merge into `out`.
// ev_start / ev_stop (may be null): events that record the kernel's own start and end.
hipError_t decode_attn_launch(const DecodeAttnArgs& a, hipStream_t st, hipEvent_t ev_start = nullptr,
                              hipEvent_t ev_stop = nullptr);
hipError_t decode_merge_launch(const DecodeAttnArgs& a, hipStream_t st, hipEvent_t ev_start = nullptr,
                               hipEvent_t ev_stop = nullptr);

// One prefill work item: queries [q0, q0 + nq) (chunk-local) of entry `entry`, kv-head
// `kvh`, attending keys of the 32-key tiles [t0, t1).  part < 0: the item covers every
// key its queries see and writes the normalized output; otherwise it writes its
// unnormalized partial (output, running max, sum) to slot `part`, and a merge job
// combines the slots of its query block by log-sum-exp.
struct PrefillItem {
  int32_t entry, kvh, q0, nq;
  int32_t t0, t1, part, pad;
};
// Merge job: partial slots [part0, part0 + n_part) of (entry, kvh, queries [q0, q0 + nq)).
struct PrefillMerge {
  int32_t entry, kvh, q0, nq;
  int32_t part0, n_part, pad0, pad1;
};
// Launch order of the prefill items: most key tiles first (equal counts keep their
// order), so that the short items fill the chip's tail instead of the long ones.
inline void order_prefill_items(PrefillItem* it, size_t n) {
  std::stable_sort(it, it + n, [](const PrefillItem& x, const PrefillItem& y) { return x.t1 - x.t0 > y.t1 - y.t0; });
}
// Workgroups of the prefill kernel resident at once (two per CU: 80 KB of LDS each),
// and the shortest key range an item is split into.
constexpr int kPrefillResident = 512;
// (query, head) pairs of one prefill item (its workgroup's columns), and of a partial slot
constexpr int kPrefillPairs = 128;
constexpr int kPrefillMinTiles = 8;
struct PrefillAttnArgs {
  const uint16_t* q;       // bf16 rows; entry e's query i at row row0[e] + i
  int q_stride;
  const int32_t* row0;     // [entries]
  const int32_t* pos0;     // [entries] position of the entry's first query
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  int64_t n_blocks;
  const int32_t* bt;       // [entries][bt_stride]
  int bt_stride;
  const PrefillItem* items;
  int n_items;
  const PrefillMerge* merges;   // merge jobs of the split items
  int n_merges;
  float* part_o;                // [slots][128 pairs][dh]: unnormalized partial outputs
  float* part_ml;               // [slots][128 pairs][2]: (max in log2 units, sum)
  uint16_t* out;
  int out_stride;
  int out_kt;                   // > 0: out in the packed tile layout with out_kt tiles per row tile
  int Hq, Hkv, dh;
  float scale_log2;
};
// The items, then (when some are split) the merge of their partials.
hipError_t prefill_attn_launch(const PrefillAttnArgs& a, hipStream_t st, hipEvent_t ev_start = nullptr,
                               hipEvent_t ev_stop = nullptr);
// Queries covered by one prefill work item for a given GQA group size.
int prefill_queries_per_item(int group);

// ------------------------------------------------------------------ 8-bit KV cache
// Per layer, kv-head major like the bf16 pools, one byte per element (e4m3) and one power-of-two
// scale per (kv-head, page) of each pool:
//   K: [Hkv][n_blocks][dh/16][16 tokens][16]  (a lane's 16-byte load is 16 dimensions of one token)
//   V: [Hkv][n_blocks][4][dh][4 tokens]       (a dimension's tokens in groups of four, as a lane of the
//                                              score tile holds them)
struct Kv8Pool {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  int64_t n_blocks;
};
// Offset of (dimension d, token t) inside a page of K
__host__ __device__ inline int k8_offset(int d, int t) { return ((d >> 4) * kPage + t) * 16 + (d & 15); }

// A launch counts its threads of each dimension in 32 bits
inline bool launch_fits(int64_t groups, int threads) { return groups <= (int64_t)UINT32_MAX / threads; }

constexpr int kSlotMapMaxSeqs = 4096;
struct SlotMapArgs {
  const int32_t* start;
  const int32_t* n_new;
  const int32_t* free_pages;
  const int32_t* n_free;
  int32_t* bt;
  int32_t* row0;
  int32_t* pos;
  int32_t* slot;
  int32_t* ctx;
  int32_t* status;
  int S, T, free_cap, bt_stride;
};
hipError_t slot_map_launch(const SlotMapArgs& a, hipStream_t st);

struct Kv8WriteArgs {
  const uint16_t* qkv;
  int64_t qkv_stride;
  const int32_t* pos;
  const int32_t* slot;
  const float2* cs;      // may be null: no rotation
  int max_pos;
  uint16_t* q_out;       // may be null
  int64_t q_stride;
  Kv8Pool pool;
  int T, Hq, Hkv, dh;
};
constexpr int kWriteRows = 16;   // rows of a workgroup
// (a workgroup of 256 for them and a head, or some q heads)
inline bool kv8_write_fits(int64_t T, int64_t Hq, int64_t Hkv) {
  return launch_fits((T + kWriteRows - 1) / kWriteRows, 256) && Hq + 2 * Hkv < (1 << 16);
}
hipError_t kv8_write_launch(const Kv8WriteArgs& a, hipStream_t st);

struct Kv8AttnArgs {
  const uint16_t* q;
  int64_t q_stride;
  Kv8Pool pool;
  const int32_t* bt;
  int bt_stride;
  const int32_t* ctx;    // decode: [B]
  const int32_t* row0;   // prefill: [S + 1]
  const int32_t* pos0;   // prefill: [S]
  uint16_t* out;
  int64_t out_stride;
  int S, T;              // sequences; prefill: rows
  int Hq, Hkv, dh;
  float scale_log2;      // log2(e) / sqrt(dh)
  uint8_t* ws;
  int64_t ws_ml;         // decode: offset of the shares of the parts
  int32_t* starts;       // decode: [B + 1] parts of a kv-head before each sequence
};
// Decode work split, made by the kernels themselves from the contexts in device memory.  As for the bf16
// cache, each (sequence, kv-head) stream of pages is cut into equal parts no longer than an even share of
// all the pages over the wavefronts the chip holds at once (or than kKv8MinPages pages, or than kv8_part_pages
// says); with fewer streams than those wavefronts the parts at most fill them.
constexpr int kKv8Resident = 3 * 1024;   // three a SIMD, at the 160 VGPRs of head size 128; 64, at 103, is split likewise,
                                         // and its fourth place is left empty
constexpr int kKv8MinPages = 4;
constexpr int kKv8WholePages = 8;    // with tables this short no stream is cut, and there is no join: 20 contexts of up
                                     // to 60 tokens 4.7 us, with parts and a join 6.3.  (A property of the table, which the
                                     // host knows: short contexts in wide tables are cut.)
__host__ __device__ inline int64_t kv8_target_pages(int64_t total_pages, int64_t n_seqs, int hkv, int bt_stride) {
  const int least = bt_stride <= kKv8WholePages ? kKv8WholePages : kKv8MinPages;
  const int64_t pairs = n_seqs * hkv;
  const int64_t slots = pairs < kKv8Resident ? kKv8Resident - pairs : kKv8Resident;
  const int64_t t = (total_pages * hkv + slots - 1) / slots;
  return t > least ? t : least;
}
// Length of a part of a stream of `pages` pages, and the number of them: at most ceil(pages / target).  A part takes as
// long as its pages, the join as its parts: for a stream alone their sum is least near sqrt(pages / 8) pages a part.  The rule
// does not look at the number of heads and streams, with which the join grows.  One context, 32 + 8 heads, us, against 8
// pages or more: 1000 tokens 7.9 / 9.0, 2000 8.1 / 9.8, 8191 11.2 / 11.2, 30000 17.5 / 19.0, 64000 29.2 / 31.9; 16 of 100 to
// 1500 10.2 / 11.3; 8 of 500 to 3000, 64 + 8 heads, 13.1 / 11.7.
__host__ __device__ inline int kv8_part_pages(int pages, int target) {
  const int least = (int)sqrtf((float)(pages / 8)), t = target > least ? target : least;
  const int n = (pages + t - 1) / t;
  return n > 0 ? (pages + n - 1) / n : 1;
}
__host__ __device__ inline int kv8_parts(int pages, int target) {
  const int len = kv8_part_pages(pages, target);
  return (pages + len - 1) / len;
}
// Wavefronts that hold every part whatever the contexts are: with fewer streams than resident wavefronts,
// sum ceil(p / t) <= sum p / t + streams <= (resident - streams) + streams; otherwise resident + streams.
inline int64_t kv8_decode_items(int64_t n_seqs, int hkv) {
  const int64_t pairs = n_seqs * hkv;
  return pairs < kKv8Resident ? kKv8Resident : kKv8Resident + pairs;
}
// Whether the launches hold a batch: the attention's, and the join's of four heads a workgroup
inline bool kv8_decode_fits(int64_t n_seqs, int hkv) { return launch_fits(kv8_decode_items(n_seqs, hkv), 64); }
inline bool kv8_decode_join_fits(int64_t n_seqs, int hq, int bt_stride) {
  return bt_stride <= kKv8WholePages || launch_fits(n_seqs * ((hq + 3) / 4), 256);
}
// Prefill work split, made by a kernel from the rows and positions in device memory.  A block of up to 128 / G queries
// of a sequence is one unit of work for every kv-head, over its key tiles of 32 positions (taken in pairs).  Where
// whole blocks would be fewer than kPrefillCutUnits, all of a head's pairs, block after block, are dealt out in equal
// shares to the workgroups resident at once: a block is cut where a share ends, unless it exceeds one by
// kPrefillMinTiles pairs at most, or the piece would be shorter than kPrefillMinTiles / 4.  32 + 8 heads, us, against
// equal parts of each block, of no more than a share and so more of them than are resident: 512 queries at 8192 104 / 137,
// 640 at 9000 140 / 163, 800 at 20000 310 / 402.  Cut / whole, us: 128 blocks (512 queries at 8192) 107 / 188, 264 (1056 at
// 6000) 154 / 178, 304 (1216 at 8192) 210 / 238, 352 (44 times 32 at 4000) 157 / 146, 352 (16 times 5 to 256 at 4000, 40 + 8
// heads) 139 / 132, 384 (1536 at 8192) 262 / 253.  The rule counts blocks and not their lengths: a first chunk of 2048
// queries, 512 blocks of 2 to 64 tiles, lasts as long as its longest (65 us).
constexpr int kCus = 256;
constexpr int kPrefillCutUnits = 320;
__host__ __device__ inline bool kv8_prefill_cuts(int64_t blocks, int hkv) {
  return blocks * hkv < kPrefillCutUnits && blocks <= kCus;   // (a thread plans a block)
}
// Sizes are counted in 2^shift pairs, so that those of all blocks that are cut stay in 32 bits
__host__ __device__ inline int kv8_prefill_shift(int bt_stride) { return bt_stride >> 24; }
__host__ __device__ inline uint32_t kv8_prefill_size(int tiles, int shift) {
  return ((uint32_t)(tiles >> 1) + (1u << shift) - 1) >> shift;
}
__host__ __device__ inline int kv8_prefill_streams(int hkv) { return kPrefillResident > hkv ? kPrefillResident / hkv : 1; }
__host__ __device__ inline uint32_t kv8_prefill_share(uint32_t total, int hkv) {
  const uint32_t n = (uint32_t)kv8_prefill_streams(hkv), t = total / n + (total % n != 0);
  return t > kPrefillMinTiles / 2 ? t : kPrefillMinTiles / 2;
}
// The block of sizes [at, at + size): its parts (at least one), which begin at 0 and, from part 1 on, where shares
// cut, cut + 1, ... end
struct Kv8Cut {
  uint32_t cut;
  int parts;
};
__host__ __device__ inline Kv8Cut kv8_prefill_cut(uint32_t at, uint32_t size, uint32_t share) {
  Kv8Cut c{0, 1};
  if (size <= share + kPrefillMinTiles) return c;
  uint32_t lo = at / share + 1, hi = (at + size - 1) / share;
  if (lo * share - at < kPrefillMinTiles / 4) ++lo;
  if (at + size - hi * share < kPrefillMinTiles / 4) --hi;
  if (lo > hi) return c;
  c.cut = lo;
  c.parts = (int)(hi - lo) + 2;
  return c;
}
// First tile of part k of a block of `tiles` tiles, and of the one after it for k + 1
__host__ __device__ inline int kv8_prefill_part_tile(Kv8Cut c, uint32_t at, uint32_t share, int shift, int tiles, int k) {
  return k == 0 ? 0 : k >= c.parts ? tiles : (int)((c.cut + k - 1) * share - at) << (shift + 1);
}
// Units that hold any batch of S sequences and T rows, and partial slots of a kv-head: blocks number at most
// T / q + S; cut ones, over all heads, under kPrefillCutUnits, with a cut for each share but one.
inline int64_t kv8_prefill_unit_cap(int64_t S, int64_t T, int queries, int hkv) {
  const int64_t cut = (kPrefillCutUnits + kPrefillResident) / hkv, whole = T / queries + S;
  return (cut > whole ? cut : whole) + 1;
}
// Blocks that the planning launch takes from its next sequences, which have `more`, after `before` others: all of them where
// row0 ascends.  Where it does not they might pass any count (each sequence may have T rows): they end with the units.
__host__ __device__ inline int kv8_prefill_take(int before, int more, int unit_cap) {
  return more < unit_cap - before ? more : unit_cap - before;
}
inline int64_t kv8_prefill_slots(int64_t S, int64_t T, int queries, int hkv) {
  const int64_t cut = (kPrefillCutUnits + kPrefillResident) / hkv, whole = T / queries + S + kv8_prefill_streams(hkv);
  return (cut < whole ? cut : whole) + 1;
}
inline bool kv8_prefill_fits(int64_t S, int64_t T, int queries, int hkv) {
  return launch_fits(kv8_prefill_unit_cap(S, T, queries, hkv) * hkv, 256);
}
int64_t kv8_decode_ws_bytes(int B, int Hq, int Hkv, int dh);
hipError_t kv8_decode_launch(const Kv8AttnArgs& a, hipStream_t st);
int64_t kv8_prefill_ws_bytes(int S, int T, int Hq, int Hkv, int dh);
hipError_t kv8_prefill_launch(const Kv8AttnArgs& a, hipStream_t st);

// ------------------------------------------------------------------ sampling / misc
// out[r] = argmax_v logits[r][v], the lowest index among equal maxima.
hipError_t argmax_launch(const float* logits, int32_t* out, int R, int V, hipStream_t st);
// dst = src (bytes % 16 == 0); HBM bandwidth probe.
hipError_t copy_launch(const void* src, void* dst, size_t bytes, hipStream_t st);
// Read-bandwidth probe: at most kReadProbeBlocks workgroups of 256 threads; thread t of
// the launch writes sink[t] (the XOR of the words it read), the rest of sink is untouched.
constexpr int kReadProbeBlocks = 4096;
hipError_t read_launch(const void* src, size_t bytes, uint32_t* sink, hipStream_t st);

}  // namespace hxf
