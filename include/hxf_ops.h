/*
 * hxf_ops.h -- the individual gfx950 kernels of one decoder iteration, exposed
 * for kernel-level parity tests, benchmarks and callers that drive their own
 * forward pass.
 *
 * All pointers are DEVICE pointers unless marked "host".  bf16 tensors are
 * uint16 bit patterns.  Every call enqueues work on `stream` (hipStream_t, may
 * be 0) and returns HXF_OK (0) or a negative hxf error code; errors are not
 * sticky and leave nothing enqueued.  The caller owns every device buffer.  Calls
 * that build a work list on the host (attention) copy it into the caller's
 * `workspace` with an asynchronous host-to-device copy and synchronise the
 * stream before returning, so their host arguments may be freed afterwards; each
 * thread that makes them keeps up to 4 MiB of pinned and 4 MiB of pageable host
 * memory for it until the thread ends.
 *
 * Physical KV layout (one layer), kv-head major: K pool [Hkv][n_blocks][dh/8][16][8]
 * (element (token t, dim d) of a page at ((d/8)*16 + t)*8 + d%8), then a separate
 * V pool [Hkv][n_blocks][dh][16] (V transposed inside a page: element (t, d) at
 * d*16 + v_pos(t), v_pos swapping bits 2 and 3 of t, i.e. the page's tokens in
 * groups of four in the order 0-3, 8-11, 4-7, 12-15); the token at
 * position p of a sequence with block table bt lives in slot bt[p/16]*16 + p%16.
 * `n_blocks` is the number of pages of the pool (its kv-head stride).
 */
#ifndef HXF_OPS_H
#define HXF_OPS_H

#include <stdint.h>

#include "hxf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* GEMM epilogues, and layout flags that may be or-ed into the epilogue argument */
enum { HXF_EPI_BF16 = 0, HXF_EPI_RESID = 1, HXF_EPI_SWIGLU = 2, HXF_EPI_F32 = 3 };
enum { HXF_GEMM_A_PACKED = 0x100, HXF_GEMM_C_PACKED = 0x200 };

/* C = A[M,K] . B[N,K]^T, bf16 inputs, fp32 accumulation.  A is row-major with row
 * stride lda; B (and B2) are PACKED weights (hxf_op_pack_weight of the row-major
 * [N,K] matrix, or [F,K] for SwiGLU).
 *   HXF_EPI_BF16:   C bf16 [M, ldc]            C = bf16(acc)
 *   HXF_EPI_RESID:  C fp32 [M, ldc]            C += acc          (residual stream)
 *   HXF_EPI_SWIGLU: B = W_gate [F,K], B2 = W_up [F,K], N = 2F; C bf16 [M, ldc],
 *                   C[:, f] = bf16(silu(gate_f) * up_f), silu(z) = z / (1 + e^-z)
 *   HXF_EPI_F32:    C fp32 [M, ldc]            C = acc
 * K % 8 == 0, lda >= K.  workspace: hxf_op_gemm_workspace_bytes(M, N, K) bytes
 * (split-K partials for M <= 512, enough for every epilogue; may be 0 bytes).
 * HXF_GEMM_A_PACKED: A is in the packed layout of the weights (hxf_op_pack_weight of the
 * row-major [M,K] activations, ceil(M/16)*16 rows; lda unused), so that a 16 x 32 block of
 * it is one contiguous kilobyte; K % 32 == 0 (and F % 32 == 0 for SwiGLU).
 * HXF_GEMM_C_PACKED (SwiGLU, F % 32 == 0): C is written in that packed layout ([M,F] with
 * F/32 tiles per row tile; ldc unused), the form in which the down projection reads it.
 * Either flag on another shape: HXF_EINVAL. */
int64_t hxf_op_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K);
int hxf_op_gemm(const void* A, int32_t lda, const void* B, const void* B2, void* C, int32_t ldc, int32_t M, int32_t N,
                int32_t K, int32_t epilogue, void* workspace, int64_t workspace_bytes, void* stream);

/* Introspection (host only, no device work): the tile and K split hxf_op_gemm takes for these sizes:
 * plan = {row tiles of 16, column tiles of 16 per wavefront, wavefronts, 1 if the weights are fetched
 * as read once, pieces of K, K per piece}. */
int hxf_op_gemm_plan(int32_t M, int32_t N, int32_t K, int32_t epilogue, int32_t plan[6]);

/* hxf_op_gemm without a workspace, for callers that cannot allocate device memory
 * (code under HIP graph capture, tight serving loops, harnesses that forbid it).
 * Same arguments and result as hxf_op_gemm (the layout flags are refused: HXF_EINVAL);
 * the split-K partials go to a device
 * array of HXF_GEMM_NOALLOC_MAX_BYTES that the library holds on each GPU it runs on
 * until the process ends (its address is looked up on the first call on a device,
 * which must be the current device).  Nothing is allocated.  HXF_ENOMEM (nothing
 * enqueued) when the plan's partials, splits * M * N * 4 bytes, exceed that size:
 * every plan with M <= 128 fits.  Calls on one GPU share the array: calls that
 * overlap on one GPU (several streams, several threads) race and must be serialised
 * by the caller. */
#define HXF_GEMM_NOALLOC_MAX_BYTES (16LL << 20)
int hxf_op_gemm_noalloc(const void* A, int32_t lda, const void* B, const void* B2, void* C, int32_t ldc, int32_t M,
                        int32_t N, int32_t K, int32_t epilogue, void* stream);

/* Packed weight layout, used for every GEMM weight: W [N,K] bf16 row-major becomes
 * tiles of 16 rows x 32 columns (1 KB), row-tiles outermost, zero padded to
 * ceil(N/16)*16 rows and ceil(K/32)*32 columns; inside a tile the 8-element chunks
 * are in the order [k%32 / 8][n%16], i.e. element (n, k) is at
 *   ((n/16) * ceil(K/32) + k/32) * 512 + ((k%32)/8) * 128 + (n%16) * 8 + k%8.
 * This is the operand order of the 16x16x32 bf16 MFMA, so a wavefront reads a tile
 * as one contiguous kilobyte.  hxf_op_pack_weight converts W (device, K % 8 == 0)
 * into out (device, hxf_packed_weight_bytes(N, K) bytes); W and out must not overlap. */
int64_t hxf_packed_weight_bytes(int32_t N, int32_t K);
int hxf_op_pack_weight(const void* W, int32_t N, int32_t K, void* out, void* stream);

/* out[r] = bf16(x[rows[r]] / sqrt(mean(x[rows[r]]^2) + eps) * g); rows may be NULL (identity).
 * x fp32 [*, d], g bf16 [d], out bf16 [n_rows, d]; d % 4 == 0. */
int hxf_op_rmsnorm(const float* x, const int32_t* rows, const void* g, void* out, int32_t n_rows, int32_t d,
                   float eps, void* stream);

/* resid[t] = float(E[ids[t]]); out[t] = rmsnorm(resid[t]) * g.  E bf16 [V, d]. */
int hxf_op_embed_rmsnorm(const int32_t* ids, const void* E, const void* g, float* resid, void* out, int32_t T,
                         int32_t d, float eps, void* stream);

/* RoPE table for positions [0, max_pos): float pairs (cos, sin) of p * base^(-2i/dh), i < dh/2,
 * computed in double on the host and copied to dst (max_pos * dh/2 * 8 bytes). */
int hxf_op_rope_table(void* dst, int32_t max_pos, int32_t head_dim, float base, void* stream);

/* qkv bf16 [T, (Hq+2Hkv)*dh] rows (q heads, k heads, v heads): rotate-half RoPE of q (in place)
 * and k at pos[t]; write rotated k and v to slot[t] of the K and V pools. */
int hxf_op_rope_kv_write(void* qkv, const int32_t* pos, const int32_t* slot, const void* rope_table, void* k_pool,
                         void* v_pool, int64_t n_blocks, int32_t T, int32_t Hq, int32_t Hkv, int32_t head_dim,
                         void* stream);

/* Write k, v bf16 [T, Hkv, dh] to slot[t] of the pools (no rotation). */
int hxf_op_kv_scatter(const void* k, const void* v, const int32_t* slot, void* k_pool, void* v_pool, int64_t n_blocks,
                      int32_t T, int32_t Hkv, int32_t head_dim, void* stream);

/* Decode attention, one query token per sequence: q bf16 [B, Hq, dh] (rotated), attends to positions
 * [0, ctx_host[b]) of sequence b through block table bt [B, bt_stride] (device); out bf16 [B, Hq, dh].
 * bt_host (may be NULL): the same block table on the host.  When given, sequences whose tables start
 * with the same physical pages (forks of one retained parent, e.g. the parallel candidate requests
 * of one query, Section 2.1) are grouped and their common full pages are read once for up to
 * min(8, 32 / (Hq/Hkv)) of them (a second 16-column MFMA tile reuses every K/V read when more
 * than 16 / (Hq/Hkv) rows share an item); the result is the same attention.  Each (sequence, kv-head) stream is
 * split into equal page-aligned partitions (at least 256 tokens, sized so that the work items fill
 * the wavefronts the chip holds at once, or, with more streams than those, no longer than an even
 * share of all the tokens over them), merged by log-sum-exp.
 * workspace: hxf_op_decode_attention_workspace_bytes(...) bytes (same ctx_host, bt_host, bt_stride). */
int64_t hxf_op_decode_attention_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t head_dim,
                                                const int32_t* ctx_host, const int32_t* bt_host, int32_t bt_stride);
/* Introspection (host only, no device work): the decode-attention work list the two calls above
 * build.  items: n_items records of 24 int32 {kvh, t0, t1, n_rows, entry[8], part[8], pad[4]}
 * (tokens [t0, t1) of kv-head kvh through the pages of entry[0], attended by the first n_rows
 * entries, partial of row r in slot part[r]); the one-tile items (n_rows <= max(1, 16 / G)) come
 * first, then the two-tile items, each longest first; merges: n_merges records of 4 int32
 * {entry, kvh, part0, n_part}.  Returns HXF_ENOMEM (with the counts set) when a capacity is short. */
int hxf_op_decode_plan(int32_t B, int32_t Hq, int32_t Hkv, const int32_t* ctx_host, const int32_t* bt_host,
                       int32_t bt_stride, int32_t* items, int32_t items_cap, int32_t* n_items, int32_t* merges,
                       int32_t merges_cap, int32_t* n_merges);
int hxf_op_decode_attention(const void* q, const void* k_pool, const void* v_pool, int64_t n_blocks, const int32_t* bt,
                            int32_t bt_stride, const int32_t* ctx_host, const int32_t* bt_host, void* out, int32_t B,
                            int32_t Hq, int32_t Hkv, int32_t head_dim, void* workspace, int64_t workspace_bytes,
                            void* stream);

/* Causal prefill attention over chunks: chunk s has n_host[s] queries at positions
 * pos0_host[s] .. pos0_host[s]+n-1, stored at rows row0_host[s].. of q bf16 [*, Hq, dh];
 * it attends to positions [0, pos0+i] of its block table row bt[s] (device).  out rows as q. */
int64_t hxf_op_prefill_attention_workspace_bytes(int32_t S, int32_t Hq, int32_t Hkv, const int32_t* n_host);
/* Introspection (host only, no device work): the prefill-attention work list the call below
 * builds for the same chunks.  items: n_items records of 8 int32 {entry, kvh, q0, nq, t0, t1, part,
 * pad} (queries [q0, q0 + nq) of chunk `entry` on kv-head kvh over key tiles [t0, t1) of 32
 * positions; part = -1 for an item that writes its output, else the partial slot of a cut item),
 * in launch order; merges: n_merges records of 8 int32 {entry, kvh, q0, nq, part0, n_part, pad,
 * pad} (the partial slots [part0, part0 + n_part) of one cut item, combined by log-sum-exp).
 * Items are cut into key ranges only when there are fewer of them than CUs: those longer than an
 * even share of all key tiles over the resident workgroups (two per CU), at least 8 tiles.
 * HXF_ENOMEM (with the counts set) when a capacity is short. */
int hxf_op_prefill_plan(int32_t S, int32_t Hq, int32_t Hkv, const int32_t* pos0_host, const int32_t* n_host,
                        int32_t* items, int32_t items_cap, int32_t* n_items, int32_t* merges, int32_t merges_cap,
                        int32_t* n_merges);
int hxf_op_prefill_attention(const void* q, const void* k_pool, const void* v_pool, int64_t n_blocks, const int32_t* bt,
                             int32_t bt_stride, const int32_t* row0_host, const int32_t* pos0_host,
                             const int32_t* n_host, void* out, int32_t S, int32_t Hq, int32_t Hkv, int32_t head_dim,
                             void* workspace, int64_t workspace_bytes, void* stream);

/* ---- The 8-bit KV cache: e4m3 pages with a scale for each block of 16 tokens and head, and the
 * operators of a step whose lengths are known on the device alone.  None of them waits for the stream or
 * reads device values on the host, so a step can be captured into a graph and replayed with other lengths.
 *
 * K pool [Hkv][n_blocks][dh/16][16][16] bytes: element (token t, dim d) of a page at
 * ((d/16)*16 + t)*16 + d%16.  V pool [Hkv][n_blocks][4][dh][4]: element (t, d) at ((t/4)*dh + d)*4 + t%4.
 * Scales: fp32 [Hkv][n_blocks] for K and for V; an element stands for its e4m3 value (OCP: largest 448, NaN, no
 * infinity) times the scale of its page.  A scale is a POWER OF TWO in [2^-100, 2^120] (hxf_op_rope_kv8_write
 * makes no other; of any other value the attention uses the exponent alone, 0 being 2^-127), so a dequantised element is
 * exactly a bf16 value and a page whose scale grows keeps its codes up to their exponents.  (But at 2^120, in a
 * page with |x| > 1.75 * 2^127, the codes from 256 on, for |x| from 1.9375 * 2^127 on, stand for values beyond bf16 and
 * fp32: outputs of queries that see one are undefined.)  (The attention holds V to
 * 2^-25 of the largest V scale among a sequence's pages of a head: exactly where scales are within 2^15 of it.)
 * k and v must be 16-byte aligned; 0 < n_blocks < 2^27.  The struct is read during the call only. */
typedef struct hxf_kv8_pool {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int64_t n_blocks;
} hxf_kv8_pool;

/* Block tables, positions and slots of a batch from its lengths: sequence s has start[s] tokens in the
 * cache and gets n_new[s] (0: none) more.  Its pages past the ceil(start/16) it holds are taken from the front
 * of free_pages, sequence by sequence, and entered into bt [S, bt_stride] (its other entries stay as they
 * are).  free_pages holds *n_free (device; at most free_cap) page numbers.  Outputs:
 *   row0 [S+1]  first row of each sequence, and the number of rows
 *   pos, slot [T]  of row row0[s] + i: start[s] + i and its place bt[s][pos/16]*16 + pos%16 in the cache;
 *                rows from row0[S] on: pos 0, slot -1 (so a batch may be padded to T rows)
 *   ctx [S]     start + n_new
 *   status [2]  pages taken, rows
 * All or nothing: when the pages or the T rows do not suffice, a sequence needs more than bt_stride pages,
 * or a length is negative, status is {-1, 0}, bt is left as it is, row0 is 0, ctx is start (0 for a negative one)
 * and every row is {pos 0, slot -1}.  S <= HXF_SLOT_MAP_MAX_SEQS, T and
 * free_cap < 2^30.  All arrays are on the device; the outputs must not overlap the inputs or each other. */
#define HXF_SLOT_MAP_MAX_SEQS 4096
int hxf_op_slot_map(const int32_t* start, const int32_t* n_new, int32_t S, const int32_t* free_pages,
                    const int32_t* n_free, int32_t free_cap, int32_t* bt, int32_t bt_stride, int32_t* row0,
                    int32_t* pos, int32_t* slot, int32_t T, int32_t* ctx, int32_t* status, void* stream);

/* RoPE and the quantised KV write.  qkv bf16, T rows of qkv_stride elements (q heads, k heads, v heads; left as it
 * is): rotate-half RoPE of q and k at pos[t] in fp32 (rope_table: max_pos rows of hxf_op_rope_table; NULL: no
 * rotation, pos unused); rotated q to q_out (bf16, rows of q_stride elements; NULL: not wanted), k and v to
 * slot[t] of the pools as e4m3 (nearest even, of the unrounded fp32 value).  A page's scale is the least power of two s with
 * max|x| <= 448 s over the finite values written to it (no less than 2^-100); values that are not finite become NaN.
 * Rows of one call that go to one page must be successive rows with successive slots, none of them skipped
 * (hxf_op_slot_map makes them so).  When they begin at the page's first token the page starts afresh; otherwise the tokens
 * before them stay: the scale is the larger of the page's and the new rows', and where it grows the old codes
 * are requantised.  Tokens behind the new rows are left as they are.  A row whose slot is not in [0, 16 n_blocks), or
 * (with a table) whose pos is not in [0, max_pos), is skipped, its q_out row included.
 * qkv and q_out 16-byte aligned, strides multiples of 8, T <= 2^28 - 16, Hq + 2 Hkv < 2^16; no buffer may overlap
 * another. */
int hxf_op_rope_kv8_write(const void* qkv, int64_t qkv_stride, const int32_t* pos, const int32_t* slot,
                          const void* rope_table, int32_t max_pos, void* q_out, int64_t q_stride,
                          const hxf_kv8_pool* pool, int32_t T, int32_t Hq, int32_t Hkv, int32_t head_dim, void* stream);

/* Decode attention over the 8-bit cache: one query per sequence, q bf16 (row b at b*q_stride, heads of
 * head_dim), attends to positions [0, ctx[b]) (ctx on the device, taken as in [0, 16 bt_stride]) through
 * bt [B, bt_stride]; out bf16 rows of out_stride elements.  ctx 0 (an empty place of a padded batch):
 * zeros.  Tokens of a block-table entry that is no page of the pool are not read and have no weight.  Entries past
 * the context are not read.  q, out, the pool and the workspace must not overlap.  workspace:
 * hxf_op_decode_attention_kv8_workspace_bytes bytes, 16-byte aligned, whose contents need not be kept between
 * calls; calls that may overlap need one each.  B * Hq < 2^29; B * Hkv < 2^26 - 3 * 2^10; and, with bt_stride > 8,
 * B * ceil(Hq / 4) < 2^24. */
int64_t hxf_op_decode_attention_kv8_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t head_dim);
int hxf_op_decode_attention_kv8(const void* q, int64_t q_stride, const hxf_kv8_pool* pool, const int32_t* bt,
                                int32_t bt_stride, const int32_t* ctx, void* out, int64_t out_stride, int32_t B,
                                int32_t Hq, int32_t Hkv, int32_t head_dim, void* workspace, int64_t workspace_bytes,
                                void* stream);

/* Causal prefill attention over the 8-bit cache: sequence s's queries are the rows row0[s] .. row0[s+1] - 1 of q
 * (row0 [S+1] ascending, on the device, as hxf_op_slot_map makes it; taken as in [0, T]; where it does not ascend
 * the T rows of out are undefined) at positions pos0[s], pos0[s]+1, ... (pos0 on the device); each attends to the
 * positions up to its own through bt[s], whose keys are in the cache already.  Rows of no sequence are left as they
 * are in out.  Positions from 16 bt_stride on are not in the cache: no key there is seen.  NaN in the cache (a value
 * that was not finite) reaches the queries that see it and no other.  Bad entries, strides and workspace as for
 * hxf_op_decode_attention_kv8.  (S + T) * Hq < 2^29; and, with Q = floor(128 / (Hq / Hkv)) queries a block,
 * (floor(T / Q) + S + 1) * Hkv < 2^24. */
int64_t hxf_op_prefill_attention_kv8_workspace_bytes(int32_t S, int32_t T, int32_t Hq, int32_t Hkv, int32_t head_dim);
int hxf_op_prefill_attention_kv8(const void* q, int64_t q_stride, const hxf_kv8_pool* pool, const int32_t* bt,
                                 int32_t bt_stride, const int32_t* row0, const int32_t* pos0, void* out,
                                 int64_t out_stride, int32_t S, int32_t T, int32_t Hq, int32_t Hkv, int32_t head_dim,
                                 void* workspace, int64_t workspace_bytes, void* stream);

/* ---- Linear layers in 8-bit integers: the rows of a matrix [R, K] (the output channels of a weight, the tokens
 * of the activations) as codes of -127..127 with one fp32 scale a row; an element stands for its code times the
 * scale of its row.  No call waits for the stream or reads device values on the host, so all of them can be captured.
 *
 * Codes are kept in tiles of 16 rows x 64 columns (1 KB), row-tiles outermost, zero padded to whole tiles: element
 * (r, k) is at
 *   ((r/16) * ceil(K/64) + k/64) * 1024 + ((k%64)/16) * 256 + (r%16) * 16 + k%16,
 * the operand order of the 16x16x64 i8 MFMA.  hxf_i8_codes_bytes(R, K) bytes (-1 for sizes the operators refuse),
 * 16-byte aligned.  0 < K < 2^17, so that no sum of products passes 32 bits; 0 <= R <= 2^22 - 16. */
int64_t hxf_i8_codes_bytes(int32_t R, int32_t K);

/* Codes and scales of bf16 rows (weights once when they are loaded, activations in each step): x bf16, R rows of
 * x_stride elements, K of them used.  With m = max|x| of a row: scale = m / 127, code = x * (127 / m) rounded to the
 * nearest whole number, ties to even; both divisions and the product in fp32.  A row with m < 2^-119 is zeros with
 * the scale 0; one that holds NaN or an infinity has zero codes and the scale NaN, so that every output it takes
 * part in is NaN and no other.  codes: hxf_i8_codes_bytes(R, K) bytes, the padding written as zeros; scale fp32
 * [R].  x 16-byte aligned, x_stride >= K and both multiples of 8.  No buffer may overlap another. */
int hxf_op_quant_i8(const void* x, int64_t x_stride, int32_t R, int32_t K, void* codes, float* scale, void* stream);

/* RMSNorm into codes: row r is y = x[rows[r]] * g / sqrt(mean(x[rows[r]]^2) + eps), without a rounding to bf16 in
 * between (rows may be NULL: row r itself).  The codes are those of x * g, formed in fp32, as hxf_op_quant_i8 makes them;
 * scale = max|x g| / 127 / sqrt(mean(x^2) + eps), the sum of squares in fp32 (beyond its range the scale is 0; eps >= 0, and
 * where mean(x^2) + eps is below 2^-100 the scale of a row that has codes is undefined).  A row with max|x g| < 2^-119,
 * or whose index is not in [0, x_rows) (an empty place of a padded batch), is zeros with the scale 0, with eps 0 too.
 * x fp32 [x_rows, d], 16-byte aligned, g bf16 [d], 8-byte aligned, d % 4 == 0, d < 2^17; codes and scale as above, for
 * [n_rows, d]; n_rows <= 2^22 - 16.  Without rows, n_rows <= x_rows.  No output may overlap another buffer. */
int hxf_op_rmsnorm_i8(const float* x, const int32_t* rows, int32_t x_rows, const void* g, void* codes, float* scale,
                      int32_t n_rows, int32_t d, float eps, void* stream);

/* C from acc = A[M,K] . B[N,K]^T of codes, summed exactly in 32-bit integers; y = (float(acc) * a_scale[m]) * b_scale[n].
 *   HXF_EPI_BF16:   C bf16 [M, ldc]            C = bf16(y)
 *   HXF_EPI_RESID:  C fp32 [M, ldc]            C += y            (residual stream)
 *   HXF_EPI_SWIGLU: B, b_scale = W_gate [F,K], B2, b2_scale = W_up [F,K], N = 2F; C bf16 [M, ldc],
 *                   C[:, f] = bf16(silu(gate_f) * up_f), silu(z) = z / (1 + e^-z)
 *   HXF_EPI_F32:    C fp32 [M, ldc]            C = y
 * A and B (and B2): codes as above, 16-byte aligned.  B2 and b2_scale are unused but for SwiGLU.  ldc >= N (SwiGLU: F);
 * elements behind a row's columns are left as they are.  M <= 2^22 - 16, 0 < N <= 2^22 - 16, 0 < K < 2^17, M * N < 2^34.
 * workspace: hxf_op_gemm_i8_workspace_bytes(M, N, K) bytes are enough for every epilogue and every product of at most M rows,
 * N columns and K (may be 0; never more than HXF_GEMM_I8_MAX_WORKSPACE, which is enough for any), 16-byte aligned, whose
 * contents need not be kept between calls; calls that may overlap need one each.  HXF_ENOMEM (nothing enqueued) only where
 * the pieces of K that this product is cut into, 4 M N bytes each, do not fit.  No buffer may overlap another. */
#define HXF_GEMM_I8_MAX_WORKSPACE (72LL << 20)
int64_t hxf_op_gemm_i8_workspace_bytes(int32_t M, int32_t N, int32_t K);
/* Introspection (host only, no device work): the plan hxf_op_gemm_i8 takes for these sizes:
 * plan = {row tiles of 16, column tiles of 16 per wavefront, wavefronts, 1 if the weights are fetched as read once,
 * pieces of K, tiles of 64 of K per piece, 1 if the wavefronts of a workgroup share out K (column tiles are then the
 * workgroup's)}. */
int hxf_op_gemm_i8_plan(int32_t M, int32_t N, int32_t K, int32_t epilogue, int32_t plan[7]);
int hxf_op_gemm_i8(const void* A, const float* a_scale, const void* B, const float* b_scale, const void* B2,
                   const float* b2_scale, void* C, int32_t ldc, int32_t M, int32_t N, int32_t K, int32_t epilogue,
                   void* workspace, int64_t workspace_bytes, void* stream);

/* out[r] = argmax over v of logits fp32 [R, V]; the lowest index wins ties. */
int hxf_op_argmax(const float* logits, int32_t* out, int32_t R, int32_t V, void* stream);

/* dst = src, bytes % 16 == 0 (HBM bandwidth probe). */
int hxf_op_copy(const void* src, void* dst, int64_t bytes, void* stream);

/* HBM read-bandwidth probe: reads src (bytes % 16 == 0) once with 16-byte loads and
 * writes to sink (device, HXF_READ_SINK_WORDS uint32 words, caller-owned) one word per
 * thread of the launch, the XOR of the 32-bit words that thread read; words of sink
 * past the launch's threads are left as they are, so the XOR of the whole sink, zeroed
 * first, is the XOR of every 32-bit word of src. */
#define HXF_READ_SINK_WORDS (4096 * 256)
int hxf_op_read(const void* src, int64_t bytes, uint32_t* sink, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HXF_OPS_H */
