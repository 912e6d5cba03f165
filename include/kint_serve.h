/*
 * kint_serve.h -- C ABI of libkint's serving operators: answering with a model whose
 * attention is K-interval attention, from a paged cache that holds keys and values in
 * 4 bits, on one NVIDIA GB300 (sm_103a).
 *
 * One serving step of a layer is, in this order on one stream,
 *   kint_blocks_extend   block tables, slots and positions from the requests' lengths
 *                        (once a step, not once a layer),
 *   kint_cache_append    the new tokens' keys (rotated) and values into the cache, and
 *                        their queries rotated in the same launch,
 *   kint_cache_attn      the new tokens' queries against the cache.
 * kint_rope rotates queries and keys on their own (training, prompts), forward and
 * backward; kint_cache_read hands cached rows back as numbers.
 *
 * Conventions
 *   - Return codes, kint_get_status, kint_strerror and the launch hook are those of
 *     kint_attn.h; errors are returned before any work is enqueued.  The library never
 *     allocates or synchronises.  Work runs on `stream`; calls that share a cache, a table
 *     or a workspace on different streams have to be ordered by the caller.
 *   - Index data that a kernel finds out of range (a block number, slot, position or
 *     length; they live on the device, so the host cannot see them) is skipped, never
 *     followed, and sets bit 8 of the status word that kint_get_status reports.
 *   - Tensors of queries, keys, values and outputs are fp32, bfloat16 or fp16 (one type
 *     a call) with any strides over batch, time and head and contiguous channels
 *     (kint_heads); they need the alignment of one element only.
 *   - Sums, row statistics and weights are fp32.  Scores are taken to be finite and below 0.9e38 in magnitude, and bfloat16 queries
 *     below 2^120.
 *   - Sizes have to fit their kernels' 32-bit indices: KINT_ERR_UNSUPPORTED past 2^30 rows (new tokens times query heads) a kv head, 2^30
 *     units (request, kv head, row tile), 2^24 heads, 2^31 - 256 tokens an append or read.
 *
 * The cache.  A pool of num_blocks blocks of block_size tokens (a power of two, 16 to
 * 4096); block n of the pool starts at pages + n * block_stride bytes and holds, for
 * each kv head, block_size / 16 slabs of 18 * d bytes.  A slab is 16 consecutive tokens:
 *   K codes  8 d bytes | K scales  d bytes | V codes  8 d bytes | V scales  d bytes
 * A channel's value is s * (code - 8) + c, with one pair of fp16 numbers (s, c) for each
 * 64 channels of a token (scales: [16 tokens][d / 64] pairs).  Storing x: lo and hi the
 * smallest and largest of the 64, s = fp16((hi - lo) * fp32(1 / 15)), c = fp16(lo + 8 s) (fp16
 * with saturation), code = clamp(rint((x - c) * (1 / s)) + 8, 0, 15) in fp32, 8 where s is 0;
 * a group that holds an infinity or a NaN is stored with c = NaN.  K codes: the 32-bit
 * word of channels 32 i + 8 t .. + 7 (lowest nibble first) of token j at byte
 * j d / 2 + t d / 8 + 4 i.  V codes: tokens 2 p and 2 p + 1 share the word of channels
 * 64 r + 8 g + 4 h .. + 3 at byte ((8 p + g) d / 32 + 2 r + h) * 4, the even token's four
 * nibbles in the low half.  (Both orders are the register order of the attention
 * kernel's tensor-core operands: a lane's codes are contiguous.)
 * A token's slot is block * block_size + offset; -1 stands for no slot.
 */
#ifndef KINT_SERVE_H
#define KINT_SERVE_H

#include "kint_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { KINT_FP32 = 0, KINT_BF16 = 1, KINT_FP16 = 2 } kint_dtype;

/* A tensor [batch][time][heads][d]: element strides, channels contiguous. */
typedef struct {
  void* ptr;
  long long stride_b, stride_t, stride_h;
  int heads;
} kint_heads;

/* A cache pool (see above).  pages and block_stride: multiples of 16 bytes. */
typedef struct {
  void* pages;
  long long block_stride; /* bytes from one block to the next */
  int num_blocks, block_size, kv_heads, d; /* d: 64 or 128 */
} kint_cache;

/* Bytes of one block (the smallest block_stride); 0 for invalid sizes. */
size_t kint_cache_block_bytes(int block_size, int kv_heads, int d);

/*
 * Block tables and slot maps of one step, from the requests' lengths.
 *   lens      in  [B] int32: tokens each request has in the cache
 *   add       in  [B] int32: new tokens of this step (0: none; negative counts as 0 and is flagged)
 *   table     in/out [B][table_stride] int32, the first `width` of a row used: the blocks of each
 *             request in order; the blocks this step takes are written behind them
 *   free_list in  [free_len] int32: free block numbers; n_free [1] of them are valid, taken from
 *             the end (the k-th block taken is free_list[n_free - 1 - k], in order of requests)
 *   lens_out  out [B], n_free_out [1]: the lengths and the free count after the step
 *   cu        out [B + 1] int32: prefix sums of add (row offsets of the requests' new tokens)
 *   slots, pos, req  out [tokens] int64, int32, int32: slot, position and request of every new
 *             token; places past cu[B] get -1.  Tokens past `tokens` places are not written, and flagged.
 *   refused   out [1] int32: requests that got no blocks: their row of the table is too short, or the
 *             free blocks ran out (requests are served in order; from the first that finds too few,
 *             every one that needs a block is refused).  Their slots are -1 and their length stays, but cu counts their
 *             tokens: hand the slots to kint_cache_attn_step, which answers them with zeros.
 * The outputs must not overlap the inputs (table apart), so the call can be repeated.  1 <= B <= 16384.
 */
int kint_blocks_extend(const int32_t* lens, const int32_t* add, int32_t* table, int table_stride, int width,
                       const int32_t* free_list, int free_len, const int32_t* n_free, int B, int block_size,
                       int tokens, int32_t* lens_out, int32_t* n_free_out, int32_t* cu, int64_t* slots, int32_t* pos,
                       int32_t* req, int32_t* refused, void* stream);

/*
 * Table of rotations: table[p][i] = (mag cos(p f_i), mag sin(p f_i)), p < max_pos, i < rot / 2, as fp32 pairs,
 * the angle and its functions in fp64.  freq: rot / 2 angles a position (host memory, read during the call).
 */
int kint_rope_table(float* table, int max_pos, int rot, const double* freq, double mag, void* stream);

/*
 * Rotary positions of queries and keys [B][T][heads][d], one launch for both (k may have 0 heads).
 * The first `rot` channels (even, 2 <= rot <= d) are pairs: (i, i + rot / 2), or with interleaved (2 i, 2 i + 1);
 *   (a, b) -> (a cos - b sin, b cos + a sin)
 * with (cos, sin) = table[pos][i]; the rest is copied.  inverse: sin -> -sin, which is the gradient's way back.
 * Outputs may be the inputs themselves (same strides); otherwise they must not overlap.
 *   pos  [B or 1][T] int32 (pos_stride_b elements between batches; 0: one row for all); -1: a padding token, copied.
 * d <= 256, even; at most 2^31 pairs of (token, pair of channels, group of 8 heads).
 */
int kint_rope(const kint_heads* q, const kint_heads* q_out, const kint_heads* k, const kint_heads* k_out,
              const int32_t* pos, long long pos_stride_b, const float* table, int max_pos, int B, int T, int d, int rot,
              int interleaved, int inverse, kint_dtype dtype, void* stream);

/*
 * New tokens into the cache: token n's keys and values k[n], v[n] ([tokens][kv_heads][d]; stride_b unused) to slots[n]
 * (-1: skipped).  With table non-NULL the keys are rotated first (kint_rope's rotation, in fp32, quantised without
 * an intermediate rounding) and, when q is non-NULL, q[n] is rotated into q_out[n] (may be q itself).
 */
int kint_cache_append(const kint_cache* cache, const kint_heads* k, const kint_heads* v, const int64_t* slots, int tokens,
                      const kint_heads* q, const kint_heads* q_out, const int32_t* pos, const float* table, int max_pos,
                      int rot, int interleaved, kint_dtype dtype, void* stream);

/* Cached keys and values of `tokens` slots as numbers, into k[n], v[n] (either may be NULL); slot -1 gives zeros. */
int kint_cache_read(const kint_cache* cache, const int64_t* slots, int tokens, const kint_heads* k, const kint_heads* v,
                    kint_dtype dtype, void* stream);

/*
 * K-interval attention of each request's new tokens over its cached keys.
 *   q, out   [rows][q_heads][d] (stride_b unused); q_heads a multiple of kv_heads (consecutive query heads share one)
 *   table    [B][table_stride] int32 block numbers, `width` of a row used
 *   lens     [B] int32: cached tokens, the new ones among them
 *   cu       [B + 1] int32: request b's new tokens are rows cu[b] .. cu[b + 1] - 1 of the `rows` there are, its last
 *            positions: row r sits at position p = lens[b] - cu[b + 1] + r
 *   A row sees keys j <= p, and with window > 0 only those with j > p - window or j < sinks.  A row that sees no key
 *   (p < 0) gives zeros.
 *   Kint, calib, tau, recon: the weights, as for kint_attn_fwd (the hard forward under Nearest); the grid is
 *   anchored at the row's extrema over the keys it sees.
 *   max_new  bound on cu[b + 1] - cu[b]; max_len bound on lens[b] (<= width * block_size): they size the launch and
 *            the workspace (with loose bounds both grow: every row that could be there has its place); rows or keys past them are left out and flagged, and so are requests whose rows do not lie
 *            within 0 .. rows.
 *   workspace: kint_cache_attn_workspace_bytes bytes (16-byte aligned).  256 bytes are asked for, and not touched, where the
 *            scores fit the shared memory of one launch.
 * Results do not depend on the order in which thread blocks run.
 */
int kint_cache_attn(const kint_heads* q, const kint_heads* out, const kint_cache* cache, const int32_t* table,
                    int table_stride, int width, const int32_t* lens, const int32_t* cu, int rows, int B, int window,
                    int sinks, int Kint, kint_calib calib, float tau, kint_recon recon, int max_new, int max_len, kint_dtype dtype,
                    void* workspace, size_t workspace_bytes, void* stream);
/*
 * kint_cache_attn for a step as kint_blocks_extend plans it, with places left over and requests refused:
 *   slots  [rows] int64, the slots of q's rows, or NULL.  A request whose first new token has none (-1) was refused: its new
 *          tokens are not in the cache, lens[b] does not count them, and its rows give zeros.  Without slots they are taken for
 *          the last lens[b] positions, which hold older tokens.
 *   fill   non-zero: rows of `out` that are no request's (before cu[0], from cu[B] on), and rows that are left out, get zeros; 0, as
 *          in kint_cache_attn: they are left as they are.
 */
int kint_cache_attn_step(const kint_heads* q, const kint_heads* out, const kint_cache* cache, const int32_t* table,
                         int table_stride, int width, const int32_t* lens, const int32_t* cu, int rows, int B, int window,
                         int sinks, int Kint, kint_calib calib, float tau, kint_recon recon, int max_new, int max_len, kint_dtype dtype,
                         const int64_t* slots, int fill, void* workspace, size_t workspace_bytes, void* stream);
size_t kint_cache_attn_workspace_bytes(int B, int q_heads, int kv_heads, int d, int window, int sinks, int max_new,
                                       int max_len);

#ifdef __cplusplus
}
#endif
#endif
