/*
 * bq4.h -- C ABI of the 4-bit variant of libbq's dynamic blockwise quantization: the same
 * method as bq.h with a 16-entry codebook and two codes per byte, so that a 16-bit hidden
 * state crosses a shard boundary in a quarter of its bytes (plus one fp32 absmax per block).
 *
 * Source of the operation: the paper's section "Compression techniques", item 1 ("Dynamic
 * Quantization") names dynamic blockwise quantization of the exchanged hidden states; the
 * 8-bit form of bq.h is the one it reports (halved bandwidth).  The bit width is a parameter
 * of the technique the paper leaves open; this header is the 4-bit point of it.
 *
 * Conventions are those of bq.h (device pointers owned by the caller, flattened row-major
 * tensor cut into blocks of `block` elements, last block may be short, work enqueued on
 * `cuda_stream`, status codes of bq.h, nothing allocated per call) with these differences:
 *   - codes: element 2i sits in the low nibble of byte i, element 2i + 1 in the high nibble;
 *     `packed` has ceil(n / 2) bytes; the unused high nibble of an odd n is written as 0.
 *   - Power-of-two blocks of 8 to 65536 elements on 16-byte aligned x / y (4-byte aligned
 *     packed) take vectorised kernels; everything else takes slower general kernels with
 *     identical results.
 */
#ifndef BQ4_H
#define BQ4_H

#include <stddef.h>
#include <stdint.h>

#include "bq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Opaque: the 16 code values and the 15 search thresholds derived from them (host memory only). */
typedef struct bq4_codebook bq4_codebook;

/*
 * bq4_make_codebook -- kind = BQ_CODEBOOK_DYNAMIC_TREE: the dynamic-tree map with 4 bits: a sign
 * bit; in the other 3 bits the first set bit picks decade k = 0..2 (scale 10^(k-2)) and leaves k
 * bits of linear fraction, m(k, j) = 10^(k-2) (0.1 + 0.9 (2j + 1) / 2^(k+1)); plus 0 and 1.
 * Ascending, the code is the index, 0.0 is code 7, +1.0 is code 15, the lowest value is -0.8875.
 * kind = BQ_CODEBOOK_USER: user_values16 (HOST, 16 floats) finite, strictly ascending, within
 * [-1, 1], no non-zero magnitude below 2^-24; else BQ_ERR_CODEBOOK.
 * host_values_out16 (HOST, may be NULL) receives the values.  No device memory is involved.
 */
int bq4_make_codebook(int kind, const float* user_values16, float* host_values_out16, bq4_codebook** out);

/* Frees the handle.  NULL is allowed. */
int bq4_free_codebook(bq4_codebook* cb);

/*
 * bq4_quantize -- per block b: absmax_out[b] = max |x_i| (fp32); xhat_i = x_i / absmax_out[b] as
 * one IEEE fp32 division (divisor 1 for an all-zero block); code_i = index of the nearest codebook
 * value, equal distances to the smaller index; codes packed two per byte.
 *   x: n elements of type xdt.  packed_out: ceil(n / 2) bytes.  absmax_out: ceil(n / block) floats.
 */
int bq4_quantize(const void* x, bq_dtype xdt, size_t n, int block, const bq4_codebook* cb,
                 uint8_t* packed_out, float* absmax_out, void* cuda_stream);

/*
 * bq4_dequantize -- y_out[i] = round-to-nearest-even to ydt of the fp32 product
 * value[code_i] * absmax[i / block].
 */
int bq4_dequantize(const uint8_t* packed, const float* absmax, size_t n, int block, const bq4_codebook* cb,
                   void* y_out, bq_dtype ydt, void* cuda_stream);

/*
 * bq4_quantize_s16 / bq4_dequantize_s16 -- the same codec with the block scale stored in two
 * bytes instead of four (at block 64 the fp32 absmax is 11 % of the 4-bit payload, the 16-bit
 * scale 6 %).  The paper fixes no format for the scale; this is a variant of its "Dynamic
 * Quantization" item.
 *   scale_b = the block's absmax rounded toward +infinity to a bf16 (1 sign, 8 exponent, 7
 *   fraction bits), so that no |x_i| / scale_b exceeds 1; never above the largest finite bf16
 *   (inputs above it are outside the contract); 0 for an all-zero block.  scale_out[b] holds the
 *   bf16's 16 bits.  xhat_i = x_i / scale_b as one IEEE fp32 division (divisor 1 for a zero
 *   block); codes and packing as in bq4_quantize.  Dequantize: y_i = round-to-nearest-even to
 *   ydt of the fp32 product value[code_i] * scale_b.
 *   scale_out / scale: ceil(n / block) 16-bit words, device memory, 2-byte aligned.
 * Arguments, errors and kernels otherwise as bq4_quantize / bq4_dequantize.
 */
int bq4_quantize_s16(const void* x, bq_dtype xdt, size_t n, int block, const bq4_codebook* cb,
                     uint8_t* packed_out, uint16_t* scale_out, void* cuda_stream);
int bq4_dequantize_s16(const uint8_t* packed, const uint16_t* scale, size_t n, int block, const bq4_codebook* cb,
                       void* y_out, bq_dtype ydt, void* cuda_stream);

/* ------------------------------------------------------------------------------------------
 * The key/value cache of a shard held in this 4-bit form, and the attention that reads it.
 *
 * Source of the operation: every node of the paper's sequential shards keeps the key/value cache of
 * its own blocks (section on the memory of a block: 2 head_dim n_heads n_layers values per token),
 * the other large activation tensor next to the exchanged hidden states.  The paper compresses the
 * latter; here the former is stored by the same codec.  The paper has no counterpart of these calls.
 *
 * Layout.  The cache is cut into pages of `page` rows; a row is one token's key (or value) of one
 * head, stored exactly as bq4_quantize_s16 stores head_dim elements with blocks of `block`:
 *     k_codes, v_codes: [n_pages, kv_heads, page, head_dim / 2] bytes (16-byte aligned)
 *     k_scale, v_scale: [n_pages, kv_heads, page, head_dim / block] bf16 words (16-byte aligned)
 * Slot j of sequence s is row j % page of page table[s * table_stride + j / page].  lens[s] counts the
 * slots of sequence s that are in use.  All pointers are DEVICE memory of the caller.  The calls take a
 * negative lens for 0 and clamp page numbers to 0 .. n_pages - 1: a table with bad entries gives
 * unspecified results, never an access outside the pools.
 *
 * Rows of a call.  append, read and attend work on `n_rows` rows, starts[s] .. starts[s + 1] - 1 being
 * those of sequence s (starts: DEVICE, n_seq + 1 ints, ascending from 0 to n_rows; NULL: one row per
 * sequence, n_rows == n_seq).  The n_s rows of a sequence are its LAST n_s slots: the caller counts
 * new tokens into lens, then appends their keys and values, then attends with their queries.
 * A sequence may have no rows, and no slots.  lens may count past the table's end, max_pages * page slots:
 * rows keep the place that lens gives them, and those whose place lies behind the end are not held.  They
 * are dropped by append, read as zeros, and attend to all slots that are held; nothing else moves for them.
 * evict sees the slots that are held.
 *
 * Limits: head_dim a multiple of 8, 8 .. 256; block a multiple of 8 that divides head_dim; kv_heads
 * 1 .. 1024, n_pages * kv_heads below 2^31; page 1 .. 65536; n_seq 1 .. 65535; max_pages * page below 2^30; max_pages <= table_stride;
 * n_rows at most 2^27.
 * Element types BQ_F16 and BQ_BF16.  Inputs must be finite, magnitudes of keys and values below 2^90
 * (a score is a product of up to 2^33 and the key's scale in fp32 before the query's factor joins it);
 * whatever lies in slots a call does not address (NaN bit patterns included) does not matter.
 */
typedef struct bqkv_cache {
    uint8_t* k_codes;
    uint8_t* v_codes;
    uint16_t* k_scale;
    uint16_t* v_scale;
    const int32_t* table;
    int32_t* lens;
    int n_pages, kv_heads, page, head_dim, block, n_seq, max_pages, table_stride;
} bqkv_cache;

/* Additional status code (the value of MMD_ERR_WORKSPACE, the same text). */
enum { BQKV_ERR_WORKSPACE = 7, BQKV_ERR_PATH = 9 };

/*
 * bqkv_append -- writes the rows of the call into their slots.
 *   k, v: [n_rows, kv_heads, head_dim] of type dt, heads contiguous, rows k_stride / v_stride ELEMENTS
 *   apart (a slice of a wider projection is taken as it is; any alignment of the elements' own size).
 *   Codes and scales are those of bq4_quantize_s16.  A row whose slot would be negative or past
 *   max_pages * page is dropped.
 */
int bqkv_append(const bqkv_cache* c, const bq4_codebook* cb, const void* k, const void* v, bq_dtype dt, int64_t k_stride, int64_t v_stride,
                const int32_t* starts, int n_rows, void* cuda_stream);

/*
 * bqkv_make_rotary -- how queries and keys turn by their positions: pair i of the first rotary_dim elements of a head's row turns
 * by the angle position * frequencies[i].  HOST memory only.
 *   rotary_dim: even, 2 .. 256 and at most the cache's head_dim; the elements behind it stay as they are.
 *   frequencies: HOST, rotary_dim / 2 radians per position, magnitudes up to 65536.
 *   axis_of_pair: HOST, rotary_dim / 2 entries of 0 .. axes - 1: whose position turns the pair, where a token has several (time, height,
 *   width); NULL with one axis.  axes: 1 .. 255.
 *   interleaved: pairs are elements (2i, 2i + 1); otherwise (i, i + rotary_dim / 2).
 */
typedef struct bqkv_rotary bqkv_rotary;
int bqkv_make_rotary(int rotary_dim, const double* frequencies, const int32_t* axis_of_pair, int axes, int interleaved, bqkv_rotary** out);

/* Frees the handle.  NULL is allowed. */
int bqkv_free_rotary(bqkv_rotary* r);

/*
 * bqkv_append_rotary -- bqkv_append with the rows' positions: (x, y) -> (x cos a - y sin a, y cos a + x sin a) for every pair of queries
 * and keys.  Keys are turned in 64 bits, rounded once to fp32 and stored as bqkv_append stores a row of those values; values are stored as
 * they are; queries are turned in fp32, rounded once to dt and written to q_out.
 *   q: [n_rows, q_heads, head_dim] of type dt, rows q_stride elements apart; any number of heads up to 65535, 0 for none (q, q_out NULL).
 *   positions: DEVICE, an int32 (negative ones too) per row and axis, axes positions_stride elements apart, at least n_rows (ignored with
 *   one axis); NULL: a row's place as lens counts it, on every axis.  The angle is right to 10^-9 radian for every position.
 *   q_out: rows q_out_stride elements apart; q itself with its stride, or memory that meets none of q, k, v (BQ_ERR_SIZE).
 *   A row without a slot has its queries turned and its key and value dropped; rows that belong to no sequence are left alone.
 * Arguments otherwise as bqkv_append.
 */
int bqkv_append_rotary(const bqkv_cache* c, const bq4_codebook* cb, const bqkv_rotary* rotary, const void* q, const void* k, const void* v, bq_dtype dt,
                       int64_t q_stride, int64_t k_stride, int64_t v_stride, int q_heads, const int32_t* positions, int64_t positions_stride,
                       const int32_t* starts, int n_rows, void* q_out, int64_t q_out_stride, void* cuda_stream);

/*
 * bqkv_read -- the inverse: k_out, v_out [n_rows, kv_heads, head_dim] of type dt, contiguous, receive
 * the values of the rows' slots as bq4_dequantize_s16 gives them (zeros for a slot that does not exist).
 */
int bqkv_read(const bqkv_cache* c, const bq4_codebook* cb, const int32_t* starts, int n_rows, void* k_out, void* v_out, bq_dtype dt,
              void* cuda_stream);

/* Kernel choice of bqkv_attend. */
enum {
    BQKV_PATH_AUTO = 0,
    BQKV_PATH_GENERAL = 1, /* any head size, block and page                                                            */
    BQKV_PATH_ROWS = 2,    /* few query rows per cached head (a decode step, a few rows over long contexts), bound by
                              the stream of the cache:
                              head_dim 64 with blocks of 64 or 32, or 128 with 128, 64 or 32; pages a multiple of 16;
                              q 4-byte aligned with an even stride (BQKV_ERR_PATH otherwise)                           */
    BQKV_PATH_TILES = 3    /* many query rows per cached head (a prompt) on the tensor cores; the same shapes          */
};

/*
 * bqkv_attend -- causal attention of the rows' queries over the cache, q_heads / kv_heads query heads
 * sharing each cached head (query head h reads cached head h / (q_heads / kv_heads)):
 *     x_j   = sm_scale * sum_d q_d key_jd        for slots j <= slot of the row itself
 *     p_j   = exp(x_j) / sum_j exp(x_j)
 *     out_d = sum_j p_j value_jd                 rounded to dt; zeros for a row that sees no slot
 *     weights[s, kv head, j] += sum of p_j over the sequence's rows and the query heads of the group
 *   q: [n_rows, q_heads, head_dim] of type dt, heads contiguous, rows q_stride elements apart.
 *   out: the same shape, contiguous; it may be q itself where q is contiguous and no weights are wanted, and shares no memory
 *   with q otherwise (BQ_ERR_SIZE).  q_heads a multiple of kv_heads, at most 1024 per cached head.
 *   weights: DEVICE floats [n_seq, kv_heads, weights_stride] that are added to, or NULL; a slot at or
 *   beyond weights_stride is not added to.  No atomics: the same call gives the same bits.
 *   max_new, max_len: the caller's (host) bounds on the rows of one sequence and on lens.  They size
 *   the launch; larger actual values still give right results.  max_len <= 0: max_pages * page.
 *   workspace: bqkv_attend_workspace bytes for the same sizes, 256-byte aligned; its first 1024 bytes
 *   are zeroed by the caller once, when it is allocated.  Calls that share a workspace must not
 *   overlap on the device.  with_weights: 0, 1, or 2 for weights on a BQKV_PATH_ROWS that is asked for
 *   by name (it keeps the scores of every row in the workspace; by itself a call with weights takes
 *   that path up to 16 query rows per cached head only).
 * Sums, maxima and softmax statistics are fp32.  BQKV_PATH_GENERAL is fp32 throughout.  The two others multiply fp16 numbers and
 * sum in fp32; what they round on the way:
 *   - codebook values to 11 significant bits, where no common factor up to 2048 makes them whole numbers of 11 bits (the dynamic
 *     tree and linear maps of up to 2048 steps are exact; an irregular USER codebook is not), in keys and values alike;
 *   - a query row's elements below 2^-29 of its largest one lose bits;
 *   - the product of a probability and the value's scale to 11 bits for bf16 outputs, 22 for fp16 outputs, in steps of no less than
 *     2^-31 (BQKV_PATH_ROWS) or 2^-34 (BQKV_PATH_TILES) of the row's largest such product;
 *   - BQKV_PATH_TILES with several blocks per row: value times scale to 11 bits for bf16 outputs (22 for fp16 outputs), and blocks
 *     whose scale is below 2^-17 of the largest scale of their row (of keys or of values) lose bits.
 * Rows whose value scales are all below 2^-80 lose their lightest slots first, below 2^-100 bits of all; scales below 2^-126 count as zero.
 */
int bqkv_attend_workspace(const bqkv_cache* c, int n_rows, int q_heads, int max_new, int max_len, int with_weights, size_t* bytes);
int bqkv_attend(const bqkv_cache* c, const bq4_codebook* cb, const void* q, bq_dtype dt, int64_t q_stride, const int32_t* starts, int n_rows,
                int q_heads, int max_new, int max_len, float sm_scale, float* weights, int64_t weights_stride, void* out, void* workspace,
                size_t workspace_bytes, int path, void* cuda_stream);

/*
 * bqkv_attend_shared -- bqkv_attend for sequences that begin with the same rows, which are attended to once for all that share them:
 * a row sees every slot of its sequence's prefix, then the sequence's own slots up to its own,
 *     x_j = sm_scale * sum_d q_d key_jd over both, p = softmax(x), out = sum_j p_j value_j.
 *   prefix: a cache (over the same pools or others) whose sequences are the prefixes; kv_heads, head_dim and block are the cache's, pages
 *   and tables its own; its lens count the prefixes' slots.  Rows of prefixes are stored with bqkv_append through that cache.
 *   members: DEVICE, prefix->n_seq + 1 ints, ascending: sequences members[p] .. members[p + 1] - 1 share prefix p; sequences outside of
 *   members[0] .. members[n] - 1 have none.  NULL: the only prefix is everybody's.
 *   weights: of the cache's own slots, as for bqkv_attend (the softmax runs over both); prefixes have none.
 *   out: as for bqkv_attend; without weights and on the kernels for head_dim 64 and 128 it may also meet q.
 *   max_shared, max_prefix: the caller's (host) bounds on the rows that share one prefix and on the prefixes' lens, for the launch's sizes
 *   only, like max_new and max_len; <= 0: n_rows, the prefix table's whole length.
 *   path: the kernel for the prefixes; the own slots' is chosen as BQKV_PATH_AUTO does (BQKV_PATH_GENERAL: both).
 *   workspace: bqkv_attend_shared_workspace bytes, otherwise as for bqkv_attend (bqkv_kernel_status reads it too).
 * The two sides' sums, in fp32, are joined in fp32: one rounding to dt at the end.  What the kernels round is said at bqkv_attend.
 */
int bqkv_attend_shared_workspace(const bqkv_cache* c, const bqkv_cache* prefix, int n_rows, int q_heads, int max_new, int max_len, int max_shared, int max_prefix,
                                 int with_weights, size_t* bytes);
int bqkv_attend_shared(const bqkv_cache* c, const bqkv_cache* prefix, const bq4_codebook* cb, const int32_t* members, const void* q, bq_dtype dt, int64_t q_stride,
                       const int32_t* starts, int n_rows, int q_heads, int max_new, int max_len, int max_shared, int max_prefix, float sm_scale, float* weights,
                       int64_t weights_stride, void* out, void* workspace, size_t workspace_bytes, int path, void* cuda_stream);

/*
 * bqkv_kernel_status -- 0, or the code a kernel of BQKV_PATH_TILES left in the workspace (its first word) when one of
 * its waits, which are bounded to about two seconds, ran out: the outputs of that call are then incomplete.
 * Synchronises the device, reads the word and clears it.  status_out: HOST.
 */
int bqkv_kernel_status(void* workspace, int* status_out);

/*
 * bqkv_evict -- bounds every sequence to `budget` slots.  For each sequence with lens[s] > budget and
 * each of its heads on its own: slots 0 .. sinks - 1 and the last `recent` slots stay; of the slots
 * between them the budget - sinks - recent with the largest weights stay (equal weights: the lower
 * slot; NaN counts below every number).  Then, in place:
 *   - the slots of [sinks, budget - recent) that do not stay are filled, in ascending order, by the
 *     staying slots of [budget - recent, lens[s] - recent), in ascending order;
 *   - the recent rows move, in order, to [budget - recent, budget);
 *   - weights move with their rows; slots at and past `budget` keep what they held;
 *   - lens[s] = budget.
 * Only rows that have to move are touched, so a step that brings one row and evicts one moves
 * recent + 1 rows at most.  The kept rows' order among themselves is not the order of arrival
 * (attention does not depend on it).
 *   weights: as for bqkv_attend, weights_stride at least every lens[s] that exceeds the budget.
 *   0 <= sinks, 0 <= recent, 1 <= budget, sinks + recent <= budget (BQ_ERR_SIZE otherwise).
 *   workspace: bqkv_evict_workspace bytes, 256-byte aligned; its contents do not matter.
 */
int bqkv_evict_workspace(const bqkv_cache* c, int budget, size_t* bytes);
int bqkv_evict(const bqkv_cache* c, float* weights, int64_t weights_stride, int budget, int sinks, int recent, void* workspace,
               size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif
