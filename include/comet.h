/*
 * libcomet -- error-bounded lossy compression of convolution activations for
 * memory-efficient CNN training (COMET), native HIP for gfx950 (MI355X).
 *
 * The codec is the paper's "modified cuSZ" (Sec. 3.4, Sec. 4.1): quantise the
 * fp32 activations against an absolute error bound eb, predict every point from
 * its neighbours (2-D Lorenzo over each H x W plane), turn the residual into an
 * integer quantisation code, Huffman-code the codes; on decompression undo the
 * steps and re-zero every value that lies within eb of zero.  The error-bounded
 * mode guarantees |x - xhat| <= eb for every element (Sec. 2.2).
 *
 * Conventions for every entry point
 *   - "dev" pointers are device memory on the current HIP device, owned by the
 *     caller; "host" pointers are ordinary host memory.  Nothing is allocated
 *     per call: all scratch lives in the comet_ctx.
 *   - Tensors are fp32, NCHW, contiguous.  N*C*H*W must be in [1, 2^31) and
 *     W <= 8192.
 *   - All device work is enqueued on `stream` (a hipStream_t passed as void*;
 *     NULL is the default stream).  A context must not be used by two calls
 *     that can overlap in time; use one context per stream.
 *   - Return value: COMET_OK or a negative COMET_ERR_* code.  Conditions that
 *     are only known on the device (container too small, malformed container)
 *     are latched in the context and reported by the next synchronising call
 *     (comet_compress with bytes_out != NULL, or comet_sync).
 *   - NaN / Inf / huge inputs are not errors: they are stored verbatim and come
 *     back bit-identical.
 */
#ifndef COMET_H
#define COMET_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define COMET_OK 0
#define COMET_ERR_INVALID (-1)     /* bad argument (null pointer, zero dimension, eb or nbins out of range, ...) */
#define COMET_ERR_CAPACITY (-2)    /* the container does not fit the caller's buffer */
#define COMET_ERR_FORMAT (-3)      /* not a valid container / does not match the shape passed */
#define COMET_ERR_HIP (-4)         /* a HIP runtime call failed; see comet_strerror */
#define COMET_ERR_NOMEM (-5)       /* workspace allocation failed / context too small for the request */
#define COMET_ERR_INTERNAL (-6)    /* a device-side safety net tripped (should not happen) */
#define COMET_ERR_CODEBOOK (-7)    /* comet_compress_with_codebook: the length table is no complete prefix code, or the
                                      tensor needs an escape and the table has no code word for the escape symbol */

#define COMET_HEADER_BYTES 128u
#define COMET_DEFAULT_CHUNK_SYMS 64u

typedef struct comet_ctx comet_ctx;                     /* opaque; owns the device workspace */
typedef struct { uint32_t n, c, h, w; } comet_shape;    /* NCHW */

/* Header of a container, as returned by comet_peek (host copy). */
typedef struct {
    comet_shape shape;
    uint32_t nbins, chunk_syms, n_chunks, n_active, max_len, n_outlier_records, n_value_records;
    float eb;
    uint64_t nnz;            /* number of non-zero input elements (R of Sec. 4.2 = nnz / elements) */
    uint64_t payload_words, total_bytes;
} comet_info;

/* Create a context able to handle tensors of up to max_elems elements and
 * max_nbins quantisation bins.  Allocates 2 bytes per element plus about 42 MB
 * (2.14 bytes per element plus about 8 MB from 240 million elements on) of device workspace
 * on the current device.  *ctx is set on success. */
int comet_create(comet_ctx **ctx, uint64_t max_elems, uint32_t max_nbins);
void comet_destroy(comet_ctx *ctx);

/* Symbols per Huffman chunk for subsequent comet_compress calls: 64 (default),
 * 128 or 256.  Stored in the container; the decompressor reads it there. */
int comet_set_chunk_syms(comet_ctx *ctx, uint32_t chunk_syms);

/* Zero-chunk containers for subsequent comet_compress calls (off by default).
 * Activations behind ReLU are sparse (the ratio R of Sec. 4.2): a run of zeros,
 * like any constant run, leaves residual 0 after prediction, i.e. the centre
 * code nbins/2.  With enable != 0 a chunk that holds nothing but that code
 * takes no payload words at all (its entry in the chunk table equals the next
 * one; a chunk with symbols otherwise has at least one bit), and the container
 * says version 2 in its header; everything else, code book included, is as in
 * version 1.  The decompressor reads the version and takes either. */
int comet_set_zero_chunks(comet_ctx *ctx, int enable);

/* Worst-case container size in bytes for a shape (every element an outlier and
 * stored verbatim); 0 if the arguments are invalid.  Realistic activations need
 * a small fraction of it; callers that pass less rely on COMET_ERR_CAPACITY,
 * the paper's "unexpectedly low compression ratio" case (Sec. 3.4). */
uint64_t comet_compress_bound(comet_shape shape, uint32_t nbins, uint32_t chunk_syms);

/* Compress one activation tensor right after its layer's forward pass
 * (Sec. 3.4): dev_in (fp32, read-only) -> container at dev_out (16-byte
 * aligned, `capacity` bytes).  eb: absolute error bound, finite, in
 * [2^-100, 2^100].  nbins: even, in [4, 65536]; residuals outside
 * (-nbins/2, nbins/2) are stored as outliers.
 * bytes_out != NULL: the call synchronises `stream`, stores the container size
 * and returns any device-side error of this call (COMET_ERR_CAPACITY leaves the
 * buffer contents undefined but never writes past capacity) or, if this call
 * raised none, the first one that earlier asynchronous calls on this context
 * have latched (*bytes_out is then still this call's valid size).
 * bytes_out == NULL: fully asynchronous; the size is in the container header
 * (comet_peek) and errors are reported by comet_sync. */
int comet_compress(comet_ctx *ctx, const float *dev_in, comet_shape shape, float eb, uint32_t nbins,
                   void *stream, void *dev_out, uint64_t capacity, uint64_t *bytes_out);

/* Compress with the code book of an earlier compression of the same layer.  COMET refreshes a
 * layer's statistics only every W iterations because they change slowly (Sec. 3.1); the same holds
 * for the layer's histogram, so the histogram and the Huffman construction (Sec. 4.1) can be skipped
 * between refreshes; with the code words known beforehand the tensor is read once, every part of it
 * quantised and encoded by the same wavefront.  dev_len: device pointer to u8[nbins] code lengths (the length section of an
 * earlier container of the same nbins starts COMET_HEADER_BYTES into it); it must stay valid and
 * unchanged until the call has completed and may lie inside another container, not inside dev_out.
 * The lengths must form a complete prefix code (or one symbol of length 1), none above 57.  A
 * quantisation code without a code word in the table is stored like a residual outside the
 * alphabet (escape symbol + outlier record); the container carries the table, so it decompresses
 * with comet_decompress to exactly the values comet_compress would give.  Everything else as
 * comet_compress.  Limits: nbins <= 8192 and planes of at most 512 columns (COMET_ERR_INVALID
 * otherwise).  A table that is no such code, that lacks a code word for the escape symbol when
 * the tensor needs one, or that spends more than 16 bits per symbol on some run of rows (a run has
 * 2048 elements or more, unless the tensor has fewer; such a table expands the data) raises COMET_ERR_CODEBOOK (device-side: returned here if bytes_out is given,
 * else by comet_sync); the caller then compresses in full. */
int comet_compress_with_codebook(comet_ctx *ctx, const float *dev_in, comet_shape shape, float eb, uint32_t nbins,
                                 const uint8_t *dev_len, void *stream, void *dev_out, uint64_t capacity,
                                 uint64_t *bytes_out);

/* Decompress a container for the backward pass (Sec. 3.4): dev_in (`bytes`
 * bytes, 16-byte aligned) -> dev_out (fp32, shape.n*c*h*w elements).  `shape`
 * is the shape the caller compressed; it sizes the launch and is checked on
 * the device against the header.  Asynchronous; a malformed container is
 * reported by comet_sync (the output is then undefined, never out of bounds). */
int comet_decompress(comet_ctx *ctx, const void *dev_in, uint64_t bytes, comet_shape shape,
                     void *stream, float *dev_out);

/* Activations held in 16 bits (mixed-precision training; the paper trains in fp32 and this goes
 * beyond it).  The codec itself is the fp32 one of Sec. 4.1: comet_compress_16 widens every input
 * element to fp32 as it is loaded (exact for both types) and from there on is comet_compress, so
 * the container is byte for byte the one comet_compress writes for the widened tensor, and either
 * decompression reads it.  comet_decompress_16 rounds the fp32 result of comet_decompress to the
 * 16-bit type (nearest, ties to even; after the re-zero filter), so a value differs from the
 * input by at most eb plus half a unit in the last place of the 16-bit type; verbatim values come
 * back exactly.  dtype: COMET_F16 (IEEE binary16) or COMET_BF16 (bfloat16); the tensor is device
 * memory of the 16-bit type, owned by the caller (input of comet_compress_16: 16-byte aligned, as
 * for comet_compress; output of comet_decompress_16: any element-aligned address).  Limit: planes
 * of at most 512 columns (COMET_ERR_INVALID otherwise).  Errors, `bytes_out`, streams: as for the
 * fp32 calls. */
#define COMET_F16 1
#define COMET_BF16 2
int comet_compress_16(comet_ctx *ctx, const void *dev_in, int dtype, comet_shape shape, float eb, uint32_t nbins,
                      void *stream, void *dev_out, uint64_t capacity, uint64_t *bytes_out);
int comet_decompress_16(comet_ctx *ctx, const void *dev_in, uint64_t bytes, comet_shape shape, int dtype,
                        void *stream, void *dev_out);

/* comet_decompress for callers that cannot allocate device memory or hold a context: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  No comet_create is needed and
 * the call allocates nothing: its control block, decode tables and work buffer live in a static device
 * array inside the library (about 11 MiB, held by every GPU the library runs on until the process
 * ends), which limits the tensor to COMET_STATIC_MAX_ELEMS elements (COMET_ERR_NOMEM beyond).
 * dev_in, bytes, shape, stream, dev_out: as for comet_decompress.  dev_status: device memory, one
 * int32 owned by the caller, or NULL; when the call's kernels have run it holds COMET_OK, or
 * COMET_ERR_FORMAT if the container was refused (dev_out is then undefined, never out of bounds).
 * Asynchronous, kernels only.  All calls on one GPU share the one array: calls that can overlap in
 * time on the same GPU (two streams, two threads) race; issue them on one stream. */
#define COMET_STATIC_MAX_ELEMS (4u << 20)
int comet_decompress_static(const void *dev_in, uint64_t bytes, comet_shape shape, void *stream, float *dev_out,
                            int32_t *dev_status);

/* Wait for `stream` and return (then clear) the first device-side error latched
 * in the context since the last synchronising call. */
int comet_sync(comet_ctx *ctx, void *stream);

/* Read and validate a container's header (synchronises `stream`). */
int comet_peek(comet_ctx *ctx, const void *dev_in, uint64_t bytes, void *stream, comet_info *info);

/* Adaptive error bound (Sec. 3.2, 3.3): sigma = sigma_frac * momentum_abs_mean;
 * eb = sigma / (a * loss_grad_mean * sqrt(batch * nonzero_ratio)), evaluated in
 * fp64 on the host, rounded to fp32, clamped to [eb_min, eb_max].  The paper's
 * constants are a = 0.32 (Sec. 5.2) and sigma_frac = 0.01 (Sec. 3.2).
 * loss_grad_mean == 0 or nonzero_ratio == 0 returns eb_max. */
typedef struct { double momentum_abs_mean, loss_grad_mean, nonzero_ratio; uint32_t batch; } comet_layer_stats;
typedef struct { double a, sigma_frac; float eb_min, eb_max; } comet_adapt_cfg;
void comet_adapt_defaults(comet_adapt_cfg *cfg);   /* 0.32, 0.01, 2^-100, 2^100 */
int comet_adapt_eb(const comet_layer_stats *stats, const comet_adapt_cfg *cfg /* NULL = defaults */, float *eb_out /* host */);

/* Semi-online statistic for comet_layer_stats (Sec. 3.1: the average of the momentum, the average
 * gradient of the loss; taken as means of absolute values): mean of |dev_in[i]| over n fp32 values
 * on the device, accumulated in fp64 by a fixed tree (the same result on every call).  Synchronises
 * `stream`; *mean_out is host memory.  Non-finite inputs give a non-finite mean.  The fraction of
 * non-zero activations comes with every compression (comet_info.nnz). */
int comet_abs_mean(comet_ctx *ctx, const float *dev_in, uint64_t n, void *stream, double *mean_out);

/* Active factor W (Sec. 3.1), a host-side counter: statistics are collected and the error bounds
 * re-estimated every W iterations, W = 1000 by default; after a re-estimation, if the bound of any
 * layer changed by more than 2x (in either direction) since the previous one, W is halved (not below
 * 1), else it returns to its default. */
typedef struct { uint32_t w_default, w, since; } comet_controller;
int comet_controller_init(comet_controller *c, uint32_t w_default /* 0 = 1000 */);
/* One training iteration has passed; *collect = 1 in every W-th call. */
int comet_controller_tick(comet_controller *c, int *collect);
/* After a re-estimation: eb_old / eb_new are host arrays of the n_layers bounds before and after
 * (all finite and > 0, else COMET_ERR_INVALID). */
int comet_controller_update(comet_controller *c, const float *eb_old, const float *eb_new, uint32_t n_layers);

/* ---- keys and values of attention layers ------------------------------------------------------
 * What an attention layer keeps from one token to the next is activations as well, the ones a language model holds longest.
 * A whole tensor's Huffman stream can neither grow by a token nor be read in place, so they have a form of their own: blocks
 * of 32 tokens of one key/value head, uniformly quantised to 8 bits against the block's largest value, one scale for the
 * keys and one for the values: |x - xhat| <= scale / 2 with scale = max(largest |x| / 127, 2^-100), up to float32 rounding.  The block a sequence
 * is still filling lies in 16 bits, so every block is quantised once and the cache holds the same bytes whether the
 * tokens came one by one or all at once.
 *
 * The cache is one device buffer of comet_cache_bytes(shape), 16-byte aligned, owned by the caller; its contents need no
 * initialisation.  n_pages pages of page_tokens tokens (a multiple of 32) for each of `heads` heads of `dim` values (a multiple
 * of 32 up to 256); n_slots sequences can have an open block.  Sections, for per = page_tokens / 32:
 *   blocks  [n_pages][heads][per][64*dim]  keys int8 [dim/32][token][32], then values int8 [dim][place of the token]
 *   scales  [n_pages][heads][per][2] float32: keys, values (the section is padded to a multiple of 256 bytes)
 *   open    [n_slots][heads][2][128*dim + 256]  float16 in the same orders, then 32 float32 scales of the keys' tokens and 32 of
 *           the values'; block j of a sequence is in half j % 2
 * Token 16u + 8w + 4h + i of a block has place 16h + 8u + 4w + i.
 *
 * A batch describes, on the device, which tokens of which sequences a call is about; all three calls of a step take the same:
 *   dev_starts  int32[n_seqs + 1]: sequence b's new tokens are rows starts[b] .. starts[b+1]-1 of the tensors passed with
 *               it (none is fine; rows behind starts[n_seqs] are neither read nor written)
 *   dev_lens    int32[n_seqs]: tokens sequence b holds once these are in: the new tokens have the places lens[b] - n .. lens[b] - 1
 *   dev_table   int32[n_seqs][table_width]: the page of the tokens p * page_tokens ..; entries that are not reached are not read
 *   dev_slots   int32[n_seqs], or NULL for slot b
 * Two sequences of one append must not share a slot or a page that the call completes a block in (values undefined, never out of
 * bounds).  Complete blocks are not written again by tokens that follow, so sequences may share the pages of a
 * common beginning that ends with a block.  A sequence's length may be set back (drafted tokens that are not taken), as often as one likes, but
 * never to less than 32 tokens below the greatest length it has had: the slot holds the block of the greatest length and the one
 * before it in 16 bits, and what is older is gone (nothing tells the library, the values of the open block are then
 * others').  A block that a set-back opens is written again when it is complete once more, so its page must not be shared.
 * Conditions known on the device only (rows outside the tensors, a page that is none, a slot that is none, lens[b] < n in an append or fetch) store
 * COMET_ERR_FORMAT in *dev_status if that is given, and leave it alone otherwise (the caller clears it); what they
 * touch is skipped: rows left as they were, tokens of a page that is none not seen.  (starts that are outside of the rows or decrease may
 * make a call skip other sequences' rows too.)  A token whose key (value) holds Inf or NaN makes NaN of
 * the keys (values) of its block and head when read back, and of the rows that see any of the block.
 *
 * Tensors are [tokens][heads][dim] with strides in elements; the dim values of a row are contiguous; in those that are written no two rows may overlap,
 * and the rows of a token lie between those of its neighbours, or the rows of a head (else COMET_ERR_INVALID).  No row of a result may overlap a row of
 * another tensor of the call, unless the result is said to be allowed to be that tensor; two tensors that lie in one another's range (slices of one
 * buffer) must have the same token stride, by which that is told (else COMET_ERR_INVALID).  dtype: COMET_F16 or COMET_BF16
 * (comet_rope: COMET_F32 too).  Everything is asynchronous on `stream` and may be captured into a HIP graph; a replay
 * goes by what the batch's arrays hold then.  Nothing is allocated. */
#define COMET_F32 0
#define COMET_CACHE_BLOCK 32u
typedef struct { uint32_t n_pages, page_tokens, n_slots, heads, dim; } comet_cache_shape;
typedef struct { uint32_t n_seqs, table_width; const int32_t *dev_starts, *dev_lens, *dev_table, *dev_slots; } comet_cache_batch;
typedef struct { void *dev; int64_t token_stride, head_stride; } comet_rows;

/* Rotary positions: pair i of the first `rot` values of a head is turned by position * steps[i] turns and multiplied with amp;
 * the values behind are left alone.  layout: COMET_ROPE_HALVES pairs (i, i + rot/2), COMET_ROPE_PAIRS (2i, 2i + 1).
 * dev_steps: uint64[rot/2], turns per position in units of 2^-64, device memory of the caller: positions and steps are multiplied
 * exactly, so angles are right to 2^-31 turns at any position below 2^31. */
#define COMET_ROPE_HALVES 0u
#define COMET_ROPE_PAIRS 1u
typedef struct { uint32_t rot, layout; float amp; const uint64_t *dev_steps; } comet_rope_plan;

/* The steps of a plan, on the host.  Frequencies base^(-2i/rot) radians per position (rot even, 2 .. 4096; base > 1), scaled for contexts `factor`
 * (>= 1) times as long as the original_len tokens of the training: not at all; every frequency divided by the factor; the base raised to
 * base * factor^(rot/(rot-2)); or by parts (arXiv 2309.00071): those of less than beta_slow turns in original_len divided, of more than
 * beta_fast kept, in between in proportion, and *amp = 0.1 ln(factor) + 1 (1 otherwise).  beta_fast > beta_slow >= 0; original_len > 0. */
#define COMET_ROPE_PLAIN 0u
#define COMET_ROPE_LINEAR 1u
#define COMET_ROPE_BASE 2u
#define COMET_ROPE_PARTS 3u
typedef struct { uint32_t rot, scaling; double base, factor, original_len, beta_fast, beta_slow; } comet_rope_cfg;
int comet_rope_steps(const comet_rope_cfg *cfg, uint64_t *host_steps, float *amp);

/* y = x turned by its tokens' positions (dev_positions: int32[n_tokens], or NULL for 0, 1, ..).  backward != 0: turned the other way, which
 * takes the gradient of y to that of x.  y may be x (same strides).  dim: any from rot on. */
int comet_rope(const comet_rope_plan *plan, comet_rows x, comet_rows y, uint32_t n_tokens, uint32_t heads, uint32_t dim, int dtype,
               const int32_t *dev_positions, int backward, void *stream);

/* Bytes of a cache, 0 if the shape is invalid. */
uint64_t comet_cache_bytes(comet_cache_shape shape);

/* Put the batch's keys and values into the cache: keys turned on the way (plan NULL: as they are) and rounded to dtype,
 * complete blocks quantised.  dev_positions: int32[n_tokens], or NULL for the tokens' places in their sequences.  q, q_out, q_heads: the
 * queries of the same tokens, turned in the same launch (q_heads 0: none; q_out may be q). */
int comet_cache_append(void *dev_cache, comet_cache_shape shape, const comet_cache_batch *batch, uint32_t n_tokens, comet_rows k, comet_rows v,
                       comet_rows q, comet_rows q_out, uint32_t q_heads, int dtype, const comet_rope_plan *plan,
                       const int32_t *dev_positions, void *stream, int32_t *dev_status);

/* Read the batch's tokens back as the cache holds them, in dtype. */
int comet_cache_fetch(const void *dev_cache, comet_cache_shape shape, const comet_cache_batch *batch, uint32_t n_tokens, comet_rows k, comet_rows v,
                      int dtype, void *stream, int32_t *dev_status);

/* Attention of the batch's queries over the cache: out = softmax(scale * q k^T) v, query heads h * q_heads/heads .. sharing key/value head h.
 * causal != 0: a query sees the tokens up to its own place (n queries are the last n of lens[b] tokens; those in front of
 * the first see nothing); 0: all lens[b].  A row that sees nothing is 0 and its lse -Inf.  dev_lse: float32[n_tokens][q_heads],
 * log of the sum of exp of the row's scores, or NULL.  scale: finite, >= 0.  dev_work: comet_cache_attend_work bytes, 16-byte aligned, whose contents
 * need no initialisation; calls that can overlap in time need one each. */
uint64_t comet_cache_attend_work(comet_cache_shape shape, uint32_t n_seqs, uint32_t n_tokens, uint32_t q_heads);
int comet_cache_attend(const void *dev_cache, comet_cache_shape shape, const comet_cache_batch *batch, uint32_t n_tokens, comet_rows q, uint32_t q_heads,
                       int dtype, float scale, int causal, comet_rows out, float *dev_lse, void *dev_work, uint64_t work_bytes,
                       void *stream, int32_t *dev_status);

/* ---- stage-level entry points: each runs one step of the pipeline alone so
 * ---- that it can be compared with the reference implementation ------------ */

/* Sec. 4.1 steps 1-3 fused: prequantise, Lorenzo-predict, emit codes, count the
 * histogram and compact the outlier records.
 * dev_codes: u16[elements]; dev_hist: u32[nbins]; dev_records: u32[2*rec_capacity]
 * (key, payload) pairs in ascending key order, key = 2*index + type (type 0: the
 * payload is the int32 residual of an escaped code, type 1: the fp32 bit pattern
 * of an element stored verbatim); dev_counts: u64[3] = records, value records,
 * non-zero inputs. */
int comet_stage_quantize(comet_ctx *ctx, const float *dev_in, comet_shape shape, float eb, uint32_t nbins,
                         void *stream, uint16_t *dev_codes, uint32_t *dev_hist,
                         uint32_t *dev_records, uint64_t rec_capacity, uint64_t *dev_counts);

/* Huffman code lengths (two-queue construction, leaf before internal node on
 * equal weight, leaves ordered by (frequency, symbol)) and canonical codes.
 * dev_hist: u32[nbins]; dev_len: u8[nbins]; dev_code: u64[nbins] (may be NULL).
 * The context keeps the table for a following comet_stage_encode. */
int comet_stage_codebook(comet_ctx *ctx, const uint32_t *dev_hist, uint32_t nbins, void *stream,
                         uint8_t *dev_len, uint64_t *dev_code);

/* Chunked Huffman encode with the table of the last comet_stage_codebook on
 * this context.  dev_chunk_off: u32[ceil(n/chunk_syms)] word offset of every
 * chunk; dev_payload: u32[payload_capacity_words]; dev_payload_words: u64[1]. */
int comet_stage_encode(comet_ctx *ctx, const uint16_t *dev_codes, uint64_t n, uint32_t nbins, uint32_t chunk_syms,
                       void *stream, uint32_t *dev_chunk_off, uint32_t *dev_payload,
                       uint64_t payload_capacity_words, uint64_t *dev_payload_words);

/* Chunk-parallel Huffman decode from a length table. dev_codes_out: u16[n]. */
int comet_stage_decode(comet_ctx *ctx, const uint8_t *dev_len, uint32_t nbins,
                       const uint32_t *dev_chunk_off, const uint32_t *dev_payload, uint64_t payload_words,
                       uint64_t n, uint32_t chunk_syms, void *stream, uint16_t *dev_codes_out);

/* Lorenzo reconstruction (plane-wise 2-D prefix sums), dequantisation, verbatim
 * values and the re-zero filter of Sec. 3.4, from a code array and records. */
int comet_stage_reconstruct(comet_ctx *ctx, const uint16_t *dev_codes, const uint32_t *dev_records, uint64_t n_records,
                            comet_shape shape, uint32_t nbins, float eb, void *stream, float *dev_out);

/* ---- per-kernel timing, for benchmarks ---------------------------------------
 * When enabled, every step below of a call on the context is bracketed by two HIP events
 * recorded on the call's stream.  comet_profile_read waits for those events and
 * returns, for `kernel_id`, the number of brackets since the last
 * comet_profile_reset ("launches") and their summed duration in milliseconds.  Kernel ids:
 * 0 quantize (sweep; alphabets beyond 8192 bins and planes of at most 512 columns: a second
 * one for the histogram of the codes the sweep does not count), 1 codebook (a large alphabet's
 * sort, merge and code kernels included), 2 encode (pack pass), 3 decode tables,
 * 4 reconstruct (scans + store; planes cut into bands, as all wider than 512 columns are: the kernels
 * of the bands together), 5 Huffman decode, 6 gather of the outlier
 * records, 7 encode (count pass), 8 decompression in one kernel (Huffman decode, reconstruction and
 * store; containers with chunks of 64 symbols and planes of at most 512 columns, unless they are cut into bands).
 * What clears a call's control block, and the general kernel that stands behind 8 for other chunk
 * sizes, are not timed.
 * At most 16384 launches are kept between resets; further ones are not timed. */
#define COMET_KERNEL_QUANTIZE 0
#define COMET_KERNEL_CODEBOOK 1
#define COMET_KERNEL_ENCODE 2
#define COMET_KERNEL_TABLES 3
#define COMET_KERNEL_RECONSTRUCT 4
#define COMET_KERNEL_DECODE 5
#define COMET_KERNEL_GATHER 6
#define COMET_KERNEL_ENCODE_COUNT 7
#define COMET_KERNEL_FUSED 8
#define COMET_KERNEL_COUNT 9
int comet_profile_enable(comet_ctx *ctx, int enable);
int comet_profile_reset(comet_ctx *ctx);
int comet_profile_read(comet_ctx *ctx, uint32_t kernel_id, uint32_t *launches /* host */, double *total_ms /* host */);

/* Text for a COMET_ERR_* code; for COMET_ERR_HIP the last HIP error string seen
 * by this thread.  Never NULL. */
const char *comet_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* COMET_H */
