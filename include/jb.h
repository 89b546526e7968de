/*
 * jb.h -- C ABI of the GB300 (sm_103a) seeded-perturbation library "libjb".
 *
 * The library implements the data-parallel hot path of the decentralized
 * shared-randomness SPSA of "Just One Byte (per gradient)" (arXiv 2306.10015):
 * regenerate a seeded Gaussian perturbation z over every model parameter, in
 * registers, and apply it in place.
 *
 *   jb_perturb        PerturbParameters(theta, eps, s): theta_i += eps z_i
 *                     (Algorithm 1, subroutine); called with +eps, -2 eps,
 *                     +eps around the two loss evaluations of one SPSA sample
 *                     (Algorithm 1, inference loop).
 *   jb_apply_updates  the step update: every machine's (seed, one-byte
 *                     projected gradient) pair applied with weight
 *                     minus the gradient times the learning rate over the
 *                     number of collected gradients, in machine-timestamp
 *                     order (Section 2, on applying the collected scalar projected
 *                     gradients; Algorithm 1), fused into one read and one
 *                     write of theta.
 *   jb_quantize_grad  the one-byte projected gradient: the logarithm of its
 *   jb_dequantize_grad magnitude with its sign, limited to +-127 (Section 3,
 *                     Training Speed).
 *
 * ---------------------------------------------------------------------------
 * Random stream. The paper names no generator (Appendix B notes that PyTorch's
 * CUDA generator is not reproducible across GPU types). This library fixes:
 *   - Philox4x32-10 (Salmon et al., SC 2011) with key = (lo, hi) words of
 *     seed.machine_id and counter = (lo(b), hi(b), seed.step, seed.sample_id)
 *     for block b = e >> 2 of global element index e; element e uses word
 *     e & 3 of its block;
 *   - Box-Muller on the word pairs (0,1) and (2,3) of a block:
 *     u_a = ((x_a >> 9) + 1/2) 2^-23, u_b = ((x_b >> 8) + 1/2) 2^-24,
 *     r = sqrt(-2 ln u_a); even element r cos(2 pi u_b), odd r sin(2 pi u_b).
 *   z depends only on (seed, e): never on the tensor split, the launch
 *   geometry or the GPU run, so every replica regenerates identical noise.
 *   Scope of that bit-identity: the Philox words are exact integers and the
 *   same on any machine; the transform is fp32 with every rounding explicit,
 *   except its reciprocal and square root, which are the GPU's
 *   rcp.approx / sqrt.approx instructions. z is therefore bitwise identical
 *   on every sm_103a (GB300) GPU, the only target of this library; on other
 *   hardware its last bits may differ, while staying within 1e-6 of the exact
 *   definition above.
 *
 * Global element index. Each tensor ("segment") carries flat_offset, the
 * global index of its element 0: element i of the segment is e = flat_offset
 * + i. Every replica must use the same table (part of the shared model
 * layout). Recommended: flat_offset of tensor t = align_up(flat_offset of
 * t-1 + numel of t-1, 8) in named_parameters() order. The vectorised path
 * needs (ptr - flat_offset * sizeof(T)) to be a multiple of 16 bytes; other
 * segments are handled with smaller accesses, at lower speed, and cost the
 * others of the table up to 2 %.
 *
 * Arithmetic. z = s r in fp32, with r the radius and s the signed cosine or
 * sine of the element; |z| <= sqrt(48 ln 2) = 5.77. A scaled draw a z is formed
 * as fma(s, a r, .) with a r rounded once to fp32. Perturb: theta + eps z as
 * one fp32 fused multiply-add, fma(s, eps r, theta), then one rounding to the
 * storage type (nearest, ties to even). Update: acc = 0; for each pair k in
 * canonical order acc = fma(s_k, c_k r_k, acc) in fp32; theta <- round(theta +
 * acc) once. No flush-to-zero. Results are bitwise repeatable.
 *
 * Memory and streams. The caller owns all device memory (e.g. torch
 * tensors). The library copies the host arrays it is given (segments, seeds,
 * codes) during the call, keeps no pointer to them, allocates no device
 * memory and holds no state between calls other than a per-device cache of
 * the SM count and of how many CTAs of a kernel run at once. Work is enqueued on `stream` (a cudaStream_t; NULL is the
 * legacy default stream) and the call returns without waiting for it. Calls on
 * different streams that touch the same parameters race.
 *
 * Errors. Every entry point returns a jb_status. Argument errors are detected
 * before anything is enqueued, and then nothing is enqueued. JB_ERR_CUDA
 * reports a failed CUDA runtime call or launch of this call (cudaGetLastError);
 * faults during execution surface at the caller's next synchronisation. The
 * library links the CUDA runtime statically, so its error state is private: an
 * error pending in the caller's runtime (torch's, say) is neither reported nor
 * cleared by libjb, and libjb clears each error it reports so that none lingers
 * into a later call. A sticky error (a fault that poisons the context) is
 * reported by every runtime. No exception, abort or exit crosses this
 * interface.
 */
#ifndef JB_H
#define JB_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

struct CUstream_st; /* cudaStream_t is struct CUstream_st* */

typedef enum {
    JB_OK = 0,
    JB_ERR_INVALID_ARG = -1,      /* NULL pointer, negative count, bad scalar, overlap */
    JB_ERR_UNSUPPORTED_DTYPE = -2,
    JB_ERR_MISALIGNED = -3,       /* segment pointer not aligned to its element size; calls say what else they need */
    JB_ERR_DUPLICATE_SEED = -4,   /* two pairs with the same (machine_id, step, sample_id) */
    JB_ERR_CUDA = -5,             /* a CUDA runtime call or launch failed */
    JB_ERR_RANGE = -6,            /* a coefficient -lr deq(q) / denom is not finite in fp32 */
    JB_ERR_TOO_MANY_SEEDS = -7,   /* K above jb_max_seeds_per_call() */
    JB_ERR_NO_MEMORY = -8         /* host memory for the call's working copy could not be had */
} jb_status;

typedef enum { JB_F32 = 0, JB_BF16 = 1 } jb_dtype;

/* One parameter tensor: `numel` contiguous elements of the call's dtype at
 * device address `ptr` (caller-owned), element i having global index
 * flat_offset + i. Segments must not overlap in memory nor in global index. */
typedef struct {
    void* ptr;
    uint64_t numel;
    uint64_t flat_offset;
} jb_segment;

/* Seed s of Algorithm 1: the machine's start time (as an identifier), the
 * iteration, and the sample's index within the iteration. 16 bytes. */
typedef struct {
    uint64_t machine_id;
    uint32_t step;
    uint32_t sample_id;
} jb_seed;

/*
 * jb_perturb -- PerturbParameters(theta, eps, s) (Algorithm 1, subroutine):
 * for every element e of every segment, theta_e <- round_T(theta_e + eps
 * z_e(seed)), the sum one fp32 fused multiply-add (see Arithmetic). In place,
 * asynchronous on `stream`.
 *   segs, n_segs  segment table (host array, copied); n_segs = 0 is a no-op.
 *   dtype         JB_F32 or JB_BF16 for all segments.
 *   eps           finite perturbation scale (use +eps, -2 eps, +eps for one
 *                 SPSA sample; eps = 0 still rewrites theta unchanged).
 */
int jb_perturb(const jb_segment* segs, int n_segs, int dtype, jb_seed seed, float eps,
               struct CUstream_st* stream);

/*
 * jb_apply_updates -- apply K machines' projected gradients in one pass
 * (Section 2; Algorithm 1, gradient application):
 *   theta_e <- round_T(theta_e + sum_k c_k z_e(seeds[k])),
 *   c_k = (float)(-(double)lr * deq(q[k]) / (double)denom) with deq as in
 *   jb_dequantize_grad, pairs taken in ascending (machine_id, step,
 *   sample_id) order whatever order they are passed in.
 * The paper divides by the number of collected gradients (denom = K);
 * Section 4 scales the learning rate with sqrt(#perturbations): denom is
 * therefore the caller's.
 *   seeds, q, K   host arrays of K pairs (copied). K = 0 is a no-op.
 *                 K <= jb_max_seeds_per_call(); duplicates are an error.
 *   lr, denom     finite, denom != 0. qscale: S > 0 of the byte code.
 * Returns JB_ERR_RANGE (nothing enqueued) if some c_k is not finite in fp32.
 */
int jb_apply_updates(const jb_segment* segs, int n_segs, int dtype, const jb_seed* seeds,
                     const int8_t* q, int K, float lr, float denom, float qscale,
                     struct CUstream_st* stream);

/*
 * jb_apply_updates_from -- the step update applied to the weight backup, fused
 * with the restore (Algorithm 1: theta is reset from the backup copy, then every
 * machine's gradients; Section 2: the backup avoids the drift of theta + z - z):
 *   dst_e <- round_T(src_e + sum_k c_k z_e(seeds[k])), one read of src and one
 *   write of dst per element (and one more write of src when write_src != 0, so
 *   the next iteration's backup is refreshed in the same pass).
 * Same pairs, coefficients, canonical order and rounding as jb_apply_updates;
 * K = 0 copies src to dst.
 *   src, dst   tables of n_segs segments: dst[i] has the numel and flat_offset of
 *              src[i]; dst[i] is either src[i] itself or overlaps no source and
 *              no other destination.
 */
int jb_apply_updates_from(const jb_segment* src, const jb_segment* dst, int n_segs, int dtype,
                          const jb_seed* seeds, const int8_t* q, int K, float lr, float denom,
                          float qscale, int write_src, struct CUstream_st* stream);

/*
 * jb_replay_updates -- a late joiner's catch-up (Appendix B): after downloading
 * the weights, apply the projected gradients of every iteration it missed. Step
 * t holds step_sizes[t] pairs (consecutive in seeds/q) and its own lr[t] and
 * denom[t]; steps are applied in order, each rounded to the storage type as
 * jb_apply_updates would round it, so the result is bitwise that of n_steps
 * successive jb_apply_updates calls -- but theta is read and written once per
 * launch instead of once per step. A step holds at most
 * jb_max_seeds_per_call() pairs; steps are packed into launches of at most
 * that many pairs.
 */
int jb_replay_updates(const jb_segment* segs, int n_segs, int dtype, const jb_seed* seeds,
                      const int8_t* q, const int* step_sizes, int n_steps, const float* lr,
                      const float* denom, float qscale, struct CUstream_st* stream);

/* A tensor of 4-bit weights: numel codes, two per byte (element 2i in the low
 * nibble of byte i; `codes` 8-byte aligned, (numel + 1) / 2 bytes), and one fp32
 * scale per block of 64 elements (`scale`, ceil(numel / 64) floats). Weight i
 * is level[code_i] * scale[i / 64] with the 16 levels of jb_q4_levels().
 * flat_offset (a multiple of 4) is the global index of element 0, as for
 * jb_segment. Device memory, caller-owned. */
typedef struct {
    uint8_t* codes;
    float* scale;
    uint64_t numel;
    uint64_t flat_offset;
} jb_q4_segment;

/*
 * jb_perturb_q4 -- PerturbParameters on 4-bit weights (Section 3, Training
 * Speed: weights are dequantized before the noise is added and quantized
 * again). For every block of 64 elements: w_i = level[code_i] * scale,
 * w'_i = w_i + eps z_i(seed) in fp32, one fused multiply-add as in jb_perturb, then
 * scale' = max_i |w'_i| and code'_i = the nearest level to w'_i / scale' (ties
 * to the lower level; scale' = 0 gives the zero level). Codes and scales are
 * rewritten in place, asynchronously on `stream`; an odd numel leaves the
 * unused high nibble of the last byte as it was. The paper fixes no 4-bit
 * format; this is a NormalFloat-style code after QLoRA (see jb_q4_levels).
 * Errors, found before anything is enqueued: JB_ERR_INVALID_ARG for n_segs < 0,
 * a null array or pointer, a non-finite eps, an index range past 2^62, or
 * tensors whose bytes or index ranges overlap; JB_ERR_MISALIGNED for codes not
 * 8-byte aligned, scale not 4-byte aligned or flat_offset not a multiple of 4.
 * Tensors with numel = 0 are skipped.
 */
int jb_perturb_q4(const jb_q4_segment* segs, int n_segs, jb_seed seed, float eps,
                  struct CUstream_st* stream);

/* The 16 levels of the 4-bit code, ascending, in [-1, 1]: quantiles of N(0,1)
 * at probabilities d + (1/2 - d) j / 7 (j = 0..7, the median 0 last) and
 * 1/2 + (1/2 - d) j / 8 (j = 1..8), d = 1/32, divided by the largest, rounded
 * to fp32. Host only; out receives 16 floats. */
int jb_q4_levels(float* out);

/*
 * jb_checksum -- hash of the model for ChecksumMatch (Algorithm 1: each machine
 * checks with a random peer that their hashed theta match). The paper fixes no
 * hash. This one: cut the global element index space into 16-byte windows of
 * storage (8 bf16 or 4 fp32 elements; window v = elements [vE, vE + E)). For
 * every segment and every window v it overlaps, take the window's four 32-bit
 * storage words (little-endian; elements outside the segment read as 0), apply
 * the first four Philox4x32 rounds under key (lo32(v) ^ 0x6A09E667,
 * hi32(v) ^ 0xF3BCC908), and add (x1:x0) + (x3:x2). The checksum is the sum
 * mod 2^64. It depends on the values, the dtype and the flat offsets, not on
 * the launch; replicas with the same table and bits get the same value.
 *   d_out   device pointer to one uint64_t (8-byte aligned, caller-owned); it is
 *           zeroed and written on `stream`.
 */
int jb_checksum(const jb_segment* segs, int n_segs, int dtype, uint64_t* d_out,
                struct CUstream_st* stream);

/*
 * jb_quantize_grad -- one-byte projected gradient (Section 3, Training
 * Speed: the sign and the logarithm of the magnitude, limited to +-127). Host
 * only, pure:
 *   *out = sign(g) * min(127, round_half_away(qscale * ln(1 + |g|))),
 *   NaN -> 0, +-inf -> +-127. qscale must be finite and > 0.
 */
int jb_quantize_grad(double g, float qscale, int8_t* out);

/*
 * jb_dequantize_grad -- inverse of the byte code, host only, pure:
 *   *out = (float)(sign(q) * expm1(min(|q|, 127) / qscale)) (code -128 reads as
 *   -127). Computed in double, rounded once; may be +-inf for small qscale.
 */
int jb_dequantize_grad(int8_t q, float qscale, float* out);

/* Largest K accepted by jb_apply_updates in one call (the pairs travel in the
 * kernel's parameter space). */
int jb_max_seeds_per_call(void);

/* Static description of a status code. Never NULL. */
const char* jb_status_string(int status);

/* ---------------------------------------------------------------------------
 * Writing answers with the perturbed model. A sample's score need not be a loss
 * with a gradient: accuracy or a reward of what the model writes serves as well.
 * The calls below are those that writing needs between two perturbations: a
 * cache of keys and values in pages, attention of new tokens over it, and the
 * draw of the next token from a given random word (the same words at +eps and
 * -eps, so that the two scores differ by the weights alone).
 *
 * All arrays named d_* and all pointers in jb_pages and jb_kv are memory of the
 * current device, caller-owned; the structures themselves are host memory, copied during the
 * call. Everything is enqueued on `stream`, and nothing is read back: lengths,
 * page tables and page counts live on the device, so a whole generation step can
 * be captured in a CUDA graph. Argument errors that the host can see are statuses,
 * as above. What only the device can see (a row index out of range, too few free
 * pages) never causes an access out of bounds; each call says what happens.
 * ------------------------------------------------------------------------- */

/* The pages of a cache: row r holds lens[r] tokens, token t in page
 * table[r * row_pages + t / page_tokens] at place t % page_tokens. Entries past a
 * row's last page are -1. refs[p] counts the entries that name page p (rows forked
 * from one another share full pages); a page with refs 0 is free. An empty cache:
 * table all -1, lens and refs all 0. The arrays are kept consistent by jb_cache_*.
 *   page_tokens  a multiple of 16, at most 1024
 *   n_rows       at most 65536;  row_pages * page_tokens below 2^31
 */
typedef struct {
    int32_t* table; /* [n_rows][row_pages] */
    int32_t* lens;  /* [n_rows] */
    int32_t* refs;  /* [n_pages] */
    int32_t n_rows;
    int32_t row_pages;
    int32_t n_pages;
    int32_t page_tokens;
} jb_pages;

/* One layer's keys and values: page p at k (v) + p * page_stride elements, in it
 * [heads][page_tokens][head_dim] (by_token = 0) or [page_tokens][heads][head_dim]
 * (by_token = 1), without gaps.
 *   dtype     JB_F32 or JB_BF16, of keys, values, queries and outputs alike
 *   head_dim  at most 256, rows of a multiple of 16 bytes; k, v 16-byte aligned,
 *             page_stride a multiple of 16 bytes and at least a page
 */
typedef struct {
    void* k;
    void* v;
    uint64_t page_stride;
    int32_t heads;
    int32_t head_dim;
    int32_t dtype;
    int32_t by_token;
} jb_kv;

/* Host threads: a call from here on may be several launches. No other call with the same workspace or the same page table may
 * be made until it returns, also not on its stream, where the other's launches would come between its own. Calls that follow
 * one another on one stream can share a workspace. */

/*
 * jb_cache_reserve -- room for new tokens: lens[d_rows[i]] += d_tokens[i], with free
 * pages taken for it, the lowest ids first, in the order of the list (i, then the
 * row's pages). The listed rows must differ. *d_status (one int32) receives
 *    0   done
 *   >0   that many free pages too few: nothing is changed
 *   -1   a row index out of range or listed twice, a negative count, or a row that
 *        would outgrow its table: nothing is changed
 *   n    at most 16384 rows a call; 0 is a no-op that writes status 0.
 */
int jb_cache_reserve(const jb_pages* pages, const int32_t* d_rows, const int32_t* d_tokens, int n,
                     int32_t* d_status, struct CUstream_st* stream);

/*
 * jb_cache_free -- the listed rows become empty; pages that no row names any more are
 * free. Listing a row twice frees it once; an index out of range is skipped.
 */
int jb_cache_free(const jb_pages* pages, const int32_t* d_rows, int n, struct CUstream_st* stream);

/*
 * jb_cache_fork -- row d_children[i] becomes a copy of row d_parents[i], for all i at
 * once (a row may be both: its state before the call is what is copied). Full pages
 * are shared; the last page, if it is not full, is copied in every layer to a page
 * that is free before the call (the lowest ids, in the order of the list): its valid
 * tokens, the rest of that page is left as it is. The child's former pages are
 * released. A pair with equal rows changes nothing. *d_status as for
 * jb_cache_reserve: -1 for an index out of range or a child listed twice.
 *   workspace  jb_cache_workspace(pages, n) bytes, 16-byte aligned, contents free
 */
int jb_cache_fork(const jb_pages* pages, const jb_kv* layers, int n_layers, const int32_t* d_parents,
                  const int32_t* d_children, int n, int32_t* d_status, void* workspace,
                  uint64_t workspace_bytes, struct CUstream_st* stream);

/*
 * jb_cache_compact -- moves pages so that the n_live pages in use are ids 0 ..
 * n_live - 1: the i-th page in use at or above n_live goes to the i-th free page below
 * it, in every layer. Tables and counts follow. *d_status receives n_live.
 *   workspace  jb_cache_workspace(pages, 0) bytes
 */
int jb_cache_compact(const jb_pages* pages, const jb_kv* layers, int n_layers, int32_t* d_status,
                     void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream);

/* Device bytes that jb_cache_fork of n pairs (n > 0) or jb_cache_compact (n = 0) works in. */
uint64_t jb_cache_workspace(const jb_pages* pages, int n);

/*
 * jb_cache_write -- new keys and values to their places: token i, d_k[i][head][:] and
 * d_v[i][head][:] of the layer's dtype, to position d_pos[i] of row d_rows[i] (room for
 * it reserved before). A token whose row, position or page is out of range is skipped;
 * two tokens with the same place race.
 *   strides  in elements, multiples of 16 bytes: from token to token and head to head
 */
int jb_cache_write(const jb_pages* pages, const jb_kv* layer, const void* d_k, uint64_t k_token_stride,
                   uint64_t k_head_stride, const void* d_v, uint64_t v_token_stride, uint64_t v_head_stride,
                   const int32_t* d_rows, const int32_t* d_pos, int n, struct CUstream_st* stream);

/* What jb_attend does to the scores, besides their scale. */
typedef struct {
    float scale;         /* x = scale q.k */
    float softcap;       /* > 0: x = softcap tanh(x / softcap), at most 1e30 and scale / softcap finite; 0: off */
    int32_t window;      /* > 0: only the last `window` positions are seen; 0: all */
    const float* slopes; /* device, one per query head: x += slope (t - pos); NULL: off */
} jb_scores;

/*
 * jb_attend -- attention of n queries over the pages: query i, head a reads key head
 * a / (q_heads / heads) of positions t <= d_pos[i] of row d_rows[i] (and
 * t > d_pos[i] - window):
 *   out = sum_t exp(x_t) v_t / sum_t exp(x_t)
 * A new token's query comes with the position that its key was written to; the tokens
 * of a prompt are queries of one row with consecutive positions, each of which reads the
 * row for itself: long prompts are slow (jb_attend_tree takes them 256 tokens at a time). A query that sees
 * nothing (position -1, or a row or position out of range) gets zeros; a position whose
 * page is missing is not seen, nor is one whose score is -inf. What a page holds past the
 * last position seen has no effect, NaN included. Results are bitwise repeatable.
 * Scores, maxima and sums are fp32 (scores beyond 2e38 in size count as infinite); fp32
 * caches are computed in fp32. With bf16 the
 * products run on the tensor cores with fp32 sums, and a weight exp(x_t) enters them
 * as the sum of two bf16 numbers (16 bits of it), so that an infinite value that is seen
 * gives an infinity or NaN.
 *   q_heads    a multiple of the layer's heads
 *   strides    in elements, multiples of 16 bytes; pointers 16-byte aligned. No two
 *              outputs (query, head) may share bytes: JB_ERR_INVALID_ARG
 *   workspace  jb_attend_workspace(...) bytes, 16-byte aligned, the first 65536 of them
 *              zero before its first use; every call leaves it ready for the next one on
 *              the stream. Calls that may run at the same time need one each.
 */
int jb_attend(const jb_pages* pages, const jb_kv* layer, const jb_scores* scores, const void* d_q,
              uint64_t q_row_stride, uint64_t q_head_stride, int q_heads, const int32_t* d_rows,
              const int32_t* d_pos, int n, void* d_out, uint64_t out_row_stride, uint64_t out_head_stride,
              void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream);

/* Device bytes that jb_attend works in, for any n. */
uint64_t jb_attend_workspace(const jb_kv* layer, int q_heads);

/* Per-row settings of jb_sample: device arrays of n entries, or NULL for the default.
 * temperature (1): below 2^-64 or NaN, the row's largest logit is taken (the first one).
 * top_k (0): <= 0 or at least the vocabulary keeps all. top_p (1): >= 1 or NaN keeps all.
 * min_p (0): <= 0 or NaN keeps all, above 1 counts as 1. */
typedef struct {
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
} jb_sampling;

/*
 * jb_sample -- the next token of each row from its logits and one random word:
 *   L = max l;  y_j = (l_j - L) (1 / temperature);  w_j = rint(2^30 exp(y_j))
 * Weights are integers, so sums of them are exact and the draw does not depend on the
 * order in which they are added. Tokens are ordered by logit, equal ones by index; kept
 * are the first top_k; of those the shortest run from the front whose weights reach
 * ceil(top_p W), W their sum; of those the ones with w_j >= ceil(min_p 2^30). Then, with
 * W the sum of the kept weights, the token is the first index whose running sum of kept
 * weights exceeds floor(word W / 2^32), and its log-probability y - ln(W / 2^30).
 * NaN logits are never drawn; logits of +inf share the draw among themselves. A row with
 * nothing to draw (all -inf or NaN) gives token -1 and -inf.
 *   d_logits   [n][vocab] of dtype, rows at row_stride elements; vocab at most 262144
 *   d_words    n random 32-bit words
 *   d_tokens, d_logprobs  n results each; d_logprobs may be NULL
 */
int jb_sample(const void* d_logits, uint64_t row_stride, int dtype, int n, int vocab,
              const jb_sampling* sampling, const uint32_t* d_words, int32_t* d_tokens, float* d_logprobs,
              struct CUstream_st* stream);

/* ---------------------------------------------------------------------------
 * Drafted tokens. Several tokens of an answer can be checked in one pass over the weights
 * and the cache: a tree of guesses is written behind its row's tokens (jb_cache_reserve,
 * jb_cache_append), attended to at once (jb_attend_tree), and of it the path that the model
 * writes itself is kept (jb_cache_keep). With random words given by position the answers
 * are those of one token at a time. A chain is a tree: the tokens of a prompt can be written
 * 256 at a time in this way.
 * ------------------------------------------------------------------------- */

/* Trees of drafted tokens: the nodes of tree i are starts[i] .. starts[i + 1] - 1 of a list of
 * n_nodes, at most 256, and they are the last tokens of row rows[i], in that order.
 * parents[] counts within the tree: the node that a node follows, before it in the list, or
 * -1 for one that follows the row's tokens before the tree. Device arrays; `starts` ascends,
 * and no row is listed twice. At most 16384 trees. */
typedef struct {
    const int32_t* rows;    /* [n] */
    const int32_t* starts;  /* [n + 1] */
    const int32_t* parents; /* [n_nodes] */
    int32_t n;
    int32_t n_nodes;
} jb_trees;

/* How queries and keys are turned by their positions. Pair j of the first `dims` elements of a
 * head (even, at most head_dim; the others stay) is turned by t steps[j] mod 2^64 parts of
 * 2^-64 of a full turn at position t: exact at any position. Pairs are (j, j + dims / 2), or
 * neighbours (2 j, 2 j + 1) with interleaved != 0. For the usual powers steps[j] is
 * 2^64 base^(-2 j / dims) / (2 pi). */
typedef struct {
    const uint64_t* steps; /* device, [dims / 2], 8-byte aligned */
    int32_t dims;
    int32_t interleaved;
} jb_rotation;

/*
 * jb_cache_append -- jb_cache_write with the rotation on the way: the key of token i is turned
 * by its position d_turns[i] and written, with its value, to position d_pos[i] of row
 * d_rows[i]; its queries are turned alike and written to d_q_out. d_turns differs from d_pos
 * for a tree's nodes (their places follow one another, their positions go by depth) and for a
 * text whose beginning the cache no longer holds; NULL: as d_pos. The rotation is computed in
 * fp32 from an angle exact to 2^-24 of itself, and rounded once.
 * A token whose row, position or page is out of range is not written (its queries are turned);
 * two tokens with the same place race.
 *   q_heads    any number of query heads, 0: none (d_q and d_q_out are not looked at)
 *   strides    in elements, multiples of 16 bytes; pointers 16-byte aligned
 *   d_q_out    d_q itself with its strides, or apart from all that is read. What shares bytes
 *              otherwise, or cannot be told not to, is refused: JB_ERR_INVALID_ARG
 */
int jb_cache_append(const jb_pages* pages, const jb_kv* layer, const jb_rotation* rotation, const void* d_q,
                    uint64_t q_token_stride, uint64_t q_head_stride, int q_heads, void* d_q_out,
                    uint64_t out_token_stride, uint64_t out_head_stride, const void* d_k, uint64_t k_token_stride,
                    uint64_t k_head_stride, const void* d_v, uint64_t v_token_stride, uint64_t v_head_stride,
                    const int32_t* d_rows, const int32_t* d_pos, const int32_t* d_turns, int n, struct CUstream_st* stream);

/*
 * jb_attend_tree -- attention of the nodes of trees, as jb_attend's: node j of tree i (query
 * starts[i] + j) sees its row's tokens before the tree, its ancestors and itself. For windows
 * and slopes a node's position is that of the token that it would be in a chain: tokens
 * before the tree plus its depth.
 * A node whose chain of parents is not valid (an index not below its own, or below -1) gets
 * zeros, and so do the nodes of a tree whose row is out of range, holds fewer tokens than the
 * tree, or that has more than 256 nodes. Queries of no tree are left as they are.
 * Accuracy, missing pages, infinite scores and what unseen places hold: as jb_attend; bf16
 * weights meet values with 16 bits.
 *   q_heads    a multiple of the layer's heads
 *   strides    in elements, multiples of 16 bytes; pointers 16-byte aligned. Outputs share bytes
 *              neither with one another nor with queries: JB_ERR_INVALID_ARG
 *   workspace  jb_attend_tree_workspace(...) bytes, 16-byte aligned, contents free. Calls that
 *              may run at the same time need one each.
 */
int jb_attend_tree(const jb_pages* pages, const jb_kv* layer, const jb_scores* scores, const jb_trees* trees, const void* d_q,
                   uint64_t q_row_stride, uint64_t q_head_stride, int q_heads, void* d_out, uint64_t out_row_stride,
                   uint64_t out_head_stride, void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream);

/* Device bytes that jb_attend_tree works in, whatever the trees. */
uint64_t jb_attend_tree_workspace(const jb_kv* layer);

/*
 * jb_cache_keep -- of each tree the path from its root to node d_leaves[i] stays (-1: nothing
 * does): the path's keys and values move, in every layer, to the places behind the tokens
 * before the tree, the row ends with them, and pages behind are given back. *d_status receives
 *    0   done
 *   -1   a tree that is not valid (see jb_attend_tree) or whose row is listed twice, a leaf out
 *        of range or without a valid path, or a token that would move from a missing page or to
 *        one that is missing or that other rows name too: nothing is changed
 *   workspace  jb_cache_keep_workspace(trees) bytes, 16-byte aligned, contents free
 */
int jb_cache_keep(const jb_pages* pages, const jb_kv* layers, int n_layers, const jb_trees* trees, const int32_t* d_leaves,
                  int32_t* d_status, void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream);

/* Device bytes that jb_cache_keep works in. */
uint64_t jb_cache_keep_workspace(const jb_trees* trees);

/*
 * jb_q4_matmul -- products of n rows with a matrix of 4-bit weights, as they are between two
 * calls of jb_perturb_q4: y_i[o] = sum_k x_i[k] level[code] scale + bias[o], the weight of
 * output o and input k being element o in_features + k of the tensor.
 *   weights       numel = out_features in_features, its codes 8-byte aligned (16-byte: large
 *                 products are faster); its flat_offset is not looked at
 *   out_features  at most 2^30
 *   in_features   a multiple of 64 (a block's scale belongs to one output), at most 65536
 *   dtype         JB_F32 or JB_BF16, of x, bias and y alike; sums are fp32. Levels enter bf16
 *                 products off by at most 1.6e-4 of themselves and fp32 products with 22 bits; x with all its bits or 22, but
 *                 nothing finer than 2^-40 of the largest element of its row
 *   d_x           [n][in_features], 16-byte aligned, rows x_row_stride elements apart (a multiple
 *                 of 16 bytes)
 *   n             at most 2^30
 *   d_bias        [out_features], or NULL
 *   d_y           [n][out_features], rows y_row_stride elements apart; shares no byte with what is
 *                 read: JB_ERR_INVALID_ARG
 *   workspace     jb_q4_matmul_workspace(...) bytes, 16-byte aligned, contents free; NULL where that
 *                 is 0. Calls that may run at the same time need one each.
 * Made for few rows: the weights are read once for each 64 of them at most.
 */
int jb_q4_matmul(const jb_q4_segment* weights, int out_features, int in_features, int dtype, const void* d_x, uint64_t x_row_stride,
                 int n, const void* d_bias, void* d_y, uint64_t y_row_stride, void* workspace, uint64_t workspace_bytes,
                 struct CUstream_st* stream);

/* Device bytes that jb_q4_matmul works in; 0 for small products. */
uint64_t jb_q4_matmul_workspace(int out_features, int in_features, int dtype, int n);

/* ---------------------------------------------------------------------------
 * Test hooks (not on the hot path). Device buffers are caller-owned.
 * ------------------------------------------------------------------------- */

/* d_out[4 i + w] = word w of Philox block first_block + i under `seed`.
 * d_out must be 16-byte aligned (JB_ERR_MISALIGNED); n_blocks <= 2^38. */
int jb_debug_philox(jb_seed seed, uint64_t first_block, uint64_t n_blocks, uint32_t* d_out,
                    struct CUstream_st* stream);

/* *d_out = XOR of all words of Philox blocks first_block .. first_block +
 * n_blocks - 1 under `seed`: the generator alone, computed as the kernels
 * compute it, on the persistent grid (the benchmark times it as the
 * generator-only rate). d_out: one uint32_t, 4-byte aligned, zeroed and written
 * on `stream`. n_blocks <= 2^46, first_block <= 2^60. */
int jb_debug_philox_fold(jb_seed seed, uint64_t first_block, uint64_t n_blocks, uint32_t* d_out,
                         struct CUstream_st* stream);

/* d_out[i] = z of global element first_elem + i under `seed` (fp32).
 * d_out must be 4-byte aligned (JB_ERR_MISALIGNED); n <= 2^38. */
int jb_debug_gaussian(jb_seed seed, uint64_t first_elem, uint64_t n, float* d_out,
                      struct CUstream_st* stream);

/* Box-Muller of raw word pairs: d_out[2 i], d_out[2 i + 1] = z of the even and
 * odd element for words (d_words[2 i], d_words[2 i + 1]). Both buffers must be
 * 4-byte aligned (JB_ERR_MISALIGNED); n_pairs <= 2^38. */
int jb_debug_box_muller(const uint32_t* d_words, uint64_t n_pairs, float* d_out,
                        struct CUstream_st* stream);

/* jb_checksum / jb_perturb / jb_apply_updates with an explicit number of CTAs
 * (0 = the default persistent grid); results must not depend on it. */
int jb_checksum_with_grid(const jb_segment* segs, int n_segs, int dtype, uint64_t* d_out,
                          int grid_ctas, struct CUstream_st* stream);
int jb_perturb_with_grid(const jb_segment* segs, int n_segs, int dtype, jb_seed seed, float eps,
                         int grid_ctas, struct CUstream_st* stream);
int jb_apply_updates_with_grid(const jb_segment* segs, int n_segs, int dtype,
                               const jb_seed* seeds, const int8_t* q, int K, float lr,
                               float denom, float qscale, int grid_ctas,
                               struct CUstream_st* stream);

#ifdef __cplusplus
}
#endif
#endif /* JB_H */
