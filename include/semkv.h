/*
 * semkv.h — C ABI of the SemKV packed mixed-precision KV cache (sm_103a).
 *
 * SemKV keeps every token of the KV cache (Eqs. 8-9) and gives each token one of
 * two adjacent fractional precisions: the top-r fraction by importance score gets
 * b_high, the rest b_low (Eqs. 4-5).  A "fractional" precision is an integer level
 * count L with log2(L) bits (Sec. 4.1: 2.585 = log2 6, 2.322 = log2 5).  Codes are
 * stored by mixed-radix packing (Sec. 4.1: 3 five-level codes in 7 bits, 5 six-level
 * codes in 13 bits) with per-row fp16 metadata (two parameters per 128-value row
 * for the affine base; one norm per row for the TurboQuant-MSE base, Sec. 4.9).
 * Generated tokens are staged at fp16 and quantized a block at a time, exactly
 * round(r*B) of each block at b_high (Sec. 3.7, Algorithm 2).
 *
 * Conventions shared by every entry point
 *  - The caller owns every buffer.  No entry point allocates, frees or synchronises;
 *    all device work is enqueued on the caller's stream `stream` (a cudaStream_t
 *    passed as void*; NULL = legacy default stream).
 *  - Pointers documented as "device" must be device (or managed) memory.
 *  - Host-checkable errors (NULL pointers, bad sizes, misalignment, unsupported
 *    level counts, capacity overflow) return an error status before anything is
 *    launched.  A failed launch returns SEMKV_ECUDA.  Kernels never trap: an
 *    anomaly seen on the device (e.g. a bulk-copy wait that timed out) is written
 *    to cache->dev_error (when given) and the host reads it when it chooses.
 *  - fp16 tensors are passed as uint16_t bit patterns (IEEE binary16).
 *  - head_dim is 128 in this version (the shape of Llama-3.1-8B / Mistral-7B KV).
 *
 * Record format (layout 1).  For level count L a 128-value row is four quarters
 * of 32 consecutive dims.  Inside a quarter the codes are grouped g(L) at a time;
 * a group's codes c_0..c_{g-1} (c_0 = lowest dim) form t = sum_k c_k L^(g-1-k) and
 * are stored as the w(L)-bit integer ceil(t * 2^w / L^g); the 32 mod g codes left at
 * the end of the quarter form one shorter group stored the same way in
 * ceil(log2 L^(32 mod g)) bits.  Quarters are concatenated least-significant-bit
 * first (stream bit i is bit i%8 of byte i/8); unused bits are zero.
 *      L : g  w   bits/quarter  row bytes RB(L)
 *      2 : 1  1        32            16
 *      3 : 5  8        52            26
 *      4 : 1  2        64            32
 *      5 : 3  7        75            38
 *      6 : 5 13        84            42
 *      7 : 1  3        96            48
 *      8 : 1  3        96            48
 *  affine record = [K row RB][V row RB][Ks f16][Kz f16][Vs f16][Vz f16]  (2RB+8 B)
 *  TQ record     = [K row RB][V row RB][Kn f16][Vn f16]                   (2RB+4 B)
 *  Pools are [batch][layers][kv_heads][cap][record]; slot s of the high pool of
 *  sequence b holds the s-th high-precision token of b in token order.
 */
#ifndef SEMKV_H_
#define SEMKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SEMKV_OK = 0,
  SEMKV_EINVAL = 1,         /* NULL pointer, bad size or inconsistent arguments   */
  SEMKV_EALIGN = 2,         /* a pointer or capacity violates an alignment rule    */
  SEMKV_ECAPACITY = 3,      /* a pool or the staging buffer would overflow         */
  SEMKV_EUNSUPPORTED = 4,   /* level count / base / head_dim not supported         */
  SEMKV_ECUDA = 5,          /* a CUDA launch or query failed                       */
  SEMKV_EWORKSPACE = 6      /* workspace NULL or smaller than the size query says  */
} semkv_status;

enum { SEMKV_BASE_AFFINE = 0, SEMKV_BASE_TQ = 1, SEMKV_BASE_AFFINE_HAD = 2,
       SEMKV_BASE_TQ_DENSE = 3 };
enum { SEMKV_HEAD_DIM = 128, SEMKV_MAX_LEVELS = 8 };
enum { SEMKV_F16 = 0, SEMKV_BF16 = 1, SEMKV_F32 = 2 };  /* types of tensors (F32: semkv_beam_select only) */

/* Quantizer description (host struct; the pointers inside are device pointers).
 * base AFFINE: per-row asymmetric min/max quantizer with fp16 scale and offset
 *   (Sec. 4.1 "two FP16 parameters (offset and scale) per head-token row").
 * base AFFINE_HAD: the same affine quantizer applied to the Hadamard-rotated row
 *   (Sec. 4.1: rows are rotated before quantization), in binary32:
 *     u = fp32(1/sqrt 128) * FWHT(x * sign)   (orthonormal (1/sqrt 128) H S; butterfly
 *                                              stages 1, 2, ..., 64, each (a+b, a-b))
 *     z = fp16 of min u rounded toward -infinity (limited to >= -65504), so z <= min u
 *     s = fp16((max u - z) / (L - 1)), rounded to nearest and limited to 65504
 *     c_j = clamp(rint((u_j - z) * fl(1/s)), 0, L - 1); all 0 unless s > 0.
 *   Records as AFFINE; decoding rotates each query once and the output back once.
 *   Needs signs.  Rows holding NaN or infinity are outside the supported inputs.
 * base TQ: TurboQuant-MSE (Sec. 4.9): sign flip + unnormalised Walsh-Hadamard
 *   transform of the row, divided by the row's fp16 norm, then a Gaussian Lloyd-Max
 *   scalar codebook with L levels (thresholds strictly-greater: ties go low).
 * base TQ_DENSE: TurboQuant-MSE with a dense random rotation (Sec. 4.9 "random
 *   rotation"): w = M x with M the stored fp16 matrix ~ sqrt(128) Q (Q orthogonal) in
 *   place of H S x; the rest as TQ (fp16 norm, u = w * fl(1/n), codebook).  w is formed
 *   on the tensor cores (exact fp16 products, fp32 accumulation), so a code can differ
 *   from the exactly rounded product's where u lies within rounding of a threshold.
 *   Records as TQ; rows dequantize to (n/128) M^T cb[c].  Needs rotation + codebooks.
 * levels_hi / levels_lo: L for b_high / b_low, each in 2..8; equal = uniform. */
typedef struct {
  int32_t base;
  int32_t levels_hi, levels_lo;
  int32_t head_dim;                 /* must be 128 */
  const int8_t* signs;              /* TQ, AFFINE_HAD: device [layers][kv_heads][128]
                                       of +-1, 4-byte aligned                       */
  const float* centroids_hi;        /* TQ, TQ_DENSE: device [levels_hi] ascending   */
  const float* thresholds_hi;       /* TQ: device [levels_hi-1] ascending           */
  const float* centroids_lo;        /* TQ: device [levels_lo]                       */
  const float* thresholds_lo;       /* TQ: device [levels_lo-1]                     */
  const uint16_t* rotation;         /* TQ_DENSE: device fp16 [layers][kv_heads][128][128]
                                       row-major (w_i = sum_j M_ij x_j), 16-byte
                                       aligned; NULL for the other bases             */
} semkv_quant_desc;

/* One mixed-precision cache Ĉ_KV (Algorithm 1 output, extended by Algorithm 2).
 * Every sequence of the batch has the same prompt length and the same r, so the
 * pool counts are equal across the batch and kept on the host.  Fields marked
 * (lib) are updated by the library; the caller initialises them to 0. */
typedef struct {
  int32_t batch, layers, kv_heads, q_heads, head_dim;  /* q_heads % kv_heads == 0 */
  int32_t block;               /* B of Algorithm 2 (1..1024)                       */
  uint8_t* hi_pool;            /* device [batch][layers][kv_heads][hi_cap][rec_hi], 16-B aligned */
  uint8_t* lo_pool;            /* device [batch][layers][kv_heads][lo_cap][rec_lo], 16-B aligned */
  int64_t hi_cap, lo_cap;      /* slots per (b, layer, head); multiples of 16, at
                                  most 2^30 (else SEMKV_EUNSUPPORTED)               */
  int32_t* hi_tok;             /* device [batch][hi_cap]: token index of each slot */
  int32_t* lo_tok;             /* device [batch][lo_cap]                            */
  int64_t hi_count, lo_count;  /* (lib) slots in use, same for every sequence      */
  int64_t n_tokens;            /* (lib) tokens quantized so far (prompt + blocks)  */
  uint16_t* stage_k;           /* device fp16 [batch][layers][kv_heads][block][128] */
  uint16_t* stage_v;           /* device fp16, same shape                           */
  float* stage_score;          /* device [batch][block]: scores of staged tokens    */
  int32_t stage_n;             /* tokens currently staged (caller writes the data
                                  at index stage_n, then increments it)            */
  uint8_t* blk_is_high;        /* device scratch [batch][block]                     */
  uint32_t* blk_slot;          /* device scratch [batch][block]                     */
  int32_t* dev_error;          /* device int32 error word (may be NULL)             */
} semkv_cache;

/* Bytes of one packed 128-value row with L levels (RB(L) above); 0 if unsupported. */
size_t semkv_row_bytes(int32_t levels);
/* Bytes of one record of the given base and level count; 0 if unsupported. */
size_t semkv_record_bytes(int32_t base, int32_t levels);

/* K = floor(r*T) with r = r_num/r_den, in 64-bit integers (Eq. 4). */
uint32_t semkv_high_count_floor(uint32_t T, uint32_t r_num, uint32_t r_den);
/* round(r*n), nearest integer with halves rounded up, in integers (Algorithm 2:
 * exactly round(rB) per block; the flush of a partial block uses n = |S|). */
uint32_t semkv_block_high_count(uint32_t n, uint32_t r_num, uint32_t r_den);

/* Gaussian N(0,1) Lloyd-Max codebook with L levels (Sec. 4.9: "Gaussian-optimal
 * Lloyd-Max codebook", extended to any integer L).  Computed on the host in fp64
 * by Lloyd iteration to convergence, then made exactly symmetric (c_l = -c_{L-1-l});
 * centroids[L] = fp32(c_l), thresholds[L-1] = fp32((c_l + c_{l+1})/2) taken in fp64.
 * Host pointers. */
semkv_status semkv_lloyd_max_gaussian(int32_t levels, float* centroids, float* thresholds);

/* Top-r selection, Eqs. 4-5 / Algorithm 1.  For each sequence b of `batch`:
 * H = the n_high tokens with the largest score, ties broken by lower token index
 * (NaN ranks below every number, -0 equals +0).  Outputs (device):
 *   is_high[b][i] = 1 if i in H else 0            (u8  [batch][T])
 *   slot[b][i]    = #{j < i : is_high[b][j] == is_high[b][i]}   (u32 [batch][T])
 *   rank[b][i]    = position of i in the (score desc, index asc) order, 0-based
 *                   (u32 [batch][T]; may be NULL).
 * scores: device f32 [batch][T].  ws/ws_bytes: device workspace of at least
 * semkv_rank_workspace_bytes(batch, T, rank != NULL) bytes, 4-byte aligned, owned by
 * the caller: 16 * batch * T bytes when ranks are wanted (keys and indices of a
 * stable radix sort, double-buffered), else 0 and ws may be NULL.
 * Errors: SEMKV_EINVAL (null pointers, T outside 1..2^24, n_high > T),
 * SEMKV_EWORKSPACE (rank set and ws missing or too small), SEMKV_EALIGN. */
size_t semkv_rank_workspace_bytes(int32_t batch, int32_t T, int32_t want_rank);
semkv_status semkv_rank_assign(const float* scores, int32_t batch, int32_t T,
                               uint32_t n_high, uint8_t* is_high, uint32_t* slot,
                               uint32_t* rank, void* ws, size_t ws_bytes, void* stream);

/* Fake quantization (Sec. 4.1: the quality experiments quantize, dequantize and compute
 * in fp16).  Every row of K and V is quantized with the same arithmetic as
 * semkv_quantize_pack at its token's level count (levels_hi where is_high[b][t], else
 * levels_lo; is_high NULL puts every token at levels_hi, a uniform grid point) and
 * reconstructed to fp16, in binary32 in this order:
 *   affine: out_d = fp16( z + s * c_d )
 *   TQ:     y = unnormalised FWHT(cb[c]) (stages 1..64);  out_d = fp16( (sign_d * y_d) * (n/128) )
 * k, v, k_out, v_out: device fp16 [batch][layers][kv_heads][T][128], 16-byte aligned
 * (rows move in 16-byte chunks), caller-owned (outputs may not alias inputs); is_high:
 * device u8 [batch][T] or NULL.
 * Errors: SEMKV_EINVAL, SEMKV_EALIGN, SEMKV_EUNSUPPORTED (level counts, base).  There is
 * no device error word: nothing in these kernels can time out (their copies are waited for
 * by group, not on a barrier). */
semkv_status semkv_fake_quant(const semkv_quant_desc* desc, const uint16_t* k, const uint16_t* v,
                              int32_t batch, int32_t layers, int32_t kv_heads, int32_t T,
                              const uint8_t* is_high, uint16_t* k_out, uint16_t* v_out,
                              void* stream);

/* KV-norm importance indicator (Sec. 3.3, "KV-norm" family: key-norm ||K_i||_2 and
 * value-norm ||V_i||_2, the magnitude of the tensor being compressed; Sec. 4.5 finds
 * value-norm the cheapest indicator profiled).  Writes
 *   scores[b][t] = || x[b][l][h][t][:] ||_2 over l in [layer_begin, layer_end) and all h
 * (a layer range restricts the score to the last m layers, as Eq. 3 does).
 * x: device fp16 [batch][layers][kv_heads][T][128] (pass the K cache for key-norm, the V
 * cache for value-norm), 8-byte aligned; scores: device f32 [batch][T], 4-byte aligned,
 * both caller-owned.  The summation order is fixed (per dim group of 4, row by row, then
 * a pairwise tree over the 32 groups), so equal inputs give bit-identical scores.
 * The scores feed semkv_rank_assign directly (only their ranking matters).
 * Errors: SEMKV_EINVAL (null pointers, empty or inverted ranges), SEMKV_EALIGN. */
semkv_status semkv_score_kv_norm(const uint16_t* x, int32_t batch, int32_t layers,
                                 int32_t kv_heads, int32_t T, int32_t layer_begin,
                                 int32_t layer_end, float* scores, void* stream);

/* Token-wise quantization, Eq. 7 / Algorithm 1: quantize every row of the prompt
 * K/V with Q_{b_i} and write token i's record (for every layer and KV head) to
 * slot[b][i] of the high pool if is_high[b][i] else of the low pool; writes
 * hi_tok/lo_tok[b][slot] = i.  k, v: device fp16 [batch][layers][kv_heads][T][128],
 * 8-byte aligned for AFFINE, 16-byte aligned for the other bases (their rows arrive by
 * bulk or tensor copies in 16-byte units); the same holds for the stage buffers in
 * semkv_append_block.  is_high, slot: as produced by semkv_rank_assign for this T.  n_high: the number
 * of high tokens per sequence (used for the capacity check and the counts).
 * Sets cache->hi_count = n_high, lo_count = T - n_high, n_tokens = T and resets
 * stage_n to 0 (a prompt replaces whatever the cache held). */
semkv_status semkv_quantize_pack(const semkv_quant_desc* desc, const uint16_t* k,
                                 const uint16_t* v, int32_t T, const uint8_t* is_high,
                                 const uint32_t* slot, uint32_t n_high, semkv_cache* cache,
                                 void* stream);

/* Block-exact deferred quantization, Sec. 3.7 / Algorithm 2: quantizes the n =
 * cache->stage_n staged tokens, exactly semkv_block_high_count(n, r_num, r_den) of
 * them (the highest staged scores, ties to the earlier token) at levels_hi, the rest
 * at levels_lo, appends them to the pools after the current counts, records their
 * token indices n_tokens + j, then advances hi_count / lo_count / n_tokens and sets
 * stage_n = 0.  Call it when stage_n == block (a full block) or at the end of a
 * turn with 0 < stage_n < block (the residual flush).  stage_n == 0 is a no-op. */
semkv_status semkv_append_block(const semkv_quant_desc* desc, semkv_cache* cache,
                                uint32_t r_num, uint32_t r_den, void* stream);

/* Single-query decode attention over the whole cache of one layer ("use Ĉ_KV for
 * decoding", Algorithm 1; the staged fp16 tokens take part, Algorithm 2):
 *   out[b][qh] = sum_i softmax_i(scale * q[b][qh] . k^_i) * v^_i
 * over i = all hi_count + lo_count quantized tokens and the stage_n staged tokens
 * of sequence b, with KV head h = qh / (q_heads / kv_heads) and k^, v^ the
 * dequantized rows (affine: z + s*c; TQ: n/128 * S H cb[c]).  Computed split-K over
 * the tokens with an online softmax and a final combine.
 * q: device fp16 [batch][q_heads][128]; out: device f32 [batch][q_heads][128].
 * ws: device workspace of semkv_decode_workspace_bytes(cache) bytes, 16-B aligned.
 * Accuracy: against fp64 attention over the same dequantized cache, max-abs error
 * <= 2e-3 and relative L2 <= 1e-3 for values of magnitude below 64; binary32 carries
 * relative error, so for larger values the absolute error grows as up to 8e-6 *
 * max|v^| (all of fp16's range, including subnormal steps, is supported). */
size_t semkv_decode_workspace_bytes(const semkv_cache* cache);
semkv_status semkv_decode_attention(const semkv_quant_desc* desc, const semkv_cache* cache,
                                    int32_t layer, const uint16_t* q, float* out,
                                    float softmax_scale, void* ws, size_t ws_bytes,
                                    void* stream);

/* Decode attention for callers that cannot allocate device memory.  The paper has
 * no counterpart: this is a deployment variant of semkv_decode_attention.
 * Who needs it: a caller whose host framework owns all device memory and gives this
 * library only the cache and the tensors of the call, or a serving loop that must
 * not call cudaMalloc between decode steps (an allocation can synchronise the device).
 * It computes what semkv_decode_attention computes, for every base, with the same
 * kernels, but keeps the split-K partial results in a static device array of 8 MiB
 * (2016 partials) that the library owns, instead of a caller workspace; it calls no
 * cudaMalloc, cudaFree or allocating routine.  Every GPU that loads the library
 * holds that array until the process exits.
 *  - Set-up: the first call on each device looks up the array's device address
 *    (cudaGetSymbolAddress) with that device current and caches it; make that first
 *    call before any stream capture.  The cached address is not refreshed after
 *    cudaDeviceReset.  Host threads may make their first calls concurrently.
 *  - Limit: each (sequence, KV head) pair gets cap = min(65, 2016 / (batch *
 *    kv_heads)) partial slots, and the split count is reduced to fit them.  The
 *    affine bases (balanced plan) need cap >= 3 + stage, i.e. batch * kv_heads <= 672,
 *    or <= 504 with staged tokens; the TQ bases (split plan) need cap >= one per
 *    non-empty pool + stage, i.e. batch * kv_heads * (pools + stage) <= 2016.
 *    Larger requests return SEMKV_EWORKSPACE before anything is launched.  The dense-
 *    rotation base (TQ_DENSE) also keeps its rotated queries in a second static array
 *    of 4096 query heads (batch * q_heads beyond it: SEMKV_EWORKSPACE).
 *  - All calls share the array, which keeps the last call's contents (each call
 *    overwrites every partial it reads, so nothing needs clearing).  Calls whose
 *    kernels overlap on the GPU (e.g. on two streams, or two host threads) race on
 *    it: serialise them.
 * Arguments and errors otherwise as semkv_decode_attention (no ws / ws_bytes). */
semkv_status semkv_decode_attention_noalloc(const semkv_quant_desc* desc,
                                            const semkv_cache* cache, int32_t layer,
                                            const uint16_t* q, float* out, float softmax_scale,
                                            void* stream);

/* One step of beam search: the best continuations of each group's beams.  Row r = group * beams + b of
 * the logits belongs to beam b of the group, which stands at scores[r] (the sum of its tokens' log
 * probabilities).  Token t of that row is a candidate with
 *   scores[r] + logits[r][t] - ln sum_u exp(logits[r][u])
 * and the k best of the group's beams * vocab candidates, best first, go to parent (the row r), token
 * and score.  The order is that of the exact scores as far as they can be told apart (see below);
 * equal ones: the lower row first, then the lower token.  (-0 equals +0.)
 *  - A logit of -infinity is no candidate (a banned token).  Neither is a NaN or +infinity, which count
 *    as -infinity; they write 4 into the error word.
 *  - A row whose score is -infinity has no candidates and is not read (the first step of a search: all
 *    beams but one).  Nor has one whose score is a NaN or +infinity, which writes 4.
 *  - done (may be NULL): device u8 [groups * beams].  A row with done != 0 is not read either; it has one
 *    candidate, end_token at scores[r].
 *  - A score below binary32's range is given as its lowest number.  Such candidates come behind all others, the
 *    lower row first, then the larger logit, then the lower token.
 *  - Where there are fewer than k candidates the rest is parent -1, token -1, score -infinity.
 * logits: device [groups * beams][vocab] of type `dtype` (SEMKV_F16, SEMKV_BF16 or SEMKV_F32), `stride`
 * >= vocab elements from row to row, aligned to its type; scores: device f32 [groups * beams]; parent,
 * token: device i32 [groups][k]; score: device f32 [groups][k].  beams, k: 1 .. 128; vocab: 1 .. 2^24;
 * groups * beams: up to 2^20.  end_token: 0 .. vocab-1 where done is given, else not used.  dev_error:
 * device i32 or NULL.  With k = beams, score may be scores: the new ones take the old ones' place.
 * Accuracy: sums of exponentials are binary32 with a known bound (2^-19 of the sum at most); where two
 * candidates of different beams whose order matters lie within it, their rows are summed again to 2^-38,
 * so that what comes out is the order by exact scores unless these agree to 2^-36, or to 2^-40 of the beams'
 * scores and of how far the logits lie below their rows' largest; equal rows with equal scores do.  score is
 * rounded once to binary32 from a sum within the first bound; its last bits may depend on where the rows lie
 * (modulo 16 bytes) and on the sizes.  Apart from that equal calls give equal bits.
 * A group sums its rows again one after the other, 44 us each at a vocabulary of 131072: few inputs have
 * more than one or two such rows, but sixteen beams that are all alike take 0.7 ms, and 1.7 ms where all their
 * logits are equal (hundreds of candidates that agree), in place of 30 us.
 * ws: device workspace of semkv_beam_select_workspace_bytes bytes, 16-byte aligned; calls that may
 * overlap on the GPU need one each.  Nothing in it has to be kept or cleared.
 * Errors: SEMKV_EINVAL, SEMKV_EALIGN, SEMKV_EUNSUPPORTED (dtype, more beams, k, vocab or rows than above),
 * SEMKV_EWORKSPACE.  groups 0 is a no-op. */
enum { SEMKV_BEAM_MAX = 128 };  /* beams of a group, and k */
size_t semkv_beam_select_workspace_bytes(int32_t groups, int32_t beams, int32_t vocab, int32_t dtype,
                                         int32_t k);
semkv_status semkv_beam_select(int32_t groups, int32_t beams, int32_t vocab, int32_t dtype,
                               const void* logits, int64_t stride, const float* scores,
                               const uint8_t* done, int32_t end_token, int32_t k, int32_t* parent,
                               int32_t* token, float* score, int32_t* dev_error, void* ws,
                               size_t ws_bytes, void* stream);

/* ------------------------------------------------ a paged cache held in 4 bits ----
 * A cache of its own beside semkv_cache, for serving: sequences of different lengths,
 * pages that several sequences share, queries of one token or of many.  The paper has no
 * counterpart (its caches are the pools above; Sec. 4.7 prunes tokens, as
 * semkv_kv4_compact does here by the flags of semkv_rank_assign).
 *
 * Format.  A row of head_dim values is held in blocks of 16 along the head dim: one e4m3
 * scale s and 16 e2m1 codes (two to a byte, the lower dim in the lower half).  With g the
 * row's float32 scale (its layer's and KV head's entry of k_scale or v_scale) a value is
 * code * s * g.  Writing a block x, in binary32:
 *   a = max |x_j| over the entries that are not NaN
 *   s = e4m3(min(448, a / (6 * g)))           nearest, ties to even
 *   code_j = e2m1(x_j / (s * g))              nearest, ties to even, limited to +-6
 * and all codes 0 where s = 0.  A NaN is stored as 0 and an infinity as the largest value
 * of its block; either writes 4 into the error word.
 * Sixteen tokens of one head form a tile of 18 * head_dim bytes:
 *   [K codes 16][head_dim/2] [V codes 16][head_dim/2] [K scales 16][head_dim/16] [V scales]
 * and a page of page_tokens tokens holds page_tokens / 16 tiles for every head.
 *
 * Error word: 1 a wait that timed out, 2 too few free pages, a table too short or a
 * destination in use, 3 an index outside its range (a page, a sequence, a row range) or
 * a sequence listed twice where it may not be, 4 a NaN or an infinity stored.  The first
 * one written stays.  What an entry does with a wrong index is given with each call; none
 * reads or writes outside the buffers it was given.
 *
 * Table, length and refs are these calls' to change.  A length lowered by hand leaves the
 * pages behind its end counted although no table entry in use names them: they do not come
 * back to the pool.
 *
 * Calls that may overlap on the GPU.  Reserve, fork, free, reorder and compact go by
 * the counts and change them without locks: on one cache they run one after the other (one
 * stream, or events between them), else a page may be given away twice.  Write, read and
 * attention may overlap with one another, and with those five where these take other
 * sequences.  No call may overlap with one that changes the length, the table row or the
 * stored rows of a sequence that it uses; the promise above holds for state that stands
 * still while the call runs. */
enum { SEMKV_KV4_MAX_SEQS = 65535 };  /* sequences of one call */

typedef struct {
  int32_t layers, kv_heads;
  int32_t head_dim;            /* 64 or 128                                          */
  int32_t page_tokens;         /* 16, 32, 64 or 128                                  */
  int32_t num_pages;           /* pages of the pool                                  */
  int32_t max_seqs, max_pages; /* sequences, and table entries of each               */
  uint8_t* pages;       /* device [layers][num_pages][kv_heads][page_tokens/16][tile],
                           16-byte aligned                                           */
  const float* k_scale; /* device [layers][kv_heads], each in 2^-40 .. 2^40; NULL = 1 */
  const float* v_scale; /* the same for V                                            */
  int32_t* table;       /* device [max_seqs][max_pages]: the page of each page_tokens
                           tokens.  Entries past a sequence's length mean nothing.   */
  int32_t* length;      /* device [max_seqs]: tokens that each sequence holds        */
  int32_t* refs;        /* device [num_pages], 16-byte aligned: table entries in use that
                           name the page; 0 = free.  All zero, like length, in a new
                           cache.                                                    */
  int32_t* dev_error;   /* device int32 error word (may be NULL)                     */
} semkv_kv4_cache;

/* The rows of one step: which sequences take part, and how many rows each has in the
 * row-major tensors of the step's calls (k, v, q, out: [total][heads][head_dim]). */
typedef struct {
  int32_t n;             /* sequences that take part, 0..SEMKV_KV4_MAX_SEQS           */
  int32_t total;         /* rows of the tensors, 0..2^30; with 0 they may be NULL     */
  int32_t max_count;     /* no sequence has more rows than this (one that has is left
                            out, 3); it chooses the kernel and sizes the workspace    */
  const int32_t* seqs;   /* device [n], or NULL for 0 .. n-1                          */
  const int32_t* cu;     /* device [n+1], ascending: rows cu[i] .. cu[i+1]-1 are the
                            i-th sequence's; rows from cu[n] on belong to nobody and are
                            left as they are.  NULL: row i is the i-th sequence's     */
  int32_t* start;        /* device [n]: token position of the i-th sequence's first row,
                            written by semkv_kv4_reserve, read by semkv_kv4_write and
                            semkv_kv4_read; negative: its rows take no part           */
} semkv_kv4_batch;

/* Bytes of a tile, 18 * head_dim; 0 if the head_dim is not supported. */
size_t semkv_kv4_tile_bytes(int32_t head_dim);

/* Room for each sequence's rows: start[i] = length, length += count, with count = cu[i+1] -
 * cu[i].  Pages come from those with refs = 0, lowest first, to the sequences in the order
 * of the list.  A sequence whose last page is part full and shared (refs > 1) first gets a
 * copy of that page (every layer) in its place, so its new rows reach nobody else.  If the
 * pool or a table has too little room for all of them nothing changes, every start[i] is -1
 * and 2 goes into the error word.  A sequence listed before, out of range, or with a wrong
 * row range gets start[i] = -1 and is left out (3).
 * ws: device workspace of semkv_kv4_pages_workspace_bytes(cache, n, -1) bytes, 16-byte aligned.
 * Errors: SEMKV_EINVAL, SEMKV_EALIGN, SEMKV_EUNSUPPORTED, SEMKV_EWORKSPACE. */
size_t semkv_kv4_pages_workspace_bytes(const semkv_kv4_cache* cache, int32_t n, int32_t tokens);
semkv_status semkv_kv4_reserve(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch,
                               void* ws, size_t ws_bytes, void* stream);

/* Quantizes rows of K and V into one layer's pages: row cu[i] + j goes to position start[i]
 * + j.  k, v: device [total][kv_heads][head_dim] of type `dtype` with k_stride and v_stride
 * elements from row to row (a multiple of 8, at least kv_heads * head_dim), 16-byte aligned.
 * A row whose position lies outside its table, or whose page index lies outside the pool, is
 * left out (3).  Two rows of a call at one position leave parts of both.
 * semkv_kv4_read is the way back: k_out, v_out [total][kv_heads][head_dim], contiguous,
 * of type `dtype`, take the values (product with g in binary32, rounded once to the type). */
semkv_status semkv_kv4_write(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch,
                             int32_t layer, int32_t dtype, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, void* stream);
semkv_status semkv_kv4_read(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch,
                            int32_t layer, int32_t dtype, void* k_out, void* v_out,
                            void* stream);

/* semkv_kv4_write of rows whose position is still to be worked into them: keys are turned on their
 * way into the pages, and the step's queries, where q_heads > 0, from q into q_out.  A pair (a, b) of
 * the first rot_dim dims of a head becomes (a c - b s, b c + a s) with c and s the table's entries of the
 * row's position, in binary32, each product, sum and difference rounded by itself; the other dims stay
 * as they are.  A query is rounded once to `dtype`; K's blocks are quantized from the binary32 values.
 * The pair's index j selects cosine j and sine j:
 *   SEMKV_KV4_HALVES  dims j and j + rot_dim / 2
 *   SEMKV_KV4_PAIRS   dims 2 j and 2 j + 1
 * positions: device i32 [total], the position of each row, or NULL: where it goes in its sequence
 * (start[i] + j).  They differ where a sequence was pruned.  A row whose position lies outside the table
 * is left out (3), queries and values too, like a row without a place in the pages; nothing of a row
 * that is left out is written.
 * q, q_out: device [total][q_heads][head_dim] of type `dtype`, with q_stride and q_out_stride
 * elements from row to row (as k's), 16-byte aligned; q_out may be q, with the same stride, and does not
 * overlap it otherwise.  With q_heads 0 they are not used.
 * Errors: SEMKV_EINVAL (rot_dim outside 1..head_dim among them), SEMKV_EALIGN, SEMKV_EUNSUPPORTED
 * (rot_dim not a multiple of 16, an unknown layout). */
enum { SEMKV_KV4_HALVES = 0, SEMKV_KV4_PAIRS = 1 };

typedef struct {
  int32_t rot_dim;       /* dims of each head that are turned: a multiple of 16, up to head_dim */
  int32_t layout;        /* SEMKV_KV4_HALVES or SEMKV_KV4_PAIRS                         */
  int32_t rows;          /* positions in the table                                      */
  const float* cos_sin;  /* device [rows][rot_dim], 16-byte aligned: the position's rot_dim / 2
                            cosines, then its sines                                      */
} semkv_kv4_rotation;

semkv_status semkv_kv4_write_rotated(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch,
                                     int32_t layer, const semkv_kv4_rotation* rotation,
                                     const int32_t* positions, int32_t dtype, const void* q,
                                     int64_t q_stride, int32_t q_heads, void* q_out,
                                     int64_t q_out_stride, const void* k, int64_t k_stride,
                                     const void* v, int64_t v_stride, void* stream);

/* Causal attention of a step's rows over one layer of their sequences.  With length L and m
 * rows, the sequence's j-th row stands at position p = L - m + j and sees the positions
 * max(0, p - window + 1) .. p (window 0: all up to p); a row at a negative position sees
 * nothing.  For query head h of row r, over the positions it sees, KV head h / (q_heads /
 * kv_heads):
 *   out[r][h] = sum_t softmax_t(softmax_scale * q[r][h] . K_t) V_t,   0 if it sees nothing
 *   lse[r][h] = ln sum_t exp(softmax_scale * q[r][h] . K_t)            (-inf if nothing)
 * q: device [total][q_heads][head_dim] of type `dtype`, q_stride elements from row to row (a
 * multiple of 8), 16-byte aligned; out: the same type, contiguous, apart from q; lse: device
 * f32 [total][q_heads] or NULL.  `start` is not used.  A sequence out of range or with a wrong row
 * range (more than max_count rows among them) is left out, its rows untouched (3); a length
 * past the table counts as the table's end and a page index outside the pool as page 0 (3).
 * Accuracy: products are exact in binary32; the weights are rounded to fp16 before they meet V
 * (relative 2^-11 each), as the result is to its type.  The sums are binary32, one chain over each
 * worker's share of the positions: every 16 of them can add 17 * 2^-23 of sum_t p_t |V_t| (2^-11 of
 * it for a share of 3800), every share that is joined 2^-20.  Logits are binary32 and may have any
 * finite size; their own rounding then decides what the softmax sees.
 * ws: device workspace of semkv_kv4_attention_workspace_bytes bytes, 16-byte aligned; calls
 * that may overlap on the GPU need one each. */
size_t semkv_kv4_attention_workspace_bytes(const semkv_kv4_cache* cache,
                                           const semkv_kv4_batch* batch, int32_t q_heads);
semkv_status semkv_kv4_attention(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch,
                                 int32_t layer, int32_t dtype, const void* q, int64_t q_stride,
                                 int32_t q_heads, void* out, float* lse, float softmax_scale,
                                 int32_t window, void* ws, size_t ws_bytes, void* stream);

/* Branches: dst[i] becomes a sequence with src[i]'s length and pages, which both then share
 * (refs + 1).  dst[i] has to be empty (length 0; else 2), and no destination may appear twice or
 * among the sources; an entry that breaks this or is out of range is left out (3).  A source
 * may appear more than once.  src, dst: device [n]. */
semkv_status semkv_kv4_fork(const semkv_kv4_cache* cache, int32_t n, const int32_t* src,
                            const int32_t* dst, void* stream);

/* Empties sequences: their pages' refs fall by one (0: free again), length = 0.  A sequence
 * listed twice is emptied once; one out of range is left out (3).  seqs: device [n] or NULL for
 * 0 .. n-1. */
semkv_status semkv_kv4_free(const semkv_kv4_cache* cache, int32_t n, const int32_t* seqs,
                            void* stream);

/* Sequences take one another's place, all at once: the i-th sequence of the list becomes a branch of
 * what the parent[i]-th of the list was before the call (its length, and its pages, which both then
 * share); parent[i] = i keeps it, parent[i] = -1 empties it.  Any map will do, a cycle among them, and a
 * state that no entry takes up is gone: its pages' refs fall.  Table entries past a new length stay
 * as they are.  An entry whose sequence was listed before or is out of range, or whose parent[i] is outside
 * -1 .. n-1 or names an entry out of range, is left out: it changes nothing (3).  (One whose sequence was
 * listed before still serves as a parent.)  seqs: device [n] or NULL for 0 .. n-1; parent: device [n], such
 * as semkv_beam_select gives for the rows that go on.
 * ws: device workspace of semkv_kv4_pages_workspace_bytes(cache, n, 0) bytes, 16-byte aligned. */
semkv_status semkv_kv4_reorder(const semkv_kv4_cache* cache, int32_t n, const int32_t* seqs,
                               const int32_t* parent, void* ws, size_t ws_bytes, void* stream);

/* Prunes sequences to some of their tokens, in order, in every layer: of the i-th sequence the
 * tokens t < tokens with keep[i][t] != 0 stay, and all from `tokens` on (they have no flag).
 * keep: device u8 [n][tokens], as semkv_rank_assign leaves is_high.  The kept rows move to
 * new pages, found as in semkv_kv4_reserve, and the old ones' refs fall by one: whoever else
 * shares those keeps its tokens.  If too few pages are free nothing changes (2).  A sequence
 * listed before or out of range is left out (3).
 * ws: semkv_kv4_pages_workspace_bytes(cache, n, tokens) bytes, 16-byte aligned. */
semkv_status semkv_kv4_compact(const semkv_kv4_cache* cache, int32_t n, const int32_t* seqs,
                               const uint8_t* keep, int32_t tokens, void* ws, size_t ws_bytes,
                               void* stream);

/* Failure-detection check (not a step of the paper's method).  Every kernel that
 * waits on a bulk copy uses one bounded mbarrier wait: after a fixed number of polls
 * (2^22) it gives up, writes 1 (a wait that timed out) into the device error word and
 * the kernel returns, so a lost copy never hangs the GPU and the context stays usable.
 * This entry point runs that same wait in one CTA of 4 warps on a barrier that nothing
 * arrives on, with the caller's poll limit `polls` (1 .. 2^22): each warp's wait runs
 * out and writes 1 into *dev_error (device int32, 4-byte aligned; the first error
 * written wins, so clear it first to see this one).  It lets a test make a wait run
 * out on purpose without faulting or hanging anything.  Stream-ordered; errors:
 * SEMKV_EINVAL (NULL dev_error, polls out of range), SEMKV_EALIGN, SEMKV_ECUDA. */
semkv_status semkv_debug_wait_timeout(int32_t* dev_error, uint32_t polls, void* stream);

/* Human-readable name of a status code (static string). */
const char* semkv_status_string(semkv_status s);

#ifdef __cplusplus
}
#endif
#endif /* SEMKV_H_ */
