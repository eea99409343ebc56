/*
 * fc.h -- C ABI of the MI355X (gfx950) Flash Communication quantization path.
 *
 * The library implements, on ONE GPU, the arithmetic that Flash Communication
 * (arXiv 2412.04964) wraps around its two exchanges (Algorithm 1, Section 3.2.2):
 *
 *     FinegrainedQuantize  ->  [All2All]  ->  Dequantize x N, ReduceSum,
 *     FinegrainedQuantize  ->  [All-Gather]  ->  Dequantize
 *
 * and, further down, the attention of a tensor-parallel rank that such all-reduces follow.
 * The exchanges themselves are not part of this library: the N partial tensors
 * (or their quantized slices) are simply N slabs in this GPU's memory.
 *
 * Quantizer (Appendix "Quantization Fundamentals", Eq. 1-2, asymmetric; groups
 * of `group` consecutive elements along `hidden`, Section 3.2.1), in fp32 with
 * round-to-nearest-even.  Results are bit-identical to evaluating, for every
 * group, exactly these operations in this order:
 *     mn, mx   = min, max of the group
 *     s        = (mx - mn) / (2^bits - 1)          one IEEE divide
 *     if !(s >= FLT_MIN):  s = |mn| >= FLT_MIN ? |mn| : 1       (constant group)
 *     inv      = 1 / s                              one IEEE divide
 *     z        = 0 - rint(mn * inv)                 integer-valued, NOT clamped
 *     q        = clamp(rint(x * inv) + z, 0, 2^bits - 1)
 * Dequantize (the inverse of Eq. 2):   x^ = (q - z) * s      (fp32 sub, fp32 mul)
 * ReduceSum: acc = +0; for j = 0..N-1 in order: acc = fma(q_j - z_j, s_j, acc).
 *
 * Data layouts (all device memory, dense, row-major):
 *   x, y     IEEE binary16 [tokens, hidden]
 *   codes    bytes [tokens, hidden*bits/8].  8 bit: one code per byte.  4 bit:
 *            two codes per byte, element 2k in bits 0-3, element 2k+1 in bits 4-7.
 *   scales   float [tokens, hidden/group]
 *   zeros    float [tokens, hidden/group]   (the zero-points z above)
 *
 * Common rules for every entry point
 *   - All pointers are DEVICE pointers unless stated otherwise, owned by the
 *     caller, 16-byte aligned (base pointers; the per-source meta slabs at
 *     +j*meta_src_stride_elems only need float alignment).  Inputs are never written; outputs must not
 *     overlap inputs.  The library allocates nothing and keeps no state except
 *     the last HIP error code.
 *   - Work is enqueued on `hip_stream` (a hipStream_t passed as void*; NULL is
 *     the default stream).  No call synchronizes.  The device that is current
 *     on the calling thread must own the buffers and the stream.
 *   - bits in {4, 8};  group a power of two in [32, 16384] (group == hidden: one group per token);
 *     hidden % group == 0;  tokens >= 0 (0 is a no-op returning FC_OK);
 *     tokens*hidden <= 2^36 (exactly 2^36 may be refused with FC_ERR_HIP: plain steps on 8-bit codes, and
 *     fc_allreduce_sim* without rotation);  1 <= n_src <= FC_MAX_SRC.
 *   - Inputs must be finite.  NaN / Inf inputs give unspecified codes.
 *   - Return value: FC_OK or a negative FC_ERR_* code.  Argument checks come
 *     first and make no HIP call, so they work on a host without a GPU.
 *     FC_ERR_HIP reports the status that the launch call itself returned (kept for
 *     fc_last_hip_error); the library never reads or clears the calling thread's
 *     HIP last-error state, so an error left there by other code is neither
 *     reported as ours nor consumed.
 */
#ifndef FC_H
#define FC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define FC_API __attribute__((visibility("default")))
#else
#define FC_API
#endif

#define FC_MAX_SRC 8

enum {
    FC_OK = 0,
    FC_ERR_NULL = -1,       /* a required pointer is NULL */
    FC_ERR_BITS = -2,       /* bit-width not 4 or 8 */
    FC_ERR_GROUP = -3,      /* unsupported group size, or hidden % group != 0 */
    FC_ERR_SHAPE = -4,      /* tokens < 0, hidden <= 0, too many elements, n_src out of range,
                               or a source stride smaller than one slab */
    FC_ERR_ALIGN = -5,      /* pointer or stride not 16-byte aligned */
    FC_ERR_WORKSPACE = -6,  /* workspace NULL or too small */
    FC_ERR_HIP = -7,        /* kernel launch failed; see fc_last_hip_error() */
    FC_ERR_TYPE = -8        /* element type, or quantizer, that the call does not take */
};

/*
 * FinegrainedQuantize of Algorithm 1 (first call), Eq. 1-2.
 *   x_f16   in   binary16 [tokens, hidden]
 *   codes   out  [tokens, hidden*bits/8] bytes
 *   scales  out  float [tokens, hidden/group]
 *   zeros   out  float [tokens, hidden/group]
 */
FC_API int fc_quantize(const void *x_f16, int64_t tokens, int64_t hidden, int group, int bits,
                       void *codes, float *scales, float *zeros, void *hip_stream);

/*
 * The body of Algorithm 1 between the two exchanges, fused: Dequantize each of
 * the n_src received slices with its own scale and zero-point, ReduceSum (fp32
 * FMA chain, source order), FinegrainedQuantize of the sum with bits_out.  The
 * fp32 sum never goes to memory.  bits_in = 4 with bits_out = 8 is the paper's
 * "INT6" setting (Section 3.2.3).
 *   codes_in   in  source j's codes start at (char*)codes_in + j*codes_src_stride_bytes,
 *                  each [tokens, hidden*bits_in/8]
 *   scales_in, zeros_in
 *              in  source j's arrays start at +j*meta_src_stride_elems floats,
 *                  each [tokens, hidden/group]
 *   codes_src_stride_bytes >= tokens*hidden*bits_in/8, multiple of 16;
 *   meta_src_stride_elems  >= tokens*hidden/group (both ignored when
 *   n_src == 1).
 *   codes_out, scales_out, zeros_out   out, as in fc_quantize with bits_out.
 */
FC_API int fc_dequant_reduce_requant(const void *codes_in, int64_t codes_src_stride_bytes,
                                     const float *scales_in, const float *zeros_in,
                                     int64_t meta_src_stride_elems,
                                     int n_src, int64_t tokens, int64_t hidden, int group,
                                     int bits_in, int bits_out,
                                     void *codes_out, float *scales_out, float *zeros_out,
                                     void *hip_stream);

/*
 * Dequantize of Algorithm 1 (last call): y = binary16_rne((q - z) * s).
 * Values beyond the binary16 range become infinities.
 */
FC_API int fc_dequantize(const void *codes, const float *scales, const float *zeros,
                         int64_t tokens, int64_t hidden, int group, int bits,
                         void *y_f16, void *hip_stream);

/*
 * Algorithm 1 end to end on one device with identity exchanges:
 * n_src x fc_quantize(bits_rs) into the workspace, fc_dequant_reduce_requant
 * (bits_rs -> bits_ag), fc_dequantize.  The volume is quantized and dequantized
 * exactly twice (Table 1, "QDQ Step").
 *   x_f16      in   binary16 [n_src, tokens, hidden]
 *   y_f16      out  binary16 [tokens, hidden]
 *   workspace  device scratch of at least fc_allreduce_sim_workspace_bytes(...)
 *              bytes, 16-byte aligned; contents on return are unspecified.
 * The call runs as ONE kernel that keeps both quantizations in
 * registers (the single fused kernel of Section 3.2.3, "Kernel Design", with identity exchanges): the
 * partials are read once and the result is written once, 2 n_src + 2 bytes per element.  It evaluates
 * the same operations in the same order, so the result is bit-identical to the three steps, and it
 * does not touch the workspace (which must still be passed).
 */
FC_API int fc_allreduce_sim(const void *x_f16, int n_src, int64_t tokens, int64_t hidden,
                            int group, int bits_rs, int bits_ag, void *y_f16,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

/* Bytes fc_allreduce_sim needs; 0 if the arguments are invalid. */
FC_API size_t fc_allreduce_sim_workspace_bytes(int n_src, int64_t tokens, int64_t hidden, int group,
                                               int bits_rs, int bits_ag);

/*
 * fc_allreduce_sim for callers that cannot allocate device memory or keep a workspace (code
 * under HIP graph capture, tight serving loops, harnesses that forbid allocation): always the
 * three steps, with the intermediate codes, scales and zero-points in a fixed array of
 * FC_STATIC_SCRATCH_BYTES that lives in the library's device image (one copy per GPU, held until
 * the process ends).  The call allocates and frees nothing.  Same arguments, results and errors
 * as fc_allreduce_sim, plus:
 *   - FC_ERR_WORKSPACE when fc_allreduce_sim_workspace_bytes(...) exceeds
 *     FC_STATIC_SCRATCH_BYTES (e.g. 8 partials of 128 x 8192 at 8 bit, group 128, need 9.6 MB;
 *     the prefill volumes do not fit and must use fc_allreduce_sim);
 *   - all calls on one GPU share that GPU's array: calls that may overlap in time on one GPU
 *     (different streams, different threads) race; serialize them;
 *   - the first call on a device looks up the array's address (hipGetSymbolAddress); make
 *     that call outside graph capture.
 */
#define FC_STATIC_SCRATCH_BYTES (32u << 20)

FC_API int fc_allreduce_sim_static(const void *x_f16, int n_src, int64_t tokens, int64_t hidden,
                                   int group, int bits_rs, int bits_ag, void *y_f16, void *hip_stream);

/*
 * Symmetric variant (Appendix "Quantization Fundamentals", Eq. 3-4; the paper's
 * INT8_Sym / INT4_Sym ablation rows).  Same layouts and rules as above except:
 * there is no zero-point array, and codes are SIGNED, stored in two's
 * complement (8 bit: one int8 per byte; 4 bit: two per byte, element 2k in bits
 * 0-3).  Results are bit-identical to evaluating, for every group,
 *     s   = max|x| / (2^(bits-1) - 1)           one IEEE divide
 *     if !(s >= FLT_MIN): s = 1                  (all-zero group)
 *     inv = 1 / s                                 one IEEE divide
 *     q   = clamp(rint(x * inv), -2^(bits-1), 2^(bits-1) - 1)
 * Dequantize: x^ = q * s.  ReduceSum: acc = +0; acc = fma(q_j, s_j, acc), j = 0..N-1.
 */
FC_API int fc_quantize_sym(const void *x_f16, int64_t tokens, int64_t hidden, int group, int bits,
                           void *codes, float *scales, void *hip_stream);

FC_API int fc_dequant_reduce_requant_sym(const void *codes_in, int64_t codes_src_stride_bytes,
                                         const float *scales_in, int64_t meta_src_stride_elems,
                                         int n_src, int64_t tokens, int64_t hidden, int group,
                                         int bits_in, int bits_out,
                                         void *codes_out, float *scales_out, void *hip_stream);

FC_API int fc_dequantize_sym(const void *codes, const float *scales,
                             int64_t tokens, int64_t hidden, int group, int bits,
                             void *y_f16, void *hip_stream);

/* Algorithm 1 end to end with the symmetric quantizer; workspace as for fc_allreduce_sim
   (fc_allreduce_sim_workspace_bytes gives a sufficient size). */
FC_API int fc_allreduce_sim_sym(const void *x_f16, int n_src, int64_t tokens, int64_t hidden,
                                int group, int bits_rs, int bits_ag, void *y_f16,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * FP8 variant (the FP8_Sym rows of the paper's precision table and rotation table;
 * format: Appendix "FP8 and FP4 Format").  Layouts and rules as for the 8-bit symmetric
 * variant, except that each code byte is one OCP FP8 E4M3 number (1 sign, 4 exponent
 * bits with bias 7, 3 fraction bits, subnormals, no infinities, largest value 448).
 * Results are bit-identical to evaluating, for every group,
 *     s   = max|x| / 448                         one IEEE divide
 *     if !(s >= FLT_MIN): s = 1                  (all-zero group)
 *     inv = 1 / s                                 one IEEE divide
 *     q   = E4M3(x * inv)     nearest, ties to the even fraction, sign kept (-0 is byte 0x80)
 * Dequantize: x^ = value(q) * s.  ReduceSum: acc = +0; acc = fma(value(q_j), s_j, acc).
 * Input bytes 0x7F / 0xFF (NaN) are outside the domain.
 */
FC_API int fc_quantize_fp8(const void *x_f16, int64_t tokens, int64_t hidden, int group,
                           void *codes, float *scales, void *hip_stream);

FC_API int fc_dequant_reduce_requant_fp8(const void *codes_in, int64_t codes_src_stride_bytes,
                                         const float *scales_in, int64_t meta_src_stride_elems,
                                         int n_src, int64_t tokens, int64_t hidden, int group,
                                         void *codes_out, float *scales_out, void *hip_stream);

FC_API int fc_dequantize_fp8(const void *codes, const float *scales,
                             int64_t tokens, int64_t hidden, int group, void *y_f16, void *hip_stream);

/* Algorithm 1 end to end with FP8 on both sides; workspace of
   fc_allreduce_sim_workspace_bytes(n_src, tokens, hidden, group, 8, 8) bytes suffices. */
FC_API int fc_allreduce_sim_fp8(const void *x_f16, int n_src, int64_t tokens, int64_t hidden, int group,
                                void *y_f16, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Compact-metadata variant of the asymmetric quantizer (Eq. 1-2; the paper does not say
 * how a group's scale and zero-point are stored or sent): both are kept in binary16, one
 * 32-bit word per group, so a group carries 4 bytes of metadata instead of 8.
 *   meta   uint32 [tokens, hidden/group]; bits 0-15 the scale, bits 16-31 the zero-point
 * Other layouts and rules as for fc_quantize.  Results are bit-identical to evaluating, for
 * every group,
 *     s   as in fc_quantize (including the constant-group rule), then
 *     s   = binary16_rne(s) kept inside [2^-24, 65504]  (zero -> 2^-24, overflow -> 65504)
 *     inv = 1 / s                                 one IEEE divide, of the stored scale
 *     z   = 0 - rint(mn * inv), then binary16_rne(z) saturated at +-65504
 *                                                 (integers up to 2048 are unchanged)
 *     q   = clamp(rint(x * inv) + z, 0, 2^bits - 1)
 * Dequantize: x^ = (q - z) * s with the two stored numbers widened to fp32; ReduceSum as in
 * fc_dequant_reduce_requant.  Input words must hold a positive finite scale and a finite
 * zero-point.  meta_src_stride_elems counts 32-bit words.
 */
FC_API int fc_quantize_cmeta(const void *x_f16, int64_t tokens, int64_t hidden, int group, int bits,
                             void *codes, uint32_t *meta, void *hip_stream);

FC_API int fc_dequant_reduce_requant_cmeta(const void *codes_in, int64_t codes_src_stride_bytes,
                                           const uint32_t *meta_in, int64_t meta_src_stride_elems,
                                           int n_src, int64_t tokens, int64_t hidden, int group,
                                           int bits_in, int bits_out,
                                           void *codes_out, uint32_t *meta_out, void *hip_stream);

FC_API int fc_dequantize_cmeta(const void *codes, const uint32_t *meta,
                               int64_t tokens, int64_t hidden, int group, int bits,
                               void *y_f16, void *hip_stream);

/* Algorithm 1 end to end with binary16 metadata; workspace as for fc_allreduce_sim
   (fc_allreduce_sim_workspace_bytes gives a sufficient size). */
FC_API int fc_allreduce_sim_cmeta(const void *x_f16, int n_src, int64_t tokens, int64_t hidden,
                                  int group, int bits_rs, int bits_ag, void *y_f16,
                                  void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Rotation variant (paper Section 4, "Naive vs. Rotation-based Quantization": the Hadamard
 * transform of QuaRot around the quantized all-reduce).  Every partial is rotated before
 * the first quantization; the rotation is linear, so the unchanged
 * fc_dequant_reduce_requant* step sums rotated partials; the inverse rotation follows the
 * last Dequantize.  `quantizer` selects the code (FC_QUANTIZER_*; FP8 needs bits == 8;
 * zeros may be NULL unless FC_QUANTIZER_ASYM).  The transform runs over every aligned block of
 * B elements of a token's row, B the largest power of two that divides hidden: the whole row when
 * hidden is a power of two, five blocks of 1024 for hidden 5120 (the rotation table's LLaMA-2-13B
 * row; the paper names no transform for such a length).  B must be 1024, 2048, 4096 or 8192
 * (FC_ERR_SHAPE otherwise); every group, a power of two dividing hidden, lies inside one block.
 * Other rules as above.  Results are bit-identical to:
 *     r = WHT_B(x) * 2^-ceil(n/2),  n = log2(B)          (fc_quantize_rot, then the quantizer on r in fp32)
 *     y = binary16(WHT_B(x^) * 2^-floor(n/2))            (fc_dequantize_rot on the dequantized fp32 x^)
 * where WHT_B applies, to each block, the natural-order Walsh-Hadamard transform evaluated in
 * fp32 as butterfly stages (a, b) -> (a + b, a - b) with spans 1, 2, 4, ..., B/2 in that order.
 */
#define FC_QUANTIZER_ASYM 0   /* Eq. 1-2 */
#define FC_QUANTIZER_SYM 1    /* Eq. 3-4 */
#define FC_QUANTIZER_FP8 2    /* E4M3 bytes */

FC_API int fc_quantize_rot(const void *x_f16, int64_t tokens, int64_t hidden, int group, int bits,
                           int quantizer, void *codes, float *scales, float *zeros, void *hip_stream);

FC_API int fc_dequantize_rot(const void *codes, const float *scales, const float *zeros,
                             int64_t tokens, int64_t hidden, int group, int bits, int quantizer,
                             void *y_f16, void *hip_stream);

/* Algorithm 1 with the rotation around it: fc_quantize_rot x n_src -> fc_dequant_reduce_requant* -> fc_dequantize_rot
   through the workspace where that is faster (some volumes of three and more sources), else one kernel, bit-identical;
   workspace as for fc_allreduce_sim. */
FC_API int fc_allreduce_sim_rot(const void *x_f16, int n_src, int64_t tokens, int64_t hidden,
                                int group, int bits_rs, int bits_ag, int quantizer, void *y_f16,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ---- Attention of a tensor-parallel rank: what runs between its projections, before the all-reduce above ----
 *
 * Activations are 16-bit (`type`: FC_TYPE_F16 or FC_TYPE_BF16) tensors [tokens, heads, dim] whose last axis is dense; token and head
 * strides are in elements, any multiple of 8 (views of a joint projection pass as they are), base pointers are 16-byte
 * aligned.  Arithmetic and sums are in fp32, except that the two attention calls round what goes into their matrix products to 16 bits:
 *     over the cache    softmax weights times their pages' scales to binary16: 11 bits for what is less than 2^26 below a row's largest,
 *                       what is 2^37 below may be lost; bfloat16 queries to binary16 after a power of two per row
 *     over prompts      softmax weights to `type`; binary16: 11 bits for what is less than 2^9 below the largest of 32 or 64 tokens
 * The weights' sum is of the unrounded ones.
 *
 * Sequences are packed: the call's new tokens of sequence b are offsets[b] <= t < offsets[b + 1] (int32 [sequences + 1], offsets[0] = 0,
 * ascending, offsets[sequences] = tokens; equal neighbours: nothing new).  All index arrays are device memory; the kernels
 * check what they read from them, and a token, page or position outside its tensor is neither read nor written.  (Where offsets do
 * not ascend, which tokens are computed is unspecified.)
 */
#define FC_TYPE_F16 0
#define FC_TYPE_BF16 1
#define FC_TYPE_F32 2         /* the weight of a norm only */

/*
 * The table of a rotation: for row r and pair i < rotary / 2, with angle = r * frequencies[i] in 64 bits,
 *     table[r, i] = magnitude * cos(angle),  table[r, rotary / 2 + i] = magnitude * sin(angle)
 * frequencies: double [rotary / 2], device memory.  table: float [rows, rotary].
 */
FC_API int fc_rotary_table(const double *frequencies, int64_t rows, int rotary, double magnitude, float *table, void *hip_stream);

/*
 * Rotary positions: of the first `rotary` elements of each head (even, at most dim), pair i turns by row positions[t] of the table,
 *     a' = a cos - b sin,  b' = b cos + a sin       (inverse != 0: with -sin, which is also the gradient)
 * a, b = elements i and i + rotary / 2, or interleaved != 0: 2 i and 2 i + 1.  Each product and sum is rounded to fp32, the
 * result once to the type; other elements are copied.  A position without a row gives NaN.  y == x with equal strides is allowed.
 * dim: a multiple of 8 up to 4096.
 */
FC_API int fc_rotary(const void *x, int64_t x_token_stride, int64_t x_head_stride, const float *table, int64_t table_rows,
                     const int32_t *positions, int64_t tokens, int heads, int dim, int rotary, int interleaved, int inverse, int type,
                     void *y, int64_t y_token_stride, int64_t y_head_stride, void *hip_stream);

/*
 * The paged cache of keys and values in 8-bit codes (quantizer FC_QUANTIZER_SYM: signed bytes, FC_QUANTIZER_FP8: E4M3):
 *     k_cache, v_cache    bytes [pages, heads, page, dim];  page in {16, 32, 64}, dim in {64, 128, 256}
 *     k_scales, v_scales  float [pages, heads]: an element is its code's value times its page's scale
 *     page_table          int32 [sequences, table_width]: page of a sequence's tokens [i * page, (i + 1) * page)
 *     held                int32 [sequences]: tokens that the sequence holds before this step's.  Negative: the step's first -held
 *                         tokens have no place and are left out (a padded batch's empty slots: held = -1 and one token)
 *
 * fc_cache_append puts the step's tokens behind those held.  Keys turn to their positions on the way if rotary > 0 (table as for
 * fc_rotary; rotary = 0: table may be NULL).  For every page and head that receives tokens, with x the fp32 key or value and top =
 * 127 or 448, results are bit-identical to
 *     s' = max(max|x| / top, FLT_MIN, s)        s: the page's scale, only if it holds tokens of the sequence already and
 *                                                the scale is a number
 *     code' = round(code * (s / s'))            of those tokens, where s' > s
 *     code' = round(x * (1 / s'))               of the new ones; signed codes are clamped to +-127
 * with IEEE divides, each operation rounded to nearest even.  A token beyond page table or rotation table is left out.
 * x must be finite.  A page that receives tokens belongs to one sequence.  longest: no sequence gets more new tokens (1: only the
 * first one of each is appended).
 */
FC_API int fc_cache_append(const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride,
                           int64_t v_head_stride, int64_t tokens, int heads, int dim, int type, const float *table, int64_t table_rows,
                           int rotary, int interleaved, int quantizer, void *k_cache, void *v_cache, float *k_scales, float *v_scales,
                           int64_t pages, int page, const int32_t *page_table, int table_width, const int32_t *offsets,
                           const int32_t *held, int sequences, int64_t longest, void *hip_stream);

/*
 * Attention over that cache, after the step's tokens were appended (same offsets, held, page_table): query i of a sequence sees its
 * tokens t < held + i + 1,
 *     o = sum_t w_t v_t,  w = softmax over t of scale * q . k_t          (scale positive and finite)
 * q, out: [tokens, heads * group, dim]; query heads h * group ... use key/value head h.  A query that sees nothing gets zeros;
 * what the pages hold beyond the tokens that it sees has no influence, NaN codes and scales that are not finite included (a NaN among
 * the value codes of a step's tokens may make NaN of all elements of the queries that see it).  Scales are positive and finite, as the append makes
 * them; sums run over weights of up to 2^8 before they are divided, so 2^8 times the tokens' |v| together must stay within fp32.
 * queries, longest: the most new tokens, and the most tokens in all, of a sequence.  They size the launch and the workspace;
 * sequences beyond them are computed all the same, more slowly.  Entries of the page table that the context uses must be pages of
 * the cache (others are not followed; what such a sequence gets is unspecified).
 * workspace: fc_cache_attention_workspace_bytes(...) bytes, 16-byte aligned, contents unspecified; may be NULL if that is 0.
 */
FC_API size_t fc_cache_attention_workspace_bytes(int64_t tokens, int sequences, int heads, int group, int dim, int64_t queries, int64_t longest);
FC_API int fc_cache_attention(const void *q, int64_t q_token_stride, int64_t q_head_stride, int64_t tokens, int heads, int group, int dim,
                              int type, int quantizer, const void *k_cache, const void *v_cache, const float *k_scales,
                              const float *v_scales, int64_t pages, int page, const int32_t *page_table, int table_width,
                              const int32_t *offsets, const int32_t *held, int sequences, int64_t queries, int64_t longest, float scale,
                              void *out, int64_t out_token_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes,
                              void *hip_stream);

/*
 * Attention of whole prompts to themselves: query i of a sequence sees all its tokens, or causal != 0: those up to i.
 * q, out: [tokens, heads * group, dim]; k, v: [tokens, heads, dim]; dim in {64, 128}; token strides of k and v below 2^25.
 * longest: the most tokens of a sequence; it only chooses the form of the launch.  No bit of a causal row depends on later tokens,
 * infinities and NaN among them included.  bfloat16: 2^8 times the tokens' |v| together must stay within fp32.
 */
FC_API int fc_prompt_attention(const void *q, int64_t q_token_stride, int64_t q_head_stride, const void *k, int64_t k_token_stride,
                               int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, int64_t tokens,
                               int heads, int group, int dim, int type, const int32_t *offsets, int sequences, int64_t longest, int causal,
                               float scale, void *out, int64_t out_token_stride, int64_t out_head_stride, void *hip_stream);

/*
 * Attention of a prompt that is taken in pieces: the step's new tokens, whose keys and values are at hand in 16 bits, over what their
 * sequences hold in the cache and over themselves.  Query i of a sequence sees the held tokens of the cache and the new tokens j <= i; with
 * held negative none of the cache, and the first -held new tokens have no place: nothing sees them, and they see nothing.
 * q, out: [tokens, heads * group, dim]; k, v: [tokens, heads, dim], keys turned; dim in {64, 128}; token strides of k and v below 2^25.  The
 * new tokens need not be in the cache, which is only read: fc_cache_append may come before or after.  Otherwise as fc_cache_attention.
 * Products are of `type`, sums in fp32.  Weights, times the scales of their pages where the values are codes, are rounded to `type`: bfloat16
 * 8 bits; binary16 11 bits for what is less than 2^8 below the largest of 64 tokens, absolutely 2^-15 of that one at least.  Sums must fit fp32 as there.
 * bfloat16: value scales may lie as far apart as fp32 has them (values below 2^-126 may count as 0).  binary16: the value scales of a sequence, and 1 for
 * its new tokens, lie within 2^56 of each other, pages of zeros alone aside (those that fc_cache_append makes of binary16 values, and 1, within 2^43); a
 * lower one may be taken for a higher.
 * What the pages hold beyond the held tokens has no influence, and no bit of a row depends on later tokens, infinities and NaN included.
 * longest: the most tokens, held and new, of a sequence; it sizes the launch and the workspace, and sequences beyond it are computed all the same.  The
 * order of sums, and so the last bits of a row, depend on it and on the other sequences of the call; the same call gives the same bits.
 * tokens * group is below 2^31 - 1024.  out may be q where their strides are equal, and otherwise overlaps nothing that is read (the Python call refuses
 * what does; rows may lie between other rows).
 * workspace: fc_chunk_attention_workspace_bytes(...) bytes, 16-byte aligned, contents unspecified; may be NULL if that is 0.
 */
FC_API size_t fc_chunk_attention_workspace_bytes(int64_t tokens, int sequences, int heads, int group, int dim, int64_t longest);
FC_API int fc_chunk_attention(const void *q, int64_t q_token_stride, int64_t q_head_stride, const void *k, int64_t k_token_stride,
                              int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, int64_t tokens,
                              int heads, int group, int dim, int type, int quantizer, const void *k_cache, const void *v_cache,
                              const float *k_scales, const float *v_scales, int64_t pages, int page, const int32_t *page_table,
                              int table_width, const int32_t *offsets, const int32_t *held, int sequences, int64_t longest, float scale,
                              void *out, int64_t out_token_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes,
                              void *hip_stream);

/*
 * ---- The cache's pages when sequences fork, grow, end, and move together ----
 *
 * page_table, held: as above.  uses: int32 [pages], in how many rows of the table a page is named; 0 is a free page.  An entry outside
 * [0, pages) is no page.  A page that is not full of a sequence's tokens, and those reserved beyond them, are not shared but as
 * fc_pages_fork leaves them.  Everything is decided on the device, in whole numbers that do not depend on the order of execution.  Where a
 * model has a cache for each layer, tables and counts are common to them and fc_cache_copy is called for each.  Arrays that a call writes, its
 * workspace among them, overlap nothing else of it but where this says so (the Python calls refuse what does).
 *
 * fc_pages_fork makes the table of the next step: its row b is what row parents[b] of the old one holds, the first ceil(held / page)
 * entries, and -1 behind them; a parent outside [0, sequences) gives an empty row (held 0).  So rows are kept, copied (they share their
 * pages, the partly filled one included), reordered and dropped at once, and their number may change.  uses gains what the new table
 * names and loses what the old one named.  page_table_out [rows, table_width], held_out [rows]: not the old ones.
 */
FC_API int fc_pages_fork(const int32_t *page_table, const int32_t *held, int sequences, int table_width, int page, int32_t *uses, int64_t pages,
                         const int32_t *parents, int rows, int32_t *page_table_out, int32_t *held_out, void *hip_stream);

/*
 * Pages for the step's tokens (offsets, held as for fc_cache_append, before it): every slot that they go to and that has no page gets one;
 * a partly filled page that is named elsewhere too gives way to a fresh one, into which fc_cache_copy copies it: source[b] -> target[b]
 * (int32 [sequences], -1 and -1 where there is nothing to copy).  If all rows that name such a page write to it, the last one keeps it.
 * Fresh pages are the lowest-numbered free ones, handed out by row, then slot; uses follows.  Slots beyond table_width are left out.
 * lacking: int32 [1], how many free pages are missing; if that is not 0, table and uses are as they were and nothing is to be copied.  So it is,
 * with lacking 0, where offsets do not ascend from 0 or more.
 * workspace: fc_pages_reserve_workspace_bytes(pages) bytes, 16-byte aligned, contents unspecified.
 */
FC_API size_t fc_pages_reserve_workspace_bytes(int64_t pages);
FC_API int fc_pages_reserve(int32_t *page_table, const int32_t *held, const int32_t *offsets, int sequences, int table_width, int page,
                            int32_t *uses, int64_t pages, int32_t *source, int32_t *target, int32_t *lacking, void *workspace,
                            size_t workspace_bytes, void *hip_stream);

/*
 * Moves the U pages in use (uses > 0) to numbers below U: the k-th free page below U, ascending, takes the k-th used page from U on,
 * source[k] -> target[k] (int32 [pages / 2], -1 behind the last), for fc_cache_copy.  page_table_out, uses_out: table and counts
 * afterwards; the table may be written in place, the counts not.  used: int32 [1], U.  Entries that name no page in use stay.
 * workspace: fc_pages_compact_workspace_bytes(pages) bytes, 16-byte aligned, contents unspecified.
 */
FC_API size_t fc_pages_compact_workspace_bytes(int64_t pages);
FC_API int fc_pages_compact(const int32_t *page_table, int64_t sequences, int table_width, const int32_t *uses, int64_t pages,
                            int32_t *page_table_out, int32_t *uses_out, int32_t *source, int32_t *target, int32_t *used, void *workspace,
                            size_t workspace_bytes, void *hip_stream);

/*
 * Copies pages of a cache: page target[i] becomes page source[i], codes and scales of keys and values.  Pairs with a page outside
 * [0, pages) are left out.  No page is a target twice, or both a target and a source (what such a page holds is unspecified).
 */
FC_API int fc_cache_copy(void *k_cache, void *v_cache, float *k_scales, float *v_scales, int64_t pages, int heads, int page, int dim,
                         const int32_t *source, const int32_t *target, int64_t count, void *hip_stream);

/*
 * ---- The norm behind an all-reduce, with the residual's addition ----
 *
 * x, residual, sum, y: 16-bit rows [tokens, hidden], dense but for the row stride (elements, a multiple of 8), 16-byte aligned; hidden a multiple
 * of 8 up to 32768.  residual may be NULL (nothing is added), sum too (x + residual is not kept).  weight [hidden]: of weight_type, which is
 * type or FC_TYPE_F32.  eps positive and finite.  sum and y may be x or residual where their strides are equal; otherwise no result overlaps what is
 * read, or another (the Python calls refuse what does; rows may lie between other rows).
 * Results are bit-identical, except where two correctly rounded 64-bit sums of the squares differ, to
 *     h   = x + residual                          fp32;  sum = h rounded to the type
 *     d   = fp32(1 / sqrt(sum of h * h / hidden + eps))          squares, sum, divides and root in 64 bits
 *     y   = (h * d) * weight                      fp32, then rounded to the type
 * or, as fc_quantize_sym (8 bit) and fc_quantize_fp8 have them, codes [tokens, hidden] and scales [tokens, hidden / group] of y in fp32:
 *     s   = max|y| / top    over the group; if !(s >= FLT_MIN): s = 1;  top 127 or 448
 *     q   = round(y * (1 / s))                    IEEE divides, ties to even
 * group: a power of two in [32, 16384] that divides hidden, or hidden itself (one scale a token, any hidden).  quantizer: FC_QUANTIZER_SYM, _FP8.
 * Inputs that are not finite give unspecified codes.
 */
FC_API int fc_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight, int weight_type,
                       int64_t tokens, int hidden, double eps, int type, void *sum, int64_t sum_stride, void *y, int64_t y_stride,
                       void *hip_stream);
FC_API int fc_rms_norm_quantize(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight,
                                int weight_type, int64_t tokens, int hidden, double eps, int type, int group, int quantizer, void *sum,
                                int64_t sum_stride, void *codes, float *scales, void *hip_stream);

/* Static, NUL-terminated description of an FC_* code.  Host pointer, never NULL. */
FC_API const char *fc_strerror(int code);

/* Raw hipError_t of the most recent failed launch on this thread (0 if none). */
FC_API int fc_last_hip_error(void);

/* major*10000 + minor*100 + patch */
FC_API int fc_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FC_H */
