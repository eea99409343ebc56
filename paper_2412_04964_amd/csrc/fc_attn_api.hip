// fc_attn_api.hip -- the extern "C" boundary of the attention operators declared in include/fc.h: argument checks (no HIP call
// before they pass) and the choice of a launch.
#include "fc.h"

#include <float.h>

#include "fc_attn.hpp"

namespace {

constexpr int kMaxHeads = 1 << 16;
constexpr int64_t kMaxTokens = 0x7FFFFFFF;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_type(int type) { return type == FC_TYPE_F16 || type == FC_TYPE_BF16 ? FC_OK : FC_ERR_TYPE; }
int check_code(int quantizer) { return quantizer == FC_QUANTIZER_SYM || quantizer == FC_QUANTIZER_FP8 ? FC_OK : FC_ERR_TYPE; }

// 128-bit accesses: base and strides in whole units of 8 elements
int check_rows(const void *p, int64_t token_stride, int64_t head_stride)
{
    if (!p) return FC_ERR_NULL;
    return aligned16(p) && token_stride % 8 == 0 && head_stride % 8 == 0 ? FC_OK : FC_ERR_ALIGN;
}

fc::Rows rows(const void *p, int64_t token_stride, int64_t head_stride) { return {const_cast<void *>(p), token_stride, head_stride}; }

int check_heads(int heads, int64_t tokens, int sequences)
{
    if (heads < 1 || heads > kMaxHeads || tokens < 0 || tokens > kMaxTokens || sequences < 0) return FC_ERR_SHAPE;
    return tokens > 0 && sequences == 0 ? FC_ERR_SHAPE : FC_OK;
}

int check_rotary(int64_t table_rows, int rotary, int dim)
{
    return rotary >= 0 && rotary % 2 == 0 && rotary <= dim && table_rows >= 0 ? FC_OK : FC_ERR_SHAPE;
}

int check_cache(const void *k, const void *v, const float *k_scales, const float *v_scales, int64_t pages, int page, const int32_t *table,
                int table_width)
{
    if ((page != 16 && page != 32 && page != 64) || pages < 1 || pages > kMaxTokens || table_width < 1) return FC_ERR_SHAPE;
    if (!k || !v || !k_scales || !v_scales || !table) return FC_ERR_NULL;
    return aligned16(k) && aligned16(v) ? FC_OK : FC_ERR_ALIGN;
}

int result(hipError_t e) { return e == fc::kTooLarge ? FC_ERR_SHAPE : fc::hip_result(e); }

// a softmax of a finite, positive multiple of the scores: the largest one stays the largest
int check_scale(float scale) { return scale > 0.0f && scale <= FLT_MAX ? FC_OK : FC_ERR_SHAPE; }

int check_attention(int64_t tokens, int sequences, int heads, int group, int dim, int64_t queries, int64_t longest)
{
    const int rc = check_heads(heads, tokens, sequences);
    if (rc != FC_OK) return rc;
    if (group < 1 || (int64_t)heads * group > kMaxHeads || (dim != 64 && dim != 128 && dim != 256)) return FC_ERR_SHAPE;
    return queries < 1 || queries > kMaxTokens || longest < 1 || longest > kMaxTokens ? FC_ERR_SHAPE : FC_OK;
}

}  // namespace

extern "C" {

int fc_rotary_table(const double *frequencies, int64_t rows_, int rotary, double magnitude, float *table, void *hip_stream)
{
    if (rotary < 2 || rotary % 2 || rotary > 4096 || rows_ < 0 || rows_ > kMaxTokens) return FC_ERR_SHAPE;
    if (rows_ == 0) return FC_OK;
    if (!frequencies || !table) return FC_ERR_NULL;
    return result(fc::launch_rotary_table(frequencies, rows_, rotary, magnitude, table, static_cast<hipStream_t>(hip_stream)));
}

int fc_rotary(const void *x, int64_t x_token_stride, int64_t x_head_stride, const float *table, int64_t table_rows,
              const int32_t *positions, int64_t tokens, int heads, int dim, int rotary, int interleaved, int inverse, int type,
              void *y, int64_t y_token_stride, int64_t y_head_stride, void *hip_stream)
{
    int rc = check_type(type);
    if (rc != FC_OK) return rc;
    if ((rc = check_heads(heads, tokens, 1)) != FC_OK) return rc;
    if (dim < 8 || dim % 8 || dim > 4096 || rotary < 2 || (rc = check_rotary(table_rows, rotary, dim)) != FC_OK) return FC_ERR_SHAPE;
    if (tokens == 0) return FC_OK;
    if (!table || !positions) return FC_ERR_NULL;
    if ((rc = check_rows(x, x_token_stride, x_head_stride)) != FC_OK) return rc;
    if ((rc = check_rows(y, y_token_stride, y_head_stride)) != FC_OK) return rc;
    fc::RotaryArgs a;
    a.x = rows(x, x_token_stride, x_head_stride);
    a.y = rows(y, y_token_stride, y_head_stride);
    a.table = table;
    a.table_rows = table_rows;
    a.tokens = tokens;
    a.positions = positions;
    a.heads = heads;
    a.dim = dim;
    a.rotary = rotary;
    a.interleaved = interleaved != 0;
    a.inverse = inverse != 0;
    a.bf16 = type == FC_TYPE_BF16;
    return result(fc::launch_rotary(a, static_cast<hipStream_t>(hip_stream)));
}

int fc_cache_append(const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride,
                    int64_t tokens, int heads, int dim, int type, const float *table, int64_t table_rows, int rotary, int interleaved,
                    int quantizer, void *k_cache, void *v_cache, float *k_scales, float *v_scales, int64_t pages, int page,
                    const int32_t *page_table, int table_width, const int32_t *offsets, const int32_t *held, int sequences, int64_t longest,
                    void *hip_stream)
{
    int rc = check_type(type);
    if (rc != FC_OK || (rc = check_code(quantizer)) != FC_OK) return rc;
    if ((rc = check_heads(heads, tokens, sequences)) != FC_OK) return rc;
    if ((dim != 64 && dim != 128 && dim != 256) || longest < 1) return FC_ERR_SHAPE;
    if ((rc = check_rotary(table_rows, rotary, dim)) != FC_OK) return rc;
    if (tokens == 0) return FC_OK;
    if ((rc = check_cache(k_cache, v_cache, k_scales, v_scales, pages, page, page_table, table_width)) != FC_OK) return rc;
    if (!offsets || !held || (rotary && !table)) return FC_ERR_NULL;
    if ((rc = check_rows(k, k_token_stride, k_head_stride)) != FC_OK) return rc;
    if ((rc = check_rows(v, v_token_stride, v_head_stride)) != FC_OK) return rc;
    fc::AppendArgs a;
    a.k = rows(k, k_token_stride, k_head_stride);
    a.v = rows(v, v_token_stride, v_head_stride);
    a.step = {offsets, held, sequences, tokens};
    a.cache = {static_cast<uint8_t *>(k_cache), static_cast<uint8_t *>(v_cache), k_scales, v_scales, page_table, pages, page, table_width};
    a.table = table;
    a.table_rows = table_rows;
    a.longest = longest;
    a.heads = heads;
    a.dim = dim;
    a.rotary = rotary;
    a.interleaved = interleaved != 0;
    a.fp8 = quantizer == FC_QUANTIZER_FP8;
    a.bf16 = type == FC_TYPE_BF16;
    return result(fc::launch_cache_append(a, static_cast<hipStream_t>(hip_stream)));
}

size_t fc_cache_attention_workspace_bytes(int64_t tokens, int sequences, int heads, int group, int dim, int64_t queries, int64_t longest)
{
    if (check_attention(tokens, sequences, heads, group, dim, queries, longest) != FC_OK) return 0;
    fc::CacheAttentionArgs a;
    fc::cache_attention_plan(sequences, heads, group, dim, queries, longest, &a);
    return fc::cache_attention_workspace(a, tokens, sequences, heads * group, dim);
}

int fc_cache_attention(const void *q, int64_t q_token_stride, int64_t q_head_stride, int64_t tokens, int heads, int group, int dim, int type,
                       int quantizer, const void *k_cache, const void *v_cache, const float *k_scales, const float *v_scales, int64_t pages,
                       int page, const int32_t *page_table, int table_width, const int32_t *offsets, const int32_t *held, int sequences,
                       int64_t queries, int64_t longest, float scale, void *out, int64_t out_token_stride, int64_t out_head_stride,
                       void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_type(type);
    if (rc != FC_OK || (rc = check_code(quantizer)) != FC_OK) return rc;
    if ((rc = check_attention(tokens, sequences, heads, group, dim, queries, longest)) != FC_OK || (rc = check_scale(scale)) != FC_OK) return rc;
    if (tokens == 0) return FC_OK;
    if ((rc = check_cache(k_cache, v_cache, k_scales, v_scales, pages, page, page_table, table_width)) != FC_OK) return rc;
    if (!offsets || !held) return FC_ERR_NULL;
    if ((rc = check_rows(q, q_token_stride, q_head_stride)) != FC_OK) return rc;
    if ((rc = check_rows(out, out_token_stride, out_head_stride)) != FC_OK) return rc;
    fc::CacheAttentionArgs a;
    fc::cache_attention_plan(sequences, heads, group, dim, queries, longest, &a);
    // ranges are counted in 32 bits: up to this many units, whatever the arrays say
    const double units = ((double)table_width * page / 32 + 1) * heads * ((double)tokens * group / 16 + sequences);
    const int64_t rows_ = tokens * heads * group;
    if (rows_ / 16 > kMaxTokens) return FC_ERR_SHAPE;
    if (units >= 2147483648.0 || !fc::launchable((rows_ + 3) / 4, 256)) {              // or more rows than are joined
        a.workgroups = 0;
        a.splits = 1;
    }
    if (!a.workgroups) {                 // a workgroup takes every row_blocks-th block of a sequence: no more of them than are launched
        const int64_t blocks = (((int64_t)1 << 32) / 512 - 1) / ((int64_t)sequences * heads * a.splits);
        if (blocks < 1) return FC_ERR_SHAPE;
        if (a.row_blocks > blocks) a.row_blocks = (int)blocks;
    }
    const size_t need = fc::cache_attention_workspace(a, tokens, sequences, heads * group, dim);
    if (need && (!workspace || workspace_bytes < need)) return FC_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return FC_ERR_ALIGN;
    a.q = rows(q, q_token_stride, q_head_stride);
    a.out = rows(out, out_token_stride, out_head_stride);
    a.step = {offsets, held, sequences, tokens};
    a.cache = {static_cast<uint8_t *>(const_cast<void *>(k_cache)), static_cast<uint8_t *>(const_cast<void *>(v_cache)),
               const_cast<float *>(k_scales), const_cast<float *>(v_scales), page_table, pages, page, table_width};
    a.plan = static_cast<uint32_t *>(workspace);       // the partials behind it, on a 16-byte boundary
    a.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + (((size_t)sequences + 1) * sizeof(uint32_t) + 15) / 16 * 16);
    a.scale = scale;
    a.heads = heads;
    a.group = group;
    a.dim = dim;
    a.fp8 = quantizer == FC_QUANTIZER_FP8;
    a.bf16 = type == FC_TYPE_BF16;
    return result(fc::launch_cache_attention(a, static_cast<hipStream_t>(hip_stream)));
}

int fc_prompt_attention(const void *q, int64_t q_token_stride, int64_t q_head_stride, const void *k, int64_t k_token_stride,
                        int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, int heads,
                        int group, int dim, int type, const int32_t *offsets, int sequences, int64_t longest, int causal, float scale,
                        void *out, int64_t out_token_stride, int64_t out_head_stride, void *hip_stream)
{
    int rc = check_type(type);
    if (rc != FC_OK) return rc;
    if ((rc = check_attention(tokens, sequences, heads, group, dim, 1, longest)) != FC_OK) return rc;
    if (dim == 256) return FC_ERR_SHAPE;
    if ((rc = check_scale(scale)) != FC_OK) return rc;
    if (tokens == 0) return FC_OK;
    if (!offsets) return FC_ERR_NULL;
    if ((rc = check_rows(q, q_token_stride, q_head_stride)) != FC_OK) return rc;
    if ((rc = check_rows(k, k_token_stride, k_head_stride)) != FC_OK) return rc;
    if ((rc = check_rows(v, v_token_stride, v_head_stride)) != FC_OK) return rc;
    if ((rc = check_rows(out, out_token_stride, out_head_stride)) != FC_OK) return rc;
    // 32-bit offsets in a tile, and tokens of a sequence
    if (tokens > kMaxTokens - 1024) return FC_ERR_SHAPE;
    if (k_token_stride >= 1 << 25 || v_token_stride >= 1 << 25 || k_token_stride < 0 || v_token_stride < 0) return FC_ERR_SHAPE;
    fc::PromptArgs a;
    a.q = rows(q, q_token_stride, q_head_stride);
    a.k = rows(k, k_token_stride, k_head_stride);
    a.v = rows(v, v_token_stride, v_head_stride);
    a.out = rows(out, out_token_stride, out_head_stride);
    a.offsets = offsets;
    a.tokens = tokens;
    a.longest = longest;
    a.scale = scale;
    a.sequences = sequences;
    a.heads = heads;
    a.group = group;
    a.dim = dim;
    a.causal = causal != 0;
    a.bf16 = type == FC_TYPE_BF16;
    return result(fc::launch_prompt_attention(a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
