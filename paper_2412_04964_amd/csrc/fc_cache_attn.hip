// fc_cache_attn.hip -- attention over the paged cache of 8-bit codes.
//
// Query i of a sequence that held L tokens before the step sees the tokens t < L + i + 1:
//     w_t = exp(scale q . (sk ck_t) - max),  o = sum w_t sv cv_t / sum w_t
// with the scales sk, sv of t's page and head.  Codes of either kind are exact in binary16, so the products run on codes: sk multiplies
// the score and sv the weight.  Rows of the matrix products are the queries of a sequence times the query heads that share a
// key/value head (16 rows); the transposed score S^T = K Q^T leaves a lane with the weights of the tokens that it needs again as the
// operand of O^T = V^T P^T, so nothing goes through LDS before the end.
//   Queries are scaled by a power of two per row so that they fit binary16 (bfloat16's 8 bits stay exact over 2^28 below a row's largest).
//   Weights are rounded to binary16 as p sv / ref, where ref is the row's largest p sv so far or less by kMost: 11 bits.
//   The running maximum is raised only when a score passes it by kSlack, and ref by kMost: the sums carry the same factors either way.
// The context is split over workgroups and their wavefronts, each with its own maximum and sums; wavefronts are joined in LDS,
// workgroups by a second kernel through the workspace.  Memory bounds it: 2 bytes per token, head and element against one multiply-add
// for each query head.
#include "fc_attn.hpp"

namespace fc {
namespace {

constexpr int kWaves = 4;
constexpr float kSlack = 8.0f;          // in powers of two
constexpr float kMost = 256.0f, kLeast = 1e-30f;
constexpr int kTile = 16;               // tokens of a matrix instruction; a page holds whole tiles

// 4 codes of a word -> binary16
template <bool FP8>
__device__ __forceinline__ uintx2 halves(uint32_t w)
{
    if constexpr (FP8) {
        return uintx2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true))};
    } else {
        // code + 128 under the exponent of 1024 is 1152 + code
        const uint32_t u = w ^ 0x80808080u;
        const half2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
        const half2 lo = __builtin_bit_cast(half2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
        const half2 hi = __builtin_bit_cast(half2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
        return uintx2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    }
}

// byte i of four words -> word i
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4])
{
    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    out[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
}

__device__ __forceinline__ float lane_f(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[1]) { w[0] = *(const uint32_t *)p; }
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[2])
{
    const uintx2 x = *(const uintx2 *)p;
    w[0] = x[0];
    w[1] = x[1];
}
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[4])
{
    const uintx4 x = *(const uintx4 *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
}

// over the four lanes that share l % 16
__device__ __forceinline__ float max4(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float sum4(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }

// pieces that a sequence of `tiles` tiles is cut into, of at most `splits`: no piece below kWaves tiles' pairs
__host__ __device__ __forceinline__ int pieces_of(int64_t tiles, int splits)
{
    const int64_t most = (tiles + 2 * kWaves - 1) / (2 * kWaves);
    return most < 1 ? 1 : most < splits ? (int)most : splits;
}

template <int DIM, bool FP8, bool BF16>
__global__ void __launch_bounds__(64 * kWaves) k_cache_attention(CacheAttentionArgs a, int page_shift)
{
    constexpr int kSteps = DIM / 32;                    // matrix instructions over the head's elements
    constexpr int kOut = DIM / 16;                      // result tiles
    constexpr int kWords = DIM / 64;                    // 4-byte words of V that a lane has of a token
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    uint32_t at = blockIdx.x;
    const int piece = at % a.splits;
    at /= a.splits;
    const int head = at % a.heads;
    at /= a.heads;
    const int row_block = at % a.row_blocks, b = at / a.row_blocks;

    const int64_t off = a.step.offsets[b], held = a.step.held[b];
    int64_t queries = (int64_t)a.step.offsets[b + 1] - off;
    if (off < 0 || queries < 0 || off + queries > a.step.tokens) return;
    const int64_t room = (int64_t)a.cache.table_width << page_shift;
    const int64_t context = held + queries < room ? held + queries : room;     // may be negative
    const int64_t tiles = context > 0 ? (context + kTile - 1) / kTile : 0;
    const int pieces = pieces_of(tiles, a.splits);
    if (piece >= pieces) return;
    // this workgroup's tiles, in pairs, then this wavefront's
    const int64_t pairs = (tiles + 1) / 2;
    const int64_t pair0 = pairs * piece / pieces, pair1 = pairs * (piece + 1) / pieces;
    const int64_t begin = 2 * (pair0 + (pair1 - pair0) * wave / kWaves), stop = 2 * (pair0 + (pair1 - pair0) * (wave + 1) / kWaves);
    const int64_t end_token = stop * kTile < context ? stop * kTile : context;  // of this wavefront

    __shared__ float join[kWaves][16][DIM + 4];
    __shared__ float join_max[kWaves][16], join_sum[kWaves][16];

    const int64_t rows = queries * a.group;
    for (int64_t row0 = (int64_t)row_block * 16; row0 < rows; row0 += (int64_t)a.row_blocks * 16) {
        const int64_t row = row0 + col;
        const int64_t query = row < rows ? row / a.group : queries - 1;
        const int64_t token = off + query;
        const int query_head = head * a.group + (int)(row - query * a.group);
        int64_t sees = held + query + 1;
        if (sees > end_token) sees = end_token;
        if (row >= rows) sees = 0;
        const int64_t all_see = held + row0 / a.group + 1 < end_token ? held + row0 / a.group + 1 : end_token;    // what every row of the block sees

        // the row's elements quad * DIM / 4 .., scaled into binary16
        uintx4 qf[kSteps];
        float factor;
        {
            float f[kSteps][8], most = 0.0f;
            const uint16_t *q = (const uint16_t *)a.q.ptr + token * a.q.token + query_head * a.q.head + quad * (DIM / 4);
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                if (row < rows) widen8<BF16>(*(const uintx4 *)(q + 8 * j), f[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (row >= rows) f[j][i] = 0.0f;
                    most = fmaxf(most, fabsf(f[j][i]));
                }
            }
            factor = 1.0f;
            if constexpr (BF16) {
                most = max4(most);
                int e = 0;
                if (most > 0.0f && most < __builtin_inff()) e = 14 - __builtin_amdgcn_frexp_expf(most);      // most * 2^e in [2^13, 2^14)
                factor = __builtin_amdgcn_ldexpf(1.0f, -e);
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[j][i] = __builtin_amdgcn_ldexpf(f[j][i], e);
            }
#pragma unroll
            for (int j = 0; j < kSteps; ++j) qf[j] = narrow8<false>(f[j]);
            factor *= a.scale * 1.4426950408889634f;    // scores in powers of two
        }

        floatx4 acc[kOut];
#pragma unroll
        for (int i = 0; i < kOut; ++i) acc[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        float top = -FLT_MAX, total = 0.0f, ref = kLeast, inv_ref = 1.0f / kLeast;
        // the sums' unit: they are acc * was, and are acc * ref afterwards
        const auto rebase = [&](float was, float least) {
            ref = fmaxf(was, least);
            inv_ref = 1.0f / ref;
            const float change = was * inv_ref;
#pragma unroll
            for (int o = 0; o < kOut; ++o) acc[o] *= change;
        };

        for (int64_t base = begin; base < stop; base += 64) {
            // page and scales of the next 64 tiles, one a lane
            int page = 0;
            float ks = 0.0f, vs = 0.0f;
            {
                const int64_t index = (base + lane) * kTile >> page_shift;
                if (base + lane < stop && (base + lane) * kTile < context) {
                    const int id = a.cache.table[(int64_t)b * a.cache.table_width + index];
                    if (id >= 0 && id < a.cache.pages) {
                        page = id;
                        ks = a.cache.k_scales[(int64_t)id * a.heads + head];
                        vs = a.cache.v_scales[(int64_t)id * a.heads + head];
                    }
                }
            }
            const int n = stop - base < 64 ? (int)(stop - base) : 64;
            for (int i = 0; i < n; i += 2) {
                const int64_t first = (base + i) * kTile;
                if (first >= end_token) break;
                uintx4 kf[2][kSteps / 2];
                uint32_t vf[2][4][kWords];
                float ksc[2], vsc[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int64_t slot = ((base + i + t) * kTile) & ((1 << page_shift) - 1);
                    const int64_t place = ((((int64_t)__builtin_amdgcn_readlane(page, i + t) * a.heads + head) << page_shift) + slot) * DIM;
                    ksc[t] = lane_f(ks, i + t);
                    vsc[t] = lane_f(vs, i + t);
                    const uint8_t *k = a.cache.k + place + col * DIM + quad * (DIM / 4);
#pragma unroll
                    for (int j = 0; j < kSteps / 2; ++j) kf[t][j] = *(const uintx4 *)(k + 16 * j);
                    const uint8_t *v = a.cache.v + place + quad * 4 * DIM + col * (DIM / 16);
#pragma unroll
                    for (int r = 0; r < 4; ++r) load_words(v + r * DIM, vf[t][r]);
                }
                floatx4 s[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    s[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) {
                        const uintx2 lo = halves<FP8>(kf[t][j / 2][(j & 1) * 2]), hi = halves<FP8>(kf[t][j / 2][(j & 1) * 2 + 1]);
                        s[t] = mma16(uintx4{lo[0], lo[1], hi[0], hi[1]}, qf[j], s[t]);
                    }
                    const float scale = factor * ksc[t];
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[t][r] *= scale;
                }
                if (first + 2 * kTile > all_see) {
                    // tokens that a row does not see: whatever the cache holds there
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int64_t tok = first + t * kTile + quad * 4 + r;
                            if (tok >= sees) s[t][r] = -__builtin_inff();
                            if (tok >= end_token)
#pragma unroll
                                for (int w = 0; w < kWords; ++w) vf[t][r][w] = 0;
                        }
                }
                float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
                if (__any(most > top + kSlack)) {
                    const float now = fmaxf(top, max4(most)), shrink = __builtin_amdgcn_exp2f(top - now);
                    top = now;
                    total *= shrink;
                    rebase(ref * shrink, kLeast);
                }
                float p[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    p[r] = __builtin_amdgcn_exp2f(s[r / 4][r % 4] - top);
                    total += p[r];
                    p[r] *= vsc[r / 4];
                }
                const float weight = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
                if (__any(weight * inv_ref > kMost)) rebase(ref, max4(weight));
                uintx4 pf;
#pragma unroll
                for (int r = 0; r < 4; ++r) pf[r] = narrow2<false>(p[2 * r] * inv_ref, p[2 * r + 1] * inv_ref);
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    uint32_t x[2][4];
#pragma unroll
                    for (int t = 0; t < 2; ++t) transpose4(vf[t][0][w], vf[t][1][w], vf[t][2][w], vf[t][3][w], x[t]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uintx2 lo = halves<FP8>(x[0][e]), hi = halves<FP8>(x[1][e]);
                        acc[w * 4 + e] = mma16(uintx4{lo[0], lo[1], hi[0], hi[1]}, pf, acc[w * 4 + e]);
                    }
                }
            }
        }
        total = sum4(total);

        // join the wavefronts
        if (quad == 0) {
            join_max[wave][col] = top;
            join_sum[wave][col] = total;
        }
        __syncthreads();
        float best = join_max[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) best = fmaxf(best, join_max[w][col]);
        const float mine = __builtin_amdgcn_exp2f(top - best) * ref;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int o = 0; o < kOut; ++o) join[wave][col][(quad * 4 + r) * kOut + o] = acc[o][r] * mine;
        __syncthreads();
        // 16 lanes a row, each DIM / 16 neighbouring elements
        const int out_row = threadIdx.x >> 4, d = (threadIdx.x & 15) * kOut;
        float best_row = join_max[0][out_row], sum_row = 0.0f, o[kOut];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) best_row = fmaxf(best_row, join_max[w][out_row]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum_row += join_sum[w][out_row] * __builtin_amdgcn_exp2f(join_max[w][out_row] - best_row);
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            o[i] = join[0][out_row][d + i];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) o[i] += join[w][out_row][d + i];
        }
        if (row0 + out_row < rows) {
            const int64_t q = (row0 + out_row) / a.group;
            const int h = head * a.group + (int)(row0 + out_row - q * a.group);
            if (pieces == 1) {
                const float inv = sum_row == 0.0f ? 0.0f : 1.0f / sum_row;      // a row that sees nothing is zero
                uint16_t *y = (uint16_t *)a.out.ptr + (off + q) * a.out.token + h * a.out.head + d;
#pragma unroll
                for (int i = 0; i < kOut; i += 2) *(uint32_t *)(y + i) = narrow2<BF16>(o[i] * inv, o[i + 1] * inv);
            } else {
                const int64_t at_row = ((off + q) * a.heads * a.group + h) * a.splits + piece;
                float *y = a.partial + at_row * DIM + d;
#pragma unroll
                for (int i = 0; i < kOut; i += 4) *(floatx4 *)(y + i) = floatx4{o[i], o[i + 1], o[i + 2], o[i + 3]};
                if ((threadIdx.x & 15) == 0) {
                    float *m = a.partial + (int64_t)a.step.tokens * a.heads * a.group * a.splits * DIM + at_row * 2;
                    m[0] = best_row;
                    m[1] = sum_row;
                }
            }
        }
        __syncthreads();
    }
}

// joins the pieces of a row: DIM / 4 lanes, 4 elements each
template <int DIM, bool BF16>
__global__ void __launch_bounds__(256) k_cache_attention_join(CacheAttentionArgs a, int page_shift)
{
    constexpr int kLanes = DIM / 4;
    const int64_t row = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
    const int d = threadIdx.x % kLanes * 4, query_heads = a.heads * a.group;
    if (row >= a.step.tokens * query_heads) return;
    const int64_t token = row / query_heads;
    const int head = (int)(row - token * query_heads);
    const int b = find_sequence(a.step.offsets, a.step.sequences, 0, 0, token);
    const int64_t off = a.step.offsets[b], next = a.step.offsets[b + 1], room = (int64_t)a.cache.table_width << page_shift;
    if (token < off || token >= next || next > a.step.tokens) return;
    int64_t context = a.step.held[b] + (next - off);
    if (context > room) context = room;
    const int pieces = pieces_of(context > 0 ? (context + kTile - 1) / kTile : 0, a.splits);
    if (pieces == 1) return;                            // written already
    const float *o = a.partial + row * a.splits * DIM + d;
    const float *m = a.partial + (int64_t)a.step.tokens * query_heads * a.splits * DIM + row * a.splits * 2;
    float best = -FLT_MAX, sum = 0.0f;
    floatx4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < pieces; ++p) best = fmaxf(best, m[2 * p]);
    for (int p = 0; p < pieces; ++p) {
        const float w = __builtin_amdgcn_exp2f(m[2 * p] - best);
        sum += w * m[2 * p + 1];
        x += *(const floatx4 *)(o + (int64_t)p * DIM) * w;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t *y = (uint16_t *)a.out.ptr + token * a.out.token + head * a.out.head + d;
    *(uintx2 *)y = uintx2{narrow2<BF16>(x[0] * inv, x[1] * inv), narrow2<BF16>(x[2] * inv, x[3] * inv)};
}

template <int DIM, bool BF16>
hipError_t attend(const CacheAttentionArgs &a, hipStream_t stream)
{
    const int shift = log2_int(a.cache.page);
    const dim3 grid((uint32_t)((int64_t)a.step.sequences * a.row_blocks * a.heads * a.splits));
    const hipError_t e = a.fp8 ? launch_kernel(k_cache_attention<DIM, true, BF16>, grid, dim3(64 * kWaves), stream, a, shift)
                               : launch_kernel(k_cache_attention<DIM, false, BF16>, grid, dim3(64 * kWaves), stream, a, shift);
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t rows = a.step.tokens * a.heads * a.group, per = 256 / (DIM / 4);
    return launch_kernel(k_cache_attention_join<DIM, BF16>, dim3((uint32_t)((rows + per - 1) / per)), dim3(256), stream, a, shift);
}

}  // namespace

void cache_attention_plan(int sequences, int heads, int group, int64_t queries, int64_t longest, int *splits, int *row_blocks)
{
    const int64_t blocks = (queries * group + 15) / 16;
    *row_blocks = blocks < 1 ? 1 : blocks > 4096 ? 4096 : (int)blocks;
    const int64_t groups = (int64_t)sequences * heads * *row_blocks;
    const int64_t want = groups ? 1024 / groups : 1, most = pieces_of((longest + kTile - 1) / kTile, 64);
    *splits = (int)(want < 1 ? 1 : want < most ? want : most);
}

hipError_t launch_cache_attention(const CacheAttentionArgs &a, hipStream_t stream)
{
    switch (a.dim) {
    case 64: return a.bf16 ? attend<64, true>(a, stream) : attend<64, false>(a, stream);
    case 128: return a.bf16 ? attend<128, true>(a, stream) : attend<128, false>(a, stream);
    default: return a.bf16 ? attend<256, true>(a, stream) : attend<256, false>(a, stream);
    }
}

}  // namespace fc
