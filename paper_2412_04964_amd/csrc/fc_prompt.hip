// fc_prompt.hip -- attention over whole prompts, packed one behind the other.
//
// Query i of a sequence sees all its tokens, or (causal) those up to i:  o = sum_t softmax_t(scale q . k_t) v_t.
// A wavefront has 32 queries of one head.  It forms the transposed score S^T = K Q^T with 32 x 32 x 16 matrix instructions, which
// leaves a lane with weights of the very tokens that it needs as operand of O^T = V^T P^T, and keeps the running maximum and sum of
// its column: one pass over K and V.  Matrix instructions and the exponentials between them bound it.
#include "fc_attn.hpp"

namespace fc {
namespace {

constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;      // queries of a workgroup

template <int DIM, bool BF16>
__global__ void __launch_bounds__(64 * kWaves) k_prompt_attention(PromptArgs a)
{
    constexpr int kSteps = DIM / 16, kOut = DIM / 32;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, side = lane >> 5;
    const int query_heads = a.heads * a.group;
    const int head = blockIdx.x % query_heads, kv_head = head / a.group;
    const int64_t unit = blockIdx.x / query_heads;
    const int b = find_sequence(a.offsets, a.sequences, 7, 1, unit);
    const int64_t off = a.offsets[b];
    int64_t n = (int64_t)a.offsets[b + 1] - off;
    if (off < 0 || n <= 0 || off + n > a.tokens) return;
    const int64_t row0 = (unit - ((off >> 7) + b)) * kRows + wave * 32;
    if (row0 >= n) return;
    const int64_t row = row0 + col, last = n - 1;
    const int64_t read_row = row < n ? row : last;

    uintx4 qf[kSteps];
    const uint16_t *q = (const uint16_t *)a.q.ptr + (off + read_row) * a.q.token + head * a.q.head + side * 8;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) qf[j] = *(const uintx4 *)(q + 16 * j);

    const uint16_t *k = (const uint16_t *)a.k.ptr + off * a.k.token + kv_head * a.k.head;
    const uint16_t *v = (const uint16_t *)a.v.ptr + off * a.v.token + kv_head * a.v.head;
    const float factor = a.scale * 1.4426950408889634f;

    floatx16 acc[kOut];
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[o][r] = 0.0f;
    float top = -FLT_MAX, total = 0.0f;
    const int64_t end = a.causal ? (row0 + 32 < n ? row0 + 32 : n) : n;
    for (int64_t t0 = 0; t0 < end; t0 += 32) {
        floatx16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.0f;
        const int64_t kt = t0 + col < n ? t0 + col : last;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) s = mma32<BF16>(*(const uintx4 *)(k + kt * a.k.token + 16 * j + side * 8), qf[j], s);
        float most = -FLT_MAX;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t t = t0 + 8 * (r / 4) + 4 * side + r % 4;
            s[r] = t < n && (!a.causal || t <= row) ? s[r] * factor : -__builtin_inff();
            most = fmaxf(most, s[r]);
        }
        most = fmaxf(most, __shfl_xor(most, 32));
        const float now = fmaxf(top, most), shrink = __builtin_amdgcn_exp2f(top - now);
        top = now;
        total *= shrink;
#pragma unroll
        for (int o = 0; o < kOut; ++o) acc[o] *= shrink;
        uintx4 pf[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] - top);
            total += s[r];
        }
#pragma unroll
        for (int r = 0; r < 16; r += 2) pf[r / 8][r % 8 / 2] = narrow2<BF16>(s[r], s[r + 1]);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                uintx4 vf;
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const int64_t t = t0 + 16 * m + 8 * (i / 4) + 4 * side + i % 4;
                    const uint32_t lo = v[(t < n ? t : last) * a.v.token + o * 32 + col], hi = v[(t + 1 < n ? t + 1 : last) * a.v.token + o * 32 + col];
                    vf[i / 2] = (t < n ? lo : 0) | (t + 1 < n ? hi << 16 : 0);
                }
                acc[o] = mma32<BF16>(vf, pf[m], acc[o]);
            }
    }
    total += __shfl_xor(total, 32);
    if (row >= n) return;
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    uint16_t *y = (uint16_t *)a.out.ptr + (off + row) * a.out.token + head * a.out.head;
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *(uintx2 *)(y + o * 32 + 2 * r + 4 * side) = uintx2{narrow2<BF16>(acc[o][r] * inv, acc[o][r + 1] * inv), narrow2<BF16>(acc[o][r + 2] * inv, acc[o][r + 3] * inv)};
}

template <bool BF16>
hipError_t prompt(const PromptArgs &a, hipStream_t stream)
{
    const int64_t units = (a.tokens >> 7) + a.sequences;
    const dim3 grid((uint32_t)(units * a.heads * a.group));
    return a.dim == 64 ? launch_kernel(k_prompt_attention<64, BF16>, grid, dim3(64 * kWaves), stream, a)
                       : launch_kernel(k_prompt_attention<128, BF16>, grid, dim3(64 * kWaves), stream, a);
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs &a, hipStream_t stream) { return a.bf16 ? prompt<true>(a, stream) : prompt<false>(a, stream); }

}  // namespace fc
