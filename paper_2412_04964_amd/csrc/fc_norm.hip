// fc_norm.hip -- root-mean-square norm behind an all-reduce: the residual's addition, the norm, and 16 bits or 8-bit codes with scales.
//
//     h = x + r,  d = fp32(1 / sqrt(sum h^2 / hidden + eps)),  y = (h d) w
//     codes: s = max|y| / top over a group (1 if that is below FLT_MIN),  code = round(y (1 / s))
// in fp32 with IEEE divides, each operation rounded to nearest even; the sum of squares, the division and the root are in 64 bits.  A
// square of an fp32 number has 48 bits, so the sum of a row is exact but for its last few bits and d does not depend on the order: one
// definition for all forms of the launch, and codes next to a border are the same in each.
// A workgroup has a row, from its first read to the last store, in registers.
#include "fc_attn.hpp"

namespace fc {
namespace {

__device__ __forceinline__ float largest(const float (&y)[8])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(y[i]));
    return m;
}

// Lane t of a row's workgroup has its 16-byte units t, t + lanes, ... : V of them
template <int V, bool BF16, int CODES>
__global__ void __launch_bounds__(1024) k_rms_norm(NormArgs a, int units)
{
    __shared__ double part[2][16];
    __shared__ float most[CODES ? 2 : 1][CODES ? 16 * V : 1];
    const int lanes = blockDim.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = lanes >> 6;
    const bool whole = CODES && a.group == a.hidden;
    const int of_group = CODES ? a.group / 8 : 1;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x, turn ^= 1) {
        const uint16_t *const x = (const uint16_t *)a.x + row * a.x_row, *const r = (const uint16_t *)a.residual + row * a.residual_row;
        float h[V][8];
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int u = i * lanes + threadIdx.x;
            if (u < units) {
                widen8<BF16>(*(const uintx4 *)(x + 8 * u), h[i]);
                if (a.residual) {
                    float f[8];
                    widen8<BF16>(*(const uintx4 *)(r + 8 * u), f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[i][j] += f[j];
                }
                if (a.sum) *(uintx4 *)((uint16_t *)a.sum + row * a.sum_row + 8 * u) = narrow8<BF16>(h[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)h[i][j], (double)h[i][j], sum);
            }
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        if (lane == 0) part[turn][wave] = sum;
        __syncthreads();
        sum = part[turn][0];
        for (int w = 1; w < waves; ++w) sum += part[turn][w];
        const float d = (float)(1.0 / __builtin_sqrt(sum / a.hidden + a.eps));
        float m[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int u = i * lanes + threadIdx.x;
            m[i] = 0.0f;
            if (u < units) {
                float w[8];
                if (a.weight_f32) {
                    const floatx4 lo = *(const floatx4 *)((const float *)a.weight + 8 * u), hi = *(const floatx4 *)((const float *)a.weight + 8 * u + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        w[j] = lo[j];
                        w[4 + j] = hi[j];
                    }
                } else {
                    widen8<BF16>(*(const uintx4 *)((const uint16_t *)a.weight + 8 * u), w);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * d * w[j];
                if constexpr (CODES == 0) *(uintx4 *)((uint16_t *)a.y + row * a.y_row + 8 * u) = narrow8<BF16>(h[i]);
                else m[i] = largest(h[i]);
            }
        }
        if constexpr (CODES != 0) {
            const int near = whole || of_group > 64 ? 64 : of_group;       // lanes of a wavefront that share a scale
#pragma unroll
            for (int i = 0; i < V; ++i)
                for (int k = 1; k < near; k <<= 1) m[i] = fmaxf(m[i], __shfl_xor(m[i], k));
            if (near == 64) {
                // and wavefronts: 64 units each, in the order of the row
                if (lane == 0)
#pragma unroll
                    for (int i = 0; i < V; ++i) most[turn][i * waves + wave] = m[i];
                __syncthreads();
                const int pieces = whole ? waves * V : of_group / 64;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int first = whole ? 0 : (i * waves + wave) / pieces * pieces;
                    for (int k = 0; k < pieces; ++k) m[i] = fmaxf(m[i], most[turn][first + k]);
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int u = i * lanes + threadIdx.x;
                if (u < units) {
                    constexpr bool fp8 = CODES == kE4M3;
                    float s = m[i] / kTop<fp8>;
                    if (!(s >= FLT_MIN)) s = 1.0f;
                    const float inv = 1.0f / s;
                    const float(&y)[8] = h[i];
                    *(uintx2 *)((uint8_t *)a.y + row * a.hidden + 8 * u) = uintx2{pack4<fp8>(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                                                                                  pack4<fp8>(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
                    if (whole ? u == 0 : u % of_group == 0) a.scales[row * (a.hidden / a.group) + u / of_group] = s;
                }
            }
        }
    }
}

template <bool BF16, int CODES>
hipError_t norm(const NormArgs &a, hipStream_t stream)
{
    const int units = a.hidden / 8;
    int v = 1;
    while ((units + v - 1) / v > 1024) v *= 2;
    const int lanes = ((units + v - 1) / v + 63) / 64 * 64;
    const int64_t grid = a.tokens < 1 << 20 ? a.tokens : 1 << 20;
    const auto go = [&](auto *kernel) { return launch_many(kernel, grid, lanes, stream, a, units); };
    return v == 1 ? go(k_rms_norm<1, BF16, CODES>) : v == 2 ? go(k_rms_norm<2, BF16, CODES>) : go(k_rms_norm<4, BF16, CODES>);
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs &a, hipStream_t stream)
{
    switch (a.codes) {
    case kSigned: return a.bf16 ? norm<true, kSigned>(a, stream) : norm<false, kSigned>(a, stream);
    case kE4M3: return a.bf16 ? norm<true, kE4M3>(a, stream) : norm<false, kE4M3>(a, stream);
    default: return a.bf16 ? norm<true, kWide16>(a, stream) : norm<false, kWide16>(a, stream);
    }
}

}  // namespace fc
