// fc_norm.hip -- root-mean-square norm behind an all-reduce: the residual's addition, the norm, and 16 bits or 8-bit codes with scales.
//
//     h = x + r,  d = fp32(1 / sqrt(sum h^2 / hidden + eps)),  y = (h d) w
//     codes: s = max|y| / top over a group (1 if that is below FLT_MIN),  code = round(y (1 / s))
// in fp32 with IEEE divides, each operation rounded to nearest even; the sum of squares, the division and the root are in 64 bits.  A
// square of an fp32 number has 48 bits, so the sum of a row is exact but for its last few bits, and d does not depend on the order but where two
// such sums lie on either side of a border between fp32 numbers: nearly one definition for all forms of the launch.
// A workgroup has a row, from its first read to the last store, in registers; wavefronts add up in LDS, once for the sum and, with scales that
// they share, once for the largest value.  Memory bounds it: 8192 rows of 8192 with a residual, 537 MB, 88 us, 6.1 TB/s; 16383 rows of 5120 into
// E4M3 with a scale a token, 587 MB, 101 to 104 us, 5.8 to 5.6 TB/s, where the two joins of a row weigh.  Few tokens are bound by the call: 8 x 8192
// 4.9 us, of which the kernel takes 3.5.
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

// A value from the lane that CTRL names: neighbours, pairs of a quad exchanged, 8 lanes mirrored, 16 lanes mirrored.  One after the other they
// bring together 2, 4, 8 and 16 lanes.
constexpr int kNeighbour = 0xB1, kPair = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;
template <int CTRL>
__device__ __forceinline__ float from_lane(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ double from_lane(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true), hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }
__device__ __forceinline__ double lane_value(double v, int lane)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane));
}

__device__ __forceinline__ double sum16(double v)
{
    v += from_lane<kNeighbour>(v);
    v += from_lane<kPair>(v);
    v += from_lane<kMirror8>(v);
    return v + from_lane<kMirror16>(v);
}
__device__ __forceinline__ double sum64(double v)
{
    v = sum16(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
// over aligned groups of `lanes`, a power of two from 4 on
__device__ __forceinline__ float max_of(float v, int lanes)
{
    v = fmaxf(v, from_lane<kNeighbour>(v));
    v = fmaxf(v, from_lane<kPair>(v));
    if (lanes >= 8) v = fmaxf(v, from_lane<kMirror8>(v));
    if (lanes >= 16) v = fmaxf(v, from_lane<kMirror16>(v));
    if (lanes == 32) v = fmaxf(v, __shfl_xor(v, 16));
    if (lanes == 64) v = fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
    return v;
}

// Lane t of a row's workgroup has its 16-byte units t, t + lanes, ... : V of them.  STREAM: rows and results are marked as used once.  F32: weights of 32 bits.
template <int V, bool BF16, int CODES, bool STREAM, bool F32>
__global__ void __launch_bounds__(1024) k_rms_norm(NormArgs a, int units)
{
    __shared__ double part[2][16];
    __shared__ float most[CODES ? 2 : 1][CODES ? 16 * V : 1];
    const int lanes = blockDim.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = lanes >> 6;
    const bool whole = CODES && a.group == a.hidden;
    const int of_group = CODES ? a.group / 8 : 1;
    const auto load = [](const uintx4 *p) {
        if constexpr (STREAM) return __builtin_nontemporal_load(p);
        else return *p;
    };
    const auto store = [](auto v, auto *p) {
        if constexpr (STREAM) __builtin_nontemporal_store(v, p);
        else *p = v;
    };
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x, turn ^= 1) {
        // all that is read is on its way at once
        constexpr bool kEarly = !(F32 && V == 4);        // (weights too, where there are registers for them)
        uintx4 x[V], r[V], w[V][F32 ? 2 : 1];
        const auto weights = [&](int i, int u) {
#pragma unroll
            for (int k = 0; k < (F32 ? 2 : 1); ++k) w[i][k] = ((const uintx4 *)a.weight)[(F32 ? 2 : 1) * u + k];
        };
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int u = i * lanes + threadIdx.x;
            x[i] = r[i] = uintx4{0, 0, 0, 0};
            if (u < units) {
                x[i] = load((const uintx4 *)((const uint16_t *)a.x + row * a.x_row + 8 * u));
                if (a.residual) r[i] = load((const uintx4 *)((const uint16_t *)a.residual + row * a.residual_row + 8 * u));
                if constexpr (kEarly) weights(i, u);
            }
        }
        float h[V][8];
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float f[8];
            widen8<BF16>(x[i], h[i]);
            widen8<BF16>(r[i], f);
            if (a.residual)
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] += f[j];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int u = i * lanes + threadIdx.x;
            if (a.sum && u < units) store(narrow8<BF16>(h[i]), (uintx4 *)((uint16_t *)a.sum + row * a.sum_row + 8 * u));
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)h[i][j], (double)h[i][j], sum);
        }
        sum = sum64(sum);
        if (waves > 1) {
            if (lane == 0) part[turn][wave] = sum;
            __syncthreads();
            sum = sum16((lane & 15) < waves ? part[turn][lane & 15] : 0.0);
        }
        const float d = (float)(1.0 / __builtin_sqrt(sum / a.hidden + a.eps));
        float m[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int u = i * lanes + threadIdx.x;
            m[i] = 0.0f;
            if (u < units) {
                float f[8];
                if constexpr (!kEarly) weights(i, u);
                if constexpr (F32)
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = __builtin_bit_cast(float, (uint32_t)w[i][j / 4][j % 4]);
                else widen8<BF16>(w[i][0], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * d * f[j];
                if constexpr (CODES == 0) store(narrow8<BF16>(h[i]), (uintx4 *)((uint16_t *)a.y + row * a.y_row + 8 * u));
                else m[i] = largest(h[i]);
            }
        }
        if constexpr (CODES != 0) {
            const int near = whole || of_group > 64 ? 64 : of_group;       // lanes of a wavefront that share a scale
#pragma unroll
            for (int i = 0; i < V; ++i)
                m[i] = max_of(m[i], near);
            if (near == 64 && (whole || of_group > 64)) {
                // and wavefronts: 64 units each, in the order of the row
                if (lane == 0)
#pragma unroll
                    for (int i = 0; i < V; ++i) most[turn][i * waves + wave] = m[i];
                __syncthreads();
                // (64 pieces at most: lane k has the k-th of the unit's group)
                const int pieces = whole ? waves * V : of_group / 64;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int first = whole ? 0 : (i * waves + wave) / pieces * pieces;
                    if (i == 0 || !whole) m[i] = max_of(lane < pieces ? most[turn][first + lane] : 0.0f, 64);
                    else m[i] = m[0];
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
                    store(uintx2{pack4<fp8>(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), pack4<fp8>(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)},
                          (uintx2 *)((uint8_t *)a.y + row * a.hidden + 8 * u));
                    if (whole ? u == 0 : u % of_group == 0) a.scales[row * (a.hidden / a.group) + u / of_group] = s;
                }
            }
        }
    }
}

template <bool BF16, int CODES, bool F32>
hipError_t norm(const NormArgs &a, hipStream_t stream)
{
    // Units of a lane.  Few rows: one, which is the shortest way through a row.  Many: two and four, which leave more rows' reads on a compute unit
    // at once.  us for 1 / 2 / 4, residual, 2^26 elements: 8192 x 8192 into 16 bits 87.6 / 87.3 / 90.9, into codes of a token's scale 90.6 / 81.4 / 81.3;
    // 13107 x 5120 codes 108.9 / 82.7 / 84.0; 4096 x 16384 codes (1024 lanes have no less than two) 101.1 with two, 83.2 with four; 131072 x 512 codes
    // 82.8 / 94.3 / 139.6.
    const int units = a.hidden / 8;
    int v = a.tokens <= 1024 || units <= 64 ? 1 : units <= 1024 ? 2 : 4;
    while ((units + v - 1) / v > 1024) v *= 2;
    const int lanes = ((units + v - 1) / v + 63) / 64 * 64;
    const int64_t grid = a.tokens < 1 << 20 ? a.tokens : 1 << 20;
    const bool once = beyond_cache((double)a.tokens * a.hidden * 4);
    const auto go = [&](auto *kernel) { return launch_many(kernel, grid, lanes, stream, a, units); };
    if (once) return v == 1 ? go(k_rms_norm<1, BF16, CODES, true, F32>) : v == 2 ? go(k_rms_norm<2, BF16, CODES, true, F32>) : go(k_rms_norm<4, BF16, CODES, true, F32>);
    return v == 1 ? go(k_rms_norm<1, BF16, CODES, false, F32>) : v == 2 ? go(k_rms_norm<2, BF16, CODES, false, F32>) : go(k_rms_norm<4, BF16, CODES, false, F32>);
}

template <bool BF16>
hipError_t norm_of(const NormArgs &a, hipStream_t stream)
{
    switch (a.codes) {
    case kSigned: return a.weight_f32 ? norm<BF16, kSigned, true>(a, stream) : norm<BF16, kSigned, false>(a, stream);
    case kE4M3: return a.weight_f32 ? norm<BF16, kE4M3, true>(a, stream) : norm<BF16, kE4M3, false>(a, stream);
    default: return a.weight_f32 ? norm<BF16, kWide16, true>(a, stream) : norm<BF16, kWide16, false>(a, stream);
    }
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs &a, hipStream_t stream) { return a.bf16 ? norm_of<true>(a, stream) : norm_of<false>(a, stream); }

}  // namespace fc
