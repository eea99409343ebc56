// fc_rotary.hip -- rotary positions: the table of angles and the rotation of queries and keys.
//
// A pair (a, b) of a head's first `rotary` elements turns by the angle position * frequency_i:
//     a' = a cos - b sin,  b' = b cos + a sin            (fp32, every product and sum rounded, then one rounding to 16 bits)
// Pair i is elements (i, i + rotary / 2) or, interleaved, (2 i, 2 i + 1); the rest of the head is copied.  The inverse turns back.
// The rotation moves 4 bytes per element for 3 operations on each, so memory bounds it: a lane has 8 pairs in 128-bit accesses and
// takes them through several heads, which share the 64 bytes of table that their 8 angles need.
#include "fc_attn.hpp"

namespace fc {
namespace {

__global__ void __launch_bounds__(256) k_rotary_table(const double *__restrict__ frequencies, int64_t rows, int half, double magnitude,
                                                      float *__restrict__ table)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * half) return;
    const int64_t row = at / half;
    const int i = (int)(at - row * half);
    double s, c;
    sincos((double)row * frequencies[i], &s, &c);      // 64 bits: the angle of a far position has few correct fraction bits in 32
    table[row * 2 * half + i] = (float)(magnitude * c);
    table[row * 2 * half + half + i] = (float)(magnitude * s);
}

// HEADS heads of one token by one lane
template <bool BF16, bool INTERLEAVED, int HEADS>
__global__ void __launch_bounds__(256) k_rotary(RotaryArgs a, int units, int head_blocks)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t item = at / units;
    const int unit = (int)(at - item * units);
    const int64_t token = item / head_blocks;
    if (token >= a.tokens) return;
    const int head0 = (int)(item - token * head_blocks) * HEADS;
    const int turned = a.rotary / 16;
    const uint16_t *x = (const uint16_t *)a.x.ptr + token * a.x.token;
    uint16_t *y = (uint16_t *)a.y.ptr + token * a.y.token;

    if (unit >= turned) {                               // 8 elements that are not turned
        const int d = a.rotary + (unit - turned) * 8;
        uintx4 w[HEADS];
#pragma unroll
        for (int j = 0; j < HEADS; ++j)
            if (head0 + j < a.heads) w[j] = *(const uintx4 *)(x + (head0 + j) * a.x.head + d);
#pragma unroll
        for (int j = 0; j < HEADS; ++j)
            if (head0 + j < a.heads) *(uintx4 *)(y + (head0 + j) * a.y.head + d) = w[j];
        return;
    }
    const int half = a.rotary / 2, pair = unit * 8;
    const int d0 = INTERLEAVED ? 2 * pair : pair, d1 = INTERLEAVED ? d0 + 8 : pair + half;
    uintx4 w[HEADS][2];
#pragma unroll
    for (int j = 0; j < HEADS; ++j)
        if (head0 + j < a.heads) {
            w[j][0] = *(const uintx4 *)(x + (head0 + j) * a.x.head + d0);
            w[j][1] = *(const uintx4 *)(x + (head0 + j) * a.x.head + d1);
        }
    const int position = a.positions[token];
    float c[8], s[8];
    if (position >= 0 && position < a.table_rows) {
        const float *row = a.table + (int64_t)position * a.rotary + pair;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = row[i];
            s[i] = a.inverse ? -row[half + i] : row[half + i];
        }
    } else {                                            // there is no such angle
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
    }
#pragma unroll
    for (int j = 0; j < HEADS; ++j)
        if (head0 + j < a.heads) {
            float u[8], v[8];
            widen8<BF16>(w[j][0], u);
            widen8<BF16>(w[j][1], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float &p = INTERLEAVED ? (i < 4 ? u[2 * i] : v[2 * i - 8]) : u[i];
                float &q = INTERLEAVED ? (i < 4 ? u[2 * i + 1] : v[2 * i - 7]) : v[i];
                const float p2 = p * c[i] - q * s[i];
                q = q * c[i] + p * s[i];
                p = p2;
            }
            *(uintx4 *)(y + (head0 + j) * a.y.head + d0) = narrow8<BF16>(u);
            *(uintx4 *)(y + (head0 + j) * a.y.head + d1) = narrow8<BF16>(v);
        }
}

// any even part of a head: one pair, or one element that is not turned, per lane
template <bool BF16>
__global__ void __launch_bounds__(256) k_rotary_any(RotaryArgs a)
{
    const int half = a.rotary / 2, units = half + a.dim - a.rotary;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = at / units;
    const int unit = (int)(at - row * units);
    const int64_t token = row / a.heads;
    if (token >= a.tokens) return;
    const int head = (int)(row - token * a.heads);
    const uint16_t *x = (const uint16_t *)a.x.ptr + token * a.x.token + head * a.x.head;
    uint16_t *y = (uint16_t *)a.y.ptr + token * a.y.token + head * a.y.head;
    if (unit >= half) {
        y[unit + half] = x[unit + half];
        return;
    }
    const int d0 = a.interleaved ? 2 * unit : unit, d1 = a.interleaved ? d0 + 1 : unit + half;
    const int position = a.positions[token];
    float c = __builtin_nanf(""), s = c;
    if (position >= 0 && position < a.table_rows) {
        c = a.table[(int64_t)position * a.rotary + unit];
        s = a.table[(int64_t)position * a.rotary + half + unit];
        if (a.inverse) s = -s;
    }
    const float p = widen<BF16>(x[d0]), q = widen<BF16>(x[d1]);
    const uint32_t w = narrow2<BF16>(p * c - q * s, q * c + p * s);
    y[d0] = (uint16_t)w;
    y[d1] = (uint16_t)(w >> 16);
}

template <bool BF16, bool INTERLEAVED>
hipError_t rotary_heads(const RotaryArgs &a, hipStream_t stream)
{
    const int units = a.rotary / 16 + (a.dim - a.rotary) / 8;
    constexpr int HEADS = 4;
    const int blocks = (a.heads + HEADS - 1) / HEADS;
    const int64_t lanes = a.tokens * blocks * units;
    return launch_kernel(k_rotary<BF16, INTERLEAVED, HEADS>, dim3((uint32_t)((lanes + 255) / 256)), dim3(256), stream, a, units, blocks);
}

}  // namespace

hipError_t launch_rotary_table(const double *frequencies, int64_t rows, int rotary, double magnitude, float *table, hipStream_t stream)
{
    const int64_t lanes = rows * (rotary / 2);
    return launch_kernel(k_rotary_table, dim3((uint32_t)((lanes + 255) / 256)), dim3(256), stream, frequencies, rows, rotary / 2, magnitude, table);
}

hipError_t launch_rotary(const RotaryArgs &a, hipStream_t stream)
{
    if (a.rotary % 16 == 0) {                           // whole 128-bit accesses, and each pair's two halves in two of them
        if (a.bf16) return a.interleaved ? rotary_heads<true, true>(a, stream) : rotary_heads<true, false>(a, stream);
        return a.interleaved ? rotary_heads<false, true>(a, stream) : rotary_heads<false, false>(a, stream);
    }
    const int64_t lanes = a.tokens * a.heads * (a.dim - a.rotary / 2);
    const dim3 grid((uint32_t)((lanes + 255) / 256));
    return a.bf16 ? launch_kernel(k_rotary_any<true>, grid, dim3(256), stream, a) : launch_kernel(k_rotary_any<false>, grid, dim3(256), stream, a);
}

}  // namespace fc
