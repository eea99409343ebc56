// fc_rotary.hip -- rotary positions: the table of angles and the rotation of queries and keys.
//
// A pair (a, b) of a head's first `rotary` elements turns by the angle position * frequency_i:
//     a' = a cos - b sin,  b' = b cos + a sin            (fp32, every product and sum rounded, then one rounding to 16 bits)
// Pair i is elements (i, i + rotary / 2) or, interleaved, (2 i, 2 i + 1); the rest of the head is copied.  The inverse turns back.
// The rotation moves 4 bytes per element for 3 operations on each, so memory bounds it: 6.2 TB/s on 16383 tokens of 80 heads of 128, what a
// copy reaches here.  The table adds little: the heads of a token follow each other in a workgroup and find it in the nearest cache.
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

// 16 elements of one head by one lane: two pieces of 8, each with a neighbouring lane's on both sides so that every access of a wavefront
// is of whole lines.  Half layout: the halves of 8 pairs, or 8 + 8 elements that are not turned; interleaved: any two pieces do, the
// two halves of the head.  Every lane loads and stores alike, so that a wavefront with both kinds does not do either twice.
// STREAM: x is marked as read once.
template <bool BF16, bool INTERLEAVED, bool STREAM>
__global__ void __launch_bounds__(256) k_rotary(RotaryArgs a, uint32_t units)
{
    const uint32_t at = blockIdx.x * 256 + threadIdx.x;
    const uint32_t item = at / units, d = (at - item * units) * 8;
    const uint32_t token = item / (uint32_t)a.heads;
    if (token >= a.tokens) return;
    const int head = (int)(item - token * a.heads), half = a.rotary / 2;
    const uint16_t *x = (const uint16_t *)a.x.ptr + token * a.x.token + head * a.x.head;
    uint16_t *y = (uint16_t *)a.y.ptr + token * a.y.token + head * a.y.head;
    const int d0 = INTERLEAVED || (int)d < half ? d : half + d, d1 = INTERLEAVED ? d + a.dim / 2 : (int)d < half ? d + half : d0 + (a.dim - a.rotary) / 2;
    uintx4 w0, w1;
    if constexpr (STREAM) {
        w0 = __builtin_nontemporal_load((const uintx4 *)(x + d0));
        w1 = __builtin_nontemporal_load((const uintx4 *)(x + d1));
    } else {
        w0 = *(const uintx4 *)(x + d0);
        w1 = *(const uintx4 *)(x + d1);
    }
    if (d0 < a.rotary) {
        const int position = a.positions[token];
        // pairs first .. first + 4 and second .. second + 4; interleaved, the second piece may be beyond what is turned
        const int first = INTERLEAVED ? d0 / 2 : d0, second = INTERLEAVED ? (d1 < a.rotary ? d1 / 2 : first) : d0 + 4;
        float c[8], s[8];
        if (position >= 0 && position < a.table_rows) {
            const float *row = a.table + (int64_t)position * a.rotary;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = row[first + i];
                c[4 + i] = row[second + i];
                s[i] = row[half + first + i];
                s[4 + i] = row[half + second + i];
            }
        } else {                                        // there is no such angle
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
        }
        if (a.inverse)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = -s[i];
        float u[8], v[8];
        widen8<BF16>(w0, u);
        widen8<BF16>(w1, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float &p = INTERLEAVED ? (i < 4 ? u[2 * i] : v[2 * i - 8]) : u[i];
            float &q = INTERLEAVED ? (i < 4 ? u[2 * i + 1] : v[2 * i - 7]) : v[i];
            const float p2 = p * c[i] - q * s[i];
            q = q * c[i] + p * s[i];
            p = p2;
        }
        w0 = narrow8<BF16>(u);
        if (!INTERLEAVED || d1 < a.rotary) w1 = narrow8<BF16>(v);
    }
    __builtin_nontemporal_store(w0, (uintx4 *)(y + d0));
    __builtin_nontemporal_store(w1, (uintx4 *)(y + d1));
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

// x beyond the memory-side cache is read as a stream: 335 MB of it (16383 x 80 heads of 128) 108 us so,
// 111 us with ordinary loads; 42 MB (2048 tokens), which a projection has just written there, 16.7 and 13.9 us.  Where only a part
// of each head turns, its halves' pieces are not whole lines and ordinary loads are faster in any case (131 and 119 us).
template <bool BF16, bool INTERLEAVED>
hipError_t rotary_pieces(const RotaryArgs &a, hipStream_t stream)
{
    const int64_t lanes = a.tokens * a.heads * (a.dim / 16);
    const int64_t grid = (lanes + 255) / 256;
    const bool stream_x = beyond_cache(lanes * 32) && (INTERLEAVED || a.rotary == a.dim);
    return stream_x ? launch_many(k_rotary<BF16, INTERLEAVED, true>, grid, 256, stream, a, a.dim / 16)
                    : launch_many(k_rotary<BF16, INTERLEAVED, false>, grid, 256, stream, a, a.dim / 16);
}

}  // namespace

hipError_t launch_rotary_table(const double *frequencies, int64_t rows, int rotary, double magnitude, float *table, hipStream_t stream)
{
    const int64_t lanes = rows * (rotary / 2);
    return launch_many(k_rotary_table, (lanes + 255) / 256, 256, stream, frequencies, rows, rotary / 2, magnitude, table);
}

hipError_t launch_rotary(const RotaryArgs &a, hipStream_t stream)
{
    if (a.rotary % 16 == 0 && a.dim % 16 == 0) {        // whole 128-bit accesses, and each pair's two halves in two of them
        if (a.bf16) return a.interleaved ? rotary_pieces<true, true>(a, stream) : rotary_pieces<true, false>(a, stream);
        return a.interleaved ? rotary_pieces<false, true>(a, stream) : rotary_pieces<false, false>(a, stream);
    }
    const int64_t lanes = a.tokens * a.heads * (a.dim - a.rotary / 2);
    const int64_t grid = (lanes + 255) / 256;
    return a.bf16 ? launch_many(k_rotary_any<true>, grid, 256, stream, a) : launch_many(k_rotary_any<false>, grid, 256, stream, a);
}

}  // namespace fc
