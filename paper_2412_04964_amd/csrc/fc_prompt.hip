// fc_prompt.hip -- attention over whole prompts, packed one behind the other.
//
// Query i of a sequence sees all its tokens, or (causal) those up to i:  o = sum_t softmax_t(scale q . k_t) v_t.
// A wavefront has 32 queries of one head and takes 64 (or 32) tokens at a time.  It forms the transposed score S^T = K Q^T with 32 x 32 x 16
// matrix instructions, which leaves a lane with weights of the very tokens that it needs as operand of O^T = V^T P^T, and keeps the
// running maximum and sum of its column: one pass over K and V, and nothing but K and V goes through LDS.
//   K and V tiles go from memory straight to LDS, one tile ahead of the arithmetic; beyond the sequence's end they are zeros.
//   Rows of a tile lie as in memory, their 16-byte units exchanged (unit ^ swizzle of the row) so that reads find every bank once.
//   Weights are rounded to the type of the values, their sum adds them before that.  Their unit is the running maximum: bfloat16 has the
//   range for all that are lower, so it is raised only, and when a score passes it by kSlack.  Binary16 has not: the unit follows a tile's
//   largest score up and down when that is kSlack away, and the largest is put at 2^kBias, so that a tile's weights have 11 bits
//   down to 2^-9 of its largest however far that is below the row's (down to 2^-kReach, where they are lost).
// Matrix instructions and the exponentials between them bound it, at a clock that falls under this load (1.5 to 1.7 GHz counted):
// 16384 tokens, 16 heads, causal, bfloat16: 965 to 1036 us by card, 1.14 to 1.06 PFLOP/s, where a library's 16384^3 product reaches 1.31.
// 11 ragged prompts, 8191 tokens, 40 heads, binary16: 129 to 136 us, where edges and what surrounds the loop weigh more.
#include "fc_attn.hpp"

namespace fc {
namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));

// in powers of two: how far a tile's largest score may be from the unit; where it is put; how far below the row's largest the unit may go
template <bool BF16> constexpr float kSlack = BF16 ? 8.0f : 10.0f;
constexpr float kBias = 5.0f, kReach = 60.0f;

// what the number of a 16-byte unit is exchanged by in row t of a tile: 16 rows of K, read one unit each, and four of V, read 64 bytes
// each, take every bank once
template <int DIM, bool K> __device__ __forceinline__ int swizzle(int t)
{
    if (K) return DIM == 128 ? t & 15 : (t >> 1) & 7;
    return DIM == 128 ? 4 * (t & 3) : 4 * ((t >> 1) & 1);
}

// buffer resource of 16 rows, of which [0, left) are there; everything else reads as zero
__device__ __forceinline__ uintx4 rows16(const uint16_t *base, int stride, int left, int dim)
{
    const int last = left < 16 ? left - 1 : 15;
    return resource(base, last < 0 ? 0u : (uint32_t)(last * stride + dim) * 2u);
}

// How a wavefront brings 16 rows of a tile to LDS, 1 KB at a time: where in memory each lane finds its 16 bytes
template <int DIM, bool K>
struct Rows16 {
    static constexpr int kPieces = 16 * DIM * 2 / 1024;
    int offset[kPieces];

    __device__ __forceinline__ Rows16(int lane, int stride)
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = i * 1024 + lane * 16, row = at / (2 * DIM), unit = at % (2 * DIM) / 16;
            offset[i] = row * stride * 2 + (unit ^ swizzle<DIM, K>(row)) * 16;
        }
    }
    __device__ __forceinline__ void load(uintx4 rsrc, const uint8_t *lds) const
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) load_to_lds<false>(rsrc, offset[i], lds_address(lds) + i * 1024);
    }
};

__device__ __forceinline__ uintx2 transposed(const uint8_t *p)
{
    return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)p));
}

template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// The sequence that has work unit u (see find_sequence), its first token and the next one's.  One read for 64 sequences instead of one
// behind the other.
struct Found {
    int b, off, next;
};
__device__ __forceinline__ Found find_sequence_wide(const int32_t *__restrict__ offsets, int sequences, int shift, int64_t u, int lane)
{
    for (int c = 0;; c += 63) {
        const int i = c + lane < sequences ? c + lane : sequences;
        const int off = offsets[i];
        // lanes up to the last sequence that begins at or before u
        const uint64_t before = __ballot(c + lane < sequences && (int64_t)(off >> shift) + i <= u);
        const int count = __builtin_popcountll(before);
        if (count < 64) {
            const int l = count ? count - 1 : 0;
            return {c + l, __builtin_amdgcn_readlane(off, l), __builtin_amdgcn_readlane(off, l + 1)};
        }
    }
}

// SPLIT: eight wavefronts have the same 32 rows and take their tiles in turn, each with a K and a V tile of its own in LDS; they are joined
// at the end.  Else four have 32 rows each and all work on the same tiles, two of each in LDS: of 64 tokens, or of 32, which leaves registers
// and LDS for three workgroups on a compute unit.
template <int DIM, bool BF16, bool SPLIT, int TOKENS>
__global__ void __launch_bounds__(SPLIT ? 512 : 256, SPLIT || TOKENS == 64 ? 2 : 3) k_prompt_attention(PromptArgs a, int units)
{
    constexpr int kWaves = SPLIT ? 8 : 4, kTokens = TOKENS;                     // tokens of a tile
    constexpr int kSteps = DIM / 16, kOut = DIM / 32, kRow = 2 * DIM, kTile = kTokens * kRow, kHalves = kTokens / 32, kGroups = kTokens / 16;
    constexpr int kShift = SPLIT ? 5 : 7, kRows = 1 << kShift;                 // queries of a workgroup
    constexpr int kOutRow = kRow + 16, kOutBytes = (SPLIT ? 1 : kWaves) * 32 * kOutRow;         // of the results on their way out
    constexpr int kTiles = SPLIT ? 2 * kWaves : 4;
    static_assert(TOKENS == 64 || TOKENS == 32, "whole matrix instructions");
    __shared__ __attribute__((aligned(1024))) uint8_t tiles[kTiles * kTile > kOutBytes ? kTiles : (kOutBytes + kTile - 1) / kTile][kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, side = lane >> 5;
    const int query_heads = a.heads * a.group;
    // workgroups go to the 8 XCDs in turn: where heads can be dealt to them, an XCD's L2 has few heads' K and V
    int head, unit;
    if (query_heads % 8 == 0) {
        const uint32_t per = query_heads / 8, j = blockIdx.x >> 3;
        head = (blockIdx.x & 7) * per + j % per;
        unit = units - 1 - j / per;
    } else {
        head = blockIdx.x % query_heads;
        unit = units - 1 - blockIdx.x / query_heads;
    }
    // late rows, which see most, come first; where (nearly) all workgroups are on the chip at once, two on a compute unit, the second ones
    // go from early rows to late ones, so that the longest run beside the shortest (8192 tokens of 8 heads, 520 workgroups, 165 -> 157 us)
    if (!SPLIT && units * query_heads > 256 && units * query_heads <= 640) {
        const int u = units - 1 - unit, once = 256 / query_heads;
        if (u >= once) unit = u - once;
    }
    const int kv_head = head / a.group;
    const Found at = find_sequence_wide(a.offsets, a.sequences, kShift, unit, lane);
    const int64_t off = at.off;
    const int n = at.next - at.off;
    if (at.off < 0 || at.next <= at.off || at.next > a.tokens) return;
    const int place = unit - ((at.off >> kShift) + at.b);
    if (place < 0 || place > (n - 1) >> kShift) return;    // (negative: tokens before the first sequence, or offsets that do not ascend)
    const int first = place * kRows, row0 = SPLIT ? first : first + wave * 32, row = row0 + col;

    uintx4 qf[kSteps];
    {
        const uint16_t *q = (const uint16_t *)a.q.ptr + (off + (row < n ? row : n - 1)) * a.q.token + head * a.q.head + side * 8;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) qf[j] = *(const uintx4 *)(q + 16 * j);
    }
    const int stride_k = (int)a.k.token, stride_v = (int)a.v.token;
    const uint16_t *k = (const uint16_t *)a.k.ptr + off * a.k.token + kv_head * a.k.head;
    const uint16_t *v = (const uint16_t *)a.v.ptr + off * a.v.token + kv_head * a.v.head;
    const float factor = a.scale * 1.4426950408889634f;       // scores in powers of two

    const Rows16<DIM, true> rows_k(lane, stride_k);
    const Rows16<DIM, false> rows_v(lane, stride_v);
    // operand addresses in a tile: K by row lane % 32, V by the row and the 8 bytes that this lane contributes to a transposing read
    const int at_k = col * kRow + (side ^ swizzle<DIM, true>(col)) * 16;
    const int v_row = 4 * side + (lane & 15) / 4;
    const int at_v = v_row * kRow + ((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ swizzle<DIM, false>(v_row)) * 16 + (lane & 1) * 8;

    floatx16 acc[kOut];
    float top, peak, total;
    const auto clear_sums = [&] {
#pragma unroll
        for (int o = 0; o < kOut; ++o)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[o][r] = 0.0f;
        top = peak = -FLT_MAX;
        total = 0.0f;
    };
    clear_sums();

    const int end = a.causal && first + kRows < n ? first + kRows : n;      // of the workgroup
    // a wavefront without rows takes no tokens (11 ragged prompts, 8191 tokens, 40 heads: 128.9 -> 125.6 us)
    const int my_end = !SPLIT && row0 >= n ? 0 : a.causal && row0 + 32 < n ? row0 + 32 : n;
    const int clear = a.causal && row0 < n ? row0 + 1 : n;                  // tokens that every row sees

    // 16 rows of a tile from token t0 on
    const auto load_k = [&](int t0, int group, const uint8_t *tile) {
        t0 += 16 * group;
        rows_k.load(rows16(k + (int64_t)t0 * stride_k, stride_k, n - t0, DIM), tile + group * 16 * kRow);
    };
    const auto load_v = [&](int t0, int group, const uint8_t *tile) {
        t0 += 16 * group;
        rows_v.load(rows16(v + (int64_t)t0 * stride_v, stride_v, n - t0, DIM), tile + group * 16 * kRow);
    };
    floatx16 s[kHalves];
    const auto scores = [&](const uint8_t *lds_k) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[h][r] = 0.0f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
                s[h] = mma32<BF16>(*(const uintx4 *)(lds_k + (at_k ^ (j << 5)) + h * 32 * kRow), qf[j], s[h]);
    };
    uintx4 pf[2 * kHalves];
    const auto mask = [&](int t0) {
        const int sees = (a.causal && row < n - 1 ? row + 1 : n) - t0 - 4 * side;
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (h * 32 + 8 * (r / 4) + r % 4 >= sees) s[h][r] = -__builtin_inff();
    };
    const auto weights = [&](int t0) {
        float most = s[0][0];
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[h][r]);
        bool away;
        if constexpr (BF16) {
            most *= factor;
            away = most > top + kSlack<BF16>;
        } else {
            most = __builtin_fmaf(most, factor, -kBias);
            if (t0 + kTokens > clear) most = fmaxf(most, __shfl_xor(most, 32));      // a lane may have nothing that its row sees
            away = fabsf(most - top) > kSlack<BF16>;
        }
        if (__any(away)) {
            most = fmaxf(most, __shfl_xor(most, 32));
            // only rows that are away themselves: no row's bits depend on others
            float now = most > top + kSlack<BF16> ? most : top;
            if constexpr (!BF16) {
                now = fabsf(most - top) > kSlack<BF16> ? fmaxf(most, peak - kReach) : top;
                peak = fmaxf(peak, now);
            }
            const float shrink = __builtin_amdgcn_exp2f(top - now);
            top = now;
            total *= shrink;
#pragma unroll
            for (int o = 0; o < kOut; ++o) acc[o] *= shrink;
        }
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][r], factor, -top));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][r + 1], factor, -top));
                total += p0 + p1;
                pf[2 * h + r / 8][r % 8 / 2] = narrow2<BF16>(p0, p1);
            }
    };
    const auto add_values = [&](const uint8_t *lds_v) {
#pragma unroll
        for (int m = 0; m < 2 * kHalves; ++m)
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                const uint8_t *p = lds_v + (at_v ^ (o << 6)) + m * 16 * kRow;
                const uintx2 lo = transposed(p), hi = transposed(p + 8 * kRow);
                acc[o] = mma32<BF16>(uintx4{lo[0], lo[1], hi[0], hi[1]}, pf[m], acc[o]);
            }
    };
    // In a tile that not all rows see whole, an infinity or NaN among the values would be NaN times the weight of 0 of those that do not.
    // Such values are left out of the products and added to the rows that see them.
    const auto not_finite = [](uint32_t w) { return (w & 0x7FFF7FFFu) + (BF16 ? 0x00800080u : 0x04000400u); };      // in the sign bits of w's halves
    const auto finite_only = [&](uint32_t w) { return w & ~(((not_finite(w) & 0x80008000u) >> 15) * 0xFFFFu); };
    const auto any_not_finite = [&](const uint8_t *lds_v) {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < kTile / 1024; ++i) {
            const uintx4 w = *(const uintx4 *)(lds_v + i * 1024 + lane * 16);
            any |= not_finite(w[0]) | not_finite(w[1]) | not_finite(w[2]) | not_finite(w[3]);
        }
        return __any(any & 0x80008000u) != 0;
    };
    const auto add_not_finite = [&](const uint8_t *lds_v, int t0) {
#pragma unroll 1
        for (int t = 0; t < kTokens; ++t) {
            const uint8_t *p = lds_v + t * kRow + side * 8;
            const bool seen = t0 + t <= row;
#pragma unroll
            for (int o = 0; o < kOut; ++o)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const uintx2 w = *(const uintx2 *)(p + ((o * 4 + r / 4) ^ swizzle<DIM, false>(t)) * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t bits = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
                        if (seen && (not_finite(bits) & 0x8000u)) acc[o][r + i] += widen<BF16>(bits);
                    }
                }
        }
    };
    // the queries are here before the loop, where waiting for them would wait for the tiles that are loaded ahead
    const auto queries_here = [&] {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) asm volatile("" : "+v"(qf[j]));
    };
    if constexpr (SPLIT) {
        constexpr int kLoads = kGroups * Rows16<DIM, true>::kPieces;
        const uint8_t *const tile_k = tiles[2 * wave], *const tile_v = tiles[2 * wave + 1];
        int t0 = wave * kTokens;
        if (t0 < end) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) load_k(t0, g, tile_k);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) load_v(t0, g, tile_v);
        }
        queries_here();
        for (; t0 < end; t0 += kWaves * kTokens) {
            const bool more = t0 + kWaves * kTokens < end;
            wait_vm<kLoads>();                           // K is here, V may be on its way
            scores(tile_k);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more)
#pragma unroll
                for (int g = 0; g < kGroups; ++g) load_k(t0 + kWaves * kTokens, g, tile_k);
            if (t0 + kTokens > clear) mask(t0);
            weights(t0);
            if (more) wait_vm<kLoads>();                 // V is here, the next K may be on its way
            else wait_vm<0>();
            if (a.causal && t0 + kTokens > clear && any_not_finite(tile_v)) {
                add_not_finite(tile_v, t0);
#pragma unroll 1
                for (int i = 0; i < kTile / 1024; ++i) {
                    uintx4 *const place = (uintx4 *)(tile_v + i * 1024 + lane * 16);
                    const uintx4 w = *place;
                    *place = uintx4{finite_only(w[0]), finite_only(w[1]), finite_only(w[2]), finite_only(w[3])};
                }
            }
            add_values(tile_v);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more)
#pragma unroll
                for (int g = 0; g < kGroups; ++g) load_v(t0 + kWaves * kTokens, g, tile_v);
        }
    } else {
        __shared__ int again;
        const auto load = [&](int t0, int to) {
            if constexpr (kGroups == kWaves) {
                load_k(t0, wave, tiles[to]);
                load_v(t0, wave, tiles[to + 1]);
            } else {                                     // half of the wavefronts bring K, half V
                if (wave < kGroups) load_k(t0, wave, tiles[to]);
                else load_v(t0, wave - kGroups, tiles[to + 1]);
            }
        };
        const auto compute = [&](int t0, int from) {
            if (t0 >= my_end) return;
            scores(tiles[from]);
            if (t0 + kTokens > clear) {
                mask(t0);
                if (a.causal && any_not_finite(tiles[from + 1])) again = 1;
            }
            weights(t0);
            add_values(tiles[from + 1]);
        };
        const auto arrived = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
        load(0, 0);
        if (threadIdx.x == 0) again = 0;
        queries_here();
        arrived();
        for (int t0 = 0; t0 < end; t0 += 2 * kTokens) {
            if (t0 + kTokens < end) load(t0 + kTokens, 2);
            compute(t0, 0);
            arrived();
            if (t0 + kTokens >= end) break;
            if (t0 + 2 * kTokens < end) load(t0 + 2 * kTokens, 0);
            compute(t0 + kTokens, 2);
            arrived();
        }
        // The workgroup's rows once more, in the same steps, where there were such values (that care in the loop above would cost all calls
        // 4 to 6 %; a tile is other wavefronts' too, so they cannot be taken out of it)
        if (__builtin_amdgcn_readfirstlane(again)) {
            clear_sums();
            for (int t0 = 0; t0 < end; t0 += kTokens) {
                load(t0, 0);
                arrived();
                if (t0 < my_end) {
                    const bool masked = t0 + kTokens > clear;
                    scores(tiles[0]);
                    if (masked) mask(t0);
                    weights(t0);
                    if (masked) add_not_finite(tiles[1], t0);
                    const uint32_t keep = masked ? 0u : 0xFFFFFFFFu;        // of what is not finite
#pragma unroll
                    for (int m = 0; m < 2 * kHalves; ++m)
#pragma unroll
                        for (int o = 0; o < kOut; ++o) {
                            const uint8_t *p = tiles[1] + (at_v ^ (o << 6)) + m * 16 * kRow;
                            const uintx2 lo = transposed(p), hi = transposed(p + 8 * kRow);
                            const uintx4 w = {lo[0], lo[1], hi[0], hi[1]};
                            acc[o] = mma32<BF16>(uintx4{finite_only(w[0]) | (w[0] & keep), finite_only(w[1]) | (w[1] & keep), finite_only(w[2]) | (w[2] & keep),
                                                        finite_only(w[3]) | (w[3] & keep)}, pf[m], acc[o]);
                        }
                }
                arrived();
            }
        }
    }

    total += __shfl_xor(total, 32);
    if constexpr (SPLIT) {
        // all in the unit of the largest maximum, then halves of the wavefronts added to the other half
        __shared__ float join_max[kWaves][32], join_sum[kWaves][32];
        float(*join)[32][DIM + 4] = reinterpret_cast<float(*)[32][DIM + 4]>(tiles);        // [kWaves / 2], when the tiles are done with
        static_assert(sizeof(tiles) >= sizeof(float) * kWaves / 2 * 32 * (DIM + 4), "the wavefronts' sums fit the tiles");
        if (side == 0) {
            join_max[wave][col] = top;
            join_sum[wave][col] = total;
        }
        __syncthreads();
        float best = join_max[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) best = fmaxf(best, join_max[w][col]);
        total = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += join_sum[w][col] * __builtin_amdgcn_exp2f(join_max[w][col] - best);
        const float unit = __builtin_amdgcn_exp2f(top - best);
#pragma unroll
        for (int o = 0; o < kOut; ++o) acc[o] *= unit;
#pragma unroll
        for (int half = kWaves / 2; half; half >>= 1) {
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int o = 0; o < kOut; ++o)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *(floatx4 *)&join[wave - half][col][o * 32 + 2 * r + 4 * side] = floatx4{acc[o][r], acc[o][r + 1], acc[o][r + 2], acc[o][r + 3]};
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int o = 0; o < kOut; ++o)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const floatx4 x = *(const floatx4 *)&join[wave][col][o * 32 + 2 * r + 4 * side];
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[o][r + i] += x[i];
                    }
            __syncthreads();
        }
        if (wave) return;
    }
    // through LDS, where the tiles are done with, so that a wavefront stores whole rows (a lane has 4 elements of a row at a time)
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    uint8_t *const mine = &tiles[0][0] + (SPLIT ? 0 : wave) * 32 * kOutRow;                     // neighbouring rows begin 4 banks apart
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *(uintx2 *)(mine + col * kOutRow + (o * 32 + 2 * r + 4 * side) * 2) = uintx2{narrow2<BF16>(acc[o][r] * inv, acc[o][r + 1] * inv), narrow2<BF16>(acc[o][r + 2] * inv, acc[o][r + 3] * inv)};
    constexpr int kLanes = DIM / 8;                      // of a row
#pragma unroll
    for (int i = 0; i < 32 * kLanes / 64; ++i) {
        const int out_row = i * (64 / kLanes) + lane / kLanes, d = lane % kLanes * 8;
        const uintx4 w = *(const uintx4 *)(mine + out_row * kOutRow + d * 2);
        if (row0 + out_row < n) *(uintx4 *)((uint16_t *)a.out.ptr + (off + row0 + out_row) * a.out.token + head * a.out.head + d) = w;
    }
}

// Whether workgroups of 32 rows whose wavefronts split the tokens are faster than those of 128 rows, by what both were measured to take
// in tenths of a microsecond.  128 rows: as long as the longest sequence's last rows, 1.1 us (0.8 with heads of 64) for 64 tokens, while
// no more than two workgroups share a compute unit.  32 rows: rounds of one workgroup (two) a compute unit, 3.2 us and 1.5 us for 256
// tokens each.  us, 8 heads of 128, causal, 128 / 32 rows: 1024 tokens 22.6 / 13.0, 2048 39.4 / 25.8, 4096 72.7 / 69.4, 8192 163 / 221;
// 16 heads, 2048 tokens 40.3 / 49.5; 8 sequences of 1024 tokens 44.0 / 88.3.
bool split_is_faster(const PromptArgs &a, int64_t wide, int64_t narrow)
{
    const int64_t heads = a.heads * a.group, longest = a.longest < a.tokens ? a.longest : a.tokens;
    if (wide * heads > 512) return false;
    const int64_t slots = a.dim == 64 ? 512 : 256, rounds = (narrow * heads + slots - 1) / slots;
    const int64_t half_steps = a.causal ? longest / 256 + 1 : longest / 128;
    return rounds * (32 + 15 * half_steps / 2) < (a.dim == 64 ? 8 : 11) * ((longest + 63) / 64);
}

template <int DIM, bool BF16>
hipError_t prompt(const PromptArgs &a, hipStream_t stream)
{
    const int query_heads = a.heads * a.group;
    const int64_t wide = (a.tokens >> 7) + a.sequences, narrow = (a.tokens >> 5) + a.sequences;
    if (split_is_faster(a, wide, narrow))
        return launch_many(k_prompt_attention<DIM, BF16, true, 32>, narrow * query_heads, 512, stream, a, (int)narrow);
    const int64_t grid = wide * query_heads;
    // Three workgroups on a compute unit, where there are two rounds of them and more; us for tiles of 64 / 32 tokens: 16384 tokens of 16 heads
    // of 128 (2064 workgroups) 1003 / 999, 8191 packed ones of 40 heads (2960) 138 / 130, but 8192 of 8 heads (520) 162 / 190, 4096 (264) 73 / 94;
    // 8 x 512 tokens of 32 heads (1280) 42 / 40.  Heads of 64 have four workgroups with 64 tokens.
    if constexpr (DIM == 128) {
        if (wide * query_heads > 1536) return launch_many(k_prompt_attention<DIM, BF16, false, 32>, grid, 256, stream, a, (int)wide);
    }
    return launch_many(k_prompt_attention<DIM, BF16, false, 64>, grid, 256, stream, a, (int)wide);
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs &a, hipStream_t stream)
{
    if (a.dim == 64) return a.bf16 ? prompt<64, true>(a, stream) : prompt<64, false>(a, stream);
    return a.bf16 ? prompt<128, true>(a, stream) : prompt<128, false>(a, stream);
}

}  // namespace fc
