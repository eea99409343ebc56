// fc_prompt.hip -- attention over whole prompts, packed one behind the other.
//
// Query i of a sequence sees all its tokens, or (causal) those up to i:  o = sum_t softmax_t(scale q . k_t) v_t.
// A wavefront has 32 queries of one head and takes 64 tokens at a time.  It forms the transposed score S^T = K Q^T with 32 x 32 x 16
// matrix instructions, which leaves a lane with weights of the very tokens that it needs as operand of O^T = V^T P^T, and keeps the
// running maximum and sum of its column: one pass over K and V, and nothing but K and V goes through LDS.
//   K and V tiles go from memory straight to LDS, one tile ahead of the arithmetic; beyond the sequence's end they are zeros.
//   Rows of a tile lie as in memory, their 16-byte units exchanged (unit ^ swizzle of the row) so that reads find every bank once.
//   The running maximum is raised only when a score passes it by kSlack; the sums carry the same factor either way.
// Matrix instructions and the exponentials between them bound it.
#include "fc_attn.hpp"

namespace fc {
namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;      // queries of a workgroup
constexpr int kTokens = 64;             // of a tile
constexpr float kSlack = 8.0f;          // in powers of two

// what the number of a 16-byte unit is exchanged by in row t of a tile: 16 rows of K, read one unit each, and four of V, read 64 bytes
// each, take every bank once
template <int DIM, bool K> __device__ __forceinline__ int swizzle(int t)
{
    if (K) return DIM == 128 ? t & 15 : (t >> 1) & 7;
    return DIM == 128 ? 4 * (t & 3) : 4 * ((t >> 1) & 1);
}

// buffer resource of rows [0, left) of a tile; everything else reads as zero
__device__ __forceinline__ uintx4 tile_rows(const uint16_t *base, int64_t stride, int64_t left, int dim)
{
    int64_t bytes = ((left - 1) * stride + dim) * 2;
    if (left <= 0) bytes = 0;
    return resource(base, bytes > 0x7FFFFFF0 ? 0x7FFFFFF0u : (uint32_t)bytes);
}

// tile positions of this lane's pieces: kPieces times 16 bytes, which land at lds + piece * 1024 + 16 lane of the wavefront's part
template <int DIM, bool K>
struct Staging {
    static constexpr int kPieces = kTokens * DIM * 2 / 1024 / kWaves;
    int offset[kPieces];

    __device__ __forceinline__ Staging(int wave, int lane, int64_t stride)
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = (wave * kPieces + i) * 1024 + lane * 16, row = at / (2 * DIM), unit = at % (2 * DIM) / 16;
            offset[i] = row * (int)stride * 2 + (unit ^ swizzle<DIM, K>(row)) * 16;
        }
    }
    __device__ __forceinline__ void load(uintx4 rsrc, const uint8_t *lds, int wave) const
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) load_to_lds<false>(rsrc, offset[i], lds_address(lds) + (wave * kPieces + i) * 1024);
    }
};

__device__ __forceinline__ uintx2 transposed(const uint8_t *p)
{
    return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)p));
}

template <int DIM, bool BF16>
__global__ void __launch_bounds__(64 * kWaves, 2) k_prompt_attention(PromptArgs a, int64_t units)
{
    constexpr int kSteps = DIM / 16, kOut = DIM / 32, kRow = 2 * DIM;
    __shared__ __attribute__((aligned(1024))) uint8_t tile_k0[kTokens * kRow], tile_v0[kTokens * kRow];
    __shared__ __attribute__((aligned(1024))) uint8_t tile_k1[kTokens * kRow], tile_v1[kTokens * kRow];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, side = lane >> 5;
    const int query_heads = a.heads * a.group;
    // workgroups go to the 8 XCDs in turn: where heads can be dealt to them, an XCD's L2 has few heads' K and V
    int head;
    int64_t unit;
    if (query_heads % 8 == 0) {
        const uint32_t per = query_heads / 8, j = blockIdx.x >> 3;
        head = (blockIdx.x & 7) * per + j % per;
        unit = units - 1 - j / per;
    } else {
        head = blockIdx.x % query_heads;
        unit = units - 1 - blockIdx.x / query_heads;
    }
    const int kv_head = head / a.group;
    const int b = find_sequence(a.offsets, a.sequences, 7, 1, unit);
    const int64_t off = a.offsets[b];
    const int64_t n = (int64_t)a.offsets[b + 1] - off;
    if (off < 0 || n <= 0 || off + n > a.tokens) return;
    const int64_t first = (unit - ((off >> 7) + b)) * kRows;
    if (first >= n) return;
    const int64_t row0 = first + wave * 32, row = row0 + col;

    uintx4 qf[kSteps];
    {
        const uint16_t *q = (const uint16_t *)a.q.ptr + (off + (row < n ? row : n - 1)) * a.q.token + head * a.q.head + side * 8;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) qf[j] = *(const uintx4 *)(q + 16 * j);
    }
    const uint16_t *k = (const uint16_t *)a.k.ptr + off * a.k.token + kv_head * a.k.head;
    const uint16_t *v = (const uint16_t *)a.v.ptr + off * a.v.token + kv_head * a.v.head;
    const float factor = a.scale * 1.4426950408889634f;       // scores in powers of two

    const Staging<DIM, true> stage_k(wave, lane, a.k.token);
    const Staging<DIM, false> stage_v(wave, lane, a.v.token);
    // operand addresses in a tile: K by row lane % 32, V by the row and the 8 bytes that this lane contributes to a transposing read
    const int at_k = col * kRow + (side ^ swizzle<DIM, true>(col)) * 16;
    const int v_row = 4 * side + (lane & 15) / 4;
    const int at_v = v_row * kRow + ((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ swizzle<DIM, false>(v_row)) * 16 + (lane & 1) * 8;

    floatx16 acc[kOut];
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[o][r] = 0.0f;
    float top = -FLT_MAX, total = 0.0f;

    const int64_t end = a.causal && first + kRows < n ? first + kRows : n;      // of the workgroup
    const int64_t my_end = a.causal && row0 + 32 < n ? row0 + 32 : n;
    const int64_t clear = a.causal && row0 < n ? row0 + 1 : n;                  // tokens that every row sees

    const auto load = [&](int64_t t0, uint8_t *lds_k, uint8_t *lds_v) {
        stage_k.load(tile_rows(k + t0 * a.k.token, a.k.token, n - t0, DIM), lds_k, wave);
        stage_v.load(tile_rows(v + t0 * a.v.token, a.v.token, n - t0, DIM), lds_v, wave);
    };
    const auto compute = [&](int64_t t0, const uint8_t *lds_k, const uint8_t *lds_v) {
        if (t0 >= my_end) return;
        floatx16 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[h][r] = 0.0f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                s[h] = mma32<BF16>(*(const uintx4 *)(lds_k + (at_k ^ (j << 5)) + h * 32 * kRow), qf[j], s[h]);
        if (t0 + kTokens > clear) {
            const int64_t sees = a.causal && row < n - 1 ? row + 1 : n;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (t0 + h * 32 + 8 * (r / 4) + 4 * side + r % 4 >= sees) s[h][r] = -__builtin_inff();
        }
        float most = s[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[h][r]);
        most *= factor;
        if (__any(most > top + kSlack)) {
            most = fmaxf(most, __shfl_xor(most, 32));
            const float now = fmaxf(top, most), shrink = __builtin_amdgcn_exp2f(top - now);
            top = now;
            total *= shrink;
#pragma unroll
            for (int o = 0; o < kOut; ++o) acc[o] *= shrink;
        }
        uintx4 pf[4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][r], factor, -top));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][r + 1], factor, -top));
                total += p0;
                total += p1;
                pf[2 * h + r / 8][r % 8 / 2] = narrow2<BF16>(p0, p1);
            }
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                const uint8_t *p = lds_v + (at_v ^ (o << 6)) + m * 16 * kRow;
                const uintx2 lo = transposed(p), hi = transposed(p + 8 * kRow);
                acc[o] = mma32<BF16>(uintx4{lo[0], lo[1], hi[0], hi[1]}, pf[m], acc[o]);
            }
    };
    const auto arrived = [] {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };

    load(0, tile_k0, tile_v0);
    // the queries are here before the loop, where waiting for them would wait for the tiles that are loaded ahead
#pragma unroll
    for (int j = 0; j < kSteps; ++j) asm volatile("" : "+v"(qf[j]));
    arrived();
    for (int64_t t0 = 0; t0 < end; t0 += 2 * kTokens) {
        if (t0 + kTokens < end) load(t0 + kTokens, tile_k1, tile_v1);
        compute(t0, tile_k0, tile_v0);
        arrived();
        if (t0 + kTokens >= end) break;
        if (t0 + 2 * kTokens < end) load(t0 + 2 * kTokens, tile_k0, tile_v0);
        compute(t0 + kTokens, tile_k1, tile_v1);
        arrived();
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
    return a.dim == 64 ? launch_kernel(k_prompt_attention<64, BF16>, grid, dim3(64 * kWaves), stream, a, units)
                       : launch_kernel(k_prompt_attention<128, BF16>, grid, dim3(64 * kWaves), stream, a, units);
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs &a, hipStream_t stream) { return a.bf16 ? prompt<true>(a, stream) : prompt<false>(a, stream); }

}  // namespace fc
