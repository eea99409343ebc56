// fc_cache.hip -- appends keys and values to the paged cache of 8-bit codes, the keys turned to their positions on the way.
//
// For each page and head that receives tokens, with top = 127 (signed codes) or 448 (E4M3):
//     s' = max(max|x| / top, FLT_MIN, the page's scale if it holds tokens of this sequence already)
//     codes that are there, if s' grew:   round(code * (s / s'))
//     new codes:                          round(x * (1 / s'))
// in fp32 with IEEE divides and rounding to nearest even, signed codes clamped to +-127.  x is the key as the rotation leaves it in fp32.
// A page of one head is one workgroup's, from the first read of its scale to the last code written, so nothing is atomic.  Whole
// pages are bound by memory (2 bytes read and 1 written per element), single tokens by the launch and a chain of four reads.
#include "fc_attn.hpp"

namespace fc {
namespace {

template <bool FP8> constexpr float kTop = FP8 ? 448.0f : 127.0f;

template <bool FP8>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d)
{
    if constexpr (FP8) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
    } else {
        const auto one = [](float v) { return (uint32_t)(int)fminf(fmaxf(rintf(v), -127.0f), 127.0f) & 0xFFu; };
        return one(a) | one(b) << 8 | one(c) << 16 | one(d) << 24;
    }
}

// the four codes of a word times r, as codes again
template <bool FP8>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float r)
{
    if constexpr (FP8) {
        const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        return pack4<FP8>(lo[0] * r, lo[1] * r, hi[0] * r, hi[1] * r);
    } else {
        return pack4<FP8>((float)(int8_t)w * r, (float)(int8_t)(w >> 8) * r, (float)(int8_t)(w >> 16) * r, (float)(int8_t)(w >> 24) * r);
    }
}

// 8 elements of a token from element d on, turned where they belong to the rotated part
template <bool BF16>
__device__ __forceinline__ void load_turned(const uint16_t *__restrict__ row, int d, const float *__restrict__ angles, int rotary, int interleaved, float (&f)[8])
{
    widen8<BF16>(*(const uintx4 *)(row + d), f);
    if (d >= rotary) return;
    const int half = rotary / 2;
    if (interleaved && rotary % 8 == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = angles[d / 2 + i], s = angles[half + d / 2 + i], a = f[2 * i], b = f[2 * i + 1];
            f[2 * i] = a * c - b * s;
            f[2 * i + 1] = b * c + a * s;
        }
    } else if (half % 8 == 0) {
        const bool first = d < half;
        const int pair = first ? d : d - half;
        float g[8];
        widen8<BF16>(*(const uintx4 *)(row + (first ? d + half : pair)), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = angles[pair + i], s = angles[half + pair + i];
            f[i] = first ? f[i] * c - g[i] * s : f[i] * c + g[i] * s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = d + i;
            if (e >= rotary) continue;
            const bool first = interleaved ? (e & 1) == 0 : e < half;
            const int pair = interleaved ? e >> 1 : first ? e : e - half;
            const float other = widen<BF16>(row[interleaved ? e ^ 1 : first ? e + half : pair]);
            const float c = angles[pair], s = angles[half + pair];
            f[i] = first ? f[i] * c - other * s : f[i] * c + other * s;
        }
    }
}

// What a workgroup does: tokens [token, token + count) of the call go to the slots from `slot` on of page `id`
struct Piece {
    int64_t token, position;
    int64_t id;
    int slot, count;
};

// the j-th page that sequence b's new tokens go to; count = 0 where there is none
__device__ __forceinline__ Piece find_piece(const AppendArgs &a, int b, int64_t j)
{
    const int64_t off = a.step.offsets[b], held = a.step.held[b];
    int64_t end = held + ((int64_t)a.step.offsets[b + 1] - off);
    if (a.rotary && end > a.table_rows) end = a.table_rows;               // tokens without an angle are not appended
    if (off >= 0 && end - held > a.step.tokens - off) end = held + a.step.tokens - off;
    Piece p = {0, 0, 0, 0, 0};
    if (off < 0) return p;
    const int64_t first = held > 0 ? held : 0;
    const int page = a.cache.page;
    const int64_t index = first / page + j, from = index * page > first ? index * page : first;
    int64_t to = (index + 1) * page;
    if (to > end) to = end;
    if (from >= to || index >= a.cache.table_width) return p;
    p.id = a.cache.table[(int64_t)b * a.cache.table_width + index];
    if (p.id < 0 || p.id >= a.cache.pages) return p;
    p.token = off + (from - held);
    p.position = from;
    p.slot = (int)(from - index * page);
    p.count = (int)(to - from);
    return p;
}

// One page of one head of K or V by one workgroup of page * DIM / 32 lanes (64 at least), 4 times 8 elements a lane
template <int DIM, bool FP8, bool BF16>
__global__ void __launch_bounds__(512) k_cache_append(AppendArgs a, int page_shift)
{
    constexpr int kPieces = 4, kRow = DIM / 8;                            // 8-element pieces of a lane, of a token
    const int which = blockIdx.x % (2 * a.heads), value = which >= a.heads, head = which - (value ? a.heads : 0);
    const int64_t unit = blockIdx.x / (2 * a.heads);
    const int b = find_sequence(a.step.offsets, a.step.sequences, page_shift, 2, unit);
    const Piece p = find_piece(a, b, unit - ((int64_t)(a.step.offsets[b] >> page_shift) + 2 * (int64_t)b));
    if (p.count <= 0) return;

    const Rows &x = value ? a.v : a.k;
    const uint16_t *rows = (const uint16_t *)x.ptr + p.token * x.token + head * x.head;
    const int rotary = value ? 0 : a.rotary;
    float f[kPieces][8], most = 0.0f;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const int piece = threadIdx.x + j * blockDim.x, row = piece / kRow, d = piece % kRow * 8;
        if (row < p.count) {
            load_turned<BF16>(rows + row * x.token, d, a.table + (p.position + row) * rotary, rotary, a.interleaved, f[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(f[j][i]));
        }
    }
    float *scale = (value ? a.cache.v_scales : a.cache.k_scales) + p.id * a.heads + head;
    const float before = p.slot ? *scale : 0.0f;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    __shared__ float waves[8];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
    __syncthreads();
    for (int w = 0; w < (int)(blockDim.x + 63) / 64; ++w) most = fmaxf(most, waves[w]);
    const float now = fmaxf(fmaxf(most / kTop<FP8>, FLT_MIN), before);
    if (threadIdx.x == 0) *scale = now;

    uint8_t *codes = (value ? a.cache.v : a.cache.k) + (p.id * a.heads + head) * ((int64_t)DIM << page_shift);
    if (p.slot && now > before) {
        const float r = before / now;
        for (int at = threadIdx.x; at < p.slot * kRow; at += blockDim.x) {
            uintx2 *w = (uintx2 *)(codes + at * 8);
            *w = uintx2{rescale4<FP8>((*w)[0], r), rescale4<FP8>((*w)[1], r)};
        }
    }
    const float inv = 1.0f / now;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const int piece = threadIdx.x + j * blockDim.x, row = piece / kRow, d = piece % kRow * 8;
        if (row < p.count) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[j][i] *= inv;
            *(uintx2 *)(codes + (p.slot + row) * DIM + d) = uintx2{pack4<FP8>(f[j][0], f[j][1], f[j][2], f[j][3]), pack4<FP8>(f[j][4], f[j][5], f[j][6], f[j][7])};
        }
    }
}

template <int DIM, bool FP8>
hipError_t append(const AppendArgs &a, hipStream_t stream)
{
    const int shift = log2_int(a.cache.page);
    const int64_t units = (a.step.tokens >> shift) + 2 * (int64_t)a.step.sequences;
    const int lanes = a.cache.page * DIM / 32 < 64 ? 64 : a.cache.page * DIM / 32;
    const dim3 grid((uint32_t)(units * 2 * a.heads));
    return a.bf16 ? launch_kernel(k_cache_append<DIM, FP8, true>, grid, dim3(lanes), stream, a, shift)
                  : launch_kernel(k_cache_append<DIM, FP8, false>, grid, dim3(lanes), stream, a, shift);
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs &a, hipStream_t stream)
{
    switch (a.dim) {
    case 64: return a.fp8 ? append<64, true>(a, stream) : append<64, false>(a, stream);
    case 128: return a.fp8 ? append<128, true>(a, stream) : append<128, false>(a, stream);
    default: return a.fp8 ? append<256, true>(a, stream) : append<256, false>(a, stream);
    }
}

}  // namespace fc
