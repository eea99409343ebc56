// fc_cache.hip -- appends keys and values to the paged cache of 8-bit codes, the keys turned to their positions on the way.
//
// For each page and head that receives tokens, with top = 127 (signed codes) or 448 (E4M3):
//     s' = max(max|x| / top, FLT_MIN, the page's scale if it holds tokens of this sequence already)
//     codes that are there, if s' grew:   round(code * (s / s'))
//     new codes:                          round(x * (1 / s'))
// in fp32 with IEEE divides and rounding to nearest even, signed codes clamped to +-127.  x is the key as the rotation leaves it in fp32.
// A page of one head is one workgroup's, from the first read of its scale to the last code written, so nothing is atomic.  Whole
// pages are bound by memory (2 bytes read and 1 written per element; 32771 tokens of 8 heads of 128 with rotation 42 us, 5.2 TB/s),
// single tokens by the launch and a chain of four reads (256 sequences of 40 heads 4.8 us).
#include "fc_attn.hpp"

namespace fc {
namespace {

template <bool FP8> constexpr float kTop = FP8 ? 448.0f : 127.0f;

// 4 values -> codes.  Signed codes: 1.5 * 2^23 added to a value in (-2^22, 2^22) leaves it, rounded to nearest even, in the low bits.
// CLAMP: a value may be beyond the codes; those of x * (1 / s') with |x| <= top * s' round to at most top.
template <bool FP8, bool CLAMP = false>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d)
{
    if constexpr (FP8) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
    } else {
        const auto one = [](float v) {
            if constexpr (CLAMP) v = fminf(fmaxf(v, -127.0f), 127.0f);
            return __builtin_bit_cast(uint32_t, v + 12582912.0f);
        };
        const uint32_t ab = __builtin_amdgcn_perm(one(b), one(a), 0x0C0C0400u), cd = __builtin_amdgcn_perm(one(d), one(c), 0x04000C0Cu);
        return ab | cd;
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
        return pack4<FP8, true>((float)(int8_t)w * r, (float)(int8_t)(w >> 8) * r, (float)(int8_t)(w >> 16) * r, (float)(int8_t)(w >> 24) * r);
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

// Two pieces of 8 elements of a token, d0 and d1 on, that a lane takes together: the two halves of 8 pairs where they are turned.  Pair
// piece i of a row's DIM / 16; needs rotary % 16 == 0.
struct PairPiece {
    int d0, d1, pair;           // pair < 0: not turned
    __device__ __forceinline__ PairPiece(int i, int dim, int rotary, int interleaved)
    {
        if (i * 16 < rotary) {
            pair = i * 8;
            d0 = interleaved ? 2 * pair : pair;
            d1 = interleaved ? d0 + 8 : pair + rotary / 2;
        } else {
            pair = -1;
            d0 = rotary + (i * 16 - rotary) / 2;
            d1 = d0 + (dim - rotary) / 2;
        }
    }
};

__device__ __forceinline__ void turn8(float (&u)[8], float (&v)[8], const float *__restrict__ angles, int half, int pair, int interleaved)
{
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c[i] = angles[pair + i];
        s[i] = angles[half + pair + i];
    }
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = u[2 * i], b = u[2 * i + 1], e = v[2 * i], f = v[2 * i + 1];
            u[2 * i] = a * c[i] - b * s[i];
            u[2 * i + 1] = b * c[i] + a * s[i];
            v[2 * i] = e * c[i + 4] - f * s[i + 4];
            v[2 * i + 1] = f * c[i + 4] + e * s[i + 4];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = u[i], b = v[i];
            u[i] = a * c[i] - b * s[i];
            v[i] = b * c[i] + a * s[i];
        }
    }
}

template <bool FP8>
__device__ __forceinline__ uintx2 pack8(float (&f)[8], float inv)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= inv;
    return uintx2{pack4<FP8>(f[0], f[1], f[2], f[3]), pack4<FP8>(f[4], f[5], f[6], f[7])};
}

// a page's scale for values up to `most`
template <bool FP8> __device__ __forceinline__ float new_scale(float most, float before) { return fmaxf(fmaxf(most / kTop<FP8>, FLT_MIN), before); }

template <int DIM, bool FP8>
__device__ __forceinline__ void rescale_page(uint8_t *codes, int slots, float r, int lane, int lanes)
{
    for (int at = lane; at < slots * (DIM / 8); at += lanes) {
        uintx2 *w = (uintx2 *)(codes + at * 8);
        *w = uintx2{rescale4<FP8>((*w)[0], r), rescale4<FP8>((*w)[1], r)};
    }
}

// One page of one head of K or V by one workgroup of page * DIM / 32 lanes (64 at least), 32 elements a lane.  PAIRS: the rotation's
// pairs are whole 8-element pieces and a lane has both halves, so it reads the key once and 2 bytes of table per byte of key; else
// each piece reads its partners too.  STREAM: keys and values are marked as read once.
template <int DIM, bool FP8, bool BF16, bool PAIRS, bool STREAM>
__global__ void __launch_bounds__(512) k_cache_append(AppendArgs a, int page_shift)
{
    constexpr int kRow = DIM / 8;                                         // 8-element pieces of a token
    // workgroups go to the 8 XCDs in turn: a page's heads all go to one, whose L2 then has their rows and angles
    const uint32_t j = blockIdx.x >> 3, which = j % (2 * (uint32_t)a.heads);
    const int value = which >= (uint32_t)a.heads, head = (int)which - (value ? a.heads : 0);
    const int64_t unit = (int64_t)(j / (2 * (uint32_t)a.heads)) * 8 + (blockIdx.x & 7);
    const int b = find_sequence(a.step.offsets, a.step.sequences, page_shift, 2, unit);
    const Piece p = find_piece(a, b, unit - ((int64_t)(a.step.offsets[b] >> page_shift) + 2 * (int64_t)b));
    if (p.count <= 0) return;

    const Rows &x = value ? a.v : a.k;
    const uint16_t *rows = (const uint16_t *)x.ptr + p.token * x.token + head * x.head;
    const int rotary = value ? 0 : a.rotary;
    float f[4][8], most = 0.0f;
    int place[4];                                                         // of a piece's codes in the page; negative: none
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        if constexpr (PAIRS) {
            const int piece = threadIdx.x + j / 2 * blockDim.x, row = piece / (kRow / 2);
            const PairPiece at(piece % (kRow / 2), DIM, rotary, a.interleaved);
            place[j] = row < p.count ? (p.slot + row) * DIM + at.d0 : -1;
            place[j + 1] = row < p.count ? (p.slot + row) * DIM + at.d1 : -1;
            if (row < p.count) {
                const uintx4 *x0 = (const uintx4 *)(rows + row * x.token + at.d0), *x1 = (const uintx4 *)(rows + row * x.token + at.d1);
                widen8<BF16>(STREAM ? __builtin_nontemporal_load(x0) : *x0, f[j]);
                widen8<BF16>(STREAM ? __builtin_nontemporal_load(x1) : *x1, f[j + 1]);
                if (at.pair >= 0) turn8(f[j], f[j + 1], a.table + (p.position + row) * rotary, rotary / 2, at.pair, a.interleaved);
            }
        } else {
#pragma unroll
            for (int i = j; i < j + 2; ++i) {
                const int piece = threadIdx.x + i * blockDim.x, row = piece / kRow, d = piece % kRow * 8;
                place[i] = row < p.count ? (p.slot + row) * DIM + d : -1;
                if (row < p.count) load_turned<BF16>(rows + row * x.token, d, a.table + (p.position + row) * rotary, rotary, a.interleaved, f[i]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (place[j] >= 0)
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(f[j][i]));
    float *scale = (value ? a.cache.v_scales : a.cache.k_scales) + p.id * a.heads + head;
    const float before = p.slot ? *scale : 0.0f;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    __shared__ float waves[8];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x / 64; ++w) most = fmaxf(most, waves[w]);
    const float now = new_scale<FP8>(most, before);
    if (threadIdx.x == 0) *scale = now;

    uint8_t *codes = (value ? a.cache.v : a.cache.k) + (p.id * a.heads + head) * ((int64_t)DIM << page_shift);
    if (p.slot && now > before) rescale_page<DIM, FP8>(codes, p.slot, before / now, threadIdx.x, blockDim.x);
    const float inv = 1.0f / now;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (place[j] >= 0) *(uintx2 *)(codes + place[j]) = pack8<FP8>(f[j], inv);
}

// Single tokens: DIM / 8 lanes for each sequence, head and K or V
template <int DIM, bool FP8, bool BF16>
__global__ void __launch_bounds__(256) k_cache_append_one(AppendArgs a, int page_shift)
{
    constexpr int kLanes = DIM / 8;
    const uint32_t item = (blockIdx.x * 256 + threadIdx.x) / kLanes;
    const int lane = threadIdx.x % kLanes, d = lane * 8;
    const uint32_t pair = item / a.heads, b = pair >> 1;
    const int head = item - pair * a.heads, value = pair & 1;
    if (b >= (uint32_t)a.step.sequences) return;
    const Piece p = find_piece(a, b, 0);
    if (p.count <= 0) return;
    const Rows &x = value ? a.v : a.k;
    float f[8], most = 0.0f;
    const int rotary = value ? 0 : a.rotary;
    load_turned<BF16>((const uint16_t *)x.ptr + p.token * x.token + head * x.head, d, a.table + p.position * rotary, rotary, a.interleaved, f);
    float *scale = (value ? a.cache.v_scales : a.cache.k_scales) + p.id * a.heads + head;
    const float before = p.slot ? *scale : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(f[i]));
#pragma unroll
    for (int m = 1; m < kLanes; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    const float now = new_scale<FP8>(most, before);
    uint8_t *codes = (value ? a.cache.v : a.cache.k) + (p.id * a.heads + head) * ((int64_t)DIM << page_shift);
    if (p.slot && now > before) rescale_page<DIM, FP8>(codes, p.slot, before / now, lane, kLanes);
    if (lane == 0) *scale = now;
    *(uintx2 *)(codes + p.slot * DIM + d) = pack8<FP8>(f, 1.0f / now);
}

template <int DIM, bool FP8, bool BF16>
hipError_t append(const AppendArgs &a, hipStream_t stream)
{
    const int shift = log2_int(a.cache.page);
    if (a.longest == 1) {
        const int64_t lanes = (int64_t)a.step.sequences * 2 * a.heads * (DIM / 8);
        return launch_many(k_cache_append_one<DIM, FP8, BF16>, (lanes + 255) / 256, 256, stream, a, shift);
    }
    const int64_t units = (a.step.tokens >> shift) + 2 * (int64_t)a.step.sequences;
    const int lanes = a.cache.page * DIM / 32 < 64 ? 64 : a.cache.page * DIM / 32;
    const int64_t grid = (units + 7) / 8 * 8 * 2 * a.heads;
    if (a.rotary % 16) return launch_many(k_cache_append<DIM, FP8, BF16, false, false>, grid, lanes, stream, a, shift);
    // us for 32771 tokens of 8 heads of 128 (134 MB) ordinary / as a stream: 45.1 / 42.3; for 4096 tokens 8.9 / 9.8
    return beyond_cache(a.step.tokens * a.heads * DIM * 4) ? launch_many(k_cache_append<DIM, FP8, BF16, true, true>, grid, lanes, stream, a, shift)
                                                           : launch_many(k_cache_append<DIM, FP8, BF16, true, false>, grid, lanes, stream, a, shift);
}

template <int DIM>
hipError_t append_types(const AppendArgs &a, hipStream_t stream)
{
    if (a.fp8) return a.bf16 ? append<DIM, true, true>(a, stream) : append<DIM, true, false>(a, stream);
    return a.bf16 ? append<DIM, false, true>(a, stream) : append<DIM, false, false>(a, stream);
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs &a, hipStream_t stream)
{
    switch (a.dim) {
    case 64: return append_types<64>(a, stream);
    case 128: return append_types<128>(a, stream);
    default: return append_types<256>(a, stream);
    }
}

}  // namespace fc
