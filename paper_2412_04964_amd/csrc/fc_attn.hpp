// fc_attn.hpp -- what the attention units share: element types, matrix instructions, the step of a batch (which tokens
// belong to which sequence), and their launch functions.  Internal to the library; the interface is include/fc.h.
#pragma once

#include <hip/hip_runtime.h>
#include <float.h>
#include <stdint.h>

#include "fc_launch.hpp"

namespace fc {

// A [tokens, heads, dim] tensor of 16-bit elements whose last axis is dense; strides in elements
struct Rows {
    void *ptr;
    int64_t token, head;
};

// The tokens that one call adds: sequence b has tokens offsets[b] .. offsets[b + 1] of the packed ones and held[b] before them
struct Step {
    const int32_t *offsets, *held;
    int sequences;
    int64_t tokens;
};

// The paged cache: codes [pages, heads, page, dim], scales [pages, heads]; table[b][i] is the page of a sequence's tokens
// [i * page, (i + 1) * page)
struct Cache {
    uint8_t *k, *v;
    float *k_scales, *v_scales;
    const int32_t *table;
    int64_t pages;
    int page, table_width;
};

// An input that does not fit the 256 MB memory-side cache beside what is made of it; smaller ones have just been written there.
inline bool beyond_cache(double bytes) { return bytes > 128 << 20; }

// Launches of `workgroups` workgroups of `lanes`, unless they are more than the runtime takes (2^32 - 1 lanes)
constexpr hipError_t kTooLarge = hipErrorInvalidConfiguration;
inline bool launchable(int64_t workgroups, int lanes) { return workgroups <= ((int64_t)1 << 32) / lanes - 1; }
template <typename K, typename... A>
inline hipError_t launch_many(K *kernel, int64_t workgroups, int lanes, hipStream_t stream, A... a)
{
    return launchable(workgroups, lanes) ? launch_kernel(kernel, dim3((uint32_t)workgroups), dim3(lanes), stream, a...) : kTooLarge;
}

struct RotaryArgs {
    Rows x, y;
    const float *table;
    int64_t table_rows, tokens;
    const int32_t *positions;
    int heads, dim, rotary, interleaved, inverse, bf16;
};
hipError_t launch_rotary_table(const double *frequencies, int64_t rows, int rotary, double magnitude, float *table, hipStream_t stream);
hipError_t launch_rotary(const RotaryArgs &a, hipStream_t stream);

struct AppendArgs {
    Rows k, v;
    Step step;
    Cache cache;
    const float *table;
    int64_t table_rows, longest;
    int heads, dim, rotary, interleaved, fp8, bf16;
};
hipError_t launch_cache_append(const AppendArgs &a, hipStream_t stream);

struct CacheAttentionArgs {
    Rows q, out;
    Step step;
    Cache cache;
    // [places, dim] sums, then [places, 2] maxima and weights.  Places: [workgroups, 2, rows of a workgroup] of equal ranges (see the join);
    // [tokens, query heads, splits] of pieces
    float *partial;
    float scale;
    int heads, group, dim, fp8, bf16;
    // cache_attention_plan's: 16-row tiles that a workgroup takes; workgroups that share all sequences' contexts evenly, or 0: one for each
    // head and sequence, and for each of `row_blocks` of its rows; whether codes are read once
    int row_tiles, row_blocks, workgroups, splits, stream;
    uint32_t *plan;            // how many units there are, and where each sequence's begin
};
void cache_attention_plan(int sequences, int heads, int group, int dim, int64_t queries, int64_t longest, CacheAttentionArgs *a);
size_t cache_attention_workspace(const CacheAttentionArgs &a, int64_t tokens, int sequences, int query_heads, int dim);
hipError_t launch_cache_attention(const CacheAttentionArgs &a, hipStream_t stream);

struct PromptArgs {
    Rows q, k, v, out;
    const int32_t *offsets;
    int64_t tokens, longest;
    float scale;
    int sequences, heads, group, dim, causal, bf16;
};
hipError_t launch_prompt_attention(const PromptArgs &a, hipStream_t stream);

// An item of the work below that begins in one range and ends in another: in how many it lies (0: there is none), its sequence's first token, its
// head, and its first row and the number of rows of its sequence
struct ChunkCut {
    int pieces, off, head, row, rows, pad[3];
};

// Attention of the step's new tokens, which are at hand in 16 bits, over what their sequences hold in the cache and over themselves
struct ChunkArgs {
    Rows q, k, v, out;
    Step step;
    Cache cache;
    // of the items that more than one workgroup has a part of: [workgroups, 2, rows of a workgroup] of normalised results, then maxima and weights
    float *partial;
    ChunkCut *cuts;                                     // [workgroups]: what each range begins and does not end
    float scale;
    int heads, group, dim, fp8, bf16;
    int waves, by_item, workgroups;                     // chunk_plan's: wavefronts of a workgroup, with 32 rows each; whether each item has a workgroup; or ranges of the work
};
void chunk_plan(int64_t tokens, int sequences, int heads, int group, int64_t longest, ChunkArgs *a);
size_t chunk_workspace(const ChunkArgs &a, int dim);
hipError_t launch_chunk_attention(const ChunkArgs &a, hipStream_t stream);

// The norm of rows [tokens, hidden]; strides in elements
struct NormArgs {
    const void *x, *residual, *weight;                  // residual may be null
    void *sum, *y;                                      // sum may be null; y: 16-bit rows, or codes
    float *scales;
    int64_t x_row, residual_row, sum_row, y_row, tokens;
    double eps;
    int hidden, group, codes, bf16, weight_f32;         // codes: 0 for 16 bits, or kSigned, kE4M3
};
enum { kWide16 = 0, kSigned = 1, kE4M3 = 2 };
hipError_t launch_rms_norm(const NormArgs &a, hipStream_t stream);

// Page tables [sequences, width], pages in use by count, and the pairs of pages that a call has copied
struct ForkArgs {
    const int32_t *table, *held, *parents;
    int32_t *uses, *table_out, *held_out;
    int64_t pages;
    int sequences, rows, width, page;                   // rows: of the new table
};
hipError_t launch_pages_fork(const ForkArgs &a, hipStream_t stream);

struct ReserveArgs {
    int32_t *table, *uses, *source, *target, *lacking, *fresh;        // fresh: [pages], scratch
    const int32_t *held, *offsets;
    int64_t pages;
    int sequences, width, page;
};
hipError_t launch_pages_reserve(const ReserveArgs &a, hipStream_t stream);

struct CompactArgs {
    const int32_t *table, *uses;
    int32_t *table_out, *uses_out, *source, *target, *used, *counts, *rank;        // counts, rank: scratch
    int64_t pages, entries;                             // entries: of the table
};
constexpr int kSegment = 4096;                          // pages that a workgroup counts
hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t stream);

struct CopyArgs {
    uint8_t *k, *v;
    float *k_scales, *v_scales;
    const int32_t *source, *target;
    int64_t pages, count, bytes;                        // bytes: of a page in one of the caches
    int heads;
};
hipError_t launch_cache_copy(const CopyArgs &a, hipStream_t stream);

#if defined(__HIPCC__)

typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 brain2 __attribute__((ext_vector_type(2)));
typedef __bf16 brain8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

// the two 16-bit element types
template <bool BF16> struct Element;
template <> struct Element<false> {
    typedef _Float16 one;
    typedef half2 two;
    typedef half8 eight;
};
template <> struct Element<true> {
    typedef __bf16 one;
    typedef brain2 two;
    typedef brain8 eight;
};

template <bool BF16>
__device__ __forceinline__ float widen(uint32_t bits16)
{
    if constexpr (BF16) return __builtin_bit_cast(float, bits16 << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
}

// 8 elements of 16 bits <-> fp32
template <bool BF16>
__device__ __forceinline__ void widen8(uintx4 w, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = widen<BF16>(w[i] & 0xFFFFu);
        f[2 * i + 1] = widen<BF16>(w[i] >> 16);
    }
}

// two fp32 values rounded to nearest, ties to even
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float a, float b)
{
    const floatx2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, typename Element<BF16>::two));
}

template <bool BF16>
__device__ __forceinline__ uintx4 narrow8(const float (&f)[8])
{
    return uintx4{narrow2<BF16>(f[0], f[1]), narrow2<BF16>(f[2], f[3]), narrow2<BF16>(f[4], f[5]), narrow2<BF16>(f[6], f[7])};
}

// what the largest magnitude of a scale's values becomes
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

// D[32][32] += A[32][16] B[16][32].  Lane l holds row (A) or column (B) l % 32, contraction indices 8 (l / 32) + 0..7; of the result
// column l % 32, rows 8 (r / 4) + 4 (l / 32) + r % 4 for r = 0..15.
template <bool BF16>
__device__ __forceinline__ floatx16 mma32(uintx4 a, uintx4 b, floatx16 c)
{
    typedef typename Element<BF16>::eight V;
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}

// D[16][16] += A[16][32] B[32][16] in binary16.  Lane l holds row (A) or column (B) l % 16, contraction indices 8 (l / 16) + 0..7;
// of the result column l % 16, rows 4 (l / 16) + 0..3.
__device__ __forceinline__ floatx4 mma16(uintx4 a, uintx4 b, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// 16 bytes per lane from memory to lds + 16 lane.  Not the builtin: the compiler would make LDS reads of what has arrived wait for what is
// on its way.  Who reads it waits for vmcnt himself, and has read what was there before.  (A wait state between the write of m0, which
// the compiler keeps nothing in, and its use.)  m0 holds the address: the kernels go up to 128 KB (prompts, split tokens).  STREAM: marked as read once.
template <bool STREAM>
__device__ __forceinline__ void load_to_lds(uintx4 rsrc, int offset, uint32_t lds)
{
    if constexpr (STREAM) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(offset), "s"(rsrc) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(rsrc) : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// A buffer resource of `bytes` from `base` on, which all lanes share; beyond them reads are zero
__device__ __forceinline__ uintx4 resource(const void *base, uint32_t bytes)
{
    const uint64_t at = (uint64_t)base;
    return uintx4{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, 0x00020000u};
}

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

// until no more than N of this wavefront's loads are on their way
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Which sequence has work unit u, where sequence b has at most (tokens of b) / 2^shift + extra units and therefore owns the numbers
// from offsets[b] / 2^shift + extra b on (these starts leave every sequence room enough, and need nothing but the offsets).
__device__ __forceinline__ int find_sequence(const int32_t *__restrict__ offsets, int sequences, int shift, int extra, int64_t u)
{
    int lo = 0, hi = sequences - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((int64_t)(offsets[mid] >> shift) + (int64_t)extra * mid <= u) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

#endif  // __HIPCC__

}  // namespace fc
