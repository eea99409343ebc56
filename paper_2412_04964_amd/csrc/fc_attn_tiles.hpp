// fc_attn_tiles.hpp -- tiles of keys and values in 16 bits in LDS, as the kernels over prompts and over chunks of them have them.
// Internal to the library.
#pragma once

#include "fc_attn.hpp"

namespace fc {
namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));

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

}  // namespace
}  // namespace fc
