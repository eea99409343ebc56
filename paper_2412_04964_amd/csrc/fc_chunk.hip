// fc_chunk.hip -- attention of a chunk of new tokens, at hand in 16 bits, over what their sequences hold in the paged cache of 8-bit codes and
// over themselves.
//
// Query i of a sequence that held L tokens before the step sees the L cached ones, k = sk ck and v = sv cv with the scales of their page
// and head, and the new tokens j <= i:  o = sum_t softmax_t(scale q . k_t) v_t.
// The rows of a key/value head are the queries times the query heads that share it.  A workgroup has 256 of them (or 128), 32 a wavefront, and takes
// 64 tokens at a time, first the cached ones, then the new.  As over prompts a wavefront forms S^T = K Q^T with 32 x 32 x 16 matrix instructions,
// which leaves a lane with weights of the very tokens that it needs as operand of O^T = V^T P^T: scores and weights stay in registers.
//   Both kinds of codes are exact in binary16 and in bfloat16: a tile's codes are converted once, on their way to LDS, for the workgroup's rows.
//   sk multiplies scores.  sv would multiply weights; it goes into their exponents instead, w = 2^(s - top + log2 c), and what sums
//   of weights then have too much is divided out once for 16 tokens.  In bfloat16 c is the part of sv in [1, 2): its power of two multiplies
//   the codes on their way to LDS, which hold it exactly (8 bits, and the exponents of fp32), so that scales of any size stand beside each
//   other.  Binary16 has not the exponents: c is sv / unit, where the unit of the sums is a power of two, common to the workgroup.
//   The unit of a row's weights is its running maximum.  Binary16 has not the range for all that are lower: there it follows a tile's
//   largest score up and down when that is kSlack away, and the largest is put at 2^kBias (kReach below the row's largest at most).
//   Weights are rounded to the type before the products with V, as over prompts: the matrix instructions take both operands in 16 bits, and a
//   second product for the bits that are cut off would make them half as many again.  The sum that divides them is of the unrounded ones.
// All work of the call, in units of a tile of 64 tokens for a workgroup's rows, is cut into equal ranges, one a workgroup: contexts of any lengths
// end together.  Rows that were cut are joined by a second kernel, from results that are normalised.
//   What bounds it.  2048 tokens over 65531, 16 query heads over 2 of 128 in E4M3, bfloat16: 1.09 to 1.17 ms by card, 1.02 PFLOP/s, where a product
//   of 16384^3 reaches 1.36.  A tile takes 4580 cycles (2.25 GHz), which is the sum of 2048 of the matrix units and 2500 of vector instructions: the two
//   wavefronts of a SIMD are mostly at the same of both.  512 tokens over 8191: 60 us, of which 43 are a range's (7.5 the way to the first tile, 35 the
//   16.6 tiles and their end, 2.3 GHz), 10 the join's (34 MB that others wrote, 3.3 TB/s) and the rest the launches'; the first calls after a pause 68, at 1.95
//   GHz.  Nine sequences of 4099 tokens over up to 4000 in signed codes, binary16, 8 heads of 4: 232 to 253 us, 13 of them the join's; a tile with
//   what surrounds the three items of a range 5300 cycles, 1920 of the matrix units and 2890 of vector instructions.  17 tokens over 129: 17 us, in
//   eight workgroups and the join as in one workgroup a head; much of it waits for the code itself, which every launch fetches anew.
//   Taken one after the other: operands ahead of their products (1.59 -> 1.42 ms for the first of these), eight wavefronts over three tiles (1.14, the
//   batch 452 -> 420 us), what surrounds an item counted as work (420 -> 270), items without a division, lanes without LDS (270 -> 240).  Two halves of
//   a workgroup half a tile apart, one at products and one at weights, took as long on the first and 10% longer on the others.
#include <cmath>
#include <type_traits>

#include "fc_attn_tiles.hpp"

namespace fc {
namespace {

constexpr int kTokens = 64;
constexpr int kRanges = 256;            // one for each compute unit
constexpr int kLeast = 2;               // units of a range
constexpr int kShort = 12;              // tiles of an item that need not be cut: sequences may be far shorter than announced
constexpr int kBegin = 3;               // units that what surrounds an item's tiles counts for (the batch below with 2, 3, 4, 6: 281, 270, 274, 276 us)
constexpr double kUnits = 4.5;          // of a range, from which on workgroups have eight wavefronts
constexpr double kJoined = 4.0;         // units that the join counts for
constexpr int rows_of(int waves) { return 32 * waves; }                  // of a workgroup
template <bool BF16> constexpr float kSlack = BF16 ? 8.0f : 10.0f;
constexpr float kBias = 4.0f, kReach = 36.0f;
// Binary16: how far below the largest unit so far the unit may go, and what a scale may be of it.  What fc_cache_append makes of binary16 values is
// between 2^-33 and 2^10 (2^-24 / 448 and 65504 / 127), or the least scale over zeros, so that neither limit is met there.  Both keep the
// sums in range: sums of values grow by 1 / kDeep where the unit falls, from 2^(kBias + kSlack + 9) a token at most; the weight of a token whose
// scale is kFaint of the unit counts up to 2^(kReach + kSlack) / kFaint = 2^102, of which fp32 has room for 2^25.
constexpr float kDeep = 0x1p-42f, kFaint = 0x1p-56f;

// What there is to do for one sequence, for each key/value head: `blocks` of a workgroup's rows, each over `cached` tiles and those new ones that it
// sees, and kBegin units for what surrounds them
struct Job {
    int64_t off, total;                                  // total: units of all blocks
    int blocks, n, held, skip, cached, fresh;            // new tokens; tokens in the cache; new ones without a place; tiles of either kind
};

// Units of new tokens of the first j blocks of ROWS: block i - 1 sees the tokens before ceil(ROWS i / group), so ceil(c i / group) tiles of them, c =
// ROWS / 64.  Every `group` blocks that is c more, and in between one more from each i > k group / c on.
template <int ROWS>
__device__ __forceinline__ int64_t fresh_units(int j, int group)
{
    constexpr int c = ROWS / kTokens;
    const auto some = [&](int r) {
        int sum = r;
#pragma unroll
        for (int k = 1; k < c; ++k) sum += r > k * group / c ? r - k * group / c : 0;
        return sum;
    };
    const int q = (int)((uint32_t)j / (uint32_t)group), r = j - q * group;
    return (int64_t)(c * group) * ((int64_t)q * (q - 1) / 2) + (int64_t)q * some(group) + (int64_t)(c * r) * q + some(r);
}

template <int ROWS>
__device__ __forceinline__ Job job_of(const ChunkArgs &a, int off, int next, int held, int page_shift)
{
    Job j;
    j.off = off;
    j.n = off < 0 || next < off || next > a.step.tokens ? 0 : next - off;
    const int64_t room = (int64_t)a.cache.table_width << page_shift;
    j.held = held < 0 ? 0 : held < room ? held : (int)room;
    j.skip = held < 0 ? -(held + 1) < j.n ? -held : j.n : 0;
    j.cached = (int)(((uint32_t)j.held + kTokens - 1) / kTokens);
    j.fresh = (int)(((uint32_t)j.n + kTokens - 1) / kTokens);
    j.blocks = (int)(((uint32_t)j.n * (uint32_t)a.group + ROWS - 1) / ROWS);             // (tokens * group is below 2^31)
    j.total = j.blocks ? (int64_t)j.blocks * (j.cached + kBegin) + fresh_units<ROWS>(j.blocks - 1, a.group) + j.fresh : 0;
    return j;
}

// units of a block
template <int ROWS>
__device__ __forceinline__ int units_of(const Job &j, int block, int group)
{
    constexpr int c = ROWS / kTokens;
    return j.cached + kBegin + (block == j.blocks - 1 ? j.fresh : (int)(((uint32_t)c * ((uint32_t)block + 1) + group - 1) / (uint32_t)group));
}

template <int ROWS>
__device__ __forceinline__ int64_t units_before(const Job &j, int block, int group)
{
    return block >= j.blocks ? j.total : (int64_t)block * (j.cached + kBegin) + fresh_units<ROWS>(block, group);
}

// the block that has unit u: a guess by the square that its sum nearly is, and the one or two beside it
template <int ROWS>
__device__ __forceinline__ int block_of(const Job &j, int64_t u, int group)
{
    const float slope = (float)(ROWS / kTokens) / (float)group, flat = (float)(j.cached + kBegin) + 0.5f * slope, x = (float)u;
    int block = (int)__builtin_amdgcn_readfirstlane((int)(2.0f * x / (flat + __builtin_sqrtf(flat * flat + 2.0f * slope * x))));
    if (block > j.blocks - 1) block = j.blocks - 1;
    while (block > 0 && units_before<ROWS>(j, block, group) > u) --block;
    while (block < j.blocks - 1 && units_before<ROWS>(j, block + 1, group) <= u) ++block;
    return block;
}

// a / b, where both are mostly small
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) { return (a | b) >> 32 ? a / b : (uint32_t)a / (uint32_t)b; }

// The units of all sequences, one behind the other, cut into ranges that differ by one unit at most; fewer of them where they would have
// less than kLeast units
struct Ranges {
    uint64_t each;
    uint32_t count, longer;                              // the first `longer` of them have one more than `each`
    static __device__ __forceinline__ Ranges of_all(uint64_t total, uint32_t workgroups)
    {
        Ranges r(0, 0);
        const uint64_t most = (total + kLeast - 1) / kLeast;
        r.count = most < workgroups ? (uint32_t)most : workgroups;
        r.each = r.count ? quotient(total, r.count) : 0;
        r.longer = (uint32_t)(total - r.count * r.each);
        return r;
    }
    __device__ __forceinline__ Ranges(uint64_t each_, uint32_t longer_) : each(each_), count(0), longer(longer_) {}
    __device__ __forceinline__ uint64_t begin(uint32_t r) const { return r * each + (r < longer ? r : longer); }
    __device__ __forceinline__ uint32_t of(uint64_t unit) const
    {
        const uint64_t split = longer * (each + 1);
        return (uint32_t)(unit < split ? quotient(unit, each + 1) : longer + quotient(unit - split, each));
    }
};

// v of the lane that CTRL names, 0 where it names none or the lane's row of 16 is not one of ROWS
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t moved(uint64_t v)
{
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)v, CTRL, ROWS, 0xF, ROWS == 0xF);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(v >> 32), CTRL, ROWS, 0xF, ROWS == 0xF);
    return (uint64_t)hi << 32 | lo;
}
// Sums of the lanes up to this one: within 16 lanes, then from the last lane of the 16 before, then from the last of the first 32
__device__ __forceinline__ uint64_t running_sum(uint64_t v)
{
    v += moved<0x111, 0xF>(v);
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);
    return v + moved<0x143, 0xC>(v);
}

// largest of a lane and the one 16 or 32 away in the pairs of rows that change places
template <int FAR>
__device__ __forceinline__ float max_across(float v)
{
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto r = FAR == 32 ? __builtin_amdgcn_permlane32_swap(x, x, false, false) : __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t a = r[0], b = r[1];                   // (a bit cast of an element itself takes the first one's bits)
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
template <int CTRL>
__device__ __forceinline__ float max_with(float v)
{
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)));
}
// largest of all lanes: of 16 by pairs, then mirrored in 8 and in 16
__device__ __forceinline__ float max_of_all(float v)
{
    return max_across<32>(max_across<16>(max_with<0x140>(max_with<0x141>(max_with<0x4E>(max_with<0xB1>(v))))));
}

__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int lane)
{
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lane), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ float lane_f(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

// Where a call gives a workgroup each item: the item of workgroup `id`; units: 0 if it has none
struct Item {
    int b, head, block, units;
};
template <int ROWS>
__device__ __forceinline__ Item item_of(const ChunkArgs &a, uint32_t id, int page_shift)
{
    const int slot = id / (uint32_t)a.heads, head = id - slot * a.heads;
    // sequence b owns the slots from offsets[b] * group / ROWS + b on (these starts leave every sequence room enough, and need nothing but the offsets)
    int lo = 0, hi = a.step.sequences - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((int64_t)a.step.offsets[mid] * a.group / ROWS + mid <= slot) lo = mid;
        else hi = mid - 1;
    }
    const Job job = job_of<ROWS>(a, a.step.offsets[lo], a.step.offsets[lo + 1], a.step.held[lo], page_shift);
    const int64_t block = slot - (job.off * a.group / ROWS + lo);
    if (block < 0 || block >= job.blocks) return {0, 0, 0, 0};
    return {lo, head, (int)block, units_of<ROWS>(job, (int)block, a.group)};
}

// 4 codes of a word -> two words of 16-bit values, which hold either kind exactly; bfloat16: times a power of two
template <bool FP8, bool BF16>
__device__ __forceinline__ uintx2 sixteen(uint32_t w, float power)
{
    asm volatile("" : "+v"(w));                          // (where it stands: the compiler would take all of a lane's together, and wait for them, far ahead)
    if constexpr (!BF16) return halves<FP8>(w);
    else if constexpr (FP8)
        return uintx2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true))};
    else
        return uintx2{narrow2<true>((float)(int8_t)w * power, (float)(int8_t)(w >> 8) * power),
                      narrow2<true>((float)(int8_t)(w >> 16) * power, (float)(int8_t)(w >> 24) * power)};
}

// N matrix instructions whose operands come from LDS: the first AHEAD of them are in `operand`, read(i) is the i-th, and later(j) does what follows
// behind the last read; use(i, operand) executes an instruction, and beside(i) is other work of the wavefront that is issued while the
// matrix unit is at it
template <int N, int AHEAD, typename R, typename L, typename U, typename B>
__device__ __forceinline__ void pipelined(uintx4 (&operand)[AHEAD], const R &read, const L &later, const U &use, const B &beside)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        use(i, operand[i % AHEAD]);
        if (i + AHEAD < N) operand[i % AHEAD] = read(i + AHEAD);
        else later(i + AHEAD - N);
        beside(i);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// W wavefronts have 32 rows each and share the tiles.  Three tiles are in LDS: while one is worked on, the next is whole, and the codes of the one
// behind that are converted; a barrier in the middle of a tile's work is all that they need.
template <int DIM, bool FP8, bool BF16, int W>
__global__ void __launch_bounds__(64 * W, W == 8 ? 2 : 1) k_chunk_attention(ChunkArgs a, int page_shift)
{
    constexpr int kSteps = DIM / 16, kOut = DIM / 32, kRow = 2 * DIM, kTile = kTokens * kRow, kRows = rows_of(W);
    constexpr int kOutRow = kRow + 16;
    constexpr int kAhead = FP8 || BF16 ? 6 : 5;         // operands on their way (4: 1152 us where 6 takes 1138); with signed codes and binary16 6 are no faster
    // A lane loads 16 codes at a time: kLoads of a tile, the first half of them K and the others V (with one load, half of the wavefronts have K)
    constexpr int kLoads = DIM / (8 * W), kEach = kLoads > 1 ? kLoads / 2 : 1, kPieces = DIM / 16, kRound = kTokens / kEach;
    __shared__ __attribute__((aligned(1024))) uint8_t tiles[4][2][kTile];       // K and V
    static_assert(sizeof(tiles) >= W * 32 * kOutRow, "the results fit the tiles");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, side = lane >> 5;
    const int sequences = a.step.sequences, group = a.group;

    // ---- this workgroup's range of all work, or its item ----
    // (What is needed between items only is kept in LDS: the loop over tiles has no registers for it.)
    __shared__ uint64_t kept[3];                         // where this range ends; each and longer of Ranges
    uint64_t at = 0, last_end = 0, each = 0;
    uint32_t range = 0, longer = 0;
    bool cut = false;                                    // an item begins here and goes on behind this range
    int b = -1, head = 0, block = 0, first_unit = 0;     // the next item, and its first unit here
    if (a.by_item) {
        const Item item = item_of<kRows>(a, blockIdx.x, page_shift);
        if (item.units == 0) return;
        b = item.b;
        head = item.head;
        block = item.block;
        last_end = item.units;
    } else {
        uint64_t sum = 0;
        bool astray = false;
        int off = 0, next = 0, held = 0;
        for (int c = 0; c < sequences; c += 64)
            if (c + lane < sequences) {
                off = a.step.offsets[c + lane];
                next = a.step.offsets[c + lane + 1];
                held = a.step.held[c + lane];
                sum += (uint64_t)job_of<kRows>(a, off, next, held, page_shift).total * a.heads;
                astray |= off < 0 || next < off || next > a.step.tokens;
            }
        const uint64_t all = running_sum(sum);
        // (units of offsets that do not ascend may be more than 64 bits count: none of them is done)
        const uint64_t total_units = __any(astray) ? 0 : lane_u64(all, 63);
        const Ranges ranges = Ranges::of_all(total_units, gridDim.x);
        if (blockIdx.x >= ranges.count) {
            if (threadIdx.x == 0) a.cuts[blockIdx.x].pieces = 0;
            return;
        }
        // workgroups go to the 8 XCDs in turn: an XCD gets neighbouring ranges, whose K and V its L2 then holds
        range = ranges.count % 8 == 0 ? (blockIdx.x & 7) * (ranges.count / 8) + (blockIdx.x >> 3) : blockIdx.x;
        at = ranges.begin(range);
        last_end = ranges.begin(range + 1);
        each = ranges.each;
        longer = ranges.longer;
        uint64_t run = 0;
        for (int c = 0; c < sequences; c += 64) {
            uint64_t work = sum, upto = all;
            if (sequences > 64) {
                work = 0;
                if (c + lane < sequences) {
                    off = a.step.offsets[c + lane];
                    next = a.step.offsets[c + lane + 1];
                    held = a.step.held[c + lane];
                    work = (uint64_t)job_of<kRows>(a, off, next, held, page_shift).total * a.heads;
                }
                upto = run + running_sum(work);
            }
            const uint64_t past = __ballot(upto > at);
            if (past) {
                const int l = __builtin_ctzll(past);
                b = c + l;
                const Job job = job_of<kRows>(a, __builtin_amdgcn_readlane(off, l), __builtin_amdgcn_readlane(next, l), __builtin_amdgcn_readlane(held, l), page_shift);
                const uint64_t within = at - lane_u64(upto - work, l);
                head = (int)quotient(within, job.total);
                const int64_t of_head = (int64_t)within - head * job.total;
                block = block_of<kRows>(job, of_head, group);
                first_unit = (int)(of_head - units_before<kRows>(job, block, group));
                break;
            }
            run = lane_u64(upto, 63);
        }
    }

    if (threadIdx.x == 0) {
        kept[0] = last_end;
        kept[1] = each;
        kept[2] = longer;
    }
    __syncthreads();

    // ---- places that do not change ----
    const int stride_k = (int)a.k.token, stride_v = (int)a.v.token;
    // (What is a few operations away from the lane's number is made where it is used: the loop has no registers for it.)
    const auto afresh = [](int v) {
        asm volatile("" : "+v"(v));
        return v;
    };
    const int at_k = col * kRow + (side ^ swizzle<DIM, true>(col)) * 16;
    const int v_row = 4 * side + (lane & 15) / 4;
    const int at_v = v_row * kRow + ((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ swizzle<DIM, false>(v_row)) * 16 + (lane & 1) * 8;
    const float factor = a.scale * 1.4426950408889634f;      // scores in powers of two
    const int half = kLoads == 1 ? wave / (W / 2) : 0, code_wave = kLoads == 1 ? wave % (W / 2) : wave;        // half: 1 for wavefronts that have V only
    const auto code_thread = [&] { return (uint32_t)afresh(kLoads == 1 ? threadIdx.x % (32 * W) : threadIdx.x); };

    while (true) {
        const uint64_t end = lane_u64(kept[0], 0);
        if (at >= end) break;
        const Job job = job_of<kRows>(a, a.step.offsets[b], a.step.offsets[b + 1], a.step.held[b], page_shift);
        if (block >= job.blocks) {                       // the next head, or sequence
            block = 0;
            if (job.blocks == 0 || ++head == a.heads) {
                head = 0;
                ++b;
            }
            continue;
        }
        // ---- the item: a head, a block of rows, and its tiles [tile0, tile1) ----
        const int block_row = block * kRows, units = units_of<kRows>(job, block, group), unit0 = first_unit;
        const uint64_t item = at - unit0;                // its first unit
        const int unit1 = end - at < (uint64_t)(units - unit0) ? unit0 + (int)(end - at) : units;
        at += unit1 - unit0;
        ++block;
        first_unit = 0;
        const int tile0 = unit0 < kBegin ? 0 : unit0 - kBegin, tile1 = unit1 - kBegin;
        if (tile1 <= tile0) continue;                    // none of its tiles
        const bool whole = tile0 == 0 && tile1 == units - kBegin;
        const int rows = job.n * group, row0 = block_row + wave * 32;
        if (tile0 == 0 && !whole) {
            cut = true;
            if (threadIdx.x == 0) {
                const uint32_t last = Ranges(kept[1], (uint32_t)kept[2]).of(item + units - 1);
                a.cuts[range] = {(int)(last - range) + 1, (int)job.off, head, block_row, rows, {0, 0, 0}};
            }
        }
        const int n = job.n, held = job.held, cached = job.cached, skip = job.skip, codes_end = cached < tile1 ? cached : tile1;
        const bool idle = row0 >= rows;                  // this wavefront has no rows

        int query;
        uintx4 qf[kSteps];
        {
            const int row = row0 + col < rows ? row0 + col : rows - 1;
            query = (int)((uint32_t)row / (uint32_t)group);
            const uint16_t *q = (const uint16_t *)a.q.ptr + (job.off + query) * a.q.token + (head * group + (row - query * group)) * a.q.head + side * 8;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) qf[j] = *(const uintx4 *)(q + 16 * j);
        }
        const int32_t *const table = a.cache.table + (int64_t)b * a.cache.table_width;

        // pages of 64 pieces of 16 tokens (16 tiles), one a lane
        const auto pages_of = [&](int batch) {
            const uint32_t token = ((uint32_t)batch * 64 + afresh(lane)) * 16;       // (below 2^31 + 2^11)
            int id = 0;
            if (token < (uint32_t)held) id = table[token >> page_shift];
            return id;
        };
        const auto scales_of = [&](int batch, int id, float &ks, float &vs) {
            const bool there = ((uint32_t)batch * 64 + afresh(lane)) * 16 < (uint32_t)held && id >= 0 && id < a.cache.pages;
            ks = vs = 0.0f;
            if (there) {
                ks = a.cache.k_scales[(int64_t)id * a.heads + head];
                vs = a.cache.v_scales[(int64_t)id * a.heads + head];
            }
        };
        // where they are in the cache
        const auto place_of = [&](int id) {
            if (id < 0 || id >= a.cache.pages) id = 0;
            return ((((uint64_t)id * a.heads + head) << page_shift) + (afresh(lane) * 16 & ((1 << page_shift) - 1))) * DIM;
        };
        uint64_t place = 0;
        int page_next = 0;
        float ks_next = 0.0f, vs_next = 0.0f;
        struct Codes {
            uintx4 w[kLoads];
            float power[kEach];                          // bfloat16: what multiplies V's
        };
        // of a scale, the power of two at or below it
        const auto power_of = [](float scale) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, scale) & 0x7F800000u); };
        // (of tile t, whose pieces' are in the lanes of `powers`; one piece for each of a wavefront's rows of codes)
        const auto raise_codes = [&](Codes &c, int t, float powers) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                c.power[i] = BF16 && (kLoads > 1 || half) ? lane_f(powers, (t & 15) * 4 + (i * kRound + code_wave * (64 / kPieces)) / 16) : 1.0f;
        };
        // the codes of tile t, from memory
        const auto fetch = [&](Codes &c, int t) {
            const int in = t & 15;
            const bool turns = t != tile0 && in == 0;
            if (turns) place = place_of(page_next);
            const uint32_t thread = code_thread(), mine = thread / kPieces % 16 * DIM + thread % kPieces * 16;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const uint64_t at_page = lane_u64(place, in * 4 + (i * kRound + code_wave * (64 / kPieces)) / 16);       // the wavefront's piece
                if constexpr (kLoads == 1) {
                    c.w[0] = *(const uintx4 *)((half ? a.cache.v : a.cache.k) + at_page + mine);
                } else {
                    c.w[i] = *(const uintx4 *)(a.cache.k + at_page + mine);
                    c.w[kEach + i] = *(const uintx4 *)(a.cache.v + at_page + mine);
                }
            }
            // (behind the codes: nothing waits for these until the next codes are there)
            if (turns) page_next = pages_of((t >> 4) + 1);
            if (in == 8) scales_of((t >> 4) + 1, page_next, ks_next, vs_next);
        };
        // and into LDS, 8 codes at a time: half a load
        const auto clear_rest = [&](Codes &c, int t) {
            if ((t + 1) * kTokens > held) {                  // whatever the page holds beyond them
                const int code_row = (int)(code_thread() / kPieces);
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    if (t * kTokens + i % kEach * kRound + code_row >= held) c.w[i] = uintx4{0, 0, 0, 0};
            }
        };
        struct Places {
            int k, v;
        };
        const Places places = [&] {
            const int thread = (int)code_thread(), r = (uint32_t)thread / kPieces, u = 2 * ((uint32_t)thread % kPieces);
            const int k = r * kRow + (u ^ swizzle<DIM, true>(r & 31)) * 16, v = r * kRow + (u ^ swizzle<DIM, false>(r & 15)) * 16 + kTile;
            return kLoads == 1 ? Places{half ? v : k, 0} : Places{k, v};
        }();
        const auto convert = [&](const Codes &c, int piece, uint8_t *to, const Places &at_lds) {
            const int i = piece >> 1, h = piece & 1;
            const float power = kLoads == 1 ? c.power[0] : i >= kEach ? c.power[i % kEach] : 1.0f;
            const uintx2 x = sixteen<FP8, BF16>(c.w[i][2 * h], power), y = sixteen<FP8, BF16>(c.w[i][2 * h + 1], power);
            *(uintx4 *)(to + ((i >= kEach ? at_lds.v : at_lds.k) ^ (h << 4)) + i % kEach * kRound * kRow) = uintx4{x[0], x[1], y[0], y[1]};
        };
        const auto convert_all = [&](const Codes &c, uint8_t *to) {
#pragma unroll
            for (int piece = 0; piece < 2 * kLoads; ++piece) convert(c, piece, to, places);
        };
        // new tokens' tile t, straight to LDS: 16 rows of K and of V a wavefront, or with eight of either
        const auto load_new = [&](int t, uint8_t *to) {
            const int16_t *const k = (const int16_t *)a.k.ptr + job.off * a.k.token + head * a.k.head;
            const int16_t *const v = (const int16_t *)a.v.ptr + job.off * a.v.token + head * a.v.head;
            const int part = wave & 3, t0 = (t - cached) * kTokens + 16 * part, mine = afresh(lane);
            if (W == 4 || wave < 4) {
                const Rows16<DIM, true> rows_k(mine, stride_k);
                rows_k.load(rows16((const uint16_t *)k + (int64_t)t0 * stride_k, stride_k, n - t0, DIM), to + part * 16 * kRow);
            }
            if (W == 4 || wave >= 4) {
                const Rows16<DIM, false> rows_v(mine, stride_v);
                rows_v.load(rows16((const uint16_t *)v + (int64_t)t0 * stride_v, stride_v, n - t0, DIM), to + kTile + part * 16 * kRow);
            }
        };

        floatx16 acc[kOut];
#pragma unroll
        for (int o = 0; o < kOut; ++o)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[o][r] = 0.0f;
        float top = -FLT_MAX, peak = -FLT_MAX, total = 0.0f, unit = 1.0f, largest_unit = 0.0f;

        floatx16 s[2];
        uintx4 pf[4];
        // Operands that are on their way from LDS: V's while the last products with K are made, the next tile's K's beside the last ones with V
        uintx4 kf[kAhead], vf[kAhead];
        const auto read_k = [&](const uint8_t *tile, int i) { return *(const uintx4 *)(tile + (at_k ^ (i / 2 << 5)) + (i & 1) * 32 * kRow); };
        const auto read_v = [&](const uint8_t *tile, int i) {
            const uint8_t *p = tile + kTile + (at_v ^ (i % kOut << 6)) + i / kOut * 16 * kRow;
            const uintx2 lo = transposed(p), hi = transposed(p + 8 * kRow);
            return uintx4{lo[0], lo[1], hi[0], hi[1]};
        };
        const auto scores = [&](const uint8_t *tile) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[h][r] = 0.0f;
            pipelined<2 * kSteps>(kf, [&](int i) { return read_k(tile, i); }, [&](int j) { vf[j] = read_v(tile, j); },
                                  [&](int i, uintx4 x) { s[i & 1] = mma32<BF16>(x, qf[i / 2], s[i & 1]); }, [](int) {});
        };
        // tokens of the tile from `first` on, and before `sees`, are seen
        const auto mask = [&](int first, int sees) {
            const int before = 4 * afresh(side);
            first -= before;
            sees -= before;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = h * 32 + 8 * (r / 4) + r % 4;
                    if (t < first || t >= sees) s[h][r] = -__builtin_inff();
                }
        };
        // The pieces of 16 tokens that the lanes have the scales of: what scores are multiplied by (powers of two), what is added to the
        // exponents for the values' scales, and what sums of weights are multiplied by for that
        float steep = 0.0f, raise = 0.0f, back = 0.0f, powers = 0.0f;
        const auto turn_to = [&](float key_scale, float value_scale) {
            float c;
            if constexpr (BF16) {
                powers = power_of(value_scale);
                c = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, value_scale) & 0x7FFFFFu) | 0x3F800000u);
            } else {
                const float widest = fmaxf(fminf(max_of_all(value_scale), 0x1p126f), FLT_MIN);
                // the unit of the sums: the power of two at or below the largest scale, or kDeep of the largest unit so far
                const float now = fmaxf(__builtin_amdgcn_ldexpf(1.0f, __builtin_amdgcn_frexp_expf(widest) - 1), fmaxf(largest_unit * kDeep, FLT_MIN));
                if (now != unit) {
                    const float change = unit / now;
#pragma unroll
                    for (int o = 0; o < kOut; ++o) acc[o] *= change;
                    unit = now;
                }
                largest_unit = fmaxf(largest_unit, now);
                c = fmaxf(value_scale / unit, kFaint);
            }
            steep = fmaxf(factor * key_scale, FLT_MIN);
            raise = __builtin_amdgcn_logf(c);            // log2
            back = 1.0f / c;
        };
        const auto raise_maxima = [&](int piece) {
            float most = -__builtin_inff();
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                float m = s[p / 2][8 * (p & 1)];
#pragma unroll
                for (int r = 1; r < 8; ++r) m = fmaxf(m, s[p / 2][8 * (p & 1) + r]);
                most = fmaxf(most, __builtin_fmaf(m, lane_f(steep, piece + p), lane_f(raise, piece + p)));
            }
            bool away;
            if constexpr (BF16) {
                away = most > top + kSlack<BF16>;
            } else {
                most = max_across<32>(most) - kBias;
                away = fabsf(most - top) > kSlack<BF16>;
            }
            if (__any(away)) {
                if constexpr (BF16) most = max_across<32>(most);
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
        };
        // The weights of 16 tokens are made beside the products of the 16 before them, and beside the last products the codes of the tile after
        // the next one are converted
        const auto add_values = [&](const uint8_t *tile, const uint8_t *behind, int piece, auto convert_codes, const Codes &c, uint8_t *to) {
            float part = 0.0f;
            const auto weigh = [&](int p, int pair) {
                const float fk = lane_f(steep, piece + p), add = lane_f(raise, piece + p) - top;
                const int r = 8 * (p & 1) + 2 * pair;
                const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[p / 2][r], fk, add)), w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[p / 2][r + 1], fk, add));
                part = pair ? part + (w0 + w1) : w0 + w1;
                pf[p][pair] = narrow2<BF16>(w0, w1);
                if (pair == 3) total = __builtin_fmaf(part, lane_f(back, piece + p), total);
            };
#pragma unroll
            for (int pair = 0; pair < 4; ++pair) weigh(0, pair);
            pipelined<4 * kOut>(vf, [&](int i) { return read_v(tile, i); }, [&](int j) { kf[j] = read_k(behind, j); },
                                [&](int i, uintx4 x) { acc[i % kOut] = mma32<BF16>(x, pf[i / kOut], acc[i % kOut]); },
                                [&](int i) {
                                    // beside each instruction 4 / kOut pairs of weights, or, for the last 16 tokens, 2 kLoads / kOut halves of loads
                                    if (i < 3 * kOut) {
#pragma unroll
                                        for (int j = i % kOut * 4 / kOut; j < (i % kOut + 1) * 4 / kOut; ++j) weigh(i / kOut + 1, j);
                                    } else if constexpr (decltype(convert_codes)::value) {
#pragma unroll
                                        for (int j = (i - 3 * kOut) * 2 * kLoads / kOut; j < (i - 3 * kOut + 1) * 2 * kLoads / kOut; ++j) convert(c, j, to, places);
                                    }
                                });
        };
        // In a tile that not all rows see whole, an infinity or NaN among the new values would be NaN times the weight of 0 of those that do
        // not.  Such values are added to the rows that see them, and taken out of the tile.
        const auto not_finite = [](uint32_t w) { return (w & 0x7FFF7FFFu) + (BF16 ? 0x00800080u : 0x04000400u); };      // in the sign bits of w's halves
        const auto finite_only = [&](uint32_t w) { return w & ~(((not_finite(w) & 0x80008000u) >> 15) * 0xFFFFu); };
        const auto any_not_finite = [&](const uint8_t *lds_v) {
            uint32_t any = 0;
            const int mine = afresh(lane);
#pragma unroll 4
            for (int i = 0; i < kTile / 1024; ++i) {
                const uintx4 w = *(const uintx4 *)(lds_v + i * 1024 + mine * 16);
                any |= not_finite(w[0]) | not_finite(w[1]) | not_finite(w[2]) | not_finite(w[3]);
            }
            return __any(any & 0x80008000u) != 0;
        };
        const auto add_not_finite = [&](const uint8_t *lds_v, int t0) {
            const int my_side = afresh(side);
#pragma unroll 1
            for (int t = 0; t < kTokens; ++t) {
                const uint8_t *p = lds_v + t * kRow + my_side * 8;
                const bool seen = t0 + t <= query && t0 + t >= skip;
#pragma unroll
                for (int o = 0; o < kOut; ++o)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const uintx2 w = *(const uintx2 *)(p + ((o * 4 + r / 4) ^ swizzle<DIM, false>(t & 15)) * 16);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t bits = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
                            if (seen && (not_finite(bits) & 0x8000u)) acc[o][r + i] += widen<BF16>(bits);
                        }
                    }
            }
        };

        // ---- the tiles ----
        // everything that this wavefront has written to LDS, or (loads) sent there straight from memory, is there, and the others' too
        const auto arrived = [](bool loads) {
            if (loads) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        };
        uint8_t *now = &tiles[0][0][0], *next = &tiles[1][0][0], *after = &tiles[2][0][0];
        Codes codes = {};
        const auto pass_on = [&] {
            uint8_t *const free = now;
            now = next;
            next = after;
            after = free;
        };
        // the powers of tile t's batch, where `batch` is the one that was turned to: it, or the next one
        const auto powers_at = [&](int t, int batch) { return t >> 4 == batch ? powers : power_of(vs_next); };
        if (tile0 < cached) {
            const int batch = tile0 >> 4, page = pages_of(batch);
            place = place_of(page);
            page_next = pages_of(batch + 1);
            float ks, vs;
            Codes first;
            fetch(first, tile0);
            scales_of(batch, page, ks, vs);
            scales_of(batch + 1, page_next, ks_next, vs_next);     // (before the next fetch may go on to that batch)
            if (tile0 + 1 < codes_end) fetch(codes, tile0 + 1);
            turn_to(ks, vs);
            clear_rest(first, tile0);
            raise_codes(first, tile0, powers);
            convert_all(first, now);
            if (tile0 + 1 < codes_end) {
                clear_rest(codes, tile0 + 1);
                raise_codes(codes, tile0 + 1, powers_at(tile0 + 1, batch));
                convert_all(codes, next);
                if (tile0 + 2 < codes_end) {
                    raise_codes(codes, tile0 + 2, powers_at(tile0 + 2, batch));
                    fetch(codes, tile0 + 2);
                }
            }
        } else {
            turn_to(1.0f, 1.0f);
            load_new(tile0, now);
        }
        if (tile0 + 1 < tile1 && tile0 + 1 >= cached) load_new(tile0 + 1, next);
        // the queries are here before the loop, where waiting for them would wait for what is loaded ahead
#pragma unroll
        for (int j = 0; j < kSteps; ++j) asm volatile("" : "+v"(qf[j]));
        arrived(true);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) kf[j] = read_k(now, j);
        int t = tile0;
        for (; t < codes_end; ++t) {
            if ((t & 15) == 0 && t != tile0) turn_to(ks_next, vs_next);
            if (!idle) scores(now);
            // the next tile is whole, and the one before this one is done with
            arrived(t + 1 >= cached);
            // (where there are no more codes the last ones go to a tile that nobody reads: one form of the products is enough)
            uint8_t *const to = t + 2 < codes_end ? after : &tiles[3][0][0];
            if (t + 2 < codes_end) clear_rest(codes, t + 2);
            else if (t + 2 < tile1) load_new(t + 2, after);
            if (!idle) {
                if ((t + 1) * kTokens > held) mask(0, held - t * kTokens);
                raise_maxima((t & 15) * 4);
                add_values(now, next, (t & 15) * 4, std::true_type(), codes, to);
            } else {
                convert_all(codes, to);
            }
            // (all that was loaded ahead is here by now; said here, where it costs nothing, and not between the next loads)
            asm volatile("" : "+v"(page_next), "+v"(ks_next), "+v"(vs_next));
            if (t + 3 < codes_end) {
                raise_codes(codes, t + 3, powers_at(t + 3, t >> 4));
                fetch(codes, t + 3);
            }
            pass_on();
        }
        if (t < tile1 && t != tile0) turn_to(1.0f, 1.0f);
        const int first_query = (int)((uint32_t)block_row / (uint32_t)group);      // of the workgroup
        const int wave_first = (int)((uint32_t)(row0 < rows ? row0 : rows - 1) / (uint32_t)group), wave_last = (int)((uint32_t)(row0 + 31 < rows ? row0 + 31 : rows - 1) / (uint32_t)group);
        for (; t < tile1; ++t) {
            const int t0 = (t - cached) * kTokens;
            const bool sees = !idle && t0 <= wave_last;
            if (sees) scores(now);
            arrived(true);
            if (t + 2 < tile1) load_new(t + 2, after);
            if (sees) {
                if (t0 + kTokens - 1 > wave_first || t0 < skip) mask(skip - t0, query + 1 - t0);
                raise_maxima(0);
            }
            if ((t0 + kTokens - 1 > first_query || t0 < skip) && any_not_finite(now + kTile)) {           // the same for all wavefronts
                uint8_t *const lds_v = now + kTile;
                const int mine = afresh(lane);
                if (sees) add_not_finite(lds_v, t0);
                arrived(false);
#pragma unroll 1
                for (int i = 0; i < kTile / 1024 / W; ++i) {
                    uintx4 *const place = (uintx4 *)(lds_v + (wave * (kTile / 1024 / W) + i) * 1024 + mine * 16);
                    const uintx4 w = *place;
                    *place = uintx4{finite_only(w[0]), finite_only(w[1]), finite_only(w[2]), finite_only(w[3])};
                }
                arrived(false);
#pragma unroll
                for (int j = 0; j < kAhead; ++j) vf[j] = read_v(now, j);
            }
            if (sees) add_values(now, next, 0, std::false_type(), codes, after);
            pass_on();
        }

        total += __shfl_xor(total, 32);
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        if (whole) {
            // through LDS, where the tiles are done with, so that a wavefront stores whole rows (a lane has 4 elements of a row at a time)
            __syncthreads();
            const int here = afresh(lane), col = here & 31, side = here >> 5;
            uint8_t *const mine = &tiles[0][0][0] + wave * 32 * kOutRow;                  // neighbouring rows begin 4 banks apart
            constexpr int kLanes = DIM / 8;                  // of a row
#pragma unroll
            for (int o = 0; o < kOut; ++o)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *(uintx2 *)(mine + col * kOutRow + (o * 32 + 2 * r + 4 * side) * 2) =
                        uintx2{narrow2<BF16>(acc[o][r] * inv * unit, acc[o][r + 1] * inv * unit), narrow2<BF16>(acc[o][r + 2] * inv * unit, acc[o][r + 3] * inv * unit)};
#pragma unroll
            for (int i = 0; i < 32 * kLanes / 64; ++i) {
                const int out_row = i * (64 / kLanes) + here / kLanes, d = here % kLanes * 8;
                const uintx4 w = *(const uintx4 *)(mine + out_row * kOutRow + d * 2);
                const int r = row0 + out_row, q = (int)((uint32_t)r / (uint32_t)group);
                if (r < rows) *(uintx4 *)((uint16_t *)a.out.ptr + (job.off + q) * a.out.token + (head * group + (r - q * group)) * a.out.head + d) = w;
            }
        } else {
            // as the lanes have them: [place][wavefront][4 elements of each][lane]
            const int64_t place = ((int64_t)range * 2 + (tile0 == 0)) * W + wave, places = (int64_t)gridDim.x * 2 * W;
            floatx4 *const y = (floatx4 *)a.partial + place * (32 * DIM / 4);
            const int mine = afresh(lane);
            if (!idle)
#pragma unroll
            for (int o = 0; o < kOut; ++o)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    y[(o * 4 + r / 4) * 64 + mine] = floatx4{acc[o][r] * inv * unit, acc[o][r + 1] * inv * unit, acc[o][r + 2] * inv * unit, acc[o][r + 3] * inv * unit};
            if (!idle && mine < 32) ((floatx2 *)(a.partial + places * (32 * DIM)))[place * 32 + mine] = floatx2{top, total};
        }
        __syncthreads();                                     // before the next item's tiles
    }
    if (!a.by_item && !cut && threadIdx.x == 0) a.cuts[range].pieces = 0;
}

// Joins what the ranges have of the items that were cut: a wavefront has 8 elements of 32 rows of the item that begins in range `first` and goes on
// behind it.  A range has two places: 1 for an item that it begins and does not end, 0 for one that began before.
template <int DIM, bool BF16, int W>
__global__ void __launch_bounds__(256) k_chunk_join(ChunkArgs a)
{
    constexpr int kEighths = DIM / 8;
    const int lane = threadIdx.x & 63, col = lane & 31, side = lane >> 5;
    const uint32_t id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = id / (W * kEighths);
    const int wave = id / kEighths % W, eighth = id % kEighths;
    const ChunkCut cut = a.cuts[first];
    if (cut.pieces == 0) return;
    const int rows = cut.rows, row0 = cut.row + wave * 32, row = row0 + col, head = cut.head;
    if (row0 >= rows) return;
    const int64_t places = (int64_t)a.workgroups * 2 * W;
    const floatx4 *const x = (const floatx4 *)a.partial + eighth * 64 + lane;
    const floatx2 *const m = (const floatx2 *)(a.partial + places * (32 * DIM)) + col;
    float best = -FLT_MAX, total = 0.0f;
    floatx4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    // N pieces on their way at a time; those behind the last one are it again, and count for nothing
    const auto add = [&](auto pieces, int r0) {
        constexpr int N = decltype(pieces)::value;
        floatx4 y[N];
        floatx2 one[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int r = r0 + k < cut.pieces ? r0 + k : cut.pieces - 1;
            const int64_t place = ((int64_t)(first + r) * 2 + (r == 0)) * W + wave;      // (the first range has it in its second place)
            one[k] = m[place * 32];
            y[k] = x[place * (32 * DIM / 4)];
        }
        float now = best;
#pragma unroll
        for (int k = 0; k < N; ++k) now = fmaxf(now, one[k][0]);
        const float shrink = __builtin_amdgcn_exp2f(best - now);
        best = now;
        total *= shrink;
        sum *= shrink;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float w = r0 + k < cut.pieces ? __builtin_amdgcn_exp2f(one[k][0] - best) * one[k][1] : 0.0f;
            total += w;
            if (w != 0.0f) sum += y[k] * w;
        }
    };
    if (cut.pieces <= 2) add(std::integral_constant<int, 2>(), 0);
    else
        for (int r = 0; r < cut.pieces; r += 8) add(std::integral_constant<int, 8>(), r);
    if (row >= rows) return;
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const int q = (int)((uint32_t)row / (uint32_t)a.group);
    *(uintx2 *)((uint16_t *)a.out.ptr + (int64_t)(cut.off + q) * a.out.token + (int64_t)(head * a.group + (row - q * a.group)) * a.out.head + 8 * eighth + 4 * side) =
        uintx2{narrow2<BF16>(sum[0] * inv, sum[1] * inv), narrow2<BF16>(sum[2] * inv, sum[3] * inv)};
}

int64_t slots_of(int64_t tokens, int group, int sequences, int waves) { return tokens * group / rows_of(waves) + sequences; }

template <int DIM, bool FP8, bool BF16, int W>
hipError_t chunk(const ChunkArgs &a, hipStream_t stream)
{
    const int shift = a.cache.page == 16 ? 4 : a.cache.page == 32 ? 5 : 6;
    const int64_t grid = a.by_item ? slots_of(a.step.tokens, a.group, a.step.sequences, W) * a.heads : a.workgroups;
    const hipError_t e = launch_many(k_chunk_attention<DIM, FP8, BF16, W>, grid, 64 * W, stream, a, shift);
    if (e != hipSuccess || a.by_item || a.workgroups == 1) return e;
    return launch_many(k_chunk_join<DIM, BF16, W>, ((int64_t)a.workgroups - 1) * W * (DIM / 8) / 4, 256, stream, a);
}

template <int DIM, bool FP8, bool BF16>
hipError_t chunk_of(const ChunkArgs &a, hipStream_t stream)
{
    return a.waves == 8 ? chunk<DIM, FP8, BF16, 8>(a, stream) : chunk<DIM, FP8, BF16, 4>(a, stream);
}

template <int DIM>
hipError_t chunk_of(const ChunkArgs &a, hipStream_t stream)
{
    if (a.fp8) return a.bf16 ? chunk_of<DIM, true, true>(a, stream) : chunk_of<DIM, true, false>(a, stream);
    return a.bf16 ? chunk_of<DIM, false, true>(a, stream) : chunk_of<DIM, false, false>(a, stream);
}

}  // namespace

// Times in what follows: keys and values of 8 heads of 128 in E4M3, bfloat16, 4 query heads each.
void chunk_plan(int64_t tokens, int sequences, int heads, int group, int64_t longest, ChunkArgs *a)
{
    const double all_rows = (double)tokens * group, tiles = (double)longest / kTokens + 2;
    const auto items = [&](int waves) { return std::fmax(sequences, all_rows / rows_of(waves) + 0.5 * sequences) * heads; };
    const auto units = [&](int waves) { return items(waves) * (tiles + kBegin) / kRanges; };             // of a range
    // Eight wavefronts convert a tile's codes for twice the rows; four leave more ranges to share the rows.  One sequence over 4000 tokens, 8 / 4 wavefronts:
    // 160 rows 33.3 / 28.7 us, 256 34.2 / 31.4, 384 35.5 / 36.0, 512 38.6 / 38.8; eight over 1000 to 2000 tokens: 64 rows each 27.6 / 29.0, 256 42.2 / 47.4
    a->waves = units(8) >= kUnits ? 8 : 4;
    // Short contexts: a workgroup for each item, and nothing to join, unless ranges would end that much sooner.  By items / by ranges: 2 items of 3 tiles
    // 12.5 / 16.3 us, of 6 20.1 / 16.7, of 11 28.7 / 17.5; about 190 items of 6 tiles 31.0 / 38.1, of 11 42.0 / 41.6
    const double slots = (double)slots_of(tokens, group, sequences, a->waves);
    a->by_item = tiles <= kShort && tiles * std::ceil(items(a->waves) / kRanges) <= units(a->waves) + kJoined && slots * heads * 512 < 4294967296.0;
    // else one for each of 256 compute units, or fewer where the announced lengths cannot make so many ranges
    const double most = slots * heads * (tiles + kBegin) / kLeast + 1;
    a->workgroups = a->by_item ? 0 : most < kRanges ? (int)most : kRanges;
}

size_t chunk_workspace(const ChunkArgs &a, int dim)
{
    return (size_t)a.workgroups * (sizeof(ChunkCut) + (a.workgroups > 1 ? 2 * rows_of(a.waves) * (dim + 2) * sizeof(float) : 0));
}

hipError_t launch_chunk_attention(const ChunkArgs &a, hipStream_t stream)
{
    return a.dim == 64 ? chunk_of<64>(a, stream) : chunk_of<128>(a, stream);
}

}  // namespace fc
