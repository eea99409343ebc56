// fc_cache_attn.hip -- attention over the paged cache of 8-bit codes.
//
// Query i of a sequence that held L tokens before the step sees the tokens t < L + i + 1:
//     w_t = exp(scale q . (sk ck_t) - max),  o = sum w_t sv cv_t / sum w_t
// with the scales sk, sv of t's page and head.  Codes of either kind are exact in binary16, so the products run on codes: sk multiplies
// the score and sv the weight.  Rows of the matrix products are the queries of a sequence times the query heads that share a
// key/value head (16 rows); the transposed score S^T = K Q^T leaves a lane with the weights of the tokens that it needs again as the
// operand of O^T = V^T P^T, so scores and weights never leave the registers.
//   Queries are scaled by a power of two per row so that they fit binary16 (bfloat16's 8 bits stay exact over 2^28 below a row's largest).
//   Weights are rounded to binary16 as p sv / ref, where ref is the row's largest p sv so far or less by kMost: 11 bits.
//   The running maximum is raised only when a score passes it by kSlack, and ref by kMost: the sums carry the same factors either way.
// The context is split over workgroups and their wavefronts, each with its own maximum and sums; wavefronts are joined in LDS,
// workgroups by a second kernel through the workspace (cache_attention_plan says which contexts are, and how).
// Memory bounds large batches: 2 bytes per token, head and element against 2 multiply-adds for each query head.  64 x 8 contexts of up to
// 8192 tokens, 807 MB: 138 us, 5.9 TB/s, where a bare stream of such pieces reaches 6.8.  Few requests are bound by latency: 8 of 1536 tokens
// 11.7 us, two launches and in each a chain of three reads; a lone step of a wavefront takes 1.2 us for its 250 to 350 vector instructions.
#include "fc_attn.hpp"

namespace fc {
namespace {

constexpr int64_t kMaxContext = 0x7FFF0000;
constexpr float kSlack = 8.0f;          // in powers of two
constexpr float kMost = 65504.0f, kAim = 4096.0f;
constexpr float kLow = 0x1p-40f, kHigh = 0x1p10f;     // what scales of values ordinarily lie between
constexpr int kLeast = 8;               // units of a range
constexpr int kPiece = 4;               // of a piece, at least (8: 16 contexts of 1536 tokens 12.4 us instead of 11.7)

constexpr int waves_of(int dim, int row_tiles) { return dim < 256 && row_tiles == 1 ? 8 : 4; }      // of a workgroup for a whole context
constexpr int kTile = 16;               // tokens of a matrix instruction; a page holds whole tiles

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

// byte i of four words -> word i
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4])
{
    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    out[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
}

__device__ __forceinline__ float lane_f(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[1]) { w[0] = *(const uint32_t *)p; }
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[2])
{
    const uintx2 x = *(const uintx2 *)p;
    w[0] = x[0];
    w[1] = x[1];
}
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[4])
{
    const uintx4 x = *(const uintx4 *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
}

// until no more than N of this wavefront's loads are on their way
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// over the four lanes that share l % 16
__device__ __forceinline__ float max4(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float sum4(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }

// What there is to do for one sequence: its queries and context, and in units of a pair of tiles for each head and block of rows.  A
// sequence without context has one unit, which writes zeros.
struct Job {
    int64_t off, held;
    int queries, context, units, blocks;                 // blocks: of rows
};

__device__ __forceinline__ Job job_of(const CacheAttentionArgs &a, int off, int next, int held, int page_shift, int block_rows)
{
    Job j;
    j.off = off;
    j.held = held;
    j.queries = off < 0 || next < off || next > a.step.tokens ? 0 : next - off;
    const int64_t room = (int64_t)a.cache.table_width << page_shift, all = j.held + j.queries;
    const int64_t seen = all < room ? all : room;
    j.context = (int)(seen < 0 ? 0 : seen < kMaxContext ? seen : kMaxContext);
    j.units = j.context > 0 ? (int)(((int64_t)j.context + 2 * kTile - 1) / (2 * kTile)) : 1;
    j.blocks = (int)(((int64_t)j.queries * a.group + block_rows - 1) / block_rows);
    return j;
}

// The units of all sequences, one behind the other, are cut into ranges that differ by one unit at most, one for a workgroup.  Fewer ranges
// than workgroups where they would have less than `least` units.
struct Ranges {
    uint32_t count, each, longer;                        // the first `longer` of them have one more than `each`
    __device__ __forceinline__ Ranges(uint32_t total, uint32_t workgroups, uint32_t least)
    {
        const uint32_t most = (total + least - 1) / least;
        count = most < workgroups ? most : workgroups;
        each = count ? total / count : 0;
        longer = total - count * each;
    }
    __device__ __forceinline__ uint32_t begin(uint32_t r) const { return r * each + (r < longer ? r : longer); }
    __device__ __forceinline__ uint32_t of(uint32_t unit) const
    {
        const uint32_t split = longer * (each + 1);
        return unit < split ? unit / (each + 1) : longer + (unit - split) / each;
    }
};

// sums of the lanes up to this one
__device__ __forceinline__ uint32_t running_sum(uint32_t v, int lane)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t u = __shfl_up(v, m);
        if (lane >= m) v += u;
    }
    return v;
}

// How a call shares out its work: one workgroup for a whole context (of a sequence, head and block of rows); contexts cut into pieces, one
// workgroup each; equal ranges of all contexts
enum { kByContext, kByPiece, kByRange };

// pieces of a context of `units`, up to `splits`
__device__ __forceinline__ int pieces_of(int units, int splits)
{
    const int most = units / kPiece;
    return most < 1 ? 1 : most < splits ? most : splits;
}

// A wavefront's part of LDS: two tiles of K and two of V, 16 tokens of DIM bytes each, which come straight from memory: those of K for the
// next step while this one's weights are made and V is read, those of V while the next step reads K.  The 16-byte units of a row are
// exchanged (unit ^ swizzle of its row): K's operand reads one unit of all 16 rows at a time, without a conflict.
template <int DIM> constexpr int kTileBytes = kTile * DIM;
template <int DIM> __device__ __forceinline__ constexpr int swizzle(int row) { return row / (256 / DIM) & (DIM / 16 - 1); }

// The rows of a sequence's queries and the heads that share K and V, 16 ROW_TILES of them at a time.  RANGES: a workgroup has a range of
// all units (Ranges); else a block of rows of one sequence and head, from its first token to its last.
template <int DIM, bool FP8, bool BF16, int ROW_TILES, int WAVES, int FORM, bool STREAM>
__global__ void __launch_bounds__(64 * WAVES, FORM != kByContext || DIM == 256 || ROW_TILES > 1 ? 2 : 4) k_cache_attention(CacheAttentionArgs a, int page_shift)
{
    constexpr int kSteps = DIM / 32;                    // matrix instructions over the head's elements
    constexpr int kOut = DIM / 16;                      // result tiles
    constexpr int kWords = DIM / 64;                    // 4-byte words of V that a lane has of a token
    constexpr int kRows = 16 * ROW_TILES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;

    constexpr bool RANGES = FORM == kByRange;
    int b, head, block, piece = 0;                      // what the workgroup is at
    uint32_t at = 0, end = 0, begins = 0;               // RANGES: its place in all units and where it ends; where the sequence's begin
    Job job;
    if constexpr (RANGES) {
        int off = 0, next = 0, held = 0;
        uint32_t sum = 0, work = 0;
        bool astray = false;
        for (int c = 0; c < a.step.sequences; c += 64)
            if (c + lane < a.step.sequences) {
                off = a.step.offsets[c + lane];
                next = a.step.offsets[c + lane + 1];
                held = a.step.held[c + lane];
                const Job j = job_of(a, off, next, held, page_shift, kRows);
                work = j.units * j.blocks * a.heads;
                sum += work;
                astray |= off < 0 || next < off || next > a.step.tokens;
            }
        uint32_t upto = running_sum(sum, lane);
        // the units of offsets that do not ascend may be more than 32 bits count: none of them is done
        const uint32_t total = __any(astray) ? 0 : __builtin_amdgcn_readlane(upto, 63);
        const Ranges ranges(total, gridDim.x, kLeast);
        if (blockIdx.x == 0 && threadIdx.x == 0) a.plan[0] = total;
        if (blockIdx.x >= ranges.count) return;
        at = ranges.begin(blockIdx.x);
        end = ranges.begin(blockIdx.x + 1);
        b = -1;
        uint32_t run = 0;
        for (int c = 0; c < a.step.sequences; c += 64) {
            if (a.step.sequences > 64) {                // else the lanes have them still
                work = 0;
                if (c + lane < a.step.sequences) {
                    off = a.step.offsets[c + lane];
                    next = a.step.offsets[c + lane + 1];
                    held = a.step.held[c + lane];
                    const Job j = job_of(a, off, next, held, page_shift, kRows);
                    work = j.units * j.blocks * a.heads;
                }
                upto = run + running_sum(work, lane);
            }
            if (blockIdx.x == 0 && wave == 0 && c + lane < a.step.sequences) a.plan[1 + c + lane] = upto - work;
            const uint64_t past = __ballot(upto > at);
            if (b < 0 && past) {
                const int l = __builtin_ctzll(past);
                b = c + l;
                begins = __builtin_amdgcn_readlane(upto - work, l);
                job = job_of(a, __builtin_amdgcn_readlane(off, l), __builtin_amdgcn_readlane(next, l), __builtin_amdgcn_readlane(held, l), page_shift, kRows);
                if (blockIdx.x) break;                  // the first one writes where every sequence begins
            }
            run = __builtin_amdgcn_readlane(upto, 63);
        }
    } else {
        uint32_t id = blockIdx.x;
        if constexpr (FORM == kByPiece) {
            piece = id % a.splits;
            id /= a.splits;
        }
        head = id % a.heads;
        id /= a.heads;
        block = id % a.row_blocks;
        b = id / a.row_blocks;
        job = job_of(a, a.step.offsets[b], a.step.offsets[b + 1], a.step.held[b], page_shift, kRows);
    }

    __shared__ __attribute__((aligned(1024))) uint8_t stages[WAVES][4 * kTileBytes<DIM>];
    __shared__ float join_max[WAVES][16], join_sum[WAVES][16];
    float(*join)[16][DIM + 4] = reinterpret_cast<float(*)[16][DIM + 4]>(stages);       // [WAVES / 2], when the stages are done with
    static_assert(sizeof(stages) >= sizeof(float) * WAVES / 2 * 16 * (DIM + 4), "the wavefronts' sums fit the stages");
    // this lane's places: of the pieces that it brings to a tile, and of its operands in one
    constexpr int kPieces = kTileBytes<DIM> / 1024, kPieceRows = 1024 / DIM;
    int bring_at[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int row = i * kPieceRows + lane / (DIM / 16);
        bring_at[i] = row * DIM + ((lane % (DIM / 16)) ^ swizzle<DIM>(row)) * 16;
    }
    const int at_k = col * DIM + (quad ^ swizzle<DIM>(col)) * 16;
    const int at_v = quad * 4 * DIM + ((col * DIM / 256) ^ swizzle<DIM>(quad * 4)) * 16 + col * (DIM / 16) % 16;
    const uint32_t lds = lds_address(&stages[wave][0]);
    const uint8_t *const tile_k = &stages[wave][0], *const tile_v = tile_k + 2 * kTileBytes<DIM>;

    while (RANGES ? at < end : block < job.blocks) {
        int pair0 = 0, pair1 = job.units;               // of the sequence
        if constexpr (RANGES) {
            const uint32_t work = job.units * job.blocks * a.heads;
            if (at >= begins + work) {
                begins += work;
                ++b;
                job = job_of(a, a.step.offsets[b], a.step.offsets[b + 1], a.step.held[b], page_shift, kRows);
                continue;
            }
            const uint32_t item = (at - begins) / job.units, item0 = begins + item * job.units;
            head = (int)(item / job.blocks);
            block = (int)(item - (uint32_t)head * job.blocks);
            pair0 = at - item0;
            if (end - item0 < (uint32_t)pair1) pair1 = end - item0;
            at = item0 + pair1;
        } else if constexpr (FORM == kByPiece) {
            const int pieces = pieces_of(job.units, a.splits);
            if (piece >= pieces) return;
            pair0 = (int)((int64_t)job.units * piece / pieces);
            pair1 = (int)((int64_t)job.units * (piece + 1) / pieces);
        }
        const bool whole = pair0 == 0 && pair1 == job.units;
        const int64_t off = job.off, held = job.held, rows = (int64_t)job.queries * a.group, row0 = (int64_t)block * kRows;
        const int context = job.context;
        const int begin = 2 * (pair0 + (pair1 - pair0) * wave / WAVES), stop = 2 * (pair0 + (pair1 - pair0) * (wave + 1) / WAVES);
        const int end_token = stop * kTile < context ? stop * kTile : context;  // of this wavefront

        // the rows: elements 64 j + 16 quad + 8 s for step 2 j + s
        uintx4 qf[ROW_TILES][kSteps];
#pragma unroll
        for (int x = 0; x < ROW_TILES; ++x) {
            const int64_t row = row0 + 16 * x + col, query = row < rows ? row / a.group : 0;
            const int query_head = head * a.group + (int)(row - query * a.group);
            const uint16_t *q = (const uint16_t *)a.q.ptr + (off + query) * a.q.token + query_head * a.q.head + quad * 16;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                qf[x][j] = uintx4{0, 0, 0, 0};
                if (row < rows) qf[x][j] = *(const uintx4 *)(q + 64 * (j / 2) + 8 * (j & 1));
            }
        }
        const int64_t least_seen = held + row0 / a.group + 1;
        const int all_see = least_seen < 0 ? 0 : least_seen < end_token ? (int)least_seen : end_token;     // what every row of the block sees

        // page and scales of 64 tiles from `base` on, one a lane
        int page = 0;
        float ks = 0.0f, vs = 0.0f;
        const auto look_up = [&](int base) {
            page = 0;
            ks = 0.0f;
            vs = kLow;                                  // (of tiles that are not there: an ordinary one, which raises nothing)
            if (base + lane < stop && (base + lane) * kTile < context) {
                const int id = a.cache.table[(int64_t)b * a.cache.table_width + ((base + lane) * kTile >> page_shift)];
                vs = 0.0f;
                if (id >= 0 && id < a.cache.pages) {
                    page = id;
                    ks = a.cache.k_scales[(int64_t)id * a.heads + head];
                    vs = a.cache.v_scales[(int64_t)id * a.heads + head];
                }
            }
        };
        // the pair of tiles of lanes i and i + 1, from base + i on; what the place held before has been read
        const auto bring = [&](const uint8_t *from, uint32_t to, int base, int i) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int slot = ((base + i + t) * kTile) & ((1 << page_shift) - 1);
                const int64_t place = ((((int64_t)__builtin_amdgcn_readlane(page, i + t) * a.heads + head) << page_shift) + slot) * DIM;
                const uintx4 tile = resource(from + place, kTileBytes<DIM>);
#pragma unroll
                for (int j = 0; j < kPieces; ++j) load_to_lds<STREAM>(tile, bring_at[j], to + t * kTileBytes<DIM> + j * 1024);
            }
        };
        const uint32_t to_k = lds, to_v = lds + 2 * kTileBytes<DIM>;
        if (begin < stop) {
            look_up(begin);
            bring(a.cache.k, to_k, begin, 0);
            bring(a.cache.v, to_v, begin, 0);
        }

        float factor[ROW_TILES];                        // scores in powers of two
#pragma unroll
        for (int x = 0; x < ROW_TILES; ++x) {
            factor[x] = a.scale * 1.4426950408889634f;
            if constexpr (BF16) {
                // into binary16, the largest magnitude times 2^e in [2^13, 2^14)
                float most = 0.0f;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    float f[8];
                    widen8<BF16>(qf[x][j], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(f[i]));
                }
                most = max4(most);
                int e = 0;
                if (most > 0.0f && most < __builtin_inff()) e = 14 - __builtin_amdgcn_frexp_expf(most);
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    float f[8];
                    widen8<BF16>(qf[x][j], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = __builtin_amdgcn_ldexpf(f[i], e);
                    qf[x][j] = narrow8<false>(f);
                }
                factor[x] = __builtin_amdgcn_ldexpf(factor[x], -e);
            }
        }

        floatx4 acc[ROW_TILES][kOut];
        float top[ROW_TILES], total[ROW_TILES], ref[ROW_TILES];
#pragma unroll
        for (int x = 0; x < ROW_TILES; ++x) {
#pragma unroll
            for (int o = 0; o < kOut; ++o) acc[x][o] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            top[x] = -FLT_MAX;
            total[x] = ref[x] = 0.0f;
        }
        // the sums' unit: they are acc * was, and are acc * ref afterwards
        const auto rebase = [&](int x, float was, float least) {
            ref[x] = fmaxf(was, least);
            const float change = was / ref[x];
#pragma unroll
            for (int o = 0; o < kOut; ++o) acc[x][o] *= change;
        };

        for (int base = begin; base < stop; base += 64) {
            const int n = stop - base < 64 ? stop - base : 64;
            if (base != begin) {
                look_up(base);
                bring(a.cache.k, to_k, base, 0);
                bring(a.cache.v, to_v, base, 0);
            }
            // the scales are here before the loop, where waiting for them would wait for all that is on its way
            asm volatile("" : "+v"(ks), "+v"(vs));
            // The sums' unit is no less than 2^-116 of these tiles' largest scale, so that a scale in it, and 2^8 times that, stay finite:
            // 2^-100 for ordinary scales
            float least = 0x1p-100f;
            if (__any(!(vs >= kLow && vs <= kHigh))) {
                const float v = vs <= FLT_MAX ? vs * 0x1p-116f : 0.0f;
                least = FLT_MIN;
#pragma unroll 1
                for (int l = 0; l < 64; ++l) least = fmaxf(least, lane_f(v, l));       // (shuffles take registers that the loop has not got)
            }
#pragma unroll
            for (int x = 0; x < ROW_TILES; ++x) {
                if (base == begin) ref[x] = least;      // there are no sums yet
                else if (__any(ref[x] < least)) rebase(x, ref[x], least);
            }
            for (int i = 0; i < n; i += 2) {
                const int first = (base + i) * kTile;
                wait_vm<2 * kPieces>();                 // K is here, V may be on its way
                floatx4 s[ROW_TILES][2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int x = 0; x < ROW_TILES; ++x) s[x][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < kWords; ++j) {
                        const uintx4 w = *(const uintx4 *)(tile_k + t * kTileBytes<DIM> + (at_k ^ (j << 6)));
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uintx2 lo = halves<FP8>(w[2 * h]), hi = halves<FP8>(w[2 * h + 1]);
#pragma unroll
                            for (int x = 0; x < ROW_TILES; ++x) s[x][t] = mma16(uintx4{lo[0], lo[1], hi[0], hi[1]}, qf[x][2 * j + h], s[x][t]);
                        }
                    }
                }
                const bool more = i + 2 < n;
                if (more) bring(a.cache.k, to_k, base, i + 2);
                const float ksc[2] = {lane_f(ks, i), lane_f(ks, i + 1)}, vsc[2] = {lane_f(vs, i), lane_f(vs, i + 1)};
                const bool masked = first + 2 * kTile > all_see;
                uintx4 pf[ROW_TILES];
#pragma unroll
                for (int x = 0; x < ROW_TILES; ++x) {
                    float scale[2], most = -__builtin_inff();
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        scale[t] = factor[x] * ksc[t];
                        if (masked) {                   // (a scale of 0 would make NaN of a masked score)
                            const int64_t row = row0 + 16 * x + col, seen = held + row / a.group + 1;
                            const int sees = row >= rows || seen < 0 ? 0 : seen < end_token ? (int)seen : end_token;
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[x][t][r] = first + t * kTile + quad * 4 + r < sees ? s[x][t][r] * scale[t] : -__builtin_inff();
                            scale[t] = 1.0f;
                        }
                        most = fmaxf(most, fmaxf(fmaxf(s[x][t][0], s[x][t][1]), fmaxf(s[x][t][2], s[x][t][3])) * scale[t]);
                    }
                    if (__any(most > top[x] + kSlack)) {
                        most = max4(most);              // only rows that passed their own: no row's bits depend on others
                        const float now = most > top[x] + kSlack ? most : top[x], shrink = __builtin_amdgcn_exp2f(top[x] - now);
                        top[x] = now;
                        total[x] *= shrink;
                        rebase(x, ref[x] * shrink, least);
                    }
                    float p[8], w[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][r / 4][r % 4], scale[r / 4], -top[x]));
                        total[x] += p[r];
                    }
                    const auto weigh = [&] {
                        const float inv = __builtin_amdgcn_rcpf(ref[x]), unit[2] = {vsc[0] * inv, vsc[1] * inv};
#pragma unroll
                        for (int r = 0; r < 8; ++r) w[r] = p[r] * unit[r / 4];
                        return fmaxf(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), fmaxf(fmaxf(w[4], w[5]), fmaxf(w[6], w[7])));
                    };
                    float weight = weigh();
                    if (__any(weight > kMost)) {
                        weight = max4(weight);
                        rebase(x, ref[x], weight > kMost ? weight * (1.0f / kAim) * ref[x] : 0.0f);
                        weigh();
                    }
                    if (masked)                         // whatever the scale of what a row does not see
#pragma unroll
                        for (int r = 0; r < 8; ++r)
                            if (p[r] == 0.0f) w[r] = 0.0f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) pf[x][r] = narrow2<false>(w[2 * r], w[2 * r + 1]);
                }
                if (more) wait_vm<2 * kPieces>();       // V is here, the next K may be on its way
                else wait_vm<0>();
                if constexpr (FP8) {
                    // E4M3's NaN among values that some rows of the block do not see: taken out, it goes into the weights of those that do
                    if (masked && job.queries > 1) {
                        uint32_t bad = 0;               // one bit for each of the tokens
#pragma unroll 1
                        for (int i = 0; i < 2 * kPieces; ++i) {
                            uintx4 *const place = (uintx4 *)(tile_v + i * 1024 + lane * 16);
                            uintx4 w = *place;
                            uint32_t any = 0;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t nan = (((w[j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;     // 1 in its byte
                                w[j] &= ~(nan * 0xFFu);
                                any |= nan;
                            }
                            if (any) *place = w;
                            for (uint64_t lanes = __ballot(any); lanes; lanes &= lanes - 1) bad |= 1u << (i * kPieceRows + __builtin_ctzll(lanes) / (DIM / 16));
                        }
                        if (bad) {
                            const uint32_t mine[2] = {bad >> (quad * 4), bad >> (kTile + quad * 4)};
#pragma unroll
                            for (int x = 0; x < ROW_TILES; ++x)
#pragma unroll
                                for (int r = 0; r < 8; ++r) {
                                    const uint32_t half = 0xFFFFu << 16 * (r & 1);
                                    if ((mine[r / 4] >> r % 4 & 1) && (pf[x][r / 2] & half)) pf[x][r / 2] |= half;
                                }
                        }
                    }
                }
                uint32_t vf[2][4][kWords];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        load_words(tile_v + t * kTileBytes<DIM> + r * DIM + (at_v ^ (swizzle<DIM>(r) << 4)), vf[t][r]);
                        // codes beyond the context: whatever the cache holds there
                        if (masked && first + t * kTile + quad * 4 + r >= end_token)
#pragma unroll
                            for (int w = 0; w < kWords; ++w) vf[t][r][w] = 0;
                    }
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    uint32_t y[2][4];
#pragma unroll
                    for (int t = 0; t < 2; ++t) transpose4(vf[t][0][w], vf[t][1][w], vf[t][2][w], vf[t][3][w], y[t]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uintx2 lo = halves<FP8>(y[0][e]), hi = halves<FP8>(y[1][e]);
#pragma unroll
                        for (int x = 0; x < ROW_TILES; ++x) acc[x][w * 4 + e] = mma16(uintx4{lo[0], lo[1], hi[0], hi[1]}, pf[x], acc[x][w * 4 + e]);
                    }
                }
                if (more) bring(a.cache.v, to_v, base, i + 2);
            }
        }

#pragma unroll
        for (int x = 0; x < ROW_TILES; ++x) {
            if (16 * x >= rows - row0) break;
            __syncthreads();                            // the stages, or the row tile before, are done with
            // join the wavefronts: all in the unit of the largest maximum, then halves of them added to the other half
            const float sum = sum4(total[x]);
            if (quad == 0) {
                join_max[wave][col] = top[x];
                join_sum[wave][col] = sum;
            }
            __syncthreads();
            float best = join_max[0][col], all = 0.0f;
#pragma unroll
            for (int w = 1; w < WAVES; ++w) best = fmaxf(best, join_max[w][col]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all += join_sum[w][col] * __builtin_amdgcn_exp2f(join_max[w][col] - best);
            const float mine = __builtin_amdgcn_exp2f(top[x] - best) * ref[x];
#pragma unroll
            for (int o = 0; o < kOut; ++o) acc[x][o] *= mine;
#pragma unroll
            for (int half = WAVES / 2; half; half >>= 1) {
                if (wave >= half && wave < 2 * half)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int o = 0; o < kOut; o += 4)
                            *(floatx4 *)&join[wave - half][col][(quad * 4 + r) * kOut + o] = floatx4{acc[x][o][r], acc[x][o + 1][r], acc[x][o + 2][r], acc[x][o + 3][r]};
                __syncthreads();
                if (wave < half)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int o = 0; o < kOut; o += 4) {
                            const floatx4 y = *(const floatx4 *)&join[wave][col][(quad * 4 + r) * kOut + o];
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[x][o + i][r] += y[i];
                        }
                __syncthreads();
            }
            const int64_t row = row0 + 16 * x + col;
            if (wave == 0 && row < rows) {
                const int64_t q = row / a.group;
                const int h = head * a.group + (int)(row - q * a.group);
                if (whole) {
                    const float inv = all == 0.0f ? 0.0f : 1.0f / all;          // a row that sees nothing is zero
                    uint16_t *y = (uint16_t *)a.out.ptr + (off + q) * a.out.token + h * a.out.head + quad * 4 * kOut;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int o = 0; o < kOut; o += 4)
                            *(uintx2 *)(y + r * kOut + o) = uintx2{narrow2<BF16>(acc[x][o][r] * inv, acc[x][o + 1][r] * inv), narrow2<BF16>(acc[x][o + 2][r] * inv, acc[x][o + 3][r] * inv)};
                } else {
                    const int64_t tokens_rows = a.step.tokens * a.heads * a.group;
                    const int64_t place = RANGES ? ((int64_t)blockIdx.x * 2 + (pair0 == 0)) * kRows + 16 * x + col
                                                 : ((off + q) * a.heads * a.group + h) * a.splits + piece;
                    const int64_t places = RANGES ? (int64_t)gridDim.x * 2 * kRows : tokens_rows * a.splits;
                    float *y = a.partial + place * DIM + quad * 4 * kOut;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int o = 0; o < kOut; o += 4)
                            *(floatx4 *)(y + r * kOut + o) = floatx4{acc[x][o][r], acc[x][o + 1][r], acc[x][o + 2][r], acc[x][o + 3][r]};
                    if (quad == 0) *(floatx2 *)(a.partial + places * DIM + place * 2) = floatx2{best, all};
                }
            }
        }
        if constexpr (!RANGES) block += a.row_blocks;
    }
}

// Joins the pieces of the rows that were cut.  A range has two places for them: 1 for an item that it begins and does not end, 0 for one
// that began before.  WAVES wavefronts for a token's row; in one, DIM / 4 lanes have 4 elements each.
template <int DIM, bool BF16, int WAVES, bool RANGES>
__global__ void __launch_bounds__(256) k_cache_attention_join(CacheAttentionArgs a, int page_shift)
{
    constexpr int kLanes = DIM / 4, kSets = 64 * WAVES / kLanes;          // every kSets-th piece is one set of lanes'
    const int block_rows = 16 * a.row_tiles, query_heads = a.heads * a.group;
    const int64_t row_id = (int64_t)blockIdx.x * (4 / WAVES) + (WAVES == 4 ? 0 : threadIdx.x / (64 * WAVES));
    if (row_id >= a.step.tokens * query_heads) return;
    const int64_t token = row_id / query_heads;
    const int h = (int)(row_id - token * query_heads), head = h / a.group;
    // single tokens: the sequence is the token's, or else it is looked for
    const int guess = token < a.step.sequences ? (int)token : a.step.sequences - 1;
    int off = a.step.offsets[guess], next = a.step.offsets[guess + 1], held = a.step.held[guess];
    uint32_t begins = 0, total = 0;
    if constexpr (RANGES) {
        begins = a.plan[1 + guess];
        total = a.plan[0];
    }
    if (off != token || next != token + 1) {
        const int b = find_sequence(a.step.offsets, a.step.sequences, 0, 0, token);
        off = a.step.offsets[b];
        next = a.step.offsets[b + 1];
        held = a.step.held[b];
        if constexpr (RANGES) begins = a.plan[1 + b];
    }
    const Job job = job_of(a, off, next, held, page_shift, block_rows);
    if (token < off || token >= off + job.queries) return;
    int64_t place0, step, places;                       // of the first piece and of the others behind it
    int pieces;
    if constexpr (RANGES) {
        if (total == 0) return;
        const Ranges ranges(total, a.workgroups, kLeast);
        const int64_t row = (token - off) * a.group + (h - head * a.group);
        const int block = (int)(row / block_rows), row_at = (int)(row - (int64_t)block * block_rows);
        const uint32_t item0 = begins + ((uint32_t)head * job.blocks + block) * job.units;
        const uint32_t first = ranges.of(item0), last = ranges.of(item0 + job.units - 1);
        pieces = (int)(last - first) + 1;
        place0 = ((int64_t)first * 2 + 1) * block_rows + row_at;
        step = 2 * block_rows;
        places = (int64_t)a.workgroups * step;
    } else {
        pieces = pieces_of(job.units, a.splits);
        place0 = row_id * a.splits;
        step = 1;
        places = a.step.tokens * query_heads * a.splits;
    }
    if (pieces == 1) return;                            // written already
    // ranges: the first piece is in the second place of its range, the others are in the first ones
    const auto place = [&](int p) { return place0 + p * step - (RANGES && p ? block_rows : 0); };

    const floatx2 *m = (const floatx2 *)(a.partial + places * DIM);
    const int lane = threadIdx.x & 63, d = threadIdx.x % kLanes * 4, set = threadIdx.x % (64 * WAVES) / kLanes;
    float best = -FLT_MAX, sum = 0.0f;
    floatx4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p0 = 0; p0 < pieces; p0 += 64) {
        const int n = pieces - p0 < 64 ? pieces - p0 : 64;
        floatx2 mine = {-FLT_MAX, 0.0f};
        if (lane < n) mine = m[place(p0 + lane)];
        // the first pieces' sums are on their way meanwhile
        floatx4 early = {0.0f, 0.0f, 0.0f, 0.0f};
        if (set < n) early = *(const floatx4 *)(a.partial + place(p0 + set) * DIM + d);
        float top = mine[0];
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) top = fmaxf(top, __shfl_xor(top, w));
        const float now = fmaxf(best, top), shrink = __builtin_amdgcn_exp2f(best - now);
        best = now;
        const float weight = __builtin_amdgcn_exp2f(mine[0] - now);
        sum = sum * shrink + weight * mine[1];          // a part of it in each lane
        x *= shrink;
        x += early * __shfl(weight, set < n ? set : 0);
        for (int p = kSets; p < n; p += kSets) {
            const float w = __shfl(weight, p + set < 64 ? p + set : 63);
            if (p + set < n) x += *(const floatx4 *)(a.partial + place(p0 + p + set) * DIM + d) * w;
        }
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) sum += __shfl_xor(sum, w);
    if constexpr (WAVES > 1) {
        __shared__ floatx4 sets[kSets][kLanes];
        sets[set][threadIdx.x % kLanes] = x;
        __syncthreads();
        if (set) return;
#pragma unroll
        for (int i = 1; i < kSets; ++i) x += sets[i][threadIdx.x];
    } else {
#pragma unroll
        for (int w = kLanes; w < 64; w <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] += __shfl_xor(x[i], w);
        if (set) return;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t *y = (uint16_t *)a.out.ptr + token * a.out.token + h * a.out.head + d;
    *(uintx2 *)y = uintx2{narrow2<BF16>(x[0] * inv, x[1] * inv), narrow2<BF16>(x[2] * inv, x[3] * inv)};
}

template <int DIM, bool FP8, bool BF16, int ROW_TILES>
hipError_t attend_rows(const CacheAttentionArgs &a, hipStream_t stream)
{
    const int shift = log2_int(a.cache.page);
    constexpr int kWaves = waves_of(DIM, ROW_TILES);
    const int64_t groups = (int64_t)a.step.sequences * a.row_blocks * a.heads;
    const auto go = [&](auto *kernel, int64_t grid, int waves) { return launch_many(kernel, grid, 64 * waves, stream, a, shift); };
    if (!a.workgroups && a.splits == 1)
        return a.stream ? go(k_cache_attention<DIM, FP8, BF16, ROW_TILES, kWaves, kByContext, true>, groups, kWaves)
                        : go(k_cache_attention<DIM, FP8, BF16, ROW_TILES, kWaves, kByContext, false>, groups, kWaves);
    hipError_t e = hipErrorInvalidValue;
    if (a.workgroups)
        e = a.stream ? go(k_cache_attention<DIM, FP8, BF16, ROW_TILES, 4, kByRange, true>, a.workgroups, 4)
                     : go(k_cache_attention<DIM, FP8, BF16, ROW_TILES, 4, kByRange, false>, a.workgroups, 4);
    else if constexpr (ROW_TILES < 3)                   // three tiles go with much more work than pieces
        e = go(k_cache_attention<DIM, FP8, BF16, ROW_TILES, 4, kByPiece, false>, groups * a.splits, 4);
    if (e != hipSuccess) return e;
    const int64_t rows = a.step.tokens * a.heads * a.group;
    // where there are many rows, there are few pieces of each
    if (rows < 1024)
        return a.workgroups ? go(k_cache_attention_join<DIM, BF16, 4, true>, rows, 4) : go(k_cache_attention_join<DIM, BF16, 4, false>, rows, 4);
    return a.workgroups ? go(k_cache_attention_join<DIM, BF16, 1, true>, (rows + 3) / 4, 4) : go(k_cache_attention_join<DIM, BF16, 1, false>, (rows + 3) / 4, 4);
}

template <int DIM, bool FP8, bool BF16>
hipError_t attend(const CacheAttentionArgs &a, hipStream_t stream)
{
    if constexpr (DIM != 256) {
        if (a.row_tiles == 2) return attend_rows<DIM, FP8, BF16, 2>(a, stream);
        if (a.row_tiles == 3) return attend_rows<DIM, FP8, BF16, 3>(a, stream);
    }
    return attend_rows<DIM, FP8, BF16, 1>(a, stream);
}

template <int DIM>
hipError_t attend_types(const CacheAttentionArgs &a, hipStream_t stream)
{
    if (a.fp8) return a.bf16 ? attend<DIM, true, true>(a, stream) : attend<DIM, true, false>(a, stream);
    return a.bf16 ? attend<DIM, false, true>(a, stream) : attend<DIM, false, false>(a, stream);
}

}  // namespace

void cache_attention_plan(int sequences, int heads, int group, int dim, int64_t queries, int64_t longest, CacheAttentionArgs *a)
{
    // what may be announced is as much as its type holds, and the products of that more than 64 bits
    const int64_t tiles = (queries * group + 15) / 16, pairs = (longest + 2 * kTile - 1) / (2 * kTile);
    const double contexts = (double)sequences * heads;
    // Three tiles of rows at a time read the context once for 48 rows, but leave fewer workgroups; us for 40 rows of 8 heads by context with
    // two and three: 4000 tokens 21.6 / 28.0, 16000 28.7 / 34.0, 131071 73.8 / 62.2
    a->row_tiles = dim == 256 || tiles == 1 ? 1 : tiles == 2 || contexts * pairs < 16384 ? 2 : 3;
    const int64_t blocks = (tiles + a->row_tiles - 1) / a->row_tiles;
    a->row_blocks = blocks > 4096 ? 4096 : (int)blocks;
    const double groups = contexts * blocks, units = groups * pairs;
    a->splits = 1;
    a->workgroups = 0;
    if (pairs <= waves_of(dim, a->row_tiles) * (groups >= 192 ? 12 : 3)) {
        // One workgroup for a whole context: no second launch, but the time of the longest context on one compute unit.  us whole / in
        // pieces: 16 contexts of 700 tokens 10.5 / 11.2, 1536 14.7 / 11.7; 128 of 1500 17.5 / 16.4; 240 of 1500 18.6 / 21.7
    } else if (units <= 16384 && a->row_tiles < 3) {
        // Pieces, a workgroup each: as many as one or two for every compute unit, and few enough to be joined quickly.  us in pieces / in equal
        // ranges, which have to be found first: 16 contexts of 3000 tokens 12.3 / 17.1, 64 of 4000 18.0 / 22.6, 8 of 40000 23.1 / 26.4;
        // 256 / 512 pieces: 16 of 3000 12.3 / 13.5, 64 of 4000 20.0 / 18.0; 2 of 32000 with 125 and 250 each 17.1 / 23.2
        const int64_t fit = (units > 4096 ? 512 : 256) / (int64_t)groups, most = pairs / kPiece, splits = fit < most ? fit : most;
        a->splits = (int)(splits < 1 ? 1 : splits < 128 ? splits : 128);
    } else {
        // Two workgroups of four wavefronts a compute unit hold enough loads in flight; 512 / 1024 / 2048 of them for 64 x 8 contexts of up to
        // 8192: 142 / 143 / 147 us.  160 contexts of up to 8192 in ranges / in pieces 52.5 / 58.2
        a->workgroups = units < 512 * kLeast ? ((int)units + kLeast - 1) / kLeast : 512;
    }
    // what one workgroup reads and the memory-side cache does not hold is marked as read once (157 -> 143 us there)
    a->stream = blocks == 1 && beyond_cache(contexts * longest * 2 * dim);
}

size_t cache_attention_workspace(const CacheAttentionArgs &a, int64_t tokens, int sequences, int query_heads, int dim)
{
    const size_t each = (size_t)(dim + 2) * sizeof(float);
    if (a.workgroups) return (size_t)a.workgroups * 2 * 16 * a.row_tiles * each + ((size_t)sequences + 5) * sizeof(uint32_t);
    return a.splits == 1 ? 0 : (size_t)tokens * query_heads * a.splits * each + ((size_t)sequences + 5) * sizeof(uint32_t);
}

hipError_t launch_cache_attention(const CacheAttentionArgs &a, hipStream_t stream)
{
    switch (a.dim) {
    case 64: return attend_types<64>(a, stream);
    case 128: return attend_types<128>(a, stream);
    default: return attend_types<256>(a, stream);
    }
}

}  // namespace fc
