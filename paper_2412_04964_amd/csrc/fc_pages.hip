// fc_pages.hip -- the pages of the cache when sequences fork, grow, end, and move together; copies of pages.
//
// A page table row names the pages of a sequence, uses[p] how many rows name page p (0: free).  All results are whole numbers that do not
// depend on the order in which workgroups run: counts are added atomically, fresh pages are the lowest free ones in the order of
// (sequence, slot), and pages move in ascending order.
#include "fc_attn.hpp"

namespace fc {
namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(4))) intx4_as_int {        // on any 4-byte boundary
    intx4 v;
};

// entries of a row that hold tokens
__device__ __forceinline__ int64_t filled_slots(int64_t held, int page_shift) { return held > 0 ? (held + (1 << page_shift) - 1) >> page_shift : 0; }

// Workgroups [0, rows) write the new table's rows; the others release or share the pages of an old row, by how many new rows have it as parent.
__global__ void __launch_bounds__(256) k_pages_fork(ForkArgs a, int page_shift)
{
    if (blockIdx.x < (uint32_t)a.rows) {
        const int b = blockIdx.x, parent = a.parents[b];
        const bool there = parent >= 0 && parent < a.sequences;
        const int64_t held = there ? a.held[parent] : 0, filled = filled_slots(held, page_shift);
        const int32_t *from = a.table + (int64_t)(there ? parent : 0) * a.width;
        for (int i = threadIdx.x; i < a.width; i += 256) {
            int id = -1;
            if (i < filled) {
                id = from[i];
                if (id < 0 || id >= a.pages) id = -1;
            }
            a.table_out[(int64_t)b * a.width + i] = id;
        }
        if (threadIdx.x == 0) a.held_out[b] = (int32_t)held;
        return;
    }
    const int b = blockIdx.x - a.rows;
    __shared__ int children;
    if (threadIdx.x == 0) children = 0;
    __syncthreads();
    int mine = 0;
    for (int i = threadIdx.x; i < a.rows; i += 256) mine += a.parents[i] == b;
    if (mine) atomicAdd(&children, mine);
    __syncthreads();
    const int64_t filled = filled_slots(a.held[b], page_shift);
    const int change = children - 1;
    for (int i = threadIdx.x; i < a.width; i += 256) {
        const int by = i < filled ? change : -1;         // what is reserved beyond the tokens held is given back
        const int id = a.table[(int64_t)b * a.width + i];
        if (by && id >= 0 && id < a.pages) atomicAdd(&a.uses[id], by);
    }
}

constexpr int kFew = 4096;                               // fresh pages that are listed in LDS
constexpr int kSegments = 8;                             // of a pool that every workgroup counts itself (20000 pages: 6.8 us, with counts ahead 5 + 4.5)

// Sums of the lanes up to this one: within 16 lanes, then from the last lane of the 16 before, then from the last of the first 32
__device__ __forceinline__ int upto(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
    return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
}

// Sum of `v` over the lanes of a workgroup of 16 wavefronts before this one, and over all; a second value's sum over all.  Two barriers.
__device__ __forceinline__ int before(int v, int (&sums)[2][16], int *all, int other = 0, int *others = nullptr)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), run = upto(v), more = others ? upto(other) : 0;
    __syncthreads();
    if (lane == 63) {
        sums[0][wave] = run;
        if (others) sums[1][wave] = more;
    }
    __syncthreads();
    const int mine = upto(sums[0][lane & 15]);           // (of the 16, in every 16 lanes; the first ones count)
    *all = __builtin_amdgcn_readlane(mine, 15);
    if (others) *others = __builtin_amdgcn_readlane(upto(sums[1][lane & 15]), 15);
    return (wave ? __builtin_amdgcn_readlane(mine, wave - 1) : 0) + run - v;
}

// The slots of a sequence's table row that its new tokens go to
struct Slots {
    int first, count;
    bool partial;                                        // the first one holds tokens already
};
__device__ __forceinline__ Slots slots_of(const ReserveArgs &a, int b, int page_shift)
{
    const int64_t held = a.held[b], end = held + ((int64_t)a.offsets[b + 1] - a.offsets[b]), begin = held > 0 ? held : 0;
    const int64_t first = begin >> page_shift;
    int64_t last = (end - 1) >> page_shift;
    if (last >= a.width) last = a.width - 1;
    if (end <= begin || first > last) return {0, 0, false};
    return {(int)first, (int)(last - first) + 1, (begin & ((1 << page_shift) - 1)) != 0};
}

// One workgroup for the step: a lane has a sequence, the first 1024 of them from beginning to end.  While it runs, source[b] is the partly filled
// page that sequence b writes to, or -1, and target[b] where its fresh pages begin among all (~ that: and it copies).
// Bound by reads that depend on each other and by the walk through `uses` up to the last page that is needed (16 counts a lane at a time): 4 sequences
// 6.4 us, 241 of which half part with a page, in a pool of 20000, 12.8 us.
__global__ void __launch_bounds__(1024) k_pages_reserve(ReserveArgs a, int page_shift)
{
    __shared__ int sums[2][16];
    __shared__ __attribute__((aligned(16))) int staged[1024];
    __shared__ int few[kFew];                            // the fresh pages, if they are few
    const auto none = [&](int id) { return id < 0 || id >= a.pages; };
    // free ones among the 16 pages from p on
    const auto free_of = [&](int64_t p) {
        uint32_t free = 0;
        if (p + 16 <= a.pages) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const intx4 u = ((const intx4_as_int *)(a.uses + p))[i].v;
#pragma unroll
                for (int j = 0; j < 4; ++j) free |= (u[j] == 0) << (4 * i + j);
            }
        } else {
            for (int i = 0; i < 16; ++i) free |= (p + i < a.pages && a.uses[p + i] == 0) << i;
        }
        return free;
    };
    uint32_t free_next = free_of(16 * threadIdx.x);      // (on its way while the rest is found out)
    Slots own = {0, 0, false};
    int own_page = -1, own_id = -1;                      // of the first slot: what the table has there; the page if it is partly filled
    const auto look = [&](int b) {
        const Slots s = slots_of(a, b, page_shift);
        const int id = s.count ? a.table[(int64_t)b * a.width + s.first] : -1;
        if (b < 1024) {
            own = s;
            own_page = id;
            own_id = s.partial && !none(id) ? id : -1;
        }
        return s.partial && !none(id) ? id : -1;
    };
    bool astray = false;                                 // offsets that do not ascend may ask for more pages than 32 bits count: none of them gets any
    for (int b = threadIdx.x; b < a.sequences; b += 1024) {
        astray |= a.offsets[b] < 0 || a.offsets[b + 1] < a.offsets[b];
        a.source[b] = look(b);
    }
    if (__syncthreads_or(astray)) {
        for (int b = threadIdx.x; b < a.sequences; b += 1024) a.source[b] = a.target[b] = -1;
        if (threadIdx.x == 0) *a.lacking = 0;
        return;
    }
    // who copies, and how many fresh pages each sequence takes
    int needed = 0;
    for (int c = 0; c < a.sequences; c += 1024) {
        const int b = c + threadIdx.x;
        const bool here = b < a.sequences;
        const int mine = !here ? -1 : c ? a.source[b] : own_id, users = mine >= 0 ? a.uses[mine] : 0;
        int writers = 0, later = 0;
        if (__syncthreads_or(users > 1)) {
            for (int d = 0; d < a.sequences; d += 1024) {
                __syncthreads();
                staged[threadIdx.x] = d + threadIdx.x < a.sequences ? d ? a.source[d + threadIdx.x] : own_id : -1;
                __syncthreads();
                if (users > 1) {
                    const int n = a.sequences - d < 1024 ? a.sequences - d : 1024;
#pragma unroll 4
                    for (int i = 0; i < n; i += 4) {     // (behind the last sequence there is no page)
                        const intx4 four = *(const intx4 *)&staged[i];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            writers += four[j] == mine;
                            later += four[j] == mine && d + i + j > b;
                        }
                    }
                }
            }
        }
        const bool copies = users > 1 && (later || writers < users);
        int want = copies;
        if (here) {
            const Slots s = c ? slots_of(a, b, page_shift) : own;
            if (c == 0) want += s.count && none(own_page);
            for (int i = c == 0; i < s.count; ++i) want += none(a.table[(int64_t)b * a.width + s.first + i]);
        }
        int all;
        const int start = needed + before(want, sums, &all);
        if (here) a.target[b] = copies ? ~start : start;
        needed += all;
    }
    // the lowest free pages
    int *const fresh = needed <= kFew ? few : a.fresh;
    int found = 0;
    for (int64_t p0 = 0; p0 < a.pages && found < needed; p0 += 16384) {
        uint32_t free = free_next;
        free_next = free_of(p0 + 16384 + 16 * threadIdx.x);
        int all;
        int at = found + before(__builtin_popcount(free), sums, &all);
        for (; free && at < needed; free &= free - 1) fresh[at++] = (int)p0 + 16 * threadIdx.x + __builtin_ctz(free);
        found += all;
    }
    __syncthreads();
    if (threadIdx.x == 0) *a.lacking = found < needed ? needed - found : 0;
    for (int b = threadIdx.x; b < a.sequences; b += 1024) {
        const int mark = a.target[b];
        const bool copies = mark < 0 && found >= needed;
        int at = mark < 0 ? ~mark : mark;
        int target = -1;
        if (found >= needed && needed) {
            const Slots s = b < 1024 ? own : slots_of(a, b, page_shift);
            int32_t *row = a.table + (int64_t)b * a.width + s.first;
            for (int i = 0; i < s.count; ++i) {
                const bool copy = copies && i == 0;
                if (!copy && !none(b < 1024 && i == 0 ? own_page : row[i])) continue;
                const int id = fresh[at++];
                row[i] = id;
                a.uses[id] = 1;
                if (copy) target = id;
            }
            if (copies) atomicAdd(&a.uses[b < 1024 ? own_id : a.source[b]], -1);
        }
        a.target[b] = target;
        if (!copies) a.source[b] = -1;
    }
}

// used ones among 4 pages from p on
__device__ __forceinline__ int used4(const CompactArgs &a, int64_t p, int (&use)[4])
{
    if (p + 4 <= a.pages) {
        const intx4 u = ((const intx4_as_int *)(a.uses + p))->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) use[i] = u[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) use[i] = p + i < a.pages ? a.uses[p + i] : 0;
    }
    return (use[0] > 0) + (use[1] > 0) + (use[2] > 0) + (use[3] > 0);
}

// used pages of each segment
__global__ void __launch_bounds__(1024) k_pages_count(CompactArgs a)
{
    __shared__ int sums[2][16];
    int use[4], n;
    before(used4(a, (int64_t)blockIdx.x * kSegment + 4 * threadIdx.x, use), sums, &n);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = n;
}

// Each segment's free pages below U (the pages in use) and used ones from U on, as the k-th of all.  COUNTED: the segments' used pages are known; in
// a small pool every workgroup counts them all itself.
template <bool COUNTED>
__global__ void __launch_bounds__(1024) k_pages_pair(CompactArgs a, int segments)
{
    __shared__ int sums[2][16];
    const int64_t p0 = (int64_t)blockIdx.x * kSegment;
    int use[4], earlier, all, below, n;                  // used pages before this segment, all of them, and those before page U
    if constexpr (!COUNTED) {
        uint32_t used = 0;                               // 4 bits for this lane's pages of each segment
#pragma unroll
        for (int i = 0; i < kSegments; ++i) {
            used4(a, (int64_t)i * kSegment + 4 * threadIdx.x, use);
#pragma unroll
            for (int j = 0; j < 4; ++j) used |= (uint32_t)(use[j] > 0) << (4 * i + j);
        }
        const auto bits = [](int n) { return n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1; };
        before(__builtin_popcount(used & bits(4 * blockIdx.x)), sums, &earlier, __builtin_popcount(used), &all);
        const int segment = all / kSegment, rest = all - segment * kSegment - 4 * (int)threadIdx.x;      // of the last segment, from this lane's on
        n = __builtin_popcount(used & bits(4 * segment + (rest < 0 ? 0 : rest > 4 ? 4 : rest)));
    } else {
        int mine = 0, sum = 0;
        for (int i = threadIdx.x; i < segments; i += 1024) {
            const int c = a.counts[i];
            mine += i < (int)blockIdx.x ? c : 0;
            sum += c;
        }
        before(mine, sums, &earlier, sum, &all);
        const int segment = all / kSegment, rest = all - segment * kSegment - 4 * (int)threadIdx.x;
        n = 0;
        for (int i = threadIdx.x; i < segment; i += 1024) n += a.counts[i];
        used4(a, (int64_t)segment * kSegment + 4 * threadIdx.x, use);
#pragma unroll
        for (int i = 0; i < 4; ++i) n += i < rest && use[i] > 0;
    }
    const int64_t p = p0 + 4 * threadIdx.x;
    const int mine = used4(a, p, use);
    int all_here;
    int at = before(mine, sums, &all_here, n, &below) + earlier;         // used pages before this lane's
    const int moves = all - below;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (p + i >= a.pages) break;
        const bool used = use[i] > 0;
        if (p + i < all) {
            if (used) a.uses_out[p + i] = use[i];
            else a.target[(int)(p + i) - at] = (int)(p + i);
        } else {
            a.uses_out[p + i] = 0;
            if (used) {
                a.source[at - below] = (int)(p + i);
                a.rank[p + i] = at - below;
            }
        }
        at += used;
    }
    // the places of pairs that there are none of
    for (int64_t k = p0 / 2 + threadIdx.x; k < (p0 + kSegment) / 2 && k < a.pages / 2; k += 1024)
        if (k >= moves) a.source[k] = a.target[k] = -1;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.used = all;
}

// The table's entries and the counts of pages that moved
__global__ void __launch_bounds__(256) k_pages_move(CompactArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int all = *a.used;
    if (i < a.entries) {
        int id = a.table[i];
        if (id >= all && id < a.pages && a.uses[id] > 0) id = a.target[a.rank[id]];
        a.table_out[i] = id;
    }
    if (i < a.pages / 2) {
        const int to = a.target[i];
        if (to >= 0) a.uses_out[to] = a.uses[a.source[i]];
    }
}

constexpr int64_t kCopy = 16384;                         // bytes of each cache that a workgroup copies

// Memory bounds it: 5000 pages of 8 heads of 16 tokens of 128, 329 MB read and written, 58 us, 5.7 TB/s.  Every lane's reads are on their way
// before it writes.  STREAM: more than the memory-side cache holds; a few pages are read again soon.
template <bool STREAM>
__global__ void __launch_bounds__(256) k_cache_copy(CopyArgs a, int parts)
{
    const int64_t pair = blockIdx.x / parts;
    const int part = blockIdx.x - (int)pair * parts;
    const int64_t from = a.source[pair], to = a.target[pair];
    if (from < 0 || to < 0 || from >= a.pages || to >= a.pages || from == to) return;
    const int64_t left = a.bytes - part * kCopy;
    constexpr int kEach = kCopy / (256 * 16);
    const int64_t at = part * kCopy + threadIdx.x * 16;
    uintx4 k[kEach], v[kEach];
    const auto load = [](const uint8_t *p) { return STREAM ? __builtin_nontemporal_load((const uintx4 *)p) : *(const uintx4 *)p; };
    const auto store = [](uintx4 w, uint8_t *p) {
        if constexpr (STREAM) __builtin_nontemporal_store(w, (uintx4 *)p);
        else *(uintx4 *)p = w;
    };
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (threadIdx.x * 16 + i * 4096 < left) {
            k[i] = load(a.k + from * a.bytes + at + i * 4096);
            v[i] = load(a.v + from * a.bytes + at + i * 4096);
        }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (threadIdx.x * 16 + i * 4096 < left) {
            store(k[i], a.k + to * a.bytes + at + i * 4096);
            store(v[i], a.v + to * a.bytes + at + i * 4096);
        }
    if (part == 0)
        for (int h = threadIdx.x; h < a.heads; h += 256) {
            a.k_scales[to * a.heads + h] = a.k_scales[from * a.heads + h];
            a.v_scales[to * a.heads + h] = a.v_scales[from * a.heads + h];
        }
}

int log2_of(int page) { return page == 16 ? 4 : page == 32 ? 5 : 6; }

}  // namespace

hipError_t launch_pages_fork(const ForkArgs &a, hipStream_t stream)
{
    return launch_many(k_pages_fork, (int64_t)a.rows + a.sequences, 256, stream, a, log2_of(a.page));
}

hipError_t launch_pages_reserve(const ReserveArgs &a, hipStream_t stream)
{
    return launch_many(k_pages_reserve, 1, 1024, stream, a, log2_of(a.page));
}

hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t stream)
{
    const int64_t segments = (a.pages + kSegment - 1) / kSegment, most = a.entries > a.pages / 2 ? a.entries : a.pages / 2;
    if (!launchable((most + 255) / 256, 256)) return kTooLarge;        // before anything is
    hipError_t e = hipSuccess;
    if (segments <= kSegments) {
        e = launch_many(k_pages_pair<false>, segments, 1024, stream, a, (int)segments);
    } else {
        e = launch_many(k_pages_count, segments, 1024, stream, a);
        if (e == hipSuccess) e = launch_many(k_pages_pair<true>, segments, 1024, stream, a, (int)segments);
    }
    if (e == hipSuccess && most) e = launch_many(k_pages_move, (most + 255) / 256, 256, stream, a);
    return e;
}

hipError_t launch_cache_copy(const CopyArgs &a, hipStream_t stream)
{
    const int64_t parts = (a.bytes + kCopy - 1) / kCopy;
    if (beyond_cache((double)a.count * a.bytes * 2)) return launch_many(k_cache_copy<true>, a.count * parts, 256, stream, a, (int)parts);
    return launch_many(k_cache_copy<false>, a.count * parts, 256, stream, a, (int)parts);
}

}  // namespace fc
