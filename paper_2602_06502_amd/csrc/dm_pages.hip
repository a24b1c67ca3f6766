// The page tables of the next step (sequences continued, forked, freed and
// grown), live pages moved together, and page data copied.
//
// Whole numbers throughout: reference counts go up and down by atomic adds,
// whose order does not matter, and every choice (which writer keeps a page,
// which free page goes where) goes by lowest index or rank, so results do not
// depend on timing.
//
// The tables' calls are chains of short passes over the pages, the sequences
// and the table entries; each pass needs the whole of the one before it, so
// launches and waits bound them.  Small calls are one workgroup with everything
// that the passes share in LDS; in large ones passes over entries take equal
// shares of them, however long the tables are.
#include <algorithm>

#include "dm_internal.h"
#include "dm_pages.h"

namespace dm {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kPageBlock = 1024;      // pages counted together
constexpr int kPlanThreads = 1024;         // the scan's workgroup
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr uint32_t kBadBlock = 1u << 31;   // of a page block's count: a negative reference count
constexpr int64_t kMaxLen = 1ll << 31;     // sequences are shorter

// ctl words: what a call has found wrong, then what its scan has found.  What the
// count pass finds has a word of its own: waves of one workgroup that read a word
// while others set it could go different ways, past barriers and each other's
// counts.
enum : int { kCtlErr = 0, kCtlNeed = 1, kCtlMoves = 2, kCtlLive = 3, kCtlBelow = 4, kCtlTurn = 5,
             kCtlCountErr = 6, kCtlWords = 8 };

// Work arrays of a call.
struct Work {
    uint32_t* ctl;     // [kCtlWords]
    uint32_t* blk;     // [blocks] free (compact: live) pages per page block, then before it
    int32_t* delta;    // [n_pages] change of the count by the tables
    uint32_t* writers; // [n_pages] sequences about to write into the page
    uint32_t* first;   // [n_pages] the first of them
    uint32_t* list;    // [n_pages] free pages in order
    uint32_t* heir;    // [n] first sequence of the result that continues s
    uint32_t* base;    // [m] new pages before j's
    uint32_t* place;   // [m] j's move, kNone: none
    int64_t* at;       // [m + 1] the result's entries before j's
};

struct ForkIn {
    const int64_t* off;
    const int32_t* page;
    const int64_t* len;
    uint32_t n;
    int64_t entries;
    const int32_t* ref;
    uint32_t n_pages, blocks;
    const int32_t* src;
    const int64_t* keep;
    const int64_t* grow;
    uint32_t m;
    uint32_t shift;  // log2(B)
};

__device__ __forceinline__ int64_t pages_of(int64_t tokens, uint32_t shift)
{
    return (tokens + (1ll << shift) - 1) >> shift;
}

// Sum over a workgroup of `threads` (a multiple of 64), in every thread.
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t* lds)
{
    const uint32_t s = (uint32_t)wave_sum_u64(v);
    __syncthreads();
    if (lane_id() == 0)
        lds[threadIdx.x / kWave] = s;
    __syncthreads();
    uint32_t t = 0;
    for (uint32_t w = 0; w < blockDim.x / kWave; w++)
        t += lds[w];
    return t;
}

// Exclusive prefix sums of K values a thread over the workgroup; tot: the sums.
template <int K>
__device__ __forceinline__ void block_scan(uint64_t (&v)[K], uint64_t (&tot)[K], uint64_t* lds)
{
    const uint32_t w = threadIdx.x / kWave, nw = blockDim.x / kWave;
    uint64_t incl[K];
#pragma unroll
    for (int k = 0; k < K; k++)
        incl[k] = wave_incl_sum_u64(v[k], 0);
    __syncthreads();
    if (lane_id() == kWave - 1)
#pragma unroll
        for (int k = 0; k < K; k++)
            lds[k * nw + w] = incl[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; k++) {
        uint64_t before = 0, all = 0;
        for (uint32_t i = 0; i < nw; i++) {
            const uint64_t x = lds[k * nw + i];
            before += i < w ? x : 0;
            all += x;
        }
        v[k] = before + incl[k] - v[k];
        tot[k] = all;
    }
}

// Entries [e0, e1) of a CSR with bounds at[0 .. n] (row r begins at at[r]), by a
// workgroup of kThreads, kEach entries a thread at once so that their reads
// overlap.  make(r): what is to be known of a row, gathered once for all of its
// entries (LDS holds it where the segment has few rows); use(entries, their
// places in their rows, rows, number of entries that exist).
constexpr int kEach = 4;
constexpr uint32_t kSegment = kThreads * kEach, kHeldRows = kThreads;

template <typename Row>
struct SegmentLds {
    int64_t at[kHeldRows];
    Row row[kHeldRows];
};

template <typename Row, typename Make, typename Use>
__device__ __forceinline__ void for_entries(const int64_t* at, uint32_t n, int64_t e0, int64_t e1,
                                            SegmentLds<Row>& lds, Make&& make, Use&& use)
{
    const uint32_t r0 = wave_find(at, n, 1, e0), rows = wave_find(at, n, 1, e1 - 1) - r0 + 1;
    const bool held = rows <= kHeldRows;
    __syncthreads();
    if (held && threadIdx.x < rows) {
        lds.at[threadIdx.x] = at[r0 + threadIdx.x];
        lds.row[threadIdx.x] = make(r0 + threadIdx.x);
    }
    __syncthreads();
    const int64_t* b = held ? lds.at : at + r0;
    int64_t e[kEach], i[kEach];
    Row row[kEach];
    int there = 0;
#pragma unroll
    for (int k = 0; k < kEach; k++) {
        e[k] = e0 + threadIdx.x + k * kThreads;
        if (e[k] >= e1)
            continue;
        there = k + 1;
        uint32_t lo = 0, hi = rows;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (b[mid] <= e[k])
                lo = mid;
            else
                hi = mid;
        }
        i[k] = e[k] - b[lo];
        row[k] = held ? lds.row[lo] : make(r0 + lo);
    }
    use(e, i, row, there);
}

// Is sequence s's table well formed?
__device__ __forceinline__ bool table_ok(const ForkIn& a, uint32_t s)
{
    const int64_t o0 = a.off[s], o1 = a.off[s + 1], len = a.len[s];
    return o0 >= 0 && o1 >= o0 && o1 <= a.entries && len >= 0 && len < kMaxLen &&
           pages_of(len, a.shift) <= o1 - o0;
}

// Is what sequence j of the result takes well formed?
__device__ __forceinline__ bool next_ok(const ForkIn& a, uint32_t j)
{
    const int64_t keep = a.keep[j], grow = a.grow[j];
    if (keep < 0 || grow < 0 || keep >= kMaxLen || grow >= kMaxLen || keep + grow >= kMaxLen)
        return false;
    const uint32_t s = keep ? (uint32_t)a.src[j] : 0;
    return !keep || (s < a.n && table_ok(a, s) && keep <= a.len[s]);
}

__device__ __forceinline__ bool writes(const ForkIn& a, int64_t keep, int64_t grow)
{
    return (keep & ((1ll << a.shift) - 1)) && grow;
}

// Rank of each thread's page among those of its kind (mine), in order over the
// workgroup's pages; rank0 moves on by their number.
__device__ __forceinline__ uint32_t rank_of(bool mine, uint32_t& rank0, uint32_t* lds)
{
    const uint64_t mask = ballot(mine);
    __syncthreads();
    if (lane_id() == 0)
        lds[threadIdx.x / kWave] = __popcll(mask);
    __syncthreads();
    uint32_t rank = rank0 + __popcll(mask & ((1ull << lane_id()) - 1));
    for (uint32_t k = 0; k < blockDim.x / kWave; k++) {
        if (k < threadIdx.x / kWave)
            rank += lds[k];
        rank0 += lds[k];
    }
    return rank;
}

// Pass 1: work arrays cleared; free pages counted per block of pages.
__global__ __launch_bounds__(kThreads) void fork_init_kernel(ForkIn a, Work w)
{
    __shared__ uint32_t lds[kThreads / kWave];
    const uint32_t b = blockIdx.x;
    if (b < a.blocks) {
        uint32_t free_pages = 0;
        for (uint32_t i = threadIdx.x; i < kPageBlock; i += kThreads) {
            const uint64_t p = (uint64_t)b * kPageBlock + i;
            if (p >= a.n_pages)
                break;
            const int32_t r = a.ref[p];
            // at most 1024 pages a block: negative counts join above bit 16
            free_pages += r == 0 ? 1u : r < 0 ? 1u << 16 : 0u;
            w.delta[p] = 0;
            w.writers[p] = 0;
            w.first[p] = kNone;
        }
        const uint32_t t = block_sum(free_pages, lds);
        if (threadIdx.x == 0)
            w.blk[b] = (t & 0xFFFFu) | (t >> 16 ? kBadBlock : 0u);
    }
    const uint64_t stride = (uint64_t)gridDim.x * kThreads;
    for (uint64_t s = (uint64_t)b * kThreads + threadIdx.x; s < a.n; s += stride)
        w.heir[s] = kNone;
    if (b == 0 && threadIdx.x < kCtlWords)
        w.ctl[threadIdx.x] = 0;
}

// Pass 2: sequences checked, the first continuation of each found; beside it,
// the last workgroup sums the page blocks' counts.
__global__ __launch_bounds__(kThreads) void fork_check_kernel(ForkIn a, Work w)
{
    __shared__ uint64_t lds[kThreads / kWave];
    bool bad = false;
    if (blockIdx.x == gridDim.x - 1) {
        uint64_t carry = 0;
        for (uint32_t b0 = 0; b0 < a.blocks; b0 += kThreads) {
            const uint32_t b = b0 + threadIdx.x;
            const uint32_t x = b < a.blocks ? w.blk[b] : 0;
            uint64_t v[1] = {x & ~kBadBlock}, tot[1];
            bad |= (x & kBadBlock) != 0;
            block_scan<1>(v, tot, lds);
            if (b < a.blocks)
                w.blk[b] = (uint32_t)(carry + v[0]);
            carry += tot[0];
        }
        if (threadIdx.x == 0)
            w.ctl[kCtlLive] = (uint32_t)carry;  // free pages
    } else {
        const uint64_t stride = (uint64_t)(gridDim.x - 1) * kThreads;
        const uint64_t t0 = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
        for (uint64_t s = t0; s < a.n; s += stride)
            bad |= !table_ok(a, (uint32_t)s);
        for (uint64_t j = t0; j < a.m; j += stride) {
            if (!next_ok(a, (uint32_t)j))
                bad = true;
            else if (a.keep[j])
                atomicMin(&w.heir[a.src[j]], (uint32_t)j);
        }
    }
    if (bad)
        atomicOr(&w.ctl[kCtlErr], kErrInval);
}

// Pass 3: the counts' changes, and the free pages listed.  The first
// continuation of s takes s's references over, so that a sequence that just
// goes on changes nothing: what it does not keep is released (equal shares of
// the entries), and every other continuation's pages get a reference more (a
// wave each).
__global__ __launch_bounds__(kThreads) void fork_count_kernel(ForkIn a, Work w, uint32_t segments)
{
    __shared__ SegmentLds<int64_t> rows;
    __shared__ uint32_t lds[kThreads / kWave];
    if (w.ctl[kCtlErr])
        return;
    bool bad = false;
    const uint64_t all = (uint64_t)a.blocks + segments + (a.m + kThreads / kWave - 1) / (kThreads / kWave);
    for (uint64_t u = blockIdx.x; u < all; u += gridDim.x) {
        if (u < segments) {
            const int64_t first = a.n ? a.off[0] : 0, last = a.n ? a.off[a.n] : 0;
            const int64_t e0 = first + (int64_t)u * kSegment;
            if (e0 >= last)
                continue;
            for_entries<int64_t>(
                a.off, a.n, e0, e0 + kSegment < last ? e0 + kSegment : last, rows,
                [&](uint32_t s) -> int64_t {
                    const uint32_t h = w.heir[s];
                    return h == kNone ? 0 : pages_of(a.keep[h], a.shift);
                },
                [&](const int64_t* e, const int64_t* i, const int64_t* kept, int there) {
                    uint32_t p[kEach];
                    int32_t r[kEach];
#pragma unroll
                    for (int k = 0; k < kEach; k++)
                        p[k] = k < there ? (uint32_t)a.page[e[k]] : 0;
#pragma unroll
                    for (int k = 0; k < kEach; k++)
                        r[k] = p[k] < a.n_pages ? a.ref[p[k]] : 0;
#pragma unroll
                    for (int k = 0; k < kEach; k++)
                        if (k < there) {
                            bad |= r[k] <= 0;
                            if (r[k] > 0 && i[k] >= kept[k])
                                atomicAdd(&w.delta[p[k]], -1);
                        }
                });
        } else if (u < (uint64_t)a.blocks + segments) {
            const uint64_t b = u - segments;
            uint32_t rank0 = w.blk[b];
            for (uint32_t i0 = 0; i0 < kPageBlock; i0 += kThreads) {
                const uint64_t p = b * kPageBlock + i0 + threadIdx.x;
                const bool mine = p < a.n_pages && a.ref[p] == 0;
                const uint32_t rank = rank_of(mine, rank0, lds);
                if (mine)
                    w.list[rank] = (uint32_t)p;
            }
        } else {
            const uint64_t j = (u - a.blocks - segments) * (kThreads / kWave) + threadIdx.x / kWave;
            const int64_t keep = j < a.m ? a.keep[j] : 0;
            if (!keep)
                continue;
            const uint32_t s = (uint32_t)a.src[j];
            const int64_t o0 = a.off[s], kept = pages_of(keep, a.shift);
            if (w.heir[s] != (uint32_t)j)
                for (int64_t i = lane_id(); i < kept; i += kWave) {
                    const uint32_t p = (uint32_t)a.page[o0 + i];
                    if (p < a.n_pages)
                        atomicAdd(&w.delta[p], 1);
                }
            if (lane_id() == 0 && writes(a, keep, a.grow[j])) {
                const uint32_t p = (uint32_t)a.page[o0 + kept - 1];
                if (p < a.n_pages) {
                    atomicAdd(&w.writers[p], 1u);
                    atomicMin(&w.first[p], (uint32_t)j);
                }
            }
        }
    }
    if (bad)
        atomicOr(&w.ctl[kCtlCountErr], kErrInval);
}

// Pass 4: new pages, entries and moves before each sequence, and whether all of
// them have room.  Whether a sequence copies a page takes a chain of scattered
// reads, a thread a sequence over the chip (by one workgroup 18 us for 4,096);
// the last workgroup to finish sums.
__global__ __launch_bounds__(kPlanThreads) void fork_scan_kernel(ForkIn a, Work w, dm_pages_out out,
                                                                 uint32_t* status)
{
    __shared__ uint64_t lds[3 * kPlanThreads / kWave];
    __shared__ uint32_t turn;
    const uint32_t err = w.ctl[kCtlErr] | w.ctl[kCtlCountErr], free_pages = w.ctl[kCtlLive];
    constexpr uint32_t kCopies = 1u << 31;  // of base: the sequence copies a page
    for (uint64_t x = (uint64_t)blockIdx.x * kPlanThreads + threadIdx.x; err == 0 && x < a.m;
         x += (uint64_t)gridDim.x * kPlanThreads) {
        const uint32_t j = (uint32_t)x;
        const int64_t keep = a.keep[j], grow = a.grow[j], kept = pages_of(keep, a.shift);
        const uint32_t all = (uint32_t)pages_of(keep + grow, a.shift);
        bool copy = false;
        if (writes(a, keep, grow)) {
            // a writer alone with its page keeps it, of several the first
            const uint32_t p = (uint32_t)a.page[a.off[a.src[j]] + kept - 1];
            copy = !(a.ref[p] + w.delta[p] == (int32_t)w.writers[p] && w.first[p] == j);
        }
        agent_store(&w.base[j], (all - (uint32_t)kept + copy) | (copy ? kCopies : 0));
        agent_store(&w.place[j], all);
    }
    if (!last_to_arrive(&w.ctl[kCtlTurn], &turn))
        return;
    constexpr int kItems = 4;
    uint64_t at[3] = {0, 0, 0};
    for (uint32_t j0 = 0; err == 0 && j0 < a.m; j0 += kPlanThreads * kItems) {
        uint64_t v[3] = {0, 0, 0}, tot[3];
        uint32_t fresh[kItems], all[kItems];
#pragma unroll
        for (int k = 0; k < kItems; k++) {
            const uint32_t j = j0 + threadIdx.x * kItems + k;
            fresh[k] = j < a.m ? agent_load(&w.base[j]) : 0;
            all[k] = j < a.m ? agent_load(&w.place[j]) : 0;
            v[0] += fresh[k] & ~kCopies;
            v[1] += all[k];
            v[2] += fresh[k] >> 31;
        }
        block_scan<3>(v, tot, lds);
#pragma unroll
        for (int k = 0; k < kItems; k++) {
            const uint32_t j = j0 + threadIdx.x * kItems + k;
            if (j < a.m) {
                w.base[j] = (uint32_t)(at[0] + v[0]);
                w.at[j] = (int64_t)(at[1] + v[1]);
                w.place[j] = fresh[k] & kCopies ? (uint32_t)(at[2] + v[2]) : kNone;
            }
            v[0] += fresh[k] & ~kCopies;
            v[1] += all[k];
            v[2] += fresh[k] >> 31;
        }
        for (int k = 0; k < 3; k++)
            at[k] += tot[k];
    }
    if (threadIdx.x)
        return;
    const uint32_t e = err ? err : at[0] > free_pages || at[1] > out.cap || at[2] > out.move_cap ? kErrFull : 0;
    w.at[a.m] = (int64_t)at[1];
    w.ctl[kCtlErr] = e;
    w.ctl[kCtlNeed] = (uint32_t)at[0];
    out.moves[0] = e ? 0 : (int64_t)at[2];
    if (e)
        atomicOr(status, e);
}

// The count of page p after the call (r: before; not free).
__device__ __forceinline__ int32_t count_after(int32_t r, int32_t delta, uint32_t writers)
{
    const int32_t total = r + delta;
    return total - (int32_t)(writers && total == (int32_t)writers ? writers - 1 : writers);
}

// What the entries of a sequence of the result are made of.
struct NextRow {
    int64_t from;           // the kept pages' first entry
    uint32_t own;           // entries that stay as they are
    uint32_t base, place;   // first new page's rank, move
};

// Pass 5: counts, bounds and lengths, and equal shares of the result's entries.
__global__ __launch_bounds__(kThreads) void fork_write_kernel(ForkIn a, Work w, dm_pages_out out,
                                                              uint32_t segments)
{
    __shared__ SegmentLds<NextRow> rows;
    __shared__ uint32_t lds[kThreads / kWave];
    if (w.ctl[kCtlErr])
        return;
    const uint32_t need = w.ctl[kCtlNeed];
    for (uint64_t u = blockIdx.x; u < (uint64_t)a.blocks + segments; u += gridDim.x) {
        if (u < segments) {
            const int64_t last = w.at[a.m], e0 = (int64_t)u * kSegment;
            if (e0 >= last)
                continue;
            for_entries<NextRow>(
                w.at, a.m, e0, e0 + kSegment < last ? e0 + kSegment : last, rows,
                [&](uint32_t j) -> NextRow {
                    const int64_t keep = a.keep[j];
                    const uint32_t place = w.place[j];
                    return NextRow{keep ? a.off[a.src[j]] : 0,
                                   (uint32_t)pages_of(keep, a.shift) - (place != kNone), w.base[j], place};
                },
                [&](const int64_t* e, const int64_t* i, const NextRow* r, int there) {
                    int32_t p[kEach];
#pragma unroll
                    for (int k = 0; k < kEach; k++)
                        if (k < there)
                            p[k] = i[k] < r[k].own ? a.page[r[k].from + i[k]]
                                                   : (int32_t)w.list[r[k].base + (i[k] - r[k].own)];
#pragma unroll
                    for (int k = 0; k < kEach; k++)
                        if (k < there) {
                            out.page[e[k]] = p[k];
                            if (r[k].place != kNone && i[k] == r[k].own) {
                                out.move_src[r[k].place] = a.page[r[k].from + i[k]];
                                out.move_dst[r[k].place] = p[k];
                            }
                        }
                });
            continue;
        }
        const uint64_t b = u - segments;
        uint32_t rank0 = w.blk[b];
        for (uint32_t i0 = 0; i0 < kPageBlock; i0 += kThreads) {
            const uint64_t p = b * kPageBlock + i0 + threadIdx.x;
            const int32_t r = p < a.n_pages ? a.ref[p] : 1;
            const uint32_t rank = rank_of(r == 0, rank0, lds);
            if (p < a.n_pages)
                out.ref[p] = r ? count_after(r, w.delta[p], w.writers[p]) : rank < need;
        }
    }
    const uint64_t stride = (uint64_t)gridDim.x * kThreads;
    for (uint64_t j = (uint64_t)blockIdx.x * kThreads + threadIdx.x; j <= a.m; j += stride) {
        out.off[j] = w.at[j];
        if (j < a.m)
            out.len[j] = a.keep[j] + a.grow[j];
    }
}

// ---------------------------------------------------------------------------
// A small call in one workgroup: the same passes, what they share in LDS.
// ---------------------------------------------------------------------------

constexpr uint32_t kSmallPages = 8192, kSmallRows = 1024;  // what LDS holds
constexpr uint64_t kSmallEntries = 32768;

// Entries of tables, by the room for them: a caller that does not wait for their number
// gives the most there can be; where that is many times the pages there are, pages
// would have to be shared by as many sequences.
uint64_t entries_about(uint64_t room, uint32_t n_pages) { return room < 4ull * n_pages ? room : 4ull * n_pages; }

// Is a call the faster in one workgroup?  us of fork there and in passes, by pages,
// sequences and entries: 767, 24, 600: 9.1 and 21.9; 2,048, 256, 4,096: 19.5 and 25.5;
// 4,096, 256, 4,096: 22.5 and 26.0; 4,096, 256, 8,192: 30.2 and 25.5; 8,192, 64, 8,192:
// 31.9 and 23.7; 8,192, 1,024, 32,768: 101 and 29.  Of compact: 2,048, 256, 4,096: 6.8
// and 15.2; 8,192, 256, 8,192: 14.8 and 15.3; 8,192, 256, 16,384: 19.0 and 15.3; with
// 65,536 sequences of 4,096 entries 20.7 and 75.8.
bool fork_is_small(uint32_t n_pages, uint64_t rows, uint64_t room)
{
    return n_pages <= kSmallPages && rows <= kSmallRows && room <= kSmallEntries &&
           n_pages + entries_about(room, n_pages) + 8 * rows < 12288;
}
bool compact_is_small(uint32_t n_pages, uint64_t room)
{
    return n_pages <= kSmallPages && room <= kSmallEntries && n_pages + entries_about(room, n_pages) / 2 <= 12288;
}

__global__ __launch_bounds__(kPlanThreads) void fork_small_kernel(ForkIn a, dm_pages_out out, uint32_t* status)
{
    __shared__ int32_t delta[kSmallPages];
    __shared__ uint32_t first[kSmallPages];
    __shared__ __attribute__((aligned(4))) uint16_t writers[kSmallPages];
    __shared__ uint16_t list[kSmallPages];
    __shared__ uint64_t lds[3 * kPlanThreads / kWave];
    __shared__ uint32_t heir[kSmallRows];
    __shared__ int64_t in_at[kSmallRows + 1], out_at[kSmallRows + 1];
    __shared__ uint32_t base[kSmallRows], place[kSmallRows], held[kSmallRows];
    __shared__ int64_t from[kSmallRows];
    __shared__ uint32_t err;
    uint32_t* words = reinterpret_cast<uint32_t*>(lds);
    const uint32_t tid = threadIdx.x, j = tid;
    if (tid == 0)
        err = 0;
    heir[tid] = kNone;
    if (tid < a.n)
        in_at[tid] = a.off[tid];
    if (tid == 0 && a.n)
        in_at[a.n] = a.off[a.n];
    __syncthreads();
    // free pages listed, arrays cleared
    bool bad = false;
    uint32_t free_pages = 0;
    for (uint32_t p0 = 0; p0 < a.n_pages; p0 += kPlanThreads) {
        const uint32_t p = p0 + tid;
        const int32_t r = p < a.n_pages ? a.ref[p] : 1;
        const uint32_t rank = rank_of(r == 0, free_pages, words);
        bad |= r < 0;
        if (r == 0)
            list[rank] = (uint16_t)p;
        if (p < a.n_pages) {
            delta[p] = 0;
            first[p] = kNone;
            writers[p] = 0;
        }
    }
    if (tid < a.n)
        bad |= !table_ok(a, tid);
    const bool mine = j < a.m;
    int64_t keep = 0, grow = 0, src_at = 0;
    uint32_t s = 0;
    if (mine) {
        if (next_ok(a, j)) {
            keep = a.keep[j];
            grow = a.grow[j];
            if (keep) {
                s = (uint32_t)a.src[j];
                src_at = in_at[s];
                atomicMin(&heir[s], j);
            }
        } else {
            bad = true;
        }
        held[j] = (uint32_t)pages_of(keep, a.shift);
        from[j] = src_at;
    }
    if (bad)
        atomicOr(&err, kErrInval);
    __syncthreads();
    if (err == 0) {
        // what the first continuations do not keep is released
        const int64_t e1 = a.n ? in_at[a.n] : 0;
        for (int64_t e = (a.n ? in_at[0] : 0) + tid; e < e1; e += kPlanThreads) {
            uint32_t lo = 0, hi = a.n;
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (in_at[mid] <= e)
                    lo = mid;
                else
                    hi = mid;
            }
            const uint32_t p = (uint32_t)a.page[e], h = heir[lo];
            if (p >= a.n_pages || a.ref[p] <= 0)
                atomicOr(&err, kErrInval);
            else if (e - in_at[lo] >= (h == kNone ? 0 : held[h]))
                atomicAdd(&delta[p], -1);
        }
    }
    __syncthreads();
    const bool ok = err == 0;
    // the other continuations' pages, a wave for one
    for (uint32_t k = tid / kWave; ok && k < a.m; k += kPlanThreads / kWave)
        if (held[k] && heir[a.src[k]] != k)
            for (uint32_t i = lane_id(); i < held[k]; i += kWave)
                atomicAdd(&delta[a.page[from[k] + i]], 1);
    const bool writer = mine && writes(a, keep, grow);
    uint32_t p = kNone;
    if (ok && writer) {
        p = (uint32_t)a.page[src_at + held[j] - 1];
        atomicMin(&first[p], j);
        // 16-bit counts in pairs
        atomicAdd(reinterpret_cast<uint32_t*>(writers) + p / 2, p % 2 ? 1u << 16 : 1u);
    }
    __syncthreads();
    uint64_t v[3] = {0, 0, 0}, tot[3];
    bool copy = false;
    if (ok && mine) {
        copy = writer && !(a.ref[p] + delta[p] == (int32_t)writers[p] && first[p] == j);
        v[1] = (uint64_t)pages_of(keep + grow, a.shift);
        v[0] = v[1] - held[j] + copy;
        v[2] = copy;
    }
    block_scan<3>(v, tot, lds);
    const uint32_t full = ok && (tot[0] > free_pages || tot[1] > out.cap || tot[2] > out.move_cap) ? kErrFull : 0;
    if (tid == 0) {
        out.moves[0] = ok && !full ? (int64_t)tot[2] : 0;
        if (err | full)
            atomicOr(status, err | full);
    }
    if (!ok || full)
        return;
    if (mine) {
        base[j] = (uint32_t)v[0];
        place[j] = copy ? (uint32_t)v[2] : kNone;
        out_at[j] = (int64_t)v[1];
        out.off[j] = (int64_t)v[1];
        out.len[j] = keep + grow;
    }
    if (tid == 0)
        out.off[a.m] = (int64_t)tot[1];
    __syncthreads();
    for (int64_t e = tid; e < (int64_t)tot[1]; e += kPlanThreads) {
        uint32_t lo = 0, hi = a.m;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (out_at[mid] <= e)
                lo = mid;
            else
                hi = mid;
        }
        const uint32_t i = (uint32_t)(e - out_at[lo]), pl = place[lo];
        const uint32_t own = held[lo] - (pl != kNone);
        if (i < own) {
            out.page[e] = a.page[from[lo] + i];
            continue;
        }
        const int32_t to = list[base[lo] + (i - own)];
        out.page[e] = to;
        if (pl != kNone && i == own) {
            out.move_src[pl] = a.page[from[lo] + i];
            out.move_dst[pl] = to;
        }
    }
    uint32_t rank0 = 0;
    for (uint32_t p0 = 0; p0 < a.n_pages; p0 += kPlanThreads) {
        const uint32_t q = p0 + tid;
        const int32_t r = q < a.n_pages ? a.ref[q] : 1;
        const uint32_t rank = rank_of(r == 0, rank0, words);
        if (q < a.n_pages)
            out.ref[q] = r ? count_after(r, delta[q], writers[q]) : rank < tot[0];
    }
}

// ---------------------------------------------------------------------------
// Compaction.
// ---------------------------------------------------------------------------

struct CompactIn {
    const int64_t* off;
    const int32_t* page;
    uint32_t n;
    int64_t entries;
    const int32_t* ref;
    uint32_t n_pages, blocks;
};

// A workgroup for a block of pages (live ones counted), then for a sequence
// (entries checked).  Each leaves its finding in a word of its own.
__global__ __launch_bounds__(kThreads) void compact_count_kernel(CompactIn a, Work w, uint32_t* flag)
{
    __shared__ uint32_t lds[kThreads / kWave];
    uint32_t bad = 0;
    for (uint64_t u = blockIdx.x; u < (uint64_t)a.blocks + a.n; u += gridDim.x) {
        if (u < a.blocks) {
            uint32_t live = 0;
            for (uint32_t i = threadIdx.x; i < kPageBlock; i += kThreads) {
                const uint64_t p = u * kPageBlock + i;
                const int32_t r = p < a.n_pages ? a.ref[p] : 0;
                live += r > 0;
                bad |= r < 0;
            }
            const uint32_t t = block_sum(live, lds);
            if (threadIdx.x == 0)
                w.blk[u] = t;
            continue;
        }
        const uint64_t s = u - a.blocks;
        const int64_t o0 = a.off[s], o1 = a.off[s + 1];
        if (o0 < 0 || o1 < o0 || o1 > a.entries) {
            bad = 1;
            continue;
        }
        for (int64_t e = o0 + threadIdx.x; e < o1; e += kThreads) {
            const uint32_t p = (uint32_t)a.page[e];
            bad |= p >= a.n_pages || a.ref[p] <= 0;
        }
    }
    const uint32_t any = block_sum(bad, lds);
    if (threadIdx.x == 0)
        flag[blockIdx.x] = any;
}

__global__ __launch_bounds__(kPlanThreads) void compact_scan_kernel(CompactIn a, Work w,
                                                                    const uint32_t* flag,
                                                                    uint32_t flags,
                                                                    dm_pages_out out,
                                                                    uint32_t* status)
{
    __shared__ uint64_t lds[kPlanThreads / kWave];
    __shared__ uint32_t err;
    if (threadIdx.x == 0)
        err = 0;
    __syncthreads();
    bool bad = false;
    for (uint32_t i = threadIdx.x; i < flags; i += kPlanThreads)
        bad |= flag[i] != 0;
    if (bad)
        atomicOr(&err, kErrInval);
    uint64_t live = 0;
    for (uint32_t b0 = 0; b0 < a.blocks; b0 += kPlanThreads) {
        const uint32_t b = b0 + threadIdx.x;
        uint64_t v[1] = {b < a.blocks ? w.blk[b] : 0}, tot[1];
        block_scan<1>(v, tot, lds);
        if (b < a.blocks)
            w.blk[b] = (uint32_t)(live + v[0]);
        live += tot[0];
    }
    __syncthreads();
    // live pages among the first `live`
    const uint32_t b = (uint32_t)live / kPageBlock, p = b * kPageBlock + threadIdx.x;
    uint64_t v[1] = {p < live && a.ref[p] > 0 ? 1ull : 0ull}, tot[1];
    block_scan<1>(v, tot, lds);
    if (threadIdx.x)
        return;
    const uint64_t below = (b < a.blocks ? w.blk[b] : live) + tot[0];
    const uint64_t moves = live - below;
    const uint32_t e = err ? err : moves > out.move_cap ? kErrFull : 0;
    w.ctl[kCtlErr] = e;
    w.ctl[kCtlLive] = (uint32_t)live;
    w.ctl[kCtlBelow] = (uint32_t)below;
    w.ctl[kCtlMoves] = (uint32_t)moves;
    out.moves[0] = e ? 0 : (int64_t)moves;
    if (e)
        atomicOr(status, e);
    else
        out.live[0] = (int64_t)live;
}

// Every page's rank among the live ones gives its end of a move.
__global__ __launch_bounds__(kThreads) void compact_list_kernel(CompactIn a, Work w, dm_pages_out out)
{
    __shared__ uint32_t lds[kThreads / kWave];
    if (w.ctl[kCtlErr])
        return;
    const uint32_t live = w.ctl[kCtlLive], below = w.ctl[kCtlBelow];
    uint32_t rank0 = w.blk[blockIdx.x];
    for (uint32_t i0 = 0; i0 < kPageBlock; i0 += kThreads) {
        const uint64_t p = (uint64_t)blockIdx.x * kPageBlock + i0 + threadIdx.x;
        const int32_t r = p < a.n_pages ? a.ref[p] : 0;
        const uint32_t rank = rank_of(r > 0, rank0, lds);
        if (p >= a.n_pages)
            continue;
        if (p < live) {
            if (r > 0)
                out.ref[p] = r;
            else
                out.move_dst[(uint32_t)p - rank] = (int32_t)p;
        } else {
            out.ref[p] = 0;
            if (r > 0) {
                out.move_src[rank - below] = (int32_t)p;
                w.first[p] = rank - below;
            }
        }
    }
}

// The moved pages' counts, and the tables' entries.
__global__ __launch_bounds__(kThreads) void compact_write_kernel(CompactIn a, Work w, dm_pages_out out)
{
    if (w.ctl[kCtlErr])
        return;
    const uint32_t live = w.ctl[kCtlLive], moves = w.ctl[kCtlMoves];
    const uint64_t stride = (uint64_t)gridDim.x * kThreads;
    const uint64_t t0 = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    for (uint64_t k = t0; k < moves; k += stride)
        out.ref[out.move_dst[k]] = a.ref[out.move_src[k]];
    for (uint64_t s = blockIdx.x; s < a.n; s += gridDim.x)
        for (int64_t e = a.off[s] + threadIdx.x; e < a.off[s + 1]; e += kThreads) {
            const int32_t p = a.page[e];
            out.page[e] = (uint32_t)p < live ? p : out.move_dst[w.first[p]];
        }
}

// A small call in one workgroup.
__global__ __launch_bounds__(kPlanThreads) void compact_small_kernel(CompactIn a, dm_pages_out out,
                                                                     uint32_t* status)
{
    __shared__ uint16_t rank_at[kSmallPages], hole[kSmallPages];
    __shared__ uint32_t words[kPlanThreads / kWave], err;
    const uint32_t tid = threadIdx.x;
    if (tid == 0)
        err = 0;
    uint32_t live = 0;
    bool bad = false;
    for (uint32_t p0 = 0; p0 < a.n_pages; p0 += kPlanThreads) {
        const uint32_t p = p0 + tid;
        const int32_t r = p < a.n_pages ? a.ref[p] : 0;
        const uint32_t rank = rank_of(r > 0, live, words);
        bad |= r < 0;
        if (p < a.n_pages)
            rank_at[p] = (uint16_t)rank;
    }
    for (uint32_t s = tid; s < a.n; s += kPlanThreads) {
        const int64_t o0 = a.off[s], o1 = a.off[s + 1];
        bad |= o0 < 0 || o1 < o0 || o1 > a.entries;
    }
    if (bad)
        atomicOr(&err, kErrInval);
    __syncthreads();
    const bool ordered = err == 0;
    __syncthreads();
    const int64_t e0 = ordered && a.n ? a.off[0] : 0, e1 = ordered && a.n ? a.off[a.n] : 0;
    for (int64_t e = e0 + tid; e < e1; e += kPlanThreads) {
        const uint32_t p = (uint32_t)a.page[e];
        if (p >= a.n_pages || a.ref[p] <= 0)
            atomicOr(&err, kErrInval);
    }
    __syncthreads();
    const uint32_t below = live < a.n_pages ? rank_at[live] : live, moves = live - below;
    const uint32_t wrong = err ? err : moves > out.move_cap ? kErrFull : 0;
    if (tid == 0) {
        out.moves[0] = wrong ? 0 : (int64_t)moves;
        if (wrong)
            atomicOr(status, wrong);
        else
            out.live[0] = live;
    }
    if (wrong)
        return;
    for (uint32_t p = tid; p < live; p += kPlanThreads)
        if (a.ref[p] == 0) {
            hole[p - rank_at[p]] = (uint16_t)p;
            out.move_dst[p - rank_at[p]] = (int32_t)p;
        } else {
            out.ref[p] = a.ref[p];
        }
    __syncthreads();
    for (uint32_t p = live + tid; p < a.n_pages; p += kPlanThreads) {
        const int32_t r = a.ref[p];
        out.ref[p] = 0;
        if (r > 0) {
            out.move_src[rank_at[p] - below] = (int32_t)p;
            out.ref[hole[rank_at[p] - below]] = r;
        }
    }
    for (int64_t e = e0 + tid; e < e1; e += kPlanThreads) {
        const uint32_t p = (uint32_t)a.page[e];
        out.page[e] = p < live ? (int32_t)p : (int32_t)hole[rank_at[p] - below];
    }
}

// ---------------------------------------------------------------------------
// Page data.
// ---------------------------------------------------------------------------

struct CopyIn {
    uint8_t* pool[2];
    uint64_t layer_bytes, page_bytes;
    uint32_t layers, n_pages;
    const int32_t* src;
    const int32_t* dst;
    const int64_t* count;
    uint64_t cap;
    uint32_t parts;       // of a page
    uint32_t part_bytes;  // a multiple of 16
};

// A workgroup moves a part of a page at a time: 16 KB, four 16-byte loads a
// thread in flight.  Bound by HBM.
constexpr uint32_t kCopyPart = 16384;

__global__ __launch_bounds__(kThreads) void pages_copy_kernel(CopyIn a, uint32_t* status)
{
    const int64_t count = *a.count;
    uint64_t moves = count < 0 ? 0 : (uint64_t)count;
    if (moves > a.cap) {
        moves = a.cap;
        if (blockIdx.x == 0 && threadIdx.x == 0)
            atomicOr(status, kErrFull);
    }
    const uint64_t per = (uint64_t)a.layers * 2 * a.parts, all = moves * per;
    for (uint64_t u = blockIdx.x; u < all; u += gridDim.x) {
        const uint64_t i = u / per;
        uint32_t x = (uint32_t)(u % per);
        const uint32_t part = x % a.parts;
        x /= a.parts;
        const uint32_t s = (uint32_t)a.src[i], d = (uint32_t)a.dst[i];
        if (s >= a.n_pages || d >= a.n_pages) {
            if (threadIdx.x == 0)
                atomicOr(status, kErrInval);
            continue;
        }
        uint8_t* pool = a.pool[x & 1] + (uint64_t)(x >> 1) * a.layer_bytes;
        const uint64_t begin = (uint64_t)part * a.part_bytes;
        const uint64_t end = begin + a.part_bytes < a.page_bytes ? begin + a.part_bytes : a.page_bytes;
        const uint8_t* from = pool + s * a.page_bytes;
        uint8_t* to = pool + d * a.page_bytes;
        v4u32 r[kCopyPart / kThreads / 16];
#pragma unroll
        for (int k = 0; k < (int)(kCopyPart / kThreads / 16); k++) {
            const uint64_t at = begin + (uint64_t)(k * kThreads + threadIdx.x) * 16;
            if (at < end)
                r[k] = *reinterpret_cast<const v4u32*>(from + at);
        }
#pragma unroll
        for (int k = 0; k < (int)(kCopyPart / kThreads / 16); k++) {
            const uint64_t at = begin + (uint64_t)(k * kThreads + threadIdx.x) * 16;
            if (at < end)
                *reinterpret_cast<v4u32*>(to + at) = r[k];
        }
    }
}

uint64_t up256(uint64_t x) { return (x + 255) & ~255ull; }

template <typename T>
T* carve(uint8_t*& p, uint64_t n)
{
    T* t = reinterpret_cast<T*>(p);
    p += up256(n * sizeof(T));
    return t;
}

uint32_t log2_of(uint32_t x)
{
    uint32_t k = 0;
    while ((1u << k) < x)
        k++;
    return k;
}

}  // namespace

hipError_t pages_fork(dm_ctx* c, const dm_page_tables& in, const int32_t* ref, uint32_t n_pages,
                      const int32_t* src, const int64_t* keep, const int64_t* grow, uint64_t m,
                      const dm_pages_out& out)
{
    const uint32_t blocks = (n_pages + kPageBlock - 1) / kPageBlock;
    const ForkIn a{in.off, in.page, in.len, (uint32_t)in.n, (int64_t)in.entries, ref, n_pages,
                   blocks, src, keep, grow, (uint32_t)m, log2_of(c->cfg.block_size)};
    hipStream_t st = c->stream;
    if (fork_is_small(n_pages, std::max(in.n, m), std::max(in.entries, out.cap))) {
        fork_small_kernel<<<1, kPlanThreads, 0, st>>>(a, out, c->d_status);
        return hipGetLastError();
    }
    hipError_t e;
    uint8_t* p = static_cast<uint8_t*>(scratch_get(
        c, kSlotPages,
        up256(4 * kCtlWords) + up256(4 * (uint64_t)blocks) + 4 * up256(4 * (uint64_t)n_pages) +
            up256(4 * in.n) + 2 * up256(4 * m) + up256(8 * (m + 1)),
        &e));
    if (!p)
        return e;
    Work w;
    w.ctl = carve<uint32_t>(p, kCtlWords);
    w.blk = carve<uint32_t>(p, blocks);
    w.delta = carve<int32_t>(p, n_pages);
    w.writers = carve<uint32_t>(p, n_pages);
    w.first = carve<uint32_t>(p, n_pages);
    w.list = carve<uint32_t>(p, n_pages);
    w.heir = carve<uint32_t>(p, in.n);
    w.base = carve<uint32_t>(p, m);
    w.place = carve<uint32_t>(p, m);
    w.at = carve<int64_t>(p, m + 1);
    const uint32_t over = grid_for(in.n > m ? in.n : m, kThreads, 4096);
    const uint32_t in_segments = (uint32_t)((in.entries + kSegment - 1) / kSegment);
    const uint32_t out_segments = (uint32_t)((out.cap + kSegment - 1) / kSegment);
    fork_init_kernel<<<blocks > over ? blocks : over, kThreads, 0, st>>>(a, w);
    fork_check_kernel<<<over + 1, kThreads, 0, st>>>(a, w);
    fork_count_kernel<<<grid_for((uint64_t)blocks + in_segments + (m + 3) / 4, 1), kThreads, 0, st>>>(
        a, w, in_segments);
    fork_scan_kernel<<<grid_for(m, kPlanThreads, 256), kPlanThreads, 0, st>>>(a, w, out, c->d_status);
    fork_write_kernel<<<grid_for((uint64_t)blocks + out_segments, 1), kThreads, 0, st>>>(a, w, out, out_segments);
    return hipGetLastError();
}

hipError_t pages_compact(dm_ctx* c, const dm_page_tables& in, const int32_t* ref,
                         uint32_t n_pages, const dm_pages_out& out)
{
    const uint32_t blocks = (n_pages + kPageBlock - 1) / kPageBlock;
    const CompactIn a{in.off, in.page, (uint32_t)in.n, (int64_t)in.entries, ref, n_pages, blocks};
    hipStream_t st = c->stream;
    if (compact_is_small(n_pages, in.entries)) {
        compact_small_kernel<<<1, kPlanThreads, 0, st>>>(a, out, c->d_status);
        return hipGetLastError();
    }
    const uint32_t grid = grid_for(blocks + in.n, 1);
    hipError_t e;
    uint8_t* p = static_cast<uint8_t*>(scratch_get(
        c, kSlotPages,
        up256(4 * kCtlWords) + up256(4 * (uint64_t)blocks) + up256(4 * (uint64_t)n_pages) +
            up256(4 * (uint64_t)grid),
        &e));
    if (!p)
        return e;
    Work w{};
    w.ctl = carve<uint32_t>(p, kCtlWords);
    w.blk = carve<uint32_t>(p, blocks);
    w.first = carve<uint32_t>(p, n_pages);
    uint32_t* flag = carve<uint32_t>(p, grid);
    compact_count_kernel<<<grid, kThreads, 0, st>>>(a, w, flag);
    compact_scan_kernel<<<1, kPlanThreads, 0, st>>>(a, w, flag, grid, out, c->d_status);
    compact_list_kernel<<<blocks, kThreads, 0, st>>>(a, w, out);
    compact_write_kernel<<<grid_for(in.n, 1), kThreads, 0, st>>>(a, w, out);
    return hipGetLastError();
}

hipError_t pages_copy(dm_ctx* c, const dm_kv_pages& kv, const int32_t* src, const int32_t* dst,
                      const int64_t* count, uint64_t cap)
{
    CopyIn a;
    a.pool[0] = static_cast<uint8_t*>(kv.k);
    a.pool[1] = static_cast<uint8_t*>(kv.v);
    a.layer_bytes = 2 * (uint64_t)kv.layer_stride;
    a.page_bytes = 2ull * kv.kv_heads * c->cfg.block_size * kv.head_dim;
    a.layers = kv.layers;
    a.n_pages = kv.n_pages;
    a.src = src;
    a.dst = dst;
    a.count = count;
    a.cap = cap;
    a.parts = (uint32_t)((a.page_bytes + kCopyPart - 1) / kCopyPart);
    a.part_bytes = kCopyPart;
    const uint64_t units = cap * kv.layers * 2 * a.parts;
    pages_copy_kernel<<<grid_for(units, 1, 16u * c->n_cu), kThreads, 0, c->stream>>>(a, c->d_status);
    return hipGetLastError();
}

}  // namespace dm
