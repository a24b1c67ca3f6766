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
// launches bound small calls and the scan by one workgroup large ones.
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

// ctl words: what a call has found wrong, then what its scan has found.
enum : int { kCtlErr = 0, kCtlNeed = 1, kCtlMoves = 2, kCtlLive = 3, kCtlBelow = 4, kCtlWords = 8 };

// Work arrays of a call.
struct Work {
    uint32_t* ctl;     // [kCtlWords]
    uint32_t* blk;     // [blocks + 1] free (compact: live) pages per page block, then before it
    int32_t* delta;    // [n_pages] change of the count by the tables
    uint32_t* writers; // [n_pages] sequences about to write into the page
    uint32_t* first;   // [n_pages] the first of them
    uint32_t* heir;    // [n] first sequence of the result that continues s
    uint32_t* base;    // [m] new pages before j's
    uint32_t* place;   // [m] j's move, kNone: none
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

// Is sequence s's table well formed?
__device__ __forceinline__ bool table_ok(const ForkIn& a, uint32_t s)
{
    const int64_t o0 = a.off[s], o1 = a.off[s + 1], len = a.len[s];
    return o0 >= 0 && o1 >= o0 && o1 <= a.entries && len >= 0 && len < kMaxLen &&
           pages_of(len, a.shift) <= o1 - o0;
}

// Pass 2: sequences checked; the first continuation of each found.
__global__ __launch_bounds__(kThreads) void fork_check_kernel(ForkIn a, Work w)
{
    const uint64_t stride = (uint64_t)gridDim.x * kThreads;
    const uint64_t t0 = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    bool bad = false;
    for (uint64_t s = t0; s < a.n; s += stride)
        bad |= !table_ok(a, (uint32_t)s);
    for (uint64_t j = t0; j < a.m; j += stride) {
        const int64_t keep = a.keep[j], grow = a.grow[j];
        if (keep < 0 || grow < 0 || keep >= kMaxLen || grow >= kMaxLen || keep + grow >= kMaxLen) {
            bad = true;
            continue;
        }
        if (!keep)
            continue;
        const uint32_t s = (uint32_t)a.src[j];
        if (s >= a.n || !table_ok(a, s) || keep > a.len[s]) {
            bad = true;
            continue;
        }
        atomicMin(&w.heir[s], (uint32_t)j);
    }
    if (bad)
        atomicOr(&w.ctl[kCtlErr], kErrInval);
}

// Pass 3, a workgroup for a sequence: the counts' changes.  The first
// continuation of s takes s's references over, so that a sequence that just
// goes on changes nothing: what it does not keep is released, and every other
// continuation's pages get a reference more.
__global__ __launch_bounds__(kThreads) void fork_count_kernel(ForkIn a, Work w)
{
    if (w.ctl[kCtlErr])
        return;
    bool bad = false;
    for (uint64_t u = blockIdx.x; u < (uint64_t)a.n + a.m; u += gridDim.x) {
        if (u < a.n) {
            const uint32_t h = w.heir[u];
            const int64_t o0 = a.off[u], o1 = a.off[u + 1];
            const int64_t kept = h == kNone ? 0 : pages_of(a.keep[h], a.shift);
            for (int64_t e = o0 + threadIdx.x; e < o1; e += kThreads) {
                const uint32_t p = (uint32_t)a.page[e];
                if (p >= a.n_pages || a.ref[p] <= 0)
                    bad = true;
                else if (e - o0 >= kept)
                    atomicAdd(&w.delta[p], -1);
            }
            continue;
        }
        const uint32_t j = (uint32_t)(u - a.n);
        const int64_t keep = a.keep[j];
        if (!keep)
            continue;
        const uint32_t s = (uint32_t)a.src[j];
        const int64_t o0 = a.off[s], kept = pages_of(keep, a.shift);
        if (w.heir[s] != j)
            for (int64_t i = threadIdx.x; i < kept; i += kThreads) {
                const uint32_t p = (uint32_t)a.page[o0 + i];
                if (p < a.n_pages)
                    atomicAdd(&w.delta[p], 1);
            }
        if (threadIdx.x == 0 && (keep & ((1ll << a.shift) - 1)) && a.grow[j]) {
            const uint32_t p = (uint32_t)a.page[o0 + kept - 1];
            if (p < a.n_pages) {
                atomicAdd(&w.writers[p], 1u);
                atomicMin(&w.first[p], j);
            }
        }
    }
    if (bad)
        atomicOr(&w.ctl[kCtlErr], kErrInval);
}

// Does writer j of page p get a page of its own?
__device__ __forceinline__ bool copies(const ForkIn& a, const Work& w, uint32_t p, uint32_t j)
{
    const bool alone = a.ref[p] + w.delta[p] == (int32_t)w.writers[p];
    return !(alone && w.first[p] == j);
}

// Pass 4, one workgroup: free pages before each block, new pages, entries and
// moves before each sequence; whether all of them have room.
__global__ __launch_bounds__(kPlanThreads) void fork_scan_kernel(ForkIn a, Work w, dm_pages_out out,
                                                                 uint32_t* status)
{
    __shared__ uint64_t lds[3 * kPlanThreads / kWave];
    __shared__ uint32_t err;
    if (threadIdx.x == 0) {
        err = w.ctl[kCtlErr];
        out.moves[0] = 0;
    }
    __syncthreads();
    uint64_t carry = 0;
    bool bad = false;
    for (uint32_t b0 = 0; b0 < a.blocks; b0 += kPlanThreads) {
        const uint32_t b = b0 + threadIdx.x;
        const uint32_t x = b < a.blocks ? w.blk[b] : 0;
        uint64_t v[1] = {x & ~kBadBlock}, tot[1];
        bad |= (x & kBadBlock) != 0;
        block_scan<1>(v, tot, lds);
        if (b < a.blocks)
            w.blk[b] = (uint32_t)(carry + v[0]);
        carry += tot[0];
    }
    if (bad)
        atomicOr(&err, kErrInval);
    __syncthreads();
    const bool ok = err == 0;
    uint64_t at[3] = {0, 0, 0};
    for (uint32_t j0 = 0; ok && j0 < a.m; j0 += kPlanThreads) {
        const uint32_t j = j0 + threadIdx.x;
        uint64_t v[3] = {0, 0, 0}, tot[3];
        bool copy = false;
        if (j < a.m) {
            const int64_t keep = a.keep[j], grow = a.grow[j];
            const int64_t kept = pages_of(keep, a.shift), all = pages_of(keep + grow, a.shift);
            if ((keep & ((1ll << a.shift) - 1)) && grow)
                copy = copies(a, w, (uint32_t)a.page[a.off[a.src[j]] + kept - 1], j);
            v[0] = all - kept + copy;
            v[1] = all;
            v[2] = copy;
        }
        block_scan<3>(v, tot, lds);
        if (j < a.m) {
            w.base[j] = (uint32_t)(at[0] + v[0]);
            w.place[j] = copy ? (uint32_t)(at[2] + v[2]) : kNone;
        }
        for (int k = 0; k < 3; k++)
            at[k] += tot[k];
    }
    // free pages, entries, moves, and entries of the reference counts
    uint32_t full = ok && (at[0] > carry || at[1] > out.cap || at[2] > out.move_cap) ? kErrFull : 0;
    if (threadIdx.x == 0) {
        w.ctl[kCtlErr] = err | full;
        w.ctl[kCtlNeed] = (uint32_t)at[0];
        if (err | full)
            atomicOr(status, err | full);
        else
            out.moves[0] = (int64_t)at[2];
    }
    if (!ok || full)
        return;
    uint64_t o = 0;
    for (uint32_t j0 = 0; j0 < a.m; j0 += kPlanThreads) {
        const uint32_t j = j0 + threadIdx.x;
        const int64_t len = j < a.m ? a.keep[j] + a.grow[j] : 0;
        uint64_t v[1] = {(uint64_t)pages_of(len, a.shift)}, tot[1];
        block_scan<1>(v, tot, lds);
        if (j < a.m) {
            out.off[j] = (int64_t)(o + v[0]);
            out.len[j] = len;
        }
        o += tot[0];
    }
    if (threadIdx.x == 0)
        out.off[a.m] = (int64_t)o;
}

// Pass 5: page blocks give their free pages away and write the counts; then
// a workgroup for a sequence copies the entries that it keeps.
__global__ __launch_bounds__(kThreads) void fork_write_kernel(ForkIn a, Work w, dm_pages_out out)
{
    if (w.ctl[kCtlErr])
        return;
    const uint32_t need = w.ctl[kCtlNeed];
    for (uint64_t u = blockIdx.x; u < (uint64_t)a.blocks + a.m; u += gridDim.x) {
        if (u < a.blocks) {
            __shared__ uint32_t lds[kThreads / kWave];
            uint32_t rank0 = w.blk[u];
            for (uint32_t i0 = 0; i0 < kPageBlock; i0 += kThreads) {
                const uint64_t p = u * kPageBlock + i0 + threadIdx.x;
                const int32_t r = p < a.n_pages ? a.ref[p] : 1;
                const uint64_t mask = ballot(r == 0);
                __syncthreads();
                if (lane_id() == 0)
                    lds[threadIdx.x / kWave] = __popcll(mask);
                __syncthreads();
                uint32_t rank = rank0;
                for (uint32_t k = 0; k < kThreads / kWave; k++) {
                    if (k < threadIdx.x / kWave)
                        rank += lds[k];
                    rank0 += lds[k];
                }
                rank += __popcll(mask & ((1ull << lane_id()) - 1));
                if (p >= a.n_pages)
                    continue;
                if (r > 0) {
                    const uint32_t wr = w.writers[p];
                    const int32_t total = r + w.delta[p];
                    out.ref[p] = total - (int32_t)(wr && total == (int32_t)wr ? wr - 1 : wr);
                } else if (rank >= need) {
                    out.ref[p] = 0;
                } else {
                    // the sequence whose new pages the rank falls among
                    uint32_t lo = 0, hi = a.m;
                    while (hi - lo > 1) {
                        const uint32_t mid = (lo + hi) / 2;
                        if (w.base[mid] <= rank)
                            lo = mid;
                        else
                            hi = mid;
                    }
                    const uint32_t k = rank - w.base[lo], place = w.place[lo];
                    const bool copy = place != kNone;
                    const int64_t kept = pages_of(a.keep[lo], a.shift);
                    out.page[out.off[lo] + kept - copy + k] = (int32_t)p;
                    if (copy && k == 0)
                        out.move_dst[place] = (int32_t)p;
                    out.ref[p] = 1;
                }
            }
            continue;
        }
        const uint32_t j = (uint32_t)(u - a.blocks);
        const int64_t keep = a.keep[j];
        if (!keep)
            continue;
        const uint32_t place = w.place[j];
        const int64_t from = a.off[a.src[j]], to = out.off[j], kept = pages_of(keep, a.shift);
        for (int64_t i = threadIdx.x; i < kept - (place != kNone); i += kThreads)
            out.page[to + i] = a.page[from + i];
        if (threadIdx.x == 0 && place != kNone)
            out.move_src[place] = a.page[from + kept - 1];
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
        const uint64_t mask = ballot(r > 0);
        __syncthreads();
        if (lane_id() == 0)
            lds[threadIdx.x / kWave] = __popcll(mask);
        __syncthreads();
        uint32_t rank = rank0;
        for (uint32_t k = 0; k < kThreads / kWave; k++) {
            if (k < threadIdx.x / kWave)
                rank += lds[k];
            rank0 += lds[k];
        }
        rank += __popcll(mask & ((1ull << lane_id()) - 1));
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
    hipError_t e;
    uint8_t* p = static_cast<uint8_t*>(scratch_get(
        c, kSlotPages,
        up256(4 * kCtlWords) + up256(4 * (uint64_t)(blocks + 1)) + 3 * up256(4 * (uint64_t)n_pages) +
            up256(4 * in.n) + 2 * up256(4 * m),
        &e));
    if (!p)
        return e;
    Work w;
    w.ctl = carve<uint32_t>(p, kCtlWords);
    w.blk = carve<uint32_t>(p, blocks + 1);
    w.delta = carve<int32_t>(p, n_pages);
    w.writers = carve<uint32_t>(p, n_pages);
    w.first = carve<uint32_t>(p, n_pages);
    w.heir = carve<uint32_t>(p, in.n);
    w.base = carve<uint32_t>(p, m);
    w.place = carve<uint32_t>(p, m);
    const ForkIn a{in.off, in.page, in.len, (uint32_t)in.n, (int64_t)in.entries, ref, n_pages,
                   blocks, src, keep, grow, (uint32_t)m, log2_of(c->cfg.block_size)};
    hipStream_t st = c->stream;
    const uint32_t over = grid_for(in.n > m ? in.n : m, kThreads, 4096);
    fork_init_kernel<<<blocks > over ? blocks : over, kThreads, 0, st>>>(a, w);
    fork_check_kernel<<<over, kThreads, 0, st>>>(a, w);
    fork_count_kernel<<<grid_for(in.n + m, 1), kThreads, 0, st>>>(a, w);
    fork_scan_kernel<<<1, kPlanThreads, 0, st>>>(a, w, out, c->d_status);
    fork_write_kernel<<<grid_for(blocks + m, 1), kThreads, 0, st>>>(a, w, out);
    return hipGetLastError();
}

hipError_t pages_compact(dm_ctx* c, const dm_page_tables& in, const int32_t* ref,
                         uint32_t n_pages, const dm_pages_out& out)
{
    const uint32_t blocks = (n_pages + kPageBlock - 1) / kPageBlock;
    const uint32_t grid = grid_for(blocks + in.n, 1);
    hipError_t e;
    uint8_t* p = static_cast<uint8_t*>(scratch_get(
        c, kSlotPages,
        up256(4 * kCtlWords) + up256(4 * (uint64_t)(blocks + 1)) + up256(4 * (uint64_t)n_pages) +
            up256(4 * (uint64_t)grid),
        &e));
    if (!p)
        return e;
    Work w{};
    w.ctl = carve<uint32_t>(p, kCtlWords);
    w.blk = carve<uint32_t>(p, blocks + 1);
    w.first = carve<uint32_t>(p, n_pages);
    uint32_t* flag = carve<uint32_t>(p, grid);
    const CompactIn a{in.off, in.page, (uint32_t)in.n, (int64_t)in.entries, ref, n_pages, blocks};
    hipStream_t st = c->stream;
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
