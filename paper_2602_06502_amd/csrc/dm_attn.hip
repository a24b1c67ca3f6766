// Attention of a batch's new tokens over KV pages, a prefix that several
// sequences share read once for all of them.
//
// For KV head h the rows of a sequence are its (token, query head of h) pairs,
// row = token * ratio + head; the rows of all sequences of a run follow each
// other the same way.  A unit is a set of rows with a range of keys: a run over
// its shared prefix (no mask: every new token comes after it), or a sequence
// over the rest of its keys.  The plan cuts units into items: a tile of rows,
// a chunk of keys, a KV head.  Each row's parts, if it has more than one, are
// joined by their maxima and sums at the end.
//
// An item makes one pass over its keys with the running maximum and sum of the
// softmax.  Products are taken transposed, S^T = K Q^T and O^T = V^T P^T, on
// 32x32x16 matrix instructions: a lane then holds one row's scores for 16 of 32
// keys, its maximum and sum are its own registers' and one exchange between
// the halves of the wave, and the scores of a lane, in the order they come, are
// the second product's right operand (the keys of its contraction in another
// order, which V's transposing LDS reads follow), so weights never leave their
// lane.
//
//   narrow tiles: 16 rows, on 16x16x32 instructions; the four waves take every
//     fourth 32 keys, each through its own part of LDS, and are joined at the
//     end.  Weights meet the values in two parts, as exactly as 32 bits nearly.
//     For rows that are few: bound by reading the pages.
//   wide tiles: 128 rows, 32 a wave, on a shared tile of 64 keys (two in LDS).
//     Bound by the matrix and vector units: two prompts of 7,000 to 8,192 tokens, 32
//     query and 8 key heads of 128, 897 to 985 us by the card, 880 to 968 TFLOP/s.
//     Weights are rounded to the pages' type: outputs are within 0.0023 relative of 64
//     bits, where one rounding makes 0.0017.  In two parts, as in narrow tiles, the same
//     prompts took 1,265 us on a card where they take 980; with the maximum moved
//     whenever it grows, so that the heaviest weight is 1 exactly, 1,028 (0.0019).
//   a few rows on a few keys: narrow tiles of more waves, nothing cut or joined.
//     Bound by launches and the chain of reads.
#include "dm_attn.h"

namespace dm {
namespace {

constexpr int kPlanThreads = 512;

// The tiles of a unit, by its rows, and their cost a key: a wide one of 128 rows takes up
// to twice a narrow one's time.  wide: rows of a wide tile, a power of two (the plan's
// kernel divides by it where its chain of steps waits); kNarrow: there are none.
__device__ __forceinline__ uint32_t tile_flags(uint64_t rows, uint32_t wide)
{
    return rows <= kNarrowRows || wide == kNarrow ? 0 : kUnitWide;
}
__device__ __forceinline__ uint64_t tiles_of(uint64_t rows, uint32_t wide)
{
    const uint32_t tile = rows <= kNarrowRows ? kNarrow : wide;
    return (rows + tile - 1) >> __builtin_ctz(tile);
}
__device__ __forceinline__ uint64_t weight_of(uint64_t rows, uint32_t wide)
{
    return tiles_of(rows, wide) * (tile_flags(rows, wide) ? wide / (kWide / 2) : 1);
}

// Are the runs' bounds in order?
__device__ __forceinline__ bool run_ok(const TokenBatch& b, uint32_t g)
{
    const int64_t g0 = b.group_off[g], g1 = b.group_off[g + 1];
    return g0 >= 0 && g1 >= g0 && g1 <= (int64_t)b.n;
}

__device__ __forceinline__ uint64_t block_sum64(uint64_t v, uint64_t* lds)
{
    const uint64_t s = wave_sum_u64(v);
    __syncthreads();
    if (lane_id() == 0)
        lds[threadIdx.x / kWave] = s;
    __syncthreads();
    uint64_t t = 0;
    for (uint32_t w = 0; w < kPlanThreads / kWave; w++)
        t += lds[w];
    return t;
}

struct PlanIn {
    TokenBatch b;
    uint32_t q_heads, kv_heads, ratio, head_dim, wide;
    uint64_t target;     // items wanted
    uint64_t part_rows;  // rows of parts there is room for (0: no unit is cut)
    uint32_t* arrived;   // workgroups that are done with their sequences; zero between calls
};

constexpr uint32_t kNoSay = 0xFFFFFFFFu;
constexpr uint32_t kLdsRuns = 1024;

// How many leading pages sequence s could share with its run's first one (kNoSay:
// it has no row that sees a key).  A shared prefix ends before the first new
// token of every sequence that has any.  By the whole workgroup (least: a word
// of LDS), or by a wave (least null).
__device__ __forceinline__ void common_pages(const PlanIn& a, const PlanView& pv, uint32_t s, uint32_t* least)
{
    const TokenBatch& b = a.b;
    const SeqView v = sequence_view(b, s);
    const RunOf r = run_of(b, s);
    uint32_t limit = 0;
    if (r.ok && (v.ntok == 0 || (!v.bad && v.len == 0))) {
        limit = kNoSay;
    } else if (r.ok && !v.bad && v.pos0 > 0) {
        // the first one's entries, and that they are there, are what is needed
        const int64_t f0 = b.off[r.g0], f1 = b.off[r.g0 + 1];
        const int64_t have = f0 < 0 || f1 < f0 || f1 > b.entries ? 0 : f1 - f0, own = v.pos0 >> b.shift;
        limit = (uint32_t)(have < own ? have : own);
        const int32_t *mine = b.page + v.off, *theirs = b.page + f0;
        if (least) {
            __syncthreads();
            if (threadIdx.x == 0)
                *least = limit;
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < limit; i += kPlanThreads)
                if (mine[i] != theirs[i]) {
                    atomicMin(least, i);
                    break;
                }
            __syncthreads();
            limit = *least;
        } else {
            constexpr uint32_t kAt = 4;  // reads of a lane at once
            for (uint32_t i0 = 0; i0 < limit; i0 += kAt * kWave) {
                uint32_t x[kAt], y[kAt], first = limit;
#pragma unroll
                for (uint32_t k = 0; k < kAt; k++) {
                    const uint32_t i = i0 + k * kWave + lane_id();
                    x[k] = i < limit ? mine[i] : 0;
                    y[k] = i < limit ? theirs[i] : 0;
                }
#pragma unroll
                for (uint32_t k = 0; k < kAt; k++) {
                    const uint64_t differ = ballot(x[k] != y[k]);
                    if (differ) {
                        const uint32_t at = i0 + k * kWave + (uint32_t)__builtin_ctzll(differ);
                        first = at < first ? at : first;
                    }
                }
                limit = first;
            }
        }
    }
    if (least ? threadIdx.x == 0 : lane_id() == 0) {
        agent_store(&pv.limit[s], limit);
        agent_store(&pv.run[s], r.ok ? r.g : kNoSay);
    }
}

// Sequences up to this many have a workgroup each, more a wave each: workgroups
// that arrive at one counter take 11 ns each.
constexpr uint32_t kPlanWorkgroups = 64;

// What the plan's last workgroup reads of a run, and of a sequence.
struct RunView {
    uint32_t tok0, ntok;
    int64_t off;
    bool ok;
};
__device__ __forceinline__ RunView run_view(const TokenBatch& b, uint32_t g)
{
    RunView r{0, 0, 0, false};
    const int64_t g0 = b.group_off[g], g1 = b.group_off[g + 1];
    if (g0 < 0 || g1 < g0 || g1 > (int64_t)b.n || g0 >= (int64_t)b.n)
        return r;
    const int64_t t0 = b.q_off[g0], t1 = b.q_off[g1];
    r.off = b.off[g0];
    r.ok = t0 >= 0 && t1 >= t0 && t1 <= (int64_t)b.q_tokens;
    r.tok0 = r.ok ? (uint32_t)t0 : 0;
    r.ntok = r.ok ? (uint32_t)(t1 - t0) : 0;
    return r;
}

// The units of a run over its shared pages, and of a sequence.
__device__ __forceinline__ Unit run_unit(const PlanIn& a, const RunView& r, uint32_t pages)
{
    Unit u{};
    if (pages == 0)
        return u;
    u.tok0 = r.tok0;
    u.ntok = r.ntok;
    u.key1 = pages << a.b.shift;
    u.off = r.off;
    u.table = pages;
    u.flags = kUnitParts | tile_flags((uint64_t)u.ntok * a.ratio, a.wide);
    return u;
}

__device__ __forceinline__ Unit sequence_unit(const PlanIn& a, const SeqView& v, uint32_t pages)
{
    Unit u{};
    u.tok0 = v.tok0;
    u.ntok = v.ntok;
    u.key0 = v.len ? pages << a.b.shift : 0;
    u.key1 = (uint32_t)v.len;
    u.off = v.off;
    u.table = (uint32_t)((v.len + (1ll << a.b.shift) - 1) >> a.b.shift);
    u.pos0 = (int32_t)v.pos0;
    u.flags = kUnitCausal | (pages ? kUnitParts : 0) | tile_flags((uint64_t)u.ntok * a.ratio, a.wide);
    return u;
}

// Is a pass of its own over `pages` common pages worth it for a run?  Where the
// run's rows together make clearly fewer tiles, over more than a chunk of keys.
__device__ __forceinline__ bool worth_sharing(const PlanIn& a, const RunView& r, uint32_t pages, uint32_t gain)
{
    return pages != 0 && pages != kNoSay && r.ok && ((uint64_t)pages << a.b.shift) >= kChunk &&
           2 * (uint64_t)gain >= 3 * weight_of((uint64_t)r.ntok * a.ratio, a.wide);
}

// Which runs share their prefixes, the chunk, and the units' items.  With
// runs, a workgroup for a sequence first, and the last one to finish goes on
// alone (a launch less).  Its threads read what they need of their first unit
// once and keep it; beyond 512 units the others are read again, and kept in the
// plan between the steps.
__global__ __launch_bounds__(kPlanThreads) void attn_plan_kernel(PlanIn a, PlanView pv, uint32_t* status)
{
    __shared__ uint64_t lds[2 * kPlanThreads / kWave];
    __shared__ uint32_t run_pages[kLdsRuns], run_gain[kLdsRuns], run_tok0[kLdsRuns], run_ntok[kLdsRuns];
    __shared__ uint32_t most, least;
    const TokenBatch& b = a.b;
    const uint32_t units = b.groups + b.n, tid = threadIdx.x;
    if (b.groups) {
        constexpr uint32_t kPlanWaves = kPlanThreads / kWave;
        if (b.n <= kPlanWorkgroups)
            for (uint32_t s = blockIdx.x; s < b.n; s += gridDim.x)
                common_pages(a, pv, s, &least);
        else
            for (uint32_t s = blockIdx.x * kPlanWaves + tid / kWave; s < b.n; s += gridDim.x * kPlanWaves)
                common_pages(a, pv, s, nullptr);
        if (!last_to_arrive(a.arrived, &least))
            return;
        if (tid == 0)
            agent_store(a.arrived, 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    }
    uint32_t* pages = b.groups <= kLdsRuns ? run_pages : pv.shared;
    uint32_t* gain = b.groups <= kLdsRuns ? run_gain : pv.gain;
    bool bad = false;
    auto settle = [&] {
        if (b.groups > kLdsRuns)
            __threadfence();
        __syncthreads();
    };
    // the thread's first unit: a run, or a sequence with its run and common pages
    const bool is_run = tid < b.groups;
    const uint32_t s0 = tid - b.groups;
    RunView rv{0, 0, 0, false};
    SeqView sv{0, 0, 0, 0, 0, false};
    uint32_t run = kNoSay, limit = kNoSay;
    if (is_run) {
        rv = run_view(b, tid);
    } else if (tid < units) {
        sv = sequence_view(b, s0);
        if (b.groups) {
            run = agent_load(&pv.run[s0]);
            limit = agent_load(&pv.limit[s0]);
        }
    }
    if (b.groups) {
        for (uint32_t g = tid; g < b.groups; g += kPlanThreads) {
            pages[g] = kNoSay;
            gain[g] = 0;
            bad |= !run_ok(b, g) || (g == 0 && b.group_off[0] != 0) ||
                   (g + 1 == b.groups && b.group_off[b.groups] != (int64_t)b.n);
        }
        settle();
        for (uint32_t i = tid; i < units; i += kPlanThreads) {
            if (i < b.groups)
                continue;
            const uint32_t s = i - b.groups;
            const uint32_t g = i == tid ? run : agent_load(&pv.run[s]);
            const SeqView v = i == tid ? sv : sequence_view(b, s);
            if (g >= b.groups)
                continue;
            atomicMin(&pages[g], i == tid ? limit : agent_load(&pv.limit[s]));
            if (v.len)
                atomicAdd(&gain[g], (uint32_t)weight_of((uint64_t)v.ntok * a.ratio, a.wide));
        }
        settle();
        for (uint32_t g = tid; g < b.groups; g += kPlanThreads) {
            const RunView r = g == tid ? rv : run_view(b, g);
            pages[g] = worth_sharing(a, r, pages[g], gain[g]) ? pages[g] : 0;
            if (b.groups <= kLdsRuns) {
                run_tok0[g] = r.tok0;
                run_ntok[g] = r.ntok;
            }
        }
        settle();
    }
    // 0: as wanted; 1: without sharing and without cuts, if the parts of the
    // first try have no room
    for (int attempt = 0; attempt < 2; attempt++) {
        auto cost_of = [&](const Unit& u) -> uint64_t {
            return u.ntok ? weight_of((uint64_t)u.ntok * a.ratio, a.wide) * (u.key1 - u.key0) : 0;
        };
        Unit mine{};
        uint64_t cost = 0;
        for (uint32_t i = tid; i < units; i += kPlanThreads) {
            Unit u{};
            if (i < b.groups) {
                u = run_unit(a, i == tid ? rv : run_view(b, i), attempt ? 0 : pages[i]);
            } else {
                const uint32_t s = i - b.groups;
                const uint32_t g = i == tid || !b.groups ? run : agent_load(&pv.run[s]);
                const SeqView v = i == tid ? sv : sequence_view(b, s);
                bad |= v.bad;
                u = sequence_unit(a, v, attempt || g >= b.groups ? 0 : pages[g]);
            }
            cost += cost_of(u);
            if (i == tid)
                mine = u;
            else
                pv.unit[i] = u;
        }
        cost = block_sum64(cost, lds) * a.kv_heads;
        uint64_t chunk = (cost / a.target + kChunk) / kChunk * kChunk;
        if (attempt || a.part_rows == 0 || chunk > 0x80000000ull)
            chunk = 0x80000000ull;
        // items and rows of parts before each unit
        if (tid == 0)
            most = 1;
        uint64_t items = 0, rows = 0;
        for (uint32_t u0 = 0; u0 < units; u0 += kPlanThreads) {
            const uint32_t i = u0 + tid;
            uint64_t it = 0, rw = 0;
            Unit u = mine;
            if (u0 && i < units)
                u = pv.unit[i];
            __syncthreads();
            if (i < units && u.ntok) {
                const uint64_t r = (uint64_t)u.ntok * a.ratio;
                u.chunks = (uint32_t)((u.key1 - u.key0 + chunk - 1) / chunk);
                if (u.chunks == 0)
                    u.chunks = 1;
                if (u.chunks > 1)
                    u.flags |= kUnitParts;
                it = tiles_of(r, a.wide) * u.chunks * a.kv_heads;
                if (u.flags & kUnitParts) {
                    rw = r * u.chunks * a.kv_heads;
                    atomicMax(&most, u.chunks);
                }
            }
            const uint64_t i1 = wave_incl_sum_u64(it, 0), r1 = wave_incl_sum_u64(rw, 0);
            constexpr uint32_t kPlanWaves = kPlanThreads / kWave;
            if (lane_id() == kWave - 1) {
                lds[tid / kWave] = i1;
                lds[kPlanWaves + tid / kWave] = r1;
            }
            __syncthreads();
            uint64_t ib = items, rb = rows;
            for (uint32_t w = 0; w < kPlanWaves; w++) {
                const uint64_t x = lds[w], y = lds[kPlanWaves + w];
                if (w < tid / kWave) {
                    ib += x;
                    rb += y;
                }
                items += x;
                rows += y;
            }
            u.item0 = (uint32_t)(ib + i1 - it);
            u.part0 = (uint32_t)(rb + r1 - rw);
            if (i < b.groups)
                gain[i] = u.part0;  // for the run's sequences, which come later
            if (b.groups)
                settle();
            if (i < units && i >= b.groups) {
                const uint32_t s = i - b.groups;
                const uint32_t g = u0 == 0 || !b.groups ? run : agent_load(&pv.run[s]);
                if (!attempt && g < b.groups && pages[g]) {
                    RunView r{0, 0, 0, true};
                    if (b.groups <= kLdsRuns) {
                        r.tok0 = run_tok0[g];
                        r.ntok = run_ntok[g];
                    } else {
                        r = run_view(b, g);
                    }
                    // sequences that are not among their run's tokens: q_off is out of order
                    const bool in = u.tok0 >= r.tok0 && u.tok0 - r.tok0 <= r.ntok && u.ntok <= r.ntok - (u.tok0 - r.tok0);
                    bad |= !in;
                    u.run_part0 = gain[g];
                    u.run_chunks = in ? (uint32_t)((((uint64_t)pages[g] << b.shift) + chunk - 1) / chunk) : 0;
                    u.run_row0 = (u.tok0 - r.tok0) * a.ratio;
                    u.run_rows = r.ntok * a.ratio;
                }
            }
            if (i < units) {
                pv.unit[i] = u;
                pv.item0[i] = u.item0;
            }
        }
        if (attempt || (rows <= a.part_rows && items < (1ull << 32))) {
            if (tid == 0) {
                PlanHead h{};
                h.n = b.n;
                h.groups = b.groups;
                h.q_tokens = b.q_tokens;
                h.q_heads = a.q_heads;
                h.kv_heads = a.kv_heads;
                h.shift = b.shift;
                h.entries = b.entries;
                h.items = (uint32_t)items;
                h.head_dim = a.head_dim;
                h.wide = a.wide;
                h.part_rows = (uint32_t)rows;
                h.most_parts = most;
                *pv.head = h;
            }
            break;
        }
        __syncthreads();
    }
    if (bad)
        atomicOr(status, kErrInval);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_kernel(AttnIn a, const PlanView pv,
                                                                          uint64_t part_rows,
                                                                          uint32_t* status)
{
    // two tiles of 64 keys and values, or four waves' 32 keys and values
    __shared__ __attribute__((aligned(16))) uint16_t lds[4 * kWideKeys * D];
    __shared__ uint32_t odd_tile;
    __shared__ Joined<kWaves> joined;
    Unit u;
    if (!item_unit(a, pv, a.b.groups + a.b.n, part_rows, D, kWide, status, u))
        return;
    bool bad = false;
    const uint32_t x = blockIdx.x - u.item0;
    if (u.flags & kUnitWide)
        wide_tile<T, D>(a, make_tile(a, u, x, kWide), lds, &odd_tile, bad);
    else
        narrow_tile<T, D, kWaves>(a, make_tile(a, u, x, kNarrow), lds, joined, bad);
    if (bad)
        atomicOr(status, kErrInval);
}

// A few rows on a few keys: narrow tiles, uncut, of as many waves as have room in LDS,
// where a second kernel that joins parts costs more than cutting gains.  A token of
// 32 query and 8 key heads of 128 on 128, 256, 512, 768 and 1,024 keys: 6.4, 7.2, 9.1,
// 11.1 and 13.5 us, in parts 8.0, 10.5, 10.5, 10.9 and 10.7 (with the plan 15.5 and 15.9
// on 768); heads of 64 on 768 and 1,024 keys 8.7 and 10.0, in parts 10.1 and 9.8; heads
// of 256 on 256 and 384 keys 12.5 and 16.0, in parts 13.8 and 13.9.  1 to 64 KV heads
// are within 0.4 us of these in this form.  Of several sequences the keys count together:
// four tokens on 768 keys 7.2, in parts 10.6.
template <typename T, int D>
__global__ __launch_bounds__(kSmallWaves<D>* kWave, 1) void attn_small_kernel(AttnIn a, const PlanView pv,
                                                                              uint32_t* status)
{
    constexpr int kW = kSmallWaves<D>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[kW * 2 * kNarrowKeys * D];
    __shared__ Joined<kW> joined;
    Unit u;
    if (!item_unit(a, pv, a.b.n, 0, D, kWide, status, u))
        return;
    bool bad = false;
    narrow_tile<T, D, kW>(a, make_tile(a, u, blockIdx.x - u.item0, kNarrow), lds, joined, bad);
    if (bad)
        atomicOr(status, kErrInval);
}

// MANY: more rows than waves (a kernel of its own: its registers would halve the
// waves of the other).  Waves a SIMD: all eight of the other up to heads of 128 (seven:
// 1.2 us more for 8,192 rows), seven of this one for heads of 64 (six: 2 us more for
// 95,488 rows).
template <typename T, int D, bool MANY>
__global__ __launch_bounds__(kThreads, D == 64 && MANY ? 7 : MANY || D == 256 ? 1 : 8) void attn_join_kernel(AttnIn a,
                                                                                       const PlanView pv,
                                                                                       uint64_t part_rows,
                                                                                       uint32_t items)
{
    constexpr int kPer = D / kWave;  // elements a lane
    __shared__ float acc[kWaves][D];
    const PlanHead& ph = *pv.head;
    if (ph.part_rows == 0 || !plan_fits(ph, a, part_rows, D, kWide, items))
        return;  // the pass has left nothing (and reported it)
    const uint32_t wave = threadIdx.x / kWave, lane = lane_id();
    const bool together = ph.most_parts > 16;
    const uint64_t all = (uint64_t)a.b.q_tokens * a.q_heads;
    const uint64_t step = together ? gridDim.x : (uint64_t)gridDim.x * kWaves;
    if (MANY && !together) {
        const uint64_t per = ((all + step - 1) / step + 3) / 4 * 4;
        const uint64_t y0 = ((uint64_t)blockIdx.x * kWaves + wave) * per;
        join_quarters<T, D>(a, pv, y0, y0 + per < all ? y0 + per : all);
        return;
    }
    for (uint64_t y0 = together ? blockIdx.x : (uint64_t)blockIdx.x * kWaves; y0 < all; y0 += step) {
        const uint64_t y = together ? y0 : y0 + wave;
        const bool mine = y < all;
        const uint32_t t = mine ? (uint32_t)(y / a.q_heads) : 0, x = mine ? (uint32_t)(y % a.q_heads) : 0;
        const uint32_t s = sequence_of(a.b, t);
        const Parts p = parts_of(pv.unit[a.b.groups + s], t, x, a.ratio);
        const uint32_t n = mine ? p.n : 0;
        const bool live = n != 0;
        auto place = [&](uint32_t i) { return p.at(i); };
        // the parts' weights, a lane each; then their rows, whose loads need not
        // wait for one another
        const uint32_t from = together ? wave * kWave : 0, by = together ? kWaves * kWave : kWave;
        float four[4][kPer];
        auto read_four = [&](uint32_t i) {
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const float* at = a.part + place(i + j < n ? i + j : n - 1) * D + lane * kPer;
#pragma unroll
                for (int c = 0; c < kPer; c++)
                    four[j][c] = at[c];
            }
        };
        const v2f none = {-INFINITY, 0};
        float m = -INFINITY;
        v2f e0 = none;
        if (n) {
            if (from + lane < n)
                e0 = a.part_stat[place(from + lane)];
            read_four(from);  // beside the weights' reads
        }
        if (together)
            for (uint32_t i = lane; i < n; i += kWave)
                m = fmaxf(m, a.part_stat[place(i)][0]);
        else
            m = e0[0];
#pragma unroll
        for (int o = 1; o < kWave; o *= 2)
            m = fmaxf(m, __shfl_xor(m, o));
        float v[kPer] = {}, total = 0;
        for (uint32_t i0 = from; i0 < n; i0 += by) {
            const uint32_t i = i0 + lane;
            const v2f e = i0 == from ? e0 : i < n ? a.part_stat[place(i)] : none;
            const float w = part_weight(e, m, a.scale2);
            total += w;
            const uint32_t k1 = n - i0 < kWave ? n - i0 : kWave;
            for (uint32_t k = 0; k < k1; k += 4) {
                float x[4];
                if (i0 != from || k)
                    read_four(i0 + k);
#pragma unroll
                for (int j = 0; j < 4; j++)
                    x[j] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), k + j));
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int c = 0; c < kPer; c++)
                        v[c] = x[j] == 0 ? v[c] : __builtin_fmaf(x[j], four[j][c], v[c]);
            }
        }
#pragma unroll
        for (int o = 1; o < kWave; o *= 2)
            total += __shfl_xor(total, o);
        if (together) {
            __shared__ float tot[kWaves];
            __syncthreads();
            if (lane == 0)
                tot[wave] = total;
#pragma unroll
            for (int k = 0; k < kPer; k++)
                acc[wave][lane * kPer + k] = v[k];
            __syncthreads();
            total = 0;
            for (int w = 0; w < kWaves; w++)
                total += tot[w];
#pragma unroll
            for (int k = 0; k < kPer; k++) {
                v[k] = 0;
                for (int w = 0; w < kWaves; w++)
                    v[k] += acc[w][lane * kPer + k];
            }
            if (wave)
                continue;
        }
        if (!live)
            continue;
        const bool seen = total > 0 || total != total;
        const float inv = seen ? 1.0f / total : 0.0f;
        typedef T vt __attribute__((ext_vector_type(kPer)));
        vt z;
        if constexpr (kPer == 1) {
            z[0] = (T)(v[0] * inv);
        } else {
#pragma unroll
            for (int k = 0; k < kPer; k++)
                z[k] = (T)(v[k] * inv);
        }
        *reinterpret_cast<vt*>(a.out + t * a.out_stride + (uint64_t)x * D + lane * kPer) = z;
        if (lane == 0 && a.lse)
            a.lse[(uint64_t)t * a.q_heads + x] =
                seen ? lse_of<T>(m, total, a.scale2) : -INFINITY;
    }
}

}  // namespace

uint64_t attn_plan_bytes(uint64_t n, uint64_t groups)
{
    return sizeof(PlanHead) + item0_bytes(n + groups) + sizeof(Unit) * (n + groups) + 2 * up16(4 * n) +
           2 * up16(4 * groups);
}

hipError_t attn_plan(dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t q_heads,
                     uint32_t wide, void* plan)
{
    PlanIn a;
    a.b = token_batch(c, b);
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.ratio = q_heads / kv.kv_heads;
    a.head_dim = kv.head_dim;
    a.wide = wide;
    a.target = item_target(c);
    a.part_rows = small(c, b, kv, a.ratio) ? 0 : part_rows_of(c, b, q_heads);
    const PlanView pv = plan_view(plan, b.tables.n, b.groups);
    a.arrived = c->d_status + 48;  // a line of its own
    const uint32_t grid = !b.groups                        ? 1
                          : b.tables.n <= kPlanWorkgroups ? (uint32_t)b.tables.n
                                                          : grid_for(b.tables.n, kPlanThreads / kWave, c->n_cu);
    attn_plan_kernel<<<grid, kPlanThreads, 0, c->stream>>>(a, pv, c->d_status);
    return hipGetLastError();
}

hipError_t attn(dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t q_heads,
                const void* plan, uint32_t layer, const void* q, int64_t q_stride, float scale,
                void* out, int64_t out_stride, float* lse)
{
    const bool is_small = small(c, b, kv, q_heads / kv.kv_heads);
    const uint64_t rows = is_small ? 0 : part_rows_of(c, b, q_heads);
    hipError_t e;
    float* part =
        is_small ? nullptr : static_cast<float*>(scratch_get(c, kSlotPages, rows * (kv.head_dim + 2) * 4, &e));
    if (!part && !is_small)
        return e;
    AttnIn a;
    a.b = token_batch(c, b);
    a.k = static_cast<const uint16_t*>(kv.k) + (uint64_t)layer * kv.layer_stride;
    a.v = static_cast<const uint16_t*>(kv.v) + (uint64_t)layer * kv.layer_stride;
    a.q = static_cast<const uint16_t*>(q);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.part = part;
    a.part_stat = is_small ? nullptr : reinterpret_cast<v2f*>(part + rows * kv.head_dim);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.n_pages = kv.n_pages;
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.ratio = q_heads / kv.kv_heads;
    a.scale2 = scale * kLog2e;
    const PlanView pv = plan_view(const_cast<void*>(plan), b.tables.n, b.groups);
    const uint64_t most = is_small ? (uint64_t)b.tables.n * kv.kv_heads : most_items(c, b, a.ratio, kv.kv_heads, kWide);
    if (most > 0x7FFFFFFFull)
        return hipErrorInvalidValue;
    by_type(kv.dtype, kv.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        if (is_small) {
            attn_small_kernel<T, D><<<(uint32_t)most, kSmallWaves<D> * kWave, 0, c->stream>>>(a, pv, c->d_status);
            return;
        }
        attn_kernel<T, D><<<(uint32_t)most, kThreads, 0, c->stream>>>(a, pv, rows, c->d_status);
        const uint64_t outs = b.q_tokens * q_heads;
        if (outs > 8ull * c->n_cu * kWaves)
            attn_join_kernel<T, D, true><<<4u * c->n_cu, kThreads, 0, c->stream>>>(a, pv, rows, (uint32_t)most);
        else
            attn_join_kernel<T, D, false>
                <<<grid_for(outs, 1, 8u * c->n_cu), kThreads, 0, c->stream>>>(a, pv, rows, (uint32_t)most);
    });
    return hipGetLastError();
}

}  // namespace dm
