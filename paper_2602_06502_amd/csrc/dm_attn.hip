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
#include "dm_internal.h"
#include "dm_pages.h"

namespace dm {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr uint32_t kNarrow = 16, kWide = 128;  // rows of a tile
// Rows of a unit, at most, that has narrow tiles.  (32 sequences of 4,096 keys, 32
// query and 8 key heads of 128: 24 rows 104 us in a wide tile, 114 in two narrow
// ones; 64 rows 112 and 158; 16 rows 103 and 106, 4 rows 100 and 102.  64 sequences of
// 64 to 8,192 keys, 4 rows: 216 narrow, 262 wide.)
constexpr uint32_t kNarrowRows = 16;
constexpr uint32_t kNarrowKeys = 32, kWideKeys = 64;
constexpr uint32_t kChunk = 128;               // keys of a chunk, at least (of the longest: a multiple)
constexpr int kPlanThreads = 512;
constexpr uint64_t kPartRows = 1ull << 20;     // rows of parts kept beyond those of cut items

// The plan in memory: a head, the numbers of items before the units, room for
// kEarlyUnits of them at least (so that a kernel may read as many beside the head,
// before it knows whose plan it is), then a unit for each run and each sequence
// (runs first), then words of the sequences.
constexpr uint32_t kEarlyUnits = 8 * kWave;
struct PlanHead {
    uint32_t n, groups, q_tokens, q_heads, kv_heads, shift;  // what it was made for
    int64_t entries;
    uint32_t items;
    uint32_t part_rows;   // rows of parts
    uint32_t most_parts;  // of a row
    uint32_t head_dim;
    uint32_t pad[4];
};
struct Unit {
    uint32_t item0;       // items before this unit
    uint32_t tok0, ntok;  // its new tokens
    uint32_t key0, key1;  // its keys
    uint32_t part0;       // its first row of parts (chunks > 1 or shared)
    uint32_t chunks;
    uint32_t table;       // pages of its table, from entry `off` on
    int64_t off;
    int32_t pos0;         // a sequence: position of its first new token
    uint32_t flags;
    // of a sequence: its run's parts (chunks; 0: none), its first row among the
    // run's, and the run's rows
    uint32_t run_part0, run_chunks, run_row0, run_rows;
};
enum : uint32_t { kUnitWide = 1, kUnitCausal = 2, kUnitParts = 4 };

struct PlanView {
    PlanHead* head;
    Unit* unit;
    uint32_t* item0;   // [n + groups] the units' again, next to each other
    uint32_t* limit;   // [n] pages that s has in common with its run's first, at most
    uint32_t* run;     // [n] its run
    // of the runs, where they are too many for LDS: pages shared, cost of its
    // sequences on their own (then its first row of parts)
    uint32_t* shared;
    uint32_t* gain;
};

__host__ __device__ inline uint64_t up16(uint64_t x) { return (x + 15) & ~15ull; }

__host__ __device__ inline uint64_t item0_bytes(uint64_t units)
{
    return up16(4 * (units < kEarlyUnits ? kEarlyUnits : units));
}

__host__ __device__ inline PlanView plan_view(void* p, uint64_t n, uint64_t groups)
{
    PlanView v;
    uint8_t* b = static_cast<uint8_t*>(p);
    v.head = reinterpret_cast<PlanHead*>(b);
    b += sizeof(PlanHead);
    v.item0 = reinterpret_cast<uint32_t*>(b);
    b += item0_bytes(n + groups);
    v.unit = reinterpret_cast<Unit*>(b);
    b += sizeof(Unit) * (n + groups);
    v.limit = reinterpret_cast<uint32_t*>(b);
    b += up16(4 * n);
    v.run = reinterpret_cast<uint32_t*>(b);
    b += up16(4 * n);
    v.shared = reinterpret_cast<uint32_t*>(b);
    b += up16(4 * groups);
    v.gain = reinterpret_cast<uint32_t*>(b);
    return v;
}

// The tiles of a unit, by its rows, and their cost a key: a wide one takes up to
// twice a narrow one's time.
__device__ __forceinline__ uint32_t tile_rows(uint64_t rows) { return rows <= kNarrowRows ? kNarrow : kWide; }
__device__ __forceinline__ uint32_t tile_flags(uint64_t rows) { return tile_rows(rows) == kWide ? kUnitWide : 0; }
__device__ __forceinline__ uint64_t tiles_of(uint64_t rows)
{
    return (rows + tile_rows(rows) - 1) / tile_rows(rows);
}
__device__ __forceinline__ uint64_t weight_of(uint64_t rows)
{
    return tiles_of(rows) * (tile_rows(rows) == kWide ? 2 : 1);
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
    uint32_t q_heads, kv_heads, ratio, head_dim;
    uint64_t target;     // items wanted
    uint64_t part_rows;  // rows of parts there is room for (0: no unit is cut)
    uint32_t* arrived;   // workgroups that are done with their sequences; zero between calls
};

constexpr uint32_t kNoSay = 0xFFFFFFFFu;
constexpr uint32_t kLdsRuns = 1024;

// The run that sequence s is in, [g0, g1), and whether there is one.
struct RunOf {
    uint32_t g;
    int64_t g0, g1;
    bool ok;
};
__device__ __forceinline__ RunOf run_of(const TokenBatch& b, uint32_t s)
{
    RunOf r;
    if (b.groups < kWave) {  // all bounds by one read
        const int64_t at = b.group_off[lane_id() < b.groups ? lane_id() : b.groups];
        const uint32_t k = __popcll(ballot(lane_id() < b.groups && at <= (int64_t)s));
        r.g = k ? k - 1 : 0;
        r.g0 = (int64_t)shfl_u64((uint64_t)at, r.g);
        r.g1 = (int64_t)shfl_u64((uint64_t)at, r.g + 1);
    } else {
        r.g = wave_find(b.group_off, b.groups, 1, (int64_t)s);
        r.g0 = b.group_off[r.g];
        r.g1 = b.group_off[r.g + 1];
    }
    r.ok = r.g0 >= 0 && r.g1 <= (int64_t)b.n && r.g0 <= (int64_t)s && (int64_t)s < r.g1;
    return r;
}

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
    u.flags = kUnitParts | tile_flags((uint64_t)u.ntok * a.ratio);
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
    u.flags = kUnitCausal | (pages ? kUnitParts : 0) | tile_flags((uint64_t)u.ntok * a.ratio);
    return u;
}

// Is a pass of its own over `pages` common pages worth it for a run?  Where the
// run's rows together make clearly fewer tiles, over more than a chunk of keys.
__device__ __forceinline__ bool worth_sharing(const PlanIn& a, const RunView& r, uint32_t pages, uint32_t gain)
{
    return pages != 0 && pages != kNoSay && r.ok && ((uint64_t)pages << a.b.shift) >= kChunk &&
           2 * (uint64_t)gain >= 3 * weight_of((uint64_t)r.ntok * a.ratio);
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
                atomicAdd(&gain[g], (uint32_t)weight_of((uint64_t)v.ntok * a.ratio));
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
            return u.ntok ? weight_of((uint64_t)u.ntok * a.ratio) * (u.key1 - u.key0) : 0;
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
                it = tiles_of(r) * u.chunks * a.kv_heads;
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

// ---------------------------------------------------------------------------
// The pass over the keys.
// ---------------------------------------------------------------------------

typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

__device__ __forceinline__ v16f mfma(v8bf a, v8bf b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v16f mfma(v8hf a, v8hf b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ v4f mfma(v8bf a, v8bf b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v4f mfma(v8hf a, v8hf b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Tiles of keys in LDS: rows of D elements in 16-byte chunks, a row's chunks in
// an order of its own, so that the 16 rows that neighbouring lanes read a
// chunk of (K), the four rows that they read 64 bytes of (V of wide tiles) or the
// eight that they read 32 bytes of (V of narrow ones) lie in different banks.
template <int D>
__device__ __forceinline__ uint32_t k_swizzle(uint32_t row)
{
    return D == 64 ? (row >> 1) & 7 : row & 15;
}
template <int D, bool WIDE = true>
__device__ __forceinline__ uint32_t v_swizzle(uint32_t row)
{
    if (!WIDE)
        return D == 64 ? ((row >> 1) & 3) << 1 : (row & 7) << 1;
    return D == 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2;
}

struct AttnIn {
    TokenBatch b;
    const uint16_t *k, *v;  // the layer's pages
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    float* part;       // [part rows][D] parts of rows
    v2f* part_stat;    // [part rows] their maxima (of raw scores) and sums
    int64_t q_stride, out_stride;
    uint32_t n_pages, q_heads, kv_heads, ratio;
    float scale2;      // scale * log2(e)
};

// Weights are raised by a power of two: a float16 one loses bits below 2^-14 and is
// nothing below 2^-25, while the sum, in 32 bits, counts it.  They reach 2^8 (see
// weights()) and float16 ends at 2^16, so 2^7 fits: a weight below 2^-21 of the
// row's largest is off by up to 2^-32 of that.  The division takes the factor out
// again, the log-sum-exp subtracts it.
template <typename T>
constexpr float kRaise = std::is_same<T, _Float16>::value ? 7.0f : 0.0f;

// What a lane keeps of its row.
template <int D>
struct Row {
    v16f o[D / 32];  // O^T: element (d = db * 32 + (i / 4) * 8 + half * 4 + i % 4, row)
    float m, l;      // maximum (of raw scores), this half's sum
    bool far;        // scores_are_far(), of some row of the wave
};

// Scores are scaled and the base taken off in one rounding, which leaves every weight
// of a row the same factor: 2 to half a unit in the base's last place.  From 2^20 on,
// before that factor could overflow or lose the weights, the maximum is taken off first.
__device__ __forceinline__ bool scores_are_far(float m, float scale2)
{
    return __any(m != -INFINITY && !(fabsf(m * scale2) < 0x1p20f));
}

// A tile of 32 keys for a wave's 32 rows: s holds S^T (key = (i / 4) * 8 + half
// * 4 + i % 4).
template <typename T, int D>
__device__ __forceinline__ v16f scores(const uint16_t* kt, const typename Vec8<T>::type (&q)[D / 16])
{
    using V = typename Vec8<T>::type;
    const uint32_t row = lane_id() % 32, half = lane_id() / 32;
    v16f s = {};
#pragma unroll
    for (int x = 0; x < D / 16; x++) {
        const uint32_t chunk = (x * 2 + half) ^ k_swizzle<D>(row);
        s = mfma(*reinterpret_cast<const V*>(kt + row * D + chunk * 8), q[x], s);
    }
    return s;
}

// V^T of 16 keys (rows key0 ..) and 32 d (from db * 32 on), keys in the order
// of the lane's weights.
template <typename T, int D>
__device__ __forceinline__ typename Vec8<T>::type values(const uint16_t* vt, uint32_t key0, uint32_t db)
{
    const uint32_t l = lane_id(), half = l / 32, sub = (l / 16) % 2;
    const uint32_t row = key0 + half * 4 + (l % 16) / 4;
    const uint32_t c = db * 4 + sub * 2 + (l % 4) / 2;  // 16-byte chunk
    const uint32_t at0 = row * D + (c ^ v_swizzle<D>(row)) * 8 + (l % 2) * 4;
    const uint32_t at1 = (row + 8) * D + (c ^ v_swizzle<D>(row + 8)) * 8 + (l % 2) * 4;
    const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(vt + at0));
    const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(vt + at1));
    typedef short v8s __attribute__((ext_vector_type(8)));
    const v8s z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(typename Vec8<T>::type, z);
}

// Is any of eight 16-bit values infinite or NaN?
template <typename T>
__device__ __forceinline__ bool not_finite(v4u32 x)
{
    const uint32_t e = std::is_same<T, __bf16>::value ? 0x7F80u : 0x7C00u;
    bool f = false;
#pragma unroll
    for (int i = 0; i < 4; i++)
        f |= (x[i] & e) == e || (x[i] & (e << 16)) == (e << 16);
    return f;
}

// The larger of a lane's value and that of the same row in the other half: the
// upper half of one register exchanged with the lower half of another (the
// compiler takes the two results of the instruction's builtin for one).  The
// waits cover what the instruction needs of the vector instructions around it.
__device__ __forceinline__ float halves_max(float x)
{
    float y = x;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(x), "+v"(y));
    return fmaxf(x, y);
}

// The running softmax of NB tiles of 32 keys: the tiles' weights in T.  limit:
// the keys that the lane's row sees (absolute), key0: the tiles' first; masked:
// some row does not see all of them; beside(): what can be done meanwhile, when
// s has been read (it may be written anew).
template <typename T, int D, int NB, typename Beside>
__device__ __forceinline__ void weights(Row<D>& r, v16f (&s)[NB], typename Vec8<T>::type (&p)[NB][2],
                                        uint32_t key0, uint32_t limit, bool masked, float scale2,
                                        Beside&& beside)
{
    const uint32_t half = lane_id() / 32;
    if (masked) {
        // behind the branch: hoisted before it, as the compiler likes to, the selects
        // of every tile were a third of the vector work
        uint32_t first = key0 + half * 4;
        asm volatile("" : "+v"(first));
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (first + b * 32 + (i / 4) * 8 + i % 4 >= limit)
                    s[b][i] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int i = 0; i < 16; i++)
            mx = fmaxf(mx, s[b][i]);
    mx = halves_max(mx);
    // The maximum moves only when some row's has grown by more than 2^8 in weight:
    // weights up to 2^8 lose nothing in 32-bit sums nor, rounded, in T.
    const float grow = (mx - r.m) * scale2;
    if (__any(!(grow <= 8.0f))) {
        const float m = fmaxf(r.m, mx);
        const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((r.m - m) * scale2);
        r.m = m;
        r.far = scores_are_far(m, scale2);
        r.l *= keep;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                r.o[d][i] *= keep;
    }
    if (r.far) {
        float m = r.m == -INFINITY ? 0.0f : r.m;
        asm volatile("" : "+v"(m));  // as above
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                s[b][i] -= m;
    }
    const float base = r.m == -INFINITY ? 0.0f : r.m * (r.far ? 0.0f : scale2) - kRaise<T>;
    const v16f now[NB] = {s[0], s[NB - 1]};
    beside();
    float sum = 0;
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(now[b][i], scale2, -base));
            sum += w;
            p[b][i / 8][i % 8] = (T)w;
        }
    r.l += sum;
}

// O^T += V^T P^T.
template <typename T, int D, int NB>
__device__ __forceinline__ void add_values(Row<D>& r, const typename Vec8<T>::type (&p)[NB][2],
                                           const uint16_t* vt)
{
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
            for (int d = 0; d < D / 32; d++)
                r.o[d] = mfma(values<T, D>(vt, b * 32 + t * 16, d), p[b][t], r.o[d]);
}

// The same for values among which are infinities or NaN that some row does not
// see: a weight of zero times such a value would be NaN.  Key by key, each row
// takes what it sees.
template <typename T, int D, int NB>
__device__ __forceinline__ void add_odd_values(Row<D>& r, const typename Vec8<T>::type (&p)[NB][2],
                                               const uint16_t* vt, uint32_t key0, uint32_t limit)
{
    const uint32_t half = lane_id() / 32;
#pragma unroll 1
    for (uint32_t key = 0; key < NB * 32; key++) {
        float w = 0;
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (key == b * 32 + (i / 4) * 8 + half * 4 + i % 4)
                    w = (float)p[b][i / 8][i % 8];
        const float other = __shfl_xor(w, 32);
        w = (key / 4) % 2 == half ? w : other;
        const bool sees = key0 + key < limit;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const uint32_t e = d * 32 + i * 2 + half * 4;
                typedef T v4t __attribute__((ext_vector_type(4)));
                const v4t x = *reinterpret_cast<const v4t*>(
                    vt + key * D + ((e / 8) ^ v_swizzle<D>(key)) * 8 + e % 8);
                for (int k = 0; k < 4; k++)
                    if (sees)
                        r.o[d][i + k] = __builtin_fmaf(w, (float)x[k], r.o[d][i + k]);
            }
    }
}

// log sum exp(scale score), from the maximum and the raised weights' sum.
template <typename T>
__device__ __forceinline__ float lse_of(float m, float l, float scale2)
{
    return (m * scale2 + (__builtin_log2f(l) - kRaise<T>)) * 0.69314718055994531f;
}

// The result of a row (o: O^T as in Row): divided by the sum, written to the
// output or to its row of parts (rows: of the unit; rows from `end` on are not
// the tile's).
template <typename T, int D>
__device__ __forceinline__ void write_row(const AttnIn& a, const Unit& u, uint32_t h, uint32_t row,
                                          uint32_t end, uint32_t chunk, const Row<D>& r, float l,
                                          uint32_t rows)
{
    const uint32_t half = lane_id() / 32;
    if (row >= end)
        return;
    const float inv = l > 0 || l != l ? 1.0f / l : 0.0f;
    const bool seen = l > 0 || l != l;
    if (u.flags & kUnitParts) {
        const uint64_t at = u.part0 + ((uint64_t)h * rows + row) * u.chunks + chunk;
        float* o = a.part + at * D;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                v4f x;
                for (int k = 0; k < 4; k++)
                    x[k] = seen ? r.o[d][i + k] * inv : 0.0f;
                *reinterpret_cast<v4f*>(o + d * 32 + i * 2 + half * 4) = x;
            }
        if (half == 0)
            a.part_stat[at] = v2f{r.m, l};
        return;
    }
    const uint32_t t = u.tok0 + row / a.ratio, x = h * a.ratio + row % a.ratio;
    uint16_t* o = a.out + t * a.out_stride + (uint64_t)x * D;
#pragma unroll
    for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            typedef T v4t __attribute__((ext_vector_type(4)));
            v4t y;
            for (int k = 0; k < 4; k++)
                y[k] = (T)(seen ? r.o[d][i + k] * inv : 0.0f);
            *reinterpret_cast<v4t*>(o + d * 32 + i * 2 + half * 4) = y;
        }
    if (half == 0 && a.lse)
        a.lse[(uint64_t)t * a.q_heads + x] = seen ? lse_of<T>(r.m, l, a.scale2) : -INFINITY;
}

// The last of up to kEarlyUnits units with item0 <= item, by one wait.
__device__ __forceinline__ uint32_t find_unit(const uint32_t* item0, uint32_t units, uint32_t item)
{
    uint32_t x[kEarlyUnits / kWave], k = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEarlyUnits / kWave; i++) {
        const uint32_t u = i * kWave + lane_id();
        x[i] = u < units ? item0[u] : 0xFFFFFFFFu;
    }
#pragma unroll
    for (uint32_t i = 0; i < kEarlyUnits / kWave; i++)
        k += __popcll(ballot(x[i] <= item));
    return k ? k - 1 : 0;
}

// Is the plan this call's, of at most `items` items?  (A batch whose q_off is out of
// order can have more than the call has workgroups.)
__device__ __forceinline__ bool plan_fits(const PlanHead& h, const AttnIn& a, uint64_t part_rows,
                                          uint32_t head_dim, uint32_t items)
{
    return h.n == a.b.n && h.groups == a.b.groups && h.q_tokens == a.b.q_tokens &&
           h.q_heads == a.q_heads && h.kv_heads == a.kv_heads && h.shift == a.b.shift &&
           h.entries == a.b.entries && h.head_dim == head_dim && h.part_rows <= part_rows &&
           h.items <= items;
}

// The unit of this workgroup's item; false: none, or the plan is another batch's
// (reported).  What the plan holds is read beside its head as far as any plan
// reaches, and beyond that only once the head has been looked at: the plan of a
// batch of fewer sequences is a smaller one.
__device__ __forceinline__ bool item_unit(const AttnIn& a, const PlanView& pv, uint32_t units,
                                          uint64_t part_rows, uint32_t head_dim, uint32_t* status, Unit& u)
{
    const PlanHead& ph = *pv.head;
    const bool early = units <= kEarlyUnits;
    uint32_t ui = early ? find_unit(pv.item0, units, blockIdx.x) : 0;
    if (!plan_fits(ph, a, part_rows, head_dim, gridDim.x)) {
        if (blockIdx.x == 0 && threadIdx.x == 0)
            atomicOr(status, kErrInval);
        return false;
    }
    if (blockIdx.x >= ph.items)
        return false;
    if (!early)
        ui = wave_find(pv.item0, units, 1, blockIdx.x);
    u = pv.unit[ui];
    return true;
}

// An item: a tile of a unit's rows, a chunk of its keys, a KV head.
struct Tile {
    Unit u;
    uint32_t h, chunk, rows;    // rows of the unit
    uint32_t first, last;       // the tile's rows
    uint32_t key0, key1;        // keys that the chunk has and some row of the tile sees
    uint32_t see_first;         // keys that the tile's first row sees, of the unit's
};

// Keys of the unit that a row sees.
__device__ __forceinline__ uint32_t sees(const Unit& u, uint32_t ratio, uint32_t row)
{
    if (!(u.flags & kUnitCausal))
        return u.key1;
    const int64_t n = (int64_t)u.pos0 + row / ratio + 1;
    return n < 0 ? 0 : n > u.key1 ? u.key1 : (uint32_t)n;
}

__device__ __forceinline__ void tile_rows_are(Tile& t, uint32_t ratio, uint32_t chunk_keys, uint32_t first,
                                              uint32_t count)
{
    t.first = first;
    t.last = first + count < t.rows ? first + count - 1 : t.rows - 1;
    t.key1 = t.u.key1 - t.key0 > chunk_keys ? t.key0 + chunk_keys : t.u.key1;
    t.see_first = sees(t.u, ratio, t.first);
    const uint32_t see_last = sees(t.u, ratio, t.last);
    if (t.key1 > see_last)
        t.key1 = see_last;
}

__device__ __forceinline__ Tile make_tile(const AttnIn& a, const Unit& u, uint32_t x, uint32_t count)
{
    Tile t;
    t.u = u;
    t.rows = u.ntok * a.ratio;
    const uint32_t tiles = (t.rows + count - 1) / count;
    t.h = x % a.kv_heads;  // neighbouring workgroups, on different dies, take different heads
    x /= a.kv_heads;
    t.chunk = x / tiles;
    // chunks of one length, none empty: the last of a unit ends no sooner than the others
    const uint32_t chunk_keys =
        ((u.key1 - u.key0 + u.chunks - 1) / u.chunks + kWideKeys - 1) / kWideKeys * kWideKeys;
    t.key0 = u.key0 + t.chunk * chunk_keys;
    // a sequence's last tiles see the most keys: they go first
    tile_rows_are(t, a.ratio, chunk_keys, (tiles - 1 - x % tiles) * count, count);
    return t;
}

// A row's query, as the right operand of K Q^T (rows past the tile's last: the
// last one's again, not written).
template <typename T, int D>
__device__ __forceinline__ void load_query(const AttnIn& a, const Tile& t, uint32_t row,
                                           typename Vec8<T>::type (&q)[D / 16])
{
    const uint32_t r = row < t.last ? row : t.last;
    const uint16_t* at = a.q + (uint64_t)(t.u.tok0 + r / a.ratio) * a.q_stride +
                         (uint64_t)(t.h * a.ratio + r % a.ratio) * D + lane_id() / 32 * 8;
#pragma unroll
    for (int k = 0; k < D / 16; k++)
        q[k] = *reinterpret_cast<const typename Vec8<T>::type*>(at + k * 16);
}

template <int D>
__device__ __forceinline__ void clear(Row<D>& r)
{
    r.m = -INFINITY;
    r.l = 0;
    r.far = false;
#pragma unroll
    for (int d = 0; d < D / 32; d++)
        r.o[d] = v16f{};
}

// Pages are looked up by scalar loads: a send's or a load's rows
// lie four to a page (tiles begin at multiples of four tokens), and vector loads would
// wait for everything that was asked for before them.
typedef const __attribute__((address_space(4))) uint32_t ScalarTable;

// A lane's share of a wave's narrow tiles: 16-byte chunk `ch` of rows r0, r0 + kStep,
// ...  A tile's pages are looked up two tiles ahead and its rows read one ahead; none
// of the reads is conditional: rows past the last key read the last key's page, and
// their values become zeros on the way to LDS.
template <typename T, int D>
struct Share {
    static constexpr int kLoads = kNarrowKeys * D / 8 / kWave;
    static constexpr uint32_t kRowChunks = D / 8, kStep = kWave / kRowChunks;
    static constexpr int kGroups = kStep > 4 ? 2 : 1, kPages = kLoads * kGroups;
    v4u32 k[kLoads], v[kLoads];
    uint32_t page[kPages];
    ScalarTable* table;
    uint32_t key1, n_pages, shift, r0, ch;
    bool halves;  // eight rows of a load are in two pages of four
    uint32_t lane_at;
    uint64_t head_at, page_size;

    __device__ __forceinline__ Share(const AttnIn& a, const Tile& t)
        : table((ScalarTable*)(a.b.page + t.u.off)), key1(t.key1), n_pages(a.n_pages), shift(a.b.shift),
          r0(lane_id() / kRowChunks), ch(lane_id() % kRowChunks), halves(kGroups == 2 && a.b.shift == 2),
          lane_at(r0 % (halves ? 4 : 8) * D + ch * 8),
          head_at((uint64_t)t.h * D << a.b.shift), page_size((uint64_t)a.kv_heads * D << a.b.shift)
    {
    }
    // r0, each time anew: what follows from it is worked out again for each tile
    // instead of being kept in registers, of which there are none to spare
    __device__ __forceinline__ uint32_t here() const
    {
        uint32_t r = r0;
        asm volatile("" : "+v"(r));
        return r;
    }
    // pages of the tile at `key` (uniform, < key1), as they are in the table
    __device__ __forceinline__ void find(uint32_t key)
    {
#pragma unroll
        for (int i = 0; i < kPages; i++) {
            const uint32_t x = key + i / kGroups * kStep + i % kGroups * 4;
            if (i % kGroups == 0 || halves)
                page[i] = table[(x < key1 ? x : key1 - 1) >> shift];
        }
    }
    __device__ __forceinline__ void fetch(const AttnIn& a, uint32_t key, bool& bad)
    {
        const uint32_t mask = (1u << shift) - 1;
        auto from = [&](int i, int g) {
            const uint32_t p = page[i * kGroups + g];
            bad |= p >= n_pages;
            return (p < n_pages ? p : 0) * page_size + head_at + ((key + i * kStep + g * 4) & mask) * D;
        };
        auto load = [&](int i, uint64_t at) {
            k[i] = *reinterpret_cast<const v4u32*>(a.k + at + lane_at);
            v[i] = *reinterpret_cast<const v4u32*>(a.v + at + lane_at);
        };
        if (kGroups == 1 || !halves) {
#pragma unroll
            for (int i = 0; i < kLoads; i++)
                load(i, from(i, 0));
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                const uint64_t low = from(i, 0), high = from(i, kGroups - 1);
                load(i, lane_id() < kWave / 2 ? low : high);
            }
        }
    }
    // into LDS; true: values that are not finite among them (asked for where some
    // row does not see all of the tile)
    __device__ __forceinline__ bool stage(uint16_t* kt, uint16_t* vt, uint32_t key, bool ask)
    {
        bool odd = false;
        if (ask) {
            const uint32_t have = key1 - key;
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                if (r0 + i * kStep >= have)
                    v[i] = v4u32{};
                odd |= not_finite<T>(v[i]);
            }
        }
        const uint32_t row = here();
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const uint32_t r = row + i * kStep;
            *reinterpret_cast<v4u32*>(kt + r * D + (ch ^ k_swizzle<D>(r)) * 8) = k[i];
            *reinterpret_cast<v4u32*>(vt + r * D + (ch ^ v_swizzle<D, false>(r)) * 8) = v[i];
        }
        return odd;
    }
};

// What the waves of a narrow tile leave for one another.
template <int WAVES>
struct Joined {
    float m[WAVES][kNarrow], l[WAVES][kNarrow];
};

// The largest of the values of a row's four lanes (16 apart), in each of them.
__device__ __forceinline__ float quarters_max(float x)
{
    float y = x;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(x), "+v"(y));
    return halves_max(fmaxf(x, y));
}

// Four elements of a row's result, d on: to the output or to its row of parts.
template <typename T, int D>
__device__ __forceinline__ void write_four(const AttnIn& a, const Tile& t, uint32_t row, uint32_t d, v4f x)
{
    const Unit& u = t.u;
    if (u.flags & kUnitParts) {
        const uint64_t at = u.part0 + ((uint64_t)t.h * t.rows + row) * u.chunks + t.chunk;
        *reinterpret_cast<v4f*>(a.part + at * D + d) = x;
        return;
    }
    typedef T v4t __attribute__((ext_vector_type(4)));
    v4t y;
    for (int k = 0; k < 4; k++)
        y[k] = (T)x[k];
    *reinterpret_cast<v4t*>(a.out + (u.tok0 + row / a.ratio) * a.out_stride +
                            (uint64_t)(t.h * a.ratio + row % a.ratio) * D + d) = y;
}

// A lane holds its row's (lane % 16) scores of 4 of 16 keys, key = h * 16 + (lane /
// 16) * 4 + i, and of O^T the elements d = block * 16 + (lane / 16) * 4 + i.
template <typename T, int D, int WAVES>
__device__ __forceinline__ void narrow_tile(const AttnIn& a, const Tile& t, uint16_t* lds, Joined<WAVES>& joined,
                                            bool& bad)
{
    using V = typename Vec8<T>::type;
    constexpr uint32_t kTurn = WAVES * kNarrowKeys;
    constexpr int kBlocks = D / 16;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t lane = lane_id(), row16 = lane % 16, g = lane / 16;
    const uint32_t row = t.first + row16, in_tile = row < t.last ? row : t.last;
    V q[D / 32];
    {
        const uint16_t* at = a.q + (uint64_t)(t.u.tok0 + in_tile / a.ratio) * a.q_stride +
                             (uint64_t)(t.h * a.ratio + in_tile % a.ratio) * D + g * 8;
#pragma unroll
        for (int k = 0; k < D / 32; k++)
            q[k] = *reinterpret_cast<const V*>(at + k * 32);
    }
    const uint32_t limit = sees(t.u, a.ratio, in_tile), end = limit < t.key1 ? limit : t.key1;
    v4f o[kBlocks];
    float m = -INFINITY, l = 0;
    bool far = false;
#pragma unroll
    for (int d = 0; d < kBlocks; d++)
        o[d] = v4f{};
    uint16_t* kt = lds + wave * 2 * kNarrowKeys * D;
    uint16_t* vt = kt + kNarrowKeys * D;
    // weights, and what their rounding has left out: the matrix unit has time for both
    // (4% busy with the weights alone, in 64 rows on up to 8,192 keys)
    V p, rest;
    // scores and weights of the tile in LDS
    auto weigh = [&](uint32_t key, bool masked) {
        v4f s[2];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            s[h] = v4f{};
            const uint32_t r = h * 16 + row16;
#pragma unroll
            for (int k = 0; k < D / 32; k++)
                s[h] = mfma(*reinterpret_cast<const V*>(kt + r * D + ((k * 4 + g) ^ k_swizzle<D>(r)) * 8), q[k],
                            s[h]);
        }
        if (masked) {
            uint32_t first = key + g * 4;
            asm volatile("" : "+v"(first));  // as in weights()
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (first + (i / 4) * 16 + i % 4 >= end)
                    s[i / 4][i % 4] = -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int i = 1; i < 8; i++)
            mx = fmaxf(mx, s[i / 4][i % 4]);
        mx = quarters_max(mx);
        // as in weights()
        if (__any(!((mx - m) * a.scale2 <= 8.0f))) {
            const float now = fmaxf(m, mx);
            const float keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - now) * a.scale2);
            m = now;
            far = scores_are_far(m, a.scale2);
            l *= keep;
#pragma unroll
            for (int d = 0; d < kBlocks; d++)
                o[d] *= keep;
        }
        float base = m == -INFINITY ? 0.0f : m * a.scale2 - kRaise<T>;
        if (far) {
            const float top = m == -INFINITY ? 0.0f : m;
            s[0] -= top;
            s[1] -= top;
            base = -kRaise<T>;
        }
        // light weights are summed before they meet a sum that a heavy one may be in
        float sum = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], a.scale2, -base));
            sum += w;
            p[i] = (T)w;
            rest[i] = (T)(w - (float)p[i]);
        }
        l += sum;
    };
    uint32_t key = t.key0 + wave * kNarrowKeys;
    if (key < t.key1) {
        Share<T, D> x(a, t);
        bool masked = false, odd = false;
        // a wave's own part of LDS: its lanes' writes and reads in order
        auto stage = [&](uint32_t key) {
            masked = key + kNarrowKeys > t.see_first || key + kNarrowKeys > t.key1;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            odd |= x.stage(kt, vt, key, masked);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        x.find(key);
        x.fetch(a, key, bad);
        if (key + kTurn < t.key1)
            x.find(key + kTurn);
        for (; key < t.key1; key += kTurn) {
            stage(key);
            if (masked && __any(odd))
                break;
            if (key + kTurn < t.key1)
                x.fetch(a, key + kTurn, bad);
            if (key + 2 * kTurn < t.key1)
                x.find(key + 2 * kTurn);
            weigh(key, masked);
            // O^T += V^T P^T, keys in the order of the lane's weights
            const uint32_t r = g * 4 + row16 / 4;
#pragma unroll
            for (int d = 0; d < kBlocks; d++) {
                const uint32_t c = d * 2 + (lane % 4) / 2, e = (lane % 2) * 4;
                const v4s v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_v4s*)(vt + r * D + (c ^ v_swizzle<D, false>(r)) * 8 + e));
                const v4s v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_v4s*)(vt + (r + 16) * D + (c ^ v_swizzle<D, false>(r + 16)) * 8 + e));
                typedef short v8s __attribute__((ext_vector_type(8)));
                const v8s f = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
                o[d] = mfma(__builtin_bit_cast(V, f), p, o[d]);
                o[d] = mfma(__builtin_bit_cast(V, f), rest, o[d]);
            }
        }
        while (key < t.key1) {
            // as add_odd_values()
            weigh(key, true);
#pragma unroll 1
            for (uint32_t k = 0; k < kNarrowKeys; k++) {
                float w = 0;
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (k / 16 * 4 + k % 4 == (uint32_t)i)
                        w = (float)p[i] + (float)rest[i];
                w = __shfl(w, (k % 16) / 4 * 16 + row16);
                const bool seen = key + k < end;
#pragma unroll
                for (int d = 0; d < kBlocks; d++) {
                    const uint32_t e = d * 16 + g * 4;
                    typedef T v4t __attribute__((ext_vector_type(4)));
                    const v4t x = *reinterpret_cast<const v4t*>(
                        vt + k * D + ((e / 8) ^ v_swizzle<D, false>(k)) * 8 + e % 8);
                    for (int i = 0; i < 4; i++)
                        if (seen)
                            o[d][i] = __builtin_fmaf(w, (float)x[i], o[d][i]);
                }
            }
            key += kTurn;
            if (key < t.key1) {
                x.find(key);
                x.fetch(a, key, bad);
                stage(key);
            }
        }
    }
    // the waves' parts joined, each wave a share of the blocks
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
        joined.m[wave][row16] = m;
        joined.l[wave][row16] = l;
    }
    v4f* sum = reinterpret_cast<v4f*>(lds);  // [wave][block][lane]
    __syncthreads();
    float all = -INFINITY, total = 0;
    for (int w = 0; w < WAVES; w++)
        all = fmaxf(all, joined.m[w][row16]);
    for (int w = 0; w < WAVES; w++) {
        const float mw = joined.m[w][row16], lw = joined.l[w][row16];
        // a wave that saw nothing adds nothing, one that saw only NaN adds it
        total += mw == -INFINITY ? (lw != lw ? lw : 0.0f) : lw * __builtin_amdgcn_exp2f((mw - all) * a.scale2);
    }
    const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - all) * a.scale2);
#pragma unroll
    for (int d = 0; d < kBlocks; d++)
        sum[(wave * kBlocks + d) * kWave + lane] = o[d] * keep;
    __syncthreads();
    const bool seen = total > 0 || total != total;
    const float inv = seen ? 1.0f / total : 0.0f;
    for (uint32_t d = wave; d < kBlocks; d += WAVES) {
        v4f x = {};
        for (int w = 0; w < WAVES; w++)
            x += sum[(w * kBlocks + d) * kWave + lane];
        for (int k = 0; k < 4; k++)
            x[k] = seen ? x[k] * inv : 0.0f;
        if (row <= t.last)
            write_four<T, D>(a, t, row, d * 16 + g * 4, x);
    }
    if (wave == 0 && g == 0 && row <= t.last) {
        if (t.u.flags & kUnitParts)
            a.part_stat[t.u.part0 + ((uint64_t)t.h * t.rows + row) * t.u.chunks + t.chunk] = v2f{all, total};
        else if (a.lse)
            a.lse[(uint64_t)(t.u.tok0 + row / a.ratio) * a.q_heads + t.h * a.ratio + row % a.ratio] =
                seen ? lse_of<T>(all, total, a.scale2) : -INFINITY;
    }
}

// A wide tile's keys and values go from memory to LDS without registers: 16 bytes a
// lane, a wave's 1024 bytes next to each other in LDS, each lane reading the chunk
// that belongs there.  The compiler does not know of these writes: wait_sent()
// and a barrier come between them and their readers.
__device__ __forceinline__ void send16(const uint16_t* from, uint32_t lds_at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :
                 : "s"(lds_at), "v"(from)
                 : "m0", "memory");
}
// The same from a uniform address and a lane's bytes on from it.  (Five wait states
// between a vector instruction that may have written the address, such as the reload
// of a spilled scalar, and its use; the compiler does not see into this.)
__device__ __forceinline__ void send16(const uint16_t* from, uint32_t lane_at, uint32_t lds_at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(lds_at), "v"(lane_at), "s"(from)
                 : "m0", "memory");
}
__device__ __forceinline__ void wait_sent() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Byte address of a place in LDS.
__device__ __forceinline__ uint32_t lds_address(const uint16_t* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint16_t*)p;
}

// A thread's share of wide tiles: LDS chunk threadIdx.x + i * 256, that is row r0 +
// i * kStep, place `ch` of the row.  What a lane adds to its rows' address does not
// change from tile to tile.
template <typename T, int D>
struct Sender {
    static constexpr int kLoads = kWideKeys * D / 8 / kThreads;
    static constexpr uint32_t kRowChunks = D / 8, kStep = kThreads / kRowChunks;
    static constexpr uint32_t kWaveRows = kWave / kRowChunks;
    static constexpr int kGroups = kWaveRows > 4 ? 2 : 1, kPages = kLoads * kGroups;
    const uint16_t *k, *v;  // the layer's pages, at the KV head
    ScalarTable* table;
    uint32_t key1, n_pages, shift, page_size, r0, ch, wave;
    bool halves;  // the wave's eight rows are in two pages of four
    uint32_t lane_row;

    __device__ __forceinline__ Sender(const AttnIn& a, const Tile& t, uint32_t wave_)
        : k(a.k + ((uint64_t)t.h * D << a.b.shift)), v(a.v + ((uint64_t)t.h * D << a.b.shift)),
          table((ScalarTable*)(a.b.page + t.u.off)), key1(t.key1), n_pages(a.n_pages), shift(a.b.shift),
          page_size(a.kv_heads * D << a.b.shift), r0(threadIdx.x / kRowChunks), ch(threadIdx.x % kRowChunks),
          wave(wave_), halves(kGroups == 2 && a.b.shift == 2), lane_row(r0 % kWaveRows % (halves ? 4 : 8) * D)
    {
    }
    // pages of the wave's rows of the tile at `key` (uniform, < key1), as they are in the
    // table; rows past the last key: the last key's
    __device__ __forceinline__ void find(uint32_t key, uint32_t (&page)[kPages]) const
    {
#pragma unroll
        for (int i = 0; i < kPages; i++) {
            const uint32_t x = key + wave * kWaveRows + i / kGroups * kStep + i % kGroups * 4;
            if (i % kGroups == 0 || halves)
                page[i] = table[(x < key1 ? x : key1 - 1) >> shift];
        }
    }
    __device__ __forceinline__ void send(const uint16_t* base, bool values, uint32_t key,
                                         const uint32_t (&page)[kPages], const uint16_t* to, bool& bad) const
    {
        const uint32_t mask = (1u << shift) - 1, at = lds_address(to) + wave * kWave * 16;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            auto from = [&](int g) {
                const uint32_t p = page[i * kGroups + g];
                bad |= p >= n_pages;
                return base + (uint64_t)(p < n_pages ? p : 0) * page_size +
                       ((key + wave * kWaveRows + i * kStep + g * 4) & mask) * D;
            };
            const uint32_t r = r0 + i * kStep;
            const uint32_t c = ch ^ (values ? v_swizzle<D>(r) : k_swizzle<D>(r));
            const uint32_t lane_at = (lane_row + c * 8) * 2, lds_at = at + i * kThreads * 16;
            if (kGroups == 1 || !halves) {
                send16(from(0), lane_at, lds_at);
            } else {
                const uint16_t *low = from(0), *high = from(kGroups - 1);
                send16((lane_id() < kWave / 2 ? low : high) + lane_at / 2, lds_at);
            }
        }
    }
    // A tile of values of which some row does not see all: zeros for the places past
    // the last key; true: values that are not finite among the others.
    __device__ __forceinline__ bool clean(uint16_t* vt, uint32_t key) const
    {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            v4u32* at = reinterpret_cast<v4u32*>(vt + (r0 + i * kStep) * D + ch * 8);
            if (key + r0 + i * kStep >= key1)
                *at = v4u32{};
            else
                odd |= not_finite<T>(*at);
        }
        return odd;
    }
};

// Tile by tile, the next one's scores are taken beside this one's weights: the
// matrix unit has work that does not wait for them.  K of tile t + 2 and V of
// tile t + 1 are on their way meanwhile, to where K of tile t and V of tile t - 1
// were.
template <typename T, int D>
__device__ __forceinline__ void wide_tile(const AttnIn& a, const Tile& t, uint16_t* lds, uint32_t* odd_tile,
                                          bool& bad)
{
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t row = t.first + wave * 32 + lane_id() % 32;
    typename Vec8<T>::type q[D / 16], p[2][2];
    load_query<T, D>(a, t, row, q);
    const uint32_t limit = sees(t.u, a.ratio, row < t.last ? row : t.last);
    const uint32_t end = limit < t.key1 ? limit : t.key1;
    Row<D> r;
    clear<D>(r);
    // keys that the wave's first and last rows see
    const uint32_t w0 = t.first + wave * 32, w1 = w0 + 31 < t.last ? w0 + 31 : t.last;
    const uint32_t wave_first = w0 <= t.last ? sees(t.u, a.ratio, w0) : 0;
    const uint32_t wave_last = w0 <= t.last ? sees(t.u, a.ratio, w1) : 0;
    auto masked = [&](uint32_t key, uint32_t first) { return key + kWideKeys > first || key + kWideKeys > t.key1; };
    constexpr uint32_t kTile = kWideKeys * D;
    uint16_t* vts = lds + 2 * kTile;  // two tiles of keys, then two of values
    if (t.key0 < t.key1) {
        const Sender<T, D> x(a, t, wave);
        uint32_t p1[Sender<T, D>::kPages], p2[Sender<T, D>::kPages];  // pages of the next tile, and the one after
        if (threadIdx.x == 0)
            *odd_tile = 0;
        x.find(t.key0, p2);
        x.send(x.k, false, t.key0, p2, lds, bad);
        x.send(x.v, true, t.key0, p2, vts, bad);
        if (t.key0 + kWideKeys < t.key1) {
            x.find(t.key0 + kWideKeys, p1);
            x.send(x.k, false, t.key0 + kWideKeys, p1, lds + kTile, bad);
        }
        if (t.key0 + 2 * kWideKeys < t.key1)
            x.find(t.key0 + 2 * kWideKeys, p2);
        wait_sent();
        __syncthreads();
        v16f s[2] = {scores<T, D>(lds, q), scores<T, D>(lds + 32 * D, q)};
        __syncthreads();  // the third tile's keys go where the first's are
        uint32_t key = t.key0, buf = 0;
        bool odd = false;
        while (true) {
            // K of the next tile and V of this one are there; everyone is done with
            // K of this tile and V of the one before
            if (masked(key, t.see_first)) {
                if (x.clean(vts + buf * kTile, key))
                    *odd_tile = 1;
                __syncthreads();
                odd = *odd_tile;
                if (odd)
                    break;
            }
            const uint32_t key1 = key + kWideKeys, key2 = key1 + kWideKeys;
            if (key2 < t.key1)
                x.send(x.k, false, key2, p2, lds + buf * kTile, bad);
            if (key1 < t.key1) {
                x.send(x.v, true, key1, p1, vts + (buf ^ 1) * kTile, bad);
#pragma unroll
                for (int i = 0; i < Sender<T, D>::kPages; i++)
                    p1[i] = p2[i];
            }
            if (key2 + kWideKeys < t.key1)
                x.find(key2 + kWideKeys, p2);
            if (key < wave_last) {
                weights<T, D, 2>(r, s, p, key, end, masked(key, wave_first), a.scale2, [&] {
                    // (of the last tile: of what is there, and not used)
                    s[0] = scores<T, D>(lds + (buf ^ 1) * kTile, q);
                    s[1] = scores<T, D>(lds + (buf ^ 1) * kTile + 32 * D, q);
                });
                add_values<T, D, 2>(r, p, vts + buf * kTile);
            }
            key = key1;
            buf ^= 1;
            if (key >= t.key1)
                break;
            wait_sent();
            __syncthreads();
        }
        while (key < t.key1) {  // rare: values that are not finite
            if (key < wave_last) {
                weights<T, D, 2>(r, s, p, key, end, true, a.scale2, [] {});
                add_odd_values<T, D, 2>(r, p, vts + buf * kTile, key, end);
            }
            key += kWideKeys;
            if (key >= t.key1)
                break;
            __syncthreads();
            x.find(key, p1);
            x.send(x.k, false, key, p1, lds + buf * kTile, bad);
            x.send(x.v, true, key, p1, vts + buf * kTile, bad);
            wait_sent();
            __syncthreads();
            x.clean(vts + buf * kTile, key);
            __syncthreads();
            s[0] = scores<T, D>(lds + buf * kTile, q);
            s[1] = scores<T, D>(lds + buf * kTile + 32 * D, q);
        }
    }
    write_row<T, D>(a, t.u, t.h, row, t.last + 1, t.chunk, r, r.l + __shfl_xor(r.l, 32), t.rows);
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
    if (!item_unit(a, pv, a.b.groups + a.b.n, part_rows, D, status, u))
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
template <int D>
constexpr int kSmallWaves = D == 256 ? 4 : 8;
template <typename T, int D>
__global__ __launch_bounds__(kSmallWaves<D>* kWave, 1) void attn_small_kernel(AttnIn a, const PlanView pv,
                                                                              uint32_t* status)
{
    constexpr int kW = kSmallWaves<D>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[kW * 2 * kNarrowKeys * D];
    __shared__ Joined<kW> joined;
    Unit u;
    if (!item_unit(a, pv, a.b.n, 0, D, status, u))
        return;
    bool bad = false;
    narrow_tile<T, D, kW>(a, make_tile(a, u, blockIdx.x - u.item0, kNarrow), lds, joined, bad);
    if (bad)
        atomicOr(status, kErrInval);
}

// ---------------------------------------------------------------------------
// Rows in parts joined: a wave for a row, or a workgroup where rows have many
// parts, or, where there are more rows than waves, a quarter of a wave.
// ---------------------------------------------------------------------------

// A row's parts: its run's chunks, then its own.
struct Parts {
    uint64_t at0, at1;
    uint32_t n0, n;
    __device__ uint64_t at(uint32_t i) const { return i < n0 ? at0 + i : at1 + (i - n0); }
};
__device__ __forceinline__ Parts parts_of(const Unit& u, uint32_t t, uint32_t x, uint32_t ratio)
{
    Parts p{0, 0, 0, 0};
    if (t - u.tok0 >= u.ntok || !(u.flags & kUnitParts))
        return p;
    const uint32_t h = x / ratio, row = (t - u.tok0) * ratio + x % ratio;
    p.n = u.chunks;
    p.at1 = u.part0 + ((uint64_t)h * u.ntok * ratio + row) * u.chunks;
    // a token before its sequence's first key sees no prefix either
    if ((int64_t)u.pos0 + (t - u.tok0) >= 0) {
        p.n0 = u.run_chunks;
        p.n += p.n0;
        p.at0 = u.run_part0 + ((uint64_t)h * u.run_rows + u.run_row0 + row) * p.n0;
    }
    return p;
}

constexpr float kLog2e = 1.44269504088896341f;

// The weight of a part among parts whose largest maximum is m.  (Their maxima and sums
// are kept apart: in one number, the log-sum-exp, scores of 2^14 would leave the sum
// eleven bits.)  A part that the row sees nothing of has none; NaN stays NaN.
__device__ __forceinline__ float part_weight(v2f stat, float m, float scale2)
{
    const float w = stat[1] * __builtin_amdgcn_exp2f((stat[0] - m) * scale2);
    return stat[1] == 0 ? 0.0f : stat[0] == -INFINITY ? stat[1] : w;
}

// Neighbouring rows of the output by a wave, four at a time (16 lanes a row, D / 16
// elements a lane); a row's sequence is looked for only where it is not the last
// one's.  Bound by reading the parts: 95,488 rows of 64 in two parts 16.6 us, 105,600
// of 128 29.7, where a wave for a row took 48 and 63.
template <typename T, int D>
__device__ __forceinline__ void join_quarters(const AttnIn& a, const PlanView& pv, uint64_t y0, uint64_t y1)
{
    constexpr int kPer = D / 16, kAtOnce = 4;
    const uint32_t g = lane_id() / 16, d = lane_id() % 16 * kPer;
    Unit u{};
    for (; y0 < y1; y0 += 4) {
        const bool mine = y0 + g < y1;
        const uint32_t y = (uint32_t)(mine ? y0 + g : y1 - 1), t = y / a.q_heads, x = y % a.q_heads;
        if (__any(t - u.tok0 >= u.ntok)) {
            uint32_t s = 0, t_last = 0xFFFFFFFFu, s_last = 0;
            for (uint32_t k = 0; k < 4; k++) {
                const uint32_t tk = __builtin_amdgcn_readlane(t, k * 16);
                s_last = tk == t_last ? s_last : sequence_of(a.b, tk);
                t_last = tk;
                s = g == k ? s_last : s;
            }
            u = pv.unit[a.b.groups + s];
        }
        const Parts p = parts_of(u, t, x, a.ratio);
        const bool live = mine && p.n;
        float m = -INFINITY, total = 0, v[kPer] = {};
        for (uint32_t i0 = 0; __any(live && i0 < p.n); i0 += kAtOnce) {
            if (!live || i0 >= p.n)
                continue;
            v2f e[kAtOnce];
            v4f r[kAtOnce][kPer / 4];
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                const uint64_t at = p.at(i0 + j < p.n ? i0 + j : p.n - 1);
                e[j] = a.part_stat[at];
#pragma unroll
                for (int c = 0; c < kPer / 4; c++)
                    r[j][c] = *reinterpret_cast<const v4f*>(a.part + at * D + d + c * 4);
            }
            float now = m;
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                if (i0 + j >= p.n)
                    e[j] = v2f{-INFINITY, 0};
                now = fmaxf(now, e[j][0]);
            }
            const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - now) * a.scale2);
            m = now;
            total *= keep;
#pragma unroll
            for (int c = 0; c < kPer; c++)
                v[c] *= keep;
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                const float w = part_weight(e[j], m, a.scale2);
                total += w;
#pragma unroll
                for (int c = 0; c < kPer; c++)
                    v[c] = w == 0 ? v[c] : __builtin_fmaf(w, r[j][c / 4][c % 4], v[c]);
            }
        }
        if (!live)
            continue;
        const bool seen = total > 0 || total != total;
        const float inv = seen ? 1.0f / total : 0.0f;
        typedef T v4t __attribute__((ext_vector_type(4)));
        uint16_t* out = a.out + t * a.out_stride + (uint64_t)x * D + d;
#pragma unroll
        for (int c = 0; c < kPer / 4; c++) {
            v4t z;
#pragma unroll
            for (int k = 0; k < 4; k++)
                z[k] = (T)(v[c * 4 + k] * inv);
            *reinterpret_cast<v4t*>(out + c * 4) = z;
        }
        if (d == 0 && a.lse)
            a.lse[(uint64_t)t * a.q_heads + x] = seen ? lse_of<T>(m, total, a.scale2) : -INFINITY;
    }
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
    if (ph.part_rows == 0 || !plan_fits(ph, a, part_rows, D, items))
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

// Is a batch small: no unit has more rows than a narrow tile, and no more keys than
// attn_small_kernel is the faster on?
bool small(const dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t ratio)
{
    const uint64_t keys = kv.head_dim == 64 ? 1024 : kv.head_dim == 128 ? 768 : 256;
    return b.groups == 0 && b.q_tokens * ratio <= kNarrowRows && b.tables.entries * c->cfg.block_size <= keys;
}

// Items wanted: three for every two places of a workgroup (two a compute unit).
// (us with one for each place, three for two, two and three: 64 decode rows of up to
// 8,192 keys 227, 217, 216 and 216; 256 rows on 8 shared prefixes 179, 178, 181 and 185; 8
// tails on 2 prefixes 753, 774, 764 and 755.)
uint64_t item_target(const dm_ctx* c) { return 3ull * c->n_cu; }

// Items that a plan can have: the tiles of its units, and what cuts add: at most
// the items wanted, and no more than the table entries' keys are chunks for each
// tile.
uint64_t most_items(const dm_ctx* c, const dm_token_batch& b, uint32_t ratio, uint32_t kv_heads)
{
    const uint64_t rows = b.q_tokens * ratio;
    auto tiles = [&](uint64_t units) { return rows / kWide + units; };
    const uint64_t uncut = tiles(b.tables.n) + (b.groups ? tiles(b.groups) : 0);
    uint64_t cuts = item_target(c);
    const uint64_t chunks = b.tables.entries * c->cfg.block_size / kChunk + 1;
    if (chunks < cuts && chunks * uncut * kv_heads < cuts)
        cuts = chunks * uncut * kv_heads;
    return uncut * kv_heads + cuts;
}

// Rows of parts that a batch can need: those of cut units, and with runs twice its
// rows (a shared prefix and the rest), up to a bound past which the plan neither
// shares nor cuts.  Cut units: a chunk is longer than an item's share of the cost,
// weight * keys over all units, and c chunks >= 2 take fewer than 2 keys / chunk, so
// that they have fewer than 2 rows / weight <= 128 rows for each item wanted.
uint64_t part_rows_of(const dm_ctx* c, const dm_token_batch& b, uint32_t q_heads)
{
    const uint64_t rows = b.groups ? 2 * b.q_tokens * q_heads : 0;
    return (rows < kPartRows ? rows : kPartRows) + kWide * item_target(c);
}

}  // namespace

uint64_t attn_plan_bytes(uint64_t n, uint64_t groups)
{
    return sizeof(PlanHead) + item0_bytes(n + groups) + sizeof(Unit) * (n + groups) + 2 * up16(4 * n) +
           2 * up16(4 * groups);
}

hipError_t attn_plan(dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t q_heads,
                     void* plan)
{
    PlanIn a;
    a.b = token_batch(c, b);
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.ratio = q_heads / kv.kv_heads;
    a.head_dim = kv.head_dim;
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
    const uint64_t most = is_small ? (uint64_t)b.tables.n * kv.kv_heads : most_items(c, b, a.ratio, kv.kv_heads);
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
