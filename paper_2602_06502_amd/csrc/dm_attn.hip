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
//   narrow tiles: 32 rows; the four waves take every fourth 32 keys, each
//     through its own part of LDS, and are joined at the end.  For rows that
//     are few: bound by reading the pages.
//   wide tiles: 128 rows, 32 a wave, on a shared tile of 64 keys (two in LDS).
//     Bound by the matrix and vector units.
#include "dm_internal.h"
#include "dm_pages.h"

namespace dm {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr uint32_t kNarrow = 32, kWide = 128;  // rows of a tile
constexpr uint32_t kNarrowKeys = 32, kWideKeys = 64;
constexpr uint32_t kChunk = 128;               // chunks are multiples of this many keys
constexpr uint32_t kLeastChunk = 128;          // and no shorter than this
constexpr int kPlanThreads = 1024;
constexpr uint64_t kPartRows = 1ull << 20;     // rows of parts kept beyond those of cut items

// The plan in memory: a head, then a unit for each run and each sequence
// (runs first), each with the number of items before it, then words of the
// sequences.
struct PlanHead {
    uint32_t n, groups, q_tokens, q_heads, kv_heads, shift;  // what it was made for
    int64_t entries;
    uint32_t items, units;
    uint32_t chunk;       // keys of a chunk
    uint32_t part_rows;   // rows of parts
    uint32_t most_parts;  // of a row
    uint32_t pad[3];
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
};
enum : uint32_t { kUnitWide = 1, kUnitCausal = 2, kUnitParts = 4 };

struct PlanView {
    PlanHead* head;
    Unit* unit;
    uint32_t* limit;   // [n] pages that s has in common with its run's first, at most
    uint32_t* run;     // [n] its run
    uint32_t* shared;  // [groups] pages shared
    uint32_t* gain;    // [groups] tiles of its sequences, each on its own
};

__host__ __device__ inline uint64_t up16(uint64_t x) { return (x + 15) & ~15ull; }

__host__ __device__ inline PlanView plan_view(void* p, uint64_t n, uint64_t groups)
{
    PlanView v;
    uint8_t* b = static_cast<uint8_t*>(p);
    v.head = reinterpret_cast<PlanHead*>(b);
    b += sizeof(PlanHead);
    v.unit = reinterpret_cast<Unit*>(b);
    b += up16(sizeof(Unit) * (n + groups));
    v.limit = reinterpret_cast<uint32_t*>(b);
    b += up16(4 * n);
    v.run = reinterpret_cast<uint32_t*>(b);
    b += up16(4 * n);
    v.shared = reinterpret_cast<uint32_t*>(b);
    b += up16(4 * groups);
    v.gain = reinterpret_cast<uint32_t*>(b);
    return v;
}

// A tile's cost a key: a wide one reads as much as a narrow one and takes
// about twice its time.
__device__ __forceinline__ uint32_t tile_rows(uint64_t rows) { return rows > 2 * kNarrow ? kWide : kNarrow; }
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
    uint32_t q_heads, kv_heads, ratio;
    uint64_t target;     // items wanted
    uint64_t part_rows;  // rows of parts there is room for
    uint32_t* arrived;   // workgroups that are done with their sequences; zero between calls
};

// Words that workgroups on other dies write or read within the launch.
__device__ __forceinline__ void agent_store(uint32_t* p, uint32_t x)
{
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t agent_load(const uint32_t* p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

constexpr uint32_t kNoSay = 0xFFFFFFFFu;
constexpr uint32_t kLdsRuns = 1024;

// How many leading pages sequence s could share with its run's first one, by
// the whole workgroup (kNoSay: it has no row that sees a key).  A shared prefix
// ends before the first new token of every sequence that has any.
__device__ void common_pages(const PlanIn& a, const PlanView& pv, uint32_t s, uint32_t* least)
{
    const TokenBatch& b = a.b;
    const uint32_t g = wave_find(b.group_off, b.groups, 1, (int64_t)s);
    const int64_t g0 = b.group_off[g];
    const bool mine = run_ok(b, g) && g0 <= (int64_t)s && (int64_t)s < b.group_off[g + 1];
    const SeqView v = sequence_view(b, s);
    uint32_t limit = 0;
    if (mine && (v.ntok == 0 || (!v.bad && v.len == 0))) {
        limit = kNoSay;
    } else if (mine && !v.bad && v.pos0 > 0) {
        const SeqView f = sequence_view(b, (uint32_t)g0);
        int64_t m = v.pos0 >> b.shift;
        const int64_t have = f.bad ? 0 : b.off[g0 + 1] - f.off;
        if (have < m)
            m = have;
        limit = (uint32_t)m;
        __syncthreads();
        if (threadIdx.x == 0)
            *least = limit;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < limit; i += kPlanThreads)
            if (b.page[v.off + i] != b.page[f.off + i]) {
                atomicMin(least, i);
                break;
            }
        __syncthreads();
        limit = *least;
    }
    if (threadIdx.x == 0) {
        agent_store(&pv.limit[s], limit);
        agent_store(&pv.run[s], mine ? g : kNoSay);
    }
}

// The units of run g over its shared pages, and of sequence s.
__device__ __forceinline__ Unit run_unit(const PlanIn& a, uint32_t g, uint32_t pages)
{
    Unit u{};
    if (pages == 0)
        return u;
    const int64_t s0 = a.b.group_off[g], s1 = a.b.group_off[g + 1];
    u.tok0 = (uint32_t)a.b.q_off[s0];
    u.ntok = (uint32_t)a.b.q_off[s1] - u.tok0;
    u.key1 = pages << a.b.shift;
    u.off = a.b.off[s0];
    u.table = pages;
    u.flags = kUnitParts | (tile_rows((uint64_t)u.ntok * a.ratio) == kWide ? kUnitWide : 0);
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
    u.flags = kUnitCausal | (pages ? kUnitParts : 0) |
              (tile_rows((uint64_t)u.ntok * a.ratio) == kWide ? kUnitWide : 0);
    return u;
}

// Is a pass of its own over `pages` common pages worth it for run g?  Where the
// run's rows together make clearly fewer tiles, over more than a chunk of keys.
__device__ __forceinline__ bool worth_sharing(const PlanIn& a, uint32_t g, uint32_t pages, uint64_t gain)
{
    if (pages == 0 || pages == kNoSay || !run_ok(a.b, g) || ((uint64_t)pages << a.b.shift) < kChunk)
        return false;
    const int64_t t0 = a.b.q_off[a.b.group_off[g]], t1 = a.b.q_off[a.b.group_off[g + 1]];
    return t0 >= 0 && t1 >= t0 && t1 <= (int64_t)a.b.q_tokens &&
           2 * gain >= 3 * weight_of((uint64_t)(t1 - t0) * a.ratio);
}

// Which runs share their prefixes, the chunk, and the units' items.  With
// runs, a workgroup for a sequence first, and the last one to finish goes on
// alone (a launch less; 10 us with two launches and every step through memory, at
// 256 sequences).  A thread keeps its unit in registers from step to step;
// beyond 1024 units the others are made again for each step.
__global__ __launch_bounds__(kPlanThreads) void attn_plan_kernel(PlanIn a, PlanView pv, uint32_t* status)
{
    __shared__ uint64_t lds[2 * kPlanThreads / kWave];
    __shared__ uint32_t run_pages[kLdsRuns], run_gain[kLdsRuns];
    __shared__ uint32_t most, least;
    const TokenBatch& b = a.b;
    const uint32_t units = b.groups + b.n, tid = threadIdx.x;
    if (b.groups) {
        for (uint32_t s = blockIdx.x; s < b.n; s += gridDim.x)
            common_pages(a, pv, s, &least);
        // thread 0 wrote the workgroup's words: its fence alone orders them (one by
        // every wave of 256 workgroups took 60 us)
        if (tid == 0) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
            least = atomicAdd(a.arrived, 1u);
        }
        __syncthreads();
        if (least != gridDim.x - 1)
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
    if (b.groups) {
        for (uint32_t g = tid; g < b.groups; g += kPlanThreads) {
            pages[g] = kNoSay;
            gain[g] = 0;
            bad |= !run_ok(b, g) || (g == 0 && b.group_off[0] != 0) ||
                   (g + 1 == b.groups && b.group_off[b.groups] != (int64_t)b.n);
        }
        settle();
        for (uint32_t s = tid; s < b.n; s += kPlanThreads) {
            const uint32_t g = agent_load(&pv.run[s]), limit = agent_load(&pv.limit[s]);
            const SeqView v = sequence_view(b, s);
            if (g >= b.groups)
                continue;
            atomicMin(&pages[g], limit);
            if (v.len)
                atomicAdd(&gain[g], (uint32_t)weight_of((uint64_t)v.ntok * a.ratio));
        }
        settle();
        for (uint32_t g = tid; g < b.groups; g += kPlanThreads)
            pages[g] = worth_sharing(a, g, pages[g], gain[g]) ? pages[g] : 0;
        settle();
    }
    // 0: as wanted; 1: without sharing and without cuts, if the parts of the
    // first try have no room
    for (int attempt = 0; attempt < 2; attempt++) {
        auto make = [&](uint32_t i) -> Unit {
            if (i < b.groups)
                return run_unit(a, i, attempt ? 0 : pages[i]);
            const uint32_t s = i - b.groups, g = b.groups ? agent_load(&pv.run[s]) : kNoSay;
            const SeqView v = sequence_view(b, s);
            bad |= v.bad;
            return sequence_unit(a, v, attempt || g >= b.groups ? 0 : pages[g]);
        };
        auto cost_of = [&](const Unit& u) -> uint64_t {
            return u.ntok ? weight_of((uint64_t)u.ntok * a.ratio) * (u.key1 - u.key0) : 0;
        };
        Unit mine{};
        if (tid < units)
            mine = make(tid);
        uint64_t cost = cost_of(mine);
        for (uint32_t i = tid + kPlanThreads; i < units; i += kPlanThreads)
            cost += cost_of(make(i));
        cost = block_sum64(cost, lds) * a.kv_heads;
        uint64_t chunk = (cost / a.target + kChunk) / kChunk * kChunk;
        if (chunk < kLeastChunk)
            chunk = kLeastChunk;
        if (attempt || chunk > 0x80000000ull)
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
                u = make(i);
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
            if (lane_id() == kWave - 1) {
                lds[tid / kWave] = i1;
                lds[kPlanThreads / kWave + tid / kWave] = r1;
            }
            __syncthreads();
            uint64_t ib = items, rb = rows;
            for (uint32_t w = 0; w < kPlanThreads / kWave; w++) {
                const uint64_t x = lds[w], y = lds[kPlanThreads / kWave + w];
                if (w < tid / kWave) {
                    ib += x;
                    rb += y;
                }
                items += x;
                rows += y;
            }
            if (i < units) {
                u.item0 = (uint32_t)(ib + i1 - it);
                u.part0 = (uint32_t)(rb + r1 - rw);
                pv.unit[i] = u;
                if (i < b.groups)
                    pv.shared[i] = u.table;
            }
        }
        if (rows <= a.part_rows && items < (1ull << 32)) {
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
                h.units = units;
                h.chunk = (uint32_t)chunk;
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

// Tiles of keys in LDS: rows of D elements in 16-byte chunks, a row's chunks in
// an order of its own, so that the 16 rows that neighbouring lanes read a
// chunk of (K), or the four rows that they read 64 bytes of (V), lie in different
// banks.
template <int D>
__device__ __forceinline__ uint32_t k_swizzle(uint32_t row)
{
    return D == 64 ? (row >> 1) & 7 : row & 15;
}
template <int D>
__device__ __forceinline__ uint32_t v_swizzle(uint32_t row)
{
    return D == 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2;
}

struct AttnIn {
    TokenBatch b;
    const uint16_t *k, *v;  // the layer's pages
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    float* part;       // [part rows][D] parts of rows, then their lse
    float* part_lse;
    int64_t q_stride, out_stride;
    uint32_t n_pages, q_heads, kv_heads, ratio;
    float scale2;      // scale * log2(e)
};

// What a lane keeps of its row.
template <int D>
struct Row {
    v16f o[D / 32];  // O^T: element (d = db * 32 + (i / 4) * 8 + half * 4 + i % 4, row)
    float m, l;      // maximum (of raw scores), this half's sum
};

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

// The running softmax of NB tiles of 32 keys: the tiles' weights in T.  limit:
// the keys that the lane's row sees (absolute), key0: the tiles' first; masked:
// some row does not see all of them.
template <typename T, int D, int NB>
__device__ __forceinline__ void weights(Row<D>& r, v16f (&s)[NB], typename Vec8<T>::type (&p)[NB][2],
                                        uint32_t key0, uint32_t limit, bool masked, float scale2)
{
    const uint32_t half = lane_id() / 32;
    if (masked) {
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (key0 + b * 32 + (i / 4) * 8 + half * 4 + i % 4 >= limit)
                    s[b][i] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int i = 0; i < 16; i++)
            mx = fmaxf(mx, s[b][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    // The maximum moves only when some row's has grown by more than 2^8 in weight:
    // weights up to 2^8 lose nothing in 32-bit sums nor, rounded, in T.
    const float grow = (mx - r.m) * scale2;
    if (__any(!(grow <= 8.0f))) {
        const float m = fmaxf(r.m, mx);
        const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((r.m - m) * scale2);
        r.m = m;
        r.l *= keep;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                r.o[d][i] *= keep;
    }
    const float base = r.m == -INFINITY ? 0.0f : r.m * scale2;
    float sum = 0;
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale2, -base));
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

// The result of a row (o: O^T as in Row): divided by the sum, written to the
// output or to its row of parts.
template <typename T, int D>
__device__ __forceinline__ void write_row(const AttnIn& a, const Unit& u, uint32_t h, uint32_t row,
                                          uint32_t rows, uint32_t chunk, const Row<D>& r, float l)
{
    const uint32_t half = lane_id() / 32;
    if (row >= rows)
        return;
    const float inv = l > 0 || l != l ? 1.0f / l : 0.0f;
    const bool seen = l > 0 || l != l;
    const float lse = seen ? (r.m * a.scale2 + __builtin_log2f(l)) * 0.69314718055994531f : -INFINITY;
    if (u.flags & kUnitParts) {
        const uint64_t at = u.part0 + ((uint64_t)h * rows + row) * u.chunks + chunk;
        float* o = a.part + at * D;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                typedef float v4f __attribute__((ext_vector_type(4)));
                v4f x;
                for (int k = 0; k < 4; k++)
                    x[k] = seen ? r.o[d][i + k] * inv : 0.0f;
                *reinterpret_cast<v4f*>(o + d * 32 + i * 2 + half * 4) = x;
            }
        if (half == 0)
            a.part_lse[at] = lse;
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
        a.lse[(uint64_t)t * a.q_heads + x] = lse;
}

// An item's place: its unit, tile, chunk and KV head.
struct Item {
    Unit u;
    uint32_t tile, chunk, h, rows;
    uint32_t key0, key1;  // keys of the chunk
};

// 16 bytes of a page's row; zeros where there is no such key or page.
struct KeyRows {
    const int32_t* table;
    uint32_t pages, key1, n_pages, shift;
    uint64_t head_at;   // elements from a page's start to the KV head's rows
    uint64_t page_size; // elements of a page
    __device__ __forceinline__ int32_t page(uint32_t key) const
    {
        const uint32_t i = key >> shift;
        if (key >= key1 || i >= pages)
            return -1;
        return table[i];
    }
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_kernel(AttnIn a, const PlanView pv,
                                                                          uint64_t part_rows,
                                                                          uint32_t* status)
{
    using V = typename Vec8<T>::type;
    // two tiles of 64 keys and values, or four waves' 32 keys and values
    __shared__ __attribute__((aligned(16))) uint16_t lds[4 * kWideKeys * D];
    __shared__ uint32_t odd_tile[2];
    __shared__ float joined[2][kWaves][kNarrow];
    const PlanHead& ph = *pv.head;
    if (ph.n != a.b.n || ph.groups != a.b.groups || ph.q_tokens != a.b.q_tokens ||
        ph.q_heads != a.q_heads || ph.kv_heads != a.kv_heads || ph.shift != a.b.shift ||
        ph.entries != a.b.entries || ph.part_rows > part_rows || ph.items > gridDim.x) {
        if (blockIdx.x == 0 && threadIdx.x == 0)
            atomicOr(status, kErrInval);  // the plan of another batch
        return;
    }
    const uint32_t items = ph.items, wave = threadIdx.x / kWave, lane = lane_id();
    const uint32_t row32 = lane % 32, half = lane / 32;
    const uint32_t item = blockIdx.x;
    if (item >= items)
        return;
    {
        const uint32_t ui = wave_find(&pv.unit[0].item0, a.b.groups + a.b.n, sizeof(Unit) / 4, item);
        const Unit u = pv.unit[ui];
        const uint32_t rows = u.ntok * a.ratio;
        const bool wide = u.flags & kUnitWide;
        const uint32_t per_tile = wide ? kWide : kNarrow, tiles = (rows + per_tile - 1) / per_tile;
        uint32_t x = item - u.item0;
        const uint32_t h = x % a.kv_heads;
        x /= a.kv_heads;
        // a sequence's last tiles see the most keys: they go first
        const uint32_t tile = tiles - 1 - x % tiles, chunk = x / tiles;
        const uint32_t first_row = tile * per_tile;
        const uint32_t last_row = first_row + per_tile < rows ? first_row + per_tile - 1 : rows - 1;
        const uint32_t key0 = u.key0 + chunk * ph.chunk;
        uint32_t key1 = u.key1 - key0 > ph.chunk ? key0 + ph.chunk : u.key1;
        // keys that a row sees, of the unit's
        auto sees = [&](uint32_t row) -> uint32_t {
            if (!(u.flags & kUnitCausal))
                return u.key1;
            const int64_t n = (int64_t)u.pos0 + row / a.ratio + 1;
            return n < 0 ? 0 : n > u.key1 ? u.key1 : (uint32_t)n;
        };
        const uint32_t see_first = sees(first_row), see_last = sees(last_row);
        if (key1 > see_last)
            key1 = see_last;

        const uint32_t row = first_row + (wide ? wave * 32 : 0) + row32;
        const uint32_t limit = sees(row < rows ? row : last_row);
        V q[D / 16];
        {
            const uint32_t rq = row < rows ? row : last_row;
            const uint16_t* at = a.q + (uint64_t)(u.tok0 + rq / a.ratio) * a.q_stride +
                                 (uint64_t)(h * a.ratio + rq % a.ratio) * D;
#pragma unroll
            for (int k = 0; k < D / 16; k++)
                q[k] = *reinterpret_cast<const V*>(at + k * 16 + half * 8);
        }
        Row<D> r;
        r.m = -INFINITY;
        r.l = 0;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
            r.o[d] = v16f{};

        KeyRows kr{a.b.page + u.off, u.table, key1, a.n_pages, a.b.shift,
                   (uint64_t)h * D << a.b.shift, (uint64_t)a.kv_heads * D << a.b.shift};
        const uint32_t slot_mask = (1u << a.b.shift) - 1;
        bool bad_page = false;
        // loads of a thread: rows r0, r0 + step, ... of a tile, chunk `ch`
        constexpr uint32_t kRowChunks = D / 8;

        if (!wide) {
            constexpr int kLoads = kNarrowKeys * D / 8 / kWave;
            constexpr uint32_t kStep = kWave / kRowChunks;  // rows a load of the wave covers
            uint16_t* kt = lds + wave * 2 * kNarrowKeys * D;
            uint16_t* vt = kt + kNarrowKeys * D;
            const uint32_t ch = lane % kRowChunks, r0 = lane / kRowChunks;
            v4u32 kx[kLoads], vx[kLoads];
            auto fetch = [&](uint32_t key, int32_t page) {  // page: of row `lane`
#pragma unroll
                for (int i = 0; i < kLoads; i++) {
                    const uint32_t rr = r0 + i * kStep;
                    const int32_t p = __shfl(page, rr);
                    kx[i] = v4u32{};
                    vx[i] = v4u32{};
                    if (p >= 0) {
                        const uint64_t at = (uint64_t)p * kr.page_size + kr.head_at +
                                            (uint64_t)((key + rr) & slot_mask) * D + ch * 8;
                        kx[i] = *reinterpret_cast<const v4u32*>(a.k + at);
                        vx[i] = *reinterpret_cast<const v4u32*>(a.v + at);
                    }
                }
            };
            auto page_of = [&](uint32_t key) -> int32_t {
                int32_t p = lane < kNarrowKeys ? kr.page(key + lane) : -1;
                if (p >= 0 && (uint32_t)p >= kr.n_pages)
                    p = -1;
                if (p < 0 && lane < kNarrowKeys && key + lane < key1)
                    bad_page = true;
                return p;
            };
            bool masked = false, odd = false;
            auto stage = [&](uint32_t key) {
                masked = key + kNarrowKeys > see_first || key + kNarrowKeys > key1;
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int i = 0; i < kLoads; i++) {
                    const uint32_t rr = r0 + i * kStep;
                    *reinterpret_cast<v4u32*>(kt + rr * D + (ch ^ k_swizzle<D>(rr)) * 8) = kx[i];
                    *reinterpret_cast<v4u32*>(vt + rr * D + (ch ^ v_swizzle<D>(rr)) * 8) = vx[i];
                    if (masked)
                        odd |= not_finite<T>(vx[i]);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            };
            uint32_t key = key0 + wave * kNarrowKeys;
            const uint32_t step = kWaves * kNarrowKeys, end = limit < key1 ? limit : key1;
            V p[1][2];
            int32_t page = page_of(key);
            if (key < key1)
                fetch(key, page);
            page = page_of(key + step);
            for (; key < key1; key += step) {
                stage(key);
                if (__any(odd))
                    break;
                if (key + step < key1)
                    fetch(key + step, page);
                page = page_of(key + 2 * step);
                v16f s[1] = {scores<T, D>(kt, q)};
                weights<T, D, 1>(r, s, p, key, end, masked, a.scale2);
                add_values<T, D, 1>(r, p, vt);
            }
            while (key < key1) {
                v16f s[1] = {scores<T, D>(kt, q)};
                weights<T, D, 1>(r, s, p, key, end, true, a.scale2);
                add_odd_values<T, D, 1>(r, p, vt, key, end);
                key += step;
                if (key < key1) {
                    fetch(key, page_of(key));
                    stage(key);
                }
            }
            // the four waves' parts joined
            float l = r.l + __shfl_xor(r.l, 32);
            if (half == 0) {
                joined[0][wave][row32] = r.m;
                joined[1][wave][row32] = l;
            }
            __syncthreads();
            float m = -INFINITY;
            for (int w = 0; w < kWaves; w++)
                m = fmaxf(m, joined[0][w][row32]);
            float total = 0;
            for (int w = 0; w < kWaves; w++) {
                const float mw = joined[0][w][row32];
                total += mw == -INFINITY ? (joined[1][w][row32] != joined[1][w][row32] ? joined[1][w][row32] : 0.0f)
                                         : joined[1][w][row32] * __builtin_amdgcn_exp2f((mw - m) * a.scale2);
            }
            const float keep = r.m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((r.m - m) * a.scale2);
            float* sum = reinterpret_cast<float*>(lds);  // [D / 4][32 rows][4] of a wave's share
            // wave w adds the waves' parts in order, a quarter of d each turn:
            // in turn each wave adds its own into LDS
            for (int w = 0; w < kWaves; w++) {
                __syncthreads();
                if ((int)wave == w)
#pragma unroll
                    for (int d = 0; d < D / 32; d++)
#pragma unroll
                        for (int i = 0; i < 16; i++) {
                            float* at = sum + (d * 16 + i) * kWave + lane;
                            const float x = r.o[d][i] * keep;
                            *at = w ? *at + x : x;
                        }
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int d = 0; d < D / 32; d++)
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        r.o[d][i] = sum[(d * 16 + i) * kWave + lane];
                r.m = m;
                write_row<T, D>(a, u, h, row, rows, chunk, r, total);
            }
        } else {
            constexpr int kLoads = kWideKeys * D / 8 / kThreads;
            constexpr uint32_t kStep = kThreads / kRowChunks;
            const uint32_t ch = threadIdx.x % kRowChunks, r0 = threadIdx.x / kRowChunks;
            v4u32 kx[kLoads], vx[kLoads];
            int32_t page[kLoads];
            auto find = [&](uint32_t key) {
#pragma unroll
                for (int i = 0; i < kLoads; i++) {
                    page[i] = kr.page(key + r0 + i * kStep);
                    if (page[i] >= 0 && (uint32_t)page[i] >= kr.n_pages)
                        page[i] = -1;
                    if (page[i] < 0 && key + r0 + i * kStep < key1)
                        bad_page = true;
                }
            };
            auto fetch = [&](uint32_t key) {
#pragma unroll
                for (int i = 0; i < kLoads; i++) {
                    kx[i] = v4u32{};
                    vx[i] = v4u32{};
                    if (page[i] >= 0) {
                        const uint64_t at = (uint64_t)page[i] * kr.page_size + kr.head_at +
                                            (uint64_t)((key + r0 + i * kStep) & slot_mask) * D + ch * 8;
                        kx[i] = *reinterpret_cast<const v4u32*>(a.k + at);
                        vx[i] = *reinterpret_cast<const v4u32*>(a.v + at);
                    }
                }
            };
            // keys that the wave's first and last rows see
            const uint32_t w0 = first_row + wave * 32, w1 = w0 + 31 < last_row ? w0 + 31 : last_row;
            const bool has_rows = w0 < rows;
            const uint32_t wave_first = has_rows ? sees(w0) : 0, wave_last = has_rows ? sees(w1) : 0;
            if (threadIdx.x < 2)
                odd_tile[threadIdx.x] = 0;
            __syncthreads();
            find(key0);
            fetch(key0);
            find(key0 + kWideKeys);
            bool odd = false;
            auto stage = [&](uint32_t key, uint16_t* kt) {
                uint16_t* vt = kt + kWideKeys * D;
                const bool masked = key + kWideKeys > see_first || key + kWideKeys > key1;
#pragma unroll
                for (int i = 0; i < kLoads; i++) {
                    const uint32_t rr = r0 + i * kStep;
                    *reinterpret_cast<v4u32*>(kt + rr * D + (ch ^ k_swizzle<D>(rr)) * 8) = kx[i];
                    *reinterpret_cast<v4u32*>(vt + rr * D + (ch ^ v_swizzle<D>(rr)) * 8) = vx[i];
                    if (masked)
                        odd |= not_finite<T>(vx[i]);
                }
            };
            const uint32_t end = limit < key1 ? limit : key1;
            V p[2][2];
            uint32_t key = key0, buf = 0;
            for (; key < key1; key += kWideKeys, buf ^= 1) {
                uint16_t* kt = lds + buf * 2 * kWideKeys * D;
                stage(key, kt);
                if (odd)
                    odd_tile[buf] = 1;
                __syncthreads();
                if (odd_tile[buf])
                    break;
                if (key + kWideKeys < key1)
                    fetch(key + kWideKeys);
                find(key + 2 * kWideKeys);
                if (key < wave_last) {
                    v16f s[2] = {scores<T, D>(kt, q), scores<T, D>(kt + 32 * D, q)};
                    weights<T, D, 2>(r, s, p, key, end, key + kWideKeys > wave_first || key + kWideKeys > key1,
                                     a.scale2);
                    add_values<T, D, 2>(r, p, kt + kWideKeys * D);
                }
            }
            while (key < key1) {
                uint16_t* kt = lds + buf * 2 * kWideKeys * D;
                if (key < wave_last) {
                    v16f s[2] = {scores<T, D>(kt, q), scores<T, D>(kt + 32 * D, q)};
                    weights<T, D, 2>(r, s, p, key, end, true, a.scale2);
                    add_odd_values<T, D, 2>(r, p, kt + kWideKeys * D, key, end);
                }
                key += kWideKeys;
                if (key < key1) {
                    find(key);
                    fetch(key);
                    __syncthreads();
                    stage(key, kt);
                    __syncthreads();
                }
            }
            const float l = r.l + __shfl_xor(r.l, 32);
            write_row<T, D>(a, u, h, row, rows, chunk, r, l);
        }
        if (bad_page)
            atomicOr(status, kErrInval);
    }
}

// ---------------------------------------------------------------------------
// Rows in parts joined: a wave for a row, or a workgroup where rows have many
// parts.
// ---------------------------------------------------------------------------

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnIn a, const PlanView pv,
                                                             uint64_t part_rows)
{
    constexpr int kPer = D / kWave;  // elements a lane
    __shared__ float acc[kWaves][D];
    const PlanHead& ph = *pv.head;
    if (ph.part_rows == 0 || ph.n != a.b.n || ph.groups != a.b.groups || ph.q_tokens != a.b.q_tokens ||
        ph.q_heads != a.q_heads || ph.kv_heads != a.kv_heads || ph.shift != a.b.shift ||
        ph.entries != a.b.entries || ph.part_rows > part_rows)
        return;
    const uint32_t wave = threadIdx.x / kWave, lane = lane_id();
    const bool together = ph.most_parts > 16;
    const uint64_t all = (uint64_t)a.b.q_tokens * a.q_heads;
    const uint64_t step = together ? gridDim.x : (uint64_t)gridDim.x * kWaves;
    for (uint64_t y0 = together ? blockIdx.x : (uint64_t)blockIdx.x * kWaves; y0 < all; y0 += step) {
        const uint64_t y = together ? y0 : y0 + wave;
        const bool mine = y < all;
        const uint32_t t = mine ? (uint32_t)(y / a.q_heads) : 0, x = mine ? (uint32_t)(y % a.q_heads) : 0;
        const uint32_t s = sequence_of(a.b, t), h = x / a.ratio;
        const Unit u = pv.unit[a.b.groups + s];
        const bool live = mine && t - u.tok0 < u.ntok && (u.flags & kUnitParts);
        const uint32_t run = a.b.groups && live ? pv.run[s] : 0xFFFFFFFFu;
        // the row's parts: its run's chunks, then its own
        uint32_t n0 = 0, n1 = 0;
        uint64_t at0 = 0, at1 = 0;
        if (live) {
            const uint32_t row = (t - u.tok0) * a.ratio + x % a.ratio;
            n1 = u.chunks;
            at1 = u.part0 + ((uint64_t)h * u.ntok * a.ratio + row) * n1;
            // a token before its sequence's first key sees no prefix either
            if (run < a.b.groups && pv.shared[run] && (int64_t)u.pos0 + (t - u.tok0) >= 0) {
                const Unit g = pv.unit[run];
                n0 = g.chunks;
                at0 = g.part0 + ((uint64_t)h * g.ntok * a.ratio + (t - g.tok0) * a.ratio + x % a.ratio) * n0;
            }
        }
        const uint32_t n = n0 + n1;
        auto place = [&](uint32_t i) { return i < n0 ? at0 + i : at1 + (i - n0); };
        // the parts' weights, a lane each; then their rows, whose loads need not
        // wait for one another
        float m = -INFINITY;
        for (uint32_t i = lane; i < n; i += kWave)
            m = fmaxf(m, a.part_lse[place(i)]);
#pragma unroll
        for (int o = 1; o < kWave; o *= 2)
            m = fmaxf(m, __shfl_xor(m, o));
        float v[kPer] = {}, total = 0;
        const uint32_t from = together ? wave * kWave : 0, by = together ? kWaves * kWave : kWave;
        for (uint32_t i0 = from; i0 < n; i0 += by) {
            const uint32_t i = i0 + lane;
            const float e = i < n ? a.part_lse[place(i)] : -INFINITY;
            // a part that the row sees nothing of has no weight; NaN stays NaN
            const float w = e == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((e - m) * 1.44269504088896341f);
            total += w;
            const uint32_t k1 = n - i0 < kWave ? n - i0 : kWave;
            for (uint32_t k = 0; k < k1; k += 4) {
                float x[4], y[4][kPer];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    x[j] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), k + j));
                    const float* at = a.part + place(i0 + (k + j < k1 ? k + j : k1 - 1)) * D + lane * kPer;
#pragma unroll
                    for (int c = 0; c < kPer; c++)
                        y[j][c] = at[c];
                }
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int c = 0; c < kPer; c++)
                        v[c] = x[j] == 0 ? v[c] : __builtin_fmaf(x[j], y[j][c], v[c]);
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
                seen ? m + __builtin_log2f(total) * 0.69314718055994531f : -INFINITY;
    }
}

// Items wanted: four for each place of a workgroup (two a compute unit).
uint64_t item_target(const dm_ctx* c) { return 8ull * c->n_cu; }

// Items that a plan can have: the tiles of its units (a unit of more than 64
// rows has wide ones), and what cuts add: at most the items wanted, and no more
// than the table entries' keys are chunks for each tile.
uint64_t most_items(const dm_ctx* c, const dm_token_batch& b, uint32_t ratio, uint32_t kv_heads)
{
    const uint64_t rows = b.q_tokens * ratio;
    auto tiles = [&](uint64_t units) {
        const uint64_t some = rows / kWide + 2 * units, few = rows / kNarrow + units;
        return some < few ? some : few;
    };
    const uint64_t uncut = tiles(b.tables.n) + (b.groups ? tiles(b.groups) : 0);
    uint64_t cuts = item_target(c);
    const uint64_t chunks = b.tables.entries * c->cfg.block_size / kChunk + 1;
    if (chunks < cuts && chunks * uncut * kv_heads < cuts)
        cuts = chunks * uncut * kv_heads;
    return uncut * kv_heads + cuts;
}

// Rows of parts that a batch can need: twice its rows (a shared prefix and the
// rest), up to a bound, and those of cut items.
uint64_t part_rows_of(const dm_ctx* c, uint64_t q_tokens, uint32_t q_heads)
{
    const uint64_t rows = 2 * q_tokens * q_heads;
    return (rows < kPartRows ? rows : kPartRows) + kWide * item_target(c);
}

}  // namespace

uint64_t attn_plan_bytes(uint64_t n, uint64_t groups)
{
    return sizeof(PlanHead) + up16(sizeof(Unit) * (n + groups)) + 2 * up16(4 * n) + 2 * up16(4 * groups);
}

hipError_t attn_plan(dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t q_heads,
                     void* plan)
{
    PlanIn a;
    a.b = token_batch(c, b);
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.ratio = q_heads / kv.kv_heads;
    a.target = item_target(c);
    a.part_rows = part_rows_of(c, b.q_tokens, q_heads);
    const PlanView pv = plan_view(plan, b.tables.n, b.groups);
    a.arrived = c->d_status + 48;  // a line of its own
    attn_plan_kernel<<<b.groups ? grid_for(b.tables.n, 1, 2u * c->n_cu) : 1, kPlanThreads, 0, c->stream>>>(
        a, pv, c->d_status);
    return hipGetLastError();
}

hipError_t attn(dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t q_heads,
                const void* plan, uint32_t layer, const void* q, int64_t q_stride, float scale,
                void* out, int64_t out_stride, float* lse)
{
    const uint64_t rows = part_rows_of(c, b.q_tokens, q_heads);
    hipError_t e;
    float* part = static_cast<float*>(scratch_get(c, kSlotPages, rows * (kv.head_dim + 1) * 4, &e));
    if (!part)
        return e;
    AttnIn a;
    a.b = token_batch(c, b);
    a.k = static_cast<const uint16_t*>(kv.k) + (uint64_t)layer * kv.layer_stride;
    a.v = static_cast<const uint16_t*>(kv.v) + (uint64_t)layer * kv.layer_stride;
    a.q = static_cast<const uint16_t*>(q);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.part = part;
    a.part_lse = part + rows * kv.head_dim;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.n_pages = kv.n_pages;
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.ratio = q_heads / kv.kv_heads;
    a.scale2 = scale * 1.44269504088896341f;
    const PlanView pv = plan_view(const_cast<void*>(plan), b.tables.n, b.groups);
    const uint64_t most = most_items(c, b, a.ratio, kv.kv_heads);
    if (most > 0x7FFFFFFFull)
        return hipErrorInvalidValue;
    const uint32_t grid = (uint32_t)most;
    by_type(kv.dtype, kv.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        attn_kernel<T, D><<<grid, kThreads, 0, c->stream>>>(a, pv, rows, c->d_status);
        attn_join_kernel<T, D><<<grid_for(b.q_tokens * q_heads, 1, 8u * c->n_cu), kThreads, 0, c->stream>>>(
            a, pv, rows);
    });
    return hipGetLastError();
}

}  // namespace dm
