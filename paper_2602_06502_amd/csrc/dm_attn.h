// What the passes of attention over KV pages share: the plan in memory, the tiles, and
// the parts of rows.
#pragma once

#include "dm_internal.h"
#include "dm_pages.h"

namespace dm {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr uint32_t kNarrow = 16, kWide = kAttnWide;  // rows of a tile
// Rows of a unit, at most, that has narrow tiles.  (32 sequences of 4,096 keys, 32
// query and 8 key heads of 128: 24 rows 104 us in a wide tile, 114 in two narrow
// ones; 64 rows 112 and 158; 16 rows 103 and 106, 4 rows 100 and 102.  64 sequences of
// 64 to 8,192 keys, 4 rows: 216 narrow, 262 wide.)
constexpr uint32_t kNarrowRows = 16;
constexpr uint32_t kNarrowKeys = 32, kWideKeys = 64;
constexpr uint32_t kChunk = 128;               // keys of a chunk, at least (of the longest: a multiple)
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
    uint32_t wide;  // rows of its wide tiles
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

// Differential attention: KV heads are pairs, their values side by side one value of D
// elements, their keys D / 2 elements each.  A row is a query head and reads the keys
// of its own map, row % 2, of the pair; ratio, kv_heads: of pairs.
struct DiffIn : AttnIn {
    const float* lambda;   // [q_heads / 2]
    const uint16_t* norm;  // [D], or null
    float eps, gain;
};
template <bool PAIR>
using InOf = std::conditional_t<PAIR, DiffIn, AttnIn>;

// Elements of a key's row of one map, and in a page: a page holds a pair's heads one
// after the other, so that place `chunk` (16 bytes) of a joint row is there.
template <int D, bool PAIR>
constexpr int kKeyElems = PAIR ? D / 2 : D;
template <int D, bool PAIR>
__device__ __forceinline__ uint32_t chunk_at(uint32_t chunk, uint32_t shift)
{
    constexpr uint32_t kOne = D / 16;  // chunks of a map's row
    return PAIR ? ((chunk / kOne) * (D / 2) << shift) + chunk % kOne * 8 : chunk * 8;
}

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

// Byte address of a place in LDS.
__device__ __forceinline__ uint32_t lds_address(const uint16_t* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint16_t*)p;
}

// A tile of 32 keys for a wave's 32 rows: s holds S^T (key = (i / 4) * 8 + half
// * 4 + i % 4).  map: of a pair.
template <typename T, int D, bool PAIR = false>
__device__ __forceinline__ v16f scores(const uint16_t* kt,
                                       const typename Vec8<T>::type (&q)[kKeyElems<D, PAIR> / 16],
                                       uint32_t map = 0)
{
    using V = typename Vec8<T>::type;
    const uint32_t row = lane_id() % 32, half = lane_id() / 32;
    v16f s = {};
#pragma unroll
    for (int x = 0; x < kKeyElems<D, PAIR> / 16; x++) {
        const uint32_t chunk = ((PAIR ? map * (D / 16) : 0) + x * 2 + half) ^ k_swizzle<D>(row);
        s = mfma(*reinterpret_cast<const V*>(kt + row * D + chunk * 8), q[x], s);
    }
    return s;
}

// The same from one register of addresses: a row's chunks are x * 2 + half, exchanged by its
// low bits, so chunk x is chunk 0's place with 32 x exchanged in (tiles begin at multiples of
// 512 bytes).  at: of the lane's row and chunk 0 of its map, in bytes.
template <int D, bool PAIR>
__device__ __forceinline__ uint32_t score_place(uint32_t map)
{
    const uint32_t row = lane_id() % 32, half = lane_id() / 32;
    return (row * D + (((PAIR ? map * (D / 16) : 0) + half) ^ k_swizzle<D>(row)) * 8) * 2;
}
// The scores of 64 keys so, a few reads ahead of the matrix instructions (left to itself the
// compiler, short of registers, waits for every read where it is used).
constexpr int kAhead = 2;
template <typename T, int D, bool PAIR>
__device__ __forceinline__ void scores_ahead(uint32_t at, const typename Vec8<T>::type (&q)[kKeyElems<D, PAIR> / 16],
                                             v16f (&s)[2])
{
    using V = typename Vec8<T>::type;
    constexpr int kSteps = kKeyElems<D, PAIR> / 8;
    V f[kAhead + 1];
    auto read = [&](int n) {
        f[n % (kAhead + 1)] = *(const __attribute__((address_space(3))) V*)(uintptr_t)(
            (at ^ (n / 2 * 32)) + n % 2 * (32 * D * 2));
    };
    s[0] = s[1] = v16f{};
#pragma unroll
    for (int n = 0; n < kAhead; n++)
        read(n);
#pragma unroll
    for (int n = 0; n < kSteps; n++) {
        if (n + kAhead < kSteps)
            read(n + kAhead);
        s[n % 2] = mfma(f[n % (kAhead + 1)], q[n / 2], s[n % 2]);
        __builtin_amdgcn_sched_barrier(0);
    }
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

// The same from one register of addresses (as score_place): block db's place is block 0's with
// 64 db exchanged in.
template <int D>
__device__ __forceinline__ uint32_t value_place()
{
    const uint32_t l = lane_id(), row = l / 32 * 4 + l % 16 / 4, c = l / 16 % 2 * 2 + l % 4 / 2;
    return (row * D + (c ^ v_swizzle<D>(row)) * 8 + l % 2 * 4) * 2;
}
template <typename T, int D>
__device__ __forceinline__ typename Vec8<T>::type values_at(uint32_t at, uint32_t key0, uint32_t db)
{
    const uint32_t here = (at ^ (db * 64)) + key0 * D * 2;
    const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(uintptr_t)here);
    const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(uintptr_t)(here + 8 * D * 2));
    typedef short v8s __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(typename Vec8<T>::type, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
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

// The running maximum over NB tiles of 32 keys, in front of their weights: what is
// taken off their scaled scores.  limit: the keys that the lane's row sees (absolute),
// key0: the tiles' first; masked: some row does not see all of them.
template <typename T, int D, int NB>
__device__ __forceinline__ float settle(Row<D>& r, v16f (&s)[NB], uint32_t key0, uint32_t limit, bool masked,
                                        float scale2)
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
    return r.m == -INFINITY ? 0.0f : r.m * (r.far ? 0.0f : scale2) - kRaise<T>;
}

// The running softmax of NB tiles of 32 keys: the tiles' weights in T.  beside(): what
// can be done meanwhile, when s has been read (it may be written anew).
template <typename T, int D, int NB, typename Beside>
__device__ __forceinline__ void weights(Row<D>& r, v16f (&s)[NB], typename Vec8<T>::type (&p)[NB][2],
                                        uint32_t key0, uint32_t limit, bool masked, float scale2,
                                        Beside&& beside)
{
    const float base = settle<T, D, NB>(r, s, key0, limit, masked, scale2);
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

// Both for two tiles, the second one's weights taken beside the first one's products, a few
// reads ahead of these.
template <typename T, int D>
__device__ __forceinline__ void weigh_and_add(Row<D>& r, v16f (&s)[2], uint32_t vt, uint32_t key0,
                                              uint32_t limit, bool masked, float scale2)
{
    using V = typename Vec8<T>::type;
    constexpr int kBlocks = D / 32, kSteps = 4 * kBlocks;
    const float base = settle<T, D, 2>(r, s, key0, limit, masked, scale2);
    V p[2][2], f[kAhead + 2];
    float sum = 0;
    auto weigh = [&](int b, int i) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale2, -base));
        sum += w;
        p[b][i / 8][i % 8] = (T)w;
    };
    auto read = [&](int n) {
        f[n % (kAhead + 2)] = values_at<T, D>(vt, n / kBlocks * 16, n % kBlocks);
    };
#pragma unroll
    for (int n = 0; n < kAhead; n++)
        read(n);
#pragma unroll
    for (int i = 0; i < 16; i++)
        weigh(0, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < kSteps; n += 2) {
#pragma unroll
        for (int k = n; k < n + 2; k++) {
            if (k + kAhead < kSteps)
                read(k + kAhead);
            r.o[k % kBlocks] = mfma(f[k % (kAhead + 2)], p[k / kBlocks / 2][k / kBlocks % 2], r.o[k % kBlocks]);
        }
        if (n < kSteps / 2) {
            constexpr int kPer = 64 / kSteps;  // two steps' share of 16
#pragma unroll
            for (int i = 0; i < kPer; i++)
                weigh(1, n / 2 * kPer + i);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    r.l += sum;
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

// Is the plan one of this batch?  (Without short cuts: the head's words by one wait, not one
// after the other, which a single token's pass would notice.)
__device__ __forceinline__ bool plan_of(const PlanHead& h, const TokenBatch& b, uint32_t q_heads, uint32_t kv_heads,
                                        uint32_t head_dim)
{
    const uint64_t entries = (uint64_t)(h.entries ^ b.entries);
    return ((h.n ^ b.n) | (h.groups ^ b.groups) | (h.q_tokens ^ b.q_tokens) | (h.q_heads ^ q_heads) | (h.kv_heads ^ kv_heads) |
            (h.shift ^ b.shift) | (h.head_dim ^ head_dim) | (uint32_t)entries | (uint32_t)(entries >> 32)) == 0;
}

// Is the plan this call's, of at most `items` items?  (A batch whose q_off is out of
// order can have more than the call has workgroups.)
__device__ __forceinline__ bool plan_fits(const PlanHead& h, const AttnIn& a, uint64_t part_rows,
                                          uint32_t head_dim, uint32_t wide, uint32_t items)
{
    return plan_of(h, a.b, a.q_heads, a.kv_heads, head_dim) & (h.wide == wide) & (h.part_rows <= part_rows) &
           (h.items <= items);
}

// The unit of this workgroup's item; false: none, or the plan is another batch's
// (reported).  What the plan holds is read beside its head as far as any plan
// reaches, and beyond that only once the head has been looked at: the plan of a
// batch of fewer sequences is a smaller one.
__device__ __forceinline__ bool item_unit(const AttnIn& a, const PlanView& pv, uint32_t units,
                                          uint64_t part_rows, uint32_t head_dim, uint32_t wide, uint32_t* status,
                                          Unit& u)
{
    const PlanHead& ph = *pv.head;
    const bool early = units <= kEarlyUnits;
    uint32_t ui = early ? find_unit(pv.item0, units, blockIdx.x) : 0;
    if (!plan_fits(ph, a, part_rows, head_dim, wide, gridDim.x)) {
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
template <typename T, int D, bool PAIR = false>
__device__ __forceinline__ void load_query(const AttnIn& a, const Tile& t, uint32_t row,
                                           typename Vec8<T>::type (&q)[kKeyElems<D, PAIR> / 16])
{
    constexpr int kElems = kKeyElems<D, PAIR>;
    const uint32_t r = row < t.last ? row : t.last;
    const uint16_t* at = a.q + (uint64_t)(t.u.tok0 + r / a.ratio) * a.q_stride +
                         (uint64_t)(t.h * a.ratio + r % a.ratio) * kElems + lane_id() / 32 * 8;
#pragma unroll
    for (int k = 0; k < kElems / 16; k++)
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
template <typename T, int D, bool PAIR = false>
struct Share {
    static constexpr int kElems = kKeyElems<D, PAIR>;
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
          lane_at(r0 % (halves ? 4 : 8) * kElems + chunk_at<D, PAIR>(ch, a.b.shift)),
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
            return (p < n_pages ? p : 0) * page_size + head_at + ((key + i * kStep + g * 4) & mask) * kElems;
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
    // keys or values alone, by way of k
    __device__ __forceinline__ void fetch_one(const uint16_t* pages, uint32_t key, bool& bad)
    {
        static_assert(kGroups == 1, "a load's rows are in one page");
        const uint32_t mask = (1u << shift) - 1;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const uint32_t p = page[i];
            bad |= p >= n_pages;
            const uint64_t at = (p < n_pages ? p : 0) * page_size + head_at + ((key + i * kStep) & mask) * kElems;
            k[i] = *reinterpret_cast<const v4u32*>(pages + at + lane_at);
        }
    }
    template <bool VALUES>
    __device__ __forceinline__ bool stage_one(uint16_t* to, uint32_t key, bool ask)
    {
        bool odd = false;
        if (VALUES && ask) {
            const uint32_t have = key1 - key;
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                if (r0 + i * kStep >= have)
                    k[i] = v4u32{};
                odd |= not_finite<T>(k[i]);
            }
        }
        const uint32_t row = here();
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const uint32_t r = row + i * kStep;
            *reinterpret_cast<v4u32*>(to + r * D + (ch ^ (VALUES ? v_swizzle<D, false>(r) : k_swizzle<D>(r))) * 8) = k[i];
        }
        return odd;
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

// 1 / sqrt(mean square + eps) of a differential row, from the sum of its D squares;
// nothing has a norm of nothing, also where eps is 0.
template <int D>
__device__ __forceinline__ float norm_of(float ss, float eps)
{
    return ss == 0 ? 0.0f : rsqrtf(ss * (1.0f / D) + eps);
}

// Four elements of a differential row, d on, times `by` and the norm's weights.  x: the
// first of the pair's query heads.
template <typename T>
__device__ __forceinline__ void write_normed(const DiffIn& a, uint32_t token, uint32_t x, int elems, uint32_t d, v4f y,
                                             float by)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    v4t w = {1, 1, 1, 1}, z;
    if (a.norm)
        w = *reinterpret_cast<const v4t*>(a.norm + d);
#pragma unroll
    for (int i = 0; i < 4; i++)
        z[i] = (T)(y[i] * by * (float)w[i]);
    *reinterpret_cast<v4t*>(a.out + token * a.out_stride + (uint64_t)x * elems + d) = z;
}

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
// 16) * 4 + i, and of O^T the elements d = block * 16 + (lane / 16) * 4 + i.  PAIR: the
// rows of a tile are of both maps in turn, so each takes the products with both maps'
// keys and keeps its own: no more instructions than one product over D.
// SPLIT: a wave's part of LDS holds a tile's keys, then its values, each on its way while
// the other is worked on: half the LDS and half the registers a wave, for twice the waves.
template <typename T, int D, int WAVES, bool PAIR = false, bool SPLIT = false>
__device__ __forceinline__ void narrow_tile(const InOf<PAIR>& a, const Tile& t, uint16_t* lds, Joined<WAVES>& joined,
                                            bool& bad)
{
    constexpr int kElems = kKeyElems<D, PAIR>;
    using V = typename Vec8<T>::type;
    constexpr uint32_t kTurn = WAVES * kNarrowKeys;
    constexpr int kBlocks = D / 16;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t lane = lane_id(), row16 = lane % 16, g = lane / 16;
    const uint32_t row = t.first + row16, in_tile = row < t.last ? row : t.last;
    V q[kElems / 32];
    {
        const uint16_t* at = a.q + (uint64_t)(t.u.tok0 + in_tile / a.ratio) * a.q_stride +
                             (uint64_t)(t.h * a.ratio + in_tile % a.ratio) * kElems + g * 8;
#pragma unroll
        for (int k = 0; k < kElems / 32; k++)
            q[k] = *reinterpret_cast<const V*>(at + k * 32);
    }
    const uint32_t limit = sees(t.u, a.ratio, in_tile), end = limit < t.key1 ? limit : t.key1;
    v4f o[kBlocks];
    float m = -INFINITY, l = 0;
    bool far = false;
#pragma unroll
    for (int d = 0; d < kBlocks; d++)
        o[d] = v4f{};
    uint16_t* kt = lds + wave * (SPLIT ? 1 : 2) * kNarrowKeys * D;
    uint16_t* vt = SPLIT ? kt : kt + kNarrowKeys * D;
    // weights, and what their rounding has left out: the matrix unit has time for both
    // (4% busy with the weights alone, in 64 rows on up to 8,192 keys)
    V p, rest;
    // a lane's number: SPLIT works places in LDS out anew for each tile, of which it has no
    // registers to keep (kept, 15 of them were spilled, and their reloads waited for the
    // pages: 297 us instead of 225 for 64 rows on up to 8,192 keys, heads of 128)
    auto here = [](uint32_t x) {
        if (SPLIT)
            asm volatile("" : "+v"(x));
        return x;
    };
    // scores and weights of the tile in LDS
    auto weigh = [&](uint32_t key, bool masked) {
        v4f s[2];
        const uint32_t at16 = here(row16);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            s[h] = v4f{};
            const uint32_t r = h * 16 + at16;
#pragma unroll
            for (int k = 0; k < kElems / 32; k++)
                s[h] = mfma(*reinterpret_cast<const V*>(kt + r * D + ((k * 4 + g) ^ k_swizzle<D>(r)) * 8), q[k],
                            s[h]);
            if constexpr (PAIR) {
                v4f other = {};
#pragma unroll
                for (int k = 0; k < kElems / 32; k++)
                    other = mfma(*reinterpret_cast<const V*>(
                                     kt + r * D + ((D / 16 + k * 4 + g) ^ k_swizzle<D>(r)) * 8),
                                 q[k], other);
#pragma unroll
                for (int i = 0; i < 4; i++)
                    s[h][i] = row16 % 2 ? other[i] : s[h][i];
            }
            if (SPLIT)
                __builtin_amdgcn_sched_barrier(0);  // (not all of a tile's reads at once, for which there is no room)
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
        Share<T, D, PAIR> x(a, t);
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
        // O^T += V^T P^T, keys in the order of the lane's weights
        auto add = [&] {
            const uint32_t own = here(lane), r = own / 16 * 4 + own % 16 / 4;
#pragma unroll
            for (int d = 0; d < kBlocks; d++) {
                const uint32_t c = d * 2 + (own % 4) / 2, e = (own % 2) * 4;
                const v4s v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_v4s*)(vt + r * D + (c ^ v_swizzle<D, false>(r)) * 8 + e));
                const v4s v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_v4s*)(vt + (r + 16) * D + (c ^ v_swizzle<D, false>(r + 16)) * 8 + e));
                typedef short v8s __attribute__((ext_vector_type(8)));
                const v8s f = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
                o[d] = mfma(__builtin_bit_cast(V, f), p, o[d]);
                o[d] = mfma(__builtin_bit_cast(V, f), rest, o[d]);
            }
        };
        // as add_odd_values()
        auto add_odd = [&](uint32_t key) {
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
        };
        x.find(key);
        if constexpr (SPLIT) {
            auto in_order = [] {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            };
            x.fetch_one(a.k, key, bad);
            for (; key < t.key1; key += kTurn) {
                const bool all = key + kNarrowKeys <= t.see_first && key + kNarrowKeys <= t.key1;
                in_order();
                x.template stage_one<false>(kt, key, false);
                in_order();
                x.fetch_one(a.v, key, bad);
                if (key + kTurn < t.key1)
                    x.find(key + kTurn);
                weigh(key, !all);
                in_order();
                const bool strange = x.template stage_one<true>(vt, key, !all);
                in_order();
                const bool odd_ones = !all && __any(strange);
                if (odd_ones)
                    add_odd(key);  // (with nothing on its way: what this needs would push the query out)
                if (key + kTurn < t.key1)
                    x.fetch_one(a.k, key + kTurn, bad);
                if (!odd_ones)
                    add();
            }
        } else {
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
                add();
            }
            while (key < t.key1) {
                weigh(key, true);
                add_odd(key);
                key += kTurn;
                if (key < t.key1) {
                    x.find(key);
                    x.fetch(a, key, bad);
                    stage(key);
                }
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
    auto block = [&](uint32_t d) {
        v4f x = {};
        for (int w = 0; w < WAVES; w++)
            x += sum[(w * kBlocks + d) * kWave + lane];
        for (int k = 0; k < 4; k++)
            x[k] = seen ? x[k] * inv : 0.0f;
        return x;
    };
    if (!PAIR || (t.u.flags & kUnitParts)) {
        for (uint32_t d = wave; d < kBlocks; d += WAVES) {
            const v4f x = block(d);
            if (row <= t.last)
                write_four<T, D>(a, t, row, d * 16 + g * 4, x);
        }
    }
    if constexpr (PAIR) {
        if (!(t.u.flags & kUnitParts)) {
            // the maps' rows are in neighbouring lanes
            constexpr int kMine = kBlocks / WAVES;
            const uint32_t x = t.h * a.ratio + in_tile % a.ratio;
            const float lambda = a.lambda[x / 2];
            v4f y[kMine];
            float ss = 0;
#pragma unroll
            for (int k = 0; k < kMine; k++) {
                y[k] = block(wave + k * WAVES);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    y[k][i] = __builtin_fmaf(-lambda, __shfl_xor(y[k][i], 1), y[k][i]);
                    ss = __builtin_fmaf(y[k][i], y[k][i], ss);
                }
            }
            float by = a.gain;
            if (a.norm) {
                ss += __shfl_xor(ss, 16);
                ss += __shfl_xor(ss, 32);
                __syncthreads();  // (the first use of joined.m is over)
                if (g == 0)
                    joined.m[wave][row16] = ss;
                __syncthreads();
                ss = 0;
                for (int w = 0; w < WAVES; w++)
                    ss += joined.m[w][row16];
                by *= norm_of<D>(ss, a.eps);
            }
            if (row16 % 2 == 0 && row <= t.last)
#pragma unroll
                for (int k = 0; k < kMine; k++) {
                    const uint32_t d = (wave + k * WAVES) * 16 + g * 4;
                    write_normed<T>(a, t.u.tok0 + row / a.ratio, x, kElems, d, y[k], by);
                }
        }
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

// A thread's share of wide tiles: LDS chunk threadIdx.x + i * 256, that is row r0 +
// i * kStep, place `ch` of the row.  What a lane adds to its rows' address does not
// change from tile to tile.
template <typename T, int D, bool PAIR = false, int WAVES = kWaves>
struct Sender {
    static constexpr int kThreads = WAVES * kWave;
    static constexpr int kElems = kKeyElems<D, PAIR>;
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
          wave(wave_), halves(kGroups == 2 && a.b.shift == 2), lane_row(r0 % kWaveRows % (halves ? 4 : 8) * kElems)
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
                       ((key + wave * kWaveRows + i * kStep + g * 4) & mask) * kElems;
            };
            const uint32_t r = r0 + i * kStep;
            const uint32_t c = ch ^ (values ? v_swizzle<D>(r) : k_swizzle<D>(r));
            const uint32_t lane_at = (lane_row + chunk_at<D, PAIR>(c, shift)) * 2, lds_at = at + i * kThreads * 16;
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
// PAIR: a wave's rows are of one map, two waves take the maps of the same 32 pairs of
// rows; each has products with its own map's keys only, both with all values.
// BESIDE: the next tile's scores are taken beside this one's weights.  Without, a wave
// has registers to spare, and another wave of its SIMD the matrix unit meanwhile.
template <typename T, int D, bool PAIR = false, int WAVES = kWaves, bool BESIDE = true>
__device__ __forceinline__ void wide_tile(const InOf<PAIR>& a, const Tile& t, uint16_t* lds, uint32_t* odd_tile,
                                          bool& bad)
{
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t map = PAIR ? wave % 2 : 0;
    // the wave's first row, and from one to the next
    const uint32_t w0 = t.first + (PAIR ? wave / 2 * 64 + map : wave * 32), step = PAIR ? 2 : 1;
    const uint32_t row = w0 + lane_id() % 32 * step;
    typename Vec8<T>::type q[kKeyElems<D, PAIR> / 16], p[2][2];
    load_query<T, D, PAIR>(a, t, row, q);
    const uint32_t limit = sees(t.u, a.ratio, row < t.last ? row : t.last);
    const uint32_t end = limit < t.key1 ? limit : t.key1;
    Row<D> r;
    clear<D>(r);
    // keys that the wave's first and last rows see
    const uint32_t w1 = w0 + 31 * step < t.last ? w0 + 31 * step : t.last;
    const uint32_t wave_first = w0 <= t.last ? sees(t.u, a.ratio, w0) : 0;
    const uint32_t wave_last = w0 <= t.last ? sees(t.u, a.ratio, w1) : 0;
    auto masked = [&](uint32_t key, uint32_t first) { return key + kWideKeys > first || key + kWideKeys > t.key1; };
    constexpr uint32_t kTile = kWideKeys * D;
    uint16_t* vts = lds + 2 * kTile;  // two tiles of keys, then two of values
    if (t.key0 < t.key1) {
        using Send = Sender<T, D, PAIR, WAVES>;
        const Send x(a, t, wave);
        const uint32_t place = score_place<D, PAIR>(map), v_place = value_place<D>();
        uint32_t p1[Send::kPages], p2[Send::kPages];  // pages of the next tile, and the one after
        if (threadIdx.x == 0)
            *odd_tile = 0;
        x.find(t.key0, p2);
        x.send(x.k, false, t.key0, p2, lds, bad);
        x.send(x.v, true, t.key0, p2, vts, bad);
        if (t.key0 + kWideKeys < t.key1) {
            x.find(t.key0 + kWideKeys, p1);
            if (BESIDE)
                x.send(x.k, false, t.key0 + kWideKeys, p1, lds + kTile, bad);
        }
        if (BESIDE && t.key0 + 2 * kWideKeys < t.key1)
            x.find(t.key0 + 2 * kWideKeys, p2);
        wait_sent();
        __syncthreads();
        v16f s[2];
        if (BESIDE) {
            s[0] = scores<T, D, PAIR>(lds, q, map);
            s[1] = scores<T, D, PAIR>(lds + 32 * D, q, map);
            __syncthreads();  // the third tile's keys go where the first's are
        } else {
            // the query is here: the compiler, which does not count the sends, would wait for
            // its reads in every tile and so for the sends
#pragma unroll
            for (int i = 0; i < kKeyElems<D, PAIR> / 16; i++)
                asm volatile("" : "+v"(q[i]));
        }
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
            if constexpr (!BESIDE) {
                if (key1 < t.key1) {
                    x.send(x.k, false, key1, p1, lds + (buf ^ 1) * kTile, bad);
                    x.send(x.v, true, key1, p1, vts + (buf ^ 1) * kTile, bad);
                }
                if (key2 < t.key1)
                    x.find(key2, p1);
                if (key < wave_last) {
                    const uint32_t at = lds_address(lds + buf * kTile) + place;
                    v16f z[2];
                    scores_ahead<T, D, PAIR>(at, q, z);
                    weigh_and_add<T, D>(r, z, lds_address(vts + buf * kTile) + v_place, key, end, masked(key, wave_first), a.scale2);
                }
                key = key1;
                buf ^= 1;
                if (key >= t.key1)
                    break;
                wait_sent();
                __syncthreads();
                continue;
            }
            if (key2 < t.key1)
                x.send(x.k, false, key2, p2, lds + buf * kTile, bad);
            if (key1 < t.key1) {
                x.send(x.v, true, key1, p1, vts + (buf ^ 1) * kTile, bad);
#pragma unroll
                for (int i = 0; i < Send::kPages; i++)
                    p1[i] = p2[i];
            }
            if (key2 + kWideKeys < t.key1)
                x.find(key2 + kWideKeys, p2);
            if (key < wave_last) {
                weights<T, D, 2>(r, s, p, key, end, masked(key, wave_first), a.scale2, [&] {
                    // (of the last tile: of what is there, and not used)
                    s[0] = scores<T, D, PAIR>(lds + (buf ^ 1) * kTile, q, map);
                    s[1] = scores<T, D, PAIR>(lds + (buf ^ 1) * kTile + 32 * D, q, map);
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
        while ((BESIDE || odd) && key < t.key1) {  // rare: values that are not finite
            if (!BESIDE) {  // (its own query, so that nothing is kept for this)
                typename Vec8<T>::type own[kKeyElems<D, PAIR> / 16];
                load_query<T, D, PAIR>(a, t, row, own);
                s[0] = scores<T, D, PAIR>(lds + buf * kTile, own, map);
                s[1] = scores<T, D, PAIR>(lds + buf * kTile + 32 * D, own, map);
            }
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
            if (BESIDE) {
                s[0] = scores<T, D, PAIR>(lds + buf * kTile, q, map);
                s[1] = scores<T, D, PAIR>(lds + buf * kTile + 32 * D, q, map);
            }
        }
    }
    const float l = r.l + __shfl_xor(r.l, 32);
    if (!PAIR || (t.u.flags & kUnitParts))
        write_row<T, D>(a, t.u, t.h, row, t.last + 1, t.chunk, r, l, t.rows);
    if constexpr (PAIR) {
        if (t.u.flags & kUnitParts)
            return;
        // the second map's rows by way of LDS to the first's wave
        const uint32_t half = lane_id() / 32;
        const uint32_t in_tile = row < t.last ? row : t.last, token = t.u.tok0 + in_tile / a.ratio;
        const uint32_t x = t.h * a.ratio + in_tile % a.ratio;
        const bool seen = l > 0 || l != l;
        const float inv = seen ? 1.0f / l : 0.0f;
        if (half == 0 && a.lse && row <= t.last)
            a.lse[(uint64_t)token * a.q_heads + x] = seen ? lse_of<T>(r.m, l, a.scale2) : -INFINITY;
        float* far = reinterpret_cast<float*>(lds) + wave / 2 * (D / 2 * kWave) + lane_id();
        __syncthreads();
        if (map)
#pragma unroll
            for (int d = 0; d < D / 32; d++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    far[(d * 16 + i) * kWave] = seen ? r.o[d][i] * inv : 0.0f;
        __syncthreads();
        if (map)
            return;
        const float lambda = a.lambda[x / 2];
        float ss = 0;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float y = __builtin_fmaf(-lambda, far[(d * 16 + i) * kWave], seen ? r.o[d][i] * inv : 0.0f);
                ss = __builtin_fmaf(y, y, ss);
                r.o[d][i] = y;
            }
        const float by = a.norm ? a.gain * norm_of<D>(ss + __shfl_xor(ss, 32), a.eps) : a.gain;
        if (row <= t.last)
#pragma unroll
            for (int d = 0; d < D / 32; d++)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    write_normed<T>(a, token, x, D / 2, d * 32 + i * 2 + half * 4,
                                    v4f{r.o[d][i], r.o[d][i + 1], r.o[d][i + 2], r.o[d][i + 3]}, by);
    }
}
// Waves of a narrow tile that is not cut (as many as have room in LDS).
template <int D>
constexpr int kSmallWaves = D == 256 ? 4 : 8;

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
template <typename T, int D, bool PAIR = false>
__device__ __forceinline__ void join_quarters(const InOf<PAIR>& a, const PlanView& pv, uint64_t y0, uint64_t y1)
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
        if constexpr (PAIR) {
            // the maps' rows are in neighbouring quarters, in the same loop or in none
            const float lambda = a.lambda[x / 2];
            float ss = 0;
#pragma unroll
            for (int c = 0; c < kPer; c++) {
                v[c] *= inv;
                v[c] = __builtin_fmaf(-lambda, __shfl_xor(v[c], 16), v[c]);
                ss = __builtin_fmaf(v[c], v[c], ss);
            }
            float by = a.gain;
            if (a.norm) {
#pragma unroll
                for (int o = 1; o < 16; o *= 2)
                    ss += __shfl_xor(ss, o);
                by *= norm_of<D>(ss, a.eps);
            }
            if (x % 2 == 0)
#pragma unroll
                for (int c = 0; c < kPer; c += 4)
                    write_normed<T>(a, t, x, D / 2, d + c, v4f{v[c], v[c + 1], v[c + 2], v[c + 3]}, by);
        } else {
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
        }
        if (d == 0 && a.lse)
            a.lse[(uint64_t)t * a.q_heads + x] = seen ? lse_of<T>(m, total, a.scale2) : -INFINITY;
    }
}

// Is a batch small: no unit has more rows than a narrow tile, and no more keys than
// attn_small_kernel is the faster on?
inline bool small(const dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t ratio)
{
    const uint64_t keys = kv.head_dim == 64 ? 1024 : kv.head_dim == 128 ? 768 : 256;
    return b.groups == 0 && b.q_tokens * ratio <= kNarrowRows && b.tables.entries * c->cfg.block_size <= keys;
}

// Items wanted: three for every two places of a workgroup (two a compute unit).
// (us with one for each place, three for two, two and three: 64 decode rows of up to
// 8,192 keys 227, 217, 216 and 216; 256 rows on 8 shared prefixes 179, 178, 181 and 185; 8
// tails on 2 prefixes 753, 774, 764 and 755.)
inline uint64_t item_target(const dm_ctx* c) { return 3ull * c->n_cu; }

// Items that a plan can have: the tiles of its units, and what cuts add: at most
// the items wanted, and no more than the table entries' keys are chunks for each
// tile.
inline uint64_t most_items(const dm_ctx* c, const dm_token_batch& b, uint32_t ratio, uint32_t kv_heads, uint32_t wide)
{
    const uint64_t rows = b.q_tokens * ratio;
    auto tiles = [&](uint64_t units) { return rows / wide + units; };
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
inline uint64_t part_rows_of(const dm_ctx* c, const dm_token_batch& b, uint32_t q_heads)
{
    const uint64_t rows = b.groups ? 2 * b.q_tokens * q_heads : 0;
    return (rows < kPartRows ? rows : kPartRows) + kWide * item_target(c);
}

}  // namespace
}  // namespace dm
