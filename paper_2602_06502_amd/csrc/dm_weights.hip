// The weight that each cached key has collected: for KV head h and token i of a sequence
//   w[h][i] = decay * prev[h][i] + sum over its new tokens t that see i, and over the query
//             heads x that read h, of exp(scale q_x,t . k_h,i - lse_x,t).
//
// Keys stay, queries pass: a wave has 64 neighbouring keys of one head in registers, as the
// right operand of S = Q K^T on 16x16x32 matrix instructions, and takes 16 rows (token,
// query head) at a time; a lane then holds scores of one key, so that their weights' sum over
// the rows is a sum over its own registers and one over four lanes at the end.  Nothing is added by two waves, so the order of
// every sum is fixed.  Blocks of 64 keys follow the tables' entries, not the sequences: a
// lane's page is known without knowing whose it is, and a block may hold the end of one
// sequence and the beginnings of others, which take their turns.
//
// Where sequences have many rows, a second kernel before the first has a workgroup for 256
// keys of a head and a stretch of rows, which pass through LDS once for its four waves; it
// leaves its sums, and the first kernel adds a key's up.
//
// The pages that a run shares (as its plan has found them) are read for four of its sequences
// at once, each with its own sums; a few rows each, several of them have one product.
//
// Bound by reading keys and carried weights where rows are few (64 tokens behind 64 to 8,192
// keys, 8 heads of 128: 107 us, 4.4 TB/s; 128 tokens on 8 shared prefixes, heads of 64: 96), by the
// exponentials beside the products where they are many (2 prompts of 7,000 to 8,192 tokens: 609
// to 625 us, 835 to 857 TFLOP/s).
#include "dm_attn.h"

namespace dm {
namespace {

constexpr uint32_t kBlockKeys = 64;
// Rows of a sequence, at most, that the blocks of 64 keys take themselves where there are
// tall blocks too.
constexpr uint32_t kFewRows = 64;
constexpr uint32_t kTallKeys = kWaves * kBlockKeys, kTallRows = 64;  // keys of a tall block, rows in LDS

struct WeightsIn {
    TokenBatch b;
    const uint16_t* k;  // the layer's pages
    const uint16_t* q;
    const float* lse;
    float* w;
    const float* prev;
    const int64_t* prev_off;
    const int32_t* src;
    const int64_t* keep;
    int64_t q_stride, w_stride, prev_stride, prev_room;
    uint32_t prev_n, n_pages, q_heads, kv_heads, ratio, last, paired;
    uint32_t plan_heads, plan_dim;  // the plan's
    float scale2, decay;
    // tall blocks: stretches of rows (0: there are none), their rows, and their sums
    // [parts][kv_heads][slots]
    uint32_t parts, part_rows;
    float* part;
    int64_t slots;
    struct SeqRow* rows;  // with runs: of each sequence
    uint32_t* order;   // [n] of each run, from its first sequence on: those that see its prefix
};

// The first row of a sequence that counts.
__device__ __forceinline__ uint32_t first_row(const WeightsIn& a, const SeqView& v)
{
    return (a.last && a.last < v.ntok ? v.ntok - a.last : 0) * a.ratio;
}
__device__ __forceinline__ bool few(const WeightsIn& a, const SeqView& v)
{
    return v.ntok * a.ratio - first_row(a, v) <= kFewRows;
}
// Rows of stretch p that see something of a block whose first key is the sequence's i0-th.
struct Stretch {
    uint32_t row0, row1;
};
__device__ __forceinline__ Stretch stretch_of(const WeightsIn& a, const SeqView& v, int64_t i0, bool causal, uint32_t p)
{
    uint32_t row0 = first_row(a, v), row1 = v.ntok * a.ratio;
    const uint64_t s0 = row0 + (uint64_t)p * a.part_rows, s1 = s0 + a.part_rows;
    if (causal && i0 > v.pos0 + row0 / a.ratio)
        row0 = (uint32_t)(i0 - v.pos0) * a.ratio;
    return Stretch{row0 > s0 ? row0 : (uint32_t)s0, row1 < s1 ? row1 : (uint32_t)s1};
}

// What is in LDS of rows: their log-sum-exps (in powers of two), and the last key that each
// sees.
template <int ROWS>
struct WordsOf {
    float lse[ROWS];
    int32_t sees[ROWS];
};

// A sum that keeps what its additions round away: tens of thousands of weights, most of
// them light, would leave 2^-18 of it (two prompts of 7,000 to 8,192 tokens: 2.4e-6
// relative of 64 bits, so 1e-7).
struct LongSum {
    float sum = 0, lost = 0;
    __device__ __forceinline__ void add(float x)
    {
        const float y = x - lost, t = sum + y;
        lost = (t - sum) - y;
        sum = t;
    }
};

// What is known of a sequence, a lane each for 64 neighbouring ones, and then of one by all
// lanes: its new tokens, its tokens, where they are (`at`), where what it carries is (`old`,
// of its first `keep` tokens), and its tokens that are its run's.
struct Known {
    uint32_t tok0, ntok, len, keep, own0;
    int64_t at, old;
};
template <bool RUNS>
__device__ __forceinline__ Known known_of(const TokenBatch& b, const PlanView& pv, uint32_t s, bool there, bool& bad)
{
    Known x{};
    if (!there)
        return x;
    const SeqView v = sequence_view(b, s);
    bad |= v.bad;
    x.tok0 = v.tok0;
    x.ntok = v.bad ? 0 : v.ntok;
    x.len = (uint32_t)v.len;
    x.at = b.off[s] << b.shift;
    if (RUNS) {
        const uint32_t g = pv.run[s];
        if (g < b.groups)
            x.own0 = x.ntok && x.len ? pv.unit[b.groups + s].key0 : 0;
    }
    return x;
}
// What it carries.
__device__ __forceinline__ void add_carried(const WeightsIn& a, uint32_t s, bool there, Known& x, bool& bad)
{
    if (!a.prev || !there)
        return;
    if (!a.prev_off) {
        x.old = x.at;
        x.keep = x.len > x.ntok ? x.len - x.ntok : 0;
    } else {
        const int64_t keep = a.keep[s];
        x.keep = keep < 0 ? 0 : keep < (int64_t)x.len ? (uint32_t)keep : x.len;
        if (x.keep) {
            const uint32_t src = (uint32_t)a.src[s];
            x.old = src < a.prev_n ? a.prev_off[src] << a.b.shift : -1;
            if (x.old < 0 || x.old + x.keep > a.prev_room) {
                bad = true;
                x.keep = 0;
            }
        }
    }
}
// What a batch with runs has of each sequence, laid out by a kernel of its own (4 us): a wave of
// the others then finds what it has to do in two reads, not in eight that wait for one another
// (128 sequences on 8 prefixes 99 to 88 us, 16 on 2 24 to 20, 4 on one 13 and 13).
constexpr uint32_t kShared = 4;  // sequences of a run that read its keys at once
struct alignas(16) SeqRow {
    Known x;
    // if it sees its run's prefix: the kShared neighbours among those that do, it among them; how
    // many they are, and from bit 8 on which of them it is
    uint32_t many, member[kShared];
};
static_assert(sizeof(SeqRow) == 64);

// A workgroup for 256 sequences, then one for each run.
__global__ __launch_bounds__(kThreads) void weights_rows_kernel(WeightsIn a, const PlanView pv, uint32_t chunks, uint32_t* status)
{
    const TokenBatch& b = a.b;
    __shared__ uint32_t counts[kWaves], order[kThreads];
    const uint32_t tid = threadIdx.x, wave = tid / kWave, lane = lane_id();
    if (!plan_of(*pv.head, b, a.q_heads, a.plan_heads, a.plan_dim))
        return;  // (the other kernel reports it, and reads nothing of these)
    if (blockIdx.x < chunks) {
        const uint32_t s = blockIdx.x * kThreads + tid;
        bool bad = false;
        Known x = known_of<true>(b, pv, s, s < b.n, bad);
        add_carried(a, s, s < b.n, x, bad);
        if (s < b.n)
            a.rows[s].x = x;
        if (bad)
            atomicOr(status, kErrInval);
        return;
    }
    const uint32_t g = blockIdx.x - chunks;
    const int64_t g0 = b.group_off[g], g1 = b.group_off[g + 1];
    if (g0 < 0 || g1 < g0 || g1 > (int64_t)b.n)
        return;
    // (as known_of has it)
    auto sees = [&](uint32_t m) {
        const Unit& u = pv.unit[b.groups + m];
        return u.ntok && u.key0 && u.key1 && pv.run[m] == g;
    };
    // ranks of those that see the prefix, for their order, then by it their neighbours; of a run
    // that the workgroup sees at once in one pass, the order in LDS
    const bool at_once = g1 - g0 <= kThreads;
    uint32_t* list = at_once ? order : a.order + g0;
    uint32_t total = 0;
    auto each = [&](auto&& f) {  // f(sequence, does it see the prefix, how many before it do)
        uint32_t seen = 0;
        for (uint32_t m0 = (uint32_t)g0; m0 < (uint32_t)g1; m0 += kThreads) {
            const uint32_t m = m0 + tid;
            const bool in = m < (uint32_t)g1 && sees(m);
            const uint64_t those = ballot(in);
            __syncthreads();
            if (lane == 0)
                counts[wave] = __popcll(those);
            __syncthreads();
            uint32_t rank = seen + __popcll(those & ((1ull << lane) - 1));
            for (uint32_t w = 0; w < kWaves; w++) {
                rank += w < wave ? counts[w] : 0;
                seen += counts[w];
            }
            total = seen;
            f(m, in, rank);
        }
    };
    auto write = [&](uint32_t m, bool in, uint32_t rank) {
        if (m >= (uint32_t)g1)
            return;
        const uint32_t mine = rank % kShared, first = rank - mine;
        const uint32_t many = !in ? 0 : total - first < kShared ? total - first : kShared;
        a.rows[m].many = many | mine << 8;
        for (uint32_t k = 0; k < many; k++)
            a.rows[m].member[k] = list[first + k];
    };
    each([&](uint32_t m, bool in, uint32_t rank) {
        if (in)
            list[rank] = m;
        if (at_once) {
            __syncthreads();
            write(m, in, rank);
        }
    });
    if (at_once)
        return;
    const uint32_t all = total;
    __syncthreads();
    each([&](uint32_t m, bool in, uint32_t rank) {
        total = all;
        write(m, in, rank);
    });
}

// Sums for sequences with up to ROWS rows each (4, 8 or 16), 16 / ROWS of them in one product:
// a lane has in sum[c] key c * 16 + lane % 16's of the sequence that has its quarter of the
// rows.  Lane n of `of` has the n-th sequence.
template <typename T, int D, int ROWS>
__device__ __forceinline__ void packed_weights(const WeightsIn& a, const Known& of, uint32_t n0, uint32_t count,
                                               uint32_t x0, uint32_t xs,
                                               const typename Vec8<T>::type (&k)[4][D / 32], WordsOf<16>& words,
                                               float (&sum)[4])
{
    using V = typename Vec8<T>::type;
    const uint32_t lane = lane_id(), quarter = lane / 16, n = n0 + lane % 16 / ROWS, r = lane % ROWS;
    const uint32_t from = n < count ? n : n0;
    const uint32_t tok0 = __shfl(of.tok0, from), ntok = __shfl(of.ntok, from);
    const uint32_t first = a.last && a.last < ntok ? ntok - a.last : 0, rows = (ntok - first) * a.ratio;
    const bool there = n < count && r < rows;
    const uint32_t row = there ? r : 0, t = first + row / a.ratio, x = x0 + row % a.ratio * xs;
    const uint16_t* at = a.q + (int64_t)(tok0 + t) * a.q_stride + (uint64_t)x * D + quarter * 8;
    V q[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; d++)
        q[d] = *reinterpret_cast<const V*>(at + d * 32);
    const float far = a.lse[(uint64_t)(tok0 + t) * a.q_heads + x] * kLog2e;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (quarter == 0)
        words.lse[lane] = there && far != -INFINITY ? far : INFINITY;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const v4f l = *reinterpret_cast<const v4f*>(&words.lse[quarter * 4]);
#pragma unroll
    for (int c = 0; c < 4; c++) {
        v4f z = {};
#pragma unroll
        for (int d = 0; d < D / 32; d++)
            z = mfma(q[d], k[c][d], z);
        sum[c] = 0;
#pragma unroll
        for (int j = 0; j < 4; j++)
            sum[c] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[j], a.scale2, -l[j]));
        if (ROWS > 4)
            sum[c] += __shfl_xor(sum[c], 16);
        if (ROWS > 8)
            sum[c] += __shfl_xor(sum[c], 32);
    }
}

__device__ __forceinline__ uint32_t from_lane(uint32_t x, uint32_t lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ int64_t from_lane(int64_t x, uint32_t lane)
{
    return (int64_t)((uint64_t)from_lane((uint32_t)((uint64_t)x >> 32), lane) << 32 | from_lane((uint32_t)x, lane));
}
__device__ __forceinline__ Known of_lane(const Known& x, uint32_t lane)
{
    Known y;
    y.tok0 = from_lane(x.tok0, lane);
    y.ntok = from_lane(x.ntok, lane);
    y.len = from_lane(x.len, lane);
    y.keep = from_lane(x.keep, lane);
    y.own0 = from_lane(x.own0, lane);
    y.at = from_lane(x.at, lane);
    y.old = from_lane(x.old, lane);
    return y;
}

// Sums over the rows [row0, end) of a sequence, for the keys in a wave's registers: of key c *
// 16 + lane % 16, a quarter of the rows a lane.
template <typename T, int D>
__device__ __forceinline__ void weights_of(const WeightsIn& a, const Known& s, uint32_t row0, uint32_t x0, uint32_t xs,
                                           int64_t i0, bool causal, const typename Vec8<T>::type (&k)[4][D / 32],
                                           WordsOf<16>& words, float (&total)[4])
{
    using V = typename Vec8<T>::type;
    LongSum sum[4];
    const uint32_t lane = lane_id(), quarter = lane / 16;
    const uint32_t end = s.ntok * a.ratio;
    const int64_t pos0 = (int64_t)s.len - s.ntok;
    if (causal && i0 > pos0 + row0 / a.ratio)
        row0 = (uint32_t)(i0 - pos0) * a.ratio;
    for (; row0 < end; row0 += 16) {
        const uint32_t mine = row0 + lane % 16, row = mine < end ? mine : end - 1;
        const uint32_t t = row / a.ratio, x = x0 + (row - t * a.ratio) * xs;
        const uint16_t* at = a.q + (int64_t)(s.tok0 + t) * a.q_stride + (uint64_t)x * D + quarter * 8;
        V q[D / 32];
#pragma unroll
        for (int d = 0; d < D / 32; d++)
            q[d] = *reinterpret_cast<const V*>(at + d * 32);
        const float far = a.lse[(uint64_t)(s.tok0 + t) * a.q_heads + x] * kLog2e;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (quarter == 0) {
            // rows past the last and rows that see nothing add nothing
            words.lse[lane] = mine < end && far != -INFINITY ? far : INFINITY;
            words.sees[lane] = (int32_t)(pos0 + t);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const v4f l = *reinterpret_cast<const v4f*>(&words.lse[quarter * 4]);
        const int4 sees = *reinterpret_cast<const int4*>(&words.sees[quarter * 4]);
        const int32_t last[4] = {sees.x, sees.y, sees.z, sees.w};
        const bool masked = causal && i0 + kBlockKeys - 1 > pos0 + row0 / a.ratio;
        const int32_t key = (int32_t)((uint32_t)i0 + lane % 16);
#pragma unroll
        for (int c = 0; c < 4; c++) {
            v4f z = {};
#pragma unroll
            for (int d = 0; d < D / 32; d++)
                z = mfma(q[d], k[c][d], z);
            float add = 0;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j], a.scale2, -l[j]));
                add += !masked || key + c * 16 <= last[j] ? w : 0.0f;
            }
            sum[c].add(add);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; c++)
        total[c] = sum[c].sum;
}

// collect(sequence, its view, the token that slot0 would be of it, tokens [from, to) that are
// meant, whether later tokens do not see them) for the sequences that have tokens in the
// slots from slot0 on; those that a run shares, for its first sequence's slots, for each of
// its sequences.  By whole waves, slot0 uniform.
template <typename F>
__device__ __forceinline__ void each_sequence(const TokenBatch& b, const PlanView& pv, int64_t slot0, uint32_t keys,
                                              bool& bad, F&& collect)
{
    const int64_t entry0 = slot0 >> b.shift, entry1 = (slot0 + keys - 1) >> b.shift;
    for (uint32_t s = wave_find(b.off, b.n, 1, entry0); s < b.n && b.off[s] <= entry1; s++) {
        const SeqView v = sequence_view(b, s);
        bad |= v.bad;
        const int64_t i0 = slot0 - (b.off[s] << b.shift);
        int64_t shared = 0;  // tokens that the run's first sequence's blocks take
        if (b.groups) {
            const RunOf r = run_of(b, s);
            shared = r.ok ? (int64_t)pv.unit[r.g].key1 : 0;
            if (r.ok && s == (uint32_t)r.g0 && i0 < shared)
                for (uint32_t m = (uint32_t)r.g0; m < (uint32_t)r.g1; m++) {
                    const SeqView x = sequence_view(b, m);
                    if (!x.bad && x.ntok && x.len && pv.unit[b.groups + m].key0)
                        collect(m, x, i0, 0, shared, false);
                }
            // one that is not among those keeps its own
            shared = v.ntok && v.len && pv.unit[b.groups + s].key0 ? shared : 0;
        }
        if (v.len > shared && i0 < v.len && i0 + (int64_t)keys > shared)
            collect(s, v, i0, shared, v.len, true);
    }
}

// A wave has 64 slots and a few heads one after another.  A run's shared keys are read for
// kShared of its sequences at once, by the blocks of one of these, or of each for some heads.
// RUNS: the batch has runs (a kernel of its own: its registers would halve the other's waves).
template <typename T, int D, bool RUNS>
__global__ __launch_bounds__(kThreads, D == 256 ? (RUNS ? 1 : 2) : RUNS && D == 128 ? 2 : 3) void weights_kernel(WeightsIn a, const PlanView pv,
                                                                            uint32_t heads, uint64_t items,
                                                                            uint32_t* status)
{
    using V = typename Vec8<T>::type;
    __shared__ __attribute__((aligned(16))) WordsOf<16> all_words[kWaves];
    const TokenBatch& b = a.b;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
    const uint64_t item = (uint64_t)blockIdx.x * kWaves + wave;
    const uint32_t sets = (a.kv_heads + heads - 1) / heads, h0 = item % sets * heads;
    const uint32_t h1 = h0 + heads < a.kv_heads ? h0 + heads : a.kv_heads;
    const int64_t slot0 = (int64_t)(item / sets) * kBlockKeys;
    const int64_t entry0 = slot0 >> b.shift, entry1 = (slot0 + kBlockKeys - 1) >> b.shift;
    // the pages of the block's keys, before it is known whose they are
    uint32_t page[4];
#pragma unroll
    for (int c = 0; c < 4; c++) {
        const int64_t e = (slot0 + c * 16 + lane % 16) >> b.shift;
        page[c] = e < b.entries ? (uint32_t)b.page[e] : 0;
    }
    if (!plan_of(*pv.head, b, a.q_heads, a.plan_heads, a.plan_dim)) {
        if (blockIdx.x == 0 && threadIdx.x == 0)
            atomicOr(status, kErrInval);
        return;
    }
    if (item >= items)
        return;
    WordsOf<16>& words = all_words[wave];
    V k[4][D / 32];
    uint32_t loaded = 0xFFFFFFFFu;  // the head whose keys k has
    bool bad = false;
    auto load = [&](uint32_t h) {
        if (loaded == h)
            return;
        loaded = h;
#pragma unroll
        for (int c = 0; c < 4; c++) {
            const uint32_t p = page[c] < a.n_pages ? page[c] : 0;
            const int64_t slot = slot0 + c * 16 + lane % 16;
            const uint16_t* at =
                a.k + ((((uint64_t)p * a.kv_heads + h) << b.shift) + (slot & ((1 << b.shift) - 1))) * D + lane / 16 * 8;
#pragma unroll
            for (int d = 0; d < D / 32; d++)
                k[c][d] = *reinterpret_cast<const V*>(at + d * 32);
        }
    };
    // sums of a sequence over its tokens [from, to) that are in the block (i0: the token that
    // slot0 would be), whose keys are here, to where the sequence has them
    auto collect = [&](const Known& s, uint32_t h, int64_t i0, int64_t from, int64_t to, bool causal) {
        const uint32_t x0 = a.paired ? h / 2 * 2 * a.ratio + h % 2 : h * a.ratio, xs = a.paired ? 2 : 1;
        const int64_t i = i0 + lane;
        const bool mine = i >= from && i < to && i < (int64_t)s.len;  // (whatever the plan says)
        float carried = 0;
        if (mine && i < s.keep)
            carried = a.decay * a.prev[(int64_t)h * a.prev_stride + s.old + i];
        float sum = 0;
        const uint32_t first = (a.last && a.last < s.ntok ? s.ntok - a.last : 0) * a.ratio;
        if (a.parts && s.ntok * a.ratio - first > kFewRows) {
            // (the tall block begins before this one, in the same sequence's numbers)
            SeqView v{0, (int64_t)s.len, (int64_t)s.len - s.ntok, s.tok0, s.ntok, false};
            const int64_t tall0 = i0 - (slot0 & (kTallKeys - 1));
            for (uint32_t p = 0; p < a.parts; p++) {
                const Stretch r = stretch_of(a, v, tall0, causal, p);
                if (mine && r.row0 < r.row1)
                    sum += a.part[((uint64_t)p * a.kv_heads + h) * a.slots + s.at + i];
            }
        } else if (s.ntok) {
            load(h);
            float part[4];
            weights_of<T, D>(a, s, first, x0, xs, i0, causal, k, words, part);
#pragma unroll
            for (int c = 0; c < 4; c++) {
                part[c] += __shfl_xor(part[c], 16);
                part[c] += __shfl_xor(part[c], 32);
                sum = lane / 16 == (uint32_t)c ? part[c] : sum;
            }
        }
        if (s.ntok)
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const int64_t key = i0 + c * 16 + lane % 16;
                bad |= key >= from && key < to && page[c] >= a.n_pages;
            }
        if (mine)
            a.w[(int64_t)h * a.w_stride + s.at + i] = carried + sum;
    };
    // The shared tokens in the block, those of sequence x, for the `count` sequences that its row
    // names (m: a lane's), of which it is number `mine`.
    auto share = [&](const Known& x, uint32_t count, uint32_t mine, uint32_t m) {
        // Where a wave has many heads, the sequences' blocks have each its own of them (128 sequences
        // on 8 prefixes 88 to 83 us); where it has few, the first sequence's have all (16 on 2: 20,
        // dealt 21).
        const bool dealt = heads >= kShared;
        const uint32_t first = dealt ? h0 + (mine + count - h0 % count) % count : mine ? h1 : h0, step = dealt ? count : 1;
        if (first >= h1)
            return;
        const bool in = lane < count && m < b.n;
        Known of{};
        if (in)
            of = a.rows[m].x;
        const uint64_t those = ballot(in);
        const uint32_t rows = (a.last && a.last < of.ntok ? a.last : of.ntok) * a.ratio;
        const int64_t i0 = slot0 - x.at;
        if (__any(in && rows > 16)) {
            for (uint32_t h = first; h < h1; h += step)
                for (uint64_t next = those; next; next &= next - 1)
                    collect(of_lane(of, (uint32_t)__builtin_ctzll(next)), h, i0, 0, x.own0, false);
            return;
        }
        auto packed = [&](auto size) {
            constexpr int kRows = decltype(size)::value;
            for (uint32_t h = first; h < h1; h += step) {
                const uint32_t x0 = a.paired ? h / 2 * 2 * a.ratio + h % 2 : h * a.ratio, xs = a.paired ? 2 : 1;
                load(h);
                for (uint32_t n0 = 0; n0 < count; n0 += 16 / kRows) {
                    const uint32_t n = n0 + lane / 16 * 4 / kRows, from = n < count ? n : n0;
                    const bool writes = n < count && lane / 16 * 4 % kRows == 0;
                    const int64_t at = __shfl((long long)of.at, from), old = __shfl((long long)of.old, from);
                    const uint32_t keep = __shfl(of.keep, from), len = __shfl(of.len, from);
                    float carried[4], sum[4];
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        const int64_t i = i0 + c * 16 + lane % 16;
                        carried[c] = writes && i >= 0 && i < keep ? a.decay * a.prev[(int64_t)h * a.prev_stride + old + i] : 0.0f;
                    }
                    packed_weights<T, D, kRows>(a, of, n0, count, x0, xs, k, words, sum);
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        const int64_t i = i0 + c * 16 + lane % 16;
                        if (writes && i >= 0 && i < x.own0 && i < len)
                            a.w[(int64_t)h * a.w_stride + at + i] = carried[c] + sum[c];
                    }
                }
            }
        };
        if (!__any(in && rows > 4))
            packed(std::integral_constant<int, 4>{});
        else if (!__any(in && rows > 8))
            packed(std::integral_constant<int, 8>{});
        else
            packed(std::integral_constant<int, 16>{});
#pragma unroll
        for (int c = 0; c < 4; c++) {
            const int64_t key = i0 + c * 16 + lane % 16;
            bad |= key >= 0 && key < x.own0 && page[c] >= a.n_pages;
        }
    };
    // the sequences in the block, 64 looked at a time
    for (uint32_t s0 = wave_find(b.off, b.n, 1, entry0); s0 < b.n; s0 += kWave) {
        const uint32_t s = s0 + lane;
        const bool in = s < b.n && b.off[s] <= entry1;
        Known all{};
        uint32_t many = 0;
        if constexpr (RUNS) {
            if (in) {
                all = a.rows[s].x;
                many = all.own0 ? a.rows[s].many : 0;
            }
        } else {
            all = known_of<false>(b, pv, s, in, bad);
        }
        const bool own = in && all.len > all.own0 && slot0 - all.at < (int64_t)all.len &&
                         slot0 - all.at + (int64_t)kBlockKeys > (int64_t)all.own0;
        if (!RUNS)
            add_carried(a, s, own, all, bad);
        for (uint64_t left = ballot(own); left; left &= left - 1) {
            const Known x = of_lane(all, (uint32_t)__builtin_ctzll(left));
            for (uint32_t h = h0; h < h1; h++)
                collect(x, h, slot0 - x.at, x.own0, x.len, true);
        }
        // a run's shared tokens
        for (uint64_t left = !RUNS ? 0 : ballot(many && slot0 - all.at < (int64_t)all.own0); left; left &= left - 1) {
            const uint32_t j = (uint32_t)__builtin_ctzll(left), word = from_lane(many, j);
            const uint32_t count = (word & 255) < kShared ? word & 255 : kShared, mine = word >> 8;
            if constexpr (RUNS)
                if (count)
                    share(of_lane(all, j), count, mine, lane < count ? a.rows[s0 + j].member[lane] : 0);
        }
        if (!__all(in))
            break;
    }
    if (bad)
        atomicOr(status, kErrInval);
}

// ---------------------------------------------------------------------------
// Many rows.
// ---------------------------------------------------------------------------

// Token and head of a thread's row, kept from tile to tile without a division.
struct RowAt {
    uint32_t t, x;
    __device__ __forceinline__ void begin(uint32_t row, uint32_t ratio)
    {
        t = row / ratio;
        x = row - t * ratio;
    }
    __device__ __forceinline__ void on(uint32_t tokens, uint32_t heads, uint32_t ratio)
    {
        t += tokens;
        x += heads;
        if (x >= ratio) {
            x -= ratio;
            t++;
        }
    }
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : D == 128 ? 2 : 3) void weights_tall_kernel(WeightsIn a, const PlanView pv,
                                                                                  uint32_t blocks, uint32_t* status)
{
    using V = typename Vec8<T>::type;
    constexpr uint32_t kRowChunks = D / 8, kStep = kThreads / kRowChunks;
    constexpr int kLoads = kTallRows * D / 8 / kThreads;
    using RowWords = WordsOf<kTallRows>;
    __shared__ __attribute__((aligned(512))) uint16_t tiles[2][kTallRows * D];
    __shared__ __attribute__((aligned(16))) RowWords words[3];  // of the tile before too, whose weights come later
    const TokenBatch& b = a.b;
    if (!plan_of(*pv.head, b, a.q_heads, a.plan_heads, a.plan_dim))
        return;  // (the other kernel reports it)
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id(), half = lane / 32;
    // the blocks that pass over the same rows at the same time are on the same die
    const uint32_t h = blockIdx.x % a.kv_heads, block = blockIdx.x / a.kv_heads % blocks,
                   p = blockIdx.x / a.kv_heads / blocks;
    const int64_t slot0 = (int64_t)block * kTallKeys;
    const uint32_t x0 = a.paired ? h / 2 * 2 * a.ratio + h % 2 : h * a.ratio, xs = a.paired ? 2 : 1;
    V k[2][D / 16];
    bool have = false, bad = false;
    const uint32_t tokens = kTallRows / a.ratio, heads = kTallRows % a.ratio;
    auto collect = [&](uint32_t s, const SeqView& v, int64_t i0, int64_t from, int64_t to, bool causal) {
        if (v.ntok == 0 || few(a, v))
            return;
        const Stretch r = stretch_of(a, v, i0, causal, p);
        if (r.row0 >= r.row1)
            return;
        if (!have) {
            have = true;
#pragma unroll
            for (int c = 0; c < 2; c++) {
                const int64_t slot = slot0 + wave * kBlockKeys + c * 32 + lane % 32, e = slot >> b.shift;
                uint32_t page = e < b.entries ? (uint32_t)b.page[e] : 0;
                page = page < a.n_pages ? page : 0;  // (the other kernel reports it)
                const uint16_t* at = a.k + ((((uint64_t)page * a.kv_heads + h) << b.shift) + (slot & ((1 << b.shift) - 1))) * D +
                                     half * 8;
#pragma unroll
                for (int d = 0; d < D / 16; d++)
                    k[c][d] = *reinterpret_cast<const V*>(at + d * 16);
            }
        }
        RowAt word;  // whose words a thread writes
        word.begin(r.row0 + threadIdx.x % kTallRows, a.ratio);
        float far = 0;
        const uint32_t to_row = threadIdx.x / kRowChunks, to_chunk = threadIdx.x % kRowChunks;
        // where a step of rows is whole tokens, a lane's place in one is the same in all of
        // them, but for k_swizzle, which goes by the row's low four bits: a uniform address
        // and the lane's bytes on from it
        const bool even = kStep % a.ratio == 0 && r.row0 % a.ratio == 0 && a.q_stride < (1 << 24);
        uint32_t lane_at[2];
#pragma unroll
        for (int i = 0; i < 2; i++)
            lane_at[i] = even ? (uint32_t)(to_row / a.ratio * a.q_stride + (x0 + to_row % a.ratio * xs) * D +
                                           (to_chunk ^ k_swizzle<D>(to_row + i * kStep)) * 8) * 2
                              : 0;
        auto send = [&](uint32_t row0, const uint16_t* to) {
            const uint32_t at = lds_address(to) + wave * kWave * 16;
            if (even && row0 + kTallRows <= r.row1) {
                // (uniform, and said so: not every optimisation level sees it)
                const uint64_t first = (uint64_t)(v.tok0 + row0 / a.ratio) * a.q_stride;
                const uint16_t* from = a.q + ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(first >> 32)) << 32 |
                                              (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)first));
#pragma unroll
                for (int i = 0; i < kLoads; i++)
                    send16(from + i * (int64_t)(kStep / a.ratio) * a.q_stride, lane_at[i % 2], at + i * kThreads * 16);
                return;
            }
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                const uint32_t row = to_row + i * kStep;
                // rows past the last: the last token's first head's again
                const bool there = row0 + row < r.row1;
                const uint32_t t = there ? (row0 + row) / a.ratio : v.ntok - 1, x = there ? (row0 + row) % a.ratio : 0;
                send16(a.q + (int64_t)(v.tok0 + t) * a.q_stride + (uint64_t)(x0 + x * xs) * D +
                           (to_chunk ^ k_swizzle<D>(row)) * 8,
                       at + i * kThreads * 16);
            }
        };
        // words of the tile at row0, read, and then written
        auto read_words = [&](uint32_t row0) {
            const uint32_t row = row0 + threadIdx.x;
            far = INFINITY;
            if (threadIdx.x < kTallRows && row < r.row1) {
                const float l = a.lse[(uint64_t)(v.tok0 + word.t) * a.q_heads + x0 + word.x * xs] * kLog2e;
                far = l != -INFINITY ? l : INFINITY;
            }
        };
        auto write_words = [&](RowWords& to) {
            if (threadIdx.x < kTallRows) {
                to.lse[threadIdx.x] = far;
                to.sees[threadIdx.x] = (int32_t)(v.pos0 + word.t);
            }
            word.on(tokens, heads, a.ratio);
        };
        const int64_t i1 = i0 + wave * kBlockKeys;  // the wave's first key
        const int32_t key = (int32_t)((uint32_t)i1 + lane % 32);
        const bool any = i1 < to && i1 + (int64_t)kBlockKeys > from;  // has the wave some of these keys?
        LongSum sum[2];
        __syncthreads();  // (the tiles' last readers)
        read_words(r.row0);
        send(r.row0, tiles[0]);
        write_words(words[0]);
        // the keys are here: the compiler, which does not count the sends, would wait for their
        // reads in every tile and so for the sends
#pragma unroll
        for (int d = 0; d < D / 16; d++)
            asm volatile("" : "+v"(k[0][d]), "+v"(k[1][d]));
        // Scores of 32 rows (at q, in LDS).  With the weights of the 32 rows before them (old, at
        // `part` of their tile) beside their products: the matrix unit has work that these do
        // not wait for.
        auto scores_of = [&](auto with, v16f (&z)[2], const uint16_t* q, const v16f (&old)[2], const RowWords& words,
                             uint32_t part) {
            constexpr int kSteps = D / 16, kPer = 32 / kSteps;
            V f[2];
            auto read = [&](int d) {
                f[d % 2] = *reinterpret_cast<const V*>(q + lane % 32 * D + ((d * 2 + half) ^ k_swizzle<D>(lane % 32)) * 8);
            };
            float add[2] = {0, 0};
            v4f l;
            z[0] = z[1] = v16f{};
            read(0);
#pragma unroll
            for (int d = 0; d < kSteps; d++) {
                if (d + 1 < kSteps)
                    read(d + 1);
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    z[c] = mfma(f[d % 2], k[c][d], z[c]);
                    if constexpr (decltype(with)::value) {
                        float w[kPer / 2];
                        if ((d * kPer + c * kPer / 2) % 8 == 0)
                            l = *reinterpret_cast<const v4f*>(&words.lse[part + (d * kPer + c * kPer / 2) / 8 * 8 + half * 4]);
#pragma unroll
                        for (int i = 0; i < kPer / 2; i++) {
                            const int at = d * kPer + c * kPer / 2 + i;
                            w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(old[at / 4 % 2][at / 8 * 4 + at % 4], a.scale2, -l[at % 4]));
                        }
#pragma unroll
                        for (int i = 0; i < kPer / 2; i++)
                            add[(d * kPer + c * kPer / 2 + i) / 4 % 2] += w[i];
                        // (they would sink to where the sums are wanted, behind all products)
                        asm volatile("" : "+v"(add[0]), "+v"(add[1]));
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (decltype(with)::value) {
                sum[0].add(add[0]);
                sum[1].add(add[1]);
            }
        };
        // the weights of 32 rows by themselves; masked: some key is later than some row
        auto finish = [&](const v16f (&z)[2], const RowWords& words, uint32_t part, bool masked) {
            float add[2] = {0, 0};
#pragma unroll
            for (int g = 0; g < 16; g += 4) {
                const v4f l = *reinterpret_cast<const v4f*>(&words.lse[part + g * 2 + half * 4]);
                const int4 sees = *reinterpret_cast<const int4*>(&words.sees[part + g * 2 + half * 4]);
                const int32_t last[4] = {sees.x, sees.y, sees.z, sees.w};
#pragma unroll
                for (int c = 0; c < 2; c++)
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(z[c][g + j], a.scale2, -l[j]));
                        add[c] += !masked || key + c * 32 <= last[j] ? w : 0.0f;
                    }
            }
            sum[0].add(add[0]);
            sum[1].add(add[1]);
        };
        const std::true_type beside;
        const std::false_type alone;
        v16f za[2], zb[2];  // of a tile's first and second half
        bool pending = false, was_masked = false;
        uint32_t buf = 0, now = 0, before = 0;
        for (uint32_t row0 = r.row0; row0 < r.row1; row0 += kTallRows, buf ^= 1) {
            wait_sent();
            __syncthreads();
            const uint16_t* q = tiles[buf];
            const bool more = row0 + kTallRows < r.row1;
            if (more) {
                read_words(row0 + kTallRows);
                send(row0 + kTallRows, tiles[buf ^ 1]);
            }
            if (any) {
                const bool masked = causal && i1 + kBlockKeys - 1 > words[now].sees[0];
                if (pending && !was_masked) {
                    scores_of(beside, za, q, zb, words[before], 32);
                } else {
                    if (pending)
                        finish(zb, words[before], 32, true);
                    scores_of(alone, za, q, zb, words[before], 32);
                }
                if (!masked) {
                    scores_of(beside, zb, q + 32 * D, za, words[now], 0);
                } else {
                    finish(za, words[now], 0, true);
                    scores_of(alone, zb, q + 32 * D, za, words[now], 0);
                }
                pending = true;
                was_masked = masked;
            }
            before = now;
            now = now == 2 ? 0 : now + 1;
            if (more)
                write_words(words[now]);
        }
        if (any)
            finish(zb, words[before], 32, was_masked);
        const float s0 = sum[0].sum + __shfl_xor(sum[0].sum, 32), s1 = sum[1].sum + __shfl_xor(sum[1].sum, 32);
        const int64_t i = i1 + lane;
        if (i >= from && i < to && i < v.len)
            a.part[((uint64_t)p * a.kv_heads + h) * a.slots + (b.off[s] << b.shift) + i] = half ? s1 : s0;
    };
    each_sequence(b, pv, slot0, kTallKeys, bad, collect);
}

// How many stretches of rows tall blocks are for (0: there are none), and their rows: some 32
// workgroups a compute unit if all sequences are alike (two prompts of 7,000 to 8,192 tokens: 6
// 728 us, 16 or 32 665), not more than kParts, nor than kSums sums.  A batch with hardly more
// tokens than sequences (kMany rows) is taken for a decode step, whose blocks would find nothing
// to do, and has none.  By these numbers alone it cannot be told from one where a few sequences
// have all the new tokens among many that have none, which is slower for it: 512 tokens of one
// sequence, 64 query and 8 key heads of 128, 4,096 keys, take 191 us among 64 places, 1,792 among
// 512 or 1,024.
uint32_t parts_of_rows(const dm_ctx* c, const dm_token_batch& b, uint32_t ratio, uint32_t last, uint64_t blocks,
                       uint32_t* part_rows)
{
    constexpr uint64_t kMany = 1024, kParts = 32, kSums = 1 << 24;
    *part_rows = 0;
    const uint64_t n = b.tables.n, tokens = last && last < b.q_tokens ? last : b.q_tokens;  // of a sequence, at most
    if (b.q_tokens <= n || (b.q_tokens - n) * ratio <= kMany || tokens * ratio <= kFewRows || blocks == 0)
        return 0;
    const uint64_t each = (last && last * n < b.q_tokens ? last * n : b.q_tokens) * ratio / n;  // rows of a sequence
    uint64_t rows = blocks * each / (32 * c->n_cu);
    rows = (rows / kTallRows + 1) * kTallRows;
    rows = rows < 256 ? 256 : rows;
    const uint64_t room = kSums / (blocks * kTallKeys);
    const uint64_t limit = room < 1 ? 1 : room < kParts ? room : kParts;
    const uint64_t most = (tokens * ratio + limit - 1) / limit;
    rows = rows < most ? (most + kTallRows - 1) / kTallRows * kTallRows : rows;
    const uint64_t parts = (tokens * ratio + rows - 1) / rows;
    if (parts * blocks > 0x7FFFFFFFull)
        return 0;
    *part_rows = (uint32_t)rows;
    return (uint32_t)parts;
}

}  // namespace

hipError_t attn_weights(dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& kv, uint32_t q_heads,
                        const void* plan, uint32_t layer, const dm_weight_args& g)
{
    WeightsIn a;
    a.b = token_batch(c, b);
    a.k = static_cast<const uint16_t*>(kv.k) + (uint64_t)layer * kv.layer_stride;
    a.q = static_cast<const uint16_t*>(g.q);
    a.lse = g.lse;
    a.w = g.w;
    a.prev = g.prev;
    a.prev_off = g.prev_off;
    a.src = g.src;
    a.keep = g.keep;
    a.q_stride = g.q_stride;
    a.w_stride = g.w_stride;
    a.prev_stride = g.prev_stride;
    a.prev_room = g.prev_room;
    a.prev_n = (uint32_t)g.prev_n;
    a.n_pages = kv.n_pages;
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.ratio = q_heads / kv.kv_heads;
    a.last = g.last;
    a.paired = g.paired;
    a.plan_heads = g.paired ? kv.kv_heads / 2 : kv.kv_heads;
    a.plan_dim = g.paired ? kv.head_dim * 2 : kv.head_dim;
    a.scale2 = g.scale * kLog2e;
    a.decay = g.decay;
    const PlanView pv = plan_view(const_cast<void*>(plan), b.tables.n, b.groups);
    const uint64_t slots = b.tables.entries * c->cfg.block_size;
    if (slots == 0)
        return hipSuccess;
    a.slots = (int64_t)slots;
    // heads of a wave: one, or as many as leave some 16 waves a SIMD
    uint64_t heads = slots / kBlockKeys * kv.kv_heads / (32 * c->n_cu);
    heads = heads < 1 ? 1 : heads > kv.kv_heads ? kv.kv_heads : heads;
    const uint64_t items = (slots + kBlockKeys - 1) / kBlockKeys * ((kv.kv_heads + heads - 1) / heads);
    const uint64_t grid = (items + kWaves - 1) / kWaves;
    if (grid > 0x7FFFFFFFull)
        return hipErrorInvalidValue;
    const uint32_t blocks = (uint32_t)((slots + kTallKeys - 1) / kTallKeys);
    a.parts = parts_of_rows(c, b, a.ratio, g.last, (uint64_t)blocks * kv.kv_heads, &a.part_rows);
    a.part = nullptr;
    a.rows = nullptr;
    a.order = nullptr;
    const uint64_t n = b.tables.n, parts = (a.parts * kv.kv_heads * slots * 4 + 15) / 16 * 16;
    const uint64_t area = parts + (b.groups ? n * (sizeof(SeqRow) + 4) : 0);
    if (area) {
        hipError_t e;
        char* at = static_cast<char*>(scratch_get(c, kSlotPages, area, &e));
        if (!at)
            return e;
        a.part = reinterpret_cast<float*>(at);
        a.rows = reinterpret_cast<SeqRow*>(at + parts);
        a.order = reinterpret_cast<uint32_t*>(a.rows + n);
    }
    const uint32_t chunks = (uint32_t)((n + kThreads - 1) / kThreads);
    if (b.groups)
        weights_rows_kernel<<<chunks + (uint32_t)b.groups, kThreads, 0, c->stream>>>(a, pv, chunks, c->d_status);
    by_type(kv.dtype, kv.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        if (a.parts)
            weights_tall_kernel<T, D>
                <<<a.parts * blocks * kv.kv_heads, kThreads, 0, c->stream>>>(a, pv, blocks, c->d_status);
        if (b.groups)
            weights_kernel<T, D, true><<<(uint32_t)grid, kThreads, 0, c->stream>>>(a, pv, (uint32_t)heads, items, c->d_status);
        else
            weights_kernel<T, D, false><<<(uint32_t)grid, kThreads, 0, c->stream>>>(a, pv, (uint32_t)heads, items, c->d_status);
    });
    return hipGetLastError();
}

}  // namespace dm
