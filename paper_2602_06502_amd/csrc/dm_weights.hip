// The weight that each cached key has collected: for KV head h and token i of a sequence
//   w[h][i] = decay * prev[h][i] + sum over its new tokens t that see i, and over the query
//             heads x that read h, of exp(scale q_x,t . k_h,i - lse_x,t).
//
// Keys stay, queries pass: a wave has 64 neighbouring keys of one head in registers, as the
// right operand of S = Q K^T on 32x32x16 matrix instructions, and takes 32 rows (token,
// query head) at a time; a lane then holds scores of one key, so that their weights' sum over
// the rows is a sum over its own registers.  Nothing is added by two waves, so the order of
// every sum is fixed.  Blocks of 64 keys follow the tables' entries, not the sequences: a
// lane's page is known without knowing whose it is, and a block may hold the end of one
// sequence and the beginnings of others, which take their turns.
//
// The pages that a run shares (as its plan has found them) are read once, by the blocks of
// its first sequence's entries, for all its sequences, each with its own sums.
//
// Bound by reading keys where rows are few, by the exponentials where they are many.
#include "dm_attn.h"

namespace dm {
namespace {

constexpr uint32_t kBlockKeys = 64;

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
};

// The rows of a sequence for one KV head.
struct Rows {
    uint32_t tok0, ntok, first;  // first row that counts
    int64_t pos0;
};

// What a wave leaves for itself of its 32 rows: their log-sum-exps (in powers of two), and
// the last key that each sees.
struct RowWords {
    float lse[32];
    int32_t sees[32];
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

template <typename T, int D>
__device__ __forceinline__ void weights_of(const WeightsIn& a, const Rows& s, uint32_t x0, uint32_t xs, int64_t i0,
                                           bool causal, const typename Vec8<T>::type (&k)[2][D / 16], RowWords& words,
                                           float (&total)[2])
{
    LongSum sum[2];
    using V = typename Vec8<T>::type;
    const uint32_t lane = lane_id(), half = lane / 32;
    const uint32_t end = s.ntok * a.ratio;
    uint32_t row0 = s.first;
    if (causal && i0 > s.pos0 + row0 / a.ratio)
        row0 = (uint32_t)(i0 - s.pos0) * a.ratio;
    for (; row0 < end; row0 += 32) {
        const uint32_t mine = row0 + lane % 32, row = mine < end ? mine : end - 1;
        const uint32_t t = row / a.ratio, x = x0 + (row - t * a.ratio) * xs;
        const uint16_t* at = a.q + (s.tok0 + t) * a.q_stride + (uint64_t)x * D + half * 8;
        V q[D / 16];
#pragma unroll
        for (int d = 0; d < D / 16; d++)
            q[d] = *reinterpret_cast<const V*>(at + d * 16);
        const float far = a.lse[(uint64_t)(s.tok0 + t) * a.q_heads + x] * kLog2e;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (half == 0) {
            // rows past the last and rows that see nothing add nothing
            words.lse[lane] = mine < end && far != -INFINITY ? far : INFINITY;
            words.sees[lane] = (int32_t)(s.pos0 + t);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        v16f z[2] = {};
#pragma unroll
        for (int d = 0; d < D / 16; d++) {
            z[0] = mfma(q[d], k[0][d], z[0]);
            z[1] = mfma(q[d], k[1][d], z[1]);
        }
        const bool masked = causal && i0 + kBlockKeys - 1 > s.pos0 + row0 / a.ratio;
        const int32_t key = (int32_t)((uint32_t)i0 + lane % 32);
        float add[2] = {0, 0};
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const v4f l = *reinterpret_cast<const v4f*>(&words.lse[r * 2 + half * 4]);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][r + j], a.scale2, -l[j]));
                float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[1][r + j], a.scale2, -l[j]));
                if (masked) {
                    const int32_t last = words.sees[r * 2 + half * 4 + j];
                    w0 = key <= last ? w0 : 0.0f;
                    w1 = key + 32 <= last ? w1 : 0.0f;
                }
                add[0] += w0;
                add[1] += w1;
            }
        }
        sum[0].add(add[0]);
        sum[1].add(add[1]);
    }
    total[0] = sum[0].sum;
    total[1] = sum[1].sum;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void weights_kernel(WeightsIn a, const PlanView pv, uint64_t items, uint32_t* status)
{
    using V = typename Vec8<T>::type;
    __shared__ __attribute__((aligned(16))) RowWords all_words[kWaves];
    const TokenBatch& b = a.b;
    const PlanHead& ph = *pv.head;
    if (!plan_of(ph, b, a.q_heads, a.plan_heads, a.plan_dim)) {
        if (blockIdx.x == 0 && threadIdx.x == 0)
            atomicOr(status, kErrInval);
        return;
    }
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id(), half = lane / 32;
    const uint64_t item = (uint64_t)blockIdx.x * kWaves + wave;
    if (item >= items)
        return;
    RowWords& words = all_words[wave];
    const uint32_t h = item % a.kv_heads;
    const int64_t slot0 = (int64_t)(item / a.kv_heads) * kBlockKeys;
    const int64_t entry0 = slot0 >> b.shift, entry1 = (slot0 + kBlockKeys - 1) >> b.shift;
    const uint32_t x0 = a.paired ? h / 2 * 2 * a.ratio + h % 2 : h * a.ratio, xs = a.paired ? 2 : 1;
    V k[2][D / 16];
    bool bad_page[2] = {};
    bool have = false, bad = false;
    auto load = [&] {
        if (have)
            return;
        have = true;
#pragma unroll
        for (int c = 0; c < 2; c++) {
            const int64_t slot = slot0 + c * 32 + lane % 32, e = slot >> b.shift;
            const uint32_t p = e < b.entries ? (uint32_t)b.page[e] : 0;
            bad_page[c] = p >= a.n_pages;
            const uint16_t* at = a.k + ((((uint64_t)(p < a.n_pages ? p : 0) * a.kv_heads + h) << b.shift) +
                                        (slot & ((1 << b.shift) - 1))) * D + half * 8;
#pragma unroll
            for (int d = 0; d < D / 16; d++)
                k[c][d] = *reinterpret_cast<const V*>(at + d * 16);
        }
    };
    // sums of sequence s over tokens [from, to) that are in the block (token 0 is slot0 -
    // i0), whose keys are here, to where s has them
    auto collect = [&](uint32_t s, const SeqView& v, int64_t i0, int64_t from, int64_t to, bool causal) {
        float sum[2] = {0, 0};
        const int64_t i = i0 + lane;
        const bool mine = i >= from && i < to;
        if (v.ntok) {
            load();
            const bool key[2] = {i0 + lane % 32 >= from && i0 + lane % 32 < to,
                                 i0 + 32 + lane % 32 >= from && i0 + 32 + lane % 32 < to};
            bad |= (key[0] && bad_page[0]) || (key[1] && bad_page[1]);
            Rows r{v.tok0, v.ntok, (a.last && a.last < v.ntok ? v.ntok - a.last : 0) * a.ratio, v.pos0};
            weights_of<T, D>(a, r, x0, xs, i0, causal, k, words, sum);
        }
        sum[0] += __shfl_xor(sum[0], 32);
        sum[1] += __shfl_xor(sum[1], 32);
        float w = half ? sum[1] : sum[0];
        if (!mine)
            return;
        const int64_t at = (v.off << b.shift) + i;
        if (a.prev) {
            if (!a.prev_off) {
                if (i < v.pos0)
                    w = __builtin_fmaf(a.decay, a.prev[(int64_t)h * a.prev_stride + at], w);
            } else if (i < a.keep[s]) {
                const uint32_t from_s = (uint32_t)a.src[s];
                const int64_t old = from_s < a.prev_n ? (a.prev_off[from_s] << b.shift) + i : -1;
                if (old >= 0 && old < a.prev_room)
                    w = __builtin_fmaf(a.decay, a.prev[(int64_t)h * a.prev_stride + old], w);
                else
                    bad = true;
            }
        }
        a.w[(int64_t)h * a.w_stride + at] = w;
    };
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
        if (v.len > shared && i0 < v.len && i0 + (int64_t)kBlockKeys > shared)
            collect(s, v, i0, shared, v.len, true);
    }
    if (bad)
        atomicOr(status, kErrInval);
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
    const uint64_t items = (slots + kBlockKeys - 1) / kBlockKeys * kv.kv_heads, grid = (items + kWaves - 1) / kWaves;
    if (grid > 0x7FFFFFFFull)
        return hipErrorInvalidValue;
    if (grid == 0)
        return hipSuccess;
    by_type(kv.dtype, kv.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        weights_kernel<T, D><<<(uint32_t)grid, kThreads, 0, c->stream>>>(a, pv, items, c->d_status);
    });
    return hipGetLastError();
}

}  // namespace dm
