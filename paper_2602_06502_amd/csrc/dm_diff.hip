// Differential attention over KV pages: a pair of query heads reads a pair of KV heads,
//   o = softmax(scale q1 K1) V - lambda softmax(scale q2 K2) V,   V = [V1 | V2],
// and, with a norm, o / sqrt(mean(o^2) + eps) * weight * gain over the pair's 2 head_dim
// elements.
//
// The pass is attention's (dm_attn.h) on pairs: a KV head of it is a pair, a row a query
// head, which map it is by its parity, the width D of a value twice head_dim.  A tile of
// keys and values is read once for both maps, and a row's products are those of its own
// map: 2 head_dim for its scores, 4 head_dim for its values a key, as the formula has
// them.  Rows that are whole are subtracted, normed and written where they end; those in
// parts are joined by a second kernel, map by map, and subtracted there.
//
// Wide tiles round a row's weights to the pages' type before they meet the values, as in plain
// attention, whose comment has the reasons; the difference, the sums and the norm are in 32 bits.
// So an error of either map's size, not of the difference's, stays where the maps cancel.  With the
// weights in two parts, as narrow tiles have them, the prompts below take 1,897 us instead of 1,196
// and the tails 510 instead of 367, for errors of 0.0017 instead of 0.0022 of the output (rounding
// it alone makes 0.0017) and of 0.00021 instead of 0.00029.
//
// Bound as attention is: narrow tiles by reading the pages, wide ones by the matrix and
// vector units (each weight meets two head_dims of values, so the matrix unit has three
// quarters of its work there, where it has half in plain attention).  32 query and 8 key heads: 64
// tokens behind 64 to 8,192 keys 221 us (4.9 TB/s), two prompts of 7,000 to 8,192 tokens 1,177 to
// 1,221 (1.05 to 1.09 PFLOP/s), heads of 128; 8 tails of 128 to 1,024 tokens on 2 prefixes, heads of
// 64, 346 to 360 (730 to 760 TFLOP/s).
#include "dm_attn.h"

namespace dm {
namespace {

// Values of 128 elements: both kinds of tiles in one kernel, two workgroups a compute unit.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, 2) void diff_kernel(DiffIn a, const PlanView pv, uint64_t part_rows,
                                                           uint32_t* status)
{
    // as attn_kernel's; the second maps' rows at the end take half of it
    __shared__ __attribute__((aligned(512))) uint16_t lds[4 * kWideKeys * D];
    __shared__ uint32_t odd_tile;
    __shared__ Joined<kWaves> joined;
    Unit u;
    if (!item_unit(a, pv, a.b.groups + a.b.n, part_rows, D, kWide, status, u))
        return;
    bool bad = false;
    const uint32_t x = blockIdx.x - u.item0;
    if (u.flags & kUnitWide)
        wide_tile<T, D, true, kWaves, false>(a, make_tile(a, u, x, kWide), lds, &odd_tile, bad);
    else
        narrow_tile<T, D, kWaves, true>(a, make_tile(a, u, x, kNarrow), lds, joined, bad);
    if (bad)
        atomicOr(status, kErrInval);
}

// Values of 256: a wide tile's keys and values leave LDS room for one workgroup a compute
// unit, which so has eight waves, two a SIMD, and 256 rows.  Narrow tiles, held apart, need
// half of that a workgroup, so that two are on a compute unit and one reads while another
// begins or ends: they have a kernel of their own.  (64 rows on up to 8,192 keys, 32 query and 8
// key heads: 222 us; in one kernel of eight waves 246, of four, keys and values together, 225.)
constexpr int kTallWaves = 8;
constexpr uint32_t kTall = 32 * kTallWaves;

template <typename T, int D>
__global__ __launch_bounds__(kTallWaves* kWave, 1) void diff_tall_kernel(DiffIn a, const PlanView pv, uint64_t part_rows,
                                                                         uint32_t* status)
{
    __shared__ __attribute__((aligned(512))) uint16_t lds[4 * kWideKeys * D];  // the second maps' rows too
    __shared__ uint32_t odd_tile;
    Unit u;
    if (!item_unit(a, pv, a.b.groups + a.b.n, part_rows, D, kTall, status, u) || !(u.flags & kUnitWide))
        return;
    bool bad = false;
    wide_tile<T, D, true, kTallWaves, false>(a, make_tile(a, u, blockIdx.x - u.item0, kTall), lds, &odd_tile, bad);
    if (bad)
        atomicOr(status, kErrInval);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 2) void diff_narrow_kernel(DiffIn a, const PlanView pv, uint64_t part_rows,
                                                                  uint32_t wide, uint32_t* status)
{
    __shared__ __attribute__((aligned(16))) uint16_t lds[kWaves * kNarrowKeys * D];
    __shared__ Joined<kWaves> joined;
    Unit u;
    if (!item_unit(a, pv, a.b.groups + a.b.n, part_rows, D, wide, status, u) || (u.flags & kUnitWide))
        return;
    bool bad = false;
    narrow_tile<T, D, kWaves, true, true>(a, make_tile(a, u, blockIdx.x - u.item0, kNarrow), lds, joined, bad);
    if (bad)
        atomicOr(status, kErrInval);
}

// A few rows on a few keys, as attn_small_kernel.
template <typename T, int D>
__global__ __launch_bounds__(kSmallWaves<D>* kWave, 1) void diff_small_kernel(DiffIn a, const PlanView pv,
                                                                              uint32_t wide, uint32_t* status)
{
    constexpr int kW = kSmallWaves<D>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[kW * 2 * kNarrowKeys * D];
    __shared__ Joined<kW> joined;
    Unit u;
    if (!item_unit(a, pv, a.b.n, 0, D, wide, status, u))
        return;
    bool bad = false;
    narrow_tile<T, D, kW, true>(a, make_tile(a, u, blockIdx.x - u.item0, kNarrow), lds, joined, bad);
    if (bad)
        atomicOr(status, kErrInval);
}

// Rows in parts where they are few: a workgroup for a pair of rows, half of its waves a map,
// each with every second or fourth part; eight parts' rows are read at once.  Eight waves where
// pairs are fewer than two a compute unit (18 pairs in up to 190 parts: 73 to 58 us with the
// pass), four otherwise (1,024 pairs: 222 us, with eight 226).
template <typename T, int D, int JOIN>
__global__ __launch_bounds__(JOIN* kWave) void diff_join_kernel(DiffIn a, const PlanView pv, uint64_t part_rows,
                                                             uint32_t wide, uint32_t items)
{
    constexpr int kPer = D / kWave, kAtOnce = 8, kEach = JOIN / 2;
    typedef float vper __attribute__((ext_vector_type(kPer)));
    __shared__ vper rows[JOIN][kWave];
    __shared__ v2f stats[JOIN];
    const PlanHead& ph = *pv.head;
    if (ph.part_rows == 0 || !plan_fits(ph, a, part_rows, D, wide, items))
        return;
    const uint32_t wave = threadIdx.x / kWave, lane = lane_id(), map = wave % 2;
    const uint32_t pairs = a.q_heads / 2, all = a.b.q_tokens * pairs;
    for (uint32_t y = blockIdx.x; y < all; y += gridDim.x) {
        const uint32_t t = y / pairs, x = y % pairs * 2;
        const Parts p = parts_of(pv.unit[a.b.groups + sequence_of(a.b, t)], t, x + map, a.ratio);
        if (p.n == 0)  // (both maps, all waves)
            continue;
        float m = -INFINITY, total = 0;
        vper v = {};
        for (uint32_t i0 = wave / 2; i0 < p.n; i0 += kEach * kAtOnce) {
            v2f e[kAtOnce];
            vper r[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                const uint64_t at = p.at(i0 + kEach * j < p.n ? i0 + kEach * j : p.n - 1);
                e[j] = a.part_stat[at];
                r[j] = *reinterpret_cast<const vper*>(a.part + at * D + lane * kPer);
            }
            float now = m;
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                if (i0 + kEach * j >= p.n)
                    e[j] = v2f{-INFINITY, 0};
                now = fmaxf(now, e[j][0]);
            }
            const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - now) * a.scale2);
            m = now;
            total *= keep;
            v *= keep;
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                const float w = part_weight(e[j], m, a.scale2);
                total += w;
#pragma unroll
                for (int c = 0; c < kPer; c++)
                    v[c] = w == 0 ? v[c] : __builtin_fmaf(w, r[j][c], v[c]);
            }
        }
        __syncthreads();
        rows[wave][lane] = v;
        if (lane == 0)
            stats[wave] = v2f{m, total};
        __syncthreads();
        if (wave)
            continue;
        // wave 0: both maps, from half of the waves each
        vper o[2];
        const float lambda = a.lambda[x / 2];
#pragma unroll
        for (uint32_t map1 = 0; map1 < 2; map1++) {
            float top = -INFINITY, sum = 0;
#pragma unroll
            for (uint32_t k = 0; k < kEach; k++)
                top = fmaxf(top, stats[map1 + 2 * k][0]);
            o[map1] = vper{};
#pragma unroll
            for (uint32_t k = 0; k < kEach; k++) {
                const v2f e = stats[map1 + 2 * k];
                // (one that saw nothing has zeros, one that saw NaN only has a sum of NaN)
                const float by = e[0] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((e[0] - top) * a.scale2);
                sum += e[1] * by;
                o[map1] += rows[map1 + 2 * k][lane] * by;
            }
            const bool seen = sum > 0 || sum != sum;
            o[map1] *= seen ? 1.0f / sum : 0.0f;
            if (lane == 0 && a.lse)
                a.lse[(uint64_t)t * a.q_heads + x + map1] = seen ? lse_of<T>(top, sum, a.scale2) : -INFINITY;
        }
        float ss = 0;
#pragma unroll
        for (int c = 0; c < kPer; c++) {
            v[c] = __builtin_fmaf(-lambda, o[1][c], o[0][c]);
            ss = __builtin_fmaf(v[c], v[c], ss);
        }
        float by = a.gain;
        typedef T vt __attribute__((ext_vector_type(kPer)));
        vt z;
        if (a.norm) {
#pragma unroll
            for (int o = 1; o < kWave; o *= 2)
                ss += __shfl_xor(ss, o);
            by *= norm_of<D>(ss, a.eps);
            z = *reinterpret_cast<const vt*>(a.norm + lane * kPer);
        }
#pragma unroll
        for (int c = 0; c < kPer; c++)
            z[c] = (T)(v[c] * by * (a.norm ? (float)z[c] : 1.0f));
        *reinterpret_cast<vt*>(a.out + t * a.out_stride + (uint64_t)x * (D / 2) + lane * kPer) = z;
    }
}

// Where they are more than the places of waves: four rows a wave (as attn_join_kernel).
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void diff_join_many_kernel(DiffIn a, const PlanView pv, uint64_t part_rows,
                                                                  uint32_t wide, uint32_t items)
{
    const PlanHead& ph = *pv.head;
    if (ph.part_rows == 0 || !plan_fits(ph, a, part_rows, D, wide, items))
        return;
    const uint64_t all = (uint64_t)a.b.q_tokens * a.q_heads, step = (uint64_t)gridDim.x * kWaves;
    const uint64_t per = ((all + step - 1) / step + 3) / 4 * 4;
    const uint64_t y0 = ((uint64_t)blockIdx.x * kWaves + threadIdx.x / kWave) * per;
    join_quarters<T, D, true>(a, pv, y0, y0 + per < all ? y0 + per : all);
}

}  // namespace

// Attention's view of a store of pairs.
dm_kv_pages pairs_of(const dm_kv_pages& kv)
{
    dm_kv_pages p = kv;
    p.kv_heads = kv.kv_heads / 2;
    p.head_dim = kv.head_dim * 2;
    return p;
}

// Heads of 128: where sequences have no more rows a pair than a narrow tile on average, and
// no runs, every tile is narrow, and one kernel has them all.  (The other one's workgroups
// would have been there only to see that they have nothing to do.)  By the mean: a chunk of 64
// tokens beside 63 single ones, 32 query and 8 key heads, 8,192 keys each, is 32 narrow tiles for
// a pair, each reading the chunk's keys: 473 us, the 63 alone 380.
uint32_t diff_wide(const dm_kv_pages& kv, const dm_token_batch& b, uint32_t q_heads)
{
    if (kv.head_dim != 128)
        return kWide;
    return b.groups == 0 && b.q_tokens * (q_heads / (kv.kv_heads / 2)) <= kNarrowRows * b.tables.n ? kNarrow : kTall;
}

hipError_t diff_attn(dm_ctx* c, const dm_token_batch& b, const dm_kv_pages& store, uint32_t q_heads,
                     const void* plan, uint32_t layer, const dm_diff_args& g)
{
    const dm_kv_pages kv = pairs_of(store);
    const uint32_t ratio = q_heads / kv.kv_heads;
    const bool is_small = small(c, b, kv, ratio);
    const uint64_t rows = is_small ? 0 : part_rows_of(c, b, q_heads);
    hipError_t e;
    float* part =
        is_small ? nullptr : static_cast<float*>(scratch_get(c, kSlotPages, rows * (kv.head_dim + 2) * 4, &e));
    if (!part && !is_small)
        return e;
    DiffIn a;
    a.b = token_batch(c, b);
    a.k = static_cast<const uint16_t*>(kv.k) + (uint64_t)layer * kv.layer_stride;
    a.v = static_cast<const uint16_t*>(kv.v) + (uint64_t)layer * kv.layer_stride;
    a.q = static_cast<const uint16_t*>(g.q);
    a.out = static_cast<uint16_t*>(g.out);
    a.lse = g.lse;
    a.part = part;
    a.part_stat = is_small ? nullptr : reinterpret_cast<v2f*>(part + rows * kv.head_dim);
    a.q_stride = g.q_stride;
    a.out_stride = g.out_stride;
    a.n_pages = kv.n_pages;
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.ratio = ratio;
    a.scale2 = g.scale * kLog2e;
    a.lambda = g.lambda;
    a.norm = static_cast<const uint16_t*>(g.norm);
    a.eps = g.eps;
    a.gain = g.gain;
    const PlanView pv = plan_view(const_cast<void*>(plan), b.tables.n, b.groups);
    const uint32_t wide = diff_wide(store, b, q_heads);
    const uint64_t most = is_small ? (uint64_t)b.tables.n * kv.kv_heads : most_items(c, b, ratio, kv.kv_heads, wide);
    if (most > 0x7FFFFFFFull)
        return hipErrorInvalidValue;
    auto launch = [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        if (is_small) {
            diff_small_kernel<T, D><<<(uint32_t)most, kSmallWaves<D> * kWave, 0, c->stream>>>(a, pv, wide, c->d_status);
            return;
        }
        if constexpr (D == 256) {
            if (wide == kTall)
                diff_tall_kernel<T, D><<<(uint32_t)most, kTallWaves * kWave, 0, c->stream>>>(a, pv, rows, c->d_status);
            diff_narrow_kernel<T, D><<<(uint32_t)most, kThreads, 0, c->stream>>>(a, pv, rows, wide, c->d_status);
        } else {
            diff_kernel<T, D><<<(uint32_t)most, kThreads, 0, c->stream>>>(a, pv, rows, c->d_status);
        }
        const uint64_t outs = b.q_tokens * q_heads;
        if (outs > 8ull * c->n_cu * kWaves)
            diff_join_many_kernel<T, D><<<4u * c->n_cu, kThreads, 0, c->stream>>>(a, pv, rows, wide, (uint32_t)most);
        else if (outs > 4ull * c->n_cu)
            diff_join_kernel<T, D, 4>
                <<<grid_for(outs / 2, 1, 8u * c->n_cu), 4 * kWave, 0, c->stream>>>(a, pv, rows, wide, (uint32_t)most);
        else
            diff_join_kernel<T, D, 8>
                <<<(uint32_t)(outs / 2), 8 * kWave, 0, c->stream>>>(a, pv, rows, wide, (uint32_t)most);
    };
    auto dims = [&](auto t) {
        if (kv.head_dim == 128)
            launch(t, std::integral_constant<int, 128>{});
        else
            launch(t, std::integral_constant<int, 256>{});
    };
    if (kv.dtype == DM_BF16)
        dims(__bf16{});
    else
        dims(_Float16{});
    return hipGetLastError();
}

}  // namespace dm
