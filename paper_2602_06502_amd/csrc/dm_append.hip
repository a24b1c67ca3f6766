// New tokens of a batch: queries and keys normed over each head and rotated
// by their positions in one pass, keys and values written to their pages.
//
// Bound by HBM: every element is read once and written once, everything between
// stays in registers.  A head is D / 8 neighbouring lanes of eight elements, 16
// bytes: its mean square is a few register exchanges between neighbouring lanes,
// and the other half of its rotated pairs is in the lane itself or D_rot / 16
// lanes on, from where the lane gets it as it was read.  (Two runs of four
// elements a lane, so that every pair is in one lane, need no exchange, but
// accesses of 8 bytes: 167 us instead of 117 for 18,700 tokens of 48 heads.)  A
// token's steps wait for one another (its sequence, page, rotation), so its
// rows, which do not depend on them, are all read first.
#include "dm_internal.h"
#include "dm_pages.h"

namespace dm {
namespace {

constexpr int kThreads = 256;

struct AppendIn {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    uint16_t* q_out;
    int64_t q_out_stride;
    const uint16_t *q_norm, *k_norm;
    const float *cos, *sin;
    uint64_t max_pos;
    uint32_t q_heads, kv_heads, rot;
    float eps;
    uint16_t *k_pages, *v_pages;  // the layer's
    uint32_t n_pages;
    TokenBatch b;
    const int64_t* first;  // AT: positions of the sequences' first new tokens
};

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL,
                                                                     0xF, 0xF, true));
}

// Sum over a head's D / 8 lanes, in each of them.
template <int D>
__device__ __forceinline__ float head_sum(float x)
{
    x = dpp_add<0xB1>(x);   // neighbours
    x = dpp_add<0x4E>(x);   // pairs
    x = dpp_add<0x141>(x);  // fours, mirrored within eight lanes
    if (D >= 128)
        x = dpp_add<0x140>(x);  // eights, mirrored within sixteen
    if (D >= 256)
        x += __shfl_xor(x, 16);
    return x;
}

// row[i] * r * w[i].
template <typename T>
__device__ __forceinline__ void scaled(const typename Vec8<T>::type& row, float r,
                                       const typename Vec8<T>::type& w, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++)
        x[i] = (float)row[i] * r * (float)w[i];
}

// A workgroup for a token; a wave takes 512 / D heads at a time, all queries,
// keys or values, kAhead times read before the first is worked on.
constexpr int kAhead = 3;

// AT: positions are given.  (A kernel of its own: with a look at a.first in one for both, 18,283
// tokens take 101.5 us, without 100.4.)
template <typename T, int D, bool INTERLEAVED, bool AT>
__global__ __launch_bounds__(kThreads, 6) void append_kernel(AppendIn a, uint32_t* status)
{
    using V = typename Vec8<T>::type;
    constexpr uint32_t kLanes = D / 8, kHeads = kWave / kLanes, kWaves = kThreads / kWave;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t li = threadIdx.x % kLanes, hi = lane_id() / kLanes;  // lane of a head, head
    const uint32_t d0 = li * 8, half = a.rot / 2;
    const bool turns = d0 < a.rot, low = d0 < half;
    // where the other half of the lane's pairs is
    const int other = (int)lane_id() + (INTERLEAVED || !turns ? 0 : low ? (int)(half / 8) : -(int)(half / 8));
    const uint32_t e0 = INTERLEAVED || !turns ? d0 : low ? d0 + half : d0 - half;
    const uint32_t gq = (a.q_heads + kHeads - 1) / kHeads, gk = (a.kv_heads + kHeads - 1) / kHeads;
    const uint32_t groups = gq + 2 * gk;
    for (uint32_t t = blockIdx.x; t < a.b.q_tokens; t += gridDim.x) {
        V rows[kAhead];
        auto fetch = [&](uint32_t g) -> V {
            const bool is_q = g < gq, is_v = g >= gq + gk;
            const uint32_t h = (g - (is_q ? 0 : is_v ? gq + gk : gq)) * kHeads + hi;
            const uint32_t n = is_q ? a.q_heads : a.kv_heads;
            const uint16_t* from = is_q   ? a.q + t * a.q_stride
                                   : is_v ? a.v + t * a.v_stride
                                          : a.k + t * a.k_stride;
            return *reinterpret_cast<const V*>(from + (uint64_t)(h < n ? h : n - 1) * D + d0);
        };
#pragma unroll
        for (int i = 0; i < kAhead; i++)
            rows[i] = fetch(wave + i * kWaves);
        const uint32_t s = sequence_of(a.b, t);
        const SeqView sv = sequence_view(a.b, s);
        if (sv.bad && threadIdx.x == 0)
            atomicOr(status, kErrInval);
        if (s >= a.b.n || !sv.covers(t))
            continue;  // a token of no sequence: its row is not written
        const int64_t pos = sv.pos0 + (t - sv.tok0);
        int64_t place = -1;  // the token's row of the pages, for KV head 0
        float cs[8], sn[8];
#pragma unroll
        for (int i = 0; i < 8; i++)
            cs[i] = 1, sn[i] = 0;
        if (!sv.bad && pos >= 0) {
            const uint32_t p = (uint32_t)a.b.page[sv.off + (pos >> a.b.shift)];
            const int64_t turn = AT ? a.first[s] + (t - sv.tok0) : pos;
            const bool past = a.rot && (uint64_t)turn >= a.max_pos;
            if (!past && turns) {
                const uint64_t at = (uint64_t)turn * half + (INTERLEAVED ? d0 / 2 : low ? d0 : d0 - half);
#pragma unroll
                for (int i = 0; i < (INTERLEAVED ? 4 : 8); i += 4) {
                    const float4 c4 = *reinterpret_cast<const float4*>(a.cos + at + i);
                    const float4 s4 = *reinterpret_cast<const float4*>(a.sin + at + i);
                    cs[i] = c4.x, cs[i + 1] = c4.y, cs[i + 2] = c4.z, cs[i + 3] = c4.w;
                    sn[i] = s4.x, sn[i + 1] = s4.y, sn[i + 2] = s4.z, sn[i + 3] = s4.w;
                }
                if (!INTERLEAVED && low)
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        sn[i] = -sn[i];
            }
            if (p < a.n_pages && !past)
                place = ((int64_t)p * a.kv_heads << a.b.shift) + (pos & ((1 << a.b.shift) - 1));
            else if (threadIdx.x == 0)
                atomicOr(status, kErrInval);
        }
        // whole waves go through this: lanes of a wave exchange values
        auto work = [&](uint32_t g, const V& row) {
            const bool is_q = g < gq, is_v = g >= gq + gk;
            const uint32_t h = (g - (is_q ? 0 : is_v ? gq + gk : gq)) * kHeads + hi;
            const uint32_t n = is_q ? a.q_heads : a.kv_heads;
            if (place < 0 && !is_q)
                return;
            uint16_t* to = is_q ? a.q_out + t * a.q_out_stride + (uint64_t)h * D + d0
                                : (is_v ? a.v_pages : a.k_pages) +
                                      (place + ((int64_t)h << a.b.shift)) * D + d0;
            if (is_v || place < 0) {
                const V zero = {};
                if (h < n)
                    *reinterpret_cast<V*>(to) = is_v ? row : zero;
                return;
            }
            // the norm's weights of the lane's elements and of their partners
            const uint16_t* w = is_q ? a.q_norm : a.k_norm;
            V w0 = {1, 1, 1, 1, 1, 1, 1, 1}, w1 = w0;
            float r = 1.0f;
            if (w) {
                w0 = *reinterpret_cast<const V*>(w + d0);
                w1 = *reinterpret_cast<const V*>(w + e0);
                float ss = 0;
#pragma unroll
                for (int i = 0; i < 8; i++)
                    ss += (float)row[i] * (float)row[i];
                r = rsqrtf(head_sum<D>(ss) * (1.0f / D) + a.eps);
            }
            float x[8];
            scaled<T>(row, r, w0, x);
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const float u = x[i], v = x[i + 1];
                    // (a pair past the rotation is left as it is: 0 times infinity is NaN)
                    x[i] = turns ? u * cs[i / 2] - v * sn[i / 2] : u;
                    x[i + 1] = turns ? v * cs[i / 2] + u * sn[i / 2] : v;
                }
            } else if (a.rot) {
                const v4u32 mine = __builtin_bit_cast(v4u32, row);
                v4u32 far;
#pragma unroll
                for (int i = 0; i < 4; i++)
                    far[i] = __shfl(mine[i], other);
                float y[8];
                scaled<T>(__builtin_bit_cast(V, far), r, w1, y);
#pragma unroll
                for (int i = 0; i < 8; i++)
                    x[i] = turns ? x[i] * cs[i] + y[i] * sn[i] : x[i];
            }
            if (h < n)
                store8<T>(to, x);
        };
#pragma unroll
        for (int i = 0; i < kAhead; i++)
            if (wave + i * kWaves < groups)
                work(wave + i * kWaves, rows[i]);
        for (uint32_t g = wave + kAhead * kWaves; g < groups; g += kWaves)
            work(g, fetch(g));
    }
}

}  // namespace

hipError_t kv_append(dm_ctx* c, const dm_kv_pages& kv, uint32_t layer, const dm_token_batch& b,
                     const dm_append_args& g, const int64_t* first)
{
    AppendIn a;
    a.q = static_cast<const uint16_t*>(g.q);
    a.k = static_cast<const uint16_t*>(g.k);
    a.v = static_cast<const uint16_t*>(g.v);
    a.q_stride = g.q_stride;
    a.k_stride = g.k_stride;
    a.v_stride = g.v_stride;
    a.q_out = static_cast<uint16_t*>(g.q_out);
    a.q_out_stride = g.q_out_stride;
    a.q_norm = static_cast<const uint16_t*>(g.q_norm);
    a.k_norm = static_cast<const uint16_t*>(g.k_norm);
    a.cos = g.cos;
    a.sin = g.sin;
    a.max_pos = g.max_pos;
    a.q_heads = g.q_heads;
    a.kv_heads = kv.kv_heads;
    a.rot = g.rot_dim;
    a.eps = g.eps;
    a.k_pages = static_cast<uint16_t*>(kv.k) + (uint64_t)layer * kv.layer_stride;
    a.v_pages = static_cast<uint16_t*>(kv.v) + (uint64_t)layer * kv.layer_stride;
    a.n_pages = kv.n_pages;
    a.b = token_batch(c, b);
    a.first = first;
    const uint32_t grid = grid_for(b.q_tokens, 1);
    by_type(kv.dtype, kv.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        auto launch = [&](auto interleaved, auto at) {
            append_kernel<T, D, decltype(interleaved)::value, decltype(at)::value>
                <<<grid, kThreads, 0, c->stream>>>(a, c->d_status);
        };
        auto by_positions = [&](auto interleaved) {
            if (first)
                launch(interleaved, std::true_type{});
            else
                launch(interleaved, std::false_type{});
        };
        if (g.interleaved)
            by_positions(std::true_type{});
        else
            by_positions(std::false_type{});
    });
    return hipGetLastError();
}

}  // namespace dm
