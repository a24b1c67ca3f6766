// New tokens of a batch: queries and keys normed over each head and rotated
// by their positions in one pass, keys and values written to their pages.
//
// Bound by HBM: every element is read once and written once (16 bytes a lane),
// everything between stays in registers.  A head is D / 8 neighbouring lanes, so
// its mean square is a few lane exchanges and the partner of a rotated pair is
// in the lane itself or D_rot / 16 lanes on.
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
};

// Eight neighbouring elements of a head, d0 the first one's place: normed
// (weight w, if any) and rotated.  cs, sn: the lane's cosines and sines.
template <int D, bool INTERLEAVED>
__device__ __forceinline__ void norm_rotate(float (&x)[8], const float* w, float eps, uint32_t rot,
                                            uint32_t d0, const float (&cs)[8], const float (&sn)[8])
{
    if (w) {
        float ss = 0;
#pragma unroll
        for (int i = 0; i < 8; i++)
            ss += x[i] * x[i];
#pragma unroll
        for (int o = 1; o < D / 8; o *= 2)
            ss += __shfl_xor(ss, o);
        const float r = rsqrtf(ss * (1.0f / D) + eps);
#pragma unroll
        for (int i = 0; i < 8; i++)
            x[i] = x[i] * r * w[i];
    }
    if (!rot)
        return;
    if (INTERLEAVED) {
        if (d0 < rot) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float a = x[i], b = x[i + 1];
                x[i] = a * cs[i / 2] - b * sn[i / 2];
                x[i + 1] = b * cs[i / 2] + a * sn[i / 2];
            }
        }
    } else {
        const bool low = d0 < rot / 2;
        const int from = lane_id() + (low ? (int)(rot / 16) : -(int)(rot / 16));
#pragma unroll
        for (int i = 0; i < 8; i++) {
            // every lane takes part; those past the rotated part keep their own
            const float y = __shfl(x[i], d0 < rot ? from : lane_id());
            if (d0 < rot)
                x[i] = x[i] * cs[i] + (low ? -y : y) * sn[i];
        }
    }
}

// A workgroup for a token; its waves take 512 / D heads at a time.
template <typename T, int D, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendIn a, uint32_t* status)
{
    constexpr int kLanes = D / 8, kHeads = kWave / kLanes;
    const uint32_t li = threadIdx.x % kLanes, hi = threadIdx.x / kLanes;  // lane of a head, head
    const uint32_t d0 = li * 8;
    float wq[8], wk[8];
    if (a.q_norm)
        load8<T>(a.q_norm + d0, wq);
    if (a.k_norm)
        load8<T>(a.k_norm + d0, wk);
    const uint32_t heads = a.q_heads + 2 * a.kv_heads;
    for (uint32_t t = blockIdx.x; t < a.b.q_tokens; t += gridDim.x) {
        const uint32_t s = sequence_of(a.b, t);
        const SeqView sv = sequence_view(a.b, s);
        if (sv.bad && threadIdx.x == 0)
            atomicOr(status, kErrInval);
        if (s >= a.b.n || !sv.covers(t))
            continue;  // a token of no sequence: its row is not written
        const int64_t pos = sv.pos0 + (t - sv.tok0);
        int64_t place = -1;  // the token's row of the pages, for KV head 0
        bool bad = sv.bad;
        if (!bad && pos >= 0) {
            const uint32_t p = (uint32_t)a.b.page[sv.off + (pos >> a.b.shift)];
            bad = p >= a.n_pages || (a.rot && (uint64_t)pos >= a.max_pos);
            if (!bad)
                place = ((int64_t)p * a.kv_heads << a.b.shift) + (pos & ((1 << a.b.shift) - 1));
        }
        if (bad && !sv.bad && threadIdx.x == 0)
            atomicOr(status, kErrInval);
        float cs[8], sn[8];
        if (place >= 0 && a.rot && d0 < a.rot) {
            const uint32_t half = a.rot / 2;
            const uint64_t at = (uint64_t)pos * half +
                                (INTERLEAVED ? d0 / 2 : d0 < half ? d0 : d0 - half);
#pragma unroll
            for (int i = 0; i < (INTERLEAVED ? 4 : 8); i += 4) {
                const float4 c4 = *reinterpret_cast<const float4*>(a.cos + at + i);
                const float4 s4 = *reinterpret_cast<const float4*>(a.sin + at + i);
                cs[i] = c4.x, cs[i + 1] = c4.y, cs[i + 2] = c4.z, cs[i + 3] = c4.w;
                sn[i] = s4.x, sn[i + 1] = s4.y, sn[i + 2] = s4.z, sn[i + 3] = s4.w;
            }
        }
        // whole waves go through the loop: lanes of a wave exchange values
        for (uint32_t h0 = hi / kHeads * kHeads; h0 < heads; h0 += kThreads / kLanes) {
            const uint32_t h = h0 + hi % kHeads;
            const bool is_q = h < a.q_heads, is_k = !is_q && h < a.q_heads + a.kv_heads;
            const uint32_t hk = is_q ? h : is_k ? h - a.q_heads : h - a.q_heads - a.kv_heads;
            float x[8] = {};
            if (h < heads && place >= 0) {
                const uint16_t* from = is_q   ? a.q + t * a.q_stride
                                       : is_k ? a.k + t * a.k_stride
                                              : a.v + t * a.v_stride;
                if (!is_q && !is_k) {
                    *reinterpret_cast<v4u32*>(a.v_pages + (place + ((int64_t)hk << a.b.shift)) * D + d0) =
                        *reinterpret_cast<const v4u32*>(from + (uint64_t)hk * D + d0);
                } else {
                    load8<T>(from + (uint64_t)hk * D + d0, x);
                }
            }
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                w[i] = is_q ? (a.q_norm ? wq[i] : 1.0f) : (a.k_norm ? wk[i] : 1.0f);
            // the branch is uniform: with one norm alone the other heads' mean
            // square is taken and not used
            if (a.q_norm || a.k_norm) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; i++)
                    y[i] = x[i];
                norm_rotate<D, INTERLEAVED>(y, w, a.eps, 0, d0, cs, sn);
                if (is_q ? a.q_norm != nullptr : a.k_norm != nullptr)
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        x[i] = y[i];
            }
            if (place >= 0)
                norm_rotate<D, INTERLEAVED>(x, nullptr, 0.0f, a.rot, d0, cs, sn);
            if (h >= heads)
                continue;
            if (is_q)
                store8<T>(a.q_out + t * a.q_out_stride + (uint64_t)hk * D + d0, x);
            else if (is_k && place >= 0)
                store8<T>(a.k_pages + (place + ((int64_t)hk << a.b.shift)) * D + d0, x);
        }
    }
}

}  // namespace

hipError_t kv_append(dm_ctx* c, const dm_kv_pages& kv, uint32_t layer, const dm_token_batch& b,
                     const dm_append_args& g)
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
    const uint32_t grid = grid_for(b.q_tokens, 1);
    by_type(kv.dtype, kv.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        if (g.interleaved)
            append_kernel<T, D, true><<<grid, kThreads, 0, c->stream>>>(a, c->d_status);
        else
            append_kernel<T, D, false><<<grid, kThreads, 0, c->stream>>>(a, c->d_status);
    });
    return hipGetLastError();
}

}  // namespace dm
