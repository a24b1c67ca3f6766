// What the kernels over KV pages share: a batch's sequences and element types.
#pragma once

#include <type_traits>

#include "dm_internal.h"

namespace dm {

typedef uint32_t v4u32 __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8hf __attribute__((ext_vector_type(8)));

// Eight neighbouring elements, and element pairs of products on the matrix
// cores, by type.
template <typename T>
struct Vec8;
template <>
struct Vec8<__bf16> {
    using type = v8bf;
};
template <>
struct Vec8<_Float16> {
    using type = v8hf;
};

// Rounds to nearest, ties to even.
template <typename T>
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8])
{
    using V = typename Vec8<T>::type;
    V v;
#pragma unroll
    for (int i = 0; i < 8; i++)
        v[i] = (T)x[i];
    *reinterpret_cast<V*>(p) = v;
}

// f(element type, head size) for the pair that the caller has checked.
template <typename F>
void by_type(uint32_t dtype, uint32_t head_dim, F&& f)
{
    auto dims = [&](auto t) {
        if (head_dim == 64)
            f(t, std::integral_constant<int, 64>{});
        else if (head_dim == 128)
            f(t, std::integral_constant<int, 128>{});
        else
            f(t, std::integral_constant<int, 256>{});
    };
    if (dtype == DM_BF16)
        dims(__bf16{});
    else
        dims(_Float16{});
}

// dm_token_batch as the kernels take it.
struct TokenBatch {
    const int64_t* off;
    const int32_t* page;
    const int64_t* len;
    const int64_t* q_off;
    const int64_t* group_off;
    int64_t entries;
    uint32_t n, q_tokens, groups;
    uint32_t shift;  // log2(B)
};

inline TokenBatch token_batch(const dm_ctx* c, const dm_token_batch& b)
{
    uint32_t shift = 0;
    while ((1u << shift) < c->cfg.block_size)
        shift++;
    return TokenBatch{b.tables.off, b.tables.page,           b.tables.len,
                      b.q_off,      b.group_off,             (int64_t)b.tables.entries,
                      (uint32_t)b.tables.n, (uint32_t)b.q_tokens, (uint32_t)b.groups, shift};
}

// Words that workgroups on other dies write or read within a launch: written
// through, and read where they arrive.
__device__ __forceinline__ void agent_store(uint32_t* p, uint32_t x)
{
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t agent_load(const uint32_t* p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A launch's workgroups, done with their agent_store()s, count themselves in
// (*arrived: zero before the launch): true for the whole of the last one, which
// finds the words of all others by agent_load().  Every wave waits for its own
// stores: a barrier waits for LDS only, and what thread 0 then orders is its own
// wave's memory.  (A fence by every wave instead: 60 us in 256 workgroups.)
// word: one of LDS.
__device__ __forceinline__ bool last_to_arrive(uint32_t* arrived, uint32_t* word)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
        *word = atomicAdd(arrived, 1u);
    }
    __syncthreads();
    return *word == gridDim.x - 1;
}

// The last i with at[i * stride] <= x, in [0, n); 0 if there is none (n >= 1, at
// non-decreasing).  A wave together, 64 places a step; every lane active, x
// uniform.
template <typename I, typename X>
__device__ __forceinline__ uint32_t wave_find(const I* at, uint32_t n, uint32_t stride, X x)
{
    uint32_t lo = 0;
    while (n > 1) {
        const uint32_t step = (n + kWave - 1) / kWave, i = lane_id() * step;
        const bool le = i < n && at[(uint64_t)(lo + i) * stride] <= (I)x;
        const uint32_t k = __popcll(ballot(le));
        const uint32_t skip = k ? (k - 1) * step : 0;
        lo += skip;
        n = k == 0 ? 1 : n - skip < step ? n - skip : step;
    }
    return lo;
}

// The sequence whose new tokens t is among (if q_off is in order).  In a decode
// step token t is sequence t's, which one look confirms.
__device__ __forceinline__ uint32_t sequence_of(const TokenBatch& b, uint32_t t)
{
    if (t < b.n && b.q_off[t] == (int64_t)t && b.q_off[t + 1] == (int64_t)t + 1)
        return t;
    return b.n ? wave_find(b.q_off, b.n, 1, (int64_t)t) : 0;
}

// A sequence of the batch.  A malformed one has length 0 (bad set), and no new
// tokens if it is its q_off that is malformed.
struct SeqView {
    int64_t off, len, pos0;  // first entry, tokens, position of the first new token
    uint32_t tok0, ntok;
    bool bad;
    __device__ bool covers(uint32_t t) const { return t - tok0 < ntok; }
};

__device__ __forceinline__ SeqView sequence_view(const TokenBatch& b, uint32_t s)
{
    SeqView v{0, 0, 0, 0, 0, false};
    if (s >= b.n)
        return v;
    const int64_t q0 = b.q_off[s], q1 = b.q_off[s + 1];
    const int64_t o0 = b.off[s], o1 = b.off[s + 1], len = b.len[s];
    if (q0 < 0 || q1 < q0 || q1 > (int64_t)b.q_tokens) {
        v.bad = true;
        return v;
    }
    v.tok0 = (uint32_t)q0;
    v.ntok = (uint32_t)(q1 - q0);
    v.bad = o0 < 0 || o1 < o0 || o1 > b.entries || len < 0 || len >= (1ll << 31) ||
            ((len + (1ll << b.shift) - 1) >> b.shift) > o1 - o0;
    v.off = v.bad ? 0 : o0;
    v.len = v.bad ? 0 : len;
    v.pos0 = v.len - (int64_t)v.ntok;
    return v;
}

}  // namespace dm
