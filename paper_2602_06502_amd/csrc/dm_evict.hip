// Eviction from KV pages by the weight that keys have collected: which tokens of a sequence
// stay within its budget, for each layer and each choice of KV heads, and their rows moved to
// the next tables' pages.
//
// The choice is the k-th largest of a sequence's scores, then one pass in order of position.
// A score is taken as a 32-bit number that orders as the float does; its digits of 11, 11
// and 10 bits are counted in LDS from the top, each time among the scores that agree with the
// digits found so far, so three passes give the k-th largest exactly, with how many of its
// equals stay (the first ones).  A workgroup takes a (layer, choice, sequence); its scores
// stay in registers where they fit; where choices are few and long, several take one.  Bound by
// reading the weights, three times where they are long (four histories of 27,000 to 124,000
// tokens, 8 layers, pairs of 8 heads: 70 us, 88 with a workgroup a choice; 86 MB a pass take 17),
// and for short sequences by the passes' barriers (16 chats, 4 layers, 8 heads: 12 us).
//
// The move takes a page of the new tables a workgroup: a row's token, that token's page, the
// row.  Bound by memory (16 histories of 2,048 to 8,192 tokens to 2,048, 4 layers, 8 heads of 128:
// 171 us, 4.6 TB/s).
#include <type_traits>

#include "dm_internal.h"
#include "dm_pages.h"

namespace dm {
namespace {

struct SelectIn {
    const int64_t *off, *len, *budget, *room;
    int64_t entries;
    const float* w;
    int64_t layer_stride, w_stride;
    int32_t* kept;
    int64_t kept_stride;
    int64_t *keep, *grow;
    uint32_t n, layers, choices, share, sink, recent, shift;
};

// A sequence's entries and tokens (none if it is malformed).
struct Held {
    int64_t off, len;
    bool bad;
};
__device__ __forceinline__ Held held(const int64_t* off, const int64_t* len, int64_t entries, uint32_t s, uint32_t shift)
{
    const int64_t o0 = off[s], o1 = off[s + 1], l = len[s];
    const bool bad = o0 < 0 || o1 < o0 || o1 > entries || l < 0 || l >= (1ll << 31) ||
                     ((l + (1ll << shift) - 1) >> shift) > o1 - o0;
    return Held{bad ? 0 : o0, bad ? 0 : l, bad};
}

// A score as a number that orders as it does, -0 as 0, NaN below all.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
    return x != x ? 0 : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Places of the digits: what is above them, and their widths.
constexpr int kDigits = 3, kBins = 2048;
__device__ __forceinline__ uint32_t digit_shift(int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit_mask(int d) { return d == 2 ? 1023 : 2047; }

template <int WAVES>
struct SelectLds {
    uint32_t bins[2][kBins];  // one is cleared while the other is looked at
    uint32_t above[WAVES];  // of a wave's bins, then of its scores
    uint32_t equal[WAVES], up[WAVES];
    uint32_t digit, left, held;
};

// The bin that the left-th score from the top is in, among those counted in bins: its number to
// lds.digit, the scores to be found in it to lds.left.  A thread has neighbouring bins.
template <int WAVES>
__device__ __forceinline__ void find_bin(SelectLds<WAVES>& lds, const uint32_t* bins, uint32_t left)
{
    const uint32_t tid = threadIdx.x, wave = tid / kWave;
    constexpr uint32_t kPer = kBins / (WAVES * kWave) ? kBins / (WAVES * kWave) : 1;
    const uint32_t top = kBins - 1 - tid * kPer;
    uint32_t own = 0;
#pragma unroll
    for (uint32_t b = 0; b < kPer; b++)
        own += bins[top - b];
    const uint32_t upto = (uint32_t)wave_incl_sum_u64(own, 0);
    if (lane_id() == kWave - 1)
        lds.above[wave] = upto;
    __syncthreads();
    uint32_t before = upto - own;
    for (uint32_t w = 0; w < wave; w++)
        before += lds.above[w];
    if (before < left && left <= before + own) {
        uint32_t b = top, x;
        while (before + (x = bins[b]) < left) {
            before += x;
            b--;
        }
        lds.digit = b;
        lds.left = left - before;
    }
    __syncthreads();
}

// The choice among n scores, of which k < n stay: each wave takes a stretch of them, R times
// 64, kept in registers.  keys(i, x): x[r] = score i + 64 r, any number where there is none.
template <int WAVES, int R, typename Keys>
__device__ __forceinline__ void choose(SelectLds<WAVES>& lds, uint32_t n, uint32_t k, int32_t first, int32_t* out,
                                       Keys&& keys)
{
    const uint32_t tid = threadIdx.x, wave = tid / kWave, lane = lane_id();
    const uint32_t begin = wave * R * kWave + lane;
    uint32_t mine[R];
    auto at = [&](uint32_t r) { return begin + r * kWave; };
    keys(begin, mine);
    // f(score, is there one, its place), step by step
    auto each = [&](auto&& f) {
#pragma unroll
        for (int r = 0; r < R; r++)
            f(mine[r], at(r) < n, at(r));
    };
    for (uint32_t b = tid; b < 2 * kBins; b += WAVES * kWave)
        lds.bins[0][b] = 0;
    __syncthreads();
    uint32_t found = 0, known = 0;  // the digits found, and their bits
    uint32_t left = k;              // to be found among those that agree with them
    for (int d = 0; d < kDigits; d++) {
        const uint32_t shift = digit_shift(d), mask = digit_mask(d);
        uint32_t* bins = lds.bins[d % 2];
        each([&](uint32_t x, bool there, uint32_t) {
            if (there && (x & known) == found)
                atomicAdd(&bins[(x >> shift) & mask], 1u);
        });
        __syncthreads();
        find_bin(lds, bins, left);
        found |= lds.digit << shift;
        known |= mask << shift;
        left = lds.left;
        if (d == 0)  // for the third digit
            for (uint32_t b = tid; b < kBins; b += WAVES * kWave)
                bins[b] = 0;
    }
    // found is the k-th largest; `left` of its equals stay.  Places of each wave's.
    uint32_t above = 0, equal = 0;
    each([&](uint32_t x, bool there, uint32_t) {
        above += __popcll(ballot(there && x > found));
        equal += __popcll(ballot(there && x == found));
    });
    if (lane == 0) {
        lds.above[wave] = above;
        lds.equal[wave] = equal;
    }
    __syncthreads();
    above = equal = 0;
    for (uint32_t w = 0; w < wave; w++) {
        above += lds.above[w];
        equal += lds.equal[w];
    }
    const uint64_t below = (1ull << lane) - 1;
    each([&](uint32_t x, bool there, uint32_t i) {
        const uint64_t up = ballot(there && x > found), same = ballot(there && x == found);
        const uint32_t e = equal + __popcll(same & below);
        // equals that stay before this one: the first `left` of all
        const uint32_t stayed = e < left ? e : left;
        const bool stays = there && (x > found || (x == found && e < left));
        if (stays)
            out[above + __popcll(up & below) + stayed] = first + (int32_t)i;
        above += __popcll(up);
        equal += __popcll(same);
    });
}

// More of them: read three times.  First for the highest digit; then for the scores that agree
// with it, of which LDS has room for kCandidates (where they are more, the other digits take a
// pass each) and how many are above them; then for the places.  A lane reads 16 bytes of
// scores at a time, kAtOnce times before the first is looked at: the reads of one workgroup
// are what bounds this (131,072 scores of two heads a choice, 128 choices: 160 us with 4 bytes
// and five passes).  keys4(i, x): x[4 u + j] = score i + 256 u + j.
template <int WAVES>
constexpr uint32_t kCandidates = WAVES * 512;
template <int WAVES, uint32_t kAtOnce, typename Keys4>
__device__ __forceinline__ void choose_long(SelectLds<WAVES>& lds, uint32_t* candidate, uint8_t* whose, uint32_t n,
                                            uint32_t k, int32_t first, int32_t* out, Keys4&& keys4)
{
    constexpr uint32_t kStep = 4 * kWave;
    const uint32_t tid = threadIdx.x, wave = tid / kWave, lane = lane_id();
    const uint32_t steps = (n + WAVES * kStep - 1) / (WAVES * kStep);
    const uint32_t begin = wave * steps * kStep;
    const uint64_t below = (1ull << lane) - 1;
    // f(four scores, place of the first) for the wave's steps; places from n on are none
    auto each = [&](auto&& f) {
        for (uint32_t r0 = 0; r0 < steps; r0 += kAtOnce) {
            uint32_t x[kAtOnce * 4];
            keys4(begin + r0 * kStep + lane * 4, x);
#pragma unroll
            for (uint32_t r = 0; r < kAtOnce; r++)
                if (r0 + r < steps)
                    f(&x[r * 4], begin + (r0 + r) * kStep + lane * 4);
        }
    };
    auto count = [&](int d, uint32_t x, uint32_t* bins) { atomicAdd(&bins[(x >> digit_shift(d)) & digit_mask(d)], 1u); };
    for (uint32_t b = tid; b < 2 * kBins; b += WAVES * kWave)
        lds.bins[0][b] = 0;
    if (tid == 0)
        lds.held = 0;
    if (tid < WAVES)
        lds.up[tid] = lds.equal[tid] = 0;
    __syncthreads();
    each([&](const uint32_t* x, uint32_t i) {
#pragma unroll
        for (uint32_t j = 0; j < 4; j++)
            if (i + j < n)
                count(0, x[j], lds.bins[0]);
    });
    __syncthreads();
    find_bin(lds, lds.bins[0], k);
    const uint32_t digit = lds.digit, many = lds.bins[0][digit];
    uint32_t left = lds.left, found = digit << digit_shift(0), known = digit_mask(0) << digit_shift(0);
    const bool fit = many <= kCandidates<WAVES>;
    if (fit) {
        uint32_t up = 0;
        each([&](const uint32_t* x, uint32_t i) {
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const bool there = i + j < n;
                up += __popcll(ballot(there && x[j] >> digit_shift(0) > digit));
                const uint64_t those = ballot(there && x[j] >> digit_shift(0) == digit);
                if (those == 0)
                    continue;
                uint32_t at = 0;
                if (lane == 0)
                    at = atomicAdd(&lds.held, (uint32_t)__popcll(those));
                at = __builtin_amdgcn_readfirstlane(at) + __popcll(those & below);
                if ((those >> lane) & 1) {
                    candidate[at] = x[j];
                    whose[at] = (uint8_t)wave;
                }
            }
        });
        if (lane == 0)
            lds.up[wave] = up;
    }
    for (int d = 1; d < kDigits; d++) {
        uint32_t* bins = lds.bins[d % 2];
        if (d == 2)  // (the first digit's)
            for (uint32_t b = tid; b < kBins; b += WAVES * kWave)
                bins[b] = 0;
        __syncthreads();
        if (fit) {
            for (uint32_t i = tid; i < many; i += WAVES * kWave)
                if ((candidate[i] & known) == found)
                    count(d, candidate[i], bins);
        } else {
            each([&](const uint32_t* x, uint32_t i) {
#pragma unroll
                for (uint32_t j = 0; j < 4; j++)
                    if (i + j < n && (x[j] & known) == found)
                        count(d, x[j], bins);
            });
        }
        __syncthreads();
        find_bin(lds, bins, left);
        found |= lds.digit << digit_shift(d);
        known |= digit_mask(d) << digit_shift(d);
        left = lds.left;
    }
    // found is the k-th largest; `left` of its equals stay.  Each wave's, above it and equal.
    if (fit) {
        for (uint32_t i = tid; i < many; i += WAVES * kWave) {
            if (candidate[i] > found)
                atomicAdd(&lds.up[whose[i]], 1u);
            else if (candidate[i] == found)
                atomicAdd(&lds.equal[whose[i]], 1u);
        }
    } else {
        uint32_t up = 0, equal = 0;
        each([&](const uint32_t* x, uint32_t i) {
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                up += __popcll(ballot(i + j < n && x[j] > found));
                equal += __popcll(ballot(i + j < n && x[j] == found));
            }
        });
        if (lane == 0) {
            lds.up[wave] = up;
            lds.equal[wave] = equal;
        }
    }
    __syncthreads();
    uint32_t above = 0, equal = 0;
    for (uint32_t w = 0; w < wave; w++) {
        above += lds.up[w];
        equal += lds.equal[w];
    }
    each([&](const uint32_t* x, uint32_t i) {
        // those before a lane's first, in the order of places: all of the lanes below it
        uint32_t up = above, same = equal;
#pragma unroll
        for (uint32_t j = 0; j < 4; j++) {
            const uint64_t more = ballot(i + j < n && x[j] > found), as = ballot(i + j < n && x[j] == found);
            up += __popcll(more & below);
            same += __popcll(as & below);
            above += __popcll(more);
            equal += __popcll(as);
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; j++) {
            if (i + j >= n || x[j] < found)
                continue;
            const bool over = x[j] > found;
            if (over || same < left)
                out[up + (same < left ? same : left)] = first + (int32_t)(i + j);
            up += over;
            same += !over;
        }
    });
}

// What a (layer, choice, sequence) is to choose: k of the n tokens from `first` on; none (k = 0)
// where the sequence is within its budget.
struct Pick {
    uint32_t len, first, tail, k, n;
    const float* w;  // of token `first`, of the choice's first head
    int32_t* out;    // the choice's first entry
    int64_t at;      // the sequence's first place
    bool past, malformed;  // (malformed: its table)
};
__device__ __forceinline__ Pick pick_of(const SelectIn& a, uint32_t x, bool& bad)
{
    const uint32_t s = x % a.n, c = x / a.n % a.choices, l = x / a.n / a.choices;
    const Held h = held(a.off, a.len, a.entries, s, a.shift);
    const int64_t budget = a.budget[s];
    Pick p{};
    bad = h.bad || budget < 0;
    p.len = (uint32_t)h.len;
    p.malformed = h.bad;
    p.past = !bad && h.len > budget;
    if (!p.past)
        return p;
    const uint32_t stay = (uint32_t)budget;
    p.first = stay < a.sink ? stay : a.sink;
    p.tail = stay - p.first < a.recent ? stay - p.first : a.recent;
    p.k = stay - p.first - p.tail;
    p.n = p.len - p.first - p.tail;
    p.at = h.off << a.shift;
    p.w = a.w + (int64_t)l * a.layer_stride + (int64_t)(c * a.share) * a.w_stride + p.at + p.first;
    p.out = a.kept + ((int64_t)l * a.choices + c) * a.kept_stride + p.at;
    return p;
}
// What needs no choosing: the first and the last tokens, and, once a sequence, the next tables'
// numbers.  Of a sequence whose table is malformed it is not known what it has: with a keep of 0
// alone the fork of other tables would free all of it before dm_sync is asked, so its grow is one
// that a fork refuses.  Room below 0 is refused alike.
__device__ __forceinline__ void settle(const SelectIn& a, const Pick& p, uint32_t x, bool bad, uint32_t threads,
                                       uint32_t* status)
{
    const uint32_t tid = threadIdx.x;
    if (x < a.n && tid == 0) {
        const int64_t room = a.room ? a.room[x] : 0;
        a.keep[x] = p.past ? 0 : p.len;
        a.grow[x] = p.malformed || room < 0 ? -1 : room + (p.past ? p.first + p.tail + p.k : 0);
        if (bad || room < 0)
            atomicOr(status, kErrInval);
    }
    if (!p.past)
        return;
    for (uint32_t i = tid; i < p.first; i += threads)
        p.out[i] = (int32_t)i;
    for (uint32_t i = tid; i < p.tail; i += threads)
        p.out[p.first + p.k + i] = (int32_t)(p.len - p.tail + i);
}

// Scores i + 256 u + j, to x[4 u + j], of those below `end`: 16 bytes of each head at a time.
template <bool WHOLE, uint32_t MANY>
__device__ __forceinline__ void scores4(const SelectIn& a, const float* w, uint32_t end, uint32_t i, uint32_t (&x)[MANY])
{
    typedef float v4 __attribute__((ext_vector_type(4), aligned(4)));
    v4 sum[MANY / 4], more[MANY / 4];
    // (waves within `end` read without a branch between their reads: the first pass of split choices
    // 24 to 21 us; one kernel by itself has no registers for it, 88 without and 100)
    const bool whole = WHOLE && __builtin_amdgcn_readfirstlane(i) + MANY * kWave <= end;
    auto read = [&](uint32_t g, v4 (&to)[MANY / 4]) {
        const float* from = w + g * a.w_stride;
        if (whole) {
#pragma unroll
            for (uint32_t u = 0; u < MANY / 4; u++)
                to[u] = *reinterpret_cast<const v4*>(from + i + u * 4 * kWave);
            return;
        }
#pragma unroll
        for (uint32_t u = 0; u < MANY / 4; u++) {
            const uint32_t p = i + u * 4 * kWave;
            to[u] = v4{};
            if (p + 3 < end) {
                to[u] = *reinterpret_cast<const v4*>(from + p);
            } else {
                for (uint32_t j = 0; j < 4; j++)
                    if (p + j < end)
                        to[u][j] = from[p + j];
            }
        }
    };
    read(0, sum);
    if (a.share > 1)
        read(1, more);  // (beside the first)
    for (uint32_t g = 1; g < a.share; g++) {
        if (g > 1)
            read(g, more);
#pragma unroll
        for (uint32_t u = 0; u < MANY / 4; u++)
            sum[u] = sum[u] + more[u];
    }
#pragma unroll
    for (uint32_t u = 0; u < MANY; u++)
        x[u] = ordered(sum[u / 4][u % 4]);
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void select_kernel(SelectIn a, uint32_t* status)
{
    constexpr int kW = THREADS / kWave;
    __shared__ SelectLds<kW> lds;
    __shared__ uint32_t candidate[kCandidates<kW>];
    __shared__ uint8_t whose[kCandidates<kW>];
    bool bad;
    const Pick p = pick_of(a, blockIdx.x, bad);
    settle(a, p, blockIdx.x, bad, THREADS, status);
    const uint32_t k = p.k, n = p.n, first = p.first;
    if (k == 0)
        return;
    const float* w = p.w;
    int32_t* out = p.out;
    // (head by head, so that reads need not wait for one another)
    auto keys = [&](uint32_t i, auto& x) {
        constexpr int kMany = sizeof(x) / sizeof(x[0]);
        float sum[kMany];
        for (uint32_t g = 0; g < a.share; g++) {
            const float* from = w + g * a.w_stride;
            float one[kMany];
#pragma unroll
            for (int r = 0; r < kMany; r++)
                one[r] = i + r * kWave < n ? from[i + r * kWave] : 0.0f;
#pragma unroll
            for (int r = 0; r < kMany; r++)
                sum[r] = g ? sum[r] + one[r] : one[r];
        }
#pragma unroll
        for (int r = 0; r < kMany; r++)
            x[r] = ordered(sum[r]);
    };
    if (n <= THREADS * 4)
        choose<kW, 4>(lds, n, k, (int32_t)first, out + first, keys);
    else if (n <= THREADS * 16)
        choose<kW, 16>(lds, n, k, (int32_t)first, out + first, keys);
    else
        choose_long<kW, THREADS == 1024 ? 4 : 1>(lds, candidate, whose, n, k, (int32_t)first, out + first,
                                                 [&](uint32_t i, auto& x) { scores4<false>(a, w, n, i, x); });
}

// Long histories where choices are too few to fill the chip: several workgroups a choice, each
// with a stretch of its scores, in three passes (the choice itself is the same):
//   count   each part's scores by their highest digit; sums of several heads are left for the
//           other passes (82 to 73 us);
//   list    every part adds these up, so it knows the digit of the k-th largest, how many
//           scores of the parts before it are above it and how many agree with it, and lists its
//           own ones that agree at their place in the choice's list;
//   place   every part finds the k-th largest among the list, and with it, as it reads its
//           scores a last time, their places.
// The last two read a round ahead, the first one beside the counts and the list (73 to 70 us).
constexpr int kPartThreads = 512, kPartWaves = kPartThreads / kWave;
constexpr uint32_t kRound = kPartThreads * 16;  // scores that a workgroup has in registers

struct Found {  // by the list pass, of a part
    uint32_t digit, left, many;  // the choice's
    uint32_t above, agree;       // of the parts before
    uint32_t mine;               // that agree, of the part
};
struct Split {
    uint32_t each;   // scores of a part, a multiple of 4
    uint32_t row;    // workgroups of a (layer, choice)
    uint32_t* bins;  // [workgroups][kBins]
    Found* found;    // [workgroups]
    uint32_t* list;  // [layers][choices], rows of `places`: where a sequence's scores are
    uint32_t* sums;  // alike, or null (one head a choice): scores, left by the first pass
    int64_t places;
};
// What a workgroup has: a stretch of a choice's scores, its number among the choice's `parts`.
struct Part {
    uint32_t x, part, parts, begin, end;
    Pick p;
    bool bad, there;
};
// A sequence has one workgroup for `each` of its scores, at least one.  By whole waves.
__device__ __forceinline__ Part part_of(const SelectIn& a, const Split& d)
{
    const uint32_t row = blockIdx.x / d.row;
    uint32_t j = blockIdx.x % d.row;
    Part t{};
    for (uint32_t s0 = 0; s0 < a.n; s0 += kWave) {
        const uint32_t s = s0 + lane_id();
        uint32_t parts = 0;
        if (s < a.n) {
            bool bad;
            const Pick p = pick_of(a, s, bad);
            parts = p.k ? (p.n - 1) / d.each + 1 : 1;
        }
        const uint32_t upto = (uint32_t)wave_incl_sum_u64(parts, 0);
        const uint32_t lane = __popcll(ballot(upto <= j));
        if (lane < kWave) {
            t.part = j - (uint32_t)__builtin_amdgcn_readlane(upto - parts, lane);
            t.parts = (uint32_t)__builtin_amdgcn_readlane(parts, lane);
            t.x = row * a.n + s0 + lane;
            t.there = true;
            break;
        }
        j -= (uint32_t)__builtin_amdgcn_readlane(upto, kWave - 1);
    }
    if (!t.there)
        return t;
    // (tables that overlap, which are malformed, can want more workgroups than there are)
    const uint32_t room = d.row - (blockIdx.x % d.row - t.part);
    t.parts = t.parts < room ? t.parts : room;
    t.p = pick_of(a, t.x, t.bad);
    const uint64_t begin = (uint64_t)t.part * d.each, end = begin + d.each;
    t.begin = begin < t.p.n ? (uint32_t)begin : t.p.n;
    t.end = end < t.p.n ? (uint32_t)end : t.p.n;
    return t;
}
// A lane's first place of a round, of the workgroup's kRound; x[j] is score i + 256 (j / 4) + j % 4.
// Places from the stretch's end on are none.
__device__ __forceinline__ uint32_t place_of(uint64_t r0)
{
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    return (uint32_t)r0 + wave * (kRound / kPartWaves) + lane_id() * 4;
}

// The second and third pass over a stretch: 16 bytes a lane at a time (a sequence's place and a
// part's begin are multiples of 4), a round ahead.  start() asks for the first round.
struct Rounds {
    typedef uint32_t v4 __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t* from;  // sums, or the one head's weights
    uint32_t begin, end;
    bool sums;
    v4 next[4];

    __device__ __forceinline__ Rounds(const SelectIn& a, const Split& d, const Part& s)
        : from(d.sums ? d.sums + (int64_t)(s.x / a.n) * d.places + s.p.at : reinterpret_cast<const uint32_t*>(s.p.w)),
          begin(s.begin), end(s.end), sums(d.sums)
    {
    }
    __device__ __forceinline__ void read(uint64_t r0)
    {
        const uint32_t i = place_of(r0);
        if (__builtin_amdgcn_readfirstlane(i) + 16 * kWave <= end) {
#pragma unroll
            for (uint32_t u = 0; u < 4; u++)
                next[u] = *reinterpret_cast<const v4*>(from + i + u * 4 * kWave);
            return;
        }
#pragma unroll
        for (uint32_t u = 0; u < 4; u++)
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const uint32_t at = i + u * 4 * kWave + j;
                next[u][j] = at < end ? from[at] : 0;
            }
    }
    __device__ __forceinline__ void start() { read(begin); }
    template <typename F>
    __device__ __forceinline__ void each(F&& f)
    {
        for (uint64_t r0 = begin; r0 < end; r0 += kRound) {
            uint32_t x[16];
#pragma unroll
            for (uint32_t j = 0; j < 16; j++)
                x[j] = sums ? next[j / 4][j % 4] : ordered(__builtin_bit_cast(float, (uint32_t)next[j / 4][j % 4]));
            if (r0 + kRound < end)
                read(r0 + kRound);
            f(x, place_of(r0));
        }
    }
};

__global__ __launch_bounds__(kPartThreads, 4) void select_count_kernel(SelectIn a, Split d, uint32_t* status)
{
    __shared__ __attribute__((aligned(16))) uint32_t bins[kBins];
    const uint32_t tid = threadIdx.x;
    const Part s = part_of(a, d);
    if (s.there && s.part == 0)
        settle(a, s.p, s.x, s.bad, kPartThreads, status);
    if (s.p.k == 0)
        return;
    for (uint32_t b = tid; b < kBins; b += kPartThreads)
        bins[b] = 0;
    __syncthreads();
    uint32_t* sums = d.sums ? d.sums + (int64_t)(s.x / a.n) * d.places + s.p.at : nullptr;
    for (uint64_t r0 = s.begin; r0 < s.end; r0 += kRound) {
        const uint32_t i = place_of(r0);
        uint32_t v[16];
        scores4<true>(a, s.p.w, s.end, i, v);
        if (sums)  // (up to 3 places past the last score, in the sequence's last page)
#pragma unroll
            for (uint32_t u = 0; u < 16; u += 4)
                if (i + u * kWave < s.end)
                    *reinterpret_cast<uint4*>(sums + i + u * kWave) = uint4{v[u], v[u + 1], v[u + 2], v[u + 3]};
#pragma unroll
        for (uint32_t j = 0; j < 16; j++)
            if (i + j / 4 * 4 * kWave + j % 4 < s.end)
                atomicAdd(&bins[v[j] >> digit_shift(0)], 1u);
    }
    __syncthreads();
    uint32_t* to = d.bins + (uint64_t)blockIdx.x * kBins;
    for (uint32_t b = tid; b < kBins; b += kPartThreads)
        to[b] = bins[b];
}

__global__ __launch_bounds__(kPartThreads, 4) void select_list_kernel(SelectIn a, Split d)
{
    constexpr uint32_t kPer = kBins / kPartThreads;
    static_assert(kPer == 4);
    __shared__ SelectLds<kPartWaves> lds;
    const uint32_t tid = threadIdx.x;
    const Part s = part_of(a, d);
    if (s.p.k == 0)
        return;
    const Pick& p = s.p;
    Rounds rounds(a, d, s);
    rounds.start();  // (beside the counts)
    const uint4* from = reinterpret_cast<const uint4*>(d.bins + (uint64_t)(blockIdx.x - s.part) * kBins) + tid;
    uint32_t all[4] = {}, before[4] = {};
#pragma unroll 8
    for (uint32_t q = 0; q < s.parts; q++) {
        const uint4 v = from[q * (kBins / 4)];
        const uint32_t one[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            all[j] += one[j];
            before[j] += q < s.part ? one[j] : 0;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; j++)
        lds.bins[0][tid * 4 + j] = all[j];
    if (tid == 0)
        lds.held = lds.up[0] = lds.equal[0] = lds.digit = lds.left = 0;
    __syncthreads();
    find_bin(lds, lds.bins[0], p.k);
    const uint32_t digit = lds.digit, left = lds.left;
    uint32_t above = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        above += tid * 4 + j > digit ? before[j] : 0;
        if (tid * 4 + j == digit)
            lds.equal[0] = before[j];
    }
    above = (uint32_t)wave_incl_sum_u64(above, 0);
    if (lane_id() == kWave - 1)
        atomicAdd(&lds.up[0], above);
    __syncthreads();
    const uint32_t agree = lds.equal[0];
    if (tid == 0)
        d.found[blockIdx.x] =
            Found{digit, left, lds.bins[0][digit], lds.up[0], agree, d.bins[(uint64_t)blockIdx.x * kBins + digit]};
    uint32_t* list = d.list + (int64_t)(s.x / a.n) * d.places + p.at;
    const uint64_t below = (1ull << lane_id()) - 1;
    rounds.each([&](const uint32_t (&v)[16], uint32_t i) {
#pragma unroll
        for (uint32_t j = 0; j < 16; j++) {
            const uint64_t those = ballot(i + j / 4 * 4 * kWave + j % 4 < s.end && v[j] >> digit_shift(0) == digit);
            if (those == 0)
                continue;
            uint32_t at = 0;
            if (lane_id() == 0)
                at = atomicAdd(&lds.held, (uint32_t)__popcll(those));
            at = agree + __builtin_amdgcn_readfirstlane(at) + __popcll(those & below);
            if ((those >> lane_id()) & 1 && at < p.n)
                list[at] = v[j];
        }
    });
}

__global__ __launch_bounds__(kPartThreads, 4) void select_place_kernel(SelectIn a, Split d)
{
    __shared__ SelectLds<kPartWaves> lds;
    __shared__ uint32_t ups[2][kPartWaves], sames[2][kPartWaves];
    const uint32_t tid = threadIdx.x;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = lane_id();
    const Part s = part_of(a, d);
    if (s.p.k == 0)
        return;
    const Pick& p = s.p;
    Rounds rounds(a, d, s);
    rounds.start();
    const Found f = d.found[blockIdx.x];
    const uint32_t* list = d.list + (int64_t)(s.x / a.n) * d.places + p.at;
    const uint32_t many = f.many < p.n ? f.many : p.n;
    uint32_t found = f.digit << digit_shift(0), known = digit_mask(0) << digit_shift(0), left = f.left;
    for (uint32_t b = tid; b < 2 * kBins; b += kPartThreads)
        lds.bins[0][b] = 0;
    if (tid == 0)
        lds.held = lds.up[0] = lds.equal[0] = lds.digit = lds.left = 0;
    __syncthreads();
    for (int e = 1; e < kDigits; e++) {
        uint32_t* bins = lds.bins[e % 2];
        for (uint32_t i = tid; i < many; i += kPartThreads) {
            const uint32_t v = list[i];
            if ((v & known) == found)
                atomicAdd(&bins[(v >> digit_shift(e)) & digit_mask(e)], 1u);
        }
        __syncthreads();
        find_bin(lds, bins, left);
        found |= lds.digit << digit_shift(e);
        known |= digit_mask(e) << digit_shift(e);
        left = lds.left;
    }
    // those before the part: above it, and equal; and equal in the part
    const uint32_t own = f.agree + f.mine < many ? f.agree + f.mine : many;
    for (uint32_t i = tid; i < own; i += kPartThreads) {
        const uint32_t v = list[i];
        if (v == found)
            atomicAdd(i < f.agree ? &lds.held : &lds.equal[0], 1u);
        else if (v > found && i < f.agree)
            atomicAdd(&lds.up[0], 1u);
    }
    __syncthreads();
    const uint32_t equal = lds.held, stay = equal < left ? equal : left;
    uint32_t above = f.above + lds.up[0] + stay, turn = 0;
    // of the part's equals all stay, or none does, or the first ones do
    const bool all = equal + lds.equal[0] <= left, some = !all && equal < left;
    const uint32_t least = all ? found : found + 1;
    uint32_t equals = left - stay;  // that stay yet, where some do
    int32_t* out = p.out + p.first;
    const uint64_t below = (1ull << lane) - 1;
    auto place = [&](auto one_by_one) {
        rounds.each([&](uint32_t (&v)[16], uint32_t i) {
            auto there = [&](uint32_t j) { return i + j / 4 * 4 * kWave + j % 4 < s.end; };
            if constexpr (decltype(one_by_one)::value) {
                // equals by their places: those that stay are raised, the workgroup's waves in turn
                uint32_t same = 0;
#pragma unroll
                for (uint32_t j = 0; j < 16; j++)
                    same += __popcll(ballot(there(j) && v[j] == found));
                if (lane == 0)
                    sames[turn][wave] = same;
                __syncthreads();
                uint32_t before = 0, sum = 0;
                for (uint32_t w = 0; w < kPartWaves; w++) {
                    before += w < wave ? sames[turn][w] : 0;
                    sum += sames[turn][w];
                }
#pragma unroll
                for (uint32_t u = 0; u < 16; u += 4) {
                    uint32_t mine = before;
#pragma unroll
                    for (uint32_t j = u; j < u + 4; j++) {
                        const uint64_t is = ballot(there(j) && v[j] == found);
                        mine += __popcll(is & below);
                        before += __popcll(is);
                    }
#pragma unroll
                    for (uint32_t j = u; j < u + 4; j++)
                        if (v[j] == found) {
                            v[j] += mine < equals;
                            mine += there(j);
                        }
                }
                equals -= sum < equals ? sum : equals;
            }
            uint32_t up = 0;
#pragma unroll
            for (uint32_t j = 0; j < 16; j++)
                up += __popcll(ballot(there(j) && v[j] >= least));
            if (lane == 0)
                ups[turn][wave] = up;
            __syncthreads();
            // what the workgroup had and the waves before have, then in the order of places: steps of
            // 256, four neighbours a lane
            up = above;
            for (uint32_t w = 0; w < kPartWaves; w++) {
                up += w < wave ? ups[turn][w] : 0;
                above += ups[turn][w];
            }
            turn ^= 1;  // (the next round's words are others: one barrier for them)
#pragma unroll
            for (uint32_t u = 0; u < 16; u += 4) {
                uint32_t at = up;
#pragma unroll
                for (uint32_t j = u; j < u + 4; j++) {
                    const uint64_t those = ballot(there(j) && v[j] >= least);
                    at += __popcll(those & below);
                    up += __popcll(those);
                }
#pragma unroll
                for (uint32_t j = u; j < u + 4; j++)
                    if (there(j) && v[j] >= least) {
                        if (at < p.k)
                            out[at] = (int32_t)(p.first + i + u / 4 * 4 * kWave + j % 4);
                        at++;
                    }
            }
        });
    };
    if (some)
        place(std::true_type{});
    else
        place(std::false_type{});
}

constexpr uint64_t kSplitArea = 1ull << 29;  // bytes of the work area, at most

// Scores of a part where choices are split (0: one kernel has them).  By itself a choice takes a
// time that goes by its length, split one that goes by all lengths, and two launches more.  us, by
// itself and split, of choices of 9,000 scores (some kept in registers): 1 11 and 21, 128 12 and
// 29; of 32,768: 16 31 and 24, 64 31 and 33, 128 36 and 48; of 65,536: 16 53 and 30, 128 61 and
// 56, 192 64 and 74; of 131,072: 1 95 and 25, 64 109 and 54, 128 110 and 83, 192 115 and 103.
// By the mean of the tables' places, so a long history among many short ones is not split, and
// the call takes what a workgroup takes for it: 16 choices of 131,072 with as many of each of seven
// of 2,000 scores 108 us, of 99 of 200 scores, where a workgroup has 256 threads, 304; alone 37.
uint32_t part_scores(const dm_ctx* c, uint64_t choices, uint64_t rows, uint64_t places, uint64_t n)
{
    constexpr uint64_t kMean = 24576, kLike = 512;
    if (places <= kMean * n || choices * kLike * n > places || choices >= c->n_cu || rows * places >= (1ull << 40))
        return 0;
    // two workgroups a compute unit, with half a part more for every choice
    const uint64_t wanted = 2 * c->n_cu - choices / 2;
    const uint64_t each = rows * places / wanted;
    return (uint32_t)(each < 4096 ? 4096 : each / 4 * 4 + 4);
}

struct GatherIn {
    const int64_t *off, *len, *budget, *to_off;
    const int32_t *page, *to_page;
    int64_t entries, to_entries;
    uint16_t *k, *v;
    int64_t layer_stride;
    const int32_t* kept;
    int64_t kept_stride;
    const float* w;
    int64_t w_layer_stride, w_stride;
    float* w_to;
    int64_t to_layer_stride, to_stride;
    uint32_t n, layers, kv_heads, share, n_pages, shift, dim;
};

constexpr int kGatherThreads = 256;

__global__ __launch_bounds__(kGatherThreads) void gather_kernel(GatherIn a, uint32_t* status)
{
    constexpr int kAtOnce = 4;
    const uint32_t tid = threadIdx.x;
    const uint64_t moves = (uint64_t)a.to_entries * a.layers;
    if (blockIdx.x >= moves) {
        // after the moves, a sequence a thread: no entry's workgroup sees the tables of one that has none
        const uint64_t s = (blockIdx.x - moves) * kGatherThreads + tid;
        if (s < a.n) {
            const int64_t t0 = a.to_off[s], t1 = a.to_off[s + 1];
            if (t0 < 0 || t1 < t0 || t1 > a.to_entries || a.budget[s] < 0 || held(a.off, a.len, a.entries, (uint32_t)s, a.shift).bad)
                atomicOr(status, kErrInval);
        }
        return;
    }
    const int64_t e = blockIdx.x / a.layers;
    const uint32_t l = blockIdx.x % a.layers;
    const uint32_t s = wave_find(a.to_off, a.n, 1, e);
    const int64_t t0 = a.to_off[s], t1 = a.to_off[s + 1];
    if (e < t0 || e >= t1)
        return;  // an entry of no sequence
    const Held h = held(a.off, a.len, a.entries, s, a.shift);
    const int64_t budget = a.budget[s];
    const bool past = h.len > budget;
    const int64_t count = past ? budget : h.len;
    const bool bad = h.bad || budget < 0 || t0 < 0 || t1 > a.to_entries || ((count + (1ll << a.shift) - 1) >> a.shift) > t1 - t0;
    const uint32_t to = bad ? 0 : (uint32_t)a.to_page[e];
    if (bad || to >= a.n_pages) {
        if (tid == 0)
            atomicOr(status, kErrInval);
        return;
    }
    const int64_t i0 = (e - t0) << a.shift;
    const uint32_t block = 1u << a.shift;
    const uint32_t here = count <= i0 ? 0 : count - i0 < block ? (uint32_t)(count - i0) : block;
    if (here == 0 || (!past && !a.w))
        return;
    bool wrong = false;
    const uint32_t choices = a.kv_heads / a.share;
    const int64_t from_at = h.off << a.shift;
    // the token that row i0 + r of head g takes
    auto token = [&](uint32_t g, uint32_t r) -> int64_t {
        if (!past)
            return i0 + r;
        const int64_t t = a.kept[((int64_t)l * choices + g / a.share) * a.kept_stride + from_at + i0 + r];
        wrong |= t < 0 || t >= h.len;
        return t < 0 || t >= h.len ? -1 : t;
    };
    if (a.w)
        for (uint32_t x = tid; x < a.kv_heads << a.shift; x += kGatherThreads) {
            const uint32_t g = x >> a.shift, r = x & (block - 1);
            if (r >= here)
                continue;
            const int64_t t = token(g, r);
            if (t >= 0)
                a.w_to[(int64_t)l * a.to_layer_stride + (int64_t)g * a.to_stride + (e << a.shift) + r] =
                    a.w[(int64_t)l * a.w_layer_stride + (int64_t)g * a.w_stride + from_at + t];
        }
    if (past) {
        const uint32_t chunks = a.dim / 8, rows = kGatherThreads / chunks, ch = tid % chunks * 8;
        const uint32_t all = a.kv_heads << a.shift;
        const uint64_t layer = (uint64_t)l * a.layer_stride;
        for (uint32_t x0 = tid / chunks; x0 < all; x0 += rows * kAtOnce) {
            int64_t t[kAtOnce];
            uint32_t p[kAtOnce];
            v4u32 kx[kAtOnce], vx[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                const uint32_t x = x0 + j * rows;
                t[j] = x < all && (x & (block - 1)) < here ? token(x >> a.shift, x & (block - 1)) : -1;
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; j++) {
                p[j] = t[j] >= 0 ? (uint32_t)a.page[h.off + (t[j] >> a.shift)] : 0;
                wrong |= p[j] >= a.n_pages;
                t[j] = p[j] >= a.n_pages ? -1 : t[j];
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; j++)
                if (t[j] >= 0) {
                    const uint64_t at = layer + ((((uint64_t)p[j] * a.kv_heads + ((x0 + j * rows) >> a.shift)) << a.shift) +
                                                 (t[j] & (block - 1))) * a.dim + ch;
                    kx[j] = *reinterpret_cast<const v4u32*>(a.k + at);
                    vx[j] = *reinterpret_cast<const v4u32*>(a.v + at);
                }
#pragma unroll
            for (int j = 0; j < kAtOnce; j++)
                if (t[j] >= 0) {
                    const uint64_t at = layer + (((uint64_t)to * a.kv_heads << a.shift) + x0 + j * rows) * a.dim + ch;
                    *reinterpret_cast<v4u32*>(a.k + at) = kx[j];
                    *reinterpret_cast<v4u32*>(a.v + at) = vx[j];
                }
        }
    }
    if (wrong)
        atomicOr(status, kErrInval);
}

uint32_t shift_of(const dm_ctx* c)
{
    uint32_t shift = 0;
    while ((1u << shift) < c->cfg.block_size)
        shift++;
    return shift;
}

}  // namespace

hipError_t evict_select(dm_ctx* c, const dm_page_tables& t, const dm_select_args& g)
{
    SelectIn a;
    a.off = t.off;
    a.len = t.len;
    a.budget = g.budget;
    a.room = g.room;
    a.entries = (int64_t)t.entries;
    a.w = g.w;
    a.layer_stride = g.w_layer_stride;
    a.w_stride = g.w_stride;
    a.kept = g.kept;
    a.kept_stride = g.kept_stride;
    a.keep = g.keep;
    a.grow = g.grow;
    a.n = (uint32_t)t.n;
    a.layers = g.layers;
    a.choices = g.kv_heads / g.share;
    a.share = g.share;
    a.sink = g.sink;
    a.recent = g.recent;
    a.shift = shift_of(c);
    const uint64_t grid = t.n * a.layers * a.choices;
    if (grid > 0x7FFFFFFFull)
        return hipErrorInvalidValue;
    const uint64_t places = t.entries * c->cfg.block_size, mean = places / t.n;
    const uint64_t rows = (uint64_t)a.layers * a.choices;
    const uint32_t each = part_scores(c, grid, rows, places, t.n);
    const uint64_t row = each ? places / each + t.n : 0, all = row * rows;
    const uint64_t bins = all * kBins * 4, found = (all * sizeof(Found) + 15) / 16 * 16;
    const uint64_t list = rows * places * 4, area = bins + found + (a.share > 1 ? 2 : 1) * list;
    if (each && area <= kSplitArea) {
        hipError_t e;
        char* at = static_cast<char*>(scratch_get(c, kSlotPages, area, &e));
        if (!at)
            return e;
        Split d;
        d.each = each;
        d.row = (uint32_t)row;
        d.bins = reinterpret_cast<uint32_t*>(at);
        d.found = reinterpret_cast<Found*>(at + bins);
        d.list = reinterpret_cast<uint32_t*>(at + bins + found);
        d.sums = a.share > 1 ? reinterpret_cast<uint32_t*>(at + bins + found + list) : nullptr;
        d.places = (int64_t)places;
        select_count_kernel<<<(uint32_t)all, kPartThreads, 0, c->stream>>>(a, d, c->d_status);
        select_list_kernel<<<(uint32_t)all, kPartThreads, 0, c->stream>>>(a, d);
        select_place_kernel<<<(uint32_t)all, kPartThreads, 0, c->stream>>>(a, d);
        return hipGetLastError();
    }
    if (mean <= 2048)
        select_kernel<256><<<(uint32_t)grid, 256, 0, c->stream>>>(a, c->d_status);
    else if (mean <= 6144)
        select_kernel<512><<<(uint32_t)grid, 512, 0, c->stream>>>(a, c->d_status);
    else
        select_kernel<1024><<<(uint32_t)grid, 1024, 0, c->stream>>>(a, c->d_status);
    return hipGetLastError();
}

hipError_t kv_gather(dm_ctx* c, const dm_kv_pages& kv, const dm_page_tables& from, const dm_page_tables& to,
                     const dm_gather_args& g)
{
    GatherIn a;
    a.off = from.off;
    a.len = from.len;
    a.budget = g.budget;
    a.to_off = to.off;
    a.page = from.page;
    a.to_page = to.page;
    a.entries = (int64_t)from.entries;
    a.to_entries = (int64_t)to.entries;
    a.k = static_cast<uint16_t*>(kv.k);
    a.v = static_cast<uint16_t*>(kv.v);
    a.layer_stride = kv.layer_stride;
    a.kept = g.kept;
    a.kept_stride = g.kept_stride;
    a.w = g.w;
    a.w_layer_stride = g.w_layer_stride;
    a.w_stride = g.w_stride;
    a.w_to = g.w_to;
    a.to_layer_stride = g.to_layer_stride;
    a.to_stride = g.to_stride;
    a.n = (uint32_t)to.n;
    a.layers = kv.layers;
    a.kv_heads = kv.kv_heads;
    a.share = g.share;
    a.n_pages = kv.n_pages;
    a.shift = shift_of(c);
    a.dim = kv.head_dim;
    const uint64_t grid = to.entries * kv.layers + (to.n + kGatherThreads - 1) / kGatherThreads;
    if (grid > 0x7FFFFFFFull)
        return hipErrorInvalidValue;
    gather_kernel<<<(uint32_t)grid, kGatherThreads, 0, c->stream>>>(a, c->d_status);
    return hipGetLastError();
}

}  // namespace dm
