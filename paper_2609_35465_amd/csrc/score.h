// Log probabilities of given tokens, entropy and likeliest tokens of rows of
// logits (log_probs).  Included by batch.hip.
//
//   d_j = x_j - m, l = sum_j 2^(c d_j), u = sum_j 2^(c d_j) d_j, c = log2(e) / T:
//   log p_j = d_j / T - ln l,  entropy = ln l - u / (l T)
//
// One pass over the logits: every lane keeps m (the largest logit so far), l and u,
// and moves them to a larger m where it meets one.  Logits of -inf and NaN, and what
// is 2^-200 and less of the largest, add nothing.  Each wave keeps its largest
// logits in order, one a lane, and looks closer only where a batch has one that
// belongs among them.  The order is by logit, then by index from the first on.
// The tokens do not depend on how a row is split, and fp32 sums have an order that the
// sizes fix.
//
// 2,048 rows of 151,936 logits in fp16, the likeliest token: 120 us, 5,180 GB/s (a
// large copy reaches 5,160); of fp32 64 rows with five tokens 18 us and one row with
// twenty 12: a chain of the loads, the bar's bisection, the list and the ranking in
// 14 and 7.5 us, and the join's 4.5.  A wave's largest kept in order by inserting, in
// place of the list, took 28 us for 64 rows with twenty tokens (now 18.6) and as long with one;
// one batch at a time in place of four 26 with five.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lanes.h"

namespace tetra_dev {

constexpr int kMostTop = 64;                 // a lane each
constexpr int kScoreBatch = 1024;            // logits that a wave takes at once: 16 a lane
constexpr int kMostScoreParts = 64;          // of a row, a lane each in the join
constexpr float kScoreFloor = -200.f;        // exponents from here down weigh nothing
constexpr uint64_t kNoPlace = 0x007FFFFFFFFFFFFFull;   // of the first token at -inf, and above those behind it

struct ScoreArgs {
    const void* logits;
    long long stride;
    const float* temperature;
    const int* tokens;
    float *out, *entropy, *top_out;
    int* top_tokens;
    int rows, vocab, given, top;
    int parts, part;                         // of a row, and the logits of each (a multiple of kScoreBatch)
    float* sums;                             // [rows][parts][4]: m, l, u of the parts
    uint64_t* places;                        // [rows][parts][top]: the parts' largest, falling
};

__device__ __forceinline__ float score_logit(uint32_t key) {
    return __builtin_bit_cast(float, key >> 31 ? key ^ 0x80000000u : ~key);
}

__device__ __forceinline__ uint64_t score_place(float x, int index) {
    return static_cast<uint64_t>(rising_key(x)) << 32 | static_cast<uint32_t>(~index);
}

// 1 / T, and c.  Temperatures end at 2^100, so that `least` is a number and -inf stays out.
struct ScoreScale {
    float inverse, c, least;                 // least: of d, below it nothing
    __device__ __forceinline__ ScoreScale(const ScoreArgs& a, int row) {
        float t = a.temperature ? a.temperature[row] : 1.f;
        if (!(t > 0.f)) t = 1.f;
        inverse = fmaxf(1.f / t, 0x1p-100f);
        c = fminf(inverse * 1.44269504f, 3e38f);
        least = kScoreFloor / c;
    }
};

struct ScoreSum {
    float m, l, u;
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = u = 0.f;
    }
    // to a largest logit of `to`, at least m
    __device__ __forceinline__ void move(float to, const ScoreScale& s) {
        const float d = m - to;
        const bool any = m > -INFINITY && d > s.least;
        const float f = any ? __builtin_amdgcn_exp2f(d * s.c) : 0.f;
        u = any ? f * (u + l * d) : m == to ? u : 0.f;
        l = any ? f * l : m == to ? l : 0.f;
        m = to;
    }
};

// How much of a wave's logits may belong to the n largest.  Every lane keeps the
// largest logits of four groups of its own: what n groups reach, n logits do, and what
// does not reach it is out.  Batches that have more raise the bar first, then put what
// passes it into a list in LDS.  Where the list is full (many equal logits), it goes
// into the n largest themselves, in order, one a lane, and those are the bar.
struct ScoreTop {
    static constexpr int kHeld = 320, kList = kHeld + kMostTop;
    uint64_t* list;                          // [kList]
    uint64_t least;                          // places up to it do not belong
    float least_logit, groups[4];
    uint64_t mine;
    int n, count;

    __device__ __forceinline__ void clear(int top, uint64_t* held) {
        list = held;
        n = top;
        count = 0;
        mine = 0;
        for (float& g : groups) g = -INFINITY;
        raise(kNoPlace);
    }
    __device__ __forceinline__ void raise(uint64_t to) {
        least = to;
        least_logit = fmaxf(score_logit(static_cast<uint32_t>(to >> 32)), -3.4028234e38f);   // -inf never belongs
    }
    // a key that at least n of the groups' reach, near the largest such; a lane's groups
    // count as one where 64 are enough
    __device__ __forceinline__ static uint32_t reached(const float (&groups)[4], int n) {
        const uint32_t key = rising_key(fmaxf(fmaxf(groups[0], groups[1]), fmaxf(groups[2], groups[3])));
        uint32_t lo = ~wave_all(Max(), ~key), hi = wave_all(Max(), key);
        if (n <= kMostTop / 2) {
            for (int step = 0; step < 10 && lo < hi; ++step) {
                const uint32_t mid = hi - (hi - lo) / 2;
                if (static_cast<int>(__popcll(__ballot(key >= mid))) >= n) lo = mid;
                else hi = mid - 1;
            }
        } else {
            uint32_t k[4];
            for (int i = 0; i < 4; ++i) k[i] = rising_key(groups[i]);
            for (int step = 0; step < 10 && lo < hi; ++step) {
                const uint32_t mid = hi - (hi - lo) / 2;
                const int c = __popcll(__ballot(k[0] >= mid)) + __popcll(__ballot(k[1] >= mid)) +
                              __popcll(__ballot(k[2] >= mid)) + __popcll(__ballot(k[3] >= mid));
                if (c >= n) lo = mid;
                else hi = mid - 1;
            }
        }
        return lo;
    }
    // the largest of a lane's 16 logits of a batch, with its groups
    __device__ __forceinline__ float add(const float (&v)[16]) {
        float all = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float m = fmaxf(fmaxf(v[4 * i], v[4 * i + 1]), fmaxf(v[4 * i + 2], v[4 * i + 3]));
            groups[i] = fmaxf(groups[i], m);
            all = fmaxf(all, m);
        }
        return all;
    }
    // whether logits of which these are the largest may belong; then the bar is raised
    __device__ __forceinline__ bool look(const float (&most)[4]) {
        if (!__any(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) >= least_logit)) return false;
        const uint64_t p = static_cast<uint64_t>(reached(groups, n)) << 32;
        if (p > least) raise(p - 1);
        return true;
    }
    // p is uniform
    __device__ __forceinline__ void insert(uint64_t p) {
        const uint32_t lo = __builtin_amdgcn_update_dpp(-1, static_cast<int>(mine), 0x138, 0xF, 0xF, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(-1, static_cast<int>(mine >> 32), 0x138, 0xF, 0xF, false);
        const uint64_t before = static_cast<uint64_t>(hi) << 32 | lo;      // of the lane before, the largest number in lane 0
        mine = mine > p ? mine : before > p ? p : before;
        const uint64_t last = lane_of(mine, n - 1);
        if (last > least) raise(last);
    }
    // all that passes the bar, of p in the lanes
    __device__ __forceinline__ void insert_all(uint64_t p) {
        unsigned long long has = __ballot(p > least);
        while (has) {
            const int l = __builtin_ctzll(has);
            insert(lane_of(p, l));
            has &= __ballot(p > least) & ~(1ull << l);
        }
    }
    __device__ __forceinline__ void insert_list() {
        const int lane = threadIdx.x & 63;
        for (int i = 0; i < count; i += 64) insert_all(i + lane < count ? list[i + lane] : 0);
        count = 0;
    }
    // The lanes' logits j whose bits are set in `which`, x and index of each from at(j): into
    // the list, one a lane at a time.
    template <class F>
    __device__ __forceinline__ void offer(uint64_t which, F at) {
        while (__any(which != 0)) {
            uint64_t p = 0;
            if (which) p = at(__builtin_ctzll(which));
            which &= which - 1;
            unsigned long long has = __ballot(p > least);
            if (count + static_cast<int>(__popcll(has)) > kHeld) {
                insert_list();
                has = __ballot(p > least);
            }
            if (p > least) list[count + __popcll(has & ((1ull << (threadIdx.x & 63)) - 1))] = p;
            count += __popcll(has);
        }
    }
    // what may belong, all in the list
    __device__ __forceinline__ void finish() {
        const unsigned long long has = __ballot(mine != 0 && static_cast<int>(threadIdx.x & 63) < n);
        if (has >> (threadIdx.x & 63) & 1) list[count + (threadIdx.x & 63)] = mine;
        count += __popcll(has);
    }
};

template <class T>
struct ScoreBatch;

template <>
struct ScoreBatch<float> {
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    vec v[4];
    __device__ __forceinline__ void load(const float* x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const vec*>(x + 256 * i + 4 * (threadIdx.x & 63));
    }
    // a row of n logits, fewer than a batch
    __device__ __forceinline__ void load_some(const float* x, int n) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j / 4][j % 4] = index(j) < n ? x[index(j)] : -INFINITY;
    }
    // the first n, which are another batch's
    __device__ __forceinline__ void leave_out(int n) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j / 4][j % 4] = index(j) < n ? -INFINITY : v[j / 4][j % 4];
    }
    __device__ __forceinline__ float at(int j) const { return v[j / 4][j % 4]; }
    // of logit j of this lane, from the batch's first on
    __device__ __forceinline__ static int index(int j) { return 256 * (j / 4) + 4 * (threadIdx.x & 63) + j % 4; }
};

template <>
struct ScoreBatch<_Float16> {
    typedef _Float16 vec __attribute__((ext_vector_type(8), aligned(2)));
    vec v[2];
    __device__ __forceinline__ void load(const _Float16* x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const vec*>(x + 512 * i + 8 * (threadIdx.x & 63));
    }
    __device__ __forceinline__ void load_some(const _Float16* x, int n) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j / 8][j % 8] = index(j) < n ? x[index(j)] : static_cast<_Float16>(-INFINITY);
    }
    __device__ __forceinline__ void leave_out(int n) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j / 8][j % 8] = index(j) < n ? static_cast<_Float16>(-INFINITY) : v[j / 8][j % 8];
    }
    __device__ __forceinline__ float at(int j) const { return static_cast<float>(v[j / 8][j % 8]); }
    __device__ __forceinline__ static int index(int j) { return 512 * (j / 8) + 8 * (threadIdx.x & 63) + j % 8; }
};

// The logits of a row's given tokens, -inf outside the vocabulary: the first 256 are on
// their way from the start, a thread each.
struct ScoreGiven {
    bool half;
    float x;
    __device__ __forceinline__ ScoreGiven(const ScoreArgs& a, int row, bool half) : half(half), x(-INFINITY) {
        if (static_cast<int>(threadIdx.x) < a.given) x = of(a, row, threadIdx.x);
    }
    __device__ __forceinline__ float of(const ScoreArgs& a, int row, int g) const {
        const int j = a.tokens[static_cast<size_t>(row) * a.given + g];
        if (j < 0 || j >= a.vocab) return -INFINITY;
        const long long at = row * a.stride + j;
        return half ? static_cast<float>(static_cast<const _Float16*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at];
    }
};

// what is known of a row, from its parts or its one workgroup: the outputs
struct ScoreRow {
    ScoreScale scale;
    ScoreSum sum;
    float log_l;
    __device__ __forceinline__ ScoreRow(const ScoreScale& scale, const ScoreSum& sum) : scale(scale), sum(sum), log_l(logf(sum.l)) {}
    __device__ __forceinline__ float log_of(float x) const {
        if (sum.m == -INFINITY || !(x > -INFINITY)) return -INFINITY;
        float t = x == sum.m ? 0.f : (x - sum.m) * scale.inverse;
        if (t == -INFINITY) t = 2.f * ((0.5f * x - 0.5f * sum.m) * scale.inverse);     // x - m past the type's end
        return t - log_l;
    }
    __device__ __forceinline__ void write(const ScoreArgs& a, int row, const ScoreGiven& given) const {
        for (int g = threadIdx.x; g < a.given; g += 256)
            a.out[static_cast<size_t>(row) * a.given + g] = log_of(g < 256 ? given.x : given.of(a, row, g));
        if (a.entropy && threadIdx.x == 0)
            a.entropy[row] = sum.m == -INFINITY ? 0.f : log_l - (sum.u == 0.f ? 0.f : sum.u / sum.l * scale.inverse);
    }
    __device__ __forceinline__ void write_top(const ScoreArgs& a, int row, int rank, uint64_t place) const {
        const size_t at = static_cast<size_t>(row) * a.top + rank;
        a.top_tokens[at] = place ? static_cast<int>(~static_cast<uint32_t>(place)) : -1;
        a.top_out[at] = place ? log_of(score_logit(static_cast<uint32_t>(place >> 32))) : -INFINITY;
    }
};

// a workgroup a part of a row, a wave every fourth batch of it, four at a time
template <class T, bool TOP>
__global__ __launch_bounds__(256, 4) void score_kernel(ScoreArgs a) {
    constexpr int kList = ScoreTop::kList, kStep = 4 * kScoreBatch;
    __shared__ float sums[4][3];
    __shared__ uint64_t lists[TOP ? 4 * kList : 1];
    __shared__ float groups[TOP ? 4 : 1][4][64];
    __shared__ int count;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    const int begin = part * a.part, end = min(a.vocab, begin + a.part);
    int i = begin + wave * kScoreBatch;
    ScoreBatch<T> batch[4];
    // batches i + k kStep; one that ends past the part lies further back, with what is not its own left out
    auto place_of = [&](int k) { return min(i + k * kStep, end - kScoreBatch); };
    auto load = [&] {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k * kStep < end) batch[k].load(x + place_of(k));
    };
    const bool small = a.vocab < kScoreBatch;
    if (!small) load();
    else if (wave == 0) batch[0].load_some(x, end);
    const ScoreScale scale(a, row);
    ScoreSum s;
    s.clear();
    ScoreTop top;
    if constexpr (TOP) top.clear(a.top, lists + wave * kList);
    for (; i < end; i += 4 * kStep, load()) {
        float most[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            most[k] = -INFINITY;
            if (i + k * kStep < end) {
                const int over = small ? 0 : i + k * kStep - place_of(k);
                if (over > 0) batch[k].leave_out(over);
                float v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = batch[k].at(j);
                float m = v[0];
                if constexpr (TOP) m = top.add(v);
                else
#pragma unroll
                    for (int j = 1; j < 16; ++j) m = fmaxf(m, v[j]);
                most[k] = m;
                if (m > s.m) s.move(m, scale);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float d = fmaxf(v[j] - s.m, scale.least);           // of NaN the bound
                    const float e = __builtin_amdgcn_exp2f(d * scale.c);
                    s.l += e;
                    s.u = __builtin_fmaf(e, d, s.u);
                }
            }
        }
        if constexpr (TOP) {
            if (top.look(most)) {
                uint64_t which = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i + k * kStep < end && __any(most[k] >= top.least_logit)) {
                        uint32_t bits = 0;
#pragma unroll
                        for (int j = 0; j < 16; ++j) bits |= static_cast<uint32_t>(batch[k].at(j) >= top.least_logit) << j;
                        which |= static_cast<uint64_t>(bits) << (16 * k);
                    }
                top.offer(which, [&](int j) {
                    const int at = (small ? 0 : place_of(j / 16)) + ScoreBatch<T>::index(j % 16);
                    return score_place(static_cast<float>(x[at]), at);
                });
            }
        }
    }
    // the lanes joined, then the waves
    float m = s.m;
    for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o, 64));
    s.move(m, scale);
    if (lane == 0) sums[wave][0] = m;
    const float l = wave_all(Sum(), s.l), u = wave_all(Sum(), s.u);
    if (lane == 0) {
        sums[wave][1] = l;
        sums[wave][2] = u;
    }
    if constexpr (TOP) {
        top.finish();
#pragma unroll
        for (int k = 0; k < 4; ++k) groups[wave][k][lane] = top.groups[k];
        if (threadIdx.x == 0) count = 0;
    }
    __syncthreads();
    float most = -INFINITY;
    for (int w = 0; w < 4; ++w) most = fmaxf(most, sums[w][0]);
    ScoreSum all;
    all.clear();
    all.m = most;
    for (int w = 0; w < 4; ++w) {
        ScoreSum o{sums[w][0], sums[w][1], sums[w][2]};
        o.move(most, scale);
        all.l += o.l;
        all.u += o.u;
    }
    if (most == INFINITY) {                  // infinities share what there is
        int n = 0;
        for (int j = begin + threadIdx.x; j < end; j += 256) n += static_cast<float>(x[j]) == INFINITY;
        n = wave_all(Sum(), n);
        __syncthreads();
        if (lane == 0) sums[wave][1] = static_cast<float>(n);
        __syncthreads();
        all.l = sums[0][1] + sums[1][1] + sums[2][1] + sums[3][1];
        all.u = 0.f;
    }
    // what of the waves' lists reaches the bar of all their groups, ranked
    int n = 0;
    if constexpr (TOP) {
        float all[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            all[k] = fmaxf(fmaxf(groups[0][k][lane], groups[1][k][lane]), fmaxf(groups[2][k][lane], groups[3][k][lane]));
        const uint64_t least = static_cast<uint64_t>(ScoreTop::reached(all, a.top)) << 32;
        constexpr int kPer = kList / 64;
        uint64_t held[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) held[k] = 64 * k + lane < top.count ? top.list[64 * k + lane] : 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const unsigned long long has = __ballot(held[k] != 0 && held[k] >= least);
            if (!has) continue;
            int to = 0;
            if (lane == 0) to = atomicAdd(&count, static_cast<int>(__popcll(has)));
            to = __builtin_amdgcn_readfirstlane(to) + __popcll(has & ((1ull << lane) - 1));
            if (has >> lane & 1) lists[to] = held[k];
        }
        __syncthreads();
        n = count;
    }
    auto ranked = [&](auto put) {
        for (int i = threadIdx.x; i < max(n, a.top); i += 256) {
            const uint64_t p = i < n ? lists[i] : 0;
            int rank = i;
            if (p) {
                rank = 0;
#pragma unroll 8
                for (int k = 0; k < n; ++k) rank += lists[k] > p;
            }
            if (rank < a.top) put(rank, p);
        }
    };
    if (a.parts > 1) {
        const size_t at = static_cast<size_t>(row) * a.parts + part;
        if (threadIdx.x == 0) {
            a.sums[4 * at] = all.m;
            a.sums[4 * at + 1] = all.l;
            a.sums[4 * at + 2] = all.u;
        }
        if constexpr (TOP) ranked([&](int rank, uint64_t p) { a.places[at * a.top + rank] = p; });
        return;
    }
    const ScoreGiven given(a, row, sizeof(T) == 2);
    const ScoreRow r(scale, all);
    r.write(a, row, given);
    if constexpr (TOP) ranked([&](int rank, uint64_t p) { r.write_top(a, row, rank, p); });
}

// A row's parts joined: a workgroup a row.  What the `deep`-th places of `of` parts
// reach, deep * of >= top places do; what reaches it is ranked.
template <class T, bool TOP>
__global__ __launch_bounds__(256) void score_join_kernel(ScoreArgs a) {
    __shared__ uint64_t found[TOP ? kMostTop * kMostScoreParts : 1];
    __shared__ unsigned count;
    constexpr int kAhead = 4;                // places of a thread on their way from the start
    const int lane = threadIdx.x & 63, row = blockIdx.x;
    const size_t first = static_cast<size_t>(row) * a.parts;
    const int n = a.parts * a.top;
    // the 60th part of a hundred of the parts, or so: fewer would set the bar too high, more too low
    const int deep = (5 * a.top + 3 * a.parts - 1) / (3 * a.parts), of = TOP ? (a.top + deep - 1) / deep : 0;
    ScoreSum s;
    s.clear();
    if (lane < a.parts) s = {a.sums[4 * (first + lane)], a.sums[4 * (first + lane) + 1], a.sums[4 * (first + lane) + 2]};
    uint64_t head = 0, ahead[kAhead];
    auto place_at = [&](int i) { return i < n ? a.places[first * a.top + i] : 0; };
    if constexpr (TOP) {
        if (lane < a.parts) head = a.places[(first + lane) * a.top + deep - 1];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) ahead[k] = place_at(threadIdx.x + 256 * k);
    }
    const ScoreGiven given(a, row, sizeof(T) == 2);
    const ScoreScale scale(a, row);
    if constexpr (TOP) {
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
    }
    float m = s.m;
    for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o, 64));
    s.move(m, scale);
    s.l = wave_all(Sum(), s.l);
    s.u = wave_all(Sum(), s.u);
    const ScoreRow r(scale, s);
    r.write(a, row, given);
    if constexpr (TOP) {
        int above = 0;
        for (int i = 0; i < a.parts; ++i) above += lane_of(head, i) > head;
        const unsigned long long at = __ballot(head != 0 && above == of - 1);
        const uint64_t least = at ? lane_of(head, __builtin_ctzll(at)) : 1;
        auto gather = [&](uint64_t p) {
            const unsigned long long has = __ballot(p >= least);
            if (!has) return;
            unsigned to = 0;
            if (lane == 0) to = atomicAdd(&count, static_cast<unsigned>(__popcll(has)));
            to = __builtin_amdgcn_readfirstlane(to) + __popcll(has & ((1ull << lane) - 1));
            if (p >= least) found[to] = p;
        };
#pragma unroll
        for (int k = 0; k < kAhead; ++k) gather(ahead[k]);
        for (int i = kAhead * 256; i < n; i += 256) gather(place_at(i + threadIdx.x));
        __syncthreads();
        const int kept = count;
        for (int i = threadIdx.x; i < kept; i += 256) {
            const uint64_t p = found[i];
            int rank = 0;
#pragma unroll 8
            for (int k = 0; k < kept; ++k) rank += found[k] > p;
            if (rank < a.top) r.write_top(a, row, rank, p);
        }
        for (int i = kept + threadIdx.x; i < a.top; i += 256) r.write_top(a, row, i, 0);
    }
}

// Parts of a row, so that there are four workgroups a CU over all rows and each wave has
// a batch; and the most that this many rows, or fewer, leave for the join.
struct ScoreShape {
    int parts, part;
};
inline int score_batches(int vocab) { return (vocab + kScoreBatch - 1) / kScoreBatch; }
inline int score_most_parts(int vocab) {
    const int most = (score_batches(vocab) + 3) / 4;
    return most < kMostScoreParts ? most : kMostScoreParts;
}
inline ScoreShape score_shape(int rows, int vocab, int cus) {
    int parts = 4 * cus / rows;
    const int most = score_most_parts(vocab), batches = score_batches(vocab);
    parts = parts < 1 ? 1 : parts < most ? parts : most;
    const int part = (batches + parts - 1) / parts;
    return {(batches + part - 1) / part, part * kScoreBatch};
}
inline size_t score_entries(int rows, int vocab, int cus) {
    const size_t n = static_cast<size_t>(rows) * score_most_parts(vocab), most = 4 * static_cast<size_t>(cus);
    return n < most ? n : most;
}

}  // namespace tetra_dev
