// Sampling a token from a row of logits: temperature, top-k, top-p and min-p,
// from a given random number.  Included by serve.hip.
//
// Weights are whole numbers, w = floor(2^40 2^t) with t = (x - max) fl(log2(e)
// / T), where 2^t is a fixed sequence of fp32 operations that each round by
// themselves.  Sums of them are exact in any order, so a token is a function
// of the inputs alone: no split of the work, and no atomic's order, can change
// it.  2^-40 of the likeliest token's weight is below what an fp32 sum of
// probabilities holds.
//
// The order of the tokens is by logit, then by index.  With k tokens of it
// left by top-k, top-p leaves the shortest prefix whose weight reaches
// ceil(p W), min-p drops what is below min_p of the likeliest, and the token
// is the first by index at which the sum of what is left exceeds floor(u W').
// So a cut of the order and the weights' sums in index order are all that is
// needed; nothing is sorted but the few candidates around the cut.
//
// Four launches, each over the rows' parts: the groups' largest logits, what
// the cut is found from, the sums, and one workgroup a row for the rest.  64
// rows of 151,936 logits with settings of every kind take 40 us, a row 16 us.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lanes.h"

namespace tetra_dev {

constexpr uint32_t kLowestKey = 0x007FFFFFu;   // of -inf
constexpr int kSampleTile = 512;               // logits of a wave's step: 8 a lane, 64 apart
constexpr int kMostGroups = 2048;              // maxima of lanes' logits that the first kernel leaves of a row
constexpr int kMostParts = 128;                // workgroups of a row
constexpr int kSampleBins = 2048;              // of the weights' logarithms, 0 down to -41
constexpr float kBinsPerUnit = kSampleBins / 41.f;
constexpr int kSampleList = 16384;             // candidates that a row's list holds
constexpr int kSortList = 1024;                // and that are sorted at once
constexpr int kTokenThreads = 1024, kTokenWaves = kTokenThreads / 64;
constexpr int kMostByGroups = 512;             // largest top-k that goes by the groups' maxima

struct SampleArgs {
    const float* logits;
    long long stride;
    const float *temperature, *top_p, *min_p, *u;
    const int* top_k;
    int* tokens;
    uint8_t* space;        // SampleSpace of every row, row_space bytes each
    size_t row_space;
    int rows, vocab, tiles, parts;
    int groups, wave_groups;      // of a row, and of each of its 4 parts waves: 16 (of four lanes) or 4 (of sixteen)
};

// What a row's kernels leave for each other, followed by the tiles' sums
// (uint64) and the groups' largest keys (uint32).
struct SampleSpace {
    unsigned long long mass[kSampleBins];
    unsigned count[kSampleBins];
    unsigned top_key;                // key of the largest logit
    int first;                       // index of the first of the largest logits (greedy rows)
    unsigned listed;                 // candidates found; the list holds the first kSampleList
    int group_bin;                   // candidates by groups: of this bin of kGroupBins and those above
    int bin_low, bin_high, bin_k;    // candidates by bin: bin_low .. bin_high, and bin_k
    unsigned count_k;                // tokens above bin_k
    unsigned long long mass_low, mass_k, mass_all;   // weight above bin_low, above bin_k, of all
    unsigned list[kSampleList];

    __device__ unsigned long long* sums() { return reinterpret_cast<unsigned long long*>(this + 1); }
    __device__ unsigned* largest(int tiles) { return reinterpret_cast<unsigned*>(sums() + tiles); }
};

// rises with x; NaN counts as -inf, and the zeros are equal
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x == 0.f ? 0.f : x);
    return x != x ? kLowestKey : b >> 31 ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float logit_of(uint32_t key) {
    return __builtin_bit_cast(float, key >> 31 ? key ^ 0x80000000u : ~key);
}

// t, a weight's logarithm; -48 and below, and of NaN, is -48 (the weight is 0)
__device__ __forceinline__ float log_of(float x, float top, float inverse) {
#pragma clang fp contract(off)
    return fmaxf(x == top ? 0.f : (x - top) * inverse, -48.f);
}

// floor(2^40 2^t): the series of 2^f to f^7 with |f| <= 1/2 (its remainder is
// 5e-9), every operation rounded by itself; then its mantissa, 2^40 for 1.0,
// shifted by the exponent
__device__ __forceinline__ uint64_t weight_of(float t) {
#pragma clang fp contract(off)
    const float whole = rintf(t), f = t - whole;
    float p = 0x1.ffcbfcp-17f;
    p = p * f + 0x1.430912p-13f;
    p = p * f + 0x1.5d87fep-10f;
    p = p * f + 0x1.3b2ab6p-7f;
    p = p * f + 0x1.c6b08ep-5f;
    p = p * f + 0x1.ebfbe0p-3f;
    p = p * f + 0x1.62e430p-1f;
    p = p * f + 1.f;
    const uint32_t q = __builtin_bit_cast(uint32_t, p) + (static_cast<uint32_t>(static_cast<int>(whole)) << 23);
    const uint32_t mantissa = (q & 0x7FFFFFu) | 0x800000u;
    return (static_cast<uint64_t>(mantissa) << 17) >> (127 - (q >> 23));
}

constexpr float kNoWeight = -41.f;     // weights of this logarithm and below are 0

// falls with t
__device__ __forceinline__ int bin_of(float t) { return min(kSampleBins - 1, static_cast<int>(t * -kBinsPerUnit)); }

// the same in 256 bins, for the groups' maxima
constexpr int kGroupBins = 256;
__device__ __forceinline__ int group_bin_of(float t) {
    return min(kGroupBins - 1, static_cast<int>(t * -(kGroupBins / 41.f)));
}

// the order of the tokens in one number: by key, then by index from the first on
__device__ __forceinline__ uint64_t place_of(uint32_t key, uint32_t index) {
    return static_cast<uint64_t>(key) << 32 | static_cast<uint32_t>(~index);
}

// the sum over WAVES (at most 16) waves, in every thread
template <int WAVES, class T>
__device__ T group_sum(T v, T* lds) {
    v = wave_all(Sum(), v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lane_of(row_upto(Sum(), lds[threadIdx.x % WAVES]), WAVES - 1);
}

// the sum over the threads up to and with this one, and over all
template <int WAVES, class T>
__device__ T group_upto(T v, T* lds, T* all) {
    v = wave_upto(Sum(), v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    const T waves = row_upto(Sum(), lds[threadIdx.x % WAVES]);
    *all = lane_of(waves, WAVES - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    return wave ? v + lane_of(waves, wave - 1) : v;
}

enum SampleKind { kFixed, kByGroups, kByBins, kUnfiltered };

// What the kernels know of a row.
struct SampleRow {
    const float* x;
    SampleSpace* space;
    float top, inverse, top_p;
    uint32_t top_key;
    uint64_t min_weight;
    int k;               // of top-k, 0: off
    SampleKind kind;     // kFixed: the token needs no weights (greedy, or nothing but -inf)
};

// before the largest logit is known: kFixed only by the temperature
__device__ __forceinline__ SampleRow sample_settings(const SampleArgs& a, int row) {
    SampleRow r;
    r.x = a.logits + row * a.stride;
    r.space = reinterpret_cast<SampleSpace*>(a.space + row * a.row_space);
    const float temperature = a.temperature[row];
    r.inverse = 0x1.715476p+0f / temperature;
    r.top_p = a.top_p[row];
    r.min_weight = static_cast<uint64_t>(ceil(fmin(fmax(static_cast<double>(a.min_p[row]), 0.0), 1.0) * 0x1p40));
    r.k = a.top_k[row];
    if (r.k < 0 || r.k >= a.vocab) r.k = 0;
    if (!(temperature > 0.f)) r.kind = kFixed;
    else if (r.k > 0 && r.k <= kMostByGroups && 2 * r.k <= a.groups) r.kind = kByGroups;
    else if (r.k > 0 || r.top_p < 1.f) r.kind = kByBins;
    else r.kind = kUnfiltered;
    return r;
}

__device__ __forceinline__ void sample_top(SampleRow& r, uint32_t top_key) {
    r.top_key = top_key;
    r.top = logit_of(top_key);
    if (r.top_key == kLowestKey) r.kind = kFixed;
}

// ceil(p mass), one at least
__device__ __forceinline__ uint64_t share_of(float p, uint64_t mass) {
    const double s = ceil(static_cast<double>(p) * static_cast<double>(mass));
    return s >= 1.0 ? static_cast<uint64_t>(s) : 1;
}

// A workgroup's candidates, gathered in LDS so that the row's list takes one
// atomic for all of them (each costs a way to memory and back).
struct Candidates {
    static constexpr int kHeld = 1024;
    unsigned count, at;
    int index[kHeld];

    __device__ __forceinline__ void clear() {
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
    }
    __device__ __forceinline__ void add(bool has, int i, SampleSpace* space) {
        const unsigned long long b = __ballot(has);
        if (!b) return;
        const int lane = threadIdx.x & 63, leader = __builtin_ctzll(b);
        unsigned n = 0;
        if (lane == leader) n = atomicAdd(&count, static_cast<unsigned>(__popcll(b)));
        n = lane_of(n, leader) + __popcll(b & ((1ull << lane) - 1));
        if (has && n < kHeld) index[n] = i;
        if (has && n >= kHeld) {       // no room: straight to the list
            const unsigned to = atomicAdd(&space->listed, 1u);
            if (to < kSampleList) space->list[to] = i;
        }
    }
    __device__ __forceinline__ void to_list(SampleSpace* space) {
        __syncthreads();
        const unsigned n = count < kHeld ? count : kHeld;
        if (n == 0) return;
        if (threadIdx.x == 0) at = atomicAdd(&space->listed, n);
        __syncthreads();
        for (unsigned i = threadIdx.x; i < n; i += blockDim.x)
            if (at + i < kSampleList) space->list[at + i] = index[i];
    }
};

// Neighbouring workgroups take different rows, one row further in every round:
// workgroups go to the XCDs and CUs in turn, and so the parts of the rows with
// most to do come to all of them (64 rows with a period of 8 settings: 49 us with
// a row's parts side by side, which put them on a quarter of the CUs, 41 so).
__device__ __forceinline__ void row_and_part(int rows, int& row, int& part) {
    part = blockIdx.x / rows;
    row = (blockIdx.x - part * rows + part) % rows;
}

// A wave's tiles of a row, `first` and every `step` further: a lane's eight logits
// of one (-inf past the row's end).  The first is on its way from the start, the
// next one during f(tile, x).
struct Tiles {
    const float* row;
    int vocab, tiles, first, step;
    float x[8];

    __device__ __forceinline__ Tiles(const SampleArgs& a, int r, int wave, int waves)
        : row(a.logits + r * a.stride), vocab(a.vocab), tiles(a.tiles), first(wave), step(waves) {
        if (first < tiles) load(x, first);
    }
    __device__ __forceinline__ void load(float (&to)[8], int t) const {
        const int i0 = t * kSampleTile + (threadIdx.x & 63);
        if ((t + 1) * kSampleTile <= vocab) {
#pragma unroll
            for (int j = 0; j < 8; ++j) to[j] = row[i0 + 64 * j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) to[j] = i0 + 64 * j < vocab ? row[i0 + 64 * j] : -INFINITY;
        }
    }
    template <class F>
    __device__ __forceinline__ void each(F f) {
        float next[8];
        for (int t = first; t < tiles; t += step) {
            if (t + step < tiles) load(next, t + step);
            f(t, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = next[j];
        }
    }
};

// First: the largest logits, a maximum for every four or sixteen lanes of a wave;
// and the row's space is cleared.  Bound by HBM, or by its start for few rows: 64
// rows, 38.9 MB, 8.0 us, 4,860 GB/s; one row 2.7 us.
__global__ __launch_bounds__(256) void sample_max_kernel(SampleArgs a) {
    int row, part;
    row_and_part(a.rows, row, part);
    const int lane = threadIdx.x & 63, wave = part * 4 + (threadIdx.x >> 6);
    SampleSpace* space = reinterpret_cast<SampleSpace*>(a.space + row * a.row_space);
    for (int i = part * 256 + threadIdx.x; i < kSampleBins; i += a.parts * 256) {
        space->mass[i] = 0;
        space->count[i] = 0;
    }
    if (part == 0 && threadIdx.x == 0) {
        space->listed = 0;
        space->first = a.vocab;
    }
    float top = -INFINITY;
    Tiles(a, row, wave, 4 * a.parts).each([&](int, const float (&x)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, x[j]);      // of NaN and a number, the number
    });
    uint32_t key = key_of(top);
    key = Max()(key, dpp<0xB1, 0xF>(key));
    key = Max()(key, dpp<0x4E, 0xF>(key));
    unsigned* largest = space->largest(a.tiles) + wave * a.wave_groups;
    if (a.wave_groups == 16) {
        if (lane % 4 == 0) largest[lane / 4] = key;
    } else {
        key = Max()(key, dpp<0x141, 0xF>(key));
        key = Max()(key, dpp<0x140, 0xF>(key));
        if (lane % 16 == 0) largest[lane / 16] = key;
    }
}

// Then the sums of rows without a cut, and what the others' cut is found from.
// A top-k of at most 512 goes by the groups: their k-th largest maximum is at
// most the k-th largest logit, so the logits from its bin on (some 1.4 k of
// them, if the large ones lie anywhere) hold the k.  Other filtered rows weigh (and
// with a top-k count) their tokens in 2,048 bins of the weight's logarithm.  Greedy rows look
// for the first of the largest logits.  64 rows 12.4 us, bound by the weights' series of
// some twenty operations a logit and the atomics on the bins in LDS; one row 4.9 us.
__global__ __launch_bounds__(256) void sample_cut_kernel(SampleArgs a) {
    __shared__ unsigned long long mass[kSampleBins];
    __shared__ unsigned count[kSampleBins];
    __shared__ Candidates found;
    __shared__ uint32_t lds[4];
    __shared__ int last;
    int row, part;
    row_and_part(a.rows, row, part);
    const int tid = threadIdx.x, lane = tid & 63, wave = part * 4 + (tid >> 6);
    Tiles tiles(a, row, wave, 4 * a.parts);
    SampleRow r = sample_settings(a, row);
    constexpr int kHeld = kMostGroups / 256;
    uint32_t held[kHeld], best = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        held[i] = tid + 256 * i < a.groups ? r.space->largest(a.tiles)[tid + 256 * i] : 0;
        best = Max()(best, held[i]);
    }
    best = wave_all(Max(), best);
    if (lane == 0) lds[tid >> 6] = best;
    count[tid] = 0;
    __syncthreads();
    sample_top(r, Max()(Max()(lds[0], lds[1]), Max()(lds[2], lds[3])));
    if (part == 0 && tid == 0) r.space->top_key = r.top_key;
    if (r.kind == kUnfiltered) {
        tiles.each([&](int t, const float (&x)[8]) {
            uint64_t sum = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint64_t w = weight_of(log_of(x[j], r.top, r.inverse));
                sum += w >= r.min_weight ? w : 0;
            }
            sum = wave_all(Sum(), sum);
            if (lane == 0) r.space->sums()[t] = sum;
        });
    } else if (r.kind == kByGroups) {
        // the bin of the k-th largest maximum (the last if fewer have a weight)
        static_assert(kGroupBins == 256, "a bin a thread");
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const float l = log_of(logit_of(held[i]), r.top, r.inverse);
            if (held[i] && l > kNoWeight) atomicAdd(&count[group_bin_of(l)], 1u);
        }
        if (tid == 0) last = kGroupBins - 1;
        found.clear();
        const uint32_t mine = count[tid];
        uint32_t all;
        const uint32_t upto = group_upto<4>(mine, lds, &all);
        if (upto >= static_cast<uint32_t>(r.k) && upto - mine < static_cast<uint32_t>(r.k)) last = tid;
        __syncthreads();
        const int bin = last;
        if (part == 0 && tid == 0) r.space->group_bin = bin;
        tiles.each([&](int t, const float (&x)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float l = log_of(x[j], r.top, r.inverse);
                const bool has = l > kNoWeight && group_bin_of(l) <= bin;
                if (__any(has)) found.add(has, t * kSampleTile + 64 * j + lane, r.space);
            }
        });
        found.to_list(r.space);
    } else if (r.kind == kByBins) {
        for (int i = tid; i < kSampleBins; i += 256) {
            mass[i] = 0;
            count[i] = 0;
        }
        __syncthreads();
        tiles.each([&](int, const float (&x)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float l = log_of(x[j], r.top, r.inverse);
                if (l > kNoWeight) {
                    atomicAdd(&mass[bin_of(l)], static_cast<unsigned long long>(weight_of(l)));
                    if (r.k) atomicAdd(&count[bin_of(l)], 1u);
                }
            }
        });
        __syncthreads();
        for (int i = tid; i < kSampleBins; i += 256) {
            if (mass[i]) atomicAdd(&r.space->mass[i], mass[i]);
            if (count[i]) atomicAdd(&r.space->count[i], count[i]);
        }
    } else if (r.top_key != kLowestKey) {
        tiles.each([&](int t, const float (&x)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = t * kSampleTile + 64 * j + lane;
                if (i < a.vocab && key_of(x[j]) == r.top_key) atomicMin(&r.space->first, i);
            }
        });
    }
}

// Then rows in bins: the bins that their cuts can lie in (top-p's share is one
// of top-k's weight, which bin_k leaves open a little), the tokens there, and
// of every tile the sum of the weights above them.  64 rows, 16 of them in bins,
// 11.9 us: the bins' sums, three tiles a wave, the list; 1.7 us where no row has any.
__global__ __launch_bounds__(256) void sample_bins_kernel(SampleArgs a, int parts) {
    __shared__ uint32_t lds[4];
    __shared__ uint64_t lds64[4];
    __shared__ unsigned long long found_mass[3];
    __shared__ unsigned found_count;
    __shared__ int found_bin[3];
    __shared__ Candidates found;
    int row, part;
    row_and_part(a.rows, row, part);
    const int tid = threadIdx.x, lane = tid & 63, wave = part * 4 + (tid >> 6);
    SampleRow r = sample_settings(a, row);
    if (r.kind != kByBins) return;
    Tiles tiles(a, row, wave, 4 * parts);
    sample_top(r, r.space->top_key);
    if (r.kind != kByBins) return;
    constexpr int kPer = kSampleBins / 256;
    uint64_t m[kPer], mine_mass = 0, all_mass;
    uint32_t c[kPer], mine_count = 0, all_count;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        m[i] = r.space->mass[tid * kPer + i];
        c[i] = r.space->count[tid * kPer + i];
        mine_mass += m[i];
        mine_count += c[i];
    }
    if (tid < 3) found_bin[tid] = -1;
    found.clear();
    const uint64_t mass0 = group_upto<4>(mine_mass, lds64, &all_mass) - mine_mass;
    const uint32_t count0 = group_upto<4>(mine_count, lds, &all_count) - mine_count;
    // the bin in which the count reaches k
    const bool by_k = r.k > 0 && static_cast<uint32_t>(r.k) < all_count;
    if (by_k) {
        uint64_t mb = mass0;
        uint32_t cb = count0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (cb < static_cast<uint32_t>(r.k) && cb + c[i] >= static_cast<uint32_t>(r.k)) {
                found_bin[0] = tid * kPer + i;
                found_count = cb;
                found_mass[0] = mb;
                found_mass[1] = mb + m[i];
            }
            mb += m[i];
            cb += c[i];
        }
    }
    __syncthreads();
    const int bin_k = found_bin[0];
    int low = bin_k, high = bin_k;
    uint64_t mass_low = by_k ? found_mass[0] : all_mass;
    if (r.top_p < 1.f) {
        const uint64_t from = share_of(r.top_p, by_k ? found_mass[0] : all_mass);
        const uint64_t to = share_of(r.top_p, by_k ? found_mass[1] : all_mass);
        uint64_t mb = mass0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (mb < from && mb + m[i] >= from) {
                found_bin[1] = tid * kPer + i;
                found_mass[2] = mb;
            }
            if (mb < to && mb + m[i] >= to) found_bin[2] = tid * kPer + i;
            mb += m[i];
        }
        __syncthreads();
        low = found_bin[1];
        high = by_k && bin_k < found_bin[2] ? bin_k : found_bin[2];
        mass_low = found_mass[2];
    } else if (!by_k) {
        low = high = kSampleBins;      // top-k leaves every token that has a weight
    }
    if (part == 0 && tid == 0) {
        r.space->bin_low = low;
        r.space->bin_high = high;
        r.space->bin_k = bin_k;
        r.space->count_k = by_k ? found_count : 0;
        r.space->mass_k = by_k ? found_mass[0] : 0;
        r.space->mass_low = mass_low;
        r.space->mass_all = all_mass;
    }
    tiles.each([&](int t, const float (&x)[8]) {
        uint64_t sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float l = log_of(x[j], r.top, r.inverse);
            const int b = bin_of(l);
            const uint64_t w = weight_of(l);
            sum += b < low && w >= r.min_weight ? w : 0;
            found.add(l > kNoWeight && ((b >= low && b <= high) || b == bin_k), t * kSampleTile + 64 * j + lane, r.space);
        }
        sum = wave_all(Sum(), sum);
        if (lane == 0) r.space->sums()[t] = sum;
    });
    found.to_list(r.space);
}

// v of lane ^ STEP
template <int STEP>
__device__ __forceinline__ uint64_t across(uint64_t v) {
    if constexpr (STEP == 1) return dpp<0xB1, 0xF>(v);
    else if constexpr (STEP == 2) return dpp<0x4E, 0xF>(v);
    else if constexpr (STEP == 4) return dpp<0x1B, 0xF>(dpp<0x141, 0xF>(v));
    else if constexpr (STEP == 8) return dpp<0x128, 0xF>(v);
    else return __shfl_xor(v, STEP, 64);
}

// sorts one number a thread, the first m (a power of two, at least 64) of the
// workgroup, falling
__device__ __forceinline__ uint64_t sorted(uint64_t v, int m, uint64_t* lds) {
    const int tid = threadIdx.x;
    for (int size = 2; size <= m; size <<= 1) {
        const bool falling = (tid & size) == 0;
        auto place = [&](uint64_t other, int step) {
            const bool larger = falling == ((tid & step) == 0);
            v = (v > other) == larger ? v : other;
        };
        for (int step = size >> 1; step >= 64; step >>= 1) {
            __syncthreads();
            lds[tid] = v;
            __syncthreads();
            place(lds[tid ^ step], step);
        }
        if (size > 32) place(across<32>(v), 32);
        if (size > 16) place(across<16>(v), 16);
        if (size > 8) place(across<8>(v), 8);
        if (size > 4) place(across<4>(v), 4);
        if (size > 2) place(across<2>(v), 2);
        place(across<1>(v), 1);
    }
    return v;
}

// Last: the cut, the tile that holds the point, and the token in it.  64 rows 8.9
// us, one row 6.4 us: a chain of loads (settings and sums, the candidates, their logits, the
// point's tile), a sort and five sums over the workgroup.  Loading all that the row's kind
// may need with the settings gained 0.1 us of it.
__global__ __launch_bounds__(kTokenThreads) void sample_token_kernel(SampleArgs a) {
    extern __shared__ unsigned long long sums[];      // of the tiles
    __shared__ uint64_t lds64[kSortList], waves64[kTokenWaves], one64[2];
    __shared__ uint32_t lds[kTokenWaves];
    __shared__ int one;
    const int row = blockIdx.x, tid = threadIdx.x;
    SampleRow r = sample_settings(a, row);
    sample_top(r, r.space->top_key);
    SampleSpace* space = r.space;
    if (r.kind == kFixed) {
        if (tid == 0) a.tokens[row] = r.top_key == kLowestKey ? -1 : space->first;
        return;
    }
    const bool by_groups = r.kind == kByGroups, by_bins = r.kind == kByBins;
    for (int i = tid; i < a.tiles; i += kTokenThreads) sums[i] = by_groups ? 0 : space->sums()[i];
    auto weigh = [&](uint32_t key) { return weight_of(log_of(logit_of(key), r.top, r.inverse)); };
    uint64_t cut = 0;                  // places from here on are left
    const int listed = r.kind == kUnfiltered ? 0 : static_cast<int>(space->listed);
    if (listed > 0) {
        const int low = by_bins ? space->bin_low : 0, high = by_bins ? space->bin_high : kSampleBins;
        const int bin_k = by_bins ? space->bin_k : -1;
        // top-k's tokens that the candidates hold (0: all of them); the weight above the candidates
        const int k = by_groups ? r.k : bin_k >= 0 ? r.k - static_cast<int>(space->count_k) : 0;
        const uint64_t above = by_bins ? space->mass_low : 0;
        auto bin_at = [&](uint64_t place) { return bin_of(log_of(logit_of(static_cast<uint32_t>(place >> 32)), r.top, r.inverse)); };
        if (listed <= kSortList) {
            uint64_t place = 0;
            if (tid < listed) {
                const uint32_t i = space->list[tid];
                place = place_of(key_of(r.x[i]), i);
            }
            int m = 64;
            while (m < listed) m <<= 1;
            place = sorted(place, m, lds64);
            const uint64_t w = tid < listed ? weigh(static_cast<uint32_t>(place >> 32)) : 0;
            uint64_t all;
            const uint64_t upto = group_upto<kTokenWaves>(w, waves64, &all);
            int before_k = 0;          // candidates above bin_k
            if (bin_k >= 0)
                before_k = static_cast<int>(group_sum<kTokenWaves>(static_cast<uint32_t>(tid < listed && bin_at(place) < bin_k), lds));
            const int last_k = k > 0 ? min(before_k + k, listed) - 1 : listed - 1;
            if (tid == last_k) one64[0] = upto;
            if (tid == before_k) one64[1] = upto - w;
            __syncthreads();
            const uint64_t left = by_groups ? one64[0] : bin_k >= 0 ? space->mass_k + one64[0] - one64[1] : space->mass_all;
            const uint64_t need = r.top_p < 1.f ? share_of(r.top_p, left) : left;
            const int end = by_bins && bin_k > high ? before_k : last_k + 1;
            const bool mine = tid < end && above + upto - w < need;
            __syncthreads();
            if (mine) lds64[tid] = place;
            const int n = static_cast<int>(group_sum<kTokenWaves>(static_cast<uint32_t>(mine), lds));
            cut = lds64[max(n, 1) - 1];
            if (mine && w >= r.min_weight)
                atomicAdd(&sums[static_cast<uint32_t>(~place) / kSampleTile], static_cast<unsigned long long>(w));
        } else {
            // many candidates (logits next to each other): bit by bit, from the list or from the row.  Of 151,936
            // logits, 2,000 equal ones and a top-k of 50: 107 us for one row, 130 for 64; all within 0.1: 64 passes over
            // the row for each filter, 3.9 ms for one and 5.4 ms for 64 rows of top-p, 6.3 and 9.2 with a top-k too
            const bool from_list = listed <= kSampleList;
            const int n = from_list ? listed : a.vocab;
            const int group_bin = by_groups ? space->group_bin : 0;
            auto each = [&](auto f) {
                for (int i = tid; i < n; i += kTokenThreads) {
                    const uint32_t index = from_list ? space->list[i] : i, key = key_of(r.x[index]);
                    const float l = log_of(logit_of(key), r.top, r.inverse);
                    const int b = bin_of(l);
                    if (from_list || (l > kNoWeight && (by_groups ? group_bin_of(l) <= group_bin : (b >= low && b <= high) || b == bin_k)))
                        f(place_of(key, index), b, l);
                }
            };
            uint64_t cut_k = 0, left = by_bins ? space->mass_all : 0;
            if (k > 0) {
                for (int bit = 63; bit >= 0; --bit) {
                    const uint64_t t = cut_k | 1ull << bit;
                    uint32_t c = 0;
                    each([&](uint64_t place, int b, float) { c += place >= t && (by_groups || b == bin_k); });
                    if (group_sum<kTokenWaves>(c, lds) >= static_cast<uint32_t>(k)) cut_k = t;
                }
                uint64_t s = 0;
                each([&](uint64_t place, int b, float l) { s += place >= cut_k && (by_groups || b == bin_k) ? weight_of(l) : 0; });
                left = group_sum<kTokenWaves>(s, waves64) + (by_bins ? space->mass_k : 0);
            }
            cut = cut_k;
            if (r.top_p < 1.f) {
                const uint64_t need = share_of(r.top_p, left);
                uint64_t c = 0;
                for (int bit = 63; bit >= 0; --bit) {
                    const uint64_t next = c | 1ull << bit, t = next > cut_k ? next : cut_k;
                    uint64_t s = 0;
                    each([&](uint64_t place, int b, float l) { s += place >= t && b >= low && b <= high ? weight_of(l) : 0; });
                    if (above + group_sum<kTokenWaves>(s, waves64) >= need) c |= 1ull << bit;
                }
                cut = c > cut_k ? c : cut_k;
            }
            each([&](uint64_t place, int b, float l) {
                const uint64_t w = weight_of(l);
                if (place >= cut && b >= low && b <= high && w >= r.min_weight)
                    atomicAdd(&sums[static_cast<uint32_t>(~place) / kSampleTile], static_cast<unsigned long long>(w));
            });
        }
    }
    __syncthreads();
    // the tile
    const int per = (a.tiles + kTokenThreads - 1) / kTokenThreads, t0 = min(a.tiles, tid * per), t1 = min(a.tiles, t0 + per);
    uint64_t mine = 0, all;
    for (int i = t0; i < t1; ++i) mine += sums[i];
    uint64_t before = group_upto<kTokenWaves>(mine, waves64, &all) - mine;
    const float u = a.u[row];
    const double at = floor((u > 0.f ? static_cast<double>(u) : 0.0) * static_cast<double>(all));
    const uint64_t point = at < static_cast<double>(all) ? min(static_cast<uint64_t>(at), all - 1) : all - 1;
    if (point >= before && point < before + mine)
        for (int i = t0; i < t1; ++i) {
            if (point < before + sums[i]) {
                one = i;
                one64[0] = before;
                break;
            }
            before += sums[i];
        }
    __syncthreads();
    const int i = one * kSampleTile + tid;
    uint64_t w = 0;
    if (tid < kSampleTile && i < a.vocab) {
        const uint32_t key = key_of(r.x[i]);
        if (place_of(key, i) >= cut) w = weigh(key);
        if (w < r.min_weight) w = 0;
    }
    const uint64_t upto = one64[0] + group_upto<kTokenWaves>(w, waves64, &all);
    if (point < upto && point >= upto - w) a.tokens[row] = i;
}

// bytes of a row's space
inline size_t sample_row_space(int vocab) {
    const size_t tiles = (vocab + kSampleTile - 1) / kSampleTile;
    return (sizeof(SampleSpace) + 8 * tiles + 4 * kMostGroups + 255) / 256 * 256;
}

}  // namespace tetra_dev
