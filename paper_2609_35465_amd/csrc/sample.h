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
// the cut is found from, the sums, and one workgroup a row for the rest.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tetra_dev {

constexpr uint32_t kLowestKey = 0x007FFFFFu;   // of -inf
constexpr int kSampleTile = 512;               // logits of a wave's step: 8 a lane, 64 apart
constexpr int kSampleGroup = 128;              // logits with a maximum of their own
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
    int vocab, tiles, groups, parts;
};

// What a row's kernels leave for each other, followed by the tiles' sums
// (uint64) and the groups' largest keys (uint32).
struct SampleSpace {
    unsigned long long mass[kSampleBins];
    unsigned count[kSampleBins];
    unsigned listed;                 // candidates found; the list holds the first kSampleList
    unsigned low_key;                // candidates by key: this and above
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

// t, a weight's logarithm
__device__ __forceinline__ float log_of(float x, float top, float inverse) {
#pragma clang fp contract(off)
    return fmaxf(x == top ? 0.f : (x - top) * inverse, -64.f);
}

// floor(2^40 2^t): the series of 2^f to f^7 with |f| <= 1/2 (its remainder is
// 5e-9), every operation rounded by itself
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
    const float s = p * __builtin_bit_cast(float, (static_cast<int>(whole) + 167) << 23);
    const uint32_t hi = static_cast<uint32_t>(s * 0x1p-20f);
    return (static_cast<uint64_t>(hi) << 20) + static_cast<uint32_t>(s - static_cast<float>(hi) * 0x1p20f);
}

constexpr float kNoWeight = -41.f;     // weights of this logarithm and below are 0

// falls with t
__device__ __forceinline__ int bin_of(float t) { return min(kSampleBins - 1, static_cast<int>(t * -kBinsPerUnit)); }

// the order of the tokens in one number: by key, then by index from the first on
__device__ __forceinline__ uint64_t place_of(uint32_t key, uint32_t index) {
    return static_cast<uint64_t>(key) << 32 | static_cast<uint32_t>(~index);
}

template <class T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <class T>
__device__ __forceinline__ T wave_max(T v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = max(v, static_cast<T>(__shfl_xor(v, o, 64)));
    return v;
}

// sum of the lanes up to and with this one
template <class T>
__device__ __forceinline__ T wave_upto(T v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T u = __shfl_up(v, o, 64);
        if ((threadIdx.x & 63) >= static_cast<unsigned>(o)) v += u;
    }
    return v;
}

// the sum over WAVES waves, in every thread
template <int WAVES, class T>
__device__ T group_sum(T v, T* lds) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += lds[w];
    return s;
}

// the sum over the threads up to and with this one, and over all
template <int WAVES, class T>
__device__ T group_upto(T v, T* lds, T* all) {
    v = wave_upto(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == static_cast<int>(threadIdx.x >> 6)) v += s;
        s += lds[w];
    }
    *all = s;
    return v;
}

enum SampleKind { kFixed, kByGroups, kByBins, kUnfiltered };

// What the kernels know of a row.
struct SampleRow {
    const float* x;
    SampleSpace* space;
    float top, inverse, top_p;
    uint32_t top_key;
    double min_weight;
    int k;               // of top-k, 0: off
    SampleKind kind;     // kFixed: the token needs no weights (greedy, or nothing but -inf)
};

// by every thread of a workgroup of WAVES waves, with a place in LDS each
template <int WAVES>
__device__ SampleRow sample_row(const SampleArgs& a, int row, uint32_t* lds) {
    SampleRow r;
    r.x = a.logits + row * a.stride;
    r.space = reinterpret_cast<SampleSpace*>(a.space + row * a.row_space);
    const unsigned* largest = r.space->largest(a.tiles);
    const float temperature = a.temperature[row];
    r.top_p = a.top_p[row];
    r.min_weight = fmin(fmax(static_cast<double>(a.min_p[row]), 0.0), 1.0) * 0x1p40;
    r.k = a.top_k[row];
    uint32_t best = 0;
    for (int i = threadIdx.x; i < a.groups; i += 64 * WAVES) best = max(best, largest[i]);
    best = wave_max(best);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) best = max(best, lds[w]);
    __syncthreads();
    r.top_key = best;
    r.top = logit_of(best);
    r.inverse = 0x1.715476p+0f / temperature;
    if (r.k < 0 || r.k >= a.vocab) r.k = 0;
    if (best == kLowestKey || !(temperature > 0.f)) r.kind = kFixed;
    else if (r.k > 0 && r.k <= kMostByGroups && 2 * r.k <= a.groups) r.kind = kByGroups;
    else if (r.k > 0 || r.top_p < 1.f) r.kind = kByBins;
    else r.kind = kUnfiltered;
    return r;
}

// ceil(p mass), one at least
__device__ __forceinline__ uint64_t share_of(float p, uint64_t mass) {
    const double s = ceil(static_cast<double>(p) * static_cast<double>(mass));
    return s >= 1.0 ? static_cast<uint64_t>(s) : 1;
}

// appends the flagged lanes' indices to the row's list
__device__ __forceinline__ void append(SampleSpace* space, bool has, int index) {
    const unsigned long long b = __ballot(has);
    if (!b) return;
    const int lane = threadIdx.x & 63, leader = __builtin_ctzll(b);
    unsigned at = 0;
    if (lane == leader) at = atomicAdd(&space->listed, static_cast<unsigned>(__popcll(b)));
    at = __shfl(at, leader, 64) + __popcll(b & ((1ull << lane) - 1));
    if (has && at < kSampleList) space->list[at] = index;
}

// First: the largest key of every 128 logits; and the row's space is cleared.
__global__ __launch_bounds__(256) void sample_max_kernel(SampleArgs a) {
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float* x = a.logits + row * a.stride;
    SampleSpace* space = reinterpret_cast<SampleSpace*>(a.space + row * a.row_space);
    for (int i = part * 256 + threadIdx.x; i < kSampleBins; i += a.parts * 256) {
        space->mass[i] = 0;
        space->count[i] = 0;
    }
    if (part == 0 && threadIdx.x == 0) space->listed = 0;
    unsigned* largest = space->largest(a.tiles);
    for (int t = part * 4 + wave; t < a.tiles; t += a.parts * 4) {
        uint32_t key[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = t * kSampleTile + 64 * j + lane;
            if (i < a.vocab) key[j / 2] = max(key[j / 2], key_of(x[i]));
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            key[g] = wave_max(key[g]);
            if (lane == g && 4 * t + g < a.groups) largest[4 * t + g] = key[g];
        }
    }
}

// Then what a filtered row's cut is found from.  A top-k of at most 512 goes by
// the groups: their k-th largest maximum is at most the k-th largest logit, so
// the logits from there on (some 1.4 k of them, if the large ones lie anywhere)
// hold the k.  Other filtered rows count and weigh their tokens in 2,048 bins of
// the weight's logarithm.
__global__ __launch_bounds__(256) void sample_cut_kernel(SampleArgs a) {
    __shared__ unsigned long long mass[kSampleBins];
    __shared__ unsigned count[kSampleBins];
    __shared__ uint32_t lds[4];
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const SampleRow r = sample_row<4>(a, row, lds);
    if (r.kind == kByGroups) {
        // the key's upper 16 bits, rounded down: a bound just as well
        const unsigned* largest = r.space->largest(a.tiles);
        constexpr int kHeld = 8;
        uint32_t held[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) held[i] = tid + 256 * i < a.groups ? largest[tid + 256 * i] : 0;
        uint32_t low = 0;
        for (int bit = 31; bit >= 16; --bit) {
            const uint32_t t = low | 1u << bit;
            uint32_t c = 0;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) c += held[i] >= t;
            for (int i = tid + 256 * kHeld; i < a.groups; i += 256) c += largest[i] >= t;
            if (group_sum<4>(c, lds) >= static_cast<uint32_t>(r.k)) low = t;
        }
        if (part == 0 && tid == 0) r.space->low_key = low;
        for (int t = part * 4 + wave; t < a.tiles; t += a.parts * 4) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = t * kSampleTile + 64 * j + lane;
                x[j] = i < a.vocab ? r.x[i] : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t key = key_of(x[j]);
                if (__any(key >= low))
                    append(r.space, key >= low && log_of(logit_of(key), r.top, r.inverse) > kNoWeight,
                           t * kSampleTile + 64 * j + lane);
            }
        }
    } else if (r.kind == kByBins) {
        for (int i = tid; i < kSampleBins; i += 256) {
            mass[i] = 0;
            count[i] = 0;
        }
        __syncthreads();
        for (int t = part * 4 + wave; t < a.tiles; t += a.parts * 4) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = t * kSampleTile + 64 * j + lane;
                x[j] = i < a.vocab ? r.x[i] : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float l = log_of(logit_of(key_of(x[j])), r.top, r.inverse);
                if (l > kNoWeight) {
                    atomicAdd(&mass[bin_of(l)], static_cast<unsigned long long>(weight_of(l)));
                    atomicAdd(&count[bin_of(l)], 1u);
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < kSampleBins; i += 256)
            if (count[i]) {
                atomicAdd(&r.space->mass[i], mass[i]);
                atomicAdd(&r.space->count[i], count[i]);
            }
    }
}

// Then the sums: of every tile's weights that are left for certain.  A row in
// bins first finds the bins that its cuts can lie in (top-p's share is one of
// top-k's weight, which bin_k leaves open a little), and lists the tokens there.
__global__ __launch_bounds__(256) void sample_sum_kernel(SampleArgs a) {
    __shared__ uint32_t lds[4];
    __shared__ unsigned long long lds64[4], found_mass[4];
    __shared__ unsigned found_count;
    __shared__ int found_bin[4];
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const SampleRow r = sample_row<4>(a, row, lds);
    if (r.kind != kByBins && r.kind != kUnfiltered) return;
    int low = kSampleBins, high = -1, bin_k = -1;
    if (r.kind == kByBins) {
        constexpr int kPer = kSampleBins / 256;
        unsigned long long m[kPer], mine_mass = 0, all_mass;
        uint32_t c[kPer], mine_count = 0, all_count;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            m[i] = r.space->mass[tid * kPer + i];
            c[i] = r.space->count[tid * kPer + i];
            mine_mass += m[i];
            mine_count += c[i];
        }
        const unsigned long long mass0 = group_upto<4>(mine_mass, lds64, &all_mass) - mine_mass;
        const uint32_t count0 = group_upto<4>(mine_count, lds, &all_count) - mine_count;
        if (tid < 4) found_bin[tid] = -1;
        __syncthreads();
        // the bin in which the count reaches k
        const bool by_k = r.k > 0 && static_cast<uint32_t>(r.k) < all_count;
        {
            unsigned long long mb = mass0;
            uint32_t cb = count0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (by_k && cb < static_cast<uint32_t>(r.k) && cb + c[i] >= static_cast<uint32_t>(r.k)) {
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
        bin_k = found_bin[0];
        const unsigned long long least = by_k ? found_mass[0] : all_mass, most = by_k ? found_mass[1] : all_mass;
        if (r.top_p < 1.f) {
            const unsigned long long from = share_of(r.top_p, least), to = share_of(r.top_p, most);
            unsigned long long mb = mass0;
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
            high = by_k ? min(found_bin[2], bin_k) : found_bin[2];
        } else {
            low = high = bin_k;
            if (tid == 0) found_mass[2] = found_mass[0];
            __syncthreads();
        }
        if (low < 0) low = high = kSampleBins;      // top-k leaves every token that has a weight
        if (part == 0 && tid == 0) {
            r.space->bin_low = low;
            r.space->bin_high = high;
            r.space->bin_k = bin_k;
            r.space->count_k = by_k ? found_count : 0;
            r.space->mass_k = by_k ? found_mass[0] : 0;
            r.space->mass_low = low < kSampleBins ? found_mass[2] : all_mass;
            r.space->mass_all = all_mass;
        }
    }
    for (int t = part * 4 + wave; t < a.tiles; t += a.parts * 4) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = t * kSampleTile + 64 * j + lane;
            x[j] = i < a.vocab ? r.x[i] : -INFINITY;
        }
        unsigned long long sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float l = log_of(logit_of(key_of(x[j])), r.top, r.inverse);
            const uint64_t w = weight_of(l);
            if (r.kind == kByBins) {
                const int b = bin_of(l);
                if (b < low && static_cast<double>(w) >= r.min_weight) sum += w;
                append(r.space, l > kNoWeight && ((b >= low && b <= high) || b == bin_k), t * kSampleTile + 64 * j + lane);
            } else if (static_cast<double>(w) >= r.min_weight) {
                sum += w;
            }
        }
        sum = wave_sum(sum);
        if (lane == 0) r.space->sums()[t] = sum;
    }
}

// sorts one number a thread, the first m (a power of two, at least 64) of the
// workgroup, falling
__device__ __forceinline__ uint64_t sorted(uint64_t v, int m, uint64_t* lds) {
    const int tid = threadIdx.x;
    for (int size = 2; size <= m; size <<= 1)
        for (int step = size >> 1; step >= 1; step >>= 1) {
            uint64_t other;
            if (step >= 64) {
                __syncthreads();
                lds[tid] = v;
                __syncthreads();
                other = lds[tid ^ step];
            } else {
                other = __shfl_xor(v, step, 64);
            }
            const bool larger_first = ((tid & size) == 0) == ((tid & step) == 0);
            v = larger_first ? max(v, other) : min(v, other);
        }
    return v;
}

// Last: the cut, the tile that holds the point, and the token in it.
__global__ __launch_bounds__(kTokenThreads) void sample_token_kernel(SampleArgs a) {
    extern __shared__ unsigned long long sums[];      // of the tiles
    __shared__ uint64_t lds64[kSortList], waves64[kTokenWaves], one64[2];
    __shared__ uint32_t lds[kTokenWaves];
    __shared__ int one;
    const int row = blockIdx.x, tid = threadIdx.x;
    const SampleRow r = sample_row<kTokenWaves>(a, row, lds);
    SampleSpace* space = r.space;
    if (r.kind == kFixed) {
        // the first of the largest
        const unsigned* largest = space->largest(a.tiles);
        if (tid == 0) one = a.groups;
        __syncthreads();
        for (int i = tid; i < a.groups; i += kTokenThreads)
            if (largest[i] == r.top_key) {
                atomicMin(&one, i);
                break;
            }
        __syncthreads();
        const int g = one, i = g * kSampleGroup + tid;
        __syncthreads();
        if (tid == 0) one = a.vocab;
        __syncthreads();
        if (tid < kSampleGroup && i < a.vocab && key_of(r.x[i]) == r.top_key) atomicMin(&one, i);
        __syncthreads();
        if (tid == 0) a.tokens[row] = r.top_key == kLowestKey ? -1 : one;
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
            if (mine && static_cast<double>(w) >= r.min_weight)
                atomicAdd(&sums[static_cast<uint32_t>(~place) / kSampleTile], static_cast<unsigned long long>(w));
        } else {
            // many candidates (logits next to each other): bit by bit, from the list or from the row
            const bool from_list = listed <= kSampleList;
            const int n = from_list ? listed : a.vocab;
            const uint32_t low_key = by_groups ? space->low_key : 0;
            auto each = [&](auto f) {
                for (int i = tid; i < n; i += kTokenThreads) {
                    const uint32_t index = from_list ? space->list[i] : i, key = key_of(r.x[index]);
                    const float l = log_of(logit_of(key), r.top, r.inverse);
                    const int b = bin_of(l);
                    if (from_list || (l > kNoWeight && (by_groups ? key >= low_key : (b >= low && b <= high) || b == bin_k)))
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
                if (place >= cut && b >= low && b <= high && static_cast<double>(w) >= r.min_weight)
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
        if (static_cast<double>(w) < r.min_weight) w = 0;
    }
    const uint64_t upto = one64[0] + group_upto<kTokenWaves>(w, waves64, &all);
    if (point < upto && point >= upto - w) a.tokens[row] = i;
}

// bytes of a row's space
inline size_t sample_row_space(int vocab) {
    const size_t tiles = (vocab + kSampleTile - 1) / kSampleTile, groups = (vocab + kSampleGroup - 1) / kSampleGroup;
    return (sizeof(SampleSpace) + 8 * tiles + 4 * groups + 255) / 256 * 256;
}

}  // namespace tetra_dev
