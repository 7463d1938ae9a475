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
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tetra_dev {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr uint32_t kLowestKey = 0x007FFFFFu;   // of -inf

struct SampleArgs {
    const float* logits;
    long long stride;
    const float *temperature, *top_p, *min_p, *u;
    const int* top_k;
    int* tokens;
    int vocab;
};

// rises with x; NaN counts as -inf, and the zeros are equal
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x == 0.f ? 0.f : x);
    return x != x ? kLowestKey : b >> 31 ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float logit_of(uint32_t key) {
    return __builtin_bit_cast(float, key >> 31 ? key ^ 0x80000000u : ~key);
}

// 2^40 2^t, t = (x - top) inverse: the series of 2^f to f^7 with |f| <= 1/2
// (its remainder is 5e-9), every operation rounded by itself
__device__ __forceinline__ uint64_t weight_of(float x, float top, float inverse) {
#pragma clang fp contract(off)
    float t = x == top ? 0.f : (x - top) * inverse;
    t = fmaxf(t, -64.f);
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

template <class T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// the sum over the workgroup, in every thread
template <class T>
__device__ T group_sum(T v, T* lds) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = 0;
    for (int w = 0; w < kSampleWaves; ++w) s += lds[w];
    return s;
}

// the sum over the threads before this one
template <class T>
__device__ T group_before(T v, T* lds) {
    T s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T u = __shfl_up(s, o, 64);
        if ((threadIdx.x & 63) >= static_cast<unsigned>(o)) s += u;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    for (unsigned w = 0; w < threadIdx.x >> 6; ++w) s += lds[w];
    return s - v;
}

// A workgroup per row; the cut of top-k and of top-p is found bit by bit.
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
    __shared__ uint64_t lds[kSampleWaves];
    const int row = blockIdx.x, tid = threadIdx.x, n = a.vocab;
    const float* x = a.logits + row * a.stride;
    uint64_t best = 0;
    for (int i = tid; i < n; i += kSampleThreads)
        best = max(best, static_cast<uint64_t>(key_of(x[i])) << 32 | static_cast<uint32_t>(~i));
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) best = max(best, static_cast<uint64_t>(__shfl_xor(best, o, 64)));
    if ((tid & 63) == 0) lds[tid >> 6] = best;
    __syncthreads();
    for (int w = 0; w < kSampleWaves; ++w) best = max(best, lds[w]);
    const uint32_t top_key = static_cast<uint32_t>(best >> 32);
    const float top = logit_of(top_key), temperature = a.temperature[row];
    if (top_key == kLowestKey || !(temperature > 0.f)) {
        if (tid == 0) a.tokens[row] = top_key == kLowestKey ? -1 : static_cast<int>(~static_cast<uint32_t>(best));
        return;
    }
    const float inverse = 0x1.715476p+0f / temperature;
    // the tokens above key `cut`, and `ties` of those at it, are left
    uint32_t cut = 0;
    int ties = n;
    const int k = a.top_k[row];
    if (k > 0 && k < n) {
        for (int b = 31; b >= 0; --b) {
            const uint32_t t = cut | 1u << b;
            int c = 0;
            for (int i = tid; i < n; i += kSampleThreads) c += key_of(x[i]) >= t;
            if (group_sum<uint64_t>(c, lds) >= static_cast<uint64_t>(k)) cut = t;
        }
        int c = 0;
        for (int i = tid; i < n; i += kSampleThreads) c += key_of(x[i]) > cut;
        ties = k - static_cast<int>(group_sum<uint64_t>(c, lds));
    }
    auto mass_from = [&](uint32_t t) {
        uint64_t s = 0;
        for (int i = tid; i < n; i += kSampleThreads)
            if (key_of(x[i]) >= t) s += weight_of(logit_of(key_of(x[i])), top, inverse);
        return group_sum(s, lds);
    };
    const float p = a.top_p[row];
    if (p < 1.f) {
        uint64_t above = mass_from(cut + 1);
        const uint64_t all = cut ? above + ties * weight_of(logit_of(cut), top, inverse) : above;
        const double part = ceil(static_cast<double>(p) * static_cast<double>(all));
        const uint64_t need = part >= 1.0 ? static_cast<uint64_t>(part) : 1;
        if (above >= need) {
            uint32_t t = 0;
            for (int b = 31; b >= 0; --b)
                if (mass_from(t | 1u << b) >= need) t |= 1u << b;
            cut = t;
            ties = n;
            above = mass_from(cut + 1);
        }
        const uint64_t w = weight_of(logit_of(cut), top, inverse);
        if (w && cut) ties = static_cast<int>(min(static_cast<uint64_t>(ties), (need - above + w - 1) / w));
    }
    const double floor_d = fmin(fmax(static_cast<double>(a.min_p[row]), 0.0), 1.0) * 0x1p40;
    // a thread takes a run of the row: its ties' ranks, its sum, and the point in it
    const int run = (n + kSampleThreads - 1) / kSampleThreads, lo = min(n, tid * run), hi = min(n, lo + run);
    uint64_t c = 0;
    for (int i = lo; i < hi; ++i) c += key_of(x[i]) == cut;
    const uint64_t rank0 = group_before(c, lds);
    auto left = [&](int i, uint64_t& rank) -> uint64_t {
        const uint32_t key = key_of(x[i]);
        if (key < cut || (key == cut && rank++ >= static_cast<uint64_t>(ties))) return 0;
        const uint64_t w = weight_of(logit_of(key), top, inverse);
        return static_cast<double>(w) >= floor_d ? w : 0;
    };
    uint64_t mine = 0, rank = rank0;
    for (int i = lo; i < hi; ++i) mine += left(i, rank);
    const uint64_t before = group_before(mine, lds), all = group_sum(mine, lds);
    const float u = a.u[row];
    const double at = floor((u > 0.f ? static_cast<double>(u) : 0.0) * static_cast<double>(all));
    const uint64_t point = at < static_cast<double>(all) ? min(static_cast<uint64_t>(at), all - 1) : all - 1;
    if (point >= before && point < before + mine) {
        uint64_t s = before;
        rank = rank0;
        for (int i = lo; i < hi; ++i)
            if ((s += left(i, rank)) > point) {
                a.tokens[row] = i;
                break;
            }
    }
}

}  // namespace tetra_dev
