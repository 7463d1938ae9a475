// Log probabilities of given tokens, entropy and likeliest tokens of rows of
// logits (log_probs).  Included by batch.hip.
//
//   t_j = (x_j - m) / T, l = sum_j exp(t_j), log p_j = t_j - ln l,
//   entropy = ln l - sum_j exp(t_j) t_j / l
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lanes.h"

namespace tetra_dev {

constexpr int kMostTop = 64;

struct ScoreArgs {
    const void* logits;
    long long stride;
    const float* temperature;
    const int* tokens;
    float *out, *entropy, *top_out;
    int* top_tokens;
    int rows, vocab, given, top;
};

__device__ __forceinline__ uint32_t score_key(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x == 0.f ? 0.f : x);
    return x != x ? 0x007FFFFFu : b >> 31 ? ~b : b | 0x80000000u;
}

template <class T>
__device__ T score_all(T v, T* lds, bool sum) {
    for (int i = 1; i < 64; i *= 2) {
        const T o = __shfl_xor(v, i, 64);
        v = sum ? v + o : v > o ? v : o;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < 4; ++w) v = sum ? v + lds[w] : v > lds[w] ? v : lds[w];
    return v;
}

// a workgroup a row
template <class T>
__global__ __launch_bounds__(256) void score_kernel(ScoreArgs a) {
    __shared__ float lds[4];
    __shared__ unsigned long long places[4];
    const int row = blockIdx.x, tid = threadIdx.x;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    auto at = [&](int j) {
        const float v = static_cast<float>(x[j]);
        return v == v ? v : -INFINITY;
    };
    float temperature = a.temperature ? a.temperature[row] : 1.f;
    if (!(temperature > 0.f)) temperature = 1.f;
    const float inverse = fmaxf(1.f / temperature, 0x1p-126f);
    float m = -INFINITY;
    for (int j = tid; j < a.vocab; j += 256) m = fmaxf(m, at(j));
    m = score_all(m, lds, false);
    auto log_of = [&](float v) { return v == m ? 0.f : (v - m) * inverse; };
    float l = 0.f, u = 0.f;
    for (int j = tid; j < a.vocab; j += 256) {
        const float t = log_of(at(j)), e = expf(t);
        l += e;
        if (e > 0.f) u += e * t;
    }
    l = score_all(l, lds, true);
    u = score_all(u, lds, true);
    const bool none = m == -INFINITY;
    const float log_l = logf(l);
    for (int g = tid; g < a.given; g += 256) {
        const int j = a.tokens[static_cast<size_t>(row) * a.given + g];
        const bool is = j >= 0 && j < a.vocab && !none;
        a.out[static_cast<size_t>(row) * a.given + g] = is ? log_of(at(j)) - log_l : -INFINITY;
    }
    if (a.entropy && tid == 0) a.entropy[row] = none ? 0.f : log_l - u / l;
    unsigned long long before = ~0ull;
    for (int n = 0; n < a.top; ++n) {
        unsigned long long best = 0;
        for (int j = tid; j < a.vocab; j += 256) {
            const float v = at(j);
            const unsigned long long place = static_cast<unsigned long long>(score_key(v)) << 32 | static_cast<uint32_t>(~j);
            if (v > -INFINITY && place < before && place > best) best = place;
        }
        before = best = score_all(best, places, false);
        if (tid == 0) {
            const int j = static_cast<int>(~static_cast<uint32_t>(best));
            a.top_tokens[static_cast<size_t>(row) * a.top + n] = best ? j : -1;
            a.top_out[static_cast<size_t>(row) * a.top + n] = best ? log_of(at(j)) - log_l : -INFINITY;
        }
    }
}

}  // namespace tetra_dev
