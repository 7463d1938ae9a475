// The attention weight that cached tokens get from a call's rows (kv_weigh).
// Included by batch.hip.
//
//   mass'[s][h][j] = decay mass[s][h][j] + sum_i exp(s_ij) / sum_t exp(s_it)
//
// over the rows i (token, q head of the cache head h) of sequence s that see
// token j.
#pragma once

#include "kv_cache.h"

namespace tetra_dev {

struct WeighArgs {
    KvCache c;
    const uint16_t* q;
    const int* starts;
    const float* mass;
    float* out;
    float* logs;      // of every row and q head: log2 of the sum of its weights
    long long q_stride;
    float scale;      // scale log2(e)
    float decay;
    int rows, max_new, q_heads, group, window, mass_tokens;
};

template <int D>
__device__ float weigh_score(const WeighArgs& a, const uint16_t* q, int seq, int token, int head, bool* there) {
    const int page = a.c.pages[static_cast<size_t>(seq) * a.c.max_pages + (token >> a.c.page_shift)];
    *there = page >= 0 && page < a.c.num_pages;
    if (!*there) return -INFINITY;
    const size_t ph = static_cast<size_t>(page) * a.c.kv_heads + head;
    const int8_t* k = a.c.k + (ph * a.c.page_tokens + (token & (a.c.page_tokens - 1))) * D;
    float s = 0.f;
    for (int d = 0; d < D; ++d) s += static_cast<float>(__builtin_bit_cast(_Float16, q[d])) * static_cast<float>(k[d]);
    return s * a.c.scales[2 * ph] * a.scale;
}

__device__ __forceinline__ int weigh_end(const KvCache& c, int len) {
    return static_cast<int>(min(static_cast<long long>(max(len, 0)), static_cast<long long>(c.max_pages) << c.page_shift));
}

// a wave a row and q head
template <int D>
__global__ __launch_bounds__(64) void weigh_logs_kernel(WeighArgs a) {
    const int row = blockIdx.x / a.q_heads, h = blockIdx.x % a.q_heads, lane = threadIdx.x;
    const Place at = locate(a.starts, a.c.lens, a.rows, a.max_new, a.c.seqs, row, [](int start, int) { return start; });
    if (at.seq < 0 || row < at.s.row0 || row >= at.s.row0 + at.s.n) return;
    const int position = at.s.first + row - at.s.row0, end = min(position + 1, weigh_end(a.c, at.s.len));
    const int begin = a.window > 0 ? max(0, max(position, 0) - a.window + 1) : 0;
    const uint16_t* q = a.q + row * a.q_stride + h * D;
    float m = -3e38f, l = 0.f;
    bool there, bad = false;
    for (int t = begin + lane; t < end; t += 64) {
        const float s = weigh_score<D>(a, q, at.seq, t, h / a.group, &there);
        if (!there) continue;
        bad |= !(fabsf(s) < INFINITY);
        const float n = fmaxf(m, s);
        l = l * exp2f(m - n) + exp2f(s - n);
        m = n;
    }
    float top = m;
    for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i, 64));
    l = wave_all(Sum(), l * exp2f(m - top));
    if (lane == 0) a.logs[static_cast<size_t>(row) * a.q_heads + h] = l > 0.f ? top + log2f(l) : 0.f;
    if (__any(bad) && lane == 0) a.logs[static_cast<size_t>(row) * a.q_heads + h] = NAN;
}

// a thread a token of a cache head
template <int D>
__global__ __launch_bounds__(256) void weigh_add_kernel(WeighArgs a) {
    const int blocks = (a.mass_tokens + 255) / 256, seq = blockIdx.x / (blocks * a.c.kv_heads);
    const int head = blockIdx.x / blocks % a.c.kv_heads, t = blockIdx.x % blocks * 256 + threadIdx.x;
    const Span s = span_of(a.starts, a.c.lens, a.rows, a.max_new, seq);
    const int all = max(min(max(a.starts[seq + 1], 0), a.rows) - s.row0, 0);
    if (t >= a.mass_tokens || t >= a.c.lens[seq]) return;
    const size_t place = (static_cast<size_t>(seq) * a.c.kv_heads + head) * a.mass_tokens + t;
    float sum = 0.f;
    if (t < weigh_end(a.c, s.len))
        for (int i = max(0, t - s.first); i < s.n; ++i) {
            const int position = s.first + i;
            if (a.window > 0 && t <= position - a.window) break;
            for (int g = 0; g < a.group; ++g) {
                bool there;
                const int h = head * a.group + g;
                const float x = weigh_score<D>(a, a.q + (s.row0 + i) * a.q_stride + h * D, seq, t, head, &there);
                if (there) sum += exp2f(x - a.logs[static_cast<size_t>(s.row0 + i) * a.q_heads + h]);
            }
        }
    const float before = a.mass && (all == 0 || t < s.first) ? a.mass[place] * (all ? a.decay : 1.f) : 0.f;
    a.out[place] = before + sum;
}

}  // namespace tetra_dev
