// Attention over the paged 8-bit cache (kv_cache.h).  Included by serve.hip.
//
//   s_j = scale * q . k_j over the keys j that a row at position p sees: those
//   of its sequence with p - window < j <= p (window 0: from 0 on);
//   out = sum_j exp(s_j - max s) v_j / sum_j exp(s_j - max s), zeros without keys.
//
// One pass with the running maximum m and sum l.  Plain form: a wave takes one
// row and head, a lane a key of each 64.
#pragma once

#include "kv_cache.h"

namespace tetra_dev {

struct AttendArgs {
    KvCache c;
    const uint16_t* q;
    const int* starts;
    uint16_t* out;
    long long q_stride, out_stride;
    float scale;      // of the scores, times log2(e)
    int rows, max_new, q_heads, window;
};

template <int D>
__global__ __launch_bounds__(64) void attend_kernel(AttendArgs a) {
    __shared__ float qs[D];
    const int lane = threadIdx.x;
    const int row = static_cast<int>(blockIdx.x) / a.q_heads, h = static_cast<int>(blockIdx.x) % a.q_heads;
    const int seq = count_upto(a.c.seqs, row, [&](int i) { return a.starts[i + 1]; });
    if (seq >= a.c.seqs) return;
    const Span s = span_of(a.starts, a.c.lens, a.rows, a.max_new, seq);
    if (row < s.row0 || row >= s.row0 + s.n) return;
    const int position = s.first + row - s.row0;
    const int head = h / (a.q_heads / a.c.kv_heads);
    const int end = static_cast<int>(min(static_cast<long long>(position) + 1,
                                         static_cast<long long>(a.c.max_pages) << a.c.page_shift));
    const int begin = a.window > 0 ? max(0, position - a.window + 1) : 0;
    const _Float16* q = reinterpret_cast<const _Float16*>(a.q) + row * a.q_stride + h * D;
    for (int d = lane; d < D; d += 64) qs[d] = static_cast<float>(q[d]);
    __syncthreads();
    float m = -1e30f, l = 0.f, o[D / 64] = {};
    for (int t0 = begin; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        float sc = -INFINITY, vs = 0.f;
        size_t base = 0;
        if (t < end) {
            const int page = a.c.pages[static_cast<size_t>(seq) * a.c.max_pages + (t >> a.c.page_shift)];
            if (page >= 0 && page < a.c.num_pages) {
                const size_t ph = static_cast<size_t>(page) * a.c.kv_heads + head;
                const int at = t & (a.c.page_tokens - 1);
                const int8_t* k = a.c.k + (ph * a.c.page_tokens + at) * D;
                float dot = 0.f;
                for (int d = 0; d < D; ++d) dot += qs[d] * static_cast<float>(k[d]);
                sc = dot * a.c.scales[2 * ph] * a.scale;
                vs = a.c.scales[2 * ph + 1];
                base = (ph * a.c.page_tokens + (at & ~15)) * D + (at & 15);
            }
        }
        float top = sc;
        for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
        top = fmaxf(top, m);
        const float alpha = exp2f(m - top), p = exp2f(sc - top);
        m = top;
        l = l * alpha + p;
        for (float& e : o) e *= alpha;
        const float pv = p * vs;
        for (int j = 0; j < 64; ++j) {
            const float w = __shfl(pv, j, 64);
            const size_t b = __shfl(static_cast<unsigned long long>(base), j, 64);
            if (w == 0.f) continue;
            for (int i = 0; i < D / 64; ++i) o[i] += w * static_cast<float>(a.c.v[b + (lane + 64 * i) * 16]);
        }
    }
    for (int x = 32; x >= 1; x >>= 1) l += __shfl_xor(l, x, 64);
    _Float16* out = reinterpret_cast<_Float16*>(a.out) + row * a.out_stride + h * D;
    for (int i = 0; i < D / 64; ++i) out[lane + 64 * i] = static_cast<_Float16>(l > 0.f ? o[i] / l : 0.f);
}

}  // namespace tetra_dev
