// Attention of a batch whose groups of sequences begin with the same pages
// (kv_attend_shared).  Included by serve.hip.
//
//   out_i = (f_0 o_0 + f_1 o_1) / (f_0 l_0 + f_1 l_1), f = 2^(m - max m),
//
// with m, l and o of attend.h over the shared tokens (0), which all rows of the
// group see, and over the sequence's own (1).  The kernels of attend.h take the
// groups and the sequences alike, as units of one launch: rows, and a range of
// the tokens of one table.  So a group's keys are read and turned into fp16 once
// for 16 rows or for 128, whichever sequences those are of, and its tokens are
// spread over the chip.  A first kernel lists the units, a last one joins the two
// sides; the sums of both are fp32 until then.
//
// 64 sequences of 32 heads over 8 of 128, 32,768 tokens in common and up to 1,000 of
// their own: 4.6 us for the list, 63 for the units (34 GFLOP, 540 TFLOP/s: matrix cores and
// vector units of the shared side, then the own side's chains of loads), 9 and 4.6 for the
// joins; kv_attend takes 587.  40 heads, 4,096 and up to 512: 4.2, 26, 7.2 and 3.6, and 78.
#pragma once

#include "attend.h"

namespace tetra_dev {

struct SharedGroup {
    int common;      // shared tokens, whole pages
    int row0, rows;  // of all its sequences
    int leader;      // the first sequence that takes part, whose table is read
};

struct SharedArgs {
    AttendArgs a;
    const int *groups, *shared;
    SharedSeq* list;         // [num_groups + seqs]: groups, then sequences
    SharedGroup* group;      // [num_groups]
    int num_groups;
};

// One workgroup.  A sequence takes part in its group (the first that holds it, of rising
// bounds) if it has rows and the first of them comes after the shared tokens.
constexpr int kListThreads = 1024;

__global__ __launch_bounds__(kListThreads) void shared_list_kernel(SharedArgs x) {
    const AttendArgs& a = x.a;
    const int seqs = a.c.seqs, tid = threadIdx.x;
    const int kept = static_cast<int>(min(static_cast<long long>(a.c.max_pages) << a.c.page_shift, 1ll << 30));
    auto bound = [&](int g) { return min(max(x.groups[g], 0), seqs); };
    // bounds that fall would put a row into two groups: then nothing is shared
    __shared__ int falls;
    if (tid == 0) falls = 0;
    __syncthreads();
    for (int g = tid; g < x.num_groups; g += kListThreads)
        if (x.groups[g + 1] < x.groups[g]) falls = 1;
    __syncthreads();
    for (int g = tid; g < x.num_groups; g += kListThreads) {
        const int from = bound(g), to = max(bound(g + 1), from);
        SharedGroup s;
        s.common = falls ? 0 : (min(max(x.shared[g], 0), kept) >> a.c.page_shift) << a.c.page_shift;
        s.row0 = min(max(a.starts[from], 0), a.rows);
        s.rows = max(min(max(a.starts[to], 0), a.rows) - s.row0, 0);
        s.leader = seqs;
        x.group[g] = s;
    }
    __threadfence_block();
    __syncthreads();
    for (int i = tid; i < seqs; i += kListThreads) {
        // the last group that begins at or before i
        int lo = 0, hi = x.num_groups;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (x.groups[mid] <= i) lo = mid;
            else hi = mid;
        }
        const Span s = span_of(a.starts, a.c.lens, a.rows, a.max_new, i);
        const Reach r = reach_of(a, s);
        SharedSeq own{s.row0, s.n, s.first, s.len, 0, r.end, i, 1};
        if (bound(lo) <= i && i < bound(lo + 1) && s.n > 0) {
            const SharedGroup g = x.group[lo];
            const bool inside = s.row0 >= g.row0 && s.row0 + s.n <= g.row0 + g.rows;
            if (g.common > 0 && s.first >= g.common && inside) {
                own.begin = g.common;
                atomicMin(&x.group[lo].leader, i);
            }
        }
        x.list[x.num_groups + i] = own;
    }
    __threadfence_block();
    __syncthreads();
    for (int g = tid; g < x.num_groups; g += kListThreads) {
        const SharedGroup s = x.group[g];
        const bool any = s.leader < seqs;
        x.list[g] = {s.row0, any ? s.rows : 0, s.common, s.common, 0, any ? s.common : 0, any ? s.leader : 0, 0};
    }
}

// The sides of a row joined: D / 4 lanes a head, 1024 / D heads a workgroup.  `begin` of
// the row's sequence tells whether it has a shared side.
template <int D>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs x) {
    const AttendArgs& a = x.a;
    constexpr int kHeads = 1024 / D;
    const int blocks = (a.q_heads + kHeads - 1) / kHeads, row = blockIdx.x / blocks;
    const int h = (blockIdx.x - row * blocks) * kHeads + static_cast<int>(threadIdx.x) / (D / 4), d = threadIdx.x % (D / 4) * 4;
    const Place at = locate(a.starts, a.c.lens, a.rows, a.max_new, a.c.seqs, row, [](int start, int) { return start; });
    if (at.seq < 0 || row < at.s.row0 || row >= at.s.row0 + at.s.n || h >= a.q_heads) return;
    const bool both = x.list[x.num_groups + at.seq].begin > 0;
    const size_t r0 = static_cast<size_t>(row) * a.q_heads + h, r1 = r0 + static_cast<size_t>(a.rows) * a.q_heads;
    const f32x2 s1 = *reinterpret_cast<const f32x2*>(a.stats + 2 * r1);
    f32x4 o = *reinterpret_cast<const f32x4*>(a.results + r1 * D + d);
    float l = s1[1];
    if (both) {
        const f32x2 s0 = *reinterpret_cast<const f32x2*>(a.stats + 2 * r0);
        const f32x4 o0 = *reinterpret_cast<const f32x4*>(a.results + r0 * D + d);
        const float m = fmaxf(s0[0], s1[0]), f0 = fast_exp2(s0[0] - m), f1 = fast_exp2(s1[0] - m);
        l = f0 * s0[1] + f1 * s1[1];
        o = f0 * o0 + f1 * o;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    f16x4 v;
    for (int i = 0; i < 4; ++i) v[i] = static_cast<_Float16>(o[i] * inv);
    *reinterpret_cast<f16x4*>(a.out + row * a.out_stride + h * D + d) = v;
}

}  // namespace tetra_dev
