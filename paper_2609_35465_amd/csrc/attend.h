// Attention over the paged 8-bit cache (kv_cache.h).  Included by serve.hip.
//
//   s_j = scale * q . k_j over the keys j that a row at position p sees: those
//   of its sequence with p - window < j <= p (window 0: from 0 on);
//   out = sum_j exp(s_j - max s) v_j / sum_j exp(s_j - max s), zeros without keys.
//
// One pass over the keys with the running maximum m and sum l (in units of
// log2).  The q heads that share a cache head are rows of one product, so a
// key is read once for all of them: the rows of a sequence and cache head are
// (token, q head of the group) in that order.
#pragma once

#include "kv_cache.h"

namespace tetra_dev {

struct AttendArgs {
    KvCache c;
    const uint16_t* q;
    const int* starts;
    uint16_t* out;
    float* partials;
    long long q_stride, out_stride;
    float scale;      // |scale| log2(e)
    uint32_t q_flip;  // 0x80008000 if the scale is negative: turns q instead
    int rows, max_new, q_heads, group, window;
};

constexpr float kNoScore = -3e38f;   // a maximum over no score
// A weight is 2^(s - m + 15) before it becomes fp16: the largest is 2^15, so
// weights down to 2^-29 of it keep their 11 bits.  l carries the same factor.
constexpr float kWeightShift = 15.f;

// four whole numbers of -128..127 as fp16, exactly: 1024 + (q + 128) is the
// byte q ^ 0x80 below the exponent byte 0x64
__device__ __forceinline__ void to_half(uint32_t q, f16x2& lo, f16x2& hi) {
    const uint32_t u = q ^ 0x80808080u;
    const f16x2 bias = {static_cast<_Float16>(-1152.f), static_cast<_Float16>(-1152.f)};
    lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + bias;
    hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + bias;
}

__device__ __forceinline__ f16x8 to_half8(uint32_t a, uint32_t b) {
    f16x2 w, x, y, z;
    to_half(a, w, x);
    to_half(b, y, z);
    return f16x8{w[0], w[1], x[0], x[1], y[0], y[1], z[0], z[1]};
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// maximum and sum over the four lanes of a row (lane % 16)
__device__ __forceinline__ float max_over_groups(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_over_groups(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// ---------------------------------------------------------------- few rows
//
// Sequences with few rows (single tokens): HBM-bound, so the work is split
// over the tokens.  A unit is 16 rows of a sequence and cache head, a tile 256
// tokens of a unit (64 for each of a workgroup's four waves).  The workgroups
// take equal contiguous ranges of all units' tiles, whatever the sequences'
// lengths (which only the device knows: every workgroup adds them up for
// itself).  Of a unit that spans several workgroups each stores its part, and
// a second kernel joins them.
//
// Products on v_mfma_f32_16x16x32_f16, transposed: S^T = K Q^T (A = 16 tokens,
// B = 16 rows) leaves a lane with scores of its own row (lane % 16), which are
// its operand of the second product O^T = V^T P^T as they stand, without any
// exchange: tile t of a wave's four takes token 16 g + 4 t + i as its row 4 g
// + i, so a lane of group g = lane / 16 gets the scores of 16 consecutive
// tokens, and its V operand is one 16-byte load of the transposed values.

constexpr int kFewWaves = 4;
constexpr int kFewTile = 64 * kFewWaves;
constexpr int kFewRows = 16;

// slots of a workgroup's parts: [2][kFewRows] m and l, [kFewRows][D] sums
template <int D>
constexpr int kFewSlot = kFewRows * (D + 2);

// the tokens that the rows of a sequence see, from a multiple of 64 on
struct Reach {
    int begin, end;
};

__device__ __forceinline__ Reach reach_of(const AttendArgs& a, const Span& s) {
    Reach r;
    const long long kept = static_cast<long long>(a.c.max_pages) << a.c.page_shift;
    r.end = static_cast<int>(min(static_cast<long long>(s.len), kept));
    r.begin = a.window > 0 ? max(0, s.first - a.window + 1) & ~63 : 0;
    return r;
}

// tiles of a sequence's unit (one at least, so that rows without keys are
// written) and its units
__device__ __forceinline__ int few_tiles(const Reach& r) { return max(1, (r.end - r.begin + kFewTile - 1) / kFewTile); }

__device__ __forceinline__ int few_work(const AttendArgs& a, int seq) {
    const Span s = span_of(a.starts, a.c.lens, a.rows, a.max_new, seq);
    const int units = (s.n * a.group + kFewRows - 1) / kFewRows * a.c.kv_heads;
    return units * few_tiles(reach_of(a, s));
}

// sum over the workgroup's four waves, in every thread
__device__ __forceinline__ int few_sum(int v, int* lds) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// the workgroups that take part, a tile each at least, and the first tile of one
__device__ __forceinline__ int few_workers(long long total, int launched) {
    return static_cast<int>(min(total, static_cast<long long>(launched)));
}
__device__ __forceinline__ long long few_from(int w, long long total, int workers) { return w * total / workers; }

template <int D>
struct FewState {
    float m, l, vref;
    f32x4 o[D / 16];
};

// A wave's blocks of a segment: tokens from `block0`, every kFewTile further, below `stop`.
template <int D>
__device__ __forceinline__ void few_segment(const AttendArgs& a, FewState<D>& st, const f16x8 (&q)[D / 32],
                                            const int* table, int head, int block0, int stop, int row_begin,
                                            int row_end) {
    constexpr int C = D / 64;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const size_t stride = static_cast<size_t>(a.c.page_tokens) * D;
    // page of the 16-token group at token t: its index in the pool times heads, or -1
    auto page_at = [&](int t) { return t < stop ? table[t >> a.c.page_shift] : -1; };
    struct Block {
        u32x4 k[4][C], v[D / 16];
        float ks, vs;
        bool there;
    };
    auto load = [&](Block& b, int t0, int pk, int pv) {
        const int tk = t0 + 16 * (r >> 2), tv = t0 + 16 * g;
        pk = pk < 0 || pk >= a.c.num_pages ? 0 : pk;
        b.there = pv >= 0 && pv < a.c.num_pages;
        pv = b.there ? pv : 0;
        const int8_t* kp = a.c.k + (static_cast<size_t>(pk) * a.c.kv_heads + head) * stride +
                           ((tk & (a.c.page_tokens - 1)) + (r & 3)) * D + 16 * g;
        const size_t ph = static_cast<size_t>(pv) * a.c.kv_heads + head;
        const int8_t* vp = a.c.v + ph * stride + (tv & (a.c.page_tokens - 1)) * D + 16 * r;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < C; ++c) b.k[t][c] = *reinterpret_cast<const u32x4*>(kp + 4 * t * D + 64 * c);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) b.v[d] = *reinterpret_cast<const u32x4*>(vp + 256 * d);
        const f32x2 s = *reinterpret_cast<const f32x2*>(a.c.scales + 2 * ph);
        b.ks = b.there ? s[0] : 0.f;
        b.vs = b.there ? s[1] : 0.f;
    };
    if (block0 >= stop) return;
    Block b;
    load(b, block0, page_at(block0 + 16 * (r >> 2)), page_at(block0 + 16 * g));
    for (int t0 = block0; t0 < stop; t0 += kFewTile) {
        const int next = t0 + kFewTile;
        const int pk = page_at(next + 16 * (r >> 2)), pv = page_at(next + 16 * g);
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const u32x4 k = b.k[t][c];
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half8(k[0], k[1]), q[2 * c], s[t], 0, 0, 0);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half8(k[2], k[3]), q[2 * c + 1], s[t], 0, 0, 0);
            }
        }
        const float sg = b.ks * a.scale;
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] *= sg;
        const int mine = t0 + 16 * g;       // the lane's 16 tokens
        if (__any(!b.there || mine < row_begin || mine + 16 > row_end)) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = mine + 4 * t + i;
                    if (!b.there || token < row_begin || token >= row_end) s[t][i] = -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
        const float m = fmaxf(st.m, max_over_groups(top));
        const float vref = fmaxf(st.vref, max_over_groups(b.vs));
        const float alpha = fast_exp2(st.m - m), beta = alpha * (st.vref / vref);
        st.l *= alpha;
        if (__any(beta != 1.f)) {
#pragma unroll
            for (f32x4& o : st.o) o *= beta;
        }
        st.m = m;
        st.vref = vref;
        // the page's scale of the values goes into the weights, relative to the largest so far
        const float rel = b.vs / vref;
        f16x8 p[2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = fast_exp2(s[t][i] - (m - kWeightShift));
                st.l += w;
                p[t / 2][4 * (t % 2) + i] = static_cast<_Float16>(w * rel);
            }
        Block n;
        if (next < stop) load(n, next, pk, pv);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            const u32x4 v = b.v[d];
            st.o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half8(v[0], v[1]), p[0], st.o[d], 0, 0, 0);
            st.o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half8(v[2], v[3]), p[1], st.o[d], 0, 0, 0);
        }
        b = n;
    }
}

template <int D>
__global__ __launch_bounds__(256, 2) void attend_few_kernel(AttendArgs a) {
    __shared__ float sums[kFewWaves][kFewRows][D + 4];
    __shared__ float stat[kFewWaves][kFewRows][2];
    __shared__ int lds[4], found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4, w = blockIdx.x;
    int mine = 0;
    for (int s = tid; s < a.c.seqs; s += 256) mine += few_work(a, s);
    const long long total = few_sum(mine, lds);
    const int W = few_workers(total, gridDim.x);
    if (w >= W) return;
    const int from = __builtin_amdgcn_readfirstlane(static_cast<int>(few_from(w, total, W)));
    const int to = __builtin_amdgcn_readfirstlane(static_cast<int>(few_from(w + 1, total, W)));
    // the sequence that holds tile `from`, and the tiles before it
    for (int s0 = 0, before = 0; s0 < a.c.seqs; s0 += 256) {
        const int n = s0 + tid < a.c.seqs ? few_work(a, s0 + tid) : 0;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(upto, o, 64);
            if (lane >= o) upto += u;
        }
        __syncthreads();
        if (lane == 63) lds[wave] = upto;
        __syncthreads();
        int all = 0;
        for (int i = 0; i < kFewWaves; ++i) {
            if (i < wave) upto += lds[i];
            all += lds[i];
        }
        upto += before;
        if (upto > from && upto - n <= from) {
            found[0] = s0 + tid;
            found[1] = upto - n;
        }
        before += all;
        if (before > from) break;
    }
    __syncthreads();
    int seq = __builtin_amdgcn_readfirstlane(found[0]), base = __builtin_amdgcn_readfirstlane(found[1]);
    bool first = true;
    for (int x = from; x < to && seq < a.c.seqs; ++seq) {
        const Span s = span_of(a.starts, a.c.lens, a.rows, a.max_new, seq);
        const Reach reach = reach_of(a, s);
        const int tiles = few_tiles(reach), rows = s.n * a.group;
        const int row_tiles = (rows + kFewRows - 1) / kFewRows, units = row_tiles * a.c.kv_heads;
        const int* table = a.c.pages + static_cast<size_t>(seq) * a.c.max_pages;
        for (int unit = (x - base) / tiles; unit < units && x < to; ++unit) {
            const int head = unit / row_tiles, row0 = (unit - head * row_tiles) * kFewRows;
            const int tile0 = x - base - unit * tiles, tile1 = min(tiles, tile0 + to - x);
            // the lane's row: its token, its q, what it sees
            const int row = row0 + r, token = row / a.group, h = head * a.group + row - token * a.group;
            const bool there = row < rows;
            const int position = s.first + token;
            const int row_end = there ? min(position + 1, reach.end) : 0;
            const int row_begin = a.window > 0 ? position - a.window + 1 : 0;
            f16x8 q[D / 32];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                u32x4 v = {0, 0, 0, 0};
                if (there)
                    v = *reinterpret_cast<const u32x4*>(a.q + (s.row0 + token) * a.q_stride + h * D + 64 * (c / 2) +
                                                        16 * g + 8 * (c % 2));
                q[c] = __builtin_bit_cast(f16x8, v ^ a.q_flip);
            }
            FewState<D> st;
            st.m = kNoScore;
            st.l = 0.f;
            st.vref = 1e-37f;
            for (f32x4& o : st.o) o = f32x4{0.f, 0.f, 0.f, 0.f};
            few_segment<D>(a, st, q, table, head, reach.begin + tile0 * kFewTile + wave * 64,
                           min(reach.end, reach.begin + tile1 * kFewTile), row_begin, row_end);
            const float l = sum_over_groups(st.l);
            __syncthreads();
            if (g == 0) {
                stat[wave][r][0] = st.m;
                stat[wave][r][1] = l;
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
                *reinterpret_cast<f32x4*>(&sums[wave][r][16 * d + 4 * g]) = st.o[d] * st.vref;
            __syncthreads();
            // the waves' sums joined, 4 dimensions a thread
            const bool whole = tile0 == 0 && tile1 == tiles;
            float* slot = a.partials + (2 * static_cast<size_t>(w) + (first ? 0 : 1)) * kFewSlot<D>;
            for (int e = tid; e < min(rows - row0, kFewRows) * (D / 4); e += 256) {
                const int er = e / (D / 4), ed = e % (D / 4) * 4;
                float m = stat[0][er][0];
                for (int i = 1; i < kFewWaves; ++i) m = fmaxf(m, stat[i][er][0]);
                float sum = 0.f;
                f32x4 o = {0.f, 0.f, 0.f, 0.f};
                for (int i = 0; i < kFewWaves; ++i) {
                    const float f = fast_exp2(stat[i][er][0] - m);
                    sum += f * stat[i][er][1];
                    o += f * *reinterpret_cast<const f32x4*>(&sums[i][er][ed]);
                }
                if (whole) {
                    const int t = (row0 + er) / a.group, eh = head * a.group + row0 + er - t * a.group;
                    const float inv = sum > 0.f ? 1.f / sum : 0.f;
                    f16x4 v;
                    for (int i = 0; i < 4; ++i) v[i] = static_cast<_Float16>(o[i] * inv);
                    *reinterpret_cast<f16x4*>(a.out + (s.row0 + t) * a.out_stride + eh * D + ed) = v;
                } else {
                    *reinterpret_cast<f32x4*>(slot + 2 * kFewRows + er * D + ed) = o;
                    if (ed == 0) {
                        slot[er] = m;
                        slot[kFewRows + er] = sum;
                    }
                }
            }
            x += tile1 - tile0;
            first = false;
        }
        base += units * tiles;
    }
}

// Joins the parts of the units that span workgroups of attend_few_kernel
// (`launched` of them): a workgroup per unit, a wave per row.
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, int launched, int row_tiles_most) {
    __shared__ int lds[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per_seq = a.c.kv_heads * row_tiles_most;
    const int seq = blockIdx.x / per_seq, unit = blockIdx.x - seq * per_seq;
    const Span s = span_of(a.starts, a.c.lens, a.rows, a.max_new, seq);
    const int rows = s.n * a.group, row_tiles = (rows + kFewRows - 1) / kFewRows;
    if (unit >= row_tiles * a.c.kv_heads) return;
    const int tiles = few_tiles(reach_of(a, s));
    if (tiles == 1) return;
    int all = 0, mine = 0;
    for (int i = tid; i < a.c.seqs; i += 256) {
        const int n = few_work(a, i);
        all += n;
        if (i < seq) mine += n;
    }
    const long long total = few_sum(all, lds);
    const int workers = few_workers(total, launched);
    const long long u0 = few_sum(mine, lds) + static_cast<long long>(unit) * tiles, u1 = u0 + tiles;
    const int w0 = static_cast<int>(((u0 + 1) * workers - 1) / total), w1 = static_cast<int>((u1 * workers - 1) / total);
    if (w0 == w1) return;
    const int head = unit / row_tiles, row0 = (unit - head * row_tiles) * kFewRows;
    const int slot0 = 2 * w0 + (few_from(w0, total, workers) >= u0 ? 0 : 1);
    auto slot = [&](int w) { return a.partials + static_cast<size_t>(w == w0 ? slot0 : 2 * w) * kFewSlot<D>; };
    for (int r = wave; r < min(kFewRows, rows - row0); r += kFewWaves) {
        float m = kNoScore;
        for (int w = w0 + lane; w <= w1; w += 64) m = fmaxf(m, slot(w)[r]);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        float l = 0.f, o[D / 64] = {};
        for (int w = w0; w <= w1; ++w) {
            const float* p = slot(w);
            const float f = fast_exp2(p[r] - m);
            l += f * p[kFewRows + r];
            for (int i = 0; i < D / 64; ++i) o[i] += f * p[2 * kFewRows + r * D + lane + 64 * i];
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const int t = (row0 + r) / a.group, h = head * a.group + row0 + r - t * a.group;
        _Float16* out = reinterpret_cast<_Float16*>(a.out) + (s.row0 + t) * a.out_stride + h * D;
        for (int i = 0; i < D / 64; ++i) out[lane + 64 * i] = static_cast<_Float16>(o[i] * inv);
    }
}

}  // namespace tetra_dev
