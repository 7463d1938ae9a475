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
    float* partials;  // of attend_few's workgroups
    float* pieces;    // of the many-row units
    long long q_stride, out_stride;
    float scale;      // |scale| log2(e)
    uint32_t q_flip;  // 0x80008000 if the scale is negative: turns q instead
    int rows, max_new, q_heads, group, window;
    int few_tile;     // tokens of a tile of attend_few: 64 for each wave of its workgroups
    int few_most;     // sequences of up to so many rows (token, q head of a group) go through attend_few_kernel
};

constexpr float kNoScore = -3e38f;   // a maximum over no score
// The scale of a key's values goes into its weight's exponent: the second product
// takes w = 2^(s + v - m + 15) in fp16, v = log2 of the scale and m the running
// maximum of s + v over the keys that the row sees, and l = sum 2^(-v) w.  So the
// largest product with a value decides what is rounded away, whatever the pages'
// scales are, and pages that a row does not see have no part in it.  fp16 keeps 11
// bits of weights down to 2^-29 of the largest where it is 2^15; attend_many_kernel
// lets m stay behind by up to kSlack, and there it is 2^-21.
//
// The matrix cores take fp16 against the values, which are exact in it; a weight's
// rounding, 2^-12 at most, takes the output's distance from 64 bits from 2.1e-4 of
// its norm (that of fp16 outputs alone) to 2.2e-4 (few rows, whose largest weight is
// exact) and 2.7e-4.  A second product with what the rounding leaves of the weights
// gives 2.1e-4 and took 4,096 tokens from 165 to 221 us, 64 single tokens from 49.3
// to 50.8.
constexpr float kWeightShift = 15.f;

// v: bounds that an fp16 output cannot tell from scales beyond them (127 times 2^-40
// is a 512th of its smallest step), so that neither w, l nor their quotient leaves
// fp32's range while the output is in fp16's
__device__ __forceinline__ float log_scale(float scale) {
    return fminf(fmaxf(__builtin_amdgcn_logf(scale), -40.f), 125.f);
}

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

// eight of a row's q, turned if the scale is negative.  An infinity becomes NaN, or
// it would leave weights of zero and no trace where all its scores are -inf.
__device__ __forceinline__ f16x8 query8(u32x4 v, uint32_t flip) {
    const f16x8 q = __builtin_bit_cast(f16x8, v ^ flip);
    return q + q * static_cast<_Float16>(0.f);
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

struct Larger {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// over the four lanes of a row (lane % 16)
template <class F>
__device__ __forceinline__ float over_groups(F f, float v) { return with_half(f, with_row(f, v)); }

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
// Measured: one sequence of 131,072 tokens, 8 heads of 128: 55 us, 4,890 GB/s of
// keys and values (a large copy reaches 5,030 here), and 6 to 7 us for the join;
// 64 sequences of up to 4,096 tokens, 182 MB: 43 us, 4,230 GB/s, and 5 us.  One
// of 203 tokens: 6 us, the way through memory four times over (the spans, the
// page table, the keys, the weighted values) and no bandwidth to speak of.
//
// Products on v_mfma_f32_16x16x32_f16, transposed: S^T = K Q^T (A = 16 tokens,
// B = 16 rows) leaves a lane with scores of its own row (lane % 16), which are
// its operand of the second product O^T = V^T P^T as they stand, without any
// exchange: tile t of a wave's four takes token 16 g + 4 t + i as its row 4 g
// + i, so a lane of group g = lane / 16 gets the scores of 16 consecutive
// tokens, and its V operand is one 16-byte load of the transposed values.

constexpr int kFewRows = 16;

// slots of a workgroup's parts: [2][kFewRows] m and l, [kFewRows][D] sums
template <int D>
constexpr int kFewSlot = kFewRows * (D + 2);

// the tokens that the rows of a sequence see, from a multiple of 64 on
struct Reach {
    int begin, end;
};

// the first token that a row at `position` may see; one below zero sees none, and
// any window may be taken from the others
__device__ __forceinline__ int window_begin(const AttendArgs& a, int position) {
    return a.window > 0 ? max(position, 0) - a.window + 1 : 0;
}

// a multiple of 64 at or below that token, and below `end` rounded up to one: a
// length may lie far past the table, whose tokens alone are counted from here
__device__ __forceinline__ int reach_begin_of(const AttendArgs& a, int position, int end) {
    return min(max(0, window_begin(a, position)), max(end, 0) + 63) & ~63;
}

__device__ __forceinline__ Reach reach_of(const AttendArgs& a, const Span& s) {
    Reach r;
    const long long kept = static_cast<long long>(a.c.max_pages) << a.c.page_shift;
    r.end = static_cast<int>(min(static_cast<long long>(s.len), kept));
    r.begin = reach_begin_of(a, s.first, r.end);
    return r;
}

// tiles of a sequence's unit (one at least, so that rows without keys are
// written) and its units
__device__ __forceinline__ int few_tiles(const AttendArgs& a, const Reach& r) {
    return max(1, (r.end - r.begin + a.few_tile - 1) / a.few_tile);
}

// row tiles of a sequence: none if it goes through attend_many_kernel
__device__ __forceinline__ int few_row_tiles(const AttendArgs& a, const Span& s) {
    const int rows = s.n * a.group;
    return rows > a.few_most ? 0 : (rows + kFewRows - 1) / kFewRows;
}

__device__ __forceinline__ int few_work(const AttendArgs& a, const Span& s) {
    return few_row_tiles(a, s) * a.c.kv_heads * few_tiles(a, reach_of(a, s));
}

// sum over the workgroup's WAVES waves, in every thread
template <int WAVES, class T>
__device__ __forceinline__ T few_sum(T v, T* lds) {
    v = wave_all(Sum(), v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < WAVES; ++w) v += lds[w];
    return v;
}

// The workgroups that take part, a tile each at least, the first tile of one and
// the one that has a tile.
struct FewPlan {
    int workers, share, more;      // `more` workgroups take share + 1 tiles, the others share

    __device__ __forceinline__ FewPlan(int total, int launched) {
        workers = min(total, launched);
        share = total / max(workers, 1);
        more = total - share * workers;
    }
    __device__ __forceinline__ int from(int w) const { return w * share + min(w, more); }
    __device__ __forceinline__ int owner(int tile) const {
        const int big = more * (share + 1);
        return tile < big ? tile / (share + 1) : more + (tile - big) / share;
    }
};

template <int D>
struct FewState {
    float m, l;
    f32x4 o[D / 16];
};

// A wave's blocks of a segment: tokens from `block0`, every STEP further, below `stop`.
template <int D, int STEP>
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
    for (int t0 = block0; t0 < stop; t0 += STEP) {
        const int next = t0 + STEP;
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
        // the lane's 16 tokens lie in one page
        const float sg = b.ks * a.scale, lv = log_scale(b.vs);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[t][i] = __builtin_fmaf(s[t][i], sg, lv);
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
        const float m = fmaxf(st.m, over_groups(Larger(), top));
        const float alpha = fast_exp2(st.m - m);
        st.l *= alpha;
        if (__any(alpha != 1.f)) {
#pragma unroll
            for (f32x4& o : st.o) o *= alpha;
        }
        st.m = m;
        f16x8 p[2];
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = fast_exp2(s[t][i] - (m - kWeightShift));
                sum += w;
                p[t / 2][4 * (t % 2) + i] = static_cast<_Float16>(w);
            }
        st.l += sum * fast_exp2(-lv);
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

template <int D, int WAVES>
struct FewLds {
    float sums[WAVES][kFewRows][D + 4];
    float stat[WAVES][kFewRows][2];
    int lds[WAVES], found[2];
    Span span;
};

// workgroup w of `launched`, WAVES waves each (a.few_tile is 64 WAVES)
template <int D, int WAVES>
__device__ __forceinline__ void attend_few(const AttendArgs& a, int w, int launched, FewLds<D, WAVES>& sh) {
    constexpr int kTile = 64 * WAVES;      // tokens, and threads
    auto& sums = sh.sums;
    auto& stat = sh.stat;
    auto& lds = sh.lds;
    auto& found = sh.found;
    Span& found_span = sh.span;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    // The total, and the sequence that holds this workgroup's first tile with the
    // tiles before it.  As many sequences as threads are one scan, more take two passes.
    auto scan = [&](int n, int& all) {
        int upto = wave_upto(Sum(), n);
        __syncthreads();
        if (lane == 63) lds[wave] = upto;
        __syncthreads();
        all = 0;
        for (int i = 0; i < WAVES; ++i) {
            if (i < wave) upto += lds[i];
            all += lds[i];
        }
        return upto;
    };
    Span mine = {};
    int n0 = 0;
    if (tid < a.c.seqs) {
        mine = span_of(a.starts, a.c.lens, a.rows, a.max_new, tid);
        n0 = few_work(a, mine);
    }
    int all, upto = scan(n0, all), total = all;
    if (a.c.seqs > kTile) {
        int more = 0;
        for (int i = tid + kTile; i < a.c.seqs; i += kTile)
            more += few_work(a, span_of(a.starts, a.c.lens, a.rows, a.max_new, i));
        total += few_sum<WAVES>(more, lds);
    }
    const FewPlan plan(__builtin_amdgcn_readfirstlane(total), launched);
    if (w >= plan.workers) return;
    const int from = plan.from(w), to = plan.from(w + 1);
    for (int s0 = 0, n = n0, before = 0;;) {
        if (upto > from && upto - n <= from) {
            found[0] = s0 + tid;
            found[1] = upto - n;
            found_span = mine;
        }
        before += all;
        s0 += kTile;
        if (before > from || s0 >= a.c.seqs) break;
        n = 0;
        if (s0 + tid < a.c.seqs) {
            mine = span_of(a.starts, a.c.lens, a.rows, a.max_new, s0 + tid);
            n = few_work(a, mine);
        }
        upto = scan(n, all) + before;
    }
    __syncthreads();
    int seq = __builtin_amdgcn_readfirstlane(found[0]), base = __builtin_amdgcn_readfirstlane(found[1]);
    Span s;
    s.row0 = __builtin_amdgcn_readfirstlane(found_span.row0);
    s.n = __builtin_amdgcn_readfirstlane(found_span.n);
    s.first = __builtin_amdgcn_readfirstlane(found_span.first);
    s.len = __builtin_amdgcn_readfirstlane(found_span.len);
    bool first = true;
    for (int x = from; x < to && seq < a.c.seqs; ++seq) {
        if (!first) s = span_of(a.starts, a.c.lens, a.rows, a.max_new, seq);
        const Reach reach = reach_of(a, s);
        const int tiles = few_tiles(a, reach), rows = s.n * a.group;
        const int row_tiles = few_row_tiles(a, s), units = row_tiles * a.c.kv_heads;
        const int* table = a.c.pages + static_cast<size_t>(seq) * a.c.max_pages;
        for (int unit = (x - base) / tiles; unit < units && x < to; ++unit) {
            const int head = unit / row_tiles, row0 = (unit - head * row_tiles) * kFewRows;
            const int tile0 = x - base - unit * tiles, tile1 = min(tiles, tile0 + to - x);
            // the lane's row: its token, its q, what it sees
            const int row = row0 + r, token = row / a.group, h = head * a.group + row - token * a.group;
            const bool there = row < rows;
            const int position = s.first + token;
            const int row_end = there ? min(position + 1, reach.end) : 0;
            const int row_begin = window_begin(a, position);
            f16x8 q[D / 32];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                u32x4 v = {0, 0, 0, 0};
                if (there)
                    v = *reinterpret_cast<const u32x4*>(a.q + (s.row0 + token) * a.q_stride + h * D + 64 * (c / 2) +
                                                        16 * g + 8 * (c % 2));
                q[c] = query8(v, a.q_flip);
            }
            FewState<D> st;
            st.m = kNoScore;
            st.l = 0.f;
            for (f32x4& o : st.o) o = f32x4{0.f, 0.f, 0.f, 0.f};
            few_segment<D, kTile>(a, st, q, table, head, reach.begin + tile0 * kTile + wave * 64,
                                  min(reach.end, reach.begin + tile1 * kTile), row_begin, row_end);
            const float l = over_groups(Sum(), st.l);
            __syncthreads();
            if (g == 0) {
                stat[wave][r][0] = st.m;
                stat[wave][r][1] = l;
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
                *reinterpret_cast<f32x4*>(&sums[wave][r][16 * d + 4 * g]) = st.o[d];
            __syncthreads();
            // the waves' sums joined, 4 dimensions a thread
            const bool whole = tile0 == 0 && tile1 == tiles;
            float* slot = a.partials + (2 * static_cast<size_t>(w) + (first ? 0 : 1)) * kFewSlot<D>;
            for (int e = tid; e < min(rows - row0, kFewRows) * (D / 4); e += kTile) {
                const int er = e / (D / 4), ed = e % (D / 4) * 4;
                float m = stat[0][er][0];
                for (int i = 1; i < WAVES; ++i) m = fmaxf(m, stat[i][er][0]);
                float sum = 0.f;
                f32x4 o = {0.f, 0.f, 0.f, 0.f};
                for (int i = 0; i < WAVES; ++i) {
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

template <int D>
__global__ __launch_bounds__(256, 2) void attend_few_kernel(AttendArgs a) {
    __shared__ FewLds<D, 4> sh;
    attend_few<D, 4>(a, blockIdx.x, gridDim.x, sh);
}

// Joins the parts of the units that span workgroups of attend_few (`launched` of
// them): a workgroup per `span` (1, 2, 4 or 8) rows of a unit, D / 4 lanes for the
// dimensions and teams of them for the rows and the parts.
struct JoinShape {
    int launched, row_tiles_most, spans, span;
};

template <int D>
__device__ __forceinline__ void attend_join(const AttendArgs& a, int block, const JoinShape& shape) {
    const int launched = shape.launched, row_tiles_most = shape.row_tiles_most, spans = shape.spans, span = shape.span;
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes;
    __shared__ unsigned long long lds[4];
    __shared__ float sums[kTeams][D + 4], stat[kTeams][2];
    const int tid = threadIdx.x;
    const int rest = block / spans, per_seq = a.c.kv_heads * row_tiles_most;
    const int seq = rest / per_seq, unit = rest - seq * per_seq;
    const Span s = span_of(a.starts, a.c.lens, a.rows, a.max_new, seq);
    const int rows = s.n * a.group, row_tiles = few_row_tiles(a, s);
    if (unit >= row_tiles * a.c.kv_heads) return;
    const int head = unit / row_tiles, row0 = (unit - head * row_tiles) * kFewRows;
    const int r0 = (block - rest * spans) * span;
    const int tiles = few_tiles(a, reach_of(a, s));
    if (tiles == 1 || row0 + r0 >= rows) return;
    unsigned long long work = 0;        // of all sequences, and above that of those before this one
    for (int i = tid; i < a.c.seqs; i += 256) {
        const unsigned n = few_work(a, span_of(a.starts, a.c.lens, a.rows, a.max_new, i));
        work += n;
        if (i < seq) work += static_cast<unsigned long long>(n) << 32;
    }
    work = few_sum<4>(work, lds);
    const FewPlan plan(static_cast<int>(work), launched);
    const int u0 = static_cast<int>(work >> 32) + unit * tiles, w0 = plan.owner(u0), w1 = plan.owner(u0 + tiles - 1);
    if (w0 == w1) return;
    // the unit's first workgroup may have begun with another unit
    const float* part0 = a.partials + (2 * static_cast<size_t>(w0) + (plan.from(w0) == u0 ? 0 : 1)) * kFewSlot<D>;
    auto part = [&](int w) { return w == w0 ? part0 : a.partials + 2 * static_cast<size_t>(w) * kFewSlot<D>; };
    // teams span t + i take row r0 + i
    const int team = tid / kLanes, r = r0 + team % span, d = tid % kLanes * 4;
    const bool there = r < kFewRows && row0 + r < rows;
    float m = kNoScore, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (there)
        for (int w = w0 + team / span; w <= w1; w += kTeams / span) {
            const float* p = part(w);
            const f32x4 x = *reinterpret_cast<const f32x4*>(p + 2 * kFewRows + r * D + d);
            const float pm = p[r], mnew = fmaxf(m, pm), fo = fast_exp2(m - mnew), fp = fast_exp2(pm - mnew);
            l = l * fo + p[kFewRows + r] * fp;
            o = o * fo + x * fp;
            m = mnew;
        }
    // the first team of a row adds the others
    if (d == 0) {
        stat[team][0] = m;
        stat[team][1] = l;
    }
    *reinterpret_cast<f32x4*>(&sums[team][d]) = o;
    __syncthreads();
    if (!there || team >= span) return;
    for (int i = team + span; i < kTeams; i += span) {
        const float pm = stat[i][0], mnew = fmaxf(m, pm), fo = fast_exp2(m - mnew), fp = fast_exp2(pm - mnew);
        l = l * fo + stat[i][1] * fp;
        o = o * fo + *reinterpret_cast<const f32x4*>(&sums[i][d]) * fp;
        m = mnew;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int t = (row0 + r) / a.group, h = head * a.group + row0 + r - t * a.group;
    f16x4 v;
    for (int i = 0; i < 4; ++i) v[i] = static_cast<_Float16>(o[i] * inv);
    *reinterpret_cast<f16x4*>(a.out + (s.row0 + t) * a.out_stride + h * D + d) = v;
}

template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, JoinShape shape) {
    attend_join<D>(a, blockIdx.x, shape);
}

// ---------------------------------------------------------------- many rows
//
// Sequences with many rows (prompts): bound by the matrix cores and the vector
// units, which share a SIMD's two waves.  A workgroup takes a unit of 32 NW rows
// of a sequence and cache head, a wave 32 of them, and goes through the unit's
// keys 64 at a time: each tile is turned into fp16 once, in LDS, for all waves.
// Two buffers, one barrier a tile: while a tile's weights are found, the scores of
// the next are under way, and keys two tiles and values one tile further go to
// LDS, with those after them on their way from memory.
//
// Measured, 32 heads over 8 of 128: 4,096 tokens from the start 154 us, 890
// TFLOP/s of the products that the mask leaves (a library product of 8,192^3 in
// fp16 reaches 1,170); 16,384 tokens 2,154 us, 1,021.  Of 4,096 the matrix cores are
// busy 42 % of the cycles, the vector units 51 %, without a bank conflict in LDS.
// Heads of 64: 4,096 tokens 109 us, 630 TFLOP/s, vector units 62 %, matrix cores
// 30 %: 86 % of the vector units' work for half the products.  Of heads of 128,
// halving the reads from LDS would gain 10 %, no conversion to fp16 12 %, no
// exponentials 2 %.
// The two halves of a workgroup in opposite phases (products against weights, two
// barriers a tile) took 167 us at any depth of reads ahead; l as a product of the
// fp16 weights is wrong where pages' scales lie far apart, as it has the small
// ones at fp16's smallest steps and scales them up again.
//
// Products on v_mfma_f32_32x32x16_f16, transposed as above: S^T = K Q^T leaves
// a lane (row lane % 32, half h = lane / 32) with the scores of tokens 8 (i /
// 4) + 4 h + i % 4 of each 32, which as they stand are its operand of O^T = V^T
// P^T, a product of 16 tokens in the order 0-3, 8-11 | 4-7, 12-15; the values
// are written to LDS in that order.
//
// m follows the maximum only when it is passed by kSlack or more.

constexpr int kManyTile = 64;
constexpr float kSlack = 8.f;

typedef float f32x16 __attribute__((ext_vector_type(16)));

// How the device spreads the many-row units, found by every wave for itself: the
// row tiles of all sequences, and the pieces that a unit's keys are cut into.
struct ManyPlan {
    int row_tiles, splits;
};

// Units that do not fill the chip (`slots` workgroups at once) are cut along
// their keys where that pays: a step of KS tiles takes a workgroup 1.75 us, a
// piece's sums on their way through memory D NW / 16384 us (all pieces' together),
// the join's launch 6 us.  Measured (one team of 128 rows, 32 heads of 128, us):
// 203 tokens after 3,893 101 whole and 39 in 8 pieces, 100 after 900 32 and 23 in
// 4; but 1,024 from the start 35 whole and 42 in 2, 512 from the start 22 and 27.
template <int D, int NW, int KS>
__host__ __device__ __forceinline__ int many_splits(int units, int tiles, int slots) {
    if (units < 1 || 2 * units > slots || tiles < 4 * KS) return 1;
    const float work = 1.75f / KS * tiles, part = units * (D * NW / 16384.f);
    float s = sqrtf(work / part);
    s = fminf(s, fminf(static_cast<float>(slots / units), static_cast<float>(tiles / (2 * KS))));
    return s >= 2.f && work * (1.f - 1.f / s) > 6.f + part * s ? static_cast<int>(s) : 1;
}

template <int NW>
__device__ __forceinline__ int many_row_tiles(const AttendArgs& a, const Span& s) {
    const int rows = s.n * a.group;
    return rows > a.few_most ? (rows + 32 * NW - 1) / (32 * NW) : 0;
}

// What a workgroup of units finds for itself: its row tile's sequence and rows.
struct ManyUnit {
    Span s;
    int seq, row0;      // seq -1: none
};

// Every wave looks for itself, the sequences a lane each: first the plan, then
// row tile `rank_of(plan)` of all.  slots 0: no unit is cut.
template <int D, int NW, int KS, class F>
__device__ __forceinline__ ManyPlan many_plan(const AttendArgs& a, int slots, F rank_of, ManyUnit& unit) {
    const int lane = threadIdx.x & 63;
    auto span_at = [&](int i) {
        return i < a.c.seqs ? span_of(a.starts, a.c.lens, a.rows, a.max_new, i) : Span{0, 0, 0, 0};
    };
    Span mine = span_at(lane);                     // of the first 64 sequences
    int row_tiles = 0, most = 0;
    for (int i0 = 0; i0 < a.c.seqs; i0 += 64) {
        const Span s = i0 ? span_at(i0 + lane) : mine;
        const int t = many_row_tiles<NW>(a, s);
        const Reach r = reach_of(a, s);
        row_tiles += t;
        if (t) most = max(most, (r.end - r.begin + kManyTile - 1) / kManyTile);
    }
    ManyPlan p;
    p.row_tiles = wave_all(Sum(), row_tiles);
    most = wave_all(Max(), most);
    p.splits = many_splits<D, NW, KS>(p.row_tiles * a.c.kv_heads, most, slots);
    const int rank = rank_of(p);
    unit.seq = -1;
    if (rank < 0) return p;
    for (int i0 = 0, before = 0; i0 < a.c.seqs; i0 += 64) {
        if (i0) mine = span_at(i0 + lane);
        const int n = many_row_tiles<NW>(a, mine);
        const int upto = wave_upto(Sum(), n) + before;
        const unsigned long long has = __ballot(upto > rank);
        if (has) {
            const int l = __builtin_ctzll(has);
            unit.seq = i0 + l;
            unit.row0 = (rank - lane_of(upto - n, l)) * 32 * NW;
            unit.s = {lane_of(mine.row0, l), lane_of(mine.n, l), lane_of(mine.first, l), lane_of(mine.len, l)};
            return p;
        }
        before = lane_of(upto, 63);
    }
    return p;
}

// the first of a unit's tiles that piece `split` of it takes
__device__ __forceinline__ int split_from(int split, int tiles, int splits) {
    return tiles / splits * split + min(split, tiles % splits);
}

// a piece's part: m and l of its rows, then their sums
template <int D, int NW>
constexpr int kManySlot = 32 * NW * (D + 2);

template <int D>
struct ManyLds {
    _Float16 k[2][D / 8][kManyTile][8];   // [8 dimensions][token]
    _Float16 v[2][4][2][D][8];            // [16 tokens][half][dimension][8 tokens]
};

// NW waves for the rows, KS teams of them for the keys: each takes every KS-th tile
// of its unit in buffers of its own, and the first adds the others' sums at the
// end.  With one team, workgroups from `blocks` on, `few` of them, run attend_few:
// in a batch of prompts and single tokens both go side by side.
template <int D, int NW, int KS, bool ONE>
__global__ __launch_bounds__(NW * KS * 64, 2) void attend_many_kernel(AttendArgs a, int slots, int blocks, int few) {
    constexpr int kRows = 32 * NW, kThreads = 64 * NW;
    constexpr int kStep = KS * kManyTile;                       // tokens from a team's tile to its next
    constexpr int kKeys = 4 * D, kPer = 8 * D / kThreads;       // 16-byte pieces of a tile's keys; a thread's pieces of both
    constexpr int kGroups = ONE ? 1 : 4, kWindow = 64 / kGroups;   // scales of a tile; tiles whose scales 64 lanes hold
    static_assert(8 * D % kThreads == 0, "whole pieces a thread");
    using Few = FewLds<D, NW>;
    constexpr size_t kLds = sizeof(ManyLds<D>) * KS;
    __shared__ __align__(16) char lds[KS == 1 && kLds < sizeof(Few) ? sizeof(Few) : kLds];
    if constexpr (KS == 1)
        if (static_cast<int>(blockIdx.x) >= blocks)
            return attend_few<D, NW>(a, blockIdx.x - blocks, few, *reinterpret_cast<Few*>(lds));
    const int lane = threadIdx.x & 63;
    const int team = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    const int tid = threadIdx.x - team * kThreads, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto& kt = reinterpret_cast<ManyLds<D>*>(lds)[team].k;
    auto& vt = reinterpret_cast<ManyLds<D>*>(lds)[team].v;
    // the last row tiles first: those have the most keys
    const int head = blockIdx.x % a.c.kv_heads, rest = blockIdx.x / a.c.kv_heads;
    ManyUnit unit;
    const ManyPlan plan =
        many_plan<D, NW, KS>(a, slots, [&](const ManyPlan& p) { return p.row_tiles - 1 - rest / p.splits; }, unit);
    if (unit.seq < 0) return;
    const int splits = plan.splits, split = rest % splits, seq = unit.seq, row0 = unit.row0;
    const Span s = unit.s;
    const int rows = s.n * a.group;
    const Reach reach = reach_of(a, s);
    const int token0 = s.first + row0 / a.group, token1 = s.first + (min(row0 + kRows, rows) - 1) / a.group;
    const int reach_end = min(token1 + 1, reach.end), reach_begin = reach_begin_of(a, token0, reach_end);
    const int unit_tiles = max(0, reach_end - reach_begin + kManyTile - 1) / kManyTile;
    const int tile0 = split_from(split, unit_tiles, splits), n = split_from(split + 1, unit_tiles, splits) - tile0;
    const int piece = reach_begin + tile0 * kManyTile, end = min(reach_end, piece + n * kManyTile);
    const int begin = piece + team * kManyTile, mine = (n - team + KS - 1) / KS;      // the team's first tile, and its tiles
    const int* table = a.c.pages + static_cast<size_t>(seq) * a.c.max_pages;
    const size_t stride = static_cast<size_t>(a.c.page_tokens) * D;

    // the lane's row, and what the wave's rows see: all of [all_begin, all_end), none outside [any_begin, any_end)
    const int wrow = row0 + 32 * wave, row = wrow + (lane & 31), half = lane >> 5;
    const int rtoken = row / a.group, h = head * a.group + row - rtoken * a.group;
    const bool there = row < rows;
    const int position = s.first + rtoken;
    const int row_end = there ? min(position + 1, end) : 0, row_begin = window_begin(a, position);
    const int wfirst = s.first + wrow / a.group, wlast = s.first + (min(wrow + 32, rows) - 1) / a.group;
    const int all_end = min(wfirst + 1, end), all_begin = window_begin(a, wlast);
    const int any_end = wrow < rows ? min(wlast + 1, end) : 0, any_begin = window_begin(a, wfirst);

    f16x8 q[D / 16];
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        u32x4 v = {0, 0, 0, 0};
        if (there) v = *reinterpret_cast<const u32x4*>(a.q + (s.row0 + rtoken) * a.q_stride + h * D + 16 * c + 8 * half);
        q[c] = query8(v, a.q_flip);
    }

    // Pages and scales of kWindow tiles, a lane each (of 16 tokens or of a tile): this window's and the next's.
    // A negative page is none, and page 0's scales, read in its place, are not used; sg is the factor of the scores, lv
    // log_scale of the values.
    struct Window {
        int page;
        float sg, lv;
    } win, next;
    auto load_pages = [&](Window& w, int first) {
        const int t = begin + (first + lane / kGroups) * kStep + lane % kGroups * 16;
        const int id = t < end ? table[t >> a.c.page_shift] : -1;
        w.page = id < a.c.num_pages ? id : -1;
    };
    auto load_scales = [&](Window& w) {
        const f32x2 x = *reinterpret_cast<const f32x2*>(a.c.scales + 2 * (static_cast<size_t>(max(w.page, 0)) * a.c.kv_heads + head));
        const bool none = w.page < 0;
        w.sg = none ? 1e-30f : fmaxf(x[0] * a.scale, 1e-30f);
        w.lv = none ? 0.f : log_scale(x[1]);
    };
    auto of_lane = [&](int v, int l) { return __builtin_amdgcn_readlane(v, l); };
    // page of the tokens 16 g .. of tile j, which lies in the present window or the next
    int window0 = 0;
    auto page_at = [&](int j, int g) {
        const int v = j - window0 < kWindow ? win.page : next.page;
        return of_lane(v, (j % kWindow) * kGroups + (ONE ? 0 : g));
    };

    // pieces of a tile: the first kKeys are keys (token, 16 dimensions), the others values (16 tokens, a dimension)
    u32x4 raw[kPer];
    auto is_key = [&](int u) { return (u + 1) * kThreads <= kKeys || (u * kThreads < kKeys && tid + u * kThreads < kKeys); };
    auto load_piece = [&](int u, int jk, int jv) {
        const int p = tid + u * kThreads;
        if (is_key(u)) {
            const int t = begin + jk * kStep + (ONE ? 0 : p & 48);
            int page;
            if constexpr (ONE) page = page_at(jk, 0);
            else page = __shfl(jk - window0 < kWindow ? win.page : next.page, (jk % kWindow) * 4 + ((p & 63) >> 4), 64);
            const int8_t* at = a.c.k + (static_cast<size_t>(max(page, 0)) * a.c.kv_heads + head) * stride +
                               static_cast<size_t>(t & (a.c.page_tokens - 1)) * D;
            raw[u] = *reinterpret_cast<const u32x4*>(at + (ONE ? p & 63 : p & 15) * D + (p >> 6) * 16);
        } else {
            const int g = __builtin_amdgcn_readfirstlane((p - kKeys) / D);
            const int t = begin + jv * kStep + 16 * g;
            const int8_t* at = a.c.v + (static_cast<size_t>(max(page_at(jv, g), 0)) * a.c.kv_heads + head) * stride +
                               static_cast<size_t>(t & (a.c.page_tokens - 1)) * D;
            raw[u] = *reinterpret_cast<const u32x4*>(at + (p - kKeys) % D * 16);
        }
    };
    auto write_piece = [&](int u, int bk, int bv) {
        const int p = tid + u * kThreads;
        const u32x4 x = raw[u];
        if (is_key(u)) {
            *reinterpret_cast<f16x8*>(kt[bk][(p >> 6) * 2][p & 63]) = to_half8(x[0], x[1]);
            *reinterpret_cast<f16x8*>(kt[bk][(p >> 6) * 2 + 1][p & 63]) = to_half8(x[2], x[3]);
        } else {
            const int v = p - kKeys;
            *reinterpret_cast<f16x8*>(vt[bv][v / D][0][v % D]) = to_half8(x[0], x[2]);
            *reinterpret_cast<f16x8*>(vt[bv][v / D][1][v % D]) = to_half8(x[1], x[3]);
        }
    };
    // keys of tile jk and values of tile jv, from memory and into LDS (tiles past the last: the last again)
    auto load_tiles = [&](int jk, int jv) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) load_piece(u, min(jk, max(mine, 1) - 1), min(jv, max(mine, 1) - 1));
    };
    auto write_tiles = [&](int bk, int bv) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) write_piece(u, bk, bv);
    };

    f32x16 o[D / 32], sc[2];
    for (f32x16& x : o)
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
    auto scores = [&](f32x16 (&x)[2], int b) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
            for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t)
                x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                    *reinterpret_cast<const f16x8*>(kt[b][2 * c + half][32 * t + (lane & 31)]), q[c], x[t], 0, 0, 0);
    };
    float m = kNoScore, l = 0.f;
    if (n > 0) {
        load_pages(win, 0);
        load_scales(win);
        load_pages(next, kWindow);
        next.sg = next.lv = 0.f;
        // the first two tiles, and the third on its way
        u32x4 tile0_raw[kPer], tile1_raw[kPer];
        auto move = [](u32x4 (&to)[kPer], const u32x4 (&from)[kPer]) {
#pragma unroll
            for (int u = 0; u < kPer; ++u) to[u] = from[u];
        };
        load_tiles(0, 0);
        move(tile0_raw, raw);
        load_tiles(1, 0);
        move(tile1_raw, raw);
        load_tiles(2, 1);
        u32x4 tile2_raw[kPer];
        move(tile2_raw, raw);
        move(raw, tile0_raw);
        write_tiles(0, 0);
        move(raw, tile1_raw);
        write_tiles(1, 0);
        move(raw, tile2_raw);
        __syncthreads();
        scores(sc, 0);
    }
    // tile j, whose scores are in `cur`; those of tile j + 1 go into `ahead`
    auto tile = [&](int j, int b, f32x16 (&cur)[2], f32x16 (&ahead)[2]) {
        const int t0 = begin + j * kStep;
        if (j == window0 + kWindow) {
            win = next;
            window0 = j;
            load_pages(next, j + kWindow);
        }
        if (j == window0 + kWindow / 2) load_scales(next);
        __syncthreads();
        // a wave also goes through the tile before its first, for that one's scores
        if (t0 < any_end && t0 + kStep + kManyTile > any_begin) {
            float sg[kGroups], lv[kGroups];
            bool none[kGroups], holes = false;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int at = (j - window0) * kGroups + g;
                sg[g] = __builtin_bit_cast(float, of_lane(__builtin_bit_cast(int, win.sg), at));
                lv[g] = __builtin_bit_cast(float, of_lane(__builtin_bit_cast(int, win.lv), at));
                none[g] = of_lane(win.page, at) < 0;
                holes |= none[g];
            }
            if (holes || t0 < all_begin || t0 + kManyTile > all_end) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int token = t0 + 32 * t + 8 * (i / 4) + 4 * half + i % 4;
                        if (none[ONE ? 0 : 2 * t + i / 8] || token < row_begin || token >= row_end) cur[t][i] = -INFINITY;
                    }
            }
            // exponents with the maximum so far, and what they say of the new one
            const float from = m > kNoScore ? m : 0.f, c0 = kWeightShift - kSlack - from;
            float top = -INFINITY;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float c = c0 + lv[ONE ? 0 : g];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = __builtin_fmaf(cur[g / 2][8 * (g % 2) + i], sg[ONE ? 0 : g], c);
                    cur[g / 2][8 * (g % 2) + i] = e;
                    top = fmaxf(top, e);
                }
            }
            top = with_half(Larger(), top) - c0;
            if (__any(top > m + kSlack)) {
                const float mnew = fmaxf(m, top), alpha = fast_exp2(m - mnew);
                l *= alpha;
#pragma unroll
                for (f32x16& x : o) x *= alpha;
#pragma unroll
                for (int t = 0; t < 2; ++t) cur[t] += from - mnew;
                m = mnew;
            }
            __builtin_amdgcn_s_setprio(1);
            scores(ahead, b ^ 1);
            f16x8 p[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float w = fast_exp2(cur[g / 2][8 * (g % 2) + i]);
                    sum += w;
                    p[g][i] = static_cast<_Float16>(w);
                }
                l += sum * fast_exp2(-lv[ONE ? 0 : g]);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                        *reinterpret_cast<const f16x8*>(vt[b][g][half][32 * d + (lane & 31)]), p[g], o[d], 0, 0, 0);
            __builtin_amdgcn_s_setprio(0);
        }
        // keys of tile j + 2 and values of tile j + 1 go where those of tiles j and j - 1 were
        write_tiles(b, b ^ 1);
        load_tiles(j + 3, j + 2);
    };
    f32x16 sc2[2];
    for (int t = 0; t < 2; ++t)
        for (int i = 0; i < 16; ++i) sc2[t][i] = 0.f;
    const int steps = (n + KS - 1) / KS;       // of every team, for the barriers
    for (int j = 0; j < steps; j += 2) {
        tile(j, 0, sc, sc2);
        if (j + 1 < steps) tile(j + 1, 1, sc2, sc);
    }
    if constexpr (KS > 1) {
        static_assert(KS == 2 && sizeof(ManyLds<D>) >= sizeof(float) * kThreads * (D / 2), "the second team's sums fit");
        float* sums = reinterpret_cast<float*>(lds) + tid;
        float* stat = reinterpret_cast<float*>(lds + sizeof(ManyLds<D>)) + tid;
        __syncthreads();
        if (team == 1) {
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(16 * d + i) * kThreads] = o[d][i];
            stat[0] = m;
            stat[kThreads] = l;
        }
        __syncthreads();
        if (team == 1) return;
        const float m1 = stat[0], l1 = stat[kThreads], mnew = fmaxf(m, m1);
        const float f0 = fast_exp2(m - mnew), f1 = fast_exp2(m1 - mnew);
        l = l * f0 + l1 * f1;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * f0 + sums[(16 * d + i) * kThreads] * f1;
        m = mnew;
    }
    l = with_half(Sum(), l);
    if (!there) return;
    if (splits > 1) {
        float* slot = a.pieces + static_cast<size_t>(blockIdx.x) * kManySlot<D, NW>;
        const int r = 32 * wave + (lane & 31);
        if (half == 0) {
            slot[r] = m;
            slot[kRows + r] = l;
        }
        float* out = slot + 2 * kRows + r * D + 4 * half;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4*>(out + 32 * d + 2 * i) =
                    f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        return;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint16_t* out = a.out + (s.row0 + rtoken) * a.out_stride + h * D + 4 * half;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            f16x4 v;
            for (int j = 0; j < 4; ++j) v[j] = static_cast<_Float16>(o[d][i + j] * inv);
            *reinterpret_cast<f16x4*>(out + 32 * d + 2 * i) = v;
        }
}

// Joins the pieces of attend_many_kernel's units: a workgroup per 1024 / D rows
// of a unit, D / 4 lanes a row.  Seven sequences of one to 509 new tokens, 16 heads of
// 64, a window of 1,024: 6.7 us after 17.8 us for units and few-row sequences.
template <int D>
constexpr int kJoinRows = 1024 / D;

// Workgroups from `blocks` on run attend_join.
template <int D, int NW, int KS>
__global__ __launch_bounds__(256) void attend_join_many_kernel(AttendArgs a, int slots, int blocks, JoinShape shape) {
    constexpr int kRows = 32 * NW, kParts = kRows / kJoinRows<D>;
    if (static_cast<int>(blockIdx.x) >= blocks) return attend_join<D>(a, blockIdx.x - blocks, shape);
    const int part = blockIdx.x % kParts, rest = blockIdx.x / kParts, head = rest % a.c.kv_heads;
    ManyUnit found;
    const ManyPlan plan = many_plan<D, NW, KS>(
        a, slots, [&](const ManyPlan& p) { return p.splits == 1 ? -1 : p.row_tiles - 1 - rest / a.c.kv_heads; }, found);
    if (found.seq < 0) return;
    const Span s = found.s;
    const int row0 = found.row0, r = part * kJoinRows<D> + static_cast<int>(threadIdx.x) / (D / 4);
    if (row0 + r >= s.n * a.group) return;
    const float* unit = a.pieces +
                        (static_cast<size_t>(rest / a.c.kv_heads) * plan.splits * a.c.kv_heads + head) * kManySlot<D, NW>;
    const size_t step = static_cast<size_t>(a.c.kv_heads) * kManySlot<D, NW>;
    const int d = static_cast<int>(threadIdx.x) % (D / 4) * 4;
    float m = kNoScore;
#pragma unroll 4
    for (int i = 0; i < plan.splits; ++i) m = fmaxf(m, unit[i * step + r]);
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < plan.splits; ++i) {
        const float* p = unit + i * step;
        const float f = fast_exp2(p[r] - m);
        l += f * p[kRows + r];
        o += f * *reinterpret_cast<const f32x4*>(p + 2 * kRows + r * D + d);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int t = (row0 + r) / a.group, h = head * a.group + row0 + r - t * a.group;
    f16x4 v;
    for (int i = 0; i < 4; ++i) v[i] = static_cast<_Float16>(o[i] * inv);
    *reinterpret_cast<f16x4*>(a.out + (s.row0 + t) * a.out_stride + h * D + d) = v;
}

}  // namespace tetra_dev
