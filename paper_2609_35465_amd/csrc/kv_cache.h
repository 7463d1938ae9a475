// The paged 8-bit cache of keys and values: appending to it and reading it
// back.  Included by serve.hip.
//
// A page holds page_tokens (16, 32, 64 or 128) consecutive tokens of one
// sequence for every head, as whole numbers of -127..127, with one fp32 scale
// for the keys and one for the values of a page and head:
//   k      int8 [num_pages][kv_heads][page_tokens][D]
//   v      int8 [num_pages][kv_heads][page_tokens / 16][D][16]
//   scales fp32 [num_pages][kv_heads][2]            (key, value)
// Values lie transposed in groups of 16 tokens: the attention's second
// product sums over tokens, and a lane's operand of it, 16 tokens of one
// dimension, is then one 16-byte load (attend.h).  8 bits with a scale per
// page: a page of Gaussian values reaches about 4.2 deviations, so a unit is
// 0.033 of a deviation and the rounding error 0.0095 of it; fp8 e4m3, with 3
// bits after the leading one, would leave 0.02.
//
// append: page_tokens' tokens of one head share a scale, so a workgroup takes
// one page and head (keys and values apart), a wave each 16 tokens of it.
// With old tokens in the page the scale can only grow: s' = max(s, amax/127),
// and if it grows they are rounded again, rint(q s / s').  A batch of single
// tokens is a chain of dependent loads (span, page, its old tokens and scale), so
// everything that does not depend on the page is loaded before it: 64 sequences
// of 8 heads by 128, 40 q heads: 6.6 us, one sequence of 32 q heads 5.5 us.  Prompts are
// bound by HBM: 4,096 tokens of 8 heads and 32 q heads by 128 from fp32, 145 MB,
// 32.5 us, 4,450 GB/s (a large copy: 5,030).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lanes.h"

namespace tetra_dev {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kGroupTokens = 16;          // tokens of a value group, and of a wave of the append
constexpr float kSmallestScale = 1e-30f;  // a page whose largest value is below 127 times this holds zeros

// tetra_kv_cache as the kernels use it
struct KvCache {
    int8_t* k;
    int8_t* v;
    float* scales;
    const int* pages;
    const int* lens;
    int num_pages, page_tokens, page_shift, kv_heads, seqs, max_pages;
};

struct AppendArgs {
    KvCache c;
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    const float *q_norm, *k_norm;
    const float* rope;
    const int* starts;
    const int* shifts;   // or NULL
    uint16_t* q_out;
    float eps;
    int rope_rows, rows, max_new, q_heads;
    int items;       // page items of all sequences
    int q_chunk;     // heads of q per wave
};

// The rows of one sequence in a call: clamped, so that no start or length can
// lead out of the arrays.
struct Span {
    int row0, n;     // rows row0 .. row0 + n - 1
    int first, len;  // their tokens first .. len - 1
};

// from the starts of the sequence and of the next, and its length.  The rows past
// max_new are the last ones, so the others' tokens end before the length there.
__device__ __forceinline__ Span span_between(int start, int next, int len, int rows, int max_new) {
    Span s;
    s.row0 = min(max(start, 0), rows);
    const int all = max(min(max(next, 0), rows) - s.row0, 0);
    s.n = min(all, max_new);
    s.first = max(len, 0) - all;   // below zero if the length does not hold the new tokens
    s.len = max(s.first + s.n, 0);
    return s;
}

__device__ __forceinline__ Span span_of(const int* starts, const int* lens, int rows, int max_new, int seq) {
    return span_between(starts[seq], starts[seq + 1], lens[seq], rows, max_new);
}

// The sequence that holds place x, and its span: the first one with base(start of
// the next, its number) above x.  Each lane loads a sequence, all at once; x and
// the result are uniform in the wave.
struct Place {
    int seq, start;    // seq -1: none; starts[seq], clamped
    Span s;
};

template <class F>
__device__ __forceinline__ Place locate(const int* starts, const int* lens, int rows, int max_new, int seqs, int x, F base) {
    const int lane = threadIdx.x & 63;
    Place p;
    p.seq = -1;
    for (int i0 = 0; i0 < seqs; i0 += 64) {
        const int i = i0 + lane;
        int a = 0, b = 0, len = 0;
        if (i < seqs) {
            a = starts[i];
            b = starts[i + 1];
            len = lens[i];
        }
        a = min(max(a, 0), rows);
        b = min(max(b, 0), rows);
        const unsigned long long has = __ballot(i < seqs && base(b, i + 1) > x);
        if (!has) continue;
        const int l = __builtin_ctzll(has);
        p.seq = i0 + l;
        p.start = __builtin_amdgcn_readlane(a, l);
        p.s = span_between(p.start, __builtin_amdgcn_readlane(b, l), __builtin_amdgcn_readlane(len, l), rows, max_new);
        break;
    }
    return p;
}

// Page items of the sequences before `seq`.  New tokens n >= 1 touch at most
// (n + B - 2) / B + 1 pages, and floor((starts + (B - 2) seq) / B) + seq grows
// by at least that from a sequence to the next; where no sequence has more
// than one, an item each.
__host__ __device__ __forceinline__ int item_base(int start, int seq, int page_shift, int max_new) {
    if (max_new == 1) return seq;
    return static_cast<int>((start + ((1ll << page_shift) - 2) * seq) >> page_shift) + seq;
}

template <bool HALF>
__device__ __forceinline__ f32x4 load4(const void* p, long long at) {
    if constexpr (HALF) {
        const f16x4 h = *reinterpret_cast<const f16x4*>(static_cast<const _Float16*>(p) + at);
        return f32x4{static_cast<float>(h[0]), static_cast<float>(h[1]), static_cast<float>(h[2]), static_cast<float>(h[3])};
    } else {
        return *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
    }
}

template <bool HALF>
__device__ __forceinline__ f32x2 load2(const void* p, long long at) {
    if constexpr (HALF) {
        const f16x2 h = *reinterpret_cast<const f16x2*>(static_cast<const _Float16*>(p) + at);
        return f32x2{static_cast<float>(h[0]), static_cast<float>(h[1])};
    } else {
        return *reinterpret_cast<const f32x2*>(static_cast<const float*>(p) + at);
    }
}

// The place in the rotation's table of a sequence's token: moved by its shift, if
// the call has any.
struct Turn {
    int shift;
    __device__ __forceinline__ Turn(const AppendArgs& a, int seq)
        : shift(a.shifts ? min(max(a.shifts[seq], 0), (1 << 30) - 1) : 0) {}
    __device__ __forceinline__ int of(int position) const { return min(position, 1 << 30) + shift; }
};

// A head of D dimensions lies in D / 8 lanes: lane `sub` holds dimensions
// 4 sub .. 4 sub + 3 (x[0..3]) and their partners D / 2 further (x[4..7]).
template <int D, bool HALF>
__device__ __forceinline__ void load_head(float (&x)[8], const void* p, long long at, int sub) {
    const f32x4 a = load4<HALF>(p, at + 4 * sub), b = load4<HALF>(p, at + D / 2 + 4 * sub);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
    }
}

// norm (if weight) and rotation (if a table) of a head of a token at `position`
template <int D>
__device__ __forceinline__ void norm_and_rotate(float (&x)[8], const float* weight, float eps, const float* rope,
                                                int rope_rows, int position, int sub) {
    if (weight) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += x[i] * x[i];
        s = __builtin_amdgcn_rsqf(team_all<D / 8>(Sum(), s) * (1.f / D) + eps);
        const f32x4 a = *reinterpret_cast<const f32x4*>(weight + 4 * sub);
        const f32x4 b = *reinterpret_cast<const f32x4*>(weight + D / 2 + 4 * sub);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] *= s * a[i];
            x[4 + i] *= s * b[i];
        }
    }
    if (rope) {
        const float* r = rope + static_cast<size_t>(min(max(position, 0), rope_rows - 1)) * D;
        const f32x4 c = *reinterpret_cast<const f32x4*>(r + 4 * sub);
        const f32x4 s = *reinterpret_cast<const f32x4*>(r + D / 2 + 4 * sub);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = x[i], b = x[4 + i];
            x[i] = a * c[i] - b * s[i];
            x[4 + i] = b * c[i] + a * s[i];
        }
    }
}

// the largest finite magnitude so far
__device__ __forceinline__ float larger(float m, float x) {
    const float a = fabsf(x);
    return a <= 3.4028234e38f ? fmaxf(m, a) : m;
}

// x in units of 1 / inverse; NaN gives 0, the infinities +-127
__device__ __forceinline__ int quantized(float x, float inverse) {
    const float v = rintf(x * inverse);
    return v == v ? static_cast<int>(fminf(fmaxf(v, -127.f), 127.f)) : 0;
}

__device__ __forceinline__ int requantized(int q, float ratio) { return static_cast<int>(rintf(static_cast<float>(q) * ratio)); }

// Scale of a page and head once `amax` (of the lane's new values) is in;
// `before` is the old tokens' scale, 0 without any.  Every wave of the
// workgroup takes part.
__device__ __forceinline__ float grown_scale(float amax, float before, float* lds, int waves) {
    amax = wave_all(Max(), amax);
    if (waves > 1) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = amax;
        __syncthreads();
        for (int w = 0; w < waves; ++w) amax = fmaxf(amax, lds[w]);
    }
    const float s = amax / 127.f;
    return fmaxf(before, s < kSmallestScale ? 0.f : s);
}

// `entry`: where the table names the page; it is on its way with the values
template <int D, bool HALF>
__device__ void append_keys(const AppendArgs& a, const Span& s, const Turn& turn, int number, const int* entry, int head, float* lds) {
    const int page = *entry;
    constexpr int kLanes = D / 8, kPerPass = 64 / kLanes, kPasses = kGroupTokens / kPerPass;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int sub = lane % kLanes, slot = lane / kLanes;
    const int page0 = number << a.c.page_shift;
    const int from = max(s.first, 0);                       // new tokens: from .. s.len - 1
    const int token0 = page0 + wave * kGroupTokens + slot;  // of the first pass
    float x[kPasses][8];
    float amax = 0.f;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int t = token0 + p * kPerPass;
        if (t >= from && t < s.len)
            load_head<D, HALF>(x[p], a.k, (s.row0 + t - s.first) * a.k_stride + head * D, sub);
        else
            for (float& e : x[p]) e = 0.f;
    }
    if (page < 0 || page >= a.c.num_pages) return;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        norm_and_rotate<D>(x[p], a.k_norm, a.eps, a.rope, a.rope_rows, turn.of(token0 + p * kPerPass), sub);
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = larger(amax, x[p][i]);
    }
    float* held = a.c.scales + (static_cast<size_t>(page) * a.c.kv_heads + head) * 2;
    const float before = from > page0 ? held[0] : 0.f;
    const float scale = grown_scale(amax, before, lds, waves);
    const float inverse = scale > 0.f ? 1.f / scale : 0.f, ratio = before * inverse;
    const bool grew = from > page0 && scale != before;
    int8_t* out = a.c.k + (static_cast<size_t>(page) * a.c.kv_heads + head) * a.c.page_tokens * D;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int t = token0 + p * kPerPass;
        uint32_t* at = reinterpret_cast<uint32_t*>(out + (t - page0) * D + 4 * sub);
        if (t >= from && t < s.len) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t w = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) w |= (quantized(x[p][4 * h + i], inverse) & 0xFF) << (8 * i);
                at[h * D / 8] = w;
            }
        } else if (grew && t < from) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t q = at[h * D / 8];
                uint32_t w = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w |= (requantized(static_cast<int8_t>(q >> (8 * i)), ratio) & 0xFF) << (8 * i);
                at[h * D / 8] = w;
            }
        }
    }
    if (threadIdx.x == 0) held[0] = scale;
}

template <int D, bool HALF>
__device__ void append_values(const AppendArgs& a, const Span& s, int number, const int* entry, int head, float* lds) {
    const int page = *entry;
    constexpr int kPairs = D / 2, kTokens = kGroupTokens * kPairs / 64;   // a lane: two dimensions of kTokens tokens
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int pair = lane % kPairs, part = lane / kPairs;
    const int page0 = number << a.c.page_shift;
    const int from = max(s.first, 0);
    const int token0 = page0 + wave * kGroupTokens + part * kTokens;
    f32x2 x[kTokens];
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
        const int t = token0 + j;
        x[j] = f32x2{0.f, 0.f};
        if (t >= from && t < s.len)
            x[j] = load2<HALF>(a.v, (s.row0 + t - s.first) * a.v_stride + head * D + 2 * pair);
    }
    if (page < 0 || page >= a.c.num_pages) return;
#pragma unroll
    for (int j = 0; j < kTokens; ++j) amax = larger(larger(amax, x[j][0]), x[j][1]);
    float* held = a.c.scales + (static_cast<size_t>(page) * a.c.kv_heads + head) * 2 + 1;
    const float before = from > page0 ? held[0] : 0.f;
    const float scale = grown_scale(amax, before, lds, waves);
    const float inverse = scale > 0.f ? 1.f / scale : 0.f, ratio = before * inverse;
    const bool grew = from > page0 && scale != before;
    if (threadIdx.x == 0) held[0] = scale;
    const bool any_new = token0 + kTokens > from && token0 < s.len, any_old = token0 < from;
    if (!any_new && !(any_old && grew)) return;
    int8_t* out = a.c.v + ((static_cast<size_t>(page) * a.c.kv_heads + head) * a.c.page_tokens + wave * kGroupTokens) * D +
                  2 * pair * kGroupTokens + part * kTokens;
    typedef uint32_t words __attribute__((ext_vector_type(kTokens / 4)));
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        words* at = reinterpret_cast<words*>(out + d * kGroupTokens);
        words w = {};
        if (any_old) w = *at;
#pragma unroll
        for (int j = 0; j < kTokens; ++j) {
            const int t = token0 + j;
            const int old = static_cast<int8_t>(w[j / 4] >> (8 * (j % 4)));
            const int q = t >= from ? quantized(x[j][d], inverse) : grew ? requantized(old, ratio) : old;
            w[j / 4] = (w[j / 4] & ~(0xFFu << (8 * (j % 4)))) | static_cast<uint32_t>(q & 0xFF) << (8 * (j % 4));
        }
        *at = w;
    }
}

// One wave: q_chunk heads of one row, D / 8 lanes a head.
template <int D, bool HALF>
__device__ void append_queries(const AppendArgs& a, int unit) {
    constexpr int kLanes = D / 8, kTeams = 64 / kLanes;
    const int lane = threadIdx.x & 63, sub = lane % kLanes;
    const int chunks = (a.q_heads + a.q_chunk - 1) / a.q_chunk;
    const int row = unit / chunks;
    if (row >= a.rows) return;
    const int head0 = (unit - row * chunks) * a.q_chunk, end = min(head0 + a.q_chunk, a.q_heads);
    const int first = head0 + lane / kLanes;
    float x0[8] = {};
    if (first < end) load_head<D, HALF>(x0, a.q, row * a.q_stride + first * D, sub);
    const Place at = locate(a.starts, a.c.lens, a.rows, a.max_new, a.c.seqs, row, [](int start, int) { return start; });
    if (at.seq < 0 || row < at.s.row0 || row >= at.s.row0 + at.s.n) return;
    const int position = Turn(a, at.seq).of(at.s.first + row - at.s.row0);
    auto finish = [&](float (&x)[8], int h) {
        norm_and_rotate<D>(x, a.q_norm, a.eps, a.rope, a.rope_rows, position, sub);
        f16x4 lo, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = static_cast<_Float16>(x[i]);
            hi[i] = static_cast<_Float16>(x[4 + i]);
        }
        uint16_t* out = a.q_out + (static_cast<size_t>(row) * a.q_heads + h) * D + 4 * sub;
        *reinterpret_cast<f16x4*>(out) = lo;
        *reinterpret_cast<f16x4*>(out + D / 2) = hi;
    };
    if (first < end) finish(x0, first);
    for (int h = first + kTeams; h < end; h += kTeams) {
        float x[8];
        load_head<D, HALF>(x, a.q, row * a.q_stride + h * D, sub);
        finish(x, h);
    }
}

// Workgroups of page_tokens / 16 waves: first the pages (item, head, keys or
// values), then the rows of q.
template <int D, bool HALF>
__global__ __launch_bounds__(512) void append_kernel(AppendArgs a) {
    __shared__ float lds[8];
    const int kv_blocks = a.items * a.c.kv_heads * 2;
    const int b = static_cast<int>(blockIdx.x);
    if (b >= kv_blocks) {
        append_queries<D, HALF>(a, (b - kv_blocks) * static_cast<int>(blockDim.x >> 6) + static_cast<int>(threadIdx.x >> 6));
        return;
    }
    const int item = b / (a.c.kv_heads * 2), rest = b - item * a.c.kv_heads * 2;
    const Place at = locate(a.starts, a.c.lens, a.rows, a.max_new, a.c.seqs, item,
                              [&](int start, int i) { return item_base(start, i, a.c.page_shift, a.max_new); });
    if (at.seq < 0) return;
    const Span s = at.s;
    const int base = item_base(at.start, at.seq, a.c.page_shift, a.max_new);
    const int number = (max(s.first, 0) >> a.c.page_shift) + item - base;
    if (item < base || s.n == 0 || number >= a.c.max_pages || (static_cast<long long>(number) << a.c.page_shift) >= s.len)
        return;
    const int* entry = a.c.pages + static_cast<size_t>(at.seq) * a.c.max_pages + number;
    if (rest & 1) append_values<D, HALF>(a, s, number, entry, rest >> 1, lds);
    else append_keys<D, HALF>(a, s, Turn(a, at.seq), number, entry, rest >> 1, lds);
}

// The last `count` tokens of every sequence as fp16, [seqs][count][kv_heads][D]
// each for keys and values; zeros before a sequence's start.  A workgroup of 2 D
// threads takes 16 tokens of a head, the first D threads its keys, the others its
// values, which LDS turns.  4,096 tokens of 8 heads by 128: 7.7 us, 3,270 GB/s.
template <int D>
__global__ __launch_bounds__(2 * D) void kv_read_kernel(KvCache c, int count, int groups, uint16_t* k_out, uint16_t* v_out) {
    __shared__ __align__(16) _Float16 turned[kGroupTokens][D + 8];
    const int tid = threadIdx.x;
    const int head = blockIdx.x % c.kv_heads, rest = blockIdx.x / c.kv_heads;
    const int seq = rest / groups, group = rest - seq * groups;
    const int len = max(c.lens[seq], 0), first = len - count;
    const int t0 = (first & ~(kGroupTokens - 1)) + group * kGroupTokens;   // a multiple of 16, below zero perhaps
    const int number = t0 >> c.page_shift;
    int page = -1;
    if (t0 >= 0 && t0 < len && number < c.max_pages) page = c.pages[static_cast<size_t>(seq) * c.max_pages + number];
    const bool there = page >= 0 && page < c.num_pages;
    const size_t ph = static_cast<size_t>(there ? page : 0) * c.kv_heads + head;
    const bool values = tid >= D;
    const int i = values ? tid - D : tid;
    u32x4 q = {0, 0, 0, 0};
    float scale = 0.f;
    if (there) {
        const int8_t* at = (values ? c.v : c.k) + (ph * c.page_tokens + (t0 & (c.page_tokens - 1))) * D + 16 * i;
        q = *reinterpret_cast<const u32x4*>(at);
        scale = c.scales[2 * ph + (values ? 1 : 0)];
    }
    // 16 keys' dimensions of a token, or a dimension's 16 tokens
    _Float16 x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = static_cast<_Float16>(static_cast<float>(static_cast<int8_t>(q[e / 4] >> (8 * (e % 4)))) * scale);
    if (values)
#pragma unroll
        for (int e = 0; e < 16; ++e) turned[e][i] = x[e];
    __syncthreads();
    const int token = i / (D / 16), part = i % (D / 16) * 16, t = t0 + token;
    if (t < first || t >= len) return;
    uint16_t* out = (values ? v_out : k_out) + ((static_cast<size_t>(seq) * count + (t - first)) * c.kv_heads + head) * D + part;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        f16x8 y;
        if (values) {
            y = *reinterpret_cast<const f16x8*>(&turned[token][part + 8 * v]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[8 * v + e];
        }
        *reinterpret_cast<f16x8*>(out + 8 * v) = y;
    }
}

}  // namespace tetra_dev
