// Eviction from the paged cache by accumulated attention weight (kv_evict).
// Included by batch.hip.
//
// Of every sequence and cache head the tokens of most weight and the last ones
// go in their order into other pages.  Two launches: which tokens (a workgroup
// a sequence and head), and their move (a workgroup a new page, head and kind).
#pragma once

#include "kv_cache.h"

namespace tetra_dev {

struct EvictArgs {
    KvCache from, to;
    const float* mass;
    float* out;
    int* tokens;          // [seqs][kv_heads][capacity]: the token that goes to each place
    int capacity;         // places of a sequence in `to`
    int mass_tokens, out_tokens, recent;
};

// n: a sequence's tokens, kept: how many stay, last: how many of those are its last ones
struct EvictShape {
    int n, kept, last;
};

__device__ __forceinline__ EvictShape evict_shape(const EvictArgs& a, int seq) {
    EvictShape s;
    s.n = static_cast<int>(min(static_cast<long long>(max(a.from.lens[seq], 0)),
                               static_cast<long long>(a.from.max_pages) << a.from.page_shift));
    s.kept = min(min(max(a.to.lens[seq], 0), s.n), a.capacity);
    s.last = min(a.recent, s.kept);
    return s;
}

// rises with the weight; NaN counts as -inf, and the zeros are equal
__device__ __forceinline__ uint32_t evict_key(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x == 0.f ? 0.f : x);
    return x != x ? 0x007FFFFFu : b >> 31 ? ~b : b | 0x80000000u;
}

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64, kEvictBins = 2048;

// The smallest key that stays is found eleven bits at a time from the histogram of the
// keys that agree so far; then every wave writes its part of the tokens.  A wave's part
// is in line, a token a lane, the first HELD of a lane in registers from the start.
template <int HELD>
__global__ __launch_bounds__(kEvictThreads) void evict_choose_kernel(EvictArgs a) {
    __shared__ unsigned count[kEvictBins], above[kEvictWaves], equal[kEvictWaves];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int seq = blockIdx.x / a.from.kv_heads, head = blockIdx.x % a.from.kv_heads;
    const EvictShape s = evict_shape(a, seq);
    if (s.kept == 0) return;
    const int old = s.n - s.last, pick = s.kept - s.last;       // `pick` of the first `old` tokens
    const size_t unit = static_cast<size_t>(seq) * a.from.kv_heads + head;
    const float* mass = a.mass + unit * a.mass_tokens;
    int* tokens = a.tokens + unit * a.capacity;
    float* out = a.out ? a.out + unit * a.out_tokens : nullptr;
    auto mass_of = [&](int t) { return t < a.mass_tokens ? mass[t] : 0.f; };
    auto put = [&](int place, int t, float x) {
        tokens[place] = t;
        if (out && place < a.out_tokens) out[place] = x;
    };
    const int part = ((old + kEvictWaves - 1) / kEvictWaves + 63) & ~63, t0 = min(old, wave * part), t1 = min(old, t0 + part);
    float held[HELD];
#pragma unroll
    for (int j = 0; j < HELD; ++j) held[j] = t0 + 64 * j + lane < t1 ? mass_of(t0 + 64 * j + lane) : 0.f;
    for (int i = tid; i < s.last; i += kEvictThreads) put(pick + i, old + i, mass_of(old + i));
    if (pick == 0) return;
    // f(token, weight) of the lane's tokens, and whether it is one
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < HELD; ++j)
            if (t0 + 64 * j < t1) f(t0 + 64 * j + lane, held[j], t0 + 64 * j + lane < t1);
        for (int i = t0 + 64 * HELD; i < t1; i += 64) f(i + lane, i + lane < t1 ? mass_of(i + lane) : 0.f, i + lane < t1);
    };
    uint32_t cut = 0;
    int left = pick;                                            // of the keys that begin like `cut`
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < kEvictBins; i += kEvictThreads) count[i] = 0;
        __syncthreads();
        each([&](int, float x, bool is) {
            const uint32_t k = evict_key(x);
            if (is && (pass == 0 || (k >> (shift + bits)) == (cut >> (shift + bits))))
                atomicAdd(&count[k >> shift & ((1u << bits) - 1)], 1u);
        });
        __syncthreads();
        // the bin in which the count from the last bin down reaches `left`: two bins a thread
        const int b = kEvictBins - 2 - 2 * tid;
        const unsigned hi = count[b + 1], lo = count[b];
        const unsigned upto = wave_upto(Sum(), hi + lo);
        if (lane == 63) above[wave] = upto;
        __syncthreads();
        unsigned before = upto - hi - lo;
        for (int w = 0; w < wave; ++w) before += above[w];
        const unsigned need = left;
        if (before < need && before + hi >= need) {
            found[0] = b + 1;
            found[1] = need - before;
        } else if (before + hi < need && before + hi + lo >= need) {
            found[0] = b;
            found[1] = need - before - hi;
        }
        __syncthreads();
        cut |= static_cast<uint32_t>(found[0]) << shift;
        left = found[1];
        __syncthreads();
    }
    unsigned n_above = 0, n_equal = 0;
    each([&](int, float x, bool is) {
        const uint32_t k = evict_key(x);
        n_above += is && k > cut;
        n_equal += is && k == cut;
    });
    n_above = wave_all(Sum(), n_above);
    n_equal = wave_all(Sum(), n_equal);
    if (lane == 0) {
        above[wave] = n_above;
        equal[wave] = n_equal;
    }
    __syncthreads();
    int place = 0, equals = 0;                                  // before this wave: above the cut, and at it
    for (int w = 0; w < wave; ++w) {
        place += above[w];
        equals += equal[w];
    }
    place += min(equals, left);
    const unsigned long long below = (1ull << lane) - 1;
    each([&](int t, float x, bool is) {
        const uint32_t k = evict_key(x);
        const unsigned long long same = __ballot(is && k == cut);
        const bool stays = is && (k > cut || (k == cut && equals + static_cast<int>(__popcll(same & below)) < left));
        const unsigned long long staying = __ballot(stays);
        if (stays) put(place + static_cast<int>(__popcll(staying & below)), t, x);
        place += __popcll(staying);
        equals += __popcll(same);
    });
}

// four whole numbers times ratio, rounded
__device__ __forceinline__ uint32_t moved4(uint32_t q, float ratio) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= static_cast<uint32_t>(requantized(static_cast<int8_t>(q >> (8 * i)), ratio) & 0xFF) << (8 * i);
    return w;
}

// A new page of a head, its keys or its values.  Keys are rows of D bytes.  Of values a
// thread takes a dimension of 16 places: 16 bytes, which come from as many groups of 16
// old tokens as the kept ones lie in (in order, so neighbours mostly share one).
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    __shared__ int from[128], where[128];
    __shared__ float ratio[128], largest[4];
    const int tid = threadIdx.x, kind = blockIdx.x & 1;
    int rest = blockIdx.x >> 1;
    const int head = rest % a.from.kv_heads;
    rest /= a.from.kv_heads;
    const int seq = rest / a.to.max_pages, number = rest - seq * a.to.max_pages;
    const EvictShape s = evict_shape(a, seq);
    const int B = a.to.page_tokens, first = number * B, n = min(B, s.kept - first);
    if (n <= 0) return;
    const int page = a.to.pages[static_cast<size_t>(seq) * a.to.max_pages + number];
    if (page < 0 || page >= a.to.num_pages) return;
    const int* tokens = a.tokens + (static_cast<size_t>(seq) * a.from.kv_heads + head) * a.capacity + first;
    float mine = 0.f;
    int token = -1, source = 0;
    if (tid < n) {
        const int t = tokens[tid], p = a.from.pages[static_cast<size_t>(seq) * a.from.max_pages + (t >> a.from.page_shift)];
        if (p >= 0 && p < a.from.num_pages) {
            token = t;
            source = p;
            mine = a.from.scales[2 * (static_cast<size_t>(p) * a.from.kv_heads + head) + kind];
        }
    }
    const float top = wave_all(Max(), mine);
    if ((tid & 63) == 0) largest[tid >> 6] = top;
    __syncthreads();
    const float grown = fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3]));
    if (tid < B) {
        from[tid] = token;
        where[tid] = source;
        ratio[tid] = grown > 0.f ? mine / grown : 0.f;
    }
    __syncthreads();
    const size_t stride = static_cast<size_t>(B) * D, to = (static_cast<size_t>(page) * a.to.kv_heads + head) * stride;
    if (tid == 0) a.to.scales[2 * (to / stride) + kind] = grown;
    auto page_of = [&](int i) { return (static_cast<size_t>(where[i]) * a.from.kv_heads + head) * stride; };
    if (kind == 0) {
        constexpr int kPieces = D / 16;
        for (int e = tid; e < n * kPieces; e += 256) {
            const int i = e / kPieces, c = e % kPieces, t = from[i];
            u32x4 q = {0, 0, 0, 0};
            if (t >= 0) q = *reinterpret_cast<const u32x4*>(a.from.k + page_of(i) + (t & (B - 1)) * D + 16 * c);
            const float f = ratio[i];
            if (f != 1.f)
#pragma unroll
                for (int k = 0; k < 4; ++k) q[k] = moved4(q[k], f);
            *reinterpret_cast<u32x4*>(a.to.k + to + i * D + 16 * c) = q;
        }
        return;
    }
    constexpr int kGroups = 256 / D;                            // groups of 16 places at once: of a wave all the same
    const int d = tid % D;
    for (int g = __builtin_amdgcn_readfirstlane(tid / D); 16 * g < n; g += kGroups) {
        u32x4 q = {0, 0, 0, 0}, held = {0, 0, 0, 0};
        int group = -1;                                         // of old tokens, in `held`
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int i = 16 * g + j;
            const int t = i < n ? __builtin_amdgcn_readfirstlane(from[i]) : -1;
            if (t < 0) continue;
            if (t >> 4 != group) {
                group = t >> 4;
                held = *reinterpret_cast<const u32x4*>(a.from.v + page_of(i) + (t & (B - 1) & ~15) * D + d * 16);
            }
            const int word = t >> 2 & 3;
            const uint32_t w = word == 0 ? held[0] : word == 1 ? held[1] : word == 2 ? held[2] : held[3];
            int x = static_cast<int8_t>(w >> (8 * (t & 3)));
            const float f = ratio[i];
            if (f != 1.f) x = requantized(x, f);
            q[j / 4] |= static_cast<uint32_t>(x & 0xFF) << (8 * (j % 4));
        }
        *reinterpret_cast<u32x4*>(a.to.v + to + 16 * g * D + d * 16) = q;
    }
}

}  // namespace tetra_dev
