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

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

// The smallest key that stays is found eight bits at a time from the histogram of
// the keys that agree so far; then every wave writes its part of the tokens.
__global__ __launch_bounds__(kEvictThreads) void evict_choose_kernel(EvictArgs a) {
    __shared__ unsigned count[256], above[kEvictWaves], equal[kEvictWaves];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int seq = blockIdx.x / a.from.kv_heads, head = blockIdx.x % a.from.kv_heads;
    const EvictShape s = evict_shape(a, seq);
    if (s.kept == 0) return;
    const int old = s.n - s.last, pick = s.kept - s.last;       // `pick` of the first `old` tokens
    const size_t unit = static_cast<size_t>(seq) * a.from.kv_heads + head;
    const float* mass = a.mass + unit * a.mass_tokens;
    int* tokens = a.tokens + unit * a.capacity;
    float* out = a.out ? a.out + unit * a.out_tokens : nullptr;
    auto mass_of = [&](int t) { return t < a.mass_tokens ? mass[t] : 0.f; };
    auto put = [&](int place, int t) {
        tokens[place] = t;
        if (out && place < a.out_tokens) out[place] = mass_of(t);
    };
    for (int i = tid; i < s.last; i += kEvictThreads) put(pick + i, old + i);
    if (pick == 0) return;
    uint32_t cut = 0;
    int left = pick;                                            // of the keys that begin like `cut`
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) count[tid] = 0;
        __syncthreads();
        for (int t = tid; t < old; t += kEvictThreads) {
            const uint32_t k = evict_key(mass_of(t));
            if (shift == 24 || (k >> (shift + 8)) == (cut >> (shift + 8))) atomicAdd(&count[k >> shift & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            int b = 255, n = left;
            while (b > 0 && static_cast<int>(count[b]) < n) n -= count[b--];
            found[0] = b;
            found[1] = n;
        }
        __syncthreads();
        cut |= static_cast<uint32_t>(found[0]) << shift;
        left = found[1];
        __syncthreads();
    }
    // a wave's tokens, in order: its part of the row
    const int part = (old + kEvictWaves - 1) / kEvictWaves, t0 = wave * part, t1 = min(old, t0 + part);
    unsigned n_above = 0, n_equal = 0;
    for (int t = t0 + lane; t < t1; t += 64) {
        const uint32_t k = evict_key(mass_of(t));
        n_above += k > cut;
        n_equal += k == cut;
    }
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
    for (int i = t0; i < t1; i += 64) {
        const int t = i + lane;
        const uint32_t k = t < t1 ? evict_key(mass_of(t)) : 0;
        const unsigned long long same = __ballot(t < t1 && k == cut);
        const bool stays = t < t1 && (k > cut || (k == cut && equals + static_cast<int>(__popcll(same & below)) < left));
        const unsigned long long staying = __ballot(stays);
        if (stays) put(place + static_cast<int>(__popcll(staying & below)), t);
        place += __popcll(staying);
        equals += __popcll(same);
    }
}

// A new page of a head, its keys or its values.
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    __shared__ int from[128];
    __shared__ float scale[128], largest[4];
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
    if (tid < B) {
        int token = -1;
        if (tid < n) {
            const int t = tokens[tid], p = a.from.pages[static_cast<size_t>(seq) * a.from.max_pages + (t >> a.from.page_shift)];
            if (p >= 0 && p < a.from.num_pages) {
                token = t;
                mine = a.from.scales[2 * (static_cast<size_t>(p) * a.from.kv_heads + head) + kind];
            }
        }
        from[tid] = token;
        scale[tid] = mine;
    }
    const float top = wave_all(Max(), mine);
    if ((tid & 63) == 0) largest[tid >> 6] = top;
    __syncthreads();
    const float grown = fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3]));
    const size_t ph = static_cast<size_t>(page) * a.to.kv_heads + head;
    if (tid == 0) a.to.scales[2 * ph + kind] = grown;
    auto moved = [&](int q, int i) {
        return grown > 0.f ? requantized(q, scale[i] / grown) & 0xFF : 0;
    };
    auto source = [&](int t) {
        const int p = a.from.pages[static_cast<size_t>(seq) * a.from.max_pages + (t >> a.from.page_shift)];
        return (static_cast<size_t>(p) * a.from.kv_heads + head) * a.from.page_tokens * D;
    };
    const int in_page = a.from.page_tokens - 1;
    for (int e = tid; e < n * D; e += 256) {
        const int i = e / D, d = e % D, t = from[i];
        int8_t q = 0;
        if (t >= 0) q = kind == 0 ? a.from.k[source(t) + (t & in_page) * D + d]
                                  : a.from.v[source(t) + (t & in_page & ~15) * D + d * 16 + (t & 15)];
        int8_t* to = kind == 0 ? a.to.k + ph * B * D + i * D + d : a.to.v + ph * B * D + (i & ~15) * D + d * 16 + (i & 15);
        *to = static_cast<int8_t>(moved(q, i));
    }
}

}  // namespace tetra_dev
