// Eviction from the paged cache by accumulated attention weight (kv_evict).
// Included by batch.hip.
//
// Of every sequence and cache head the tokens of most weight and the last ones
// go in their order into other pages.  Two launches: which tokens (a workgroup
// a sequence and head), and their move (a workgroup a new page, head and kind).
#pragma once

#include "kv_cache.h"

namespace tetra_dev {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64, kEvictBins = 2048;
constexpr int kEvictHeld = 8;         // weights that a thread keeps in registers
constexpr int kEvictParts = 16;       // of a long sequence and head, at most

struct EvictArgs {
    KvCache from, to;
    const float* mass;
    float* out;
    int* tokens;          // [seqs][kv_heads][capacity]: the token that goes to each place
    int capacity;         // places of a sequence in `to`
    int mass_tokens, out_tokens, recent;
    // of long sequences
    unsigned* bins;       // [3 passes][seqs * kv_heads][parts][kEvictBins]: how many keys of a part
    int* state;           // [2][seqs * kv_heads][2 + parts]
    int parts;
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


// The smallest key that stays is found eleven bits at a time from the histogram of the
// keys that agree so far; then every wave writes its part of the tokens.  A wave's part
// is in line, a token a lane, the first kEvictHeld of a lane in registers from the start.
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
    float held[kEvictHeld];
#pragma unroll
    for (int j = 0; j < kEvictHeld; ++j) held[j] = t0 + 64 * j + lane < t1 ? mass_of(t0 + 64 * j + lane) : 0.f;
    for (int i = tid; i < s.last; i += kEvictThreads) put(pick + i, old + i, mass_of(old + i));
    if (pick == 0) return;
    // f(token, weight) of the lane's tokens, and whether it is one
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < kEvictHeld; ++j)
            if (t0 + 64 * j < t1) f(t0 + 64 * j + lane, held[j], t0 + 64 * j + lane < t1);
        for (int i = t0 + 64 * kEvictHeld; i < t1; i += 64) f(i + lane, i + lane < t1 ? mass_of(i + lane) : 0.f, i + lane < t1);
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

// The same for long sequences, in parts of a row: a launch for each eleven bits, which
// leaves the parts' histograms, and one that writes the tokens.  Each adds up the last
// histograms for itself: where the count reaches the cut, and how many before its own
// part stay.

template <int PASS>
__global__ __launch_bounds__(kEvictThreads) void evict_part_kernel(EvictArgs a) {
    __shared__ unsigned count[kEvictBins], above[kEvictWaves], equal[kEvictWaves];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int units = a.from.seqs * a.from.kv_heads, unit = blockIdx.x / a.parts, mine = blockIdx.x - unit * a.parts;
    const int seq = unit / a.from.kv_heads;
    const EvictShape s = evict_shape(a, seq);
    const int old = s.n - s.last, pick = s.kept - s.last;
    if (s.kept == 0) return;
    const float* mass = a.mass + static_cast<size_t>(unit) * a.mass_tokens;
    auto mass_of = [&](int t) { return t < a.mass_tokens ? mass[t] : 0.f; };
    // the part, and of that the wave's
    const int part = (old + a.parts - 1) / a.parts, p0 = min(old, mine * part), p1 = min(old, p0 + part);
    const int share = ((p1 - p0 + kEvictWaves - 1) / kEvictWaves + 63) & ~63;
    const int t0 = min(p1, p0 + wave * share), t1 = min(p1, t0 + share);
    float held[kEvictHeld];
#pragma unroll
    for (int j = 0; j < kEvictHeld; ++j) held[j] = t0 + 64 * j + lane < t1 ? mass_of(t0 + 64 * j + lane) : 0.f;
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < kEvictHeld; ++j)
            if (t0 + 64 * j < t1) f(t0 + 64 * j + lane, held[j], t0 + 64 * j + lane < t1);
        for (int i = t0 + 64 * kEvictHeld; i < t1; i += 64 * kEvictHeld) {
            float x[kEvictHeld];
#pragma unroll
            for (int j = 0; j < kEvictHeld; ++j) x[j] = i + 64 * j + lane < t1 ? mass_of(i + 64 * j + lane) : 0.f;
#pragma unroll
            for (int j = 0; j < kEvictHeld; ++j)
                if (i + 64 * j < t1) f(i + 64 * j + lane, x[j], i + 64 * j + lane < t1);
        }
    };
    auto bins = [&](int pass, int p) { return a.bins + ((static_cast<size_t>(pass) * units + unit) * a.parts + p) * kEvictBins; };
    uint32_t cut = 0;
    int left = pick, before_part = 0, equals_before = 0;
    if constexpr (PASS > 0) {
        constexpr int shift = PASS == 1 ? 21 : PASS == 2 ? 10 : 0;
        // cut and left after the pass before, and what stays before each part; one to read, one to write
        auto state_of = [&](int which) { return a.state + (static_cast<size_t>(which) * units + unit) * (2 + a.parts); };
        int* state = state_of(PASS & 1);
        if constexpr (PASS > 1) {
            const int* last = state_of(PASS & 1 ^ 1);
            cut = last[0];
            left = last[1];
            before_part = last[2 + mine];
        }
        const int b = kEvictBins - 2 - 2 * tid;
        unsigned hi = 0, lo = 0, hi_before = 0, lo_before = 0;
#pragma unroll
        for (int p = 0; p < kEvictParts; ++p)
            if (p < a.parts) {
                const u32x2 c = *reinterpret_cast<const u32x2*>(bins(PASS - 1, p) + b);
                if (p < mine) {
                    hi_before += c[1];
                    lo_before += c[0];
                }
                hi += c[1];
                lo += c[0];
            }
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
        const int bin = found[0];
        left = found[1];
        cut |= static_cast<uint32_t>(bin) << shift;
        const unsigned over = wave_all(Sum(), (b + 1 > bin ? hi_before : 0) + (b > bin ? lo_before : 0));
        const unsigned same = wave_all(Sum(), (b + 1 == bin ? hi_before : 0) + (b == bin ? lo_before : 0));
        if (lane == 0) {
            above[wave] = over;
            equal[wave] = same;
        }
        __syncthreads();
        for (int w = 0; w < kEvictWaves; ++w) {
            before_part += above[w];
            equals_before += equal[w];
        }
        __syncthreads();
        if (PASS < 3 && tid == 0) {
            if (mine == 0) {
                state[0] = cut;
                state[1] = left;
            }
            state[2 + mine] = before_part;
        }
    }
    if constexpr (PASS < 3) {
        constexpr int shift = PASS == 0 ? 21 : PASS == 1 ? 10 : 0, bits = PASS == 2 ? 10 : 11;
        for (int i = tid; i < kEvictBins; i += kEvictThreads) count[i] = 0;
        __syncthreads();
        each([&](int, float x, bool is) {
            const uint32_t k = evict_key(x);
            if (is && (PASS == 0 || (k >> (shift + bits)) == (cut >> (shift + bits))))
                atomicAdd(&count[k >> shift & ((1u << bits) - 1)], 1u);
        });
        __syncthreads();
        for (int i = tid; i < kEvictBins; i += kEvictThreads) bins(PASS, mine)[i] = count[i];
    } else {
        int* tokens = a.tokens + static_cast<size_t>(unit) * a.capacity;
        float* out = a.out ? a.out + static_cast<size_t>(unit) * a.out_tokens : nullptr;
        auto put = [&](int place, int t, float x) {
            tokens[place] = t;
            if (out && place < a.out_tokens) out[place] = x;
        };
        for (int i = mine * kEvictThreads + tid; i < s.last; i += a.parts * kEvictThreads) put(pick + i, old + i, mass_of(old + i));
        if (pick == 0) return;
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
        int place = before_part, equals = equals_before;
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
}

// four whole numbers times ratio, rounded
__device__ __forceinline__ uint32_t moved4(uint32_t q, float ratio) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= static_cast<uint32_t>(requantized(static_cast<int8_t>(q >> (8 * i)), ratio) & 0xFF) << (8 * i);
    return w;
}

// A new page of a head: half of the workgroup its keys, the other its values.  Keys are
// rows of D bytes, moved in pieces of 16.  Of values a thread takes a dimension of 16
// places, whose bytes lie in as many groups of 16 old tokens as the kept ones do: they are
// loaded one by one, all at once.
template <int D>
__global__ __launch_bounds__(512) void evict_move_kernel(EvictArgs a) {
    __shared__ int from[128], where[128];
    __shared__ float ratio[2][128], largest[2][4];
    const int kind = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255;
    int rest = blockIdx.x;
    const int head = rest % a.from.kv_heads;
    rest /= a.from.kv_heads;
    const int seq = rest / a.to.max_pages, number = rest - seq * a.to.max_pages;
    const int B = a.to.page_tokens, first = number * B;
    const int page = a.to.pages[static_cast<size_t>(seq) * a.to.max_pages + number];
    const EvictShape s = evict_shape(a, seq);
    const int n = min(B, s.kept - first);
    if (n <= 0 || page < 0 || page >= a.to.num_pages) return;
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
    if ((tid & 63) == 0) largest[kind][tid >> 6] = top;
    __syncthreads();
    const float grown = fmaxf(fmaxf(largest[kind][0], largest[kind][1]), fmaxf(largest[kind][2], largest[kind][3]));
    if (tid < B) {
        if (kind == 0) {
            from[tid] = token;
            where[tid] = source;
        }
        ratio[kind][tid] = grown > 0.f ? mine / grown : 0.f;
    }
    __syncthreads();
    const size_t stride = static_cast<size_t>(B) * D, to = (static_cast<size_t>(page) * a.to.kv_heads + head) * stride;
    if (tid == 0) a.to.scales[2 * (static_cast<size_t>(page) * a.to.kv_heads + head) + kind] = grown;
    auto page_of = [&](int i) { return (static_cast<size_t>(where[i]) * a.from.kv_heads + head) * stride; };
    if (kind == 0) {
        constexpr int kPieces = D / 16;
#pragma unroll 4
        for (int e = tid; e < n * kPieces; e += 256) {
            const int i = e / kPieces, c = e % kPieces, t = from[i];
            u32x4 q = {0, 0, 0, 0};
            if (t >= 0) q = *reinterpret_cast<const u32x4*>(a.from.k + page_of(i) + (t & (B - 1)) * D + 16 * c);
            const float f = ratio[0][i];
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
        int x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int t = 16 * g + j < n ? __builtin_amdgcn_readfirstlane(from[16 * g + j]) : -1;
            x[j] = 0;
            if (t >= 0) x[j] = a.from.v[page_of(16 * g + j) + (t & (B - 1) & ~15) * D + d * 16 + (t & 15)];
        }
        u32x4 q = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int v = requantized(x[j], 16 * g + j < n ? ratio[1][16 * g + j] : 0.f);
            q[j / 4] |= static_cast<uint32_t>(v & 0xFF) << (8 * (j % 4));
        }
        *reinterpret_cast<u32x4*>(a.to.v + to + 16 * g * D + d * 16) = q;
    }
}

}  // namespace tetra_dev
