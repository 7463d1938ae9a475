// Eviction from the paged cache by accumulated attention weight (kv_evict).
// Included by batch.hip.
//
// Of every sequence and cache head the tokens of most weight and the last ones
// go in their order into other pages: first which tokens, then their move.  Which
// ones is a selection by a 32-bit key that rises with the weight, found from
// histograms of its bits, so equal weights are told apart by the token alone and
// nothing depends on the order of atomics.
//
// The move is bound by HBM where most tokens stay: 64 sequences of 4,096 tokens
// kept whole, 8 heads of 128, 1,074 MB, 233 us with the choice, 4,610 GB/s (a large copy:
// 5,160).  With gaps between the kept tokens it reads more than it needs: values lie
// transposed in groups of 16 tokens, and a group is read whole (2 KB for a head of
// 128) for any token of it.  Half of the tokens kept: 176 us for 537 MB; one in 32 of
// 131,072: 18 us.
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

// What the two forms of the choice have in common: a workgroup's bins and its waves' counts.
struct EvictLds {
    unsigned count[kEvictBins], above[kEvictWaves], equal[kEvictWaves];
    int found[2];

    // found: the bin in which the count from the last bin down reaches `need`, and what it has to give; a thread has two
    // neighbouring bins, hi of the last but 2 tid and lo below it
    __device__ __forceinline__ void find(unsigned hi, unsigned lo, unsigned need) {
        const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = kEvictBins - 2 - 2 * tid;
        const unsigned upto = wave_upto(Sum(), hi + lo);
        if ((tid & 63) == 63) above[wave] = upto;
        __syncthreads();
        unsigned before = upto - hi - lo;
        for (int w = 0; w < wave; ++w) before += above[w];
        if (before < need && before + hi >= need) {
            found[0] = b + 1;
            found[1] = need - before;
        } else if (before + hi < need && before + hi + lo >= need) {
            found[0] = b;
            found[1] = need - before - hi;
        }
        __syncthreads();
    }

    // Puts the tokens of `each` above the cut, and as many at it that `left` are put with the `equals` before them, in
    // their order from `place` + min(equals, left) on.
    template <class Each, class Put>
    __device__ __forceinline__ void select(Each each, uint32_t cut, int left, int place, int equals, Put put) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        unsigned n_above = 0, n_equal = 0;
        each([&](int, float x, bool is) {
            const uint32_t k = rising_key(x);
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
        for (int w = 0; w < wave; ++w) {
            place += above[w];
            equals += equal[w];
        }
        place += min(equals, left);
        const unsigned long long below = (1ull << lane) - 1;
        each([&](int t, float x, bool is) {
            const uint32_t k = rising_key(x);
            const unsigned long long same = __ballot(is && k == cut);
            const bool stays = is && (k > cut || (k == cut && equals + static_cast<int>(__popcll(same & below)) < left));
            const unsigned long long staying = __ballot(stays);
            if (stays) put(place + static_cast<int>(__popcll(staying & below)), t, x);
            place += __popcll(staying);
            equals += __popcll(same);
        });
    }
};

// The smallest key that stays is found eleven bits at a time from the histogram of the
// keys that agree so far; then every wave writes its part of the tokens.  64 sequences
// of up to 4,096 tokens, 8 heads: 12.5 us, three rounds of LDS atomics and scans.  A wave's part
// is in line, a token a lane, kEvictHeld of a lane in registers from the start: all of them,
// as tables with room for more than kEvictHeld kEvictThreads tokens take the form below.
__global__ __launch_bounds__(kEvictThreads) void evict_choose_kernel(EvictArgs a) {
    __shared__ EvictLds sh;
    unsigned(&count)[kEvictBins] = sh.count;
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
    };
    uint32_t cut = 0;
    int left = pick;                                            // of the keys that begin like `cut`
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < kEvictBins; i += kEvictThreads) count[i] = 0;
        __syncthreads();
        each([&](int, float x, bool is) {
            const uint32_t k = rising_key(x);
            if (is && (pass == 0 || (k >> (shift + bits)) == (cut >> (shift + bits))))
                atomicAdd(&count[k >> shift & ((1u << bits) - 1)], 1u);
        });
        __syncthreads();
        const int b = kEvictBins - 2 - 2 * tid;
        sh.find(count[b + 1], count[b], left);
        cut |= static_cast<uint32_t>(sh.found[0]) << shift;
        left = sh.found[1];
        __syncthreads();
    }
    sh.select(each, cut, left, 0, 0, put);
}

// The same for long sequences, in parts of a row: a launch for each eleven bits, which
// leaves the parts' histograms, and one that writes the tokens.  Each adds up the last
// histograms for itself: where the count reaches the cut, and how many before its own
// part stay.  8 heads of 131,072 tokens in 16 parts each: 4.7, 8, 7.8 and 11 us (one
// workgroup a head: 144); with 8 parts as long, with 4 half as long again.

template <int PASS>
__global__ __launch_bounds__(kEvictThreads) void evict_part_kernel(EvictArgs a) {
    __shared__ EvictLds sh;
    unsigned(&count)[kEvictBins] = sh.count;
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
        u32x2 c[kEvictParts];                  // all on their way at once
#pragma unroll
        for (int p = 0; p < kEvictParts; ++p) c[p] = *reinterpret_cast<const u32x2*>(bins(PASS - 1, min(p, a.parts - 1)) + b);
#pragma unroll
        for (int p = 0; p < kEvictParts; ++p) {
            hi += p < a.parts ? c[p][1] : 0;
            lo += p < a.parts ? c[p][0] : 0;
            hi_before += p < mine ? c[p][1] : 0;
            lo_before += p < mine ? c[p][0] : 0;
        }
        sh.find(hi, lo, left);
        const int bin = sh.found[0];
        left = sh.found[1];
        cut |= static_cast<uint32_t>(bin) << shift;
        const unsigned over = wave_all(Sum(), (b + 1 > bin ? hi_before : 0) + (b > bin ? lo_before : 0));
        const unsigned same = wave_all(Sum(), (b + 1 == bin ? hi_before : 0) + (b == bin ? lo_before : 0));
        if (lane == 0) {
            sh.above[wave] = over;
            sh.equal[wave] = same;
        }
        __syncthreads();
        for (int w = 0; w < kEvictWaves; ++w) {
            before_part += sh.above[w];
            equals_before += sh.equal[w];
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
            const uint32_t k = rising_key(x);
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
        sh.select(each, cut, left, before_part, equals_before, put);
    }
}

// four whole numbers times ratio, rounded
__device__ __forceinline__ uint32_t moved4(uint32_t q, float ratio) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= static_cast<uint32_t>(requantized(static_cast<int8_t>(q >> (8 * i)), ratio) & 0xFF) << (8 * i);
    return w;
}

// 16 places of a new page and head, keys or values: a wave each, for itself.  Every wave
// finds the page's scale from the scales of all its tokens, while what it moves is on its
// way.  Keys are rows of D bytes, moved in pieces of 16.  Of values a lane takes a
// dimension of the 16 places, whose bytes lie in as many groups of 16 old tokens as the
// kept ones do: it loads those groups' 16 bytes and picks from them with byte permutes,
// whose selectors are the same for all dimensions.  (Bytes loaded one by one took 73
// cycles of a CU for each load of a wave.)
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    const int lane = threadIdx.x & 63, B = a.to.page_tokens, groups = B / kGroupTokens;
    unsigned rest = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = rest % groups;
    rest /= groups;
    const int kind = rest & 1;
    rest >>= 1;
    const int head = rest % a.from.kv_heads;
    rest /= a.from.kv_heads;
    const int seq = rest / a.to.max_pages, number = rest - seq * a.to.max_pages;
    if (seq >= a.from.seqs) return;
    const int page = a.to.pages[static_cast<size_t>(seq) * a.to.max_pages + number];
    const EvictShape s = evict_shape(a, seq);
    const int n = min(B, s.kept - number * B), n_group = min(kGroupTokens, n - kGroupTokens * group);
    if (n_group <= 0 || page < 0 || page >= a.to.num_pages) return;
    const int* tokens = a.tokens + (static_cast<size_t>(seq) * a.from.kv_heads + head) * a.capacity + static_cast<size_t>(number) * B;
    const int* table = a.from.pages + static_cast<size_t>(seq) * a.from.max_pages;
    const size_t stride = static_cast<size_t>(B) * D;
    auto page_of = [&](int t) {
        const int p = table[t >> a.from.page_shift];
        return p >= 0 && p < a.from.num_pages ? p : -1;
    };
    auto head_of = [&](int p) { return static_cast<size_t>(p) * a.from.kv_heads + head; };
    auto scale_of = [&](int p) { return p >= 0 ? a.from.scales[2 * head_of(p) + kind] : 0.f; };
    // the wave's tokens, in each 16 lanes; then the page's
    const int i = lane & 15, t = i < n_group ? tokens[kGroupTokens * group + i] : -1;
    const int t_lo = lane < n ? tokens[lane] : -1, t_hi = lane + 64 < n ? tokens[lane + 64] : -1;
    const int p = t >= 0 ? page_of(t) : -1;
    const int p_lo = t_lo >= 0 ? page_of(t_lo) : -1, p_hi = t_hi >= 0 ? page_of(t_hi) : -1;
    constexpr int kPer = kGroupTokens * D / 16 / 64;
    u32x4 piece[kPer];
    const int t0 = __builtin_amdgcn_readfirstlane(t), p0 = __builtin_amdgcn_readfirstlane(p);
    if (kind == 0) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int at = (64 * u + lane) / (D / 16), tj = __shfl(t, at, 64), pj = __shfl(p, at, 64);
            piece[u] = u32x4{0, 0, 0, 0};
            if (pj >= 0)
                piece[u] = *reinterpret_cast<const u32x4*>(a.from.k + head_of(pj) * stride + (tj & (B - 1)) * D + 16 * (lane % (D / 16)));
        }
    } else {
        auto old_group = [&](int tj, int pj, u32x4 (&to)[kPer]) {
#pragma unroll
            for (int u = 0; u < kPer; ++u)
                to[u] = *reinterpret_cast<const u32x4*>(a.from.v + head_of(pj) * stride + (tj & (B - 1) & ~15) * D + (64 * u + lane) * 16);
        };
        if (p0 >= 0 && (t0 & 15) == 0 && __all(t == t0 + i)) {
            old_group(t0, p0, piece);
        } else {
            // Where the next old group begins among the places (those without a page left out), four on their way at
            // once.  Lane 4 k + w has how word w of an old group goes into word k: its byte, or the one that is there.
            const int before = __shfl(t, i ? i - 1 : 0, 64);
            unsigned begins = __ballot(p >= 0 && (i == 0 || t >> 4 != before >> 4)) & 0xFFFF;
            int word_t[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) word_t[b] = __shfl(t, (lane & 12) + b, 64);
#pragma unroll
            for (int u = 0; u < kPer; ++u) piece[u] = u32x4{0, 0, 0, 0};
            while (begins) {
                u32x4 old[4][kPer];
                int group_t[4];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    group_t[m] = -1;
                    if (begins) {
                        const int j = __builtin_ctz(begins);
                        begins &= begins - 1;
                        group_t[m] = __builtin_amdgcn_readlane(t, j);
                        old_group(group_t[m], __builtin_amdgcn_readlane(p, j), old[m]);
                    }
                }
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (group_t[m] < 0) break;
                    uint32_t choice = 0x07060504u;
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if (word_t[b] >> 2 == (group_t[m] >> 4) * 4 + (lane & 3))
                            choice = (choice & ~(0xFFu << (8 * b))) | static_cast<uint32_t>(word_t[b] & 3) << (8 * b);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const uint32_t c = __builtin_amdgcn_readlane(choice, 4 * k + w);
#pragma unroll
                            for (int u = 0; u < kPer; ++u) piece[u][k] = __builtin_amdgcn_perm(piece[u][k], old[m][u][w], c);
                        }
                }
            }
        }
    }
    const float mine = scale_of(p), grown = wave_all(Max(), fmaxf(scale_of(p_lo), scale_of(p_hi)));
    const float ratio = grown > 0.f ? mine / grown : 0.f;
    const size_t to = static_cast<size_t>(page) * a.to.kv_heads + head;
    if (group == 0 && lane == 0) a.to.scales[2 * to + kind] = grown;
    if (kind == 0) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int at = (64 * u + lane) / (D / 16);
            const float f = __shfl(ratio, at, 64);
            if (f != 1.f)
#pragma unroll
                for (int k = 0; k < 4; ++k) piece[u][k] = moved4(piece[u][k], f);
            if (at < n_group)
                *reinterpret_cast<u32x4*>(a.to.k + to * stride + (kGroupTokens * group + at) * D + 16 * (lane % (D / 16))) = piece[u];
        }
        return;
    }
    if (__any(ratio != 1.f && i < n_group))
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float f = lane_of(ratio, j);
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int q = requantized(static_cast<int8_t>(piece[u][j / 4] >> (8 * (j % 4))), f);
                piece[u][j / 4] = (piece[u][j / 4] & ~(0xFFu << (8 * (j % 4)))) | static_cast<uint32_t>(q & 0xFF) << (8 * (j % 4));
            }
        }
#pragma unroll
    for (int u = 0; u < kPer; ++u)
        *reinterpret_cast<u32x4*>(a.to.v + to * stride + kGroupTokens * group * D + (64 * u + lane) * 16) = piece[u];
}

}  // namespace tetra_dev
