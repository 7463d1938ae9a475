// The attention weight that cached tokens get from a call's rows (kv_weigh).
// Included by batch.hip.
//
//   mass'[s][h][j] = decay mass[s][h][j] + sum_i 2^(s_ij - L_i), L_i = log2 sum_t 2^(s_it)
//
// over the rows i (token, q head of the cache head h: in that order) of sequence
// s that see token j, with s_ij = scale log2(e) q_i . k_j.  L must be known before
// the sum over rows, so the scores are found twice: once for L (a row's largest
// score and sum over each span of tokens, then joined), once for the weights.
//
// Prompts: the keys stay and the rows pass by.  A wave holds 32 tokens in fp16
// as operands of v_mfma_f32_32x32x16_f16, S^T = K Q^T, and a workgroup's eight waves
// share the rows, 32 at a time, from LDS.  A lane then has scores of one row (lane
// % 32) and 16 tokens: 8 (i / 4) + 4 (lane / 32) + i % 4.  A row's maximum and sum
// stay within a lane and its other half; a token's sum over the rows is one addition
// a score, and one exchange over the lanes at the end.  The lengths are the device's,
// so every workgroup plans for itself: blocks of tokens by chunks of rows, some eight
// of them each.  4,096 tokens of 32 heads over 8 of 128: 148 and 133 us, 466 and 518
// TFLOP/s; vector units busy 66 % of the cycles and matrix cores 30 %, which take turns
// on a SIMD: an exponential a score and pass is 45 % of the former.  64 tokens a wave and four
// waves 158 and 146 us with more instructions and 165 and 154 with fewer, two tiles of rows
// a barrier 164 and 160, half as many items 171 and 167.
//
// Single tokens: see weigh_few_kernel.
#pragma once

#include <type_traits>

#include "attend.h"

namespace tetra_dev {

constexpr int kWeighBlock = 256;          // tokens of a workgroup
constexpr int kWeighWaves = kWeighBlock / 32;
constexpr int kWeighRows = 32;            // rows of a tile
constexpr int kWeighSpans = 256;          // of a sequence's tokens, for the sums, at most
constexpr int kWeighMostTiles = 16;       // row tiles whose sums a workgroup holds in LDS
constexpr int kWeighItems = 8;            // of a workgroup, where there are enough
constexpr float kWeighNone = -3e38f;      // a maximum over no score
constexpr long long kWeighScores = 16 << 20;   // scores that single tokens' first pass leaves for the second, at most

struct WeighArgs {
    KvCache c;
    const uint16_t* q;
    const int* starts;
    const float* mass;
    float* out;
    float* spans;         // [spans_most][rows][q_heads][2]: largest score and sum of a row over a span
    float* logs;          // [rows][q_heads]: L, +inf where a row sees nothing
    float* parts;         // [2 items_most][kWeighBlock]: a block's sums over some of its rows
    long long q_stride;
    float scale;          // |scale| log2(e)
    uint32_t q_flip;      // 0x80008000 if the scale is negative: turns q instead
    float decay;
    int rows, max_new, q_heads, group, window, mass_tokens;
    int workers;          // workgroups, or waves, that share the items of a launch
    int block, spans_most;   // tokens of a block; spans of a sequence at most
    int* span;               // the blocks of a span, at least, for the kernel of the logs
    int items_most;          // chunks of rows are so long that no more items than this have one
    float* scores;           // [blocks of all sequences and heads][rows of a sequence][64], of weigh_few_kernel
    long long scores_most;   // that there is room for
    int score_rows;          // rows of a sequence and cache head at most
};

// What a sequence asks for.
struct WeighSeq {
    Span s;
    int all;              // its rows, those past max_new among them
    int end;              // tokens that may be seen: below this
    int written;          // tokens that have a place in mass_out
    int blocks, tiles;    // of its tokens, of its rows

    __device__ __forceinline__ WeighSeq() : s{0, 0, 0, 0}, all(0), end(0), written(0), blocks(0), tiles(0) {}
    __device__ __forceinline__ WeighSeq(const WeighArgs& a, int seq) {
        const int start = a.starts[seq], next = a.starts[seq + 1], len = a.c.lens[seq];
        s = span_between(start, next, len, a.rows, a.max_new);
        all = max(min(max(next, 0), a.rows) - s.row0, 0);
        const long long kept = static_cast<long long>(a.c.max_pages) << a.c.page_shift;
        end = static_cast<int>(min(static_cast<long long>(s.len), kept));
        written = min(max(len, 0), a.mass_tokens);
        // a sequence that keeps what it has needs no visit where it has that already
        if (all == 0 && a.mass == a.out) written = 0;
        blocks = (max(s.n ? end : 0, written) + a.block - 1) / a.block;
        tiles = (s.n * a.group + kWeighRows - 1) / kWeighRows;
    }
};

// Items of a launch: a sequence's (head, block or span of blocks, chunk of row tiles).
struct WeighItem {
    int seq, head, block, blocks, tile, tiles;      // blocks `block` .. block + blocks - 1, tiles likewise
    int chunks;                                     // of the block
    int slot;                                       // of the item's part, where there are several chunks
    int before;                                     // slots of the sequences before
    WeighSeq q;
};

enum WeighPass { kWeighSpanSums, kWeighTokens, kWeighJoin };

// Row tiles of a chunk, so that there are some items_most items (kWeighItems a workgroup,
// where a full table has as many): then no more than twice that many have a part of a
// block's sums to leave.
struct WeighPlan {
    int chunk, total;             // row tiles of a chunk; items
    int span;                     // blocks of a span, at least
    bool keep;                    // there is room for all scores
    int lane_items, lane_slots;   // of a lane's sequence, the first 64

    __device__ __forceinline__ static int span_blocks(const WeighArgs& a, const WeighSeq& q, int least) {
        return max(least, (q.blocks + a.spans_most - 1) / a.spans_most);
    }
    __device__ __forceinline__ static int spans_of(const WeighArgs& a, const WeighSeq& q, int least) {
        const int n = span_blocks(a, q, least);
        return (q.blocks + n - 1) / n;
    }
    __device__ __forceinline__ int chunks_of(const WeighSeq& q) const { return max(1, (q.tiles + chunk - 1) / chunk); }
    __device__ __forceinline__ int slots_of(const WeighArgs& a, const WeighSeq& q) const {
        const int n = chunks_of(q);
        return n > 1 ? n * q.blocks * a.c.kv_heads : 0;
    }
    template <WeighPass PASS>
    __device__ __forceinline__ int items_of(const WeighArgs& a, const WeighSeq& q) const {
        if (PASS == kWeighSpanSums) return spans_of(a, q, span) * a.c.kv_heads * chunks_of(q);
        if (PASS == kWeighTokens) return q.blocks * a.c.kv_heads * chunks_of(q);
        return chunks_of(q) > 1 ? q.blocks * a.c.kv_heads : 0;
    }

    template <WeighPass PASS, bool FEW>
    __device__ __forceinline__ WeighPlan(const WeighArgs& a, WeighSeq& mine, std::integral_constant<WeighPass, PASS>,
                                         std::integral_constant<bool, FEW>) {
        const int lane = threadIdx.x & 63;
        unsigned long long steps = 0, blocks = 0;
        int live = 0;
        for (int i = lane; i < a.c.seqs; i += 64) {
            const WeighSeq q(a, i);
            if (i < 64) mine = q;
            steps += static_cast<unsigned long long>(q.blocks) * q.tiles * a.c.kv_heads;
            blocks += q.blocks;
            live += q.blocks > 0;
        }
        steps = wave_all(Sum(), steps);
        span = 1;
        keep = false;
        if (FEW) {
            // an item a wave, of equal spans: each sequence and head may have one that is not full
            const long long ends = static_cast<long long>(wave_all(Sum(), live)) * a.c.kv_heads;
            const long long room = max(static_cast<long long>(a.workers) - ends, static_cast<long long>(a.workers / 2));
            blocks = wave_all(Sum(), blocks) * a.c.kv_heads;
            span = static_cast<int>(max(1ll, min((static_cast<long long>(blocks) + room - 1) / room, 1ll << 24)));
            keep = static_cast<long long>(blocks) * 64 * a.score_rows <= a.scores_most;
        }
        const unsigned long long most = a.items_most;
        chunk = static_cast<int>(max(1ull, min((steps + most - 1) / most, 1ull << 26)));
        if (PASS == kWeighSpanSums) chunk = min(chunk, kWeighMostTiles);
        lane_items = items_of<PASS>(a, mine);
        lane_slots = FEW ? mine.blocks * a.c.kv_heads : slots_of(a, mine);
        total = wave_all(Sum(), lane_items);
        for (int i0 = 64; i0 < a.c.seqs; i0 += 64) {
            int n = 0;
            if (i0 + lane < a.c.seqs) n = items_of<PASS>(a, WeighSeq(a, i0 + lane));
            total += wave_all(Sum(), n);
        }
    }

    // item x of all; the sequences a lane each
    template <WeighPass PASS, bool FEW = false>
    __device__ __forceinline__ WeighItem find(const WeighArgs& a, const WeighSeq& first, int x,
                                              std::integral_constant<WeighPass, PASS>,
                                              std::integral_constant<bool, FEW> = {}) const {
        const int lane = threadIdx.x & 63;
        WeighItem w;
        w.seq = -1;
        int before = 0, slots = 0;
        for (int i0 = 0; i0 < a.c.seqs; i0 += 64) {
            WeighSeq q = first;
            int n = lane_items, m = lane_slots;
            if (i0) {
                q = WeighSeq();
                if (i0 + lane < a.c.seqs) q = WeighSeq(a, i0 + lane);
                n = items_of<PASS>(a, q);
                m = FEW ? q.blocks * a.c.kv_heads : slots_of(a, q);
            }
            const int upto = wave_upto(Sum(), n) + before, slots_upto = wave_upto(Sum(), m) + slots;
            const unsigned long long has = __ballot(upto > x);
            if (has) {
                const int l = __builtin_ctzll(has);
                w.seq = i0 + l;
                w.q.s = {lane_of(q.s.row0, l), lane_of(q.s.n, l), lane_of(q.s.first, l), lane_of(q.s.len, l)};
                w.q.all = lane_of(q.all, l);
                w.q.end = lane_of(q.end, l);
                w.q.written = lane_of(q.written, l);
                w.q.blocks = lane_of(q.blocks, l);
                w.q.tiles = lane_of(q.tiles, l);
                const int at = x - lane_of(upto - n, l), per = PASS == kWeighJoin ? 1 : chunks_of(w.q);
                const int place = at / per, part = at - place * per;
                w.chunks = chunks_of(w.q);
                w.head = place % a.c.kv_heads;
                w.block = place / a.c.kv_heads;
                w.blocks = 1;
                if (PASS == kWeighSpanSums) {
                    w.blocks = span_blocks(a, w.q, span);
                    w.block *= w.blocks;
                    w.blocks = min(w.blocks, w.q.blocks - w.block);
                }
                w.tile = part * chunk;
                w.tiles = min(chunk, w.q.tiles - w.tile);
                w.before = lane_of(slots_upto - m, l);
                w.slot = w.before + (place * w.chunks) + part;
                return w;
            }
            before = lane_of(upto, 63);
            slots = lane_of(slots_upto, 63);
        }
        return w;
    }
};

// Items of a workgroup: every `workers`-th, every other round from the other end, so
// that a prompt's first blocks, which all rows see, and its last, which few do, come
// to the same workgroups.
__device__ __forceinline__ int weigh_item(const WeighArgs& a, int round) {
    const int w = blockIdx.x;
    return round * a.workers + (round & 1 ? a.workers - 1 - w : w);
}

// sums over 16 neighbouring lanes of 16 numbers: lane e of them gets that of v[e]
__device__ __forceinline__ float weigh_scatter(float (&v)[16]) {
    const int lane = threadIdx.x & 63;
    auto halve = [&](int bit, auto other) {
#pragma unroll
        for (int j = 0; j < bit; ++j) {
            const bool up = lane & bit;
            const float keep = up ? v[j + bit] : v[j], give = up ? v[j] : v[j + bit];
            v[j] = keep + other(give);
        }
    };
    halve(8, [](float x) { return dpp<0x128, 0xF>(x); });
    halve(4, [](float x) { return dpp<0x141, 0xF>(x); });
    halve(2, [](float x) { return dpp<0x4E, 0xF>(x); });
    halve(1, [](float x) { return dpp<0xB1, 0xF>(x); });
    return v[0];
}

// a block's new mass: what token t had, and `sum`
__device__ __forceinline__ void weigh_write(const WeighArgs& a, const WeighItem& w, int t, float sum) {
    if (t >= w.q.written) return;
    const size_t at = (static_cast<size_t>(w.seq) * a.c.kv_heads + w.head) * a.mass_tokens + t;
    float before = 0.f;
    if (a.mass && (w.q.all == 0 || t < w.q.s.first)) before = a.mass[at] * (w.q.all ? a.decay : 1.f);
    a.out[at] = before + sum;
}

template <int D, WeighPass PASS>
__global__ __launch_bounds__(64 * kWeighWaves, 2 * kWeighWaves / 4) void weigh_kernel(WeighArgs a) {
    constexpr int kThreads = 64 * kWeighWaves, kSlices = D / 8;
    constexpr int kPieces = kSlices * kWeighRows;               // of 8 dimensions, of a tile of rows
    constexpr int kPer = (kPieces + kThreads - 1) / kThreads;   // and of a thread
    static_assert(kPieces % kThreads == 0 || kPer == 1, "all of a thread's or none");
    constexpr std::integral_constant<WeighPass, PASS> pass;
    constexpr bool kSums = PASS == kWeighSpanSums;
    // a slice's rows, and one row more, so that neither a slice's rows nor a row's slices meet in a bank
    __shared__ __align__(16) _Float16 rows[2][kSlices][kWeighRows + 1][8];
    __shared__ float row_logs[2][kWeighRows];
    __shared__ float sums[kSums ? kWeighWaves : 1][kSums ? kWeighMostTiles * kWeighRows : 1][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lrow = lane & 31, half = lane >> 5;
    const float inverse_group = 1.f / static_cast<float>(a.group);
    const int step_t = kWeighRows / a.group, step_g = kWeighRows - step_t * a.group;
    WeighSeq first;
    const WeighPlan plan(a, first, pass, std::false_type());
    if (kSums && blockIdx.x == 0 && threadIdx.x == 0) *a.span = plan.span;
    const size_t stride = static_cast<size_t>(a.c.page_tokens) * D;
    for (int round = 0;; ++round) {
        if (static_cast<long long>(round) * a.workers >= plan.total) break;
        const int x = weigh_item(a, round);
        if (x >= plan.total) continue;
        const WeighItem w = plan.find(a, first, x, pass);
        const Span& s = w.q.s;
        const int* table = a.c.pages + static_cast<size_t>(w.seq) * a.c.max_pages;
        const int all_rows = s.n * a.group;
        if constexpr (kSums) {
            __syncthreads();
            for (int i = lane; i < w.tiles * kWeighRows; i += 64) {
                sums[wave][i][0] = kWeighNone;
                sums[wave][i][1] = 0.f;
            }
        }
        float total[16];
        if constexpr (!kSums)
            for (float& v : total) v = 0.f;
        for (int block = w.block; block < w.block + w.blocks; ++block) {
            // the rows that see something of the block: tiles tile0 .. tile1 - 1
            const int t_begin = block * kWeighBlock, t_end = min(t_begin + kWeighBlock, w.q.end);
            int row_a = max(0, t_begin - s.first), row_b = s.n;
            if (a.window > 0)
                row_b = static_cast<int>(max(0ll, min(static_cast<long long>(row_b), static_cast<long long>(t_end) - 1 + a.window - s.first)));
            int tile0 = max(w.tile, static_cast<int>(min(static_cast<long long>(row_a) * a.group, static_cast<long long>(all_rows)) / kWeighRows));
            int tile1 = min(w.tile + w.tiles, static_cast<int>((static_cast<long long>(row_b) * a.group + kWeighRows - 1) / kWeighRows));
            if (t_end <= t_begin) tile1 = tile0;
            if (tile0 >= tile1) continue;
            // the wave's tokens
            const int mine = t_begin + 32 * wave;
            f16x8 k[D / 16];
            float unit[2];                        // of 16 tokens each: scale of the scores
            unsigned there = 0;                   // which of those have a page
            {
                const int token = mine + lrow;
                const int page = token < t_end ? table[token >> a.c.page_shift] : -1;
                const bool is = page >= 0 && page < a.c.num_pages;
                const size_t ph = static_cast<size_t>(is ? page : 0) * a.c.kv_heads + w.head;
                const int8_t* kp = a.c.k + ph * stride + (token & (a.c.page_tokens - 1)) * D + 16 * half;
                u32x4 raw[D / 32];
#pragma unroll
                for (int c = 0; c < D / 32; ++c) raw[c] = *reinterpret_cast<const u32x4*>(kp + 32 * c);
                const float scale = a.c.scales[2 * ph] * a.scale;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    k[2 * c] = to_half8(raw[c][0], raw[c][1]);
                    k[2 * c + 1] = to_half8(raw[c][2], raw[c][3]);
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    unit[g] = lane_of(scale, 16 * g);
                    there |= static_cast<unsigned>(__builtin_amdgcn_readlane(is, 16 * g)) << g;
                }
            }
            // Row r of the sequence is token r / group, head r % group; a tile's first row as both, uniform.
            struct TileAt {
                int t, g;
            };
            auto step = [&](TileAt& p) {
                p.t += step_t;
                p.g += step_g;
                if (p.g >= a.group) {
                    p.g -= a.group;
                    ++p.t;
                }
            };
            auto row_of = [&](const TileAt& p, int i, int& token) {
                const int j = static_cast<int>((static_cast<float>(p.g + i) + 0.5f) * inverse_group);
                token = p.t + j;
                return w.head * a.group + p.g + i - j * a.group;
            };
            // a tile on its way, and the place of the next to load
            u32x4 piece[kPer];
            float next_log = 0.f;
            TileAt ahead;
            ahead.t = __builtin_amdgcn_readfirstlane(tile0 * kWeighRows / a.group);
            ahead.g = tile0 * kWeighRows - ahead.t * a.group;
            TileAt now = ahead;
            const int pc = tid % kSlices;
            // where the heads of a cache head divide a tile, a thread's pieces of a tile are step_t tokens after those before
            const uint16_t* from[kPer];
            int from_token[kPer];
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int h = row_of(ahead, (tid + u * kThreads) / kSlices, from_token[u]);
                from[u] = a.q + (s.row0 + from_token[u]) * a.q_stride + h * D + pc * 8;
            }
            auto load = [&] {
                int token;
#pragma unroll
                for (int u = 0; u < kPer; ++u) {
                    piece[u] = u32x4{0, 0, 0, 0};
                    if (kPieces < kThreads && tid >= kPieces) continue;
                    if (step_g == 0) {
                        if (from_token[u] < s.n) piece[u] = *reinterpret_cast<const u32x4*>(from[u]);
                        from_token[u] += step_t;
                        from[u] += step_t * a.q_stride;
                    } else {
                        const int h = row_of(ahead, (tid + u * kThreads) / kSlices, token);
                        if (token < s.n) piece[u] = *reinterpret_cast<const u32x4*>(a.q + (s.row0 + token) * a.q_stride + h * D + pc * 8);
                    }
                }
                if (!kSums && wave == 0) {
                    const int h = row_of(ahead, lrow, token);
                    next_log = token < s.n ? a.logs[static_cast<size_t>(s.row0 + token) * a.q_heads + h] : INFINITY;
                }
                step(ahead);
            };
            auto store = [&](int b) {
#pragma unroll
                for (int u = 0; u < kPer; ++u)
                    if (kPieces >= kThreads || tid < kPieces)
                        *reinterpret_cast<f16x8*>(rows[b][pc][(tid + u * kThreads) / kSlices]) = query8(piece[u], a.q_flip);
                if (!kSums && wave == 0) row_logs[b][lrow] = next_log;
            };
            load();
            __syncthreads();                      // the block before is done with the rows
            store(0);
            if (tile0 + 1 < tile1) load();
            for (int tile = tile0; tile < tile1; ++tile) {
                const int b = (tile - tile0) & 1;
                __syncthreads();
                if (tile + 1 < tile1) {
                    store(b ^ 1);
                    if (tile + 2 < tile1) load();
                }
                const float my_log = kSums ? 0.f : row_logs[b][lrow];
                f32x16 z;
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        z = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                            k[2 * c + u], *reinterpret_cast<const f16x8*>(rows[b][4 * c + 2 * half + u][lrow]), z, 0, 0, 0);
                // do all of the tile's rows see all of the wave's tokens (rows past the last matter to none)?
                const int position0 = s.first + now.t, position1 = position0 + step_t + 1;
                const bool all = there == 3u && mine + 32 <= min(position0 + 1, t_end) &&
                                 (a.window == 0 || position1 - a.window < mine);
                const TileAt at = now;
                step(now);
                auto finish = [&](auto masked) {
                    unsigned lo = 0, n = 0;                // tokens [lo, lo + n) of the lane's half, of those with a page
                    if constexpr (masked) {
                        int token;
                        row_of(at, lrow, token);
                        const int position = s.first + token;
                        const int see_end = token < s.n ? min(position + 1, t_end) : 0;
                        const int see_begin = a.window > 0 ? max(0, max(position, 0) - a.window + 1) : 0;
                        lo = static_cast<unsigned>(see_begin - mine - 4 * half);
                        n = static_cast<unsigned>(max(see_end - see_begin, 0));
                    }
                    auto unseen = [&](int e) { return static_cast<unsigned>(8 * (e / 4) + e % 4) - lo >= n || !(there >> (e / 8) & 1); };
                    if constexpr (kSums) {
                        // the largest before the scale, which is the same for 8 of a lane and not below 0
                        float top = kWeighNone;
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            float most = -INFINITY;
#pragma unroll
                            for (int e = 8 * g; e < 8 * g + 8; ++e) {
                                if constexpr (masked) z[e] = unseen(e) ? -INFINITY : z[e];
                                most = fmaxf(most, z[e]);
                            }
                            top = fmaxf(top, most > -INFINITY ? most * unit[g] : -INFINITY);
                        }
                        float* at_row = sums[wave][(tile - w.tile) * kWeighRows + lrow];
                        const float m0 = at_row[0], l0 = at_row[1];
                        const float m = fmaxf(with_half(Larger(), top), m0);
                        float l = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float v = fast_exp2(__builtin_fmaf(z[e], unit[e / 8], -m));
                            if constexpr (masked) v = z[e] == -INFINITY ? 0.f : v;
                            l += v;
                        }
                        l = with_half(Sum(), l) + l0 * fast_exp2(m0 - m);
                        if (half == 0) {
                            at_row[0] = m;
                            at_row[1] = l;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float v = fast_exp2(__builtin_fmaf(z[e], unit[e / 8], -my_log));
                            if constexpr (masked) v = unseen(e) ? 0.f : v;
                            total[e] += v;
                        }
                    }
                };
                if (all) finish(std::false_type());
                else finish(std::true_type());
            }
        }
        if constexpr (kSums) {
            __syncthreads();
            for (int r = tid; r < w.tiles * kWeighRows; r += kThreads) {
                const int row = w.tile * kWeighRows + r;
                if (row >= all_rows) break;
                float m = kWeighNone, l = 0.f;
                for (int i = 0; i < kWeighWaves; ++i) m = fmaxf(m, sums[i][r][0]);
                for (int i = 0; i < kWeighWaves; ++i) l += sums[i][r][1] * fast_exp2(sums[i][r][0] - m);
                const int token = row / a.group, h = w.head * a.group + row - token * a.group;
                const size_t span = w.block / WeighPlan::span_blocks(a, w.q, plan.span);
                float* to = a.spans + ((span * a.rows + s.row0 + token) * a.q_heads + h) * 2;
                *reinterpret_cast<f32x2*>(to) = f32x2{m, l};
            }
        } else {
            // lane e of 16 gets the sum of total[e] over them, then over the other 16 of the half
            const float sum = with_row(Sum(), weigh_scatter(total));
            const int place = 32 * wave + 8 * ((lrow & 15) >> 2) + 4 * half + (lrow & 3);
            if (lrow < 16) {
                if (w.chunks == 1) weigh_write(a, w, w.block * kWeighBlock + place, sum);
                else a.parts[static_cast<size_t>(w.slot) * kWeighBlock + place] = sum;
            }
        }
    }
}

// L of row `lane` of a sequence's `rows` (64 at most) of a cache head, from its spans' largest
// scores and sums: 64 / R lanes a row, R the next power of two.  Every wave that asks
// joins them in the same order.  With up to 16 rows this costs less than the launch of
// weigh_logs_kernel: 4 rows over 203 tokens 11.0 and 12.5 us, 64 sequences of 5 rows over up to
// 4,096 37 and 40, 5 rows over 131,072 (256 spans) 49 and 54.  With 32 over 65,536 it took 51
// and the launch 44.
__device__ __forceinline__ float weigh_log(const WeighArgs& a, const WeighItem& w, int rows, int spans) {
    const int lane = threadIdx.x & 63;
    int R = 1;
    while (R < rows) R *= 2;
    const int i = lane & (R - 1), token = i / a.group;
    const size_t step = static_cast<size_t>(a.rows) * a.q_heads;
    const f32x2* p = reinterpret_cast<const f32x2*>(a.spans) + static_cast<size_t>(w.q.s.row0 + token) * a.q_heads + w.head * a.group + i -
                     token * a.group;
    float m = kWeighNone, l = 0.f;
    if (i < rows)
#pragma unroll 4
        for (int k = lane / R; k < spans; k += 64 / R) {
            const f32x2 x = p[k * step];
            const float n = fmaxf(m, x[0]);
            l = l * fast_exp2(m - n) + x[1] * fast_exp2(x[0] - n);
            m = n;
        }
    for (int k = R; k < 64; k *= 2) {
        const float m1 = __shfl_xor(m, k, 64), l1 = __shfl_xor(l, k, 64), n = fmaxf(m, m1);
        l = l * fast_exp2(m - n) + l1 * fast_exp2(m1 - n);
        m = n;
    }
    return lane >= rows || l == 0.f ? INFINITY : m + __builtin_amdgcn_logf(l);
}

// The same for sequences of up to 16 RT rows (single tokens), on v_mfma_f32_16x16x32_f16:
// every wave for itself, a span of blocks of 64 tokens at a time, the rows in its
// registers and the next block's keys on their way.  The first pass also leaves the scores
// where there is room for them (16 M), so that the second reads those and not the keys again:
// of 5 rows 20 bytes for 128.  64 sequences of 6,528 tokens, whose scores fit, take 144 us, of
// 6,656, whose do not, 185.  All blocks of a sequence are gone through, also those before a
// window: one token of 131,072, 40 heads over 8, 48 us with a window of 1,024 as without.
// 64 sequences of up to 4,096 tokens, 40 heads over 8 of 128:
// 24 us (91 MB of keys, 14 of scores, 4,400 GB/s) and 13, with the keys read twice 21
// and 22.  In 32 rows a tile, a block a wave at a time, both took 27.  Tile t of four takes
// token 16 g + 4 t + i as its row 4 g + i, so that a lane of group g = lane / 16 gets the
// scores of 16 neighbouring tokens, all of one page, for row lane % 16.
template <int D, WeighPass PASS, int RT>
__global__ __launch_bounds__(256, 4) void weigh_few_kernel(WeighArgs a) {
    constexpr std::integral_constant<WeighPass, kWeighSpanSums> pass;       // spans are the items both times
    constexpr int C = D / 64;
    constexpr bool kJoins = RT == 1;              // the rows' spans itself
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x + gridDim.x * (threadIdx.x >> 6));
    const size_t stride = static_cast<size_t>(a.c.page_tokens) * D;
    WeighSeq first;
    const WeighPlan plan(a, first, pass, std::true_type());
    if (PASS == kWeighSpanSums && wave == 0 && lane == 0) *a.span = plan.span;
    for (int x = wave; x < plan.total; x += a.workers) {
        const WeighItem w = plan.find(a, first, x, pass, std::true_type());
        const Span& s = w.q.s;
        const int* table = a.c.pages + static_cast<size_t>(w.seq) * a.c.max_pages;
        const int blocks_end = w.block + w.blocks;
        // the block's scores: a row after another, a token a lane
        auto scores_of = [&](int block) {
            return a.scores + (static_cast<size_t>(w.before) + static_cast<size_t>(w.head) * w.q.blocks + block) * a.score_rows * 64;
        };
        if (PASS == kWeighTokens && plan.keep) {
            // the rows' sums a lane each; eight rows' scores of a block at once, the first of the next on their way
            constexpr int kAhead = 8;
            const int rows = s.n * a.group, token = lane / a.group;
            float logs = INFINITY, z[kAhead];
            if (kJoins && rows > 0) logs = weigh_log(a, w, rows, WeighPlan::spans_of(a, w.q, plan.span));
            if (!kJoins && lane < rows) logs = a.logs[static_cast<size_t>(s.row0 + token) * a.q_heads + w.head * a.group + lane - token * a.group];
            auto load = [&](int block, int i0) {
                const float* p = scores_of(block) + lane;
#pragma unroll
                for (int j = 0; j < kAhead; ++j) z[j] = rows > 0 ? p[64 * min(i0 + j, rows - 1)] : -INFINITY;
            };
            load(w.block, 0);
            for (int block = w.block; block < blocks_end; ++block) {
                float sum = 0.f;
                for (int i0 = 0; i0 < max(rows, 1); i0 += kAhead) {
                    float now[kAhead];
#pragma unroll
                    for (int j = 0; j < kAhead; ++j) now[j] = z[j];
                    if (i0 + kAhead < rows) load(block, i0 + kAhead);
                    else if (block + 1 < blocks_end) load(block + 1, 0);
#pragma unroll
                    for (int j = 0; j < kAhead; ++j)      // of rows past the last L is infinite
                        sum += now[j] == -INFINITY ? 0.f : fast_exp2(now[j] - lane_of(logs, min(i0 + j, 63)));
                }
                weigh_write(a, w, block * 64 + lane, sum);
            }
            continue;
        }
        auto page_at = [&](int t) { return t < w.q.end ? table[t >> a.c.page_shift] : -1; };
        struct Keys {
            u32x4 raw[4][C];
            float scale;
            bool there;
        };
        auto load = [&](Keys& k, int t0, int pk, int ps) {
            const int tk = t0 + 16 * (r >> 2);
            pk = pk < 0 || pk >= a.c.num_pages ? 0 : pk;
            k.there = ps >= 0 && ps < a.c.num_pages;
            const int8_t* kp = a.c.k + (static_cast<size_t>(pk) * a.c.kv_heads + w.head) * stride +
                               ((tk & (a.c.page_tokens - 1)) + (r & 3)) * D + 16 * g;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < C; ++c) k.raw[t][c] = *reinterpret_cast<const u32x4*>(kp + 4 * t * D + 64 * c);
            k.scale = a.c.scales[2 * (static_cast<size_t>(k.there ? ps : 0) * a.c.kv_heads + w.head)];
        };
        Keys k;
        load(k, w.block * 64, page_at(w.block * 64 + 16 * (r >> 2)), page_at(w.block * 64 + 16 * g));
        f16x8 q[RT][D / 32];
        bool is[RT];
        size_t row[RT];
        int see_all[RT], see_begin[RT];
        float m[RT], l[RT], log[RT], logs = INFINITY;
        if (PASS == kWeighTokens && kJoins && s.n > 0) logs = weigh_log(a, w, s.n * a.group, WeighPlan::spans_of(a, w.q, plan.span));
#pragma unroll
        for (int n = 0; n < RT; ++n) {
            const int i = 16 * n + r, token = i / a.group, h = w.head * a.group + i - token * a.group;
            is[n] = token < s.n;
            row[n] = static_cast<size_t>(s.row0 + token) * a.q_heads + h;
            const int position = s.first + token;
            see_all[n] = is[n] ? position + 1 : 0;
            see_begin[n] = a.window > 0 ? max(0, max(position, 0) - a.window + 1) : 0;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                u32x4 v = {0, 0, 0, 0};
                if (is[n])
                    v = *reinterpret_cast<const u32x4*>(a.q + (s.row0 + token) * a.q_stride + h * D + 64 * (c / 2) + 16 * g + 8 * (c % 2));
                q[n][c] = query8(v, a.q_flip);
            }
            m[n] = kWeighNone;
            l[n] = 0.f;
            log[n] = INFINITY;
            if (PASS == kWeighTokens) {
                if (kJoins) log[n] = __shfl(logs, 16 * n + r, 64);
                else if (is[n]) log[n] = a.logs[row[n]];
            }
        }
        for (int block = w.block; block < blocks_end; ++block) {
            const int t0 = block * 64, mine = t0 + 16 * g;
            const bool more = block + 1 < blocks_end;
            int pk = -1, ps = -1;
            if (more) {
                pk = page_at(t0 + 64 + 16 * (r >> 2));
                ps = page_at(t0 + 64 + 16 * g);
            }
            f32x4 z[RT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int n = 0; n < RT; ++n) z[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const f16x8 k0 = to_half8(k.raw[t][c][0], k.raw[t][c][1]), k1 = to_half8(k.raw[t][c][2], k.raw[t][c][3]);
#pragma unroll
                    for (int n = 0; n < RT; ++n) {
                        z[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[n][2 * c], z[n][t], 0, 0, 0);
                        z[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[n][2 * c + 1], z[n][t], 0, 0, 0);
                    }
                }
            }
            const float unit = k.scale * a.scale;
            const bool there = k.there;
            if (more) load(k, t0 + 64, pk, ps);
            float total[16];
#pragma unroll
            for (int n = 0; n < RT; ++n) {
                // the lane's tokens that its row sees: e in [lo, lo + seen)
                const unsigned lo = static_cast<unsigned>(see_begin[n] - mine);
                const unsigned seen = there ? static_cast<unsigned>(max(min(see_all[n], w.q.end) - see_begin[n], 0)) : 0u;
                if constexpr (PASS == kWeighSpanSums) {
                    float top = m[n];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float v = z[n][e / 4][e % 4] * unit;
                        total[e] = static_cast<unsigned>(e) - lo >= seen ? -INFINITY : v;
                        top = fmaxf(top, total[e]);
                    }
                    top = over_groups(Larger(), top);
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += fast_exp2(total[e] - top);
                    if (plan.keep && is[n])
#pragma unroll
                        for (int e = 0; e < 16; e += 4)
                            *reinterpret_cast<f32x4*>(scores_of(block) + (16 * n + r) * 64 + 16 * g + e) =
                                f32x4{total[e], total[e + 1], total[e + 2], total[e + 3]};
                    l[n] = l[n] * fast_exp2(m[n] - top) + sum;      // of this lane's tokens
                    m[n] = top;
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float v = fast_exp2(__builtin_fmaf(z[n][e / 4][e % 4], unit, -log[n]));
                        v = static_cast<unsigned>(e) - lo >= seen ? 0.f : v;
                        total[e] = n ? total[e] + v : v;
                    }
                }
            }
            if constexpr (PASS == kWeighTokens) weigh_write(a, w, mine + r, weigh_scatter(total));
        }
        if constexpr (PASS == kWeighSpanSums) {
            const size_t span = w.block / WeighPlan::span_blocks(a, w.q, plan.span);
#pragma unroll
            for (int n = 0; n < RT; ++n) {
                const float sum = over_groups(Sum(), l[n]);
                if (is[n] && g == 0)
                    *reinterpret_cast<f32x2*>(a.spans + (span * a.rows * a.q_heads + row[n]) * 2) = f32x2{m[n], sum};
            }
        }
    }
}

// L of a row: a head a lane, the spans in turns over the waves
constexpr int kLogWaves = 4;
__global__ __launch_bounds__(kLogWaves * 64) void weigh_logs_kernel(WeighArgs a) {
    __shared__ f32x2 part[kLogWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x;
    const Place at = locate(a.starts, a.c.lens, a.rows, a.max_new, a.c.seqs, row, [](int start, int) { return start; });
    if (at.seq < 0 || row < at.s.row0 || row >= at.s.row0 + at.s.n) return;
    const int spans = WeighPlan::spans_of(a, WeighSeq(a, at.seq), *a.span);
    const size_t step = static_cast<size_t>(a.rows) * a.q_heads;
    for (int h0 = 0; h0 < a.q_heads; h0 += 64) {
        const int h = h0 + lane;
        const f32x2* p = reinterpret_cast<const f32x2*>(a.spans) + static_cast<size_t>(row) * a.q_heads + h;
        float m = kWeighNone, l = 0.f;
        if (h < a.q_heads)
#pragma unroll 4
            for (int i = wave; i < spans; i += kLogWaves) {
                const f32x2 x = p[i * step];
                const float n = fmaxf(m, x[0]);
                l = l * fast_exp2(m - n) + x[1] * fast_exp2(x[0] - n);
                m = n;
            }
        __syncthreads();
        part[wave][lane] = f32x2{m, l};
        __syncthreads();
        if (wave == 0 && h < a.q_heads) {
            for (int i = 1; i < kLogWaves; ++i) m = fmaxf(m, part[i][lane][0]);
            l = 0.f;
            for (int i = 0; i < kLogWaves; ++i) l += part[i][lane][1] * fast_exp2(part[i][lane][0] - m);
            a.logs[static_cast<size_t>(row) * a.q_heads + h] = l == 0.f ? INFINITY : m + __builtin_amdgcn_logf(l);
        }
    }
}

// blocks whose rows were several items': the parts, in their order
__global__ __launch_bounds__(256) void weigh_join_kernel(WeighArgs a) {
    constexpr std::integral_constant<WeighPass, kWeighJoin> pass;
    WeighSeq first;
    const WeighPlan plan(a, first, pass, std::false_type());
    for (int x = blockIdx.x; x < plan.total; x += a.workers) {
        const WeighItem w = plan.find(a, first, x, pass);
        const float* part = a.parts + static_cast<size_t>(w.slot) * kWeighBlock + threadIdx.x;
        float sum = 0.f;
#pragma unroll 4
        for (int i = 0; i < w.chunks; ++i) sum += part[i * kWeighBlock];
        weigh_write(a, w, w.block * kWeighBlock + threadIdx.x, sum);
    }
}

}  // namespace tetra_dev
