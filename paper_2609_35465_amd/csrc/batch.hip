// What a server does with a batch's cache and logits beside attention and
// sampling, for MI355X (gfx950): the weights of cached tokens, eviction by them,
// log probabilities.  The entry points of include/tetra.h: host code here
// validates arguments and launches the kernels of weigh.h, evict.h and score.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/tetra.h"
#include "evict.h"
#include "host.h"
#include "score.h"
#include "weigh.h"

using namespace tetra_host;

namespace {

constexpr size_t kMinWorkspace = 256;

size_t rounded(size_t bytes) { return std::max(kMinWorkspace, (bytes + 255) / 256 * 256); }

// a cache's sizes alone, as tetra_kv_cache limits them
bool sizes_ok(const tetra_kv_cache* c) {
    if (!c || c->num_pages < 1 || c->kv_heads < 1 || c->seqs < 1 || c->max_pages < 1) return false;
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return false;
    return c->max_pages <= kMaxTokens / c->page_tokens && (c->head_dim == 64 || c->head_dim == 128);
}

// As many as a CU holds by their registers.
constexpr int kWeighGroupsPerCU = 2, kWeighFewGroupsPerCU = 4;

// Sequences whose rows a wave holds in registers beside its keys: 16 of a cache head of 128, 32
// of one of 64.  Then the keys are what is read: 64 sequences of up to 4,096 tokens, 5 rows
// 37 us by weigh_few_kernel and 73 by weigh_kernel, whose rows go through LDS with a barrier; 16
// rows 22-41 and 30-73 by batch; heads of 64, 32 rows 14-43 and 16-62.  With heads of
// 128, 20 rows took 28 and 22 (8 sequences) to 62 and 73 (64), 32 rows 37 and 30 (16): the rule
// is for batches of up to some 32 sequences there and does not look at their count.
constexpr long long kWeighFew = 2048;
bool weigh_few(int max_new, int group, int head_dim) { return static_cast<long long>(max_new) * group * head_dim <= kWeighFew; }

// Places of kv_weigh's workspace, in floats, for up to `rows` rows: what full tables ask for.  A sequence that goes by
// weigh_few_kernel has few_rows rows at most; a batch of more rows than those, as where there are rows past the last
// start, has longer spans.  Lengths past the table make spans and chunks longer too, so nothing depends on the lengths.
struct WeighSpace {
    int few_spans, many_spans;      // of a sequence at most, in weigh_few_kernel and in weigh_kernel
    int items;                      // of weigh_kernel, whose parts there is room for
    size_t spans, logs, scores, bytes;
    WeighSpace(const tetra_kv_cache& c, int rows, int q_heads, int cus) {
        using namespace tetra_dev;
        const long long tokens = static_cast<long long>(c.max_pages) * c.page_tokens, group = q_heads / c.kv_heads;
        const long long few_blocks = (tokens + 63) / 64, blocks = (tokens + kWeighBlock - 1) / kWeighBlock;
        few_spans = static_cast<int>(std::min<long long>(kWeighSpans, few_blocks));
        many_spans = static_cast<int>(std::min<long long>(kWeighSpans / 4, blocks));
        const long long few_rows = std::min<long long>(rows, kWeighFew / (group * c.head_dim));
        const long long few = std::min<long long>(rows, few_rows * c.seqs);
        logs = (static_cast<size_t>(rows) * q_heads + 63) / 64 * 64;
        spans = std::max(2 * logs * many_spans, (2 * static_cast<size_t>(few) * q_heads * few_spans + 63) / 64 * 64);
        // and single tokens' scores, or prompts' parts: blocks of each sequence by row tiles of all
        const long long units = static_cast<long long>(c.seqs) * c.kv_heads, block_scores = 64 * few_rows * group;
        scores = 0;
        if (few_rows) scores = few_blocks > kWeighScores / block_scores / units ? kWeighScores : few_blocks * units * block_scores;
        const long long tiles = rows * group / kWeighRows + std::min(rows, c.seqs);
        const double steps = static_cast<double>(blocks) * c.kv_heads * static_cast<double>(tiles);
        items = static_cast<int>(std::min<double>(kWeighItems * kWeighGroupsPerCU * cus, steps));
        bytes = rounded(256 + sizeof(float) * (spans + logs + std::max(scores, 2 * static_cast<size_t>(items) * kWeighBlock)));
    }
    int spans_most(bool few, int rows, int q_heads) const {
        return static_cast<int>(std::min<size_t>(few ? few_spans : many_spans, spans / (2 * static_cast<size_t>(rows) * q_heads)));
    }
};

template <int D>
int weigh_launch(tetra_dev::WeighArgs& a, const WeighSpace& space, int cus, hipStream_t stream) {
    const bool few = weigh_few(a.max_new, a.group, D);
    const dim3 b(256), m(64 * tetra_dev::kWeighWaves), g(static_cast<unsigned>(cus * (few ? kWeighFewGroupsPerCU : kWeighGroupsPerCU)));
    a.workers = static_cast<int>(few ? 4 * g.x : g.x);
    a.block = few ? 64 : tetra_dev::kWeighBlock;
    a.spans_most = space.spans_most(few, a.rows, a.q_heads);
    a.items_most = space.items;
    a.scores_most = static_cast<long long>(space.scores);
    const bool two = D == 64 && static_cast<long long>(a.max_new) * a.group > 16;
#define TETRA_WEIGH_FEW(PASS) \
    if (two) hipLaunchKernelGGL((tetra_dev::weigh_few_kernel<D, PASS, D == 64 ? 2 : 1>), g, b, 0, stream, a); \
    else hipLaunchKernelGGL((tetra_dev::weigh_few_kernel<D, PASS, 1>), g, b, 0, stream, a)
    if (few) { TETRA_WEIGH_FEW(tetra_dev::kWeighSpanSums); }
    else hipLaunchKernelGGL((tetra_dev::weigh_kernel<D, tetra_dev::kWeighSpanSums>), g, m, 0, stream, a);
    if (!few || two)                  // one tile of rows is joined by the second pass
        hipLaunchKernelGGL(tetra_dev::weigh_logs_kernel, dim3(static_cast<unsigned>(a.rows)), dim3(64 * tetra_dev::kLogWaves), 0, stream, a);
    if (few) {
        TETRA_WEIGH_FEW(tetra_dev::kWeighTokens);
    } else {
        hipLaunchKernelGGL((tetra_dev::weigh_kernel<D, tetra_dev::kWeighTokens>), g, m, 0, stream, a);
        hipLaunchKernelGGL(tetra_dev::weigh_join_kernel, g, b, 0, stream, a);
    }
#undef TETRA_WEIGH_FEW
    return launch_status();
}

// Places of kv_evict's workspace.  A sequence and head whose weights a workgroup holds in
// registers is one workgroup's, in one launch; longer ones are cut in parts, two workgroups a
// CU in all, in four launches (8 heads of 131,072 tokens 32 us in place of 144; what the
// first form takes is 12.5 us for 512 units of up to 4,096).  The host does not know the
// lengths, so the table's width decides: 64 sequences of 300 tokens, 8 heads, cut to 150
// take 23 us with tables of up to 8,192 tokens and 48 with wider ones.
struct EvictSpace {
    int parts;            // 0: not cut
    size_t tokens, state, bytes;
    EvictSpace(const tetra_kv_cache* from, const tetra_kv_cache* to) {
        const size_t units = static_cast<size_t>(from->seqs) * from->kv_heads;
        parts = 0;
        if (static_cast<long long>(from->max_pages) * from->page_tokens > tetra_dev::kEvictHeld * tetra_dev::kEvictThreads)
            parts = static_cast<int>(std::max<size_t>(1, std::min<size_t>(tetra_dev::kEvictParts, 512 / units)));
        tokens = units * to->max_pages * to->page_tokens;
        state = (2 * units * (2 + parts) + 63) / 64 * 64;
        bytes = rounded(sizeof(int) * (tokens + state + 3 * units * parts * tetra_dev::kEvictBins));
    }
};

template <class T, bool TOP>
int score_launch(const tetra_dev::ScoreArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((tetra_dev::score_kernel<T, TOP>), dim3(static_cast<unsigned>(a.rows * a.parts)), dim3(256), 0, stream, a);
    if (a.parts > 1)
        hipLaunchKernelGGL((tetra_dev::score_join_kernel<T, TOP>), dim3(static_cast<unsigned>(a.rows)), dim3(256), 0, stream, a);
    return launch_status();
}

}  // namespace

extern "C" {

size_t tetra_kv_weigh_workspace_bytes(const tetra_kv_cache* cache, int rows, int q_heads) {
    int cus = 0;
    if (!sizes_ok(cache) || rows < 1 || q_heads < 1 || q_heads % cache->kv_heads || rows > kMaxGrid / q_heads || device_cus(&cus))
        return 0;
    return WeighSpace(*cache, rows, q_heads, cus).bytes;
}

int tetra_kv_weigh(const tetra_kv_cache* cache, const uint16_t* q, long long q_stride, const int* starts, int rows,
                   int max_new, int q_heads, float scale, int window, const float* mass, float* mass_out,
                   int mass_tokens, float decay, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    tetra_dev::WeighArgs a;
    if (int st = cache_of(cache, &a.c)) return st;
    if (!q || !starts || !mass_out || !workspace || rows < 1 || max_new < 1 || max_new > rows || window < 0) return TETRA_EINVAL;
    if (q_heads < 1 || q_heads % a.c.kv_heads || !std::isfinite(scale) || mass_tokens < 1) return TETRA_EINVAL;
    if (!(decay >= 0.f && decay <= 1.f)) return TETRA_EINVAL;
    if (q_stride < static_cast<long long>(q_heads) * cache->head_dim || rows > kMaxGrid / q_heads || rows > kMaxGroups)
        return TETRA_EINVAL;
    if (!aligned(q, 16) || q_stride % 8 || !aligned(starts, 4) || !aligned(mass, 4) || !aligned(mass_out, 4) ||
        !aligned(workspace, 256))
        return TETRA_EALIGN;
    // items of a launch are counted in an int: the blocks of all heads, and kWeighItems times the workgroups
    const long long tokens = std::max<long long>(static_cast<long long>(a.c.max_pages) << a.c.page_shift, mass_tokens);
    if ((tokens + 63) / 64 * a.c.kv_heads > (1 << 30) / a.c.seqs) return TETRA_EINVAL;
    int cus = 0;
    if (workspace_bytes < kMinWorkspace) return TETRA_EINVAL;
    if (int st = device_cus(&cus)) return st;
    const WeighSpace space(*cache, rows, q_heads, cus);
    if (workspace_bytes < space.bytes) return TETRA_EINVAL;
    a.q = q;
    a.starts = starts;
    a.mass = mass;
    a.out = mass_out;
    a.span = static_cast<int*>(workspace);
    a.spans = static_cast<float*>(workspace) + 64;
    a.logs = a.spans + space.spans;
    a.parts = a.scores = a.logs + space.logs;
    a.q_stride = q_stride;
    a.scale = std::fabs(scale) * 1.44269504f;
    a.q_flip = scale < 0.f ? 0x80008000u : 0u;
    a.decay = decay;
    a.rows = rows;
    a.max_new = max_new;
    a.q_heads = q_heads;
    a.group = q_heads / a.c.kv_heads;
    a.window = window;
    a.mass_tokens = mass_tokens;
    a.score_rows = static_cast<int>(std::min<long long>(static_cast<long long>(max_new) * a.group, tetra_dev::kWeighRows));
    return cache->head_dim == 64 ? weigh_launch<64>(a, space, cus, stream) : weigh_launch<128>(a, space, cus, stream);
}

size_t tetra_kv_evict_workspace_bytes(const tetra_kv_cache* from, const tetra_kv_cache* to) {
    if (!sizes_ok(from) || !sizes_ok(to)) return 0;
    return EvictSpace(from, to).bytes;
}

int tetra_kv_evict(const tetra_kv_cache* from, const tetra_kv_cache* to, const float* mass, int mass_tokens, int recent,
                   float* mass_out, int out_tokens, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    tetra_dev::EvictArgs a;
    if (int st = cache_of(from, &a.from)) return st;
    if (int st = cache_of(to, &a.to)) return st;
    if (from->kv_heads != to->kv_heads || from->head_dim != to->head_dim || from->page_tokens != to->page_tokens ||
        from->seqs != to->seqs)
        return TETRA_EINVAL;
    if (!mass || !workspace || mass_tokens < 1 || recent < 0 || (mass_out && out_tokens < 1) || mass_out == mass)
        return TETRA_EINVAL;
    if (!aligned(mass, 4) || !aligned(mass_out, 4) || !aligned(workspace, 256)) return TETRA_EALIGN;
    if (from->pages == to->pages && from->k == to->k) return TETRA_EINVAL;      // into the pages that it reads
    const EvictSpace space(from, to);
    if (workspace_bytes < space.bytes) return TETRA_EINVAL;
    const long long units = static_cast<long long>(a.from.seqs) * a.from.kv_heads;
    const long long moves = 2 * (to->page_tokens / tetra_dev::kGroupTokens);         // waves of a page and head
    if (units > kMaxGrid / 16 / a.to.max_pages || (units * a.to.max_pages * moves + 3) / 4 > kMaxGroups) return TETRA_EINVAL;
    if (units * std::max(space.parts, 1) > kMaxGroups * 256 / tetra_dev::kEvictThreads) return TETRA_EINVAL;
    a.mass = mass;
    a.out = mass_out;
    a.tokens = static_cast<int*>(workspace);
    a.capacity = to->max_pages * to->page_tokens;
    a.mass_tokens = mass_tokens;
    a.out_tokens = out_tokens;
    a.recent = recent;
    a.state = a.tokens + space.tokens;
    a.bins = reinterpret_cast<unsigned*>(a.state + space.state);
    a.parts = space.parts;
    const dim3 u(static_cast<unsigned>(units)), t(tetra_dev::kEvictThreads);
    if (space.parts == 0) {
        hipLaunchKernelGGL(tetra_dev::evict_choose_kernel, u, t, 0, stream, a);
    } else {
        const dim3 p(static_cast<unsigned>(units * space.parts));
        hipLaunchKernelGGL(tetra_dev::evict_part_kernel<0>, p, t, 0, stream, a);
        hipLaunchKernelGGL(tetra_dev::evict_part_kernel<1>, p, t, 0, stream, a);
        hipLaunchKernelGGL(tetra_dev::evict_part_kernel<2>, p, t, 0, stream, a);
        hipLaunchKernelGGL(tetra_dev::evict_part_kernel<3>, p, t, 0, stream, a);
    }
    const dim3 g(static_cast<unsigned>((units * a.to.max_pages * moves + 3) / 4)), m(256);
    if (from->head_dim == 64) hipLaunchKernelGGL((tetra_dev::evict_move_kernel<64>), g, m, 0, stream, a);
    else hipLaunchKernelGGL((tetra_dev::evict_move_kernel<128>), g, m, 0, stream, a);
    return launch_status();
}

size_t tetra_log_probs_workspace_bytes(int rows, int vocab, int top) {
    int cus = 0;
    if (rows < 1 || vocab < 1 || vocab > kMaxVocab || top < 0 || top > tetra_dev::kMostTop || device_cus(&cus)) return 0;
    return rounded(tetra_dev::score_entries(rows, vocab, cus) * (16 + 8 * static_cast<size_t>(top)));
}

int tetra_log_probs(const void* logits, int half, long long stride, int rows, int vocab, const float* temperature,
                    const int* tokens, int given, float* out, float* entropy, int top, int* top_tokens, float* top_out,
                    void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!logits || !workspace || (half != 0 && half != 1) || rows < 1 || vocab < 1 || vocab > kMaxVocab || stride < vocab)
        return TETRA_EINVAL;
    if (given < 0 || top < 0 || top > tetra_dev::kMostTop || rows > kMaxGroups) return TETRA_EINVAL;
    if ((given && (!tokens || !out)) || (top && (!top_tokens || !top_out))) return TETRA_EINVAL;
    if (!given && !top && !entropy) return TETRA_EINVAL;
    if (!aligned(logits, half ? 2 : 4) || !aligned(temperature, 4) || !aligned(tokens, 4) || !aligned(out, 4) ||
        !aligned(entropy, 4) || !aligned(top_tokens, 4) || !aligned(top_out, 4) || !aligned(workspace, 256))
        return TETRA_EALIGN;
    int cus = 0;
    if (workspace_bytes < kMinWorkspace) return TETRA_EINVAL;
    if (int st = device_cus(&cus)) return st;
    if (workspace_bytes < tetra_log_probs_workspace_bytes(rows, vocab, top)) return TETRA_EINVAL;
    tetra_dev::ScoreArgs a;
    a.logits = logits;
    a.stride = stride;
    a.temperature = temperature;
    a.tokens = tokens;
    a.out = out;
    a.entropy = entropy;
    a.top_out = top_out;
    a.top_tokens = top_tokens;
    a.rows = rows;
    a.vocab = vocab;
    a.given = given;
    a.top = top;
    const tetra_dev::ScoreShape shape = tetra_dev::score_shape(rows, vocab, cus);
    a.parts = shape.parts;
    a.part = shape.part;
    a.sums = static_cast<float*>(workspace);
    a.places = reinterpret_cast<uint64_t*>(a.sums + 4 * static_cast<size_t>(rows) * shape.parts);
    if (half) return top ? score_launch<_Float16, true>(a, stream) : score_launch<_Float16, false>(a, stream);
    return top ? score_launch<float, true>(a, stream) : score_launch<float, false>(a, stream);
}

}  // extern "C"
