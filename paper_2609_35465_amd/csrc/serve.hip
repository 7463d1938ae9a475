// The serving operators around the projections for MI355X (gfx950): the paged
// 8-bit cache of keys and values, the attention over it and sampling.  The
// entry points of include/tetra.h: host code here validates arguments and
// launches the kernels of kv_cache.h, attend.h and sample.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/tetra.h"
#include "attend.h"
#include "host.h"
#include "kv_cache.h"
#include "sample.h"
#include "shared.h"

namespace {

using namespace tetra_host;

constexpr int kFewGroupsPerCU = 2;
constexpr size_t kMinAttendWorkspace = 4096;

// the parts of attend_few's workgroups, and behind them the pieces of the
// many-row units
size_t few_parts(int cus) { return static_cast<size_t>(cus) * kFewGroupsPerCU * 2 * tetra_dev::kFewSlot<128>; }
size_t attend_workspace(int cus) {
    return ((few_parts(cus) + 2 * static_cast<size_t>(cus) * tetra_dev::kManySlot<128, 4>) * sizeof(float) + 255) / 256 * 256;
}


// How a call of tetra_kv_attend is spread; the lengths, and with them the
// pieces, are the device's own matter.
struct AttendPlan {
    long long few_grid = 0, join_grid = 0;            // attend_few_kernel, 0: none
    int row_tiles = 0, spans = 0, span = 1;           // of a sequence in it: row tiles; the join's rows a workgroup
    long long many_grid = 0, many_join_grid = 0;      // attend_many_kernel, 0: none
    int waves = 0, teams = 0;                         // of its workgroups
    int slots = 0;                                    // workgroups at once, 0: units are not cut
};

template <int D>
AttendPlan attend_plan(tetra_dev::AttendArgs& a, int cus) {
    AttendPlan p;
    a.few_tile = 256;
    const long long kept = static_cast<long long>(a.c.max_pages) << a.c.page_shift;
    const long long reach = a.window > 0 ? std::min<long long>(kept, static_cast<long long>(a.window) + a.max_new + 64) : kept;
    const long long tiles = (reach + a.few_tile - 1) / a.few_tile;
    const long long most = static_cast<long long>(a.max_new) * a.group;      // rows of a sequence
    const long long most_tiles = (most + tetra_dev::kFewRows - 1) / tetra_dev::kFewRows;
    const long long few_groups = static_cast<long long>(cus) * kFewGroupsPerCU;
    // attend_few_kernel reads the keys once for 16 rows.  Up to there it is ahead (64 sequences of 1,000 tokens, 8
    // heads by 16 rows: 33 us against 59); with several row tiles only where few sequences leave the other kernel
    // short of units (32 rows: 1 sequence of 4,096 13 us against 22, 8 of them 33 and 33, 32 of 1,000 31 and 27;
    // 64 rows: 16 and 23, 51 and 35, 52 and 29).  Of contexts that one tile holds it also takes prompts whose row
    // tiles are one round of the chip: one short loop and no join (203 tokens of 40 heads over 8 of 128 9.8 us against
    // 15.7, 64 tokens 6.7 and 12.7, 8 times 20 after 183 11 and 15, 8 times 64 of 16 heads of 64 6.1 and 9.0).  What a
    // context may be is told by the table's width, for the host does not know the lengths.
    const int few_rows = static_cast<int>(std::min<long long>(64, std::max<long long>(16, 2048 / (static_cast<long long>(a.c.seqs) * a.c.kv_heads))));
    const bool all_few = most <= few_rows || (tiles == 1 && most_tiles * a.c.kv_heads * a.c.seqs <= few_groups);
    a.few_most = static_cast<int>(all_few ? most : few_rows);
    if (!all_few) {
        // sequences of the most rows that the rows would make, and their units
        const long long full = (a.rows + a.max_new - 1) / a.max_new;
        const long long units4 = full * ((most + 127) / 128) * a.c.kv_heads;
        // Where every sequence fills max_new rows there are no few-row sequences; should `starts` end before the last
        // row after all, attend_many_kernel takes what there is.
        const bool mixed = static_cast<long long>(a.c.seqs) * a.max_new != a.rows;
        if (!mixed) a.few_most = 0;
        // Three forms of the workgroup.  128 rows with two teams for the keys, so that a CU has eight waves for few rows,
        // where they are one round of the chip, or two rounds of long prompts from the start, whose short units even out.
        // 256 rows for more: a tile is turned into fp16 for twice as many.  Of batches that may have few-row sequences,
        // 128 rows with one team up to two rounds, since those run beside it.  Measured (128 rows with one team, with two,
        // 256 rows; heads of 128, us): 1,024 tokens of 32 heads 34, 29, 41; 2,048 68, 61, 72; 2,800 93, 105, 95; 8 x 203
        // tokens of 40 heads after 1,797 85, 92, 79; 2 x 500 of 32 from the start 22, 20, 25.
        p.waves = 8;
        if (mixed ? units4 <= 2 * cus : units4 <= cus || (units4 <= 2 * cus && a.max_new >= 1024)) p.waves = 4;
        p.teams = p.waves == 4 && !mixed ? 2 : 1;
        const int at_once = p.waves * p.teams == 4 ? 2 * cus : cus;
        const long long rows = 32 * p.waves, all = static_cast<long long>(a.rows) * a.group;
        const long long sequences = std::min<long long>(a.c.seqs, all / (a.few_most + 1));
        const long long units = (all / rows + sequences) * a.c.kv_heads;     // at most
        p.many_grid = std::max<long long>(units, at_once);
        // the device may cut units of 128 rows if it would at the fewest units and the most keys
        const int least = static_cast<int>(std::min<long long>(std::max<long long>(all / rows, 1) * a.c.kv_heads, kMaxGrid));
        const int longest = static_cast<int>((reach + tetra_dev::kManyTile - 1) / tetra_dev::kManyTile);
        if (p.waves == 4 && (p.teams == 2 ? tetra_dev::many_splits<D, 4, 2>(least, longest, at_once)
                                          : tetra_dev::many_splits<D, 4, 1>(least, longest, at_once)) > 1) {
            p.slots = at_once;
            p.many_join_grid = std::min<long long>(units, at_once / 2) * (rows / tetra_dev::kJoinRows<D>);
        }
        if (!mixed) return p;
    }
    p.row_tiles = (a.few_most + tetra_dev::kFewRows - 1) / tetra_dev::kFewRows;
    // in workgroups of the size of attend_many_kernel's, which they run beside
    p.few_grid = p.waves == 8 ? cus : few_groups;
    a.few_tile = p.waves == 8 ? 512 : 256;
    const long long units = static_cast<long long>(p.row_tiles) * a.c.kv_heads * a.c.seqs;
    if (units > kMaxGrid / tiles) p.few_grid = kMaxGrid + 1;
    if (tiles > 1) {
        // a row a workgroup where that is few of them, and the parts may be many
        const int rows_most = std::min(a.few_most, tetra_dev::kFewRows);
        while (p.span < 8 && p.span < rows_most && units * rows_most > 2 * p.span * cus) p.span *= 2;
        p.spans = (rows_most + p.span - 1) / p.span;
        p.join_grid = units * p.spans;
    }
    return p;
}

template <int D, int NW, int KS>
void attend_many_launch(const tetra_dev::AttendArgs& a, const AttendPlan& p, hipStream_t stream) {
    const dim3 g(static_cast<unsigned>(p.many_grid + p.few_grid)), b(64 * NW * KS);
    const int blocks = static_cast<int>(p.many_grid), few = static_cast<int>(p.few_grid);
    if (a.c.page_tokens >= tetra_dev::kManyTile)
        hipLaunchKernelGGL((tetra_dev::attend_many_kernel<D, NW, KS, true>), g, b, 0, stream, a, p.slots, blocks, few);
    else
        hipLaunchKernelGGL((tetra_dev::attend_many_kernel<D, NW, KS, false>), g, b, 0, stream, a, p.slots, blocks, few);
}

template <int D>
int attend_launch(tetra_dev::AttendArgs& a, int cus, hipStream_t stream) {
    const AttendPlan p = attend_plan<D>(a, cus);
    if (p.few_grid > kMaxGrid || p.many_grid + p.few_grid > kMaxGrid || p.many_join_grid + p.join_grid > kMaxGrid)
        return TETRA_EINVAL;
    if (p.waves == 8) attend_many_launch<D, 8, 1>(a, p, stream);
    else if (p.teams == 2) attend_many_launch<D, 4, 2>(a, p, stream);
    else if (p.teams == 1) attend_many_launch<D, 4, 1>(a, p, stream);
    else hipLaunchKernelGGL((tetra_dev::attend_few_kernel<D>), dim3(static_cast<unsigned>(p.few_grid)), dim3(256), 0, stream, a);
    if (int st = launch_status()) return st;
    const tetra_dev::JoinShape shape{static_cast<int>(p.few_grid), p.row_tiles, p.spans, p.span};
    const int blocks = static_cast<int>(p.many_join_grid);
    const dim3 g(static_cast<unsigned>(p.many_join_grid + p.join_grid));
    if (blocks && p.teams == 1)
        hipLaunchKernelGGL((tetra_dev::attend_join_many_kernel<D, 4, 1>), g, dim3(256), 0, stream, a, p.slots, blocks, shape);
    else if (blocks)
        hipLaunchKernelGGL((tetra_dev::attend_join_many_kernel<D, 4, 2>), g, dim3(256), 0, stream, a, p.slots, blocks, shape);
    else if (p.join_grid)
        hipLaunchKernelGGL((tetra_dev::attend_join_kernel<D>), g, dim3(256), 0, stream, a, shape);
    return launch_status();
}

// the arguments of tetra_kv_attend, checked
int attend_args(const tetra_kv_cache* cache, const uint16_t* q, long long q_stride, const int* starts, int rows,
                int max_new, int q_heads, float scale, int window, uint16_t* out, long long out_stride,
                void* workspace, size_t workspace_bytes, tetra_dev::AttendArgs& a) {
    if (int st = cache_of(cache, &a.c)) return st;
    if (!q || !starts || !out || !workspace || rows < 1 || max_new < 1 || max_new > rows || window < 0) return TETRA_EINVAL;
    if (q_heads < 1 || q_heads % a.c.kv_heads || !std::isfinite(scale)) return TETRA_EINVAL;
    const long long width = static_cast<long long>(q_heads) * cache->head_dim;
    if (q_stride < width || out_stride < width || rows > kMaxGrid / q_heads) return TETRA_EINVAL;
    if (!aligned(q, 16) || !aligned(out, 16) || q_stride % 8 || out_stride % 8 || !aligned(starts, 4) ||
        !aligned(workspace, 256))
        return TETRA_EALIGN;
    if (workspace_bytes < kMinAttendWorkspace) return TETRA_EINVAL;
    a.q = q;
    a.starts = starts;
    a.out = out;
    a.partials = static_cast<float*>(workspace);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.scale = std::fabs(scale) * 1.44269504f;
    a.q_flip = scale < 0.f ? 0x80008000u : 0u;
    a.rows = rows;
    a.max_new = max_new;
    a.q_heads = q_heads;
    a.group = q_heads / a.c.kv_heads;
    a.window = window;
    return TETRA_OK;
}

// the device's part of them
int attend_device(tetra_dev::AttendArgs& a, size_t workspace_bytes, int& cus) {
    if (int st = device_cus(&cus)) return st;
    if (workspace_bytes < attend_workspace(cus)) return TETRA_EINVAL;
    a.pieces = a.partials + few_parts(cus);
    return TETRA_OK;
}

// What a call with shared prefixes may be to go by its groups: rows of a sequence and cache
// head, rows times q heads, groups and sequences, and these times cache heads (at most 8
// workgroups of the join for each).  The first is what was measured to pay, the others are
// what the workspace holds, whose size does not depend on the call: 1,600 sequences of 1,044
// tokens with 1,024 in common, 40 heads over 8 of 128, take 280 us by groups and 472 by
// kv_attend, 1,700 go by kv_attend and take 507.
constexpr int kSharedMost = 64, kSharedRows = 65536, kSharedList = 131072, kSharedHeads = 1 << 20;

// bytes of kv_attend_shared's workspace, behind those of kv_attend
struct SharedSpace {
    size_t list, group, results, stats, bytes;
    explicit SharedSpace(int cus) {
        list = attend_workspace(cus);
        group = list + sizeof(tetra_dev::SharedSeq) * kSharedList;
        results = group + sizeof(tetra_dev::SharedGroup) * kSharedList;
        stats = results + 2 * sizeof(float) * 128 * kSharedRows;
        bytes = stats + 4 * sizeof(float) * kSharedRows;
    }
};

// Whether a call goes by its groups.  That takes two launches more and the sums' way through
// memory, some 14 us, and saves what kv_attend reads of keys and values more than once: of
// pages that sequences share it has much from the caches.  What it may read is told by the
// table's width, for the host does not know the lengths, and it reads it for each 16 rows
// of a sequence.  So short sequences in wide tables take the four launches: 4 sequences of
// 1,056 tokens 15.7 us with tables of 20,480 tokens and more, 10.7 by kv_attend.  Measured (40 heads over 8 of 128, us by groups and by kv_attend): 8
// sequences of 4,196 tokens (69 MB) 28 and 22, 64 of 1,124 (151 MB) 29 and 27, 12 of 8,292
// (204 MB) 33 and 39, 64 of 4,196 in 8 groups (554 MB) 43 and 56, with four rows each in one
// group 64 and 179.
constexpr long long kSharedBytes = 160ll << 20;

bool shared_pays(const tetra_dev::AttendArgs& a, int num_groups, int dim) {
    const long long most = static_cast<long long>(a.max_new) * a.group, seqs = static_cast<long long>(num_groups) + a.c.seqs;
    if (most > kSharedMost || a.rows > kSharedRows / a.q_heads || seqs > kSharedList) return false;
    if (seqs > kSharedHeads / a.c.kv_heads) return false;
    const double tokens = static_cast<double>(static_cast<long long>(a.c.max_pages) << a.c.page_shift) * a.c.seqs;
    const long long tiles = (most + tetra_dev::kFewRows - 1) / tetra_dev::kFewRows;
    return tokens * a.c.kv_heads * 2 * dim * tiles >= kSharedBytes;
}

// Groups of up to 32 rows of a cache head go 16 rows at a time, like the sequences' own
// tokens, others 128 at a time (groups of 20 rows over 8,192 tokens 27 us so and 29 by 128;
// of 40 rows 28 by 128 and 25 so, but over 32,768 51 and 58).  The latter fill one and a
// half workgroups a CU, so that the former begin beside them: 64 sequences of 32 heads with
// 32,768 tokens in common 74 us, two workgroups a CU 83, one 77.
constexpr int kSharedFew = 32;

int shared_few(const tetra_dev::AttendArgs& a) { return std::max(a.max_new * a.group, kSharedFew); }
constexpr int kSharedTile = 256;

// Tiles of attend_few where groups and sequences all fill the table: the device counts them in an int.
double shared_tiles(const tetra_dev::AttendArgs& a, int num_groups) {
    auto row_tiles = [](int rows) { return (rows + tetra_dev::kFewRows - 1) / tetra_dev::kFewRows; };
    const double units = static_cast<double>(num_groups) * row_tiles(shared_few(a)) +
                         static_cast<double>(a.c.seqs) * row_tiles(a.max_new * a.group);
    const long long kept = static_cast<long long>(a.c.max_pages) << a.c.page_shift;
    return units * a.c.kv_heads * static_cast<double>((kept + kSharedTile - 1) / kSharedTile);
}

template <int D>
int shared_launch(tetra_dev::SharedArgs& x, int cus, hipStream_t stream) {
    tetra_dev::AttendArgs& a = x.a;
    const int slots = cus + cus / 2, few = kFewGroupsPerCU * cus;
    a.few_most = shared_few(a);
    a.few_tile = kSharedTile;
    const long long all = static_cast<long long>(a.rows) * a.group;
    const long long units = (all / 128 + std::min<long long>(x.num_groups, all / (a.few_most + 1))) * a.c.kv_heads;   // at most
    const long long blocks = units ? std::max<long long>(units, slots) : 0;
    const long long join_many = std::min<long long>(units, slots / 2) * (128 / tetra_dev::kJoinRows<D>);
    tetra_dev::JoinShape shape{few, (a.few_most + tetra_dev::kFewRows - 1) / tetra_dev::kFewRows, 1, 1};
    const long long few_units = static_cast<long long>(shape.row_tiles_most) * a.c.kv_heads * a.num_seqs;
    while (shape.span < 8 && few_units * tetra_dev::kFewRows > 2ll * shape.span * cus) shape.span *= 2;
    shape.spans = tetra_dev::kFewRows / shape.span;
    const long long join = join_many + few_units * shape.spans;
    const long long last = static_cast<long long>(a.rows) * ((a.q_heads + 1024 / D - 1) / (1024 / D));
    if (blocks + few > kMaxGrid || join > kMaxGrid || last > kMaxGrid) return TETRA_EINVAL;
    hipLaunchKernelGGL(tetra_dev::shared_list_kernel, dim3(1), dim3(tetra_dev::kListThreads), 0, stream, x);
    const dim3 g(static_cast<unsigned>(blocks + few)), b(256);
    const int many = static_cast<int>(blocks);
    if (a.c.page_tokens >= tetra_dev::kManyTile)
        hipLaunchKernelGGL((tetra_dev::attend_many_kernel<D, 4, 1, true, true>), g, b, 0, stream, a, slots, many, few);
    else
        hipLaunchKernelGGL((tetra_dev::attend_many_kernel<D, 4, 1, false, true>), g, b, 0, stream, a, slots, many, few);
    hipLaunchKernelGGL((tetra_dev::attend_join_many_kernel<D, 4, 1, true>), dim3(static_cast<unsigned>(join)), b, 0, stream, a, slots,
                       static_cast<int>(join_many), shape);
    hipLaunchKernelGGL((tetra_dev::shared_join_kernel<D>), dim3(static_cast<unsigned>(last)), b, 0, stream, x);
    return launch_status();
}

int append(const tetra_kv_cache* cache, const tetra_kv_input* in, const int* starts, const int* shifts, int rows, int max_new,
           hipStream_t stream) {
    tetra_dev::AppendArgs a;
    if (int st = cache_of(cache, &a.c)) return st;
    if (!in || !in->k || !in->v || !starts || rows < 1 || max_new < 1 || max_new > rows) return TETRA_EINVAL;
    if (!in->q != !in->q_out || (in->q && in->q_heads < 1)) return TETRA_EINVAL;
    if ((in->half != 0 && in->half != 1) || (in->rope && in->rope_rows < 1)) return TETRA_EINVAL;
    if (!(in->eps >= 0.f) || std::isinf(in->eps)) return TETRA_EINVAL;
    const int D = cache->head_dim;
    const long long kv_width = static_cast<long long>(a.c.kv_heads) * D, q_width = static_cast<long long>(in->q_heads) * D;
    if (in->k_stride < kv_width || in->v_stride < kv_width || (in->q && in->q_stride < q_width)) return TETRA_EINVAL;
    if (!aligned(in->k, 16) || !aligned(in->v, 16) || in->k_stride % 8 || in->v_stride % 8 || !aligned(starts, 4) ||
        (in->q && (!aligned(in->q, 16) || in->q_stride % 8 || !aligned(in->q_out, 16))) || !aligned(in->q_norm, 16) ||
        !aligned(in->k_norm, 16) || !aligned(in->rope, 16) || !aligned(shifts, 4))
        return TETRA_EALIGN;
    a.q = in->q;
    a.k = in->k;
    a.v = in->v;
    a.q_stride = in->q_stride;
    a.k_stride = in->k_stride;
    a.v_stride = in->v_stride;
    a.q_norm = in->q_norm;
    a.k_norm = in->k_norm;
    a.rope = in->rope;
    a.starts = starts;
    a.shifts = shifts;
    a.q_out = in->q_out;
    a.eps = in->eps;
    a.rope_rows = in->rope_rows;
    a.rows = rows;
    a.max_new = max_new;
    a.q_heads = in->q ? in->q_heads : 0;
    const int waves = a.c.page_tokens / tetra_dev::kGroupTokens;
    const long long items =
        max_new == 1 ? a.c.seqs : ((rows + ((1ll << a.c.page_shift) - 2) * a.c.seqs) >> a.c.page_shift) + a.c.seqs;
    const long long kv_blocks = items * a.c.kv_heads * 2;
    // 16 heads of a row per wave where that still leaves waves enough, so that a
    // lane's part of the rotation table is read once for several heads
    a.q_chunk = static_cast<long long>(rows) * a.q_heads >= 65536 ? 16 : 512 / D;
    const long long q_units = a.q_heads ? static_cast<long long>(rows) * ((a.q_heads + a.q_chunk - 1) / a.q_chunk) : 0;
    const long long grid = kv_blocks + (q_units + waves - 1) / waves;
    if (kv_blocks > kMaxGrid || q_units > kMaxGrid - 8 || grid > kMaxGrid) return TETRA_EINVAL;
    a.items = static_cast<int>(items);
    const dim3 g(static_cast<unsigned>(grid)), b(static_cast<unsigned>(waves * 64));
#define TETRA_APPEND(D_, H) hipLaunchKernelGGL((tetra_dev::append_kernel<D_, H>), g, b, 0, stream, a)
    if (D == 64) {
        if (in->half) TETRA_APPEND(64, true);
        else TETRA_APPEND(64, false);
    } else {
        if (in->half) TETRA_APPEND(128, true);
        else TETRA_APPEND(128, false);
    }
#undef TETRA_APPEND
    return launch_status();
}

}  // namespace

extern "C" {

int tetra_kv_append(const tetra_kv_cache* cache, const tetra_kv_input* in, const int* starts, int rows, int max_new,
                    hipStream_t stream) {
    return append(cache, in, starts, nullptr, rows, max_new, stream);
}

int tetra_kv_append_at(const tetra_kv_cache* cache, const tetra_kv_input* in, const int* starts, const int* shifts,
                       int rows, int max_new, hipStream_t stream) {
    if (!shifts) return TETRA_EINVAL;
    return append(cache, in, starts, shifts, rows, max_new, stream);
}

int tetra_kv_read(const tetra_kv_cache* cache, int count, uint16_t* k_out, uint16_t* v_out, hipStream_t stream) {
    tetra_dev::KvCache c;
    if (int st = cache_of(cache, &c)) return st;
    if (count < 1 || !k_out || !v_out) return TETRA_EINVAL;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return TETRA_EALIGN;
    // groups of 16 tokens that `count` tokens can touch
    const int groups = count / tetra_dev::kGroupTokens + 2;
    const long long grid = static_cast<long long>(groups) * c.seqs;
    if (grid > kMaxGrid / c.kv_heads) return TETRA_EINVAL;
    const dim3 g(static_cast<unsigned>(grid * c.kv_heads));
    if (cache->head_dim == 64)
        hipLaunchKernelGGL((tetra_dev::kv_read_kernel<64>), g, dim3(128), 0, stream, c, count, groups, k_out, v_out);
    else
        hipLaunchKernelGGL((tetra_dev::kv_read_kernel<128>), g, dim3(256), 0, stream, c, count, groups, k_out, v_out);
    return launch_status();
}

size_t tetra_kv_attend_workspace_bytes(void) {
    int cus = 0;
    if (device_cus(&cus)) return 0;
    return attend_workspace(cus);
}

int tetra_kv_attend(const tetra_kv_cache* cache, const uint16_t* q, long long q_stride, const int* starts, int rows,
                    int max_new, int q_heads, float scale, int window, uint16_t* out, long long out_stride,
                    void* workspace, size_t workspace_bytes, hipStream_t stream) {
    tetra_dev::AttendArgs a;
    int cus = 0;
    if (int st = attend_args(cache, q, q_stride, starts, rows, max_new, q_heads, scale, window, out, out_stride, workspace,
                             workspace_bytes, a))
        return st;
    if (int st = attend_device(a, workspace_bytes, cus)) return st;
    return cache->head_dim == 64 ? attend_launch<64>(a, cus, stream) : attend_launch<128>(a, cus, stream);
}

size_t tetra_kv_attend_shared_workspace_bytes(void) {
    int cus = 0;
    if (device_cus(&cus)) return 0;
    return SharedSpace(cus).bytes;
}

int tetra_kv_attend_shared(const tetra_kv_cache* cache, const uint16_t* q, long long q_stride, const int* starts, int rows,
                           int max_new, int q_heads, float scale, const int* groups, const int* shared, int num_groups,
                           uint16_t* out, long long out_stride, void* workspace, size_t workspace_bytes,
                           hipStream_t stream) {
    tetra_dev::SharedArgs x;
    int cus = 0;
    if (cache && (!groups || !shared || num_groups < 1 || num_groups > cache->seqs)) return TETRA_EINVAL;
    if (!aligned(groups, 4) || !aligned(shared, 4)) return TETRA_EALIGN;
    if (int st = attend_args(cache, q, q_stride, starts, rows, max_new, q_heads, scale, 0, out, out_stride, workspace,
                             workspace_bytes, x.a))
        return st;
    const bool pays = shared_pays(x.a, num_groups, cache->head_dim);
    if (pays && shared_tiles(x.a, num_groups) > kMaxGrid) return TETRA_EINVAL;
    if (int st = attend_device(x.a, workspace_bytes, cus)) return st;
    const SharedSpace space(cus);
    if (workspace_bytes < space.bytes) return TETRA_EINVAL;
    x.groups = groups;
    x.shared = shared;
    x.num_groups = num_groups;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    x.list = reinterpret_cast<tetra_dev::SharedSeq*>(at + space.list);
    x.group = reinterpret_cast<tetra_dev::SharedGroup*>(at + space.group);
    x.a.seqs = x.list;
    x.a.results = reinterpret_cast<float*>(at + space.results);
    x.a.stats = reinterpret_cast<float*>(at + space.stats);
    if (!pays)
        return cache->head_dim == 64 ? attend_launch<64>(x.a, cus, stream) : attend_launch<128>(x.a, cus, stream);
    x.a.num_seqs = num_groups + cache->seqs;
    return cache->head_dim == 64 ? shared_launch<64>(x, cus, stream) : shared_launch<128>(x, cus, stream);
}

size_t tetra_sample_workspace_bytes(int rows, int vocab) {
    if (rows < 1 || vocab < 1 || vocab > kMaxVocab) return 0;
    return static_cast<size_t>(rows) * tetra_dev::sample_row_space(vocab);
}

int tetra_sample(const float* logits, long long stride, int rows, int vocab, const float* temperature,
                 const int* top_k, const float* top_p, const float* min_p, const float* u, int* tokens,
                 void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!logits || !temperature || !top_k || !top_p || !min_p || !u || !tokens || !workspace) return TETRA_EINVAL;
    if (rows < 1 || vocab < 1 || vocab > kMaxVocab || stride < vocab) return TETRA_EINVAL;
    if (workspace_bytes < tetra_sample_workspace_bytes(rows, vocab)) return TETRA_EINVAL;
    if (!aligned(logits, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
        !aligned(min_p, 4) || !aligned(u, 4) || !aligned(tokens, 4) || !aligned(workspace, 256))
        return TETRA_EALIGN;
    tetra_dev::SampleArgs a;
    a.logits = logits;
    a.stride = stride;
    a.temperature = temperature;
    a.top_p = top_p;
    a.min_p = min_p;
    a.u = u;
    a.top_k = top_k;
    a.tokens = tokens;
    a.space = static_cast<uint8_t*>(workspace);
    a.row_space = tetra_dev::sample_row_space(vocab);
    a.rows = rows;
    a.vocab = vocab;
    a.tiles = (vocab + tetra_dev::kSampleTile - 1) / tetra_dev::kSampleTile;
    // A tile a wave where the chip has the room: two workgroups a CU over all rows, or up to 16 a row and four a CU.
    // More of them take longer over the bins, which each adds to the row's (top-p 0.9 of 151,936: 16 rows 33 us in 32
    // parts each, 40 in 64; 32 rows 44 in 16, 49 in 32; without a filter one row 12 us in 75, 16 in 16).
    int cus = 0;
    if (int st = device_cus(&cus)) return st;
    a.parts = std::max(1, std::min({(a.tiles + 3) / 4, std::max(2 * cus / rows, std::min(16, 4 * cus / rows)),
                                    tetra_dev::kMostParts}));
    a.wave_groups = a.parts * 4 * 16 <= tetra_dev::kMostGroups ? 16 : 4;
    a.groups = a.parts * 4 * a.wave_groups;
    if (static_cast<long long>(rows) * a.parts > kMaxGrid) return TETRA_EINVAL;
    const dim3 g(static_cast<unsigned>(rows * a.parts)), b(256);
    hipLaunchKernelGGL(tetra_dev::sample_max_kernel, g, b, 0, stream, a);
    hipLaunchKernelGGL(tetra_dev::sample_cut_kernel, g, b, 0, stream, a);
    // few rows go by bins, and each of their parts has the more to do
    const int bins_parts = std::min((a.tiles + 3) / 4, 2 * a.parts);
    hipLaunchKernelGGL(tetra_dev::sample_bins_kernel, dim3(static_cast<unsigned>(rows * bins_parts)), b, 0, stream, a, bins_parts);
    hipLaunchKernelGGL(tetra_dev::sample_token_kernel, dim3(static_cast<unsigned>(rows)), dim3(tetra_dev::kTokenThreads),
                       8 * static_cast<size_t>(a.tiles), stream, a);
    return launch_status();
}

}  // extern "C"
