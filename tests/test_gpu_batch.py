"""Attention over shared prefixes, weights of cached tokens, eviction and log probabilities on the GPU against float64
(run on an MI355X).

Bounds, from the formats:
* shared prefixes: as for the attention, fp16 output, 2^-11 |o|, weights rounded to fp16 and fp32 scores, 1.5 * 2^-11
  of sum w |v|;
* weights: q and whole keys are exact in fp16; a score is a sum of D products with D + 4 roundings at most (the sum,
  scale, logarithm's unit and reference), off by (D + 4) 2^-24 of sum |q k|; a weight by that twice (its own and its
  sum's), the exponentials and logarithm by 2^-20, and sums over n tokens and r rows by (n + r) 2^-24 at most;
* evicted pages: equal, the new rounding being two fixed steps in float32;
* log probabilities: t = (x - m) / T has three roundings, 2^-22 |t|; the sum of exponentials is off by 2^-20 and by
  2^-24 for each of the vocab / 256 terms that a lane adds in line; the entropy by that times sum p (1 + |t|)^2, each
  exponential being off by 2^-22 |t|.
"""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2609_35465_amd as tt  # noqa: E402
from oracle import batch as ref  # noqa: E402
from oracle import serving  # noqa: E402
from test_gpu_serving import Cache, _dev, _starts  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    torch.cuda.init()


# ------------------------------------------------------------------ shared prefixes

class Shared(Cache):
    """A pool in which the sequences of a group name the same pages for its whole shared pages.  groups: (tokens
    shared, [own tokens of each sequence]) after another; `loose`: lengths of sequences after the groups."""

    def __init__(self, seed, groups, heads, page, dim, loose=(), max_pages=None):
        lens, plan, used = [], [], 0
        self.first, self.shared = [0], []
        for shared, own in groups:
            whole = list(range(used, used + shared // page))
            used += len(whole)
            for n in own:
                lens.append(shared + n if n else 0)
                more = -(-lens[-1] // page) - len(whole) if n else 0
                plan.append((whole if n else []) + list(range(used, used + more)))
                used += more
            self.first.append(len(lens))
            self.shared.append(shared)
        for n in loose:
            lens.append(n)
            plan.append(list(range(used, used - (-n // page))))
            used += len(plan[-1])
        order = np.random.default_rng(seed + 100).permutation(used + 3)
        table = np.full((len(lens), max_pages or max(1, max(map(len, plan)))), -1, np.int32)
        for i, p in enumerate(plan):
            table[i, :len(p)] = order[p]
        super().__init__(seed, [(used) * page], heads, page, dim)
        self.table, self.lens, self.max_pages = table, np.array(lens, np.int32), table.shape[1]


_SPACE = []


def _shared_space():
    if not _SPACE:
        _SPACE.append(tt.kv_attend_shared_workspace())
    return _SPACE[0]


def _widen(c):
    """Gives the table room for 256 MB of keys and values."""
    wide = max(c.max_pages, -(-(1 << 28) // (2 * c.heads * c.dim * len(c.lens) * c.page)))
    c.table = np.pad(c.table, ((0, 0), (0, wide - c.table.shape[1])), constant_values=-1)
    c.max_pages = wide


def _check_shared(c, news, q_heads, **kw):
    """With the table as it is and with one that has room for far longer sequences, by whose size calls go by groups."""
    got = _check_shared_once(c, news, q_heads, **kw)
    _widen(c)
    _check_shared_once(c, news, q_heads, **kw)
    return got


def _check_shared_once(c, news, q_heads, scale=None, strided=False, slack=0, seed=2, first=None, shared=None, q_size=2.0):
    rng = np.random.default_rng(seed)
    starts, rows = _starts(news), int(sum(news))
    q = (rng.standard_normal((rows, q_heads, c.dim)) * q_size).astype(np.float16)
    cache, width = c.upload(), q_heads * c.dim
    groups = _dev(np.array(c.first if first is None else first, np.int32))
    lengths = _dev(np.array(c.shared if shared is None else shared, np.int32))
    outs = []
    for _ in range(2):
        if strided:
            qd = torch.zeros((rows, width + 40), dtype=torch.float16, device="cuda")[:, 32:32 + width]
            qd.copy_(_dev(q).flatten(1))
            wide = torch.full((rows + 1, width + 16), 7.0, dtype=torch.float16, device="cuda")
            out = wide[:rows, 8:8 + width]
        else:
            qd = _dev(q)
            wide = torch.full((rows + 1, q_heads, c.dim), 7.0, dtype=torch.float16, device="cuda")
            out = wide[:rows]
        tt.kv_attend_shared(cache, qd, _dev(starts), int(max(news)) + slack, groups, lengths, out, _shared_space(), scale)
        torch.cuda.synchronize()
        assert torch.all(wide[rows] == 7)
        if strided:
            assert torch.all(wide[:, :8] == 7) and torch.all(wide[:, 8 + width:] == 7)
        outs.append(out.contiguous().view(torch.int16))
    assert torch.equal(*outs)
    got = outs[0].view(torch.float16).reshape(rows, q_heads, c.dim).cpu().numpy().astype(np.float64)
    worst = 0.0
    for i, n in enumerate(news):
        if n == 0:
            continue
        ks, vs, there = c.sequence(i)
        want, size = serving.attend(q[starts[i]:starts[i + 1]], ks, vs, there, int(c.lens[i]) - int(n),
                                    c.dim ** -0.5 if scale is None else scale, 0)
        bound = 2.0 ** -11 * np.abs(want) + 1.5 * 2.0 ** -11 * size + 2.0 ** -24
        mine = got[starts[i]:starts[i + 1]]
        # fp16 rounds 65520 and more to an infinity
        past, fits = np.abs(want) - bound >= 65520, np.abs(want) + bound < 65520
        assert np.array_equal(mine[past], np.sign(want[past]) * np.inf)
        if fits.any():
            worst = max(worst, float((np.abs(mine - want) / bound)[fits].max()))
    print(f"[shared] dim={c.dim} page={c.page} heads={q_heads}/{c.heads} groups={c.shared[:6]} news={list(news)[:6]} "
          f"worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0
    return got


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_shared_single_tokens(dim, page):
    """Groups of several lengths, one that ends inside a page, one of a single sequence, an idle slot, and sequences of
    no group behind them."""
    c = Shared(1, [(3 * page, [1, 2, page, 40]), (page + 7, [5, 9, 0, 1]), (700, [30])], 2, page, dim, loose=[90, 1])
    _check_shared(c, [1, 1, 1, 1, 1, 1, 0, 1, 1, 1, 1], 6)


@pytest.mark.parametrize("heads,q_heads", [(1, 1), (8, 40), (2, 14), (4, 4), (1, 16), (1, 17), (2, 80)])
@pytest.mark.parametrize("dim", [64, 128])
def test_shared_head_layouts(heads, q_heads, dim):
    c = Shared(2, [(512, [7, 33, 1, 64, 20, 3, 3, 90])], heads, 32, dim)
    _check_shared(c, [1] * 8, q_heads, strided=True)


@pytest.mark.parametrize("news", [(2, 3, 1), (8, 8, 8), (16, 5, 1), (40, 0, 17), (130, 1, 70)])
@pytest.mark.parametrize("group", [1, 5])
@pytest.mark.parametrize("slack", [0, 300])
def test_shared_several_tokens(news, group, slack):
    """Drafts of a few tokens, chunks of prompts, both; max_new far above what any sequence has."""
    slack = min(slack, sum(news) - max(news))
    c = Shared(3, [(200, [n + 30 if n else 0 for n in news]), (96, [n for n in news])], 2, 16, 64)
    _check_shared(c, list(news) * 2, 2 * group, slack=slack)


@pytest.mark.parametrize("seqs,groups", [(64, 1), (130, 1), (300, 3), (300, 100), (600, 290)])
def test_shared_many_sequences(seqs, groups):
    rng = np.random.default_rng(4)
    sizes = np.diff(np.sort(np.concatenate([[0, seqs], rng.choice(np.arange(1, seqs), groups - 1, replace=False)])))
    plan = [(int(rng.integers(0, 200)), [int(n) for n in rng.integers(0, 40, size)]) for size in sizes]
    c = Shared(4, plan, 1, 16, 64)
    news = [int(n > 0) for n in c.lens]
    _check_shared(c, news, 3)


@pytest.mark.parametrize("prefix,seqs", [(5000, 3), (5000, 40), (33000, 20)])
def test_shared_long_prefixes(prefix, seqs):
    c = Shared(5, [(prefix, [int(n) for n in np.random.default_rng(0).integers(1, 200, seqs)])], 2, 64, 128)
    _check_shared(c, [1] * seqs, 10)


@pytest.mark.parametrize("news", [[1, 1, 1, 1], [1, 2, 40, 1]])
def test_shared_sequences_that_do_not_reach_the_prefix(news):
    """Sequences whose new rows begin before the shared tokens' end see what they would without a group; also the first
    of a group, whose table then does not hold the prefix."""
    c = Shared(6, [(320, [4, 50, 60, 70])], 2, 32, 64)
    c.lens[0], c.table[0, 3:] = 70, -1
    c.lens[2] = 325
    _check_shared(c, news, 4)


@pytest.mark.parametrize("first,shared", [([0, 0, 4], [64, 320]), ([2, 4], [320]), ([0, 4], [0]), ([0, 4], [-5]),
                                          ([0, 2], [31]), ([1, 3, 3, 4], [320, 96, 160]), ([0, 2, 4], [320, 64]),
                                          ([0, 99], [320]), ([-7, 4], [320]), ([3, 1], [320])])
def test_shared_groups_of_any_kind(first, shared):
    """Empty groups, groups of some sequences, no or little in common, bounds outside the batch or falling."""
    _check_shared(Shared(7, [(320, [4, 50, 60, 70])], 2, 32, 128), [1, 1, 2, 1], 10, first=first, shared=shared)


@pytest.mark.parametrize("roomy", [False, True])
def test_shared_lengths_past_the_table(roomy):
    """The table is what counts: tokens past it are not seen, and shared lengths past it are all of it."""
    c = Shared(8, [(320, [4, 50, 60])], 2, 32, 64)
    wide = 16384 if roomy else 10
    c.table = np.pad(c.table[:, :10], ((0, 0), (0, wide - 10)), constant_values=-1)
    c.max_pages = wide
    cache = c.upload()
    q = _dev((np.random.default_rng(1).standard_normal((3, 4, 64)) * 2).astype(np.float16))
    at, out = _dev(_starts([1, 1, 1])), [torch.empty((3, 4, 64), dtype=torch.float16, device="cuda") for _ in range(3)]
    tt.kv_attend(cache, q, at, 1, out[0], tt.kv_attend_workspace())
    for o, n in zip(out[1:], (320, (1 << 31) - 1)):
        tt.kv_attend_shared(cache, q, at, 1, _dev(np.array([0, 3], np.int32)), _dev(np.array([n], np.int32)), o, _shared_space())
    torch.cuda.synchronize()
    for o in out[1:]:
        assert float((o.float() - out[0].float()).abs().max()) <= 4 * 2.0 ** -11 * float(out[0].abs().max())


@pytest.mark.parametrize("news", [(1, 1, 1, 1), (30, 1, 1, 3)])
def test_shared_missing_pages_and_scales(news):
    """A prefix page of no pool place, one of scale 0, one far larger and one far smaller than the others."""
    c = Shared(9, [(320, [n + 20 for n in news])], 2, 32, 128)
    c.table[:, 2] = len(c.k) + 5
    for j, f in ((1, 0.0), (3, 2.0 ** 20), (4, 2.0 ** -30), (5, 2.0 ** 9)):
        c.scales[c.table[0, j]] *= np.float32(f)
    _check_shared(c, list(news), 4, q_size=1e-6)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("news", [(1, 1, 1, 1), (9, 1, 30, 2)])
@pytest.mark.parametrize("roomy", [False, True])
def test_shared_not_finite_queries_stay_alone(news, bad, roomy):
    c = Shared(10, [(320, [n + 20 for n in news])], 2, 32, 64)
    if roomy:
        _widen(c)
    starts, rows = _starts(news), sum(news)
    q = np.random.default_rng(3).standard_normal((rows, 6, 64)).astype(np.float16)
    spoiled = q.copy()
    spoiled[starts[2], 4, 11] = bad
    cache, at = c.upload(), _dev(starts)
    groups, lengths = _dev(np.array(c.first, np.int32)), _dev(np.array(c.shared, np.int32))
    out = [torch.empty((rows, 6, 64), dtype=torch.float16, device="cuda") for _ in range(2)]
    for x, o in zip((q, spoiled), out):
        tt.kv_attend_shared(cache, _dev(x), at, max(news), groups, lengths, o, _shared_space())
    torch.cuda.synchronize()
    assert torch.isnan(out[1][starts[2], 4]).all()
    out[1][starts[2], 4] = out[0][starts[2], 4]
    assert torch.equal(*out)


@pytest.mark.parametrize("roomy", [False, True])
def test_shared_rows_of_no_sequence_are_left_alone(roomy):
    """Starts that end before the last row, as where a graph is captured for a full batch; bad starts."""
    c = Shared(11, [(320, [24, 30, 50])], 2, 32, 64)
    if roomy:
        _widen(c)
    cache, q = c.upload(), _dev(np.random.default_rng(3).standard_normal((9, 6, 64)).astype(np.float16))
    groups, lengths = _dev(np.array([0, 3], np.int32)), _dev(np.array([320], np.int32))
    want = torch.full((3, 6, 64), 7.0, dtype=torch.float16, device="cuda")
    tt.kv_attend_shared(cache, q[:3], _dev(_starts([1, 1, 1])), 1, groups, lengths, want, _shared_space())
    for starts, rows in (([0, 1, 2, 3], 3), ([0, 1, 1, 1], 1), ([-4, 1, 2, 3], 3), ([0, 1, 2, -9], 2), ([9, 0, 0, 0], 0),
                         ([0, 0, 0, 0], 0)):
        out = torch.full((9, 6, 64), 7.0, dtype=torch.float16, device="cuda")
        tt.kv_attend_shared(cache, q, _dev(np.array(starts, np.int32)), 2, groups, lengths, out, _shared_space())
        torch.cuda.synchronize()
        assert torch.all(out[rows:] == 7), starts
        if starts[:2] == [0, 1]:
            assert float((out[:1] - want[:1]).abs().max()) < 1e-2


# ------------------------------------------------------------------ weights of cached tokens

def _check_weigh(c, news, q_heads, window=0, scale=None, decay=1.0, mass="own", strided=False, slack=0, places=None, seed=3,
                 q_size=2.0):
    """mass "own": a buffer of its own, "in place", or None."""
    rng = np.random.default_rng(seed)
    starts, rows, D = _starts(news), int(sum(news)), c.dim
    q = (rng.standard_normal((rows, q_heads, D)) * q_size).astype(np.float16)
    places = places or int(max(1, c.lens.max()))
    before = rng.exponential(1, (len(news), c.heads, places)).astype(np.float32)
    # places of the rows' own tokens are not read
    for i, n in enumerate(news):
        if n:
            before[i, :, max(0, int(c.lens[i]) - int(n)):] = np.nan
        else:
            before[i, :, max(0, int(c.lens[i])):] = np.nan
    cache, width = c.upload(), q_heads * D
    qd = _dev(q)
    if strided:
        qd = torch.zeros((rows, width + 40), dtype=torch.float16, device="cuda")[:, 32:32 + width]
        qd.copy_(_dev(q).flatten(1))
    got = []
    space = tt.kv_weigh_workspace(cache, rows, q_heads)
    for fill in (255, 0):
        space.fill_(fill)
        old = _dev(before)
        out = old if mass == "in place" else torch.full_like(old, -7.0)
        tt.kv_weigh(cache, qd, _dev(starts), int(max(news)) + slack, old if mass else None, out, space, scale, window, decay)
        torch.cuda.synchronize()
        got.append(out.cpu().numpy())
    assert np.array_equal(got[0].view(np.uint32), got[1].view(np.uint32))
    worst, scale = 0.0, D ** -0.5 if scale is None else scale
    for i, n in enumerate(news):
        L = int(c.lens[i])
        ks, _, there = c.sequence(i)
        want, size = ref.weigh(q[starts[i]:starts[i + 1]], ks, there, L - int(n), scale, window)
        past = np.zeros((c.heads, places))
        if mass:
            past[:, :max(0, L - int(n))] = before[i, :, :max(0, L - int(n))].astype(np.float64) * (decay if n else 1)
        seen = min(L, places)
        want, size, past = want[:, :seen], size[:, :seen], past[:, :seen]
        bound = size * 2 * (D + 4) * 2.0 ** -24 + want * (2.0 ** -20 + (L + int(n) * q_heads) * 2.0 ** -24) + \
            past * 2.0 ** -22 + 1e-35
        if seen:
            worst = max(worst, float((np.abs(got[0][i, :, :seen] - want - past) / bound).max()))
        rest = got[0][i, :, seen:]
        if mass != "in place":
            assert np.all(rest == -7)
        else:
            assert np.array_equal(rest.view(np.uint32), before[i, :, seen:].view(np.uint32))
        if n and not mass and places >= L and there[:L].all() and window == 0:
            assert abs(got[0][i].astype(np.float64)[:, :L].sum() - int(n) * q_heads) < 1e-3 * n * q_heads
    print(f"[weigh] dim={D} page={c.page} heads={q_heads}/{c.heads} news={list(news)[:6]} lens={list(c.lens)[:6]} "
          f"window={window} worst {worst:.4f} of the bound", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("mass", ["own", "in place", None])
def test_weigh_single_tokens(dim, page, mass):
    lens = [1, 2, 16, 17, 63, 64, 65, 200, 0, 1000, 256, 257, 511]
    _check_weigh(Cache(21, lens, 2, page, dim), [1, 1, 1, 1, 1, 1, 1, 1, 0, 1, 1, 1, 1], 6, mass=mass)


@pytest.mark.parametrize("heads,q_heads", [(1, 1), (8, 40), (2, 14), (4, 4), (1, 16), (1, 33), (2, 80)])
@pytest.mark.parametrize("dim", [64, 128])
def test_weigh_head_layouts(heads, q_heads, dim):
    _check_weigh(Cache(22, [300, 40, 77], heads, 32, dim), [1, 3, 1], q_heads, strided=True, decay=0.9)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("group", [1, 5])
def test_weigh_prompts(dim, page, group):
    """From the start, after a context, a few last rows, sequences that wait, together."""
    _check_weigh(Cache(23, [300, 333, 64, 500, 90, 700], 2, page, dim), [300, 70, 64, 1, 0, 33], 2 * group, decay=0.5)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 200, 5000, (1 << 31) - 1])
@pytest.mark.parametrize("news", [(1, 1, 1), (130, 1, 70)])
def test_weigh_windows(window, news):
    _check_weigh(Cache(24, [400, 70, 333], 2, 32, 64), list(news), 4, window=window)


@pytest.mark.parametrize("news", [(1,), (40,), (1500,)])
def test_weigh_long_context(news):
    _check_weigh(Cache(25, [9000], 1, 64, 128), list(news), 2, decay=0.0)


@pytest.mark.parametrize("places", [1, 100, 255, 2000])
def test_weigh_fewer_or_more_places_than_tokens(places):
    _check_weigh(Cache(26, [300, 77, 0, 256], 2, 32, 64), [1, 20, 0, 40], 4, places=places)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
@pytest.mark.parametrize("news", [(1, 3), (90, 70)])
def test_weigh_scale_argument(scale, news):
    _check_weigh(Cache(32, [300, 77], 2, 32, 64), list(news), 6, scale=scale, q_size=0.5)


def test_weigh_many_sequences():
    rng = np.random.default_rng(0)
    news = rng.integers(0, 4, 300)
    lens = [int(n + rng.integers(0, 90)) if n else int(rng.integers(0, 2)) * 40 for n in news]
    _check_weigh(Cache(27, lens, 1, 16, 64), news, 3, slack=5)


@pytest.mark.parametrize("news", [(1, 1), (40, 70)])
def test_weigh_missing_pages_and_scales(news):
    """Pages of no pool place get no weight; scales of 0, far larger and far smaller than the others."""
    c = Cache(28, [300, 333], 2, 32, 64)
    c.table[0, 2], c.table[1, 0] = -1, len(c.k)
    for j, f in ((1, 0.0), (3, 2.0 ** 10), (5, 2.0 ** -30)):
        c.scales[c.table[0, j]] *= np.float32(f)
    _check_weigh(c, list(news), 4, q_size=0.01)


@pytest.mark.parametrize("news", [(1, 1), (60, 20)])
def test_weigh_lengths_below_the_rows(news):
    """A length that does not hold the new rows: those before its start see nothing and give nothing."""
    c = Cache(29, [100, 90], 2, 16, 64)
    c.lens = np.array([0 if news[0] == 1 else 30, 90], np.int32)
    _check_weigh(c, list(news), 4)


def test_weigh_length_past_the_table_and_rows_past_the_starts():
    c = Cache(30, [128, 90], 2, 16, 64)
    cache = c.upload()
    q = _dev(np.random.default_rng(1).standard_normal((8, 4, 64)).astype(np.float16))
    space = tt.kv_weigh_workspace(cache, 8, 4)
    out = [torch.full((2, 2, 300), -7.0, device="cuda") for _ in range(2)]
    tt.kv_weigh(cache, q[:2], _dev(np.array([0, 1, 2], np.int32)), 1, None, out[0], space)
    c.d[4].copy_(torch.tensor([128, 90], dtype=torch.int32))
    tt.kv_weigh(cache, q, _dev(np.array([0, 1, 2], np.int32)), 3, None, out[1], space)
    torch.cuda.synchronize()
    assert torch.equal(*out)
    # far past the table: what the table holds is weighed, the places behind it get nothing
    c.d[4].copy_(torch.tensor([(1 << 31) - 1, 90], dtype=torch.int32))
    tt.kv_weigh(cache, q[:2], _dev(np.array([0, 1, 2], np.int32)), 1, None, out[1], space)
    torch.cuda.synchronize()
    assert torch.all(out[1][0, :, 128:] == 0) and torch.equal(out[1][1], out[0][1])
    assert float((out[1][0, :, :128].sum(-1) - 2).abs().max()) < 1e-4


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_weigh_not_finite_query_stays_in_its_head_and_sequence(bad):
    c = Cache(31, [100, 300], 2, 16, 64)
    cache, q = c.upload(), np.random.default_rng(1).standard_normal((2, 6, 64)).astype(np.float16)
    out = [torch.zeros((2, 2, 300), device="cuda") for _ in range(2)]
    space = tt.kv_weigh_workspace(cache, 2, 6)
    spoiled = q.copy()
    spoiled[1, 1, 5] = bad
    for x, o in zip((q, spoiled), out):
        tt.kv_weigh(cache, _dev(x), _dev(_starts([1, 1])), 1, None, o, space)
    torch.cuda.synchronize()
    assert torch.isnan(out[1][1, 0]).all()
    assert torch.equal(out[1][0], out[0][0]) and torch.equal(out[1][1, 1], out[0][1, 1])


# ------------------------------------------------------------------ eviction

def _pages(c, i, k, v, scales, table, n):
    """Whole numbers [n, heads, dim] and scales [n, heads] of a sequence, keys and values."""
    B, out = c.page, []
    for which in (0, 1):
        q, s = np.zeros((n, c.heads, c.dim), np.int8), np.zeros((n, c.heads), np.float32)
        for j in range(-(-n // B)):
            p = table[i, j] if j < table.shape[1] else -1
            if not 0 <= p < len(k):
                continue
            page = k[p] if which == 0 else v[p].transpose(0, 1, 3, 2).reshape(k.shape[1:])
            hi = min(n, (j + 1) * B)
            q[j * B:hi] = page.transpose(1, 0, 2)[:hi - j * B]
            s[j * B:hi] = scales[p, :, which]
        out.append((q, s))
    return out


def _check_evict(c, kept, recent, mass=None, places=None, out_places=None, wide=None, drop=None, seed=5):
    """Evicts into fresh pages of the same pool and checks every byte of it."""
    rng = np.random.default_rng(seed)
    seqs, B, kept = len(c.lens), c.page, np.array(kept, np.int32)
    places = places or int(max(1, c.lens.max()))
    if mass is None:
        mass = rng.exponential(1, (seqs, c.heads, places)).astype(np.float32)
    need = [-(-max(0, min(int(k), int(n))) // B) for k, n in zip(kept, c.lens)]
    wide = wide or max(1, max(need))
    old = len(c.k)
    pages = old + sum(need) + 2
    to_table = np.full((seqs, wide), -1, np.int32)
    order, at = old + rng.permutation(sum(need) + 2), 0
    for i, n in enumerate(need):
        n = min(n, wide)
        to_table[i, :n] = order[at:at + n]
        at += n
    if drop is not None:
        to_table[drop] = -1
    grow = pages - old
    c.k = np.concatenate([c.k, np.full((grow,) + c.k.shape[1:], 99, np.int8)])
    c.v = np.concatenate([c.v, np.full((grow,) + c.v.shape[1:], 99, np.int8)])
    c.scales = np.concatenate([c.scales, np.full((grow,) + c.scales.shape[1:], -5, np.float32)])
    cache = c.upload()
    to_d = (_dev(to_table), _dev(kept))
    to = tt.make_kv_cache(*c.d[:3], *to_d)
    out_places = out_places or int(max(1, kept.max()))
    out = torch.full((seqs, c.heads, out_places), -7.0, device="cuda")
    space = tt.kv_evict_workspace(cache, to)
    space.fill_(255)
    tt.kv_evict(cache, to, _dev(mass), out, space, recent)
    torch.cuda.synchronize()
    k1, v1, s1 = c.download()
    out = out.cpu().numpy()
    want_k, want_v, want_s = c.k.copy(), c.v.copy(), c.scales.copy()
    for i in range(seqs):
        n = min(int(max(0, c.lens[i])), c.table.shape[1] * B)
        b = min(int(max(0, kept[i])), n, wide * B)
        held = _pages(c, i, c.k, c.v, c.scales, c.table, n)
        for h in range(c.heads):
            chosen = ref.choose(mass[i, h], n, b, recent)
            assert len(chosen) == b
            m = np.zeros(n, np.float32)
            m[:min(n, places)] = mass[i, h, :n]
            row = np.full(out_places, -7, np.float32)
            row[:min(b, out_places)] = m[chosen][:out_places]
            assert np.array_equal(out[i, h].view(np.uint32), row.view(np.uint32)), (i, h)
            for j in range(-(-b // B)):
                page = to_table[i, j]
                if not 0 <= page < pages:
                    continue
                part = chosen[j * B:(j + 1) * B]
                for which, (q, s) in enumerate(held):
                    whole, top = ref.moved(q[part, h], s[part, h])
                    want_s[page, h, which] = top
                    if which == 0:
                        want_k[page, h, :len(part)] = whole
                    else:
                        flat = want_v[page, h].transpose(0, 2, 1).reshape(B, c.dim).copy()
                        flat[:len(part)] = whole
                        want_v[page, h] = flat.reshape(B // 16, 16, c.dim).transpose(0, 2, 1)
    live = np.zeros((pages, B), bool)                   # places that hold a kept token; the others may hold anything
    live[:old] = True
    for i in range(seqs):
        b = min(int(max(0, kept[i])), int(max(0, c.lens[i])), wide * B)
        for j in range(-(-b // B)):
            if to_table[i, j] >= 0:
                live[to_table[i, j], :b - j * B] = True
    spare = sorted(set(range(old, pages)) - set(to_table.flatten().tolist()))
    live[spare] = True
    flat1, flat0 = (x.transpose(0, 1, 2, 4, 3).reshape(pages, c.heads, B, c.dim) for x in (v1, want_v))
    sel = np.broadcast_to(live[:, None, :, None], k1.shape)
    assert np.array_equal(k1[sel], want_k[sel]) and np.array_equal(flat1[sel], flat0[sel])
    assert np.array_equal(s1.view(np.uint32), want_s.view(np.uint32))
    return to, out


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("recent", [0, 1, 20, 1000])
def test_evict(dim, page, recent):
    """Lengths around pages, budgets of none, one, a page, all and more than all, an idle slot."""
    lens = [1, 17, 64, 200, 300, 0, 130, 129, 500]
    kept = [1, 16, 1, 100, 299, 5, 200, 129, 0]
    print(f"[evict] dim={dim} page={page} recent={recent}", flush=True)
    _check_evict(Cache(41, lens, 3, page, dim), kept, recent)


@pytest.mark.parametrize("recent", [0, 100])
@pytest.mark.parametrize("kept", [1, 64, 4097, 20000])
def test_evict_long(recent, kept):
    print(f"[evict long] kept={kept}", flush=True)
    _check_evict(Cache(42, [20001, 1500], 2, 64, 64), [kept, 700], recent)


@pytest.mark.parametrize("seqs", [3, 100, 300])
def test_evict_tables_for_long_sequences(seqs):
    """Tables with room for more than 8,192 tokens: rows are cut in parts, few or one of them where sequences are many;
    short ones leave parts without tokens."""
    rng = np.random.default_rng(3)
    lens = [int(n) for n in rng.integers(0, 300, seqs)]
    lens[1] = 9000
    kept = [int(n) for n in rng.integers(0, 300, seqs)]
    kept[1] = 4000
    print(f"[evict wide] seqs={seqs}", flush=True)
    _check_evict(Cache(52, lens, 2, 16, 64, max_pages=700), kept, 12)


def test_evict_ties_and_not_finite_weights():
    """Equal weights go by the first token; NaN is the least, zeros of both signs are equal, infinities as they are."""
    c = Cache(43, [700, 700, 700, 700], 2, 16, 64)
    mass = np.zeros((4, 2, 700), np.float32)
    mass[0] = 1.0
    mass[1] = np.random.default_rng(0).integers(0, 5, (2, 700))
    mass[2] = np.random.default_rng(1).choice([0.0, -0.0, np.nan, np.inf, -np.inf, 1e-40, 3.0], (2, 700))
    mass[3] = np.nan
    for recent in (0, 33):
        print(f"[evict ties] recent={recent}", flush=True)
        _check_evict(Cache(43, [700] * 4, 2, 16, 64), [300, 333, 250, 90], recent, mass=mass)
    assert c.heads == 2


def test_evict_places_and_pages_that_are_missing():
    """Fewer weights than tokens, fewer or more places for them, tables narrower or wider than what is kept, source pages
    of no pool place, new pages that are missing."""
    for kw in (dict(places=50), dict(out_places=7), dict(out_places=400), dict(wide=3), dict(wide=40), dict(drop=(0, 1))):
        print(f"[evict missing] {kw}", flush=True)
        c = Cache(44, [300, 120], 2, 16, 64)
        c.table[0, 3], c.table[0, 5] = -1, 1 << 20
        _check_evict(c, [150, 60], 10, **kw)


def test_evict_scales_far_apart():
    c = Cache(45, [300, 120], 2, 16, 128)
    c.scales *= np.float32(2.0) ** np.random.default_rng(0).integers(-60, 60, c.scales.shape).astype(np.float32)
    c.scales[c.table[0, 2]] = 0
    print("[evict scales]", flush=True)
    _check_evict(c, [150, 60], 10)


def test_evict_many_sequences_and_bad_lengths():
    rng = np.random.default_rng(0)
    c = Cache(46, [int(n) for n in rng.integers(0, 120, 200)], 1, 16, 64)
    c.lens[5], c.lens[9] = -3, -(1 << 31)
    kept = rng.integers(0, 90, 200)
    kept[17], kept[30] = -4, -(1 << 31)
    print("[evict many]", flush=True)
    _check_evict(c, kept, 8)


def test_evict_keeps_a_prefix_of_scales_exactly():
    """Where nothing is taken the new pages are the old ones, byte by byte."""
    c = Cache(47, [100, 64], 2, 32, 64)
    to, _ = _check_evict(c, [100, 64], 0)
    k, v, s = c.download()
    to_pages = to.tensors[3].cpu().numpy()
    for i, n in enumerate((4, 2)):
        for j in range(n):
            a, b = c.table[i, j], to_pages[i, j]
            assert np.array_equal(s[a], s[b])
            if (j + 1) * 32 <= c.lens[i]:
                assert np.array_equal(k[a], k[b]) and np.array_equal(v[a], v[b])


# ------------------------------------------------------------------ positions after an eviction

@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("news", [(1, 1, 0, 1), (30, 1, 0, 17)])
def test_append_shifted_is_the_append_further_on(dim, news):
    """Rows with a shift come out as those of a longer sequence: the same bytes as from an append with a table of the
    rotation that begins so many places later."""
    lens, shifts = [40, 21, 9, 64], np.array([100, 0, 7, 1000], np.int32)
    starts, rows = _starts(news), sum(news)
    rng = np.random.default_rng(2)
    k, v, q = (_dev(rng.standard_normal((rows, n, dim)).astype(np.float32)) for n in (2, 2, 4))
    rope = tt.rope_table(1100, dim)
    c = Cache(48, lens, 2, 16, dim)
    out = torch.zeros((rows, 4, dim), dtype=torch.float16, device="cuda")
    tt.kv_append(c.upload(), q, k, v, _dev(starts), max(news), rope, out, shifts=_dev(shifts))
    got = [t.clone() for t in c.d[:3]] + [out]
    for i in range(4):
        if not news[i]:
            continue
        part = torch.zeros_like(out)
        alone = Cache(48, lens, 2, 16, dim)
        tt.kv_append(alone.upload(), q, k, v, _dev(starts), max(news), rope[int(shifts[i]):].contiguous(), part)
        torch.cuda.synchronize()
        assert torch.equal(part[starts[i]:starts[i + 1]], out[starts[i]:starts[i + 1]])
        pages = torch.from_numpy(c.table[i][c.table[i] >= 0].astype(np.int64)).cuda()
        for a, b in zip(got[:3], alone.d[:3]):
            assert torch.equal(a[pages], b[pages])


@pytest.mark.parametrize("dim", [64, 128])
def test_append_shifted_from_fp16_with_norms(dim):
    """fp16 rows, strided, with norms: the bytes of an append whose table of the rotation begins at the shift."""
    lens, news, shift = [40, 23, 130], [1, 17, 70], 333
    starts, rows = _starts(news), sum(news)
    rng = np.random.default_rng(3)
    wide = _dev(rng.standard_normal((rows, 8 * dim + 16)).astype(np.float16))
    q, k, v = (wide[:, 8 + a * dim:8 + b * dim] for a, b in ((0, 4), (4, 6), (6, 8)))
    norms = [_dev(rng.uniform(0.5, 1.5, dim).astype(np.float32)) for _ in range(2)]
    rope, got = tt.rope_table(600, dim), []
    for table, shifts in ((rope, torch.full((3,), shift, dtype=torch.int32, device="cuda")), (rope[shift:].contiguous(), None)):
        c = Cache(50, lens, 2, 16, dim)
        out = torch.zeros((rows, 4, dim), dtype=torch.float16, device="cuda")
        tt.kv_append(c.upload(), q, k, v, _dev(starts), max(news), table, out, *norms, shifts=shifts)
        torch.cuda.synchronize()
        got.append([*c.d[:3], out])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_append_shifts_are_clamped():
    c = Cache(49, [40, 21], 1, 16, 64)
    x, rope = _dev(np.random.default_rng(2).standard_normal((2, 1, 64)).astype(np.float32)), tt.rope_table(50, 64)
    want = []
    for shifts in ([-5, (1 << 31) - 1], [0, 1 << 30], [-(1 << 31), 29]):
        out = torch.zeros((2, 1, 64), dtype=torch.float16, device="cuda")
        tt.kv_append(c.upload(), x, x, x, _dev(_starts([1, 1])), 1, rope, out, shifts=_dev(np.array(shifts, np.int32)))
        torch.cuda.synchronize()
        want.append(out)
    assert torch.equal(want[0], want[1]) and torch.equal(want[0], want[2])       # the table's last row


# ------------------------------------------------------------------ log probabilities

def _check_score(x, tokens=None, top=5, temperature=None, pad=0, entropy=True, half=False, lead=0):
    """x float32 or float16 [rows, vocab]; lead: elements before the first row, so that rows begin off any boundary."""
    rows, vocab = x.shape
    rng = np.random.default_rng(vocab)
    if tokens is None:
        tokens = rng.integers(0, vocab, (rows, 1))
    tokens = np.array(tokens, np.int32).reshape(rows, -1)
    x = x.astype(np.float16 if half else np.float32)
    flat = torch.full((rows * (vocab + pad) + lead,), float("nan"), dtype=torch.float16 if half else torch.float32, device="cuda")
    logits = flat[lead:].view(rows, vocab + pad)[:, :vocab]
    logits.copy_(_dev(x))
    t = None if temperature is None else _dev(np.broadcast_to(np.float32(temperature), (rows,)).copy())
    runs = []
    for fill in (255, 0):
        space = tt.log_probs_workspace(rows, vocab, top).fill_(fill)
        out = torch.full((rows, tokens.shape[1]), 7.0, device="cuda")
        ent = torch.full((rows,), 7.0, device="cuda")
        ids = torch.full((rows, top), 7, dtype=torch.int32, device="cuda")
        logs = torch.full((rows, top), 7.0, device="cuda")
        tt.log_probs(logits, _dev(tokens), out, space, entropy=ent if entropy else None, top_tokens=ids if top else None,
                     top_out=logs if top else None, temperature=t)
        torch.cuda.synchronize()
        runs.append([a.cpu().numpy() for a in (out, ent, ids, logs)])
    for a, b in zip(*runs):
        assert np.array_equal(a.view(np.uint32), b.view(np.uint32))
    out, ent, ids, logs = runs[0]
    chain, worst = 2.0 ** -20 + (vocab // 256 + 1) * 2.0 ** -24, 0.0

    def near(got, want, extra=0.0):
        nonlocal worst
        want = np.where(want < -float(np.finfo(np.float32).max), -np.inf, want)      # past the type's end
        with np.errstate(invalid="ignore"):
            assert np.array_equal(np.isneginf(got), np.isneginf(want)), (got, want)
            fine = ~np.isneginf(want)
            # t = want + ln l, and ln l is at most ln vocab
            bound = chain + 2.0 ** -22 * (np.abs(want[fine]) + np.log(vocab))
            if fine.any():
                worst = max(worst, float((np.abs(got[fine].astype(np.float64) - want[fine]) / bound).max()))

    for i in range(rows):
        T = 1.0 if temperature is None else float(np.broadcast_to(np.float32(temperature), (rows,))[i])
        given, h, spread, order, theirs = ref.log_probs(x[i], T, tokens[i], top)
        near(out[i], given)
        assert np.array_equal(ids[i], order), (i, ids[i][:8], order[:8])
        near(logs[i], theirs)
        if entropy:
            worst = max(worst, abs(float(ent[i]) - h) / (chain * max(spread, 1.0)))
    print(f"[score] rows={rows} vocab={vocab} top={top} half={half} T={temperature} worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 65, 1000, 1023, 1025, 4097, 50001, 151936])
@pytest.mark.parametrize("half", [False, True])
def test_score_vocabularies(vocab, half):
    rng = np.random.default_rng(vocab)
    x = rng.standard_normal((3, vocab)) * 3
    _check_score(x, rng.integers(0, vocab, (3, 4)), top=20, half=half)
    _check_score(x, top=1, half=half, pad=5, lead=3)


@pytest.mark.parametrize("top", [0, 1, 2, 5, 20, 63, 64])
@pytest.mark.parametrize("rows", [1, 7, 300])
def test_score_alternatives(top, rows):
    _check_score(np.random.default_rng(top).standard_normal((rows, 3001)) * 2, top=top, pad=top)


@pytest.mark.parametrize("rows", [1, 40, 1100])
@pytest.mark.parametrize("half", [False, True])
def test_score_rows(rows, half):
    x = np.random.default_rng(rows).standard_normal((rows, 9001)) * 2
    _check_score(x, top=3, half=half, temperature=np.random.default_rng(1).uniform(0.2, 2, rows))


@pytest.mark.parametrize("vocab", [700, 20000, 151936])
@pytest.mark.parametrize("rows", [1, 600])
def test_score_orders_and_ties(vocab, rows):
    """Rising, falling, equal logits, few values, many equal at the top, in the first and the last places."""
    if rows * vocab > 2e7:
        rows = 100
    base = np.arange(vocab, dtype=np.float32)
    rng = np.random.default_rng(0)
    kinds = [base / vocab, -base / vocab, base * 0 + 3, rng.integers(0, 3, vocab), np.where(base < 70, 5, 0),
             np.where(base >= vocab - 70, 5, 0), np.where(base % 2 == 0, 1, 1 + 2.0 ** -20), -np.abs(base - vocab // 2) / 10]
    x = np.stack([kinds[i % len(kinds)] for i in range(max(rows, len(kinds)))])
    _check_score(x, top=64)
    _check_score(x[:len(kinds)], top=5, half=True)


def test_score_not_finite():
    """NaN is -inf, infinities share, rows of nothing but -inf, masks of the type's lowest, alternatives that are none."""
    vocab, inf = 5000, np.inf
    rng = np.random.default_rng(0)
    x = rng.standard_normal((10, vocab)).astype(np.float32)
    x[0, ::2] = np.nan
    x[1] = -inf
    x[2] = np.nan
    x[3, [7, 4000]] = inf
    x[4] = np.where(rng.random(vocab) < 0.999, -inf, x[4])
    x[5] = np.where(rng.random(vocab) < 0.99, np.finfo(np.float32).min, x[5])
    x[6] = np.where(np.arange(vocab) == 4999, 2.0, -inf)
    x[7] = np.where(np.arange(vocab) == 0, 2.0, -inf)
    x[8] = np.finfo(np.float32).min
    x[9, 17] = -inf
    tokens = np.stack([np.full(10, 17), np.full(10, 4999), np.full(10, 0), np.full(10, -1), np.full(10, vocab),
                       np.full(10, -(1 << 31)), np.full(10, 4000)], 1)
    for top in (5, 20, 64):
        _check_score(x, tokens, top=top)
        _check_score(x, tokens, top=top, temperature=0.5)
    x = np.clip(x, np.finfo(np.float16).min, None)
    x[8] = np.finfo(np.float16).min
    _check_score(np.where(np.isneginf(x), -inf, x), tokens, top=20, half=True)


@pytest.mark.parametrize("temperature", [0.0, -1.0, np.nan, np.inf, 1e-3, 1e-30, 1e-42, 30.0, 1e30])
def test_score_temperatures(temperature):
    x = np.random.default_rng(0).standard_normal((2, 3000))
    x[1, 5] = -np.inf
    _check_score(x, [[3, 5], [3, 5]], top=5, temperature=temperature)


def test_score_large_logits():
    x = np.random.default_rng(0).standard_normal((3, 3000)) * np.array([[1e4], [1e30], [3e38 / 5]])
    _check_score(x, top=5)


@pytest.mark.parametrize("temperature", [1.0, 1.5, 4.0, 1e30])
def test_score_differences_past_the_type(temperature):
    """Logits that lie further apart than the type reaches, at temperatures that bring them back into it."""
    x = np.random.default_rng(0).uniform(-3.4e38, 3.4e38, (2, 3000)).astype(np.float32)
    x[0, 7], x[0, 8], x[1, 9] = np.finfo(np.float32).min, np.finfo(np.float32).max, np.inf
    _check_score(x, [[7, 8, 5], [9, 5, 6]], top=64, temperature=temperature)


def test_score_workspace_serves_fewer_rows():
    """One for the largest batch serves every smaller one, whose rows are cut in more parts."""
    vocab, top = 30000, 7
    x = _dev(np.random.default_rng(0).standard_normal((900, vocab)).astype(np.float32))
    space = tt.log_probs_workspace(900, vocab, top)
    for rows in (900, 513, 300, 64, 5, 1):
        ids, logs = torch.zeros((rows, top), dtype=torch.int32, device="cuda"), torch.zeros((rows, top), device="cuda")
        tt.log_probs(x[:rows], None, None, space, top_tokens=ids, top_out=logs)
        torch.cuda.synchronize()
        want = torch.log_softmax(x[:rows].double(), -1).topk(top)
        assert torch.equal(ids.long(), want.indices) and torch.allclose(logs.double(), want.values, atol=1e-4)


def test_score_nothing_but_what_is_asked_for():
    x = _dev(np.random.default_rng(0).standard_normal((3, 400)).astype(np.float32))
    space, ent = tt.log_probs_workspace(3, 400), torch.zeros(3, device="cuda")
    tt.log_probs(x, None, None, space, entropy=ent)
    out = torch.zeros(3, device="cuda")
    tt.log_probs(x, torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda"), out, space)
    torch.cuda.synchronize()
    want = torch.log_softmax(x.double(), -1)
    assert torch.allclose(ent.double(), -(want.exp() * want).sum(-1), atol=1e-5)
    assert torch.allclose(out.double(), want[torch.arange(3), torch.tensor([5, 6, 7])], atol=1e-5)


@pytest.mark.parametrize("vocab", [524289, 1 << 22])
def test_score_up_to_the_largest_vocabulary(vocab):
    _check_score(np.random.default_rng(0).standard_normal((2, vocab)).astype(np.float32) * 3, top=64)


def test_score_offsets_past_four_gib():
    """Rows of a buffer of 5 GiB."""
    rows, vocab = 9000, 151936
    x = torch.zeros((rows, vocab), device="cuda")
    x[:, 77] = torch.arange(rows, device="cuda") % 50 / 10
    ids, logs = torch.zeros((rows, 1), dtype=torch.int32, device="cuda"), torch.zeros((rows, 1), device="cuda")
    tt.log_probs(x, None, None, tt.log_probs_workspace(rows, vocab, 1), top_tokens=ids, top_out=logs)
    torch.cuda.synchronize()
    t = x[:, 77].double()
    assert torch.equal(ids[:, 0], torch.where(t > 0, 77, 0).int())
    assert torch.allclose(logs[:, 0].double(), t - (vocab - 1 + t.exp()).log(), atol=1e-5)


# ------------------------------------------------------------------ together

def _serving_state():
    """A batch of two groups over a shared pool, its buffers, and room for an eviction."""
    c = Shared(61, [(64, [20, 5, 9]), (96, [30, 31])], 2, 16, 64, max_pages=20)
    used = int(c.table.max()) + 1
    grow = 60
    c.k, c.v = (np.concatenate([a, np.zeros((grow,) + a.shape[1:], np.int8)]) for a in (c.k, c.v))
    c.scales = np.concatenate([c.scales, np.zeros((grow, 2, 2), np.float32)])
    spare = iter(range(used + 3, used + grow))
    for i in range(5):
        n = -(-int(c.lens[i]) // 16)
        c.table[i, n] = next(spare)
    return c, spare


@pytest.mark.parametrize("roomy", [False, True])
def test_a_served_step_of_all_operators_in_a_graph(roomy):
    """Append, attention over the groups, weights, log probabilities, captured once and replayed with other lengths and
    groups; every replay is what the calls give by themselves."""
    c, _ = _serving_state()
    if roomy:
        _widen(c)
    cache, rng = c.upload(), np.random.default_rng(0)
    x = _dev(rng.standard_normal((5, 2, 64)).astype(np.float32))
    q = _dev(rng.standard_normal((5, 6, 64)).astype(np.float32))
    logits, rope = _dev(rng.standard_normal((5, 3000)).astype(np.float32)), tt.rope_table(400, 64)
    at, shifts = _dev(_starts([1] * 5)), torch.zeros(5, dtype=torch.int32, device="cuda")
    groups, shared = _dev(np.array(c.first, np.int32)), _dev(np.array(c.shared, np.int32))
    tokens = _dev(rng.integers(0, 3000, 5).astype(np.int32))
    spaces = (tt.kv_attend_shared_workspace(), tt.kv_weigh_workspace(cache, 5, 6), tt.log_probs_workspace(5, 3000, 4))

    def step(qo, out, mass, logs, ent, ids, top):
        tt.kv_append(cache, q, x, x, at, 1, rope, qo, shifts=shifts)
        tt.kv_attend_shared(cache, qo, at, 1, groups, shared, out, spaces[0])
        tt.kv_weigh(cache, qo, at, 1, mass, mass, spaces[1], decay=0.9)
        tt.log_probs(logits, tokens, logs, spaces[2], entropy=ent, top_tokens=ids, top_out=top)

    def buffers():
        return (torch.zeros((5, 6, 64), dtype=torch.float16, device="cuda"), torch.zeros((5, 6, 64), dtype=torch.float16, device="cuda"),
                torch.zeros((5, 2, 320), device="cuda"), torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda"),
                torch.zeros((5, 4), dtype=torch.int32, device="cuda"), torch.zeros((5, 4), device="cuda"))

    captured, eager = buffers(), buffers()
    step(*eager)
    torch.cuda.synchronize()
    for t in eager:
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    for rep in range(5):
        c.d[4].add_(1)
        shifts.add_(rep)
        shared.copy_(torch.tensor([64 if rep % 2 else 32, 96 if rep < 3 else 0], dtype=torch.int32))
        x.normal_()
        logits.normal_()
        torch.cuda.synchronize()
        before = [t.clone() for t in c.d[:3]]
        graph.replay()
        torch.cuda.synchronize()
        for t, b in zip(c.d, before):
            t.copy_(b)
        step(*eager)
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b), rep
        assert float(captured[2].sum()) > 0


def test_generation_goes_on_after_an_eviction():
    """Weights over steps, an eviction into other pages, appends with shifts, attention: as the oracle computes each from
    what the cache holds.  Evicting nothing changes no result."""
    c, spare = _serving_state()
    cache, rng = c.upload(), np.random.default_rng(0)
    at, rope = _dev(_starts([1] * 5)), tt.rope_table(500, 64)
    mass = torch.zeros((5, 2, 320), device="cuda")
    spaces = (tt.kv_attend_workspace(), tt.kv_weigh_workspace(cache, 5, 6))

    def step(cache, lens, shifts, mass):
        x = _dev(rng.standard_normal((5, 2, 64)).astype(np.float32))
        q = _dev(rng.standard_normal((5, 6, 64)).astype(np.float32))
        lens.add_(1)
        qo, out = (torch.empty((5, 6, 64), dtype=torch.float16, device="cuda") for _ in range(2))
        tt.kv_append(cache, q, x, x, at, 1, rope, qo, shifts=shifts)
        tt.kv_attend(cache, qo, at, 1, out, spaces[0])
        tt.kv_weigh(cache, qo, at, 1, mass, mass, spaces[1])
        return qo, out

    shifts = torch.zeros(5, dtype=torch.int32, device="cuda")
    for _ in range(4):
        step(cache, c.d[4], shifts, mass)
    lens = c.d[4].clone()
    kept = torch.minimum(lens, torch.tensor([40, 40, 300, 50, 128], dtype=torch.int32, device="cuda"))
    table = torch.full((5, 20), -1, dtype=torch.int32)
    for i in range(5):
        for j in range(-(-int(kept[i]) // 16) + 1):
            table[i, j] = next(spare)
    to_lens = kept.clone()
    to = tt.make_kv_cache(*c.d[:3], table.cuda(), to_lens)
    new_mass = torch.full((5, 2, 320), float("nan"), device="cuda")
    tt.kv_evict(cache, to, mass, new_mass, tt.kv_evict_workspace(cache, to), recent=8)
    dropped = (lens - kept).int()
    assert dropped.tolist()[2] == 0 and min(dropped[i] for i in (0, 1, 3)) > 0
    # the step after it, on the thinned cache
    state = torch.get_rng_state()
    qo, out = step(to, to_lens, dropped, new_mass)
    torch.cuda.synchronize()
    k, v, s = c.download()
    for i in range(5):
        n = int(to_lens[i])
        ks, vs, there = serving.sequence(k, v, s, table[i].numpy(), n)
        want, size = serving.attend(qo[i:i + 1].cpu().numpy(), ks, vs, there, n - 1, 64 ** -0.5, 0)
        bound = 2.0 ** -11 * np.abs(want) + 1.5 * 2.0 ** -11 * size + 2.0 ** -24
        assert np.all(np.abs(out[i:i + 1].cpu().numpy() - want) <= bound), i
        assert torch.isfinite(new_mass[i, :, :n]).all() and torch.isnan(new_mass[i, :, n:]).all()
    torch.set_rng_state(state)


def test_operators_on_other_streams():
    """Two streams at once, each with workspaces of its own, not torch's current one."""
    setups = []
    for i in range(2):
        c = Shared(71 + i, [(640, [20, 50, 90, 33]), (320, [300, 7])], 2, 32, 64)
        _widen(c)
        cache = c.upload()
        q = _dev(np.random.default_rng(i).standard_normal((6, 6, 64)).astype(np.float16))
        x = _dev(np.random.default_rng(i).standard_normal((6, 20000)).astype(np.float32))
        kept = _dev(np.minimum(c.lens, 100).astype(np.int32))
        pages = len(c.k)
        pool = [torch.zeros((6 * 7,) + t.shape[1:], dtype=t.dtype, device="cuda") for t in c.d[:3]]
        to = tt.make_kv_cache(*pool, torch.arange(42, dtype=torch.int32, device="cuda").view(6, 7), kept)
        spaces = [(tt.kv_attend_shared_workspace(), tt.kv_weigh_workspace(cache, 6, 6), tt.kv_evict_workspace(cache, to),
                   tt.log_probs_workspace(6, 20000, 9)) for _ in range(2)]
        setups.append((c, cache, q, x, to, pool, spaces, _dev(np.array(c.first, np.int32)), _dev(np.array(c.shared, np.int32))))
        assert pages
    at, tokens = _dev(_starts([1] * 6)), _dev(np.arange(6, dtype=np.int32))

    def results():
        return (torch.zeros((6, 6, 64), dtype=torch.float16, device="cuda"), torch.zeros((6, 2, 960), device="cuda"),
                torch.zeros((6, 2, 100), device="cuda"), torch.zeros(6, device="cuda"),
                torch.zeros((6, 9), dtype=torch.int32, device="cuda"), torch.zeros((6, 9), device="cuda"))

    def calls(i, o, which, stream):
        _, cache, q, x, to, _, spaces, groups, shared = setups[i]
        w = spaces[which]
        tt.kv_attend_shared(cache, q, at, 1, groups, shared, o[0], w[0], stream=stream)
        tt.kv_weigh(cache, q, at, 1, None, o[1], w[1], stream=stream)
        tt.kv_evict(cache, to, o[1], o[2], w[2], recent=5, stream=stream)
        tt.log_probs(x, tokens, o[3], w[3], top_tokens=o[4], top_out=o[5], stream=stream)

    want, pools = [results() for _ in range(2)], []
    for i in range(2):
        calls(i, want[i], 0, None)
        torch.cuda.synchronize()
        pools.append([t.clone() for t in setups[i][5]])
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[results() for _ in range(4)] for _ in range(2)]
    torch.cuda.synchronize()
    for rep in range(4):
        for i in range(2):
            calls(i, outs[i][rep], 1, streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            for a, b in zip(o, want[i]):
                assert torch.equal(a, b)
        for a, b in zip(setups[i][5], pools[i]):
            assert torch.equal(a, b)
