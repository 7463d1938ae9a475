"""Weights of cached tokens over the plans that the device makes for them: items of several row tiles, spans of several
blocks, scores that find no room, more items than waves; and the workspace (run on an MI355X).

Which of these a call meets goes by its sizes, so every case asks a copy of the plan on the host whether it meets what it
is for.  The pages of a small pool are shared by all tables, in any order and more than once.

Bounds: a score is a sum of D products with D + 4 roundings at most, off by (D + 4) 2^-24 of sum |q k|, a weight by that
twice (its own and its sum's); exponentials and logarithm by 2^-20; a row's sum takes 16 additions and 4 roundings of its
rescaling a block of a span, 4 roundings a span and 64 from lanes and waves, a token's sum an addition for each 32 rows
and 64 from lanes and chunks: 2^-24 each.
"""

from types import SimpleNamespace

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2609_35465_amd as tt  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    torch.cuda.init()


def _up(a, b):
    return -(-a // b)


def _plan(lens, news, heads, group, dim, places, cus, max_new):
    few = max_new * group * dim <= 2048
    block, most_spans, workers = (64, 256, 16 * cus) if few else (256, 64, 2 * cus)
    blocks = [_up(max(n if m else 0, min(n, places)), block) for n, m in zip(lens, news)]
    tiles = [_up(m * group, 32) for m in news]
    steps = heads * sum(b * t for b, t in zip(blocks, tiles))
    chunk, span, keep = max(1, _up(steps, 16 * cus)), 1, False
    if few:
        ends = heads * sum(b > 0 for b in blocks)
        span = max(1, _up(heads * sum(blocks), max(workers - ends, workers // 2)))
        keep = heads * sum(blocks) * 64 * max_new * group <= 1 << 24
    per = [max(span, _up(b, most_spans)) for b in blocks]
    items = sum(heads * _up(b, p) for b, p in zip(blocks, per))
    return SimpleNamespace(few=few, keep=keep, chunk=chunk, items=items, workers=workers, block=block, span=per,
                           spans=[_up(b, p) for b, p in zip(blocks, per)], two=few and max_new * group > 16)


def _want(q, k, scales, first, seen_to, scale, window):
    """(weights, their error's size) float64 of tokens [0, seen_to) from rows q [rows, group, dim] at positions first.. over
    one cache head's keys k int8 [tokens, dim] of scales [tokens]."""
    rows, group, dim = q.shape
    keys = (k.double() * scales.double()[:, None]).T.contiguous()
    out, size = (torch.zeros(k.shape[0], dtype=torch.float64, device="cuda") for _ in range(2))
    token, step = torch.arange(k.shape[0], device="cuda"), max(1, (1 << 25) // max(1, k.shape[0] * group))
    for i in range(0, rows, step):
        x = q[i:i + step].double()
        n = x.shape[0]
        x = x.reshape(n * group, dim)
        position = (first + i + torch.arange(n, device="cuda")).repeat_interleave(group)[:, None]
        seen = (token <= position) & (token < seen_to)
        if window:
            seen &= token > position - window
        z = (x @ keys * scale).masked_fill_(~seen, -float("inf"))
        w = (z - z.amax(-1, keepdim=True).clamp(min=-1e300)).exp()
        w /= w.sum(-1, keepdim=True).clamp(min=1e-300)            # rows before the start see nothing
        largest = (x.abs() @ keys.abs() * abs(scale)).masked_fill_(~seen, 0).amax(-1, keepdim=True)
        out += w.sum(0)
        size += (w * largest).sum(0)
    return out, size


def _check(lens, news, heads, group, dim, page=64, window=0, decay=0.9, places=None, table_tokens=None, extra_rows=0, slack=0,
           in_place=False, seed=1):
    """Checks every place of the result, that a second run in a workspace with other contents gives the same bits, and
    that nothing is written behind a workspace of just the size asked for.  Returns the plan."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    seqs, rows, q_heads, max_new = len(lens), int(sum(news)), heads * group, int(max(news)) + slack
    places, width = places or max(lens), _up(table_tokens or max(lens), page)
    pool = 48
    k = (torch.randn((pool, heads, page, dim), device="cuda", generator=gen) * 30).round().clamp(-127, 127).to(torch.int8)
    v = torch.zeros((pool, heads, page // 16, dim, 16), dtype=torch.int8, device="cuda")
    scales = (0.8 + 0.4 * torch.rand((pool, heads, 2), device="cuda", generator=gen)) * (4.2 / 127)
    table = torch.from_numpy(rng.integers(0, pool, (seqs, width)).astype(np.int32)).cuda()
    cache = tt.make_kv_cache(k, v, scales, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    at = torch.from_numpy(starts).cuda()
    q = (2 * torch.randn((rows + extra_rows, q_heads, dim), device="cuda", generator=gen)).half()
    mass = torch.rand((seqs, heads, places), device="cuda", generator=gen)
    size = tt.kv_weigh_workspace(cache, rows + extra_rows, q_heads).numel()
    got = []
    for fill in (255, 0):
        space = torch.full((size + 4096,), fill, dtype=torch.uint8, device="cuda")
        out = mass.clone() if in_place else torch.full_like(mass, -7.0)
        tt.kv_weigh(cache, q, at, max_new, out if in_place else mass, out, space[:size], window=window, decay=decay)
        torch.cuda.synchronize()
        assert torch.all(space[size:] == fill)
        got.append(out)
    assert torch.equal(got[0].view(torch.int32), got[1].view(torch.int32))
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    plan = _plan(lens, news, heads, group, dim, places, cus, max_new)
    worst = 0.0
    for i, (n, m) in enumerate(zip(lens, news)):
        held = min(n, width * page)
        pages, shown = table[i].long(), min(n, places)
        past = torch.zeros((heads, shown), dtype=torch.float64, device="cuda")
        old = min(max(0, n - m), shown)
        past[:, :old] = mass[i, :, :old].double() * (float(np.float32(decay)) if m else 1.0)
        for h in range(heads):
            want, err = (torch.zeros(shown, dtype=torch.float64, device="cuda") for _ in range(2))
            if m:
                keys, units = k[pages, h].reshape(-1, dim)[:held], scales[pages, h, 0].repeat_interleave(page)[:held]
                x = q[starts[i]:starts[i + 1], h * group:(h + 1) * group]
                w, e = _want(x, keys, units, n - m, held, dim ** -0.5, window)
                want[:min(held, shown)], err[:min(held, shown)] = w[:shown], e[:shown]
            path = 20 * plan.span[i] * (plan.block // 64) + 4 * plan.spans[i] + 64 + _up(m * group, 32) + 64
            bound = err * 2 * (dim + 4) * 2.0 ** -24 + want * (2.0 ** -20 + path * 2.0 ** -24) + past[h] * 2.0 ** -22 + 1e-35
            if shown:
                diff = (got[0][i, h, :shown].double() - want - past[h]).abs()
                assert not torch.isnan(diff).any()
                worst = max(worst, float((diff / bound).max()))
        rest = got[0][i, :, shown:]
        assert torch.equal(rest, mass[i, :, shown:] if in_place else torch.full_like(rest, -7.0))
    print(f"[plan] dim={dim} heads={q_heads}/{heads} seqs={seqs} rows={rows} longest={max(lens)} window={window} few={plan.few} "
          f"keep={plan.keep} chunk={plan.chunk} span={max(plan.span)} items={plan.items} worst {worst:.4f} of the bound", flush=True)
    assert worst <= 1.0
    return plan


def _ragged(seed, seqs, most, least=1):
    return [int(n) for n in np.random.default_rng(seed).integers(least, most + 1, seqs - 1)] + [most]


# ------------------------------------------------------------------ single tokens

@pytest.mark.parametrize("window", [0, 1000])
@pytest.mark.parametrize("heads,group,dim,seqs,most", [(8, 5, 128, 9, 9000), (4, 20, 64, 18, 7000), (1, 16, 128, 3, 90001)])
def test_single_tokens_spans_of_several_blocks(heads, group, dim, seqs, most, window):
    """Keys on their way over blocks of a span, running maxima and sums; one and two tiles of rows."""
    plan = _check(_ragged(2, seqs, most, most // 2), [1] * seqs, heads, group, dim, window=window)
    assert plan.few and plan.keep and max(plan.span) > 1 and plan.two == (group == 20)


@pytest.mark.parametrize("window", [0, 5000])
@pytest.mark.parametrize("heads,group,dim,seqs,most,new", [(1, 16, 128, 10, 131072, 1), (8, 7, 64, 50, 8192, 1),
                                                           (2, 16, 64, 7, 70000, 2), (1, 5, 64, 6, 300000, 6)])
def test_single_tokens_without_room_for_their_scores(heads, group, dim, seqs, most, new, window):
    """The second pass finds the scores again: one and two tiles of rows, a window, drafts of several tokens."""
    news = [new] * (seqs - 2) + [1, new]
    plan = _check(_ragged(3, seqs, most, most * 4 // 5), news, heads, group, dim, page=128, window=window)
    assert plan.few and not plan.keep and max(plan.span) > 1 and plan.two == (new * group > 16)


def test_a_step_of_64_long_sequences():
    """A decode step of ordinary size whose scores find no room, with sequences that wait."""
    news = [1] * 64
    news[5] = news[40] = 0
    plan = _check(_ragged(4, 64, 8192, 6000), news, 8, 5, 128, page=32)
    assert plan.few and not plan.keep and max(plan.span) > 1


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dim,group", [(128, 3), (64, 30)])
def test_single_tokens_of_more_items_than_waves(dim, group, in_place):
    news = [int(n) for n in np.random.default_rng(5).integers(0, 8, 700) > 0]
    plan = _check(_ragged(5, 700, 200), news, 8, group, dim, page=16, in_place=in_place)
    assert plan.few and plan.items > plan.workers


# ------------------------------------------------------------------ prompts

@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("heads,group,dim", [(8, 3, 128), (8, 5, 64), (8, 8, 128), (6, 40, 64)])
def test_prompts_of_several_tiles_an_item(heads, group, dim, window):
    """Rows through both buffers, heads of a cache head that divide a tile, do not, and are more than one."""
    rows = 400 if group == 40 else 2048
    plan = _check([rows + 133, 2049, 70], [rows, 31, 0], heads, group, dim, window=window)
    assert not plan.few and plan.chunk > 1


@pytest.mark.parametrize("window", [0, 1500])
def test_prompts_of_more_tiles_than_the_first_pass_holds(window):
    """The two passes cut the rows apart differently."""
    plan = _check([4096], [4096], 8, 5, 64, window=window)
    assert not plan.few and plan.chunk > 16


@pytest.mark.parametrize("window", [0, 400, 9000])
@pytest.mark.parametrize("dim,group", [(128, 3), (64, 4)])
def test_prompts_over_long_contexts(dim, group, window):
    """Spans of several blocks, of which a window leaves some out."""
    plan = _check([20000, 33001, 257], [300, 33, 200], 2, group, dim, page=128, window=window)
    assert not plan.few and max(plan.span) > 1 and plan.chunk > 1


@pytest.mark.parametrize("group", [1, 3])
def test_prompts_of_more_sequences_than_lanes(group):
    rng = np.random.default_rng(6)
    news = [int(n) for n in rng.integers(0, 60, 150)]
    lens = [n + int(rng.integers(0, 600)) for n in news]
    plan = _check(lens, news, 2, group, 128, page=16, slack=9)
    assert not plan.few


# ------------------------------------------------------------------ the workspace

def _sizes(seqs, kv_heads, dim, tokens, page=64):
    c = tt.KVCache()
    c.num_pages, c.page_tokens, c.kv_heads, c.head_dim, c.seqs, c.max_pages = 10, page, kv_heads, dim, seqs, _up(tokens, page)
    return c


def test_workspace_is_what_a_call_can_use():
    """Not the most that any call could: a prompt's 64 spans of the table's blocks, a short sequence's scores."""
    import ctypes

    def size(rows, q_heads, *sizes):
        cache = _sizes(*sizes)
        return tt.library().tetra_kv_weigh_workspace_bytes(ctypes.addressof(cache), rows, q_heads)

    assert 0 < size(1, 32, 1, 8, 128, 203) <= 1 << 17
    # 64 MiB of scores (the rows may be three a sequence: 8 * 64 * 64 blocks * 64 * 15 are more), and the spans of 64 rows
    assert size(64, 40, 64, 8, 128, 4096) <= (64 << 20) + 64 * 40 * (64 * 8 + 4) + 512
    assert size(64, 40, 64, 8, 128, 131072) <= (64 << 20) + 64 * 40 * (256 * 8 + 4) + 512
    assert size(16, 40, 16, 8, 128, 2048) <= 16 * 8 * 32 * 64 * 15 * 4 + 16 * 40 * (32 * 8 + 4) + 512
    assert size(4096, 32, 1, 8, 128, 4096) <= 32 << 20
    # scores of three rows of five heads over the table: 15.7 MB
    assert size(32768, 40, 1, 8, 128, 32768) <= 32768 * 40 * (64 * 8 + 4) + 8 * 32768 * 15 * 4 + 512
    # one for many rows serves fewer
    for cache in ((1, 8, 128, 203), (3, 2, 64, 100000), (64, 8, 128, 4096)):
        for q_heads in (8, 40, 320):
            sizes = [size(n, q_heads, *cache) for n in (1, 2, 3, 4, 5, 15, 16, 17, 31, 32, 33, 64, 200, 1000, 5000)]
            assert sizes == sorted(sizes)


@pytest.mark.parametrize("dim,group", [(128, 5), (64, 20)])
def test_rows_far_past_the_last_start(dim, group):
    """As in a graph captured for a larger batch: the spans of the rows that count are longer then."""
    plan = _check([40000, 33], [1, 1], 2, group, dim, extra_rows=700)
    assert plan.few


@pytest.mark.parametrize("news", [(1, 1), (60, 300)])
def test_lengths_and_places_far_past_the_table(news):
    """What the table does not hold gets no weight and keeps what it had, in a workspace of the table's size."""
    _check([90000, 5000], list(news), 2, 4, 128, table_tokens=700, places=100000)
    _check([300000, 200], list(news), 1, 3, 64, table_tokens=400, places=200000, in_place=True)
