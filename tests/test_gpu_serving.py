"""Cache append, attention and sampling on the GPU against float64 (run on an MI355X).

Bounds, from the formats:
* a value stored in 8 bits is off by half a unit of its page's scale, s / 2, plus the float32 arithmetic before it
  (rotation and norm: a few 2^-24 of a value of at most 127 units, below 1e-3 unit); a value rounded again on a
  grown scale by half a unit of the new one;
* scales are fp32 quotients of fp32 values that went through a norm and a rotation: 1e-6 relative to the largest
  input of a rotated pair (three or four roundings of 2^-24);
* q out: one fp16 rounding, 2^-11, and the float32 arithmetic, 1e-6 of the pair's size;
* attention: fp16 output, 2^-11 |o|; a weight rounded to fp16, 2^-11 of sum w |v|; and scores of magnitude S in
  float32 over D products, whose error 2^-24 sqrt(D) S moves the weights by less than another 2^-12 for S < 100;
* sampled tokens: equal.
"""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2609_35465_amd as tt  # noqa: E402
from oracle import serving as ref  # noqa: E402

EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    torch.cuda.init()


_WS = []


def _workspace():
    if not _WS:
        _WS.append(tt.kv_attend_workspace())
    return _WS[0]


def _dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


class Cache:
    """A pool on the device with its host copies; pages of the sequences in a shuffled order."""

    def __init__(self, seed, lens, heads, page, dim, max_pages=None, spare=3, table=None):
        rng = self.rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in lens]
        pages = sum(need) + spare
        self.max_pages = max_pages or max(1, max(need))
        self.table = np.full((len(lens), self.max_pages), -1, np.int32)
        order = rng.permutation(pages)
        at = 0
        for i, n in enumerate(need):
            n = min(n, self.max_pages)
            self.table[i, :n] = order[at:at + n]
            at += n
        if table is not None:
            self.table = table
        self.lens, self.heads, self.page, self.dim = np.array(lens, np.int32), heads, page, dim
        self.k = np.clip(np.rint(rng.standard_normal((pages, heads, page, dim)) * 30), -127, 127).astype(np.int8)
        self.v = np.clip(np.rint(rng.standard_normal((pages, heads, page // 16, dim, 16)) * 30), -127, 127).astype(np.int8)
        self.scales = (rng.uniform(0.8, 1.2, (pages, heads, 2)) * 4.2 / 127).astype(np.float32)

    def upload(self):
        self.d = [_dev(a) for a in (self.k, self.v, self.scales, self.table, self.lens)]
        return tt.make_kv_cache(*self.d)

    def download(self):
        return [t.cpu().numpy() for t in self.d[:3]]

    def sequence(self, i, k=None, v=None, scales=None):
        return ref.sequence(self.k if k is None else k, self.v if v is None else v,
                            self.scales if scales is None else scales, self.table[i], int(self.lens[i]))


def _starts(news):
    return np.concatenate([[0], np.cumsum(news)]).astype(np.int32)


# ------------------------------------------------------------------ append

def _check_append(c, news, q_heads, half=False, norm=False, rotate=True, spoil=None, strided=False, slack=0, seed=1):
    """Appends, then checks every page byte by byte against what may be there."""
    rng = np.random.default_rng(seed)
    news = np.array(news)
    starts, rows, D, H, B = _starts(news), int(sum(news)), c.dim, c.heads, c.page
    kind = np.float16 if half else np.float32
    k, v, q = (rng.standard_normal((rows, n, D)).astype(kind) for n in (H, H, q_heads))
    if spoil is not None:
        spoil(k, v)
    qn, kn = ((1 + 0.2 * rng.standard_normal((2, D))).astype(np.float32) if norm else (None, None))
    rope = tt.rope_table(int(max(1, c.lens.max())), D) if rotate else None
    cache = c.upload()

    def dev(x):
        if not strided:
            return _dev(x)
        wide = torch.zeros((rows, x.shape[1] * D + 24), dtype=torch.from_numpy(x).dtype, device="cuda")
        wide[:, 16:16 + x.shape[1] * D] = _dev(x).flatten(1)
        return wide[:, 16:16 + x.shape[1] * D]

    out = torch.full((rows, q_heads, D), float("nan"), dtype=torch.float16, device="cuda")
    tt.kv_append(cache, dev(q), dev(k), dev(v), _dev(starts), int(news.max()) + slack, rope, out,
                 None if qn is None else _dev(qn), None if kn is None else _dev(kn), EPS)
    torch.cuda.synchronize()
    k1, v1, s1 = c.download()
    touched = set()
    got_q = out.cpu().numpy().astype(np.float64)
    for i, n in enumerate(news):
        L, first = int(c.lens[i]), int(c.lens[i]) - int(n)
        if n == 0:
            continue
        mine = slice(starts[i], starts[i + 1])
        position = np.arange(first, L) if rotate else None
        want = ref.norm_and_rotate(q[mine], qn, EPS, position)
        size = np.hypot(*np.split(want, 2, -1))
        size = np.concatenate([size, size], -1)
        assert np.all(np.abs(got_q[mine] - want) <= 2.0 ** -11 * np.abs(want) + 1e-6 * size + 2.0 ** -25)
        with np.errstate(invalid="ignore"):
            new = (ref.norm_and_rotate(k[mine], kn, EPS, position), v[mine].astype(np.float64))
        for j in range(first // B, -(-L // B)):
            if j >= c.max_pages or not 0 <= c.table[i, j] < len(c.k):
                continue
            page = c.table[i, j]
            touched.add(int(page))
            lo, hi = max(first, j * B), min(L, (j + 1) * B)
            old = lo - j * B
            for which, x in enumerate(new):
                q1 = k1[page] if which == 0 else v1[page].transpose(0, 1, 3, 2).reshape(H, B, D)
                q0 = c.k[page] if which == 0 else c.v[page].transpose(0, 1, 3, 2).reshape(H, B, D)
                s, s0 = s1[page, :, which].astype(np.float64), c.scales[page, :, which].astype(np.float64)
                x = x[lo - first:hi - first].transpose(1, 0, 2)
                fine = np.isfinite(x)
                largest = np.abs(np.where(fine, x, 0)).max((1, 2)) / 127
                largest[largest < 1e-30] = 0
                want_s = np.maximum(largest, s0) if old else largest
                # a pair's rotation errs by the pair's size, at most sqrt(2) of the largest value
                assert np.all(np.abs(s - want_s) <= 2e-6 * want_s), (i, j, which)
                assert not old or np.all(s >= s0)
                value = q1[:, old:old + hi - lo].astype(np.float64)
                unit = np.where(s > 0, s, 1)[:, None, None]
                assert np.all(np.abs(value - np.where(fine, x, 0) / unit)[fine] <= 0.5 + 1e-3)
                zero = np.broadcast_to((s == 0)[:, None, None], value.shape)
                assert np.all(value[np.isnan(x) | zero] == 0)
                assert np.all(value[np.isinf(x) & ~zero] == 127 * np.sign(x[np.isinf(x) & ~zero]))
                if old:
                    grew = (s != s0)[:, None, None]
                    again = q0[:, :old].astype(np.float64) * (s0 / np.where(s > 0, s, 1))[:, None, None]
                    kept = q1[:, :old].astype(np.float64)
                    assert np.all(np.where(grew, np.abs(kept - again) <= 0.5 + 1e-3, kept == q0[:, :old])), (i, j, which)
                    assert np.all(np.abs(kept) <= 127)
    for page in set(range(len(c.k))) - touched:
        assert np.array_equal(k1[page], c.k[page]) and np.array_equal(v1[page], c.v[page])
        assert np.array_equal(s1[page].view(np.uint32), c.scales[page].view(np.uint32))
    return cache


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("half,norm", [(False, True), (True, False)])
def test_append_single_tokens(dim, page, half, norm):
    """Lengths on both sides of page and group ends, a first token, an idle slot."""
    lens = [1, 2, 16, 17, page - 1, page, page + 1, 3 * page + 5, 0, 200]
    print(f"[append 1] dim={dim} page={page}", flush=True)
    _check_append(Cache(3, lens, 3, page, dim), [1, 1, 1, 1, 1, 1, 1, 1, 0, 1], 6, half, norm)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("slack", [0, 70])
def test_append_chunks(dim, page, slack):
    """Prompts from the start, chunks into the middle of pages, whole pages, single tokens and none, together."""
    news = [70, 1, 0, 2 * page, 3, page + 1, 33, 16]
    lens = [70, 50, 0, 2 * page, 18, 2 * page + 1, 33 + page - 1, 48]
    print(f"[append chunks] dim={dim} page={page} slack={slack}", flush=True)
    _check_append(Cache(4, lens, 2, page, dim), news, 5, slack % 4 == 0, slack == 0, slack=slack)


@pytest.mark.parametrize("heads,q_heads", [(1, 1), (8, 40), (5, 35), (2, 128)])
def test_append_heads_and_strides(heads, q_heads):
    c = Cache(5, [40, 21], heads, 32, 128)
    print(f"[append heads] {heads} {q_heads}", flush=True)
    _check_append(c, [9, 21], q_heads, strided=True, norm=True)


def test_append_many_sequences():
    """More sequences than a wave has lanes, idle ones among them."""
    rng = np.random.default_rng(0)
    news = rng.integers(0, 4, 150)
    lens = [int(n + rng.integers(0, 90)) if n else int(rng.integers(0, 2)) * 40 for n in news]
    print("[append many]", flush=True)
    _check_append(Cache(6, lens, 1, 16, 64), news, 2)


def test_append_without_rotation_or_q():
    c = Cache(7, [30], 2, 16, 64)
    print("[append plain]", flush=True)
    _check_append(c, [30], 2, rotate=False)
    cache = c.upload()
    k = _dev(np.ones((30, 2, 64), np.float32))
    tt.kv_append(cache, None, k, k, _dev(_starts([30])), 30, None, None)
    kb, vb = (torch.empty((1, 30, 2, 64), dtype=torch.float16, device="cuda") for _ in "kv")
    tt.kv_read(cache, 30, kb, vb)
    assert torch.all(kb == 1) and torch.all(vb == 1)


def test_append_ignores_what_a_reused_page_held():
    """A page that starts afresh takes nothing from its last use: huge, NaN and zero scales."""
    c = Cache(8, [20, 16, 5], 2, 16, 128)
    c.scales[:] = np.array([1e30, np.nan, 0, np.inf], np.float32)[np.arange(c.scales.size) % 4].reshape(c.scales.shape)
    print("[append reuse]", flush=True)
    _check_append(c, [20, 16, 5], 3)


def test_append_not_finite_and_zero_values():
    def spoil(k, v):
        k[3, 0, 5], k[4, 0, 6], k[5, 1, 7] = np.nan, np.inf, -np.inf
        v[2, 0, 1], v[6, 1, 2], v[7, 1, 63] = np.nan, np.inf, -np.inf
        k[16:32], v[16:32] = 0, 0
        v[32:48] = 1e-35
    c = Cache(9, [50], 2, 16, 64)
    print("[append spoilt]", flush=True)
    _check_append(c, [50], 2, rotate=False, spoil=spoil)


def test_append_zero_page_then_values():
    """A page of zeros (scale 0) whose scale grows from nothing."""
    c = Cache(10, [3], 1, 16, 64)
    cache = c.upload()
    zero, some = (_dev(np.full((n, 1, 64), x, np.float32)) for n, x in ((3, 0.0), (2, 2.0)))
    one, two = _dev(_starts([3])), _dev(_starts([2]))
    tt.kv_append(cache, None, zero, zero, one, 3, None, None)
    c.d[4].fill_(5)
    tt.kv_append(cache, None, some, some, two, 2, None, None)
    kb, vb = (torch.empty((1, 5, 1, 64), dtype=torch.float16, device="cuda") for _ in "kv")
    tt.kv_read(cache, 5, kb, vb)
    want = torch.tensor([0, 0, 0, 2, 2], device="cuda").view(1, 5, 1, 1)
    assert torch.all(kb == want) and torch.all(vb == want)


def test_append_outside_the_pool_is_dropped():
    """Page ids that are none, and lengths past the table: the rest is as without them."""
    c = Cache(11, [40, 40, 60], 2, 16, 64, max_pages=3)
    c.table[0, 1], c.table[1, 2] = -1, len(c.k)
    print("[append outside]", flush=True)
    _check_append(c, [40, 3, 30], 2)


def test_append_clamps_bad_rows():
    """Starts past the rows and lengths shorter than the new rows stay inside the arrays."""
    c = Cache(12, [4, 8], 1, 16, 64)
    cache = c.upload()
    x = _dev(np.ones((10, 1, 64), np.float32))
    out = torch.zeros((10, 1, 64), dtype=torch.float16, device="cuda")
    for starts in ([0, 10, 99], [-5, 3, 2], [7, 3, 10], [0, 1 << 30, -(1 << 31)]):
        tt.kv_append(cache, x, x, x, _dev(np.array(starts, np.int32)), 10, tt.rope_table(4, 64), out)
        tt.kv_attend(cache, out, _dev(np.array(starts, np.int32)), 10, torch.empty_like(out), _workspace())
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()


def test_append_token_by_token_stays_near():
    """A sequence appended one token a call: each growth of a scale rounds again, half a unit at most; a page of
    32 tokens of growing size grows 32 times, and an old value is off by half a unit of every scale it had."""
    c = Cache(13, [0], 2, 32, 128)
    c.table[0, 0] = 0
    cache = c.upload()
    rng = np.random.default_rng(3)
    x = rng.standard_normal((32, 2, 128)).astype(np.float32) * np.linspace(1, 3, 32)[:, None, None].astype(np.float32)
    at = _dev(_starts([1]))
    for i in range(32):
        c.d[4].fill_(i + 1)
        tt.kv_append(cache, None, _dev(x[i:i + 1]), _dev(x[i:i + 1]), at, 1, None, None)
    kb, vb = (torch.empty((1, 32, 2, 128), dtype=torch.float16, device="cuda") for _ in "kv")
    tt.kv_read(cache, 32, kb, vb)
    sofar = np.maximum.accumulate(np.abs(x).max(2), 0) / 127         # the scale after each token
    for t in range(32):
        bound = 0.5 * sofar[t:].sum(0) * (1 + 1e-3) + 2.0 ** -11 * np.abs(x[t]).max(1)
        for b in (kb, vb):
            assert np.all(np.abs(b[0, t].cpu().numpy().astype(np.float64) - x[t]).max(1) <= bound), t


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 128), (128, 32)])
@pytest.mark.parametrize("count", [1, 16, 37])
def test_read_matches_pages(dim, page, count):
    c = Cache(14, [5, 0, 37, 300], 3, page, dim)
    c.table[2, 0] = -1
    cache = c.upload()
    kb, vb = (torch.full((4, count, 3, dim), float("nan"), dtype=torch.float16, device="cuda") for _ in "kv")
    print(f"[read] dim={dim} page={page} count={count}", flush=True)
    tt.kv_read(cache, count, kb, vb)
    for i in range(4):
        for got, x in zip((kb, vb), c.sequence(i)[:2]):
            want = np.zeros((count, 3, dim))
            tail = x[-count:] if len(x) else x
            want[count - len(tail):] = tail
            want = want.astype(np.float32)                          # products of whole numbers and an fp32 scale
            got_i = got[i].cpu().numpy().astype(np.float64)
            assert np.all(np.abs(got_i - want) <= 2.0 ** -11 * np.abs(want) * (1 + 1e-6))


# ------------------------------------------------------------------ attention

def _check_attend(c, news, q_heads, window=0, scale=None, q_size=2.0, strided=False, slack=0, seed=2):
    rng = np.random.default_rng(seed)
    starts, rows = _starts(news), int(sum(news))
    q = (rng.standard_normal((rows, q_heads, c.dim)) * q_size).astype(np.float16)
    cache = c.upload()
    width = q_heads * c.dim
    if strided:
        qd = torch.zeros((rows, width + 40), dtype=torch.float16, device="cuda")[:, 32:32 + width]
        qd.copy_(_dev(q).flatten(1))
        wide = torch.full((rows, width + 16), 7.0, dtype=torch.float16, device="cuda")
        out = wide[:, 8:8 + width]
    else:
        qd, out = _dev(q), torch.full((rows, q_heads, c.dim), float("nan"), dtype=torch.float16, device="cuda")
    tt.kv_attend(cache, qd, _dev(starts), int(max(news)) + slack, out, _workspace(), scale, window)
    again = torch.full_like(out, float("nan"))
    tt.kv_attend(cache, qd, _dev(starts), int(max(news)) + slack, again, _workspace(), scale, window)
    torch.cuda.synchronize()
    assert torch.equal(out.contiguous().view(torch.int16), again.contiguous().view(torch.int16))
    if strided:
        assert torch.all(wide[:, :8] == 7) and torch.all(wide[:, 8 + width:] == 7)
    got = out.reshape(rows, q_heads, c.dim).cpu().numpy().astype(np.float64)
    worst = 0.0
    for i, n in enumerate(news):
        if n == 0:
            continue
        ks, vs, there = c.sequence(i)
        want, size = ref.attend(q[starts[i]:starts[i + 1]], ks, vs, there, int(c.lens[i]) - int(n),
                                c.dim ** -0.5 if scale is None else scale, window)
        bound = 2.0 ** -11 * np.abs(want) + 1.5 * 2.0 ** -11 * size + 2.0 ** -24
        worst = max(worst, float((np.abs(got[starts[i]:starts[i + 1]] - want) / bound).max()))
    print(f"[attend] dim={c.dim} page={c.page} heads={q_heads}/{c.heads} news={list(news)[:6]} window={window} "
          f"worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0
    return got


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attend_single_tokens(dim, page):
    """Lengths of one and around 16, 64, 256 and page ends, an idle slot."""
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 0, 255, 256, 257, page, 2 * page + 1, 700]
    _check_attend(Cache(20, lens, 2, page, dim), [int(n > 0) for n in lens], 8)


@pytest.mark.parametrize("heads,q_heads", [(1, 1), (8, 40), (2, 14), (4, 4), (1, 16), (1, 17), (2, 80)])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_head_layouts(heads, q_heads, dim):
    _check_attend(Cache(21, [300, 77], heads, 32, dim), [1, 1], q_heads)


@pytest.mark.parametrize("news", [(2, 3, 1), (3, 0, 4), (16, 5, 1), (17, 1, 1)])
@pytest.mark.parametrize("group", [1, 5, 8])
def test_attend_few_tokens(news, group):
    lens = [n + 90 * i for i, n in enumerate(news)]
    _check_attend(Cache(22, lens, 2, 16, 128), news, 2 * group)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("group", [1, 5])
def test_attend_prompts(dim, page, group):
    """Whole prompts, chunks after a context, and single tokens in one call."""
    news = [65, 130, 1, 0, 33, 7]
    lens = [65, 130, 400, 0, 300, 7]
    _check_attend(Cache(23, lens, 2, page, dim), news, 2 * group)
    _check_attend(Cache(23, lens, 2, page, dim), news, 2 * group, slack=100, strided=True)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 200, 5000])
@pytest.mark.parametrize("news", [(1, 1, 1), (130, 1, 70)])
def test_attend_windows(window, news):
    lens = [500, 3, 333]
    lens = [max(a, b) for a, b in zip(lens, news)]
    _check_attend(Cache(24, lens, 2, 32, 128), news, 10, window=window)


@pytest.mark.parametrize("seqs", [257, 600])
@pytest.mark.parametrize("prompts", [False, True])
def test_attend_many_sequences(seqs, prompts):
    """More sequences than a workgroup scans at once, idle ones and (in some) prompts among them."""
    rng = np.random.default_rng(seqs)
    news = rng.integers(0, 3, seqs)
    if prompts:
        news[rng.integers(0, seqs, 6)] = rng.integers(40, 150, 6)
    lens = [int(n + rng.integers(0, 500) * (n > 0)) for n in news]
    _check_attend(Cache(34, lens, 1, 16, 64), news, 2)


@pytest.mark.parametrize("news,rows", [((60, 2), 120), ((1, 0, 1), 3), ((300, 1, 0), 900), ((7, 3), 14)])
def test_attend_rows_past_the_last_start(news, rows):
    """Fewer rows in use than the buffers hold, as where a graph is captured for a full batch: the used ones come out
    as ever, the others stay untouched."""
    lens = [n + 40 * (n > 0) for n in news]
    c = Cache(35, lens, 2, 16, 128)
    want = _check_attend(c, news, 8)
    used = sum(news)
    q = np.zeros((rows, 8, 128), np.float16)
    q[:used] = (np.random.default_rng(2).standard_normal((used, 8, 128)) * 2).astype(np.float16)
    out = torch.full((rows, 8, 128), 7.0, dtype=torch.float16, device="cuda")
    tt.kv_attend(c.upload(), _dev(q), _dev(_starts(news)), rows // len(news), out, _workspace())
    got = out.cpu().numpy()
    assert np.all(got[used:] == 7)
    # the split of the keys may differ with the rows' count: two fp16 roundings and those of the weights
    assert np.all(np.abs(got[:used].astype(np.float64) - want) <= 2.0 ** -9 * np.abs(want) + 2.0 ** -8)


@pytest.mark.parametrize("news", [(1, 3), (10, 5), (100, 64)])
@pytest.mark.parametrize("window", [1, 200, (1 << 31) - 1])
def test_attend_windows_and_lengths_up_to_the_type_s_end(news, window):
    """The largest window is none, also for rows before a sequence's start; of a length far past the table the tokens
    in the table are seen, as far as the window reaches back to them."""
    c = Cache(37, [480, 480], 2, 16, 64)
    c.lens[:] = [news[0] // 2, news[1] - 2]
    got = _check_attend(c, news, 4, window=window)
    assert np.all(got[:news[0] - news[0] // 2] == 0)
    c.lens[:] = 480
    rows = sum(news)
    q = _dev(np.random.default_rng(4).standard_normal((rows, 4, 64)).astype(np.float16))
    all_seen, far = (torch.full_like(q, float("nan")) for _ in range(2))
    cache = c.upload()
    c.d[4].fill_(480 + max(news))
    tt.kv_attend(cache, q, _dev(_starts(news)), max(news), all_seen, _workspace())
    c.d[4].fill_((1 << 31) - 1)
    print(f"[attend far lengths] news={news} window={window}", flush=True)
    tt.kv_attend(cache, q, _dev(_starts(news)), max(news), far, _workspace(), window=window)
    assert torch.equal(far, all_seen if window > 1 << 30 else torch.zeros_like(q))


def _attend_rows(c, q, news, window=0):
    """out of rows q [rows, heads, dim] (fp16) over c, and the oracle's (out, size), one array each."""
    out = torch.full(q.shape, float("nan"), dtype=torch.float16, device="cuda")
    tt.kv_attend(c.upload(), _dev(q), _dev(_starts(news)), int(max(news)), out, _workspace(), window=window)
    starts, want, size = _starts(news), [], []
    for i, n in enumerate(news):
        w, s = ref.attend(q[starts[i]:starts[i + 1]], *c.sequence(i), int(c.lens[i]) - int(n), c.dim ** -0.5, window)
        want.append(w)
        size.append(s)
    return out.cpu().numpy().astype(np.float64), np.concatenate(want), np.concatenate(size)


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 32)])
@pytest.mark.parametrize("news,lens", [((6, 1), (35, 30)), ((100, 64), (100, 64)), ((100, 1), (100, 31))])
@pytest.mark.parametrize("window", [0, 9])
@pytest.mark.parametrize("power", [26, 60])
def test_attend_large_page_that_a_row_does_not_see(dim, page, news, lens, window, power):
    """Values 2^26 and 2^60 times as large from token 32 on, in the tile that holds the earlier tokens too: a row
    before them, or (with the window) past them, keeps its precision."""
    c = Cache(39, lens, 2, page, dim)
    for i in range(2):
        if lens[i] > 32:
            c.scales[c.table[i, 32 // page], :, 1] *= np.float32(2.0 ** power)
    q = (c.rng.standard_normal((sum(news), 8, dim)) * 2).astype(np.float16)
    got, want, size = _attend_rows(c, q, news, window)
    position = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, news)])
    apart = (position < 32) | ((position >= 32 + page + window) if window else False)
    assert apart.any()
    bound = 2.0 ** -11 * np.abs(want) + 1.5 * 2.0 ** -11 * size + 2.0 ** -24
    worst = float((np.abs(got - want) / bound)[apart].max())
    print(f"[attend large page] dim={dim} page={page} news={news} window={window} 2^{power} worst {worst:.3f}", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("news,lens", [((1, 3), (100, 300)), ((100, 70), (100, 300))])
@pytest.mark.parametrize("power", [26, 40])
def test_attend_large_page_without_weight(dim, page, news, lens, power):
    """A page of values 2^26 and 2^40 times as large whose keys lie against every q, so that its weights are below
    2^-80 of the others' sum: the output is the others' mean to its last bits."""
    c = Cache(40, lens, 2, page, dim)
    for i in range(2):
        p = c.table[i, 0]
        c.scales[p, :, 1] *= np.float32(2.0 ** power)
        c.k[p] = -127
        c.scales[p, :, 0] = 8.0 * (128 / dim) ** 0.5 / 127
    rng = c.rng
    q = np.maximum(np.abs(rng.standard_normal((sum(news), 8, dim)) * 2), 0.5).astype(np.float16)
    got, want, size = _attend_rows(c, q, news)
    position = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, news)])
    others = position >= page                 # the rows that see another page too
    scores = -8.0 * (128 / dim) ** 0.5 * q.astype(np.float64).sum(-1) * dim ** -0.5 / np.log(2)
    assert scores.max() < -130                 # the others' best are above -40: at most 2^-90 of them, times 2^40
    bound = 2.0 ** -11 * np.abs(want) + 1.5 * 2.0 ** -11 * size + 2.0 ** -24
    worst = float((np.abs(got - want) / bound)[others].max())
    print(f"[attend page without weight] dim={dim} page={page} news={news} 2^{power} worst {worst:.3f}", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("news", [(5, 1), (100, 90)])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("sign", [-1, 0, 1])
def test_attend_not_finite_queries_over_keys_of_one_sign(news, bad, sign):
    """Keys that all have one sign (or nothing) where q is not finite, so that every score may be -inf, from the row
    that sees one key on: NaN all the same, and zeros where a row sees no key."""
    c = Cache(41, news, 2, 16, 64)
    c.k[..., 7] = sign * 90
    starts, rows = _starts(news), sum(news)
    q = c.rng.standard_normal((rows, 8, 64)).astype(np.float16)
    spoilt = np.array([0, 2, news[0] - 1, news[0]])
    q[spoilt, 5, 7] = bad
    out = torch.zeros((rows, 8, 64), dtype=torch.float16, device="cuda")
    cache = c.upload()
    tt.kv_attend(cache, _dev(q), _dev(starts), max(news), out, _workspace())
    got = out.cpu().numpy()
    mine = np.zeros((rows, 8), bool)
    mine[spoilt, 5] = True
    assert np.isnan(got[mine]).all() and np.isfinite(got[~mine]).all()
    c.d[4].copy_(torch.tensor([news[0] - 1, 0], dtype=torch.int32))      # the first rows see nothing now
    tt.kv_attend(cache, _dev(q), _dev(starts), max(news), out, _workspace())
    got = out.cpu().numpy()
    assert np.all(got[0] == 0) and np.all(got[news[0]:] == 0) and np.isnan(got[2, 5]).all()


@pytest.mark.parametrize("news,most", [((3, 1), 1), ((5, 9), 4), ((100, 30, 2), 40), ((90, 120), 100)])
def test_rows_past_max_new_are_ignored(news, most):
    """Sequences of more rows than max_new: the rows before it are appended and attend at the positions that `starts`
    and the lengths give them, as in a call that takes all rows; the rows past it leave nothing."""
    lens = [n + 37 * i + 5 for i, n in enumerate(news)]
    c, rows = Cache(42, lens, 2, 16, 64), sum(news)
    rope, starts = tt.rope_table(max(lens), 64), _dev(_starts(news))
    q, k, v = (_dev(c.rng.standard_normal((rows, n, 64)).astype(np.float32)) for n in (4, 2, 2))
    taken = np.concatenate([np.arange(n) < most for n in news])
    print(f"[past max_new] news={news} max_new={most}", flush=True)
    got = []
    for m in (max(news), most):
        cache = c.upload()
        turned, out = (torch.full((rows, 4, 64), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
        tt.kv_append(cache, q, k, v, starts, m, rope, turned)
        pool = c.download()
        tt.kv_attend(c.upload(), turned, starts, m, out, _workspace())
        got.append((turned.cpu().numpy(), out.cpu().numpy(), pool))
    (turned, out, pool), (turned1, out1, pool1) = got
    assert np.array_equal(turned1[taken], turned[taken]) and np.all(turned1[~taken] == 7) and np.all(out1[~taken] == 7)
    # the split of the keys may differ with max_new: two fp16 roundings and those of the weights
    assert np.all(np.abs(out1[taken].astype(np.float64) - out[taken]) <= 2.0 ** -9 * np.abs(out[taken]) + 2.0 ** -8)
    for i, n in enumerate(news):
        first, end = lens[i] - n, lens[i] - n + min(n, most)
        for j in range(-(-lens[i] // 16)):
            page, lo, hi = c.table[i, j], min(16, max(0, first - 16 * j)), min(16, max(0, end - 16 * j))
            whole = 16 * j + 16 <= end                  # no ignored row lies in the page
            assert np.array_equal(pool1[0][page, :, hi:], c.k[page, :, hi:])
            if whole or hi <= lo:
                want = pool if whole else (c.k, c.v, c.scales)
                assert all(np.array_equal(a[page], b[page]) for a, b in zip(pool1, want))
            else:                                       # its scale may be below that of the whole call
                now = ref.page_tokens_of(*pool1, page, 0)[:, lo:hi]
                all_rows = ref.page_tokens_of(*pool, page, 0)[:, lo:hi]
                unit = pool[2][page, :, 0].astype(np.float64)[:, None, None]
                assert np.all(np.abs(now - all_rows) <= 1.001 * unit)


@pytest.mark.parametrize("rows", [10, 100])
@pytest.mark.parametrize("after", [-(1 << 31), -(1 << 31) + 1, -7, 0, 3, 1 << 30, (1 << 31) - 1])
def test_attend_bad_starts_stay_in_the_arrays(rows, after):
    """Starts outside [0, rows]: q and out lie between guard rows, which come out as they were, and the rows that the
    starts do name are those of a call without the bad ones."""
    c = Cache(36, [rows - 4, 8], 2, 16, 64, max_pages=32)
    cache, guard = c.upload(), 128
    q = torch.full((rows + 2 * guard, 4, 64), float("nan"), dtype=torch.float16, device="cuda")
    q[guard:guard + rows] = _dev(c.rng.standard_normal((rows, 4, 64)).astype(np.float16))
    outs = []
    print(f"[attend bad starts] rows={rows} after={after}", flush=True)
    for starts in ([0, rows, rows], [0, (1 << 31) - 1, after], [-(1 << 31), rows, after]):
        wide = torch.full_like(q, 7.0)
        tt.kv_attend(cache, q[guard:guard + rows], _dev(np.array(starts, np.int32)), rows, wide[guard:guard + rows],
                     _workspace())
        assert torch.all(wide[:guard] == 7) and torch.all(wide[guard + rows:] == 7)
        outs.append(wide[guard:guard + rows])
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("news", [(1,), (40,), (200,)])
def test_attend_long_context(news):
    """Many pieces of one sequence, with the context's end inside a page."""
    _check_attend(Cache(25, [9001], 2, 64, 128), news, 4)


@pytest.mark.parametrize("news", [(1, 1), (40, 70)])
def test_attend_missing_pages_are_not_seen(news):
    """Holes in a table, a sequence without any page, lengths past the table."""
    c = Cache(26, [400, 200], 2, 16, 64, max_pages=14)
    c.table[0, 2], c.table[0, 7], c.table[1, :] = -1, len(c.k), -7
    got = _check_attend(c, news, 4)
    assert np.all(got[news[0]:] == 0)


@pytest.mark.parametrize("news", [(1, 1), (60, 20)])
def test_attend_lengths_below_the_rows(news):
    """Rows before a sequence's start see nothing and give zeros."""
    c = Cache(27, [100, 30], 1, 16, 64)
    c.lens[:] = [news[0] // 2, 0]
    got = _check_attend(c, news, 2)
    assert np.all(got[:news[0] - news[0] // 2] == 0) and np.all(got[news[0]:] == 0)


@pytest.mark.parametrize("news", [(1, 1), (80, 33)])
def test_attend_unused_places_do_not_matter(news):
    """What lies past a sequence's end in its page, and in pages of no sequence, is never seen: -128 values there,
    NaN and infinite scales of unused pages."""
    lens = [85, 333]
    c = Cache(28, lens, 2, 64, 128)
    first = _check_attend(c, news, 4)
    used = np.zeros(len(c.k), bool)
    for i, n in enumerate(lens):
        for j in range(-(-n // 64)):
            p = c.table[i, j]
            used[p] = True
            end = min(64, n - 64 * j)
            c.k[p, :, end:] = -128
            flat = c.v[p].transpose(0, 1, 3, 2).reshape(2, 64, 128)
            flat[:, end:] = -128
            c.v[p] = flat.reshape(2, 4, 16, 128).transpose(0, 1, 3, 2)
    c.scales[~used] = np.nan
    c.table[c.table < 0] = int(np.flatnonzero(~used)[0])
    assert np.array_equal(_check_attend(c, news, 4), first)


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("news", [(1, 1, 1), (70, 33, 1), (81, 130, 7)])
@pytest.mark.parametrize("scale", [1e30, np.inf, np.nan, 0.0])
def test_attend_scales_of_other_pages_do_not_matter(page, news, scale):
    """Scales of pages that are no sequence's, page 0 of the pool among them, at prompts' ends inside a tile and at
    holes of the table: the outputs keep every bit."""
    c = Cache(38, [81, 333, 215], 2, page, 128)
    c.table[1:, 2] = -1
    if (c.table == 0).any():                   # page 0 is left to no one: its sequence takes a spare one
        c.table[c.table == 0] = np.setdiff1d(np.arange(len(c.k)), c.table)[0]
    unused = np.setdiff1d(np.arange(len(c.k)), c.table)
    assert unused[0] == 0
    first = _check_attend(c, news, 4)
    c.scales[unused] = scale
    c.k[unused], c.v[unused] = 127, 127
    assert np.array_equal(_check_attend(c, news, 4), first)


@pytest.mark.parametrize("news", [(1, 1, 1), (40, 3, 1), (100, 80, 33)])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_attend_not_finite_queries_stay_alone(news, bad):
    """A q that is not finite makes its own output NaN and no other: the rest stay as far from the output without it
    as two outputs within _check_attend's bound can be, whose |weight| |value| sums are at most the largest value."""
    c = Cache(29, (170, 500, 3000), 2, 64, 128)
    starts, rows = _starts(news), sum(news)
    q = c.rng.standard_normal((rows, 8, c.dim)).astype(np.float16)
    spoilt = q.copy()
    mine = np.zeros((rows, 8), bool)
    for row, head in ((0, 3), (rows - 1, 0)):
        spoilt[row, head, 5] = bad
        mine[row, head] = True
    cache, outs = c.upload(), []
    for x in (q, spoilt):
        out = torch.zeros((rows, 8, c.dim), dtype=torch.float16, device="cuda")
        tt.kv_attend(cache, _dev(x), _dev(starts), max(news), out, _workspace())
        outs.append(out.cpu().numpy().astype(np.float64))
    largest = max(float(np.abs(c.sequence(i)[1]).max()) for i in range(3))
    assert np.isnan(outs[1][mine]).all()
    assert np.abs(outs[1][~mine] - outs[0][~mine]).max() <= 2 * (2.5 * 2.0 ** -11 * largest + 2.0 ** -24)


@pytest.mark.parametrize("news", [(1,), (100,)])
@pytest.mark.parametrize("kind", ["large", "apart", "zero", "small"])
def test_attend_scales(news, kind):
    """Peaked scores, pages whose scales are orders apart, pages of zeros."""
    c = Cache(29, [700], 2, 16, 128)
    rng = np.random.default_rng(1)
    if kind == "large":
        c.scales[..., 0] *= 4
    elif kind == "apart":
        c.scales[..., 1] *= 10.0 ** rng.integers(-4, 4, c.scales[..., 1].shape)
    elif kind == "zero":
        some = rng.random(len(c.k)) < 0.5
        c.scales[some] = 0
        c.k[some], c.v[some] = 0, 0
    else:
        c.scales[..., 1] *= 1e-4
    _check_attend(c, news, 4)


def test_attend_scale_argument_and_large_scores():
    """Scores of some hundreds: one key takes all; the float32 scores' error, 2^-24 of a few thousand, stays small."""
    _check_attend(Cache(30, [300], 1, 32, 64), [1], 4, scale=0.5)
    _check_attend(Cache(30, [300], 1, 32, 64), [90], 4, scale=0.0)


def test_attend_offsets_past_four_gib():
    """A pool of 5 GiB a side whose last pages are used."""
    heads, page, dim = 8, 128, 128
    pages = (5 << 30) // (heads * page * dim)
    k = torch.zeros((pages, heads, page, dim), dtype=torch.int8, device="cuda")
    v = torch.zeros((pages, heads, page // 16, dim, 16), dtype=torch.int8, device="cuda")
    scales = torch.zeros((pages, heads, 2), device="cuda")
    table = torch.tensor([[pages - 1, pages // 2, pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([300], dtype=torch.int32, device="cuda")
    cache = tt.make_kv_cache(k, v, scales, table, lens)
    rng = np.random.default_rng(5)
    x = rng.standard_normal((2, 300, heads, dim)).astype(np.float32)
    q = rng.standard_normal((300, heads, dim)).astype(np.float32)
    starts, qo = _dev(_starts([300])), torch.empty((300, heads, dim), dtype=torch.float16, device="cuda")
    tt.kv_append(cache, _dev(q), _dev(x[0]), _dev(x[1]), starts, 300, None, qo)
    out = torch.empty_like(qo)
    tt.kv_attend(cache, qo, starts, 300, out, _workspace())
    last = torch.empty_like(qo[:1])
    tt.kv_attend(cache, qo[-1:], _dev(_starts([1])), 1, last, _workspace())
    kb, vb = (torch.empty((1, 300, heads, dim), dtype=torch.float16, device="cuda") for _ in "kv")
    tt.kv_read(cache, 300, kb, vb)
    torch.cuda.synchronize()
    for b, w in ((kb, x[0]), (vb, x[1])):
        assert float((b[0].cpu().float() - torch.from_numpy(w)).abs().max()) < 0.03
    ks, vs = (b[0].cpu().numpy().astype(np.float64) for b in (kb, vb))
    want, size = ref.attend(qo.cpu().numpy(), ks, vs, np.ones(300, bool), 0, dim ** -0.5, 0)
    # the values read back are rounded to fp16 themselves: one more 2^-11 of the scores' and values' size
    assert np.all(np.abs(out.cpu().numpy() - want) <= 2.0 ** -11 * np.abs(want) + 8 * 2.0 ** -11 * size + 2.0 ** -24)
    assert np.all(np.abs(last.cpu().numpy() - want[-1:]) <= 2.0 ** -11 * np.abs(want[-1:]) + 8 * 2.0 ** -11 * size[-1:] + 2.0 ** -24)


def test_attend_on_other_streams():
    """Two streams at once, each with its own workspace; a call on a stream that is not torch's current one."""
    caches = [Cache(31 + i, [2000, 900], 2, 32, 128) for i in range(2)]
    handles = [c.upload() for c in caches]
    q = [_dev(np.random.default_rng(i).standard_normal((2, 8, 128)).astype(np.float16)) for i in range(2)]
    at = _dev(_starts([1, 1]))
    want = [torch.empty_like(x) for x in q]
    for h, x, w in zip(handles, q, want):
        tt.kv_attend(h, x, at, 1, w, _workspace())
    torch.cuda.synchronize()
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [tt.kv_attend_workspace() for _ in range(2)]
    outs = [[torch.empty_like(q[i]) for _ in range(6)] for i in range(2)]
    torch.cuda.synchronize()
    for rep in range(6):
        for i in range(2):
            tt.kv_attend(handles[i], q[i], at, 1, outs[i][rep], spaces[i], stream=streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o, want[i])


def test_decode_step_in_a_graph_follows_the_lengths():
    """Append, attention and sampling captured once; every replay sees the lengths and pages of its time."""
    c = Cache(33, [90, 200], 2, 32, 64, max_pages=12)
    c.table[0, :6], c.table[1, :8] = np.arange(6), np.arange(6, 14)
    c.k, c.v = (np.zeros((20,) + a.shape[1:], np.int8) for a in (c.k, c.v))
    c.scales = np.zeros((20, 2, 2), np.float32)
    cache = c.upload()
    rng = np.random.default_rng(9)
    x = _dev(rng.standard_normal((2, 2, 64)).astype(np.float32))
    q = _dev(rng.standard_normal((2, 6, 64)).astype(np.float32))
    logits, rope = _dev(rng.standard_normal((2, 500)).astype(np.float32)), tt.rope_table(400, 64)
    f = [_dev(np.array(a, np.float32)) for a in ([1, 0.7], [0.9, 1], [0, 0.1], [0.3, 0.8])]
    top_k = _dev(np.array([20, 0], np.int32))
    at, ws, sws = _dev(_starts([1, 1])), tt.kv_attend_workspace(), tt.sample_workspace(2, 500)

    def step(qo, out, tokens):
        tt.kv_append(cache, q, x, x, at, 1, rope, qo)
        tt.kv_attend(cache, qo, at, 1, out, ws)
        tt.sample(logits, f[0], top_k, f[1], f[2], f[3], tokens, sws)

    def buffers():
        return (torch.zeros((2, 6, 64), dtype=torch.float16, device="cuda"),
                torch.zeros((2, 6, 64), dtype=torch.float16, device="cuda"),
                torch.zeros(2, dtype=torch.int32, device="cuda"))

    captured, eager = buffers(), buffers()
    step(*eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    for rep in range(5):
        c.d[4].copy_(torch.tensor([91 + 3 * rep, 201 + rep], dtype=torch.int32))
        x.normal_()
        logits.normal_()
        torch.cuda.synchronize()
        before = [t.clone() for t in c.d[:3]]
        graph.replay()
        torch.cuda.synchronize()
        after = [t.clone() for t in c.d[:3]]
        for t, b in zip(c.d, before):
            t.copy_(b)
        step(*eager)
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b), rep
        for t, b in zip(c.d, after):
            assert torch.equal(t, b), rep


# ------------------------------------------------------------------ sampling

def _sample(x, temperature, top_k, top_p, min_p, u, pad=0):
    rows, n = x.shape
    full = [np.broadcast_to(np.asarray(a), (rows,)) for a in (temperature, top_k, top_p, min_p, u)]
    wide = torch.full((rows, n + pad), 1e4, dtype=torch.float32, device="cuda")
    wide[:, :n] = _dev(x, np.float32)
    tokens = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    f = [_dev(a, np.int32 if i == 1 else np.float32) for i, a in enumerate(full)]
    tt.sample(wide[:, :n], f[0], f[1], f[2], f[3], f[4], tokens, tt.sample_workspace(rows, n))
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), full


def _check_sample(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.5, pad=0):
    got, full = _sample(x, temperature, top_k, top_p, min_p, u, pad)
    want = [ref.sample(r, *(a[i] for a in full)) for i, r in enumerate(np.asarray(x, np.float32))]
    assert got.tolist() == want
    return got


@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 1000, 1023, 1025, 4097, 50001, 151936])
def test_sample_every_filter(vocab):
    """Rows of one call with settings of their own."""
    rng = np.random.default_rng(vocab)
    rows = 24
    x = (rng.standard_normal((rows, vocab)) * 2.5).astype(np.float32)
    t = rng.choice([0.0, 0.3, 0.7, 1.0, 1.7], rows)
    k = rng.choice([-1, 0, 1, 2, 20, 50, 1000, vocab, vocab + 5], rows)
    p = rng.choice([0.0, 0.1, 0.5, 0.9, 0.99, 1.0, 1.5], rows)
    m = rng.choice([-1.0, 0.0, 0.01, 0.2, 1.0, 2.0], rows)
    print(f"[sample] vocab={vocab}", flush=True)
    _check_sample(x, t, k, p, m, rng.random(rows), pad=vocab % 5)


@pytest.mark.parametrize("vocab", [700, 20000])
@pytest.mark.parametrize("which", ["top_k", "top_p", "min_p", "none", "both"])
def test_sample_ties(vocab, which):
    """Few distinct logits: ties at the cut go to the lowest indices."""
    rng = np.random.default_rng(7)
    rows = 16
    x = rng.integers(-3, 3, (rows, vocab)).astype(np.float32)
    x[0] = 1.25
    x[1] = -0.0
    x[1, ::2] = 0.0
    arg = {"top_k": {"top_k": rng.integers(1, vocab, rows)}, "top_p": {"top_p": rng.random(rows)},
           "min_p": {"min_p": rng.random(rows)}, "none": {},
           "both": {"top_k": rng.integers(1, vocab, rows), "top_p": rng.random(rows), "min_p": rng.random(rows) * 0.1}}[which]
    print(f"[sample ties] {vocab} {which}", flush=True)
    _check_sample(x, u=rng.random(rows), **arg)


def test_sample_spread_of_values():
    """Wide and narrow rows, one far ahead, subnormal differences, the type's ends."""
    rng = np.random.default_rng(11)
    n = 5000
    x = np.stack([rng.standard_normal(n) * s for s in (1e-6, 0.01, 0.1, 1, 30, 1e4, 1e30)] +
                 [np.linspace(-40, 0, n), np.linspace(100, 100.5, n), rng.standard_normal(n) + 1e6 * (np.arange(n) == 77),
                  np.full(n, 3.4e38) * np.sign(rng.standard_normal(n)), rng.standard_normal(n) * 1e-40]).astype(np.float32)
    rows = len(x)
    for p, k in ((1.0, 0), (0.9, 0), (0.95, 700), (1.0, 2500)):
        for t in (0.05, 1.0, 50.0, 1e-42, 1e30):
            print(f"[sample spread] p={p} k={k} t={t}", flush=True)
            _check_sample(x, t, k, p, 0.0, rng.random(rows))


def test_sample_masks():
    """-inf, the type's lowest value and NaN as masks; rows with one token, and with none, left."""
    rng = np.random.default_rng(13)
    n = 3000
    x = rng.standard_normal((10, n)).astype(np.float32)
    x[0, 5:] = -np.inf
    x[1, :-1] = -np.inf
    x[2] = -np.inf
    x[3, ::2] = np.nan
    x[4] = np.nan
    x[5, 10:] = np.finfo(np.float32).min
    x[6] = np.finfo(np.float32).min
    x[7, [3, 900]] = np.inf
    x[8, 17] = np.inf
    x[9, 100:] = -np.inf
    for args in ({}, {"top_k": 7}, {"top_p": 0.9}, {"min_p": 0.3}, {"top_k": 500, "top_p": 0.99, "min_p": 0.01},
                 {"temperature": 0.0}):
        print(f"[sample masks] {args}", flush=True)
        got = _check_sample(x, u=rng.random(10), **args)
        assert got[2] == got[4] == -1 and got[1] == n - 1


@pytest.mark.parametrize("vocab", [524289, (1 << 22) - 77, 1 << 22])
def test_sample_up_to_the_largest_vocabulary(vocab):
    """More tiles than the last kernel has threads, and the most LDS that it asks for; the row's end inside a tile."""
    rng = np.random.default_rng(vocab)
    x = (rng.standard_normal((6, vocab)) * 2.5).astype(np.float32)
    x[5, -1] = 30
    print(f"[sample large] vocab={vocab}", flush=True)
    got = _check_sample(x, [1.0, 0.7, 1.0, 0.8, 0.0, 1.0], [0, 50, 0, 3000, 0, 0], [1.0, 0.9, 0.9, 0.99, 1.0, 0.5],
                        [0.0, 0.01, 0.0, 0.0, 0.0, 0.0], [0.999, 0.3, 0.7, 0.5, 0.0, 0.9])
    assert got[5] == vocab - 1


@pytest.mark.parametrize("equal", [1000, 1500, 16384, 16385, 40000])
def test_sample_many_equal_logits_at_the_cut(equal):
    """As many candidates as are sorted at once, as the row's list holds and more, for a top-k that goes by groups, one
    that goes by bins, and a top-p alone."""
    rng = np.random.default_rng(equal)
    n = 60000
    x = (rng.standard_normal((8, n)) * 0.5 - 8).astype(np.float32)
    for r in range(8):
        x[r, rng.choice(n, equal, replace=False)] = 2.5
        x[r, rng.choice(n, 5, replace=False)] = 3.0
    print(f"[sample equal] {equal}", flush=True)
    _check_sample(x, 1.0, [50, 50, 512, 600, 600, 0, 0, 30000], [1.0, 0.5, 0.99, 1.0, 0.3, 0.5, 0.01, 0.9],
                  [0.0, 0.0, 0.1, 0.0, 0.7, 0.0, 0.0, 0.0], rng.random(8))


def test_sample_ends_of_u():
    rng = np.random.default_rng(17)
    x = rng.standard_normal((4, 2000)).astype(np.float32)
    for args in ({}, {"top_k": 9}, {"top_p": 0.8}):
        got = _check_sample(x, u=np.array([0.0, np.nextafter(np.float32(1), np.float32(0)), 1e-30, 0.25]), **args)
        assert got[0] >= 0
    # outside [0, 1): the ends
    one, _ = _sample(x, 1.0, 0, 1.0, 0.0, np.array([1.0, -3.0, np.nan, np.inf]))
    last = [int(np.flatnonzero(ref.weights(r, 1.0))[-1]) for r in x]
    assert one[0] == last[0] and one[3] == last[3] and one[1] == one[2] == 0


def test_sample_frequencies():
    """Chi-squared of 20,000 draws over ten kept tokens (9 degrees of freedom: 33.7 at 1e-4)."""
    rng = np.random.default_rng(19)
    x = np.tile((rng.standard_normal(64) * 1.5).astype(np.float32), (20000, 1))
    got, _ = _sample(x, 0.9, 10, 1.0, 0.0, rng.random(20000))
    kept = np.argsort(-x[0], kind="stable")[:10]
    p = np.exp(x[0, kept].astype(np.float64) / 0.9)
    p /= p.sum()
    seen = np.array([(got == t).sum() for t in kept])
    assert seen.sum() == 20000
    assert float(((seen - 20000 * p) ** 2 / (20000 * p)).sum()) < 33.7


def test_sample_many_rows_and_workspace_contents():
    """A workspace's contents do not matter, and a call leaves nothing that the next one needs."""
    rng = np.random.default_rng(23)
    x = (rng.standard_normal((700, 3001)) * 3).astype(np.float32)
    u = rng.random(700)
    args = (np.float32(0.8), 40, np.float32(0.9), np.float32(0.02), u)
    want, full = _sample(x, *args)
    some = rng.integers(0, 700, 20)
    for i in some:
        assert want[i] == ref.sample(x[i], *(a[i] for a in full))
    ws = tt.sample_workspace(700, 3001)
    f = [_dev(a, np.int32 if i == 1 else np.float32) for i, a in enumerate(full)]
    xd = _dev(x)
    for fill in (0, 255, 17):
        ws.fill_(fill)
        tokens = torch.empty(700, dtype=torch.int32, device="cuda")
        for _ in range(2):
            tt.sample(xd, f[0], f[1], f[2], f[3], f[4], tokens, ws)
            assert np.array_equal(tokens.cpu().numpy(), want)
