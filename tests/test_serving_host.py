"""Host-side checks of the serving operators (no GPU needed): argument validation returns the documented status
codes before any launch, the binding refuses tensors of other shapes and types, and the oracle's sampling agrees
with a plain float64 draw."""

import ctypes

import numpy as np
import pytest

import paper_2609_35465_amd as tt
from oracle import serving as ref

torch = pytest.importorskip("torch")

FAKE = 0x1000                    # never dereferenced: validation fails first


def _cache(**change):
    c = dict(k=FAKE, v=FAKE, scales=FAKE, pages=FAKE, lens=FAKE, num_pages=4, page_tokens=16, kv_heads=2, head_dim=64,
             seqs=3, max_pages=5)
    c.update(change)
    return tt.KVCache(**c)


def _input(**change):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_stride=256, k_stride=128, v_stride=128, half=0, q_norm=None, k_norm=None,
             eps=1e-6, rope=FAKE, rope_rows=9, q_heads=4, q_out=FAKE)
    a.update(change)
    return tt.KVInput(**a)


def _append(cache=None, inp=None, starts=FAKE, rows=6, max_new=2):
    cache, inp = cache or _cache(), inp or _input()
    return tt.library().tetra_kv_append(ctypes.addressof(cache), ctypes.addressof(inp), starts, rows, max_new, None)


def _attend(cache=None, q=FAKE, q_stride=256, starts=FAKE, rows=6, max_new=2, heads=4, scale=0.1, window=0, out=FAKE,
            out_stride=256, ws=FAKE, ws_bytes=1 << 40):
    cache = cache or _cache()
    return tt.library().tetra_kv_attend(ctypes.addressof(cache), q, q_stride, starts, rows, max_new, heads, scale, window,
                                        out, out_stride, ws, ws_bytes, None)


def _read(cache=None, count=4, k=FAKE, v=FAKE):
    cache = cache or _cache()
    return tt.library().tetra_kv_read(ctypes.addressof(cache), count, k, v, None)


def _sample(logits=FAKE, stride=100, rows=2, vocab=100, t=FAKE, k=FAKE, p=FAKE, m=FAKE, u=FAKE, tokens=FAKE, ws=FAKE,
            ws_bytes=1 << 40):
    return tt.library().tetra_sample(logits, stride, rows, vocab, t, k, p, m, u, tokens, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), tt.EINVAL), (dict(v=None), tt.EINVAL), (dict(scales=None), tt.EINVAL), (dict(pages=None), tt.EINVAL),
    (dict(lens=None), tt.EINVAL), (dict(num_pages=0), tt.EINVAL), (dict(page_tokens=0), tt.EINVAL),
    (dict(page_tokens=8), tt.EINVAL), (dict(page_tokens=48), tt.EINVAL), (dict(page_tokens=256), tt.EINVAL),
    (dict(kv_heads=0), tt.EINVAL), (dict(head_dim=0), tt.EINVAL), (dict(head_dim=96), tt.EUNSUPPORTED),
    (dict(head_dim=256), tt.EUNSUPPORTED), (dict(seqs=0), tt.EINVAL), (dict(max_pages=0), tt.EINVAL),
    (dict(k=FAKE + 8), tt.EALIGN), (dict(v=FAKE + 8), tt.EALIGN), (dict(scales=FAKE + 4), tt.EALIGN),
    (dict(pages=FAKE + 2), tt.EALIGN), (dict(lens=FAKE + 1), tt.EALIGN)])
def test_cache_validation(change, status):
    assert _append(_cache(**change)) == status
    assert _attend(_cache(**change)) == status
    assert _read(_cache(**change)) == status


def test_append_validation():
    lib, c, a = tt.library(), _cache(), _input()
    assert lib.tetra_kv_append(None, ctypes.addressof(a), FAKE, 6, 2, None) == tt.EINVAL
    assert lib.tetra_kv_append(ctypes.addressof(c), None, FAKE, 6, 2, None) == tt.EINVAL
    for args in (dict(starts=None), dict(rows=0), dict(max_new=0), dict(max_new=7)):
        assert _append(**args) == tt.EINVAL, args
    assert _append(starts=FAKE + 2) == tt.EALIGN
    for change in (dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(q_heads=0), dict(half=2),
                   dict(rope_rows=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                   dict(k_stride=64), dict(v_stride=120), dict(q_stride=192)):
        assert _append(inp=_input(**change)) == tt.EINVAL, change
    for change in (dict(k=FAKE + 8), dict(v=FAKE + 4), dict(q=FAKE + 8), dict(q_out=FAKE + 8), dict(q_norm=FAKE + 4),
                   dict(k_norm=FAKE + 8), dict(rope=FAKE + 4), dict(k_stride=132), dict(v_stride=132), dict(q_stride=260)):
        assert _append(inp=_input(**change)) == tt.EALIGN, change


def test_read_validation():
    assert _read(count=0) == tt.EINVAL and _read(k=None) == tt.EINVAL and _read(v=None) == tt.EINVAL
    assert _read(k=FAKE + 8) == tt.EALIGN and _read(v=FAKE + 2) == tt.EALIGN
    assert _read(count=(1 << 31) - 1, cache=_cache(seqs=1 << 20)) == tt.EINVAL


def test_attend_validation():
    for args in (dict(q=None), dict(starts=None), dict(out=None), dict(ws=None), dict(rows=0), dict(max_new=0),
                 dict(max_new=7), dict(heads=0), dict(heads=3), dict(scale=float("nan")), dict(scale=float("inf")),
                 dict(window=-1), dict(q_stride=128), dict(out_stride=192), dict(ws_bytes=0)):
        assert _attend(**args) == tt.EINVAL, args
    for args in (dict(q=FAKE + 8), dict(out=FAKE + 8), dict(q_stride=260), dict(out_stride=260), dict(starts=FAKE + 2),
                 dict(ws=FAKE + 16)):
        assert _attend(**args) == tt.EALIGN, args


def test_sample_validation():
    for args in (dict(logits=None), dict(t=None), dict(k=None), dict(p=None), dict(m=None), dict(u=None),
                 dict(tokens=None), dict(ws=None), dict(rows=0), dict(vocab=0), dict(vocab=(1 << 22) + 1, stride=1 << 23),
                 dict(stride=99), dict(ws_bytes=0)):
        assert _sample(**args) == tt.EINVAL, args
    for name in ("logits", "t", "k", "p", "m", "u", "tokens"):
        assert _sample(**{name: FAKE + 2}) == tt.EALIGN, name
    assert _sample(ws=FAKE + 16) == tt.EALIGN
    size = tt.library().tetra_sample_workspace_bytes
    assert size(0, 5) == size(5, 0) == size(1, (1 << 22) + 1) == 0 and size(3, 151936) > 0


def test_binding_refuses_other_shapes_and_types():
    def cache_args(**change):
        t = dict(k=torch.zeros((4, 2, 32, 64), dtype=torch.int8), v=torch.zeros((4, 2, 2, 64, 16), dtype=torch.int8),
                 scales=torch.zeros((4, 2, 2)), pages=torch.zeros((3, 5), dtype=torch.int32),
                 lens=torch.zeros(3, dtype=torch.int32))
        t.update(change)
        return tuple(t.values())

    def refused(call, *args, **kw):
        with pytest.raises(tt.TetraError) as e:
            call(*args, **kw)
        assert e.value.status == tt.EINVAL

    cache = tt.make_kv_cache(*cache_args())
    assert (cache.num_pages, cache.kv_heads, cache.page_tokens, cache.head_dim, cache.seqs, cache.max_pages) == \
        (4, 2, 32, 64, 3, 5)
    for change in (dict(k=torch.zeros((4, 2, 32, 64))), dict(v=torch.zeros((4, 2, 32, 64, 1), dtype=torch.int8)),
                   dict(scales=torch.zeros((4, 2))), dict(scales=torch.zeros((4, 2, 2)).half()),
                   dict(pages=torch.zeros((3, 5))), dict(lens=torch.zeros(4, dtype=torch.int32)),
                   dict(pages=torch.zeros((5, 3), dtype=torch.int32).T)):
        refused(tt.make_kv_cache, *cache_args(**change))
    q, k = torch.zeros((3, 4, 64)), torch.zeros((3, 2, 64))
    out, starts, rope = torch.zeros((3, 4, 64)).half(), torch.zeros(4, dtype=torch.int32), torch.zeros((9, 64))
    refused(tt.kv_append, cache, q, k.double(), k.double(), starts, 1, rope, out)
    refused(tt.kv_append, cache, q, k, k.half(), starts, 1, rope, out)
    refused(tt.kv_append, cache, q.half(), k, k, starts, 1, rope, out)
    refused(tt.kv_append, cache, q, k, k[:2], starts, 1, rope, out)
    refused(tt.kv_append, cache, q, k, k, starts[:3], 1, rope, out)
    refused(tt.kv_append, cache, q, k, k, starts.long(), 1, rope, out)
    refused(tt.kv_append, cache, q, k, k, starts, 1, rope[:, :32], out)
    refused(tt.kv_append, cache, q, k, k, starts, 1, rope, out.float())
    refused(tt.kv_append, cache, q, k, k, starts, 1, rope, out[:2])
    refused(tt.kv_append, cache, q, k.transpose(1, 2).contiguous().transpose(1, 2), k, starts, 1, rope, out)
    refused(tt.kv_append, cache, q, k, k, starts, 1, rope, out, torch.zeros(32))
    refused(tt.kv_read, cache, 4, torch.zeros((3, 4, 2, 64)).half(), torch.zeros((3, 4, 2, 32)).half())
    refused(tt.kv_attend, cache, q, starts, 1, out, out)
    refused(tt.kv_attend, cache, out, starts[:2], 1, out, out)
    refused(tt.kv_attend, cache, out, starts, 1, out[:, :2], out)
    x, f, i = torch.zeros((3, 10)), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    refused(tt.sample, x.half(), f, i, f, f, f, i, f)
    refused(tt.sample, x, f, f, f, f, f, i, f)
    refused(tt.sample, x, f[:2], i, f, f, f, i, f)
    refused(tt.sample, x.T, f, i, f, f, f, i, f)


def _small_cache():
    return tt.make_kv_cache(torch.zeros((4, 2, 32, 64), dtype=torch.int8), torch.zeros((4, 2, 2, 64, 16), dtype=torch.int8),
                            torch.zeros((4, 2, 2)), torch.zeros((3, 5), dtype=torch.int32),
                            torch.zeros(3, dtype=torch.int32))


@pytest.mark.parametrize("starts", [torch.zeros((4, 2), dtype=torch.int32)[:, 1], torch.zeros(1, dtype=torch.int32).expand(4)])
def test_binding_refuses_starts_with_gaps(starts):
    """A column of a wider tensor, or one number spread over all places: the kernels read `seqs + 1` numbers in line."""
    cache, k = _small_cache(), torch.zeros((3, 2, 64))
    out = torch.zeros((3, 4, 64)).half()
    for call in (lambda: tt.kv_append(cache, None, k, k, starts, 1, None, None),
                 lambda: tt.kv_attend(cache, out, starts, 1, out, torch.zeros(64, dtype=torch.uint8))):
        with pytest.raises(tt.TetraError) as e:
            call()
        assert e.value.status == tt.EINVAL


def test_binding_refuses_q_and_q_out_apart():
    """kv_append takes both or neither; one without the other is refused with its status."""
    cache, k, starts = _small_cache(), torch.zeros((3, 2, 64)), torch.zeros(4, dtype=torch.int32)
    for q, out in ((torch.zeros((3, 4, 64)), None), (None, torch.zeros((3, 4, 64)).half())):
        with pytest.raises(tt.TetraError) as e:
            tt.kv_append(cache, q, k, k, starts, 1, None, out)
        assert e.value.status == tt.EINVAL


def test_oracle_sampling_is_the_plain_draw():
    """The whole weights leave the distribution as it is: against a float64 draw with the same random number, the
    tokens agree (a cumulative sum would have to lie within 1e-7 of u to differ)."""
    rng = np.random.default_rng(0)
    for i in range(200):
        n = int(rng.integers(2, 400))
        x = (rng.standard_normal(n) * 2).astype(np.float32)
        t, k = float(np.float32(rng.uniform(0.3, 2))), int(rng.integers(0, n))
        p, m = float(np.float32(rng.random())), float(np.float32(rng.random() * 0.2))
        u = float(np.float32(rng.random()))
        w = np.exp((x.astype(np.float64) - float(x.max())) / t)
        order = np.argsort(-x, kind="stable")[:k if k else n]
        above = np.cumsum(w[order]) - w[order]
        order = order[above < p * w[order].sum()]
        keep = np.zeros(n, bool)
        keep[order] = True
        keep &= w >= m
        c = np.cumsum(np.where(keep, w, 0))
        assert ref.sample(x, t, k, p, m, u) == int(np.searchsorted(c, u * c[-1], side="right")), i
