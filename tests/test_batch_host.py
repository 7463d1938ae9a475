"""Host-side checks of shared prefixes, weights, eviction and log probabilities (no GPU needed): arguments that do not fit
are refused with their status before any launch, also by the binding, and the oracle agrees with plain float64."""

import ctypes

import numpy as np
import pytest

import paper_2609_35465_amd as tt
from oracle import batch as ref
from test_serving_host import FAKE, _cache, _input

torch = pytest.importorskip("torch")


def _shared(cache=None, q=FAKE, q_stride=256, starts=FAKE, rows=6, max_new=2, heads=4, scale=0.1, groups=FAKE, shared=FAKE, n=2,
            out=FAKE, out_stride=256, ws=FAKE, ws_bytes=1 << 40):
    cache = cache or _cache()
    return tt.library().tetra_kv_attend_shared(ctypes.addressof(cache), q, q_stride, starts, rows, max_new, heads, scale, groups,
                                               shared, n, out, out_stride, ws, ws_bytes, None)


def _weigh(cache=None, q=FAKE, q_stride=256, starts=FAKE, rows=6, max_new=2, heads=4, scale=0.1, window=0, mass=FAKE, out=FAKE,
           places=100, decay=1.0, ws=FAKE, ws_bytes=1 << 40):
    cache = cache or _cache()
    return tt.library().tetra_kv_weigh(ctypes.addressof(cache), q, q_stride, starts, rows, max_new, heads, scale, window, mass,
                                       out, places, decay, ws, ws_bytes, None)


def _evict(cache=None, to=None, mass=FAKE, places=100, recent=2, out=FAKE + 4096, out_places=50, ws=FAKE, ws_bytes=1 << 40):
    cache, to = cache or _cache(), to or _cache()
    return tt.library().tetra_kv_evict(ctypes.addressof(cache), ctypes.addressof(to), mass, places, recent, out, out_places, ws,
                                       ws_bytes, None)


def _score(logits=FAKE, half=0, stride=100, rows=2, vocab=100, t=FAKE, tokens=FAKE, given=1, out=FAKE, entropy=FAKE, top=3,
           ids=FAKE, logs=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return tt.library().tetra_log_probs(logits, half, stride, rows, vocab, t, tokens, given, out, entropy, top, ids, logs, ws,
                                        ws_bytes, None)


def _append_at(cache=None, inp=None, starts=FAKE, shifts=FAKE, rows=6, max_new=2):
    cache, inp = cache or _cache(), inp or _input()
    return tt.library().tetra_kv_append_at(ctypes.addressof(cache), ctypes.addressof(inp), starts, shifts, rows, max_new, None)


CACHES = [
    (dict(k=None), tt.EINVAL), (dict(v=None), tt.EINVAL), (dict(scales=None), tt.EINVAL), (dict(pages=None), tt.EINVAL),
    (dict(lens=None), tt.EINVAL), (dict(num_pages=0), tt.EINVAL), (dict(page_tokens=0), tt.EINVAL),
    (dict(page_tokens=48), tt.EINVAL), (dict(kv_heads=0), tt.EINVAL), (dict(head_dim=0), tt.EINVAL),
    (dict(head_dim=96), tt.EUNSUPPORTED), (dict(seqs=0), tt.EINVAL), (dict(max_pages=0), tt.EINVAL),
    (dict(max_pages=(1 << 26) + 1), tt.EINVAL), (dict(k=FAKE + 8), tt.EALIGN), (dict(v=FAKE + 8), tt.EALIGN),
    (dict(scales=FAKE + 4), tt.EALIGN), (dict(pages=FAKE + 2), tt.EALIGN), (dict(lens=FAKE + 1), tt.EALIGN)]


@pytest.mark.parametrize("change,status", CACHES)
def test_cache_validation(change, status):
    assert _shared(_cache(**change)) == status
    assert _weigh(_cache(**change)) == status
    assert _evict(_cache(**change)) == status and _evict(to=_cache(**change)) == status
    assert _append_at(_cache(**change)) == status


ROWS = [dict(q=None), dict(starts=None), dict(out=None), dict(ws=None), dict(rows=0), dict(max_new=0), dict(max_new=7),
        dict(heads=0), dict(heads=3), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride=128), dict(ws_bytes=0)]


def test_shared_validation():
    for args in ROWS + [dict(groups=None), dict(shared=None), dict(n=0), dict(n=4), dict(out_stride=192)]:
        assert _shared(**args) == tt.EINVAL, args
    for args in (dict(q=FAKE + 8), dict(out=FAKE + 8), dict(q_stride=260), dict(out_stride=260), dict(starts=FAKE + 2),
                 dict(groups=FAKE + 2), dict(shared=FAKE + 1), dict(ws=FAKE + 16)):
        assert _shared(**args) == tt.EALIGN, args


def test_weigh_validation():
    for args in ROWS + [dict(window=-1), dict(places=0), dict(decay=-0.1), dict(decay=1.5), dict(decay=float("nan"))]:
        assert _weigh(**args) == tt.EINVAL, args
    for args in (dict(q=FAKE + 8), dict(out=FAKE + 2), dict(q_stride=260), dict(mass=FAKE + 2), dict(starts=FAKE + 2),
                 dict(ws=FAKE + 16)):
        assert _weigh(**args) == tt.EALIGN, args
    size, c = tt.library().tetra_kv_weigh_workspace_bytes, _cache()
    for bad in (dict(head_dim=96), dict(seqs=0), dict(page_tokens=8), dict(max_pages=1 << 30), dict(kv_heads=0)):
        assert size(ctypes.addressof(_cache(**bad)), 6, 4) == 0, bad
    assert size(None, 6, 4) == size(ctypes.addressof(c), 0, 4) == size(ctypes.addressof(c), 6, 3) == 0
    assert size(ctypes.addressof(c), 6, 0) == 0


def test_evict_validation():
    for args in (dict(mass=None), dict(ws=None), dict(places=0), dict(recent=-1), dict(out_places=0), dict(ws_bytes=0),
                 dict(out=FAKE)):
        assert _evict(**args) == tt.EINVAL, args
    for args in (dict(mass=FAKE + 2), dict(out=FAKE + 1), dict(ws=FAKE + 16)):
        assert _evict(**args) == tt.EALIGN, args
    assert _evict(to=_cache(lens=FAKE + 64, num_pages=9)) == tt.EINVAL            # into the pages that it reads
    for change in (dict(kv_heads=1), dict(head_dim=128), dict(page_tokens=32), dict(seqs=2)):
        assert _evict(to=_cache(**change)) == tt.EINVAL, change
    size, c = tt.library().tetra_kv_evict_workspace_bytes, _cache()
    assert size(None, ctypes.addressof(c)) == size(ctypes.addressof(c), None) == 0
    assert size(ctypes.addressof(c), ctypes.addressof(_cache(seqs=0))) == 0
    assert size(ctypes.addressof(c), ctypes.addressof(c)) > 0
    # sizes past 32 bits are refused or counted, never wrapped
    big = _cache(seqs=1 << 15, max_pages=1 << 10, page_tokens=128, kv_heads=64)
    assert size(ctypes.addressof(big), ctypes.addressof(big)) > 1 << 36
    assert _evict(big, big, ws_bytes=1 << 30) == tt.EINVAL


def test_append_at_validation():
    assert _append_at(shifts=None) == tt.EINVAL and _append_at(shifts=FAKE + 2) == tt.EALIGN
    for args in (dict(starts=None), dict(rows=0), dict(max_new=0), dict(max_new=7)):
        assert _append_at(**args) == tt.EINVAL, args
    for change in (dict(k=None), dict(q_out=None), dict(half=2), dict(k_stride=64)):
        assert _append_at(inp=_input(**change)) == tt.EINVAL, change


def test_score_validation():
    for args in (dict(logits=None), dict(half=2), dict(half=-1), dict(rows=0), dict(vocab=0), dict(stride=99),
                 dict(vocab=(1 << 22) + 1, stride=1 << 23), dict(given=-1), dict(tokens=None), dict(out=None), dict(top=-1),
                 dict(top=65), dict(ids=None), dict(logs=None), dict(ws=None), dict(ws_bytes=0),
                 dict(given=0, top=0, entropy=None)):
        assert _score(**args) == tt.EINVAL, args
    for name in ("logits", "t", "tokens", "out", "entropy", "ids", "logs"):
        assert _score(**{name: FAKE + 2}) == tt.EALIGN, name
    assert _score(half=1, logits=FAKE + 1) == tt.EALIGN and _score(ws=FAKE + 16) == tt.EALIGN
    size = tt.library().tetra_log_probs_workspace_bytes
    assert size(0, 5, 0) == size(5, 0, 0) == size(1, (1 << 22) + 1, 0) == size(1, 5, 65) == size(1, 5, -1) == 0


def test_launches_past_the_thread_limit_are_refused():
    """A launch holds less than 2^32 threads: calls that need one more are refused before their first launch."""
    wide = _cache(kv_heads=8, page_tokens=128, max_pages=1 << 23, seqs=1)
    for pages in (1 << 19, 1 << 20, 1 << 23):             # 2^24 workgroups of 256 threads from the first on
        to = _cache(kv_heads=8, page_tokens=128, max_pages=pages, seqs=1, k=FAKE + 4096)
        assert _evict(wide, to, ws_bytes=1 << 62) == tt.EINVAL, pages
    assert _weigh(rows=1 << 24, max_new=1) == tt.EINVAL
    assert _score(rows=1 << 24) == tt.EINVAL


def _refused(call, *args, **kw):
    with pytest.raises(tt.TetraError) as e:
        call(*args, **kw)
    assert e.value.status == tt.EINVAL


def _tensors(pages=5):
    return tt.make_kv_cache(torch.zeros((4, 2, 32, 64), dtype=torch.int8), torch.zeros((4, 2, 2, 64, 16), dtype=torch.int8),
                            torch.zeros((4, 2, 2)), torch.zeros((3, pages), dtype=torch.int32),
                            torch.zeros(3, dtype=torch.int32))


def test_binding_refuses_other_shapes_types_and_places():
    """Every call here would be refused for its host tensors at last; what is wrong before that has the same status."""
    cache, q, i32 = _tensors(), torch.zeros((3, 4, 64)).half(), torch.int32
    starts, groups, shared = torch.zeros(4, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32)
    ws, mass = torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros((3, 2, 100))
    gap = torch.zeros((4, 2), dtype=i32)
    for args in ((q, starts, 1, groups, shared, q, ws), (q.float(), starts, 1, groups, shared, q, ws),
                 (q, starts[:3], 1, groups, shared, q, ws), (q, starts, 1, shared, shared, q, ws),
                 (q, starts, 1, groups.long(), shared, q, ws), (q, starts, 1, groups, shared.float(), q, ws),
                 (q, starts, 1, gap[:3, 1], shared, q, ws), (q, gap[:, 0], 1, groups, shared, q, ws),
                 (q, starts, 1, groups, shared, q.float(), ws), (q, starts, 1, groups, shared, q[:2], ws),
                 (q.transpose(1, 2), starts, 1, groups, shared, q, ws)):
        _refused(tt.kv_attend_shared, cache, *args)
    for args in ((q, starts, 1, mass, mass, ws), (q, starts, 1, None, mass.half(), ws), (q, starts, 1, mass[:2], mass, ws),
                 (q, starts, 1, mass[:, :, :50], mass, ws), (q, starts, 1, None, mass.transpose(0, 1), ws),
                 (q, starts, 1, torch.zeros((3, 2, 99)), mass, ws), (q.float(), starts, 1, None, mass, ws),
                 (q[:0], starts, 1, None, mass, ws)):
        _refused(tt.kv_weigh, cache, *args)
    for args in ((cache, mass, mass, ws), (cache, mass.double(), None, ws), (cache, mass[:, :1], None, ws),
                 (cache, mass, mass[:2], ws)):
        _refused(tt.kv_evict, cache, *args)
    x, t1, f = torch.zeros((3, 10)), torch.zeros((3, 1), dtype=i32), torch.zeros(3)
    out, top = torch.zeros((3, 1)), torch.zeros((3, 5), dtype=i32)
    for args, kw in (((x, t1, out, ws), {}), ((x.double(), t1, out, ws), {}), ((x.T, t1, out, ws), {}),
                     ((x, t1.long(), out, ws), {}), ((x, t1, out.half(), ws), {}), ((x, t1[:2], out, ws), {}),
                     ((x, t1, torch.zeros((3, 2)), ws), {}), ((x, None, out, ws), {}), ((x, t1, None, ws), {}),
                     ((x, torch.zeros((1, 3), dtype=i32), torch.zeros((1, 3)), ws), {}),
                     ((x, t1, out, ws), dict(entropy=f[:2])), ((x, t1, out, ws), dict(temperature=f.half())),
                     ((x, t1, out, ws), dict(top_tokens=top)), ((x, t1, out, ws), dict(top_tokens=top, top_out=f)),
                     ((x[:0], t1, out, ws), {}), ((x, t1, out, ws), dict(entropy=f[0])), ((x[:1], t1[0, 0], out[0, 0], ws), {})):
        _refused(tt.log_probs, *args, **kw)
    k = torch.zeros((3, 2, 64))
    for shifts in (torch.zeros(2, dtype=i32), torch.zeros(3), torch.zeros((3, 2), dtype=i32)[:, 0]):
        _refused(tt.kv_append, cache, None, k, k, starts, 1, None, None, shifts=shifts)


def test_oracle_of_weights_and_scores_is_the_plain_one():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((5, 4, 8)), rng.standard_normal((9, 2, 8))
    got, _ = ref.weigh(q, k, np.ones(9, bool), 4, 0.3, 3)
    want = np.zeros((2, 9))
    for i in range(5):
        for h in range(4):
            z = np.array([q[i, h] @ k[t, h // 2] * 0.3 if 4 + i - 3 < t <= 4 + i else -np.inf for t in range(9)])
            want[h // 2] += np.exp(z - z.max()) / np.exp(z - z.max()).sum()
    assert np.allclose(got, want)
    x = torch.from_numpy(rng.standard_normal(50).astype(np.float32))
    given, h, _, order, theirs = ref.log_probs(x.numpy(), 0.7, [3, 99], 4)
    logs = torch.log_softmax(x.double() / 0.7, 0)
    assert abs(given[0] - float(logs[3])) < 1e-7 and given[1] == -np.inf
    assert abs(h + float((logs.exp() * logs).sum())) < 1e-6
    assert order.tolist() == x.topk(4).indices.tolist() and np.allclose(theirs, logs.topk(4).values, atol=1e-6)


def test_oracle_of_the_choice_keeps_order_and_the_last():
    m = np.array([5, 1, 5, 2, 9, 5, 0, 0], np.float32)
    assert ref.choose(m, 8, 4, 0).tolist() == [0, 2, 4, 5]
    assert ref.choose(m, 8, 4, 2).tolist() == [0, 4, 6, 7]
    assert ref.choose(m, 8, 1, 5).tolist() == [7] and ref.choose(m, 8, 0, 5).tolist() == []
    assert ref.choose(m, 5, 9, 1).tolist() == [0, 1, 2, 3, 4]
    q, s = ref.moved(np.array([[10, -7], [100, 3]], np.int8), np.array([1.0, 4.0], np.float32))
    assert s == 4 and q.tolist() == [[2, -2], [100, 3]]


def test_shifts_on_the_host_do_not_reach_the_library(monkeypatch):
    """What kv_append takes with shifts lies on the current GPU, all of it: an address of host memory never gets to a
    kernel."""
    cache, i32 = _tensors(), torch.int32
    calls, call = [], tt._call
    monkeypatch.setattr(tt, "_call", lambda name, *a: calls.append(name) or tt.OK if name.startswith("tetra_kv") else call(name, *a))
    k, q, starts, shifts = torch.zeros((3, 2, 64)), torch.zeros((3, 4, 64)), torch.zeros(4, dtype=i32), torch.zeros(3, dtype=i32)
    _refused(tt.kv_append, cache, None, k, k, starts, 1, None, None, shifts=shifts, stream=0)
    _refused(tt.kv_append, cache, q, k, k, starts, 1, torch.zeros((9, 64)), q.half(), torch.zeros(64), torch.zeros(64),
             shifts=shifts, stream=0)
    assert calls == []

    # each of them by itself: the others as if on the current GPU
    seen = []
    monkeypatch.setattr(tt, "_here", lambda *t: bool(seen.append(t)))
    rope, out, norms = torch.zeros((9, 64)), q.half(), [torch.zeros(64), torch.zeros(64)]
    _refused(tt.kv_append, cache, q, k, k, starts, 1, rope, out, *norms, shifts=shifts, stream=0)
    for t in (q, k, starts, rope, out, *norms, shifts, *cache.tensors):
        assert any(t is x for x in seen[0])


def test_shared_tables_of_more_tiles_than_an_int_counts():
    """Room for 2^31 tiles and more, over groups, sequences, cache heads and row tiles, is refused as kv_attend refuses it:
    the kernels count them in an int.  The workspace is too small for a launch in any case."""
    def call(pages, seqs=1024, n=1024, heads=64, new=1):
        wide = _cache(kv_heads=heads, page_tokens=128, max_pages=pages, seqs=seqs)
        return _shared(wide, q_stride=heads * 64, rows=1024, max_new=new, heads=heads, n=n, out_stride=heads * 64, ws_bytes=4096)

    # row tiles of 1,024 groups of up to 32 rows (two) and of as many sequences, by 64 heads, of pages / 2 tiles each
    for new, row_tiles in ((1, 3), (20, 4)):
        least = 2 * -(-(1 << 31) // (row_tiles * 1024 * 64))
        assert call(least, new=new) == call(1 << 23, new=new) == tt.EINVAL
        if not torch.cuda.is_available():
            assert call(least - 2, new=new) == tt.EDEVICE                    # on to the device, which is none
