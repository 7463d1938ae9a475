"""The operators of a batch that shares, thins out and scores what it has in the cache: what they are timed on.

share - attention of the new tokens' q over the paged 8-bit cache where groups of sequences begin with the same
        pages (a system prompt, a document, several answers to one prompt), which are read once for a group.
weigh - the attention weight that every cached token gets from the new tokens, added up over calls.
evict - the tokens of most weight, and the last ones, of every sequence and cache head into fewer pages; then they are
        read back as the values they stand for.
score - log probabilities of given tokens, the entropy and the likeliest alternatives, from rows of logits.

A case holds plain sizes.  A ragged case spreads its counts over its sequences, down to one new token and a sixteenth
of the context, and its last sequence is an idle slot of the batch with nothing in it.
"""

import math
import random

import torch

own = False


def listed():
    def heads(model):
        # q and kv heads of 128 of the dense Qwen3 layers
        return {"q_heads": {"4B": 32, "8B": 32, "14B": 40}[model], "kv_heads": 8, "dim": 128}

    return [
        # four answers to one prompt, a few tokens in: the smallest call
        {"name": "share-14b-b4-1024", "kind": "share", "groups": 1, "seqs": 4, "prefix": 1024, "own": 32, "new": 1,
         "ragged": False, **heads("14B"), "page": 32},
        # a decode step of 64 conversations that begin with one system prompt
        {"name": "share-14b-b64-4096", "kind": "share", "groups": 1, "seqs": 64, "prefix": 4096, "own": 512, "new": 1,
         "ragged": True, **heads("14B"), "page": 16},
        # 64 questions about one long document
        {"name": "share-8b-b64-32768", "kind": "share", "groups": 1, "seqs": 64, "prefix": 32768, "own": 1000, "new": 1,
         "ragged": True, **heads("8B"), "page": 64},
        # seven prompts of different lengths, six drafts of each checked three tokens at a time; narrow heads of their own
        {"name": "share-groups-d64", "kind": "share", "groups": 7, "seqs": 42, "prefix": 2000, "own": 301, "new": 3,
         "ragged": True, "q_heads": 16, "kv_heads": 16, "dim": 64, "page": 32},
        # the weights of one 4B token: the smallest call
        {"name": "weigh-4b-b1-203", "kind": "weigh", "seqs": 1, "new": 1, "ragged": False, "context": 203, **heads("4B"),
         "page": 32, "window": 0, "decay": 1.0},
        # a decode step of 64 sequences of 14B at different lengths
        {"name": "weigh-14b-b64-4096", "kind": "weigh", "seqs": 64, "new": 1, "ragged": True, "context": 4096,
         **heads("14B"), "page": 64, "window": 0, "decay": 1.0},
        # every row of a long 8B prompt
        {"name": "weigh-8b-4096", "kind": "weigh", "seqs": 1, "new": 4096, "ragged": False, "context": 4096, **heads("8B"),
         "page": 64, "window": 0, "decay": 1.0},
        # 64 sequences of 14B cut to half of what they hold at most
        {"name": "evict-14b-b64-4096", "kind": "evict", "seqs": 64, "ragged": True, "context": 4096, "keep": 2048,
         "recent": 64, **heads("14B"), "page": 64},
        # a long document cut to a thirty-second
        {"name": "evict-8b-b1-131072", "kind": "evict", "seqs": 1, "ragged": False, "context": 131072, "keep": 4096,
         "recent": 256, **heads("8B"), "page": 64},
        # the token of one sequence with the alternatives that an interface shows
        {"name": "score-b1", "kind": "score", "rows": 1, "vocab": 151936, "given": 1, "top": 20, "half": False,
         "tempered": False, "masked": False},
        # the tokens of 64 sequences, as drawn at temperatures of their own
        {"name": "score-b64", "kind": "score", "rows": 64, "vocab": 151936, "given": 1, "top": 5, "half": False,
         "tempered": True, "masked": False},
        # every token of a long prompt, whose logits are kept in 16 bits
        {"name": "score-prompt-2048", "kind": "score", "rows": 2048, "vocab": 151936, "given": 1, "top": 1, "half": True,
         "tempered": False, "masked": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["share", "share", "weigh", "weigh", "evict", "score"])
    if kind == "score":
        vocab = _log(rng, 1000, 151936)
        return {"kind": kind, "rows": _log(rng, 1, min(2048, 2048 * 75968 // vocab)), "vocab": vocab,
                "given": rng.choice([1, 1, 1, 2, 7]), "top": rng.choice([0, 1, 5, 20, 64]), "half": rng.random() < 0.4,
                "tempered": rng.random() < 0.4, "masked": rng.random() < 0.3}
    kv_heads, group, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8]), rng.choice([64, 128, 128])
    c = {"kind": kind, "q_heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "page": rng.choice([16, 32, 64, 128]),
         "ragged": rng.random() < 0.6}
    if kind == "share":
        c["seqs"], c["new"] = _log(rng, 2, 64), rng.choice([1, 1, 1, 1, 2, 4, 8])
        c["groups"] = min(c["seqs"] // 2, rng.choice([1, 1, 1, 2, 5, 9]))
        most = 64 * 32 * 32768 * 128 // (c["seqs"] * c["new"] * c["q_heads"] * dim)
        c["own"] = c["new"] + _log(rng, 1, min(1000, most // 4)) - 1
        return {**c, "prefix": _log(rng, 100, max(100, min(most // 2, 32768 // c["groups"])))}
    if kind == "evict":
        c["seqs"] = _log(rng, 1, 64)
        c["context"] = _log(rng, 1, min(131072, 131072 * 1024 // (c["seqs"] * kv_heads * dim)))
        c["keep"] = _log(rng, max(1, c["context"] // 32), c["context"])
        return {**c, "recent": rng.choice([0, 1, 32, 100])}
    c["decay"], most = rng.choice([1.0, 1.0, 0.9]), 4096 ** 3
    if rng.random() < 0.6:
        c["seqs"], c["new"] = _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 3])
        c["context"] = c["new"] + _log(rng, 1, min(131072, 131072 * 1024 // (c["seqs"] * kv_heads * dim)) - 3)
    else:
        c["seqs"] = _log(rng, 1, 8)
        c["new"] = _log(rng, 2, min(4096, int((most // (c["seqs"] * c["q_heads"] * dim)) ** 0.5)))
        c["context"] = _log(rng, c["new"], max(c["new"], min(32768, most // (2 * c["seqs"] * c["q_heads"] * dim * c["new"]))))
    return {**c, "window": 0 if rng.random() < 0.7 else _log(rng, 1, c["context"])}


# ------------------------------------------------------------------ the sequences of a case

def _spread(lo, hi, n, seed):
    v = [int(round(hi * (lo / hi) ** (i / (n - 1)))) for i in range(n)] if n > 1 else [hi]
    random.Random(seed).shuffle(v)
    return v


def _sequences(case):
    """New tokens, and tokens in the cache after the call, of every sequence."""
    n, new, context = case["seqs"], case.get("new", 0), case["context"]
    if not case["ragged"] or n < 2:
        return [new] * n, [context] * n
    news = _spread(1, new, n - 1, 1) if new else [0] * (n - 1)
    return news + [0], [max(a, b) for a, b in zip(news, _spread(max(1, context // 16), context, n - 1, 2))] + [0]


def _groups(case):
    """First sequence of every group and behind the last, tokens shared in each; new tokens and own tokens (the new ones
    among them) of every sequence."""
    n, g = case["seqs"], case["groups"]
    first = [i * n // g for i in range(g + 1)]
    shared = _spread(max(1, case["prefix"] // 4), case["prefix"], g, 3)
    news, own_tokens = _sequences({**case, "context": case["own"]})
    return first, shared, news, own_tokens


def _starts(news):
    at = [0]
    for n in news:
        at.append(at[-1] + n)
    return at


def _gen(seed, index):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 16 + index)


def _randn(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen)


def _whole(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pool(case, seed, pages):
    """A cache's pages, values as calls before this one left them, and the pages in no order."""
    heads, dim, page, gen = case["kv_heads"], case["dim"], case["page"], _gen(seed, 1)
    pages += 3

    def values(*shape):                # about 4.2 deviations at 127, as the largest of a page of Gaussian values is
        out = torch.empty(shape, dtype=torch.int8, device="cuda")
        for part in out.split(max(1, (1 << 28) // out[0].numel())):
            part.copy_((_randn(gen, *part.shape) * 30).round_().clamp_(-127, 127))
        return out

    return {"k": values(pages, heads, page, dim), "v": values(pages, heads, page // 16, dim, 16),
            "scales": (0.8 + 0.4 * torch.rand((pages, heads, 2), device="cuda", generator=gen)) * (4.2 / 127),
            "order": torch.randperm(pages, device="cuda", generator=gen).int()}


def _table(rows, order):
    """A page table from lists of places in `order`."""
    wide = max(1, max(len(r) for r in rows))
    at = torch.tensor([r + [-1] * (wide - len(r)) for r in rows], device="cuda")
    return torch.where(at < 0, -1, order[at.clamp(min=0)]).int()


def _share_inputs(case, seed):
    first, shared, news, own_tokens = _groups(case)
    page, rows, used = case["page"], [[] for _ in news], 0
    lens = [0] * len(news)
    for g in range(case["groups"]):
        whole = shared[g] // page                      # pages that the group's sequences have in common
        for i in range(first[g], first[g + 1]):
            if own_tokens[i]:
                lens[i] = shared[g] + own_tokens[i]
                rows[i] = list(range(used, used + whole))
        used += whole
    for i, n in enumerate(lens):
        more = -(-n // page) - len(rows[i])
        rows[i] += list(range(used, used + more))
        used += more
    starts, pool = _starts(news), _pool(case, seed, used)
    return {**pool, "pages": _table(rows, pool["order"]), "lens": _whole(lens), "starts": _whole(starts), "new": max(news),
            "groups": _whole(first), "shared": _whole(shared), "first": first, "common": [n // page * page for n in shared],
            "rows": starts, "counts": lens, "page": page,
            "q": (2 * _randn(_gen(seed, 2), starts[-1], case["q_heads"], case["dim"])).half()}


def _cache_inputs(case, seed):
    news, lens = _sequences(case)
    page, used, rows = case["page"], 0, []
    for n in lens:
        rows.append(list(range(used, used - (-n // page))))
        used += len(rows[-1])
    state = {"new": case.get("new", 0), "context": case["context"], "page": page}
    gen = _gen(seed, 3)
    # what calls before this one found: some tokens have most of the weight
    state["mass"] = torch.exp(1.5 * _randn(gen, len(lens), case["kv_heads"], case["context"]))
    if case["kind"] == "evict":
        kept = [min(n, case["keep"]) for n in lens]
        to = []
        for n in kept:
            to.append(list(range(used, used - (-n // page))))
            used += len(to[-1])
        pool = _pool(case, seed, used)
        return {**state, **pool, "pages": _table(rows, pool["order"]), "lens": _whole(lens), "to": _table(to, pool["order"]),
                "kept": _whole(kept), "recent": case["recent"], "count": max(kept)}
    starts, pool = _starts(news), _pool(case, seed, used)
    return {**state, **pool, "pages": _table(rows, pool["order"]), "lens": _whole(lens), "starts": _whole(starts),
            "window": case["window"], "decay": case["decay"],
            # queries of normed heads: scores of a few units
            "q": (2 * _randn(_gen(seed, 2), starts[-1], case["q_heads"], case["dim"])).half()}


def _score_inputs(case, seed):
    rows, vocab, gen = case["rows"], case["vocab"], _gen(seed, 4)
    x = _randn(gen, rows, vocab) * 2.5
    # the handful of tokens that the context makes likely
    likely = torch.randint(0, vocab, (rows, 8), device="cuda", generator=gen)
    x.scatter_add_(1, likely, 6 + 3 * _randn(gen, rows, 8))
    given = torch.randint(0, vocab, (rows, case["given"]), device="cuda", generator=gen)
    given[:, 0] = torch.where(torch.rand(rows, device="cuda", generator=gen) < 0.8, likely[:, 0], given[:, 0])
    if case["masked"]:
        # a grammar leaves a tenth of the vocabulary, the given tokens among it; it masks with -inf or the type's lowest
        keep = torch.rand((rows, vocab), device="cuda", generator=gen) < 0.1
        keep.scatter_(1, given, True)
        low = torch.full((rows, 1), -math.inf, device="cuda")
        low[1::2] = torch.finfo(torch.float16 if case["half"] else torch.float32).min
        x = torch.where(keep, x, low)
    state = {"logits": x.half() if case["half"] else x, "given": given.int(), "top": case["top"], "temperature": None}
    if case["tempered"]:
        state["temperature"] = 0.3 + 1.2 * torch.rand(rows, device="cuda", generator=gen)
    return state


def _inputs(case, seed):
    make = {"share": _share_inputs, "weigh": _cache_inputs, "evict": _cache_inputs, "score": _score_inputs}
    return make[case["kind"]](case, seed)


def prepare(case, seed):
    kind = case["kind"]
    state = {"kind": kind, **_inputs(case, seed)}
    if not own:
        return state
    import paper_2609_35465_amd as tt
    if kind == "score":
        rows, top = case["rows"], case["top"]
        state["workspace"] = tt.log_probs_workspace(rows, case["vocab"], top)
        state["out"] = torch.empty((rows, case["given"]), device="cuda")
        state["entropy"] = torch.empty(rows, device="cuda")
        state["top_tokens"] = torch.empty((rows, top), dtype=torch.int32, device="cuda")
        state["top_out"] = torch.empty((rows, top), device="cuda")
        return state
    state["cache"] = cache = tt.make_kv_cache(*(state[k] for k in ("k", "v", "scales", "pages", "lens")))
    if kind == "share":
        state["out"], state["workspace"] = torch.empty_like(state["q"]), tt.kv_attend_shared_workspace()
    elif kind == "weigh":
        state["mass_out"] = torch.zeros_like(state["mass"])
        state["workspace"] = tt.kv_weigh_workspace(cache, *state["q"].shape[:2])
    else:
        state["to_cache"] = to = tt.make_kv_cache(*(state[k] for k in ("k", "v", "scales", "to", "kept")))
        state["mass_out"] = torch.zeros((case["seqs"], case["kv_heads"], state["count"]), device="cuda")
        state["workspace"] = tt.kv_evict_workspace(cache, to)
        back = (case["seqs"], state["count"], case["kv_heads"], case["dim"])
        state["k_back"], state["v_back"] = (torch.empty(back, dtype=torch.float16, device="cuda") for _ in "kv")
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    kind = state["kind"]
    if not own:
        return {"share": _share, "weigh": _weigh, "evict": _evict, "score": _score}[kind](state)
    import paper_2609_35465_amd as tt
    s = state
    if kind == "share":
        tt.kv_attend_shared(s["cache"], s["q"], s["starts"], s["new"], s["groups"], s["shared"], s["out"], s["workspace"])
        return {"out": s["out"]}
    if kind == "weigh":
        tt.kv_weigh(s["cache"], s["q"], s["starts"], s["new"], s["mass"], s["mass_out"], s["workspace"],
                    window=s["window"], decay=s["decay"])
        return {"mass": s["mass_out"]}
    if kind == "evict":
        tt.kv_evict(s["cache"], s["to_cache"], s["mass"], s["mass_out"], s["workspace"], recent=s["recent"])
        tt.kv_read(s["to_cache"], s["count"], s["k_back"], s["v_back"])
        return {"k": s["k_back"], "v": s["v_back"], "mass": s["mass_out"]}
    tt.log_probs(s["logits"], s["given"], s["out"], s["workspace"], entropy=s["entropy"], top_tokens=s["top_tokens"],
                 top_out=s["top_out"], temperature=s["temperature"])
    return {k: s[k] for k in ("out", "entropy", "top_tokens", "top_out")}


def _gather(state, pages, tokens):
    """float32 k and v [.., n, heads, dim] of token numbers [.., n] of a table's rows [.., pages]."""
    t, page = tokens.clamp(min=0), state["page"]
    ids = pages.long().gather(-1, (t // page).clamp(max=pages.shape[-1] - 1)).clamp(min=0)
    scale, at = state["scales"][ids], t % page
    return (state["k"][ids, :, at].float() * scale[..., :1],
            state["v"][ids, :, at // 16, :, at % 16].float() * scale[..., 1:])


def _part(q, k, v, seen):
    """Largest score, sum of weights and weighted values of rows q [.., rows, dim] over keys [.., n, dim]."""
    z = q @ k.transpose(-1, -2) * q.shape[-1] ** -0.5
    if seen is not None:
        z.masked_fill_(~seen, -math.inf)
    m = z.amax(-1, keepdim=True).clamp(min=-3e38)
    p = z.sub_(m).exp_()
    return m, p.sum(-1, keepdim=True), p @ v


def _share(state):
    """A group's prefix against all its rows, every sequence's own tokens against its rows, joined."""
    q, lens, starts = state["q"], state["lens"].long(), state["starts"].long()
    rows, q_heads, dim = q.shape
    heads = state["k"].shape[1]
    group, seqs = q_heads // heads, lens.shape[0]
    common = torch.zeros(seqs, dtype=torch.long, device="cuda")
    parts = [torch.zeros((heads, rows, group, n), device="cuda") for n in (1, 1, dim)]
    parts[0].fill_(-3e38)
    by_head = q.float().view(rows, heads, group, dim).transpose(0, 1)                   # [heads, rows, group, dim]
    for g, n in enumerate(state["common"]):
        a, b = state["first"][g], state["first"][g + 1]
        common[a:b] = n
        lo, hi = state["rows"][a], state["rows"][b]
        if n and hi > lo:
            k, v = _gather(state, state["pages"][a], torch.arange(n, device="cuda"))
            mine = by_head[:, lo:hi].flatten(1, 2)
            for part, x in zip(parts, _part(mine, k.transpose(0, 1), v.transpose(0, 1), None)):
                part[:, lo:hi] = x.unflatten(1, (hi - lo, group))
    new, most = state["new"], max(n - c for n, c in zip(state["counts"], _common_of(state)))
    tokens = common[:, None] + torch.arange(max(1, most), device="cuda")
    k, v = (x.transpose(1, 2) for x in _gather(state, state["pages"], tokens))          # [seqs, heads, most, dim]
    j = torch.arange(new, device="cuda")
    counts = (starts[1:] - starts[:-1])[:, None]
    at = (starts[:-1, None] + j).clamp(max=rows - 1)
    padded = by_head[:, at].transpose(0, 1).flatten(2, 3)                               # [seqs, heads, new * group, dim]
    seen = (tokens[:, None] <= (lens[:, None] - counts + j)[..., None]) & (j < counts)[..., None]
    own_parts = _part(padded, k, v, seen.repeat_interleave(group, 1)[:, None])
    live = j < counts                                                                   # [seqs, new]
    m1, l1, o1 = (x.unflatten(2, (new, group)).transpose(1, 2)[live].transpose(0, 1) for x in own_parts)
    m0, l0, o0 = parts
    m = torch.maximum(m0, m1)
    f0, f1 = (m0 - m).exp(), (m1 - m).exp()
    out = (o0 * f0 + o1 * f1) / (l0 * f0 + l1 * f1).clamp(min=1e-37)
    return {"out": out.transpose(0, 1).reshape(q.shape).half()}


def _common_of(state):
    """Tokens in whole common pages of every sequence (0 for an idle slot)."""
    out = []
    for g, n in enumerate(state["common"]):
        out += [n if state["counts"][i] else 0 for i in range(state["first"][g], state["first"][g + 1])]
    return out


def _weigh(state):
    q, lens, starts, new = state["q"], state["lens"].long(), state["starts"].long(), state["new"]
    seqs, heads, dim = lens.shape[0], state["k"].shape[1], q.shape[-1]
    group = q.shape[1] // heads
    token = torch.arange(state["context"], device="cuda")
    ids = state["pages"].long().gather(1, (token // state["page"]).expand(seqs, -1)).clamp(min=0)
    at = (token % state["page"]).expand(seqs, -1)
    k = (state["k"][ids, :, at].float() * state["scales"][ids][..., :1]).transpose(1, 2)
    j = torch.arange(new, device="cuda")
    counts = (starts[1:] - starts[:-1])[:, None]
    rows = (starts[:-1, None] + j).clamp(max=q.shape[0] - 1)
    padded = q[rows].float().view(seqs, new, heads, group, dim).permute(0, 2, 1, 3, 4).flatten(2, 3)
    z = padded @ k.transpose(-1, -2) * dim ** -0.5                                      # [seqs, heads, new * group, context]
    position = (lens[:, None] - counts + j)[..., None]
    seen = (token <= position) & (j < counts)[..., None]
    if state["window"]:
        seen &= token > position - state["window"]
    z.masked_fill_(~seen.repeat_interleave(group, 1)[:, None], -math.inf)
    p = z.sub_(z.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    # a sum over thousands of rows in 64 bits: the weights of far tokens are small next to it
    added = (p / p.sum(-1, keepdim=True).clamp(min=1e-37)).sum(2, dtype=torch.float64)
    old = token < (lens[:, None] - counts)
    before = state["mass"] * torch.where(counts > 0, state["decay"], 1.0)[..., None]
    total = torch.where(old[:, None], before, 0) + added
    return {"mass": torch.where((token < lens[:, None])[:, None], total, 0).float()}


def _evict(state):
    page, lens, kept, count, recent = (state[k] for k in ("page", "lens", "kept", "count", "recent"))
    lens, kept = lens.long()[:, None, None], torch.minimum(kept, lens).long()[:, None, None]
    last = kept.clamp(max=recent)
    token = torch.arange(state["context"], device="cuda")
    # the heaviest of those that are not among the last
    mass = torch.where(state["mass"].isnan(), -math.inf, state["mass"])
    order = torch.where(token < lens - last, mass, -math.inf).sort(dim=-1, descending=True, stable=True).indices
    chosen = torch.zeros(mass.shape, dtype=torch.bool, device="cuda")
    chosen.scatter_(-1, order, (token < kept - last).expand(mass.shape))
    chosen |= (token >= lens - last) & (token < lens)
    slot = torch.arange(count, device="cuda")
    tokens = torch.where(chosen, token, state["context"]).sort(-1).values[..., :count]  # [seqs, heads, count]
    there = slot < kept
    tokens = torch.where(there, tokens, 0)
    out_mass = torch.where(there, mass.gather(-1, tokens), 0)
    seqs, heads, dim = mass.shape[0], mass.shape[1], state["k"].shape[3]
    ids = state["pages"].long()[:, None].expand(-1, heads, -1).gather(2, tokens // page).clamp(min=0)
    h, at = torch.arange(heads, device="cuda")[:, None], tokens % page
    n = -(-count // page)
    pad = n * page - count
    result = {}
    to = state["to"].long()
    live = to >= 0                                                                      # [seqs, pages kept]
    for which, name in enumerate("kv"):
        q = state["k"][ids, h, at] if which == 0 else state["v"][ids, h, at // 16, :, at % 16]
        scale = torch.where(there, state["scales"][ids, h, which], 0)
        wide = torch.nn.functional.pad(scale, (0, pad)).unflatten(-1, (n, page))
        top = wide.amax(-1)                                                             # [seqs, heads, n]
        grown = top.repeat_interleave(page, -1)[..., :count]
        ratio = torch.where(grown > 0, scale / grown, 0)
        whole = (q.float() * ratio[..., None]).round()
        value = torch.where(there[..., None], whole * grown[..., None], 0).half()
        # into the new pages
        paged = torch.nn.functional.pad(whole, (0, 0, 0, pad)).to(torch.int8).view(seqs, heads, n, page, dim).transpose(1, 2)
        if which == 0:
            state["k"][to[live]] = paged[live]
        else:
            state["v"][to[live]] = paged[live].unflatten(2, (page // 16, 16)).transpose(-1, -2)
        state["scales"][to[live], :, which] = top.transpose(1, 2)[live]
        # the last `count` tokens of every sequence, as a reader of the cache gets them
        back = slot - count + kept
        back = torch.where((back >= 0)[..., None], value.gather(2, back.clamp(min=0).expand(seqs, heads, -1)[..., None]
                                                                .expand(-1, -1, -1, dim)), 0)
        result[name] = back.transpose(1, 2)
    return {**result, "mass": out_mass}


def _score(state):
    x = state["logits"].float()
    x = torch.where(x.isnan(), -math.inf, x)
    rows, vocab = x.shape
    inverse = 1.0 if state["temperature"] is None else 1 / state["temperature"][:, None]
    t = (x - x.amax(-1, keepdim=True)) * inverse
    e = t.exp()
    total = e.sum(-1, keepdim=True)
    log_total = total.log()
    entropy = log_total[:, 0] - torch.where(e > 0, e * t, 0).sum(-1) / total[:, 0]
    # the order by logit, then by index from the first on, in one number
    b = torch.where(x == 0, 0.0, x).view(torch.int32)
    key = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long() << 32 | (vocab - torch.arange(vocab, device="cuda"))
    top = key.topk(state["top"], sorted=True).indices
    return {"out": t.gather(1, state["given"].long()) - log_total, "entropy": entropy, "top_tokens": top.int(),
            "top_out": t.gather(1, top) - log_total}


# ------------------------------------------------------------------ what a pass cannot do without

def _keys(first, count, window):
    """Sum over `count` rows at positions first.. of the keys that each sees."""
    last = first + count
    if not window:
        return (last * (last + 1) - first * (first + 1)) // 2
    turn = min(max(window, first), last)                             # from here on a row sees the whole window
    return (turn * (turn + 1) - first * (first + 1)) // 2 + (last - turn) * window


def work(case):
    if case["kind"] == "score":
        n = case["rows"] * case["vocab"]
        return {"bytes": (2 if case["half"] else 4) * n + case["rows"] * (8 * case["given"] + 8 * case["top"] + 8),
                "flops": 6 * n}
    heads, dim, page, q_heads = case["kv_heads"], case["dim"], case["page"], case["q_heads"]
    token = 2 * heads * dim + 8 * heads / page                       # keys, values and their scales
    if case["kind"] == "share":
        first, shared, news, own_tokens = _groups(case)
        tokens, pairs = 0, 0
        for g, n in enumerate(shared):
            common = n // page * page
            tokens += common
            for i in range(first[g], first[g + 1]):
                if own_tokens[i]:
                    tokens += n - common + own_tokens[i]
                    pairs += _keys(n + own_tokens[i] - news[i], news[i], 0)
        return {"bytes": int(tokens * token) + 4 * sum(news) * q_heads * dim, "flops": 4 * dim * q_heads * pairs}
    news, lens = _sequences(case)
    if case["kind"] == "weigh":
        window = case["window"]
        seen = sum(n if not window else min(n, m + window - 1) for n, m in zip(lens, news) if m)
        return {"bytes": int(seen * token / 2) + 8 * heads * sum(lens) + 2 * sum(news) * q_heads * dim,
                "flops": 2 * dim * q_heads * sum(_keys(n - m, m, window) for n, m in zip(lens, news))}
    kept = [min(n, case["keep"]) for n in lens]
    back = 2 * heads * dim * (2 * case["seqs"] * max(kept) + sum(kept))              # read again, and out in fp16
    return {"bytes": 4 * heads * (sum(lens) + sum(kept)) + int(2 * token * sum(kept)) + back,
            "flops": 2 * heads * dim * sum(kept)}


# ------------------------------------------------------------------ 64 bits, from the definitions

def exact(case, seed):
    s, dim = _inputs(case, seed), case.get("dim")
    if case["kind"] == "score":
        rows, vocab = s["logits"].shape
        out = {"out": [], "entropy": [], "top_tokens": [], "top_out": []}
        for lo in range(0, rows, 256):
            x = s["logits"][lo:lo + 256].double()
            given = s["given"][lo:lo + 256].long()
            order = x.sort(dim=-1, descending=True, stable=True).indices[:, :case["top"]]
            if s["temperature"] is not None:
                x = x / s["temperature"][lo:lo + 256, None].double()
            logs = x - x.logsumexp(-1, keepdim=True)
            out["out"].append(logs.gather(1, given))
            out["entropy"].append(torch.special.entr(logs.exp()).sum(-1))
            out["top_tokens"].append(order.int())
            out["top_out"].append(logs.gather(1, order))
        return {k: torch.cat(v) for k, v in out.items()}
    heads, q_heads, page = case["kv_heads"], case["q_heads"], case["page"]
    scales = s["scales"].double()

    def tokens_of(i, n):
        """whole numbers and scales of the first n tokens of sequence i: [n, heads, dim], [n, heads]"""
        at = torch.arange(n, device="cuda")
        ids = s["pages"][i].long()[at // page]
        return (s["k"][ids, :, at % page].double(), scales[ids][..., 0],
                s["v"][ids, :, at % page // 16, :, at % 16].double(), scales[ids][..., 1])

    if case["kind"] == "evict":
        _, lens = _sequences(case)
        count, page_of = s["count"], torch.arange(s["count"], device="cuda") // page
        out = {n: torch.zeros((case["seqs"], count, heads, dim), dtype=torch.float64, device="cuda") for n in "kv"}
        out["mass"] = torch.zeros((case["seqs"], heads, count), dtype=torch.float64, device="cuda")
        for i, n in enumerate(lens):
            b = min(n, case["keep"])
            r = min(case["recent"], b)
            if n == 0:
                continue
            k, ks, v, vs = tokens_of(i, n)
            for h in range(heads):
                weight = s["mass"][i, h, :n - r].double()
                heavy = (-weight).sort(stable=True).indices[:b - r]
                kept = torch.cat([heavy.sort().values, torch.arange(n - r, n, device="cuda")])
                out["mass"][i, h, :b] = s["mass"][i, h].double()[kept]
                for name, x, unit in (("k", k, ks), ("v", v, vs)):
                    unit = unit[kept, h]
                    top = torch.zeros(-(-count // page), dtype=torch.float64, device="cuda")
                    top = top.index_reduce(0, page_of[:b], unit, "amax")[page_of[:b], None]
                    out[name][i, count - b:, h] = (x[kept, h] * unit[:, None] / top).round() * top
        return out

    if case["kind"] == "share":
        _, _, news, _ = _groups(case)
        lens, starts, window = s["counts"], s["rows"], 0
        result = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    else:
        news, lens = _sequences(case)
        starts, window = _starts(news), case["window"]
        result = torch.zeros(s["mass"].shape, dtype=torch.float64, device="cuda")
    group = q_heads // heads
    for i, (n, m) in enumerate(zip(lens, news)):
        if n == 0:
            continue
        k, ks, v, vs = tokens_of(i, n)
        k, v = k * ks[..., None], v * vs[..., None]
        position, token = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")
        hidden = token > position
        if window:
            hidden |= token <= position - window
        if case["kind"] == "weigh":
            result[i, :, :n - m] = s["mass"][i, :, :n - m].double() * (case["decay"] if m else 1)
        for h in range(q_heads if m else 0):
            z = s["q"][starts[i]:starts[i + 1], h].double() @ k[:, h // group].T / math.sqrt(dim)
            p = z.masked_fill(hidden, -math.inf).softmax(-1)
            if case["kind"] == "share":
                result[starts[i]:starts[i + 1], h] = p @ v[:, h // group]
            else:
                result[i, h // group, :n] += p.sum(0)
    return {"out" if case["kind"] == "share" else "mass": result}
