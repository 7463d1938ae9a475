"""The served decoder of examples/serve.py: cache, attention and sampling as a program uses them (run on an MI355X)."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve  # noqa: E402

SHAPE = {"hidden": 512, "q": 768, "kv": 256, "inter": 1024}
VOCAB = 3000


def _model(seqs=3):
    return serve.Model(SHAPE, 2, VOCAB, seqs, 90, page_tokens=16)


def test_step_by_step_is_the_prompt():
    """The logits after a prompt and some single tokens are those after the longer prompt: what differs is the
    rounding of weights for prompts (2^-11 of sum |w x|) and of values again as a page's scale grows (a unit of 1/127
    of the page's largest), some hundredths of the logits' size after two layers."""
    assert torch.cuda.is_available(), "GPU test"
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens = torch.randint(0, VOCAB, (3, 40), dtype=torch.int32, device="cuda", generator=gen)
    whole = _model().forward(tokens.flatten(), [40] * 3)
    model = _model()
    model.forward(tokens[:, :21].flatten(), [21] * 3)
    for i in range(21, 40):
        logits = model.forward(tokens[:, i].contiguous(), [1] * 3)
    # and ragged: chunks of different lengths, one sequence waiting
    ragged = _model()
    for lo, hi in (((0, 0, 0), (40, 7, 0)), ((40, 7, 0), (40, 40, 33)), ((40, 40, 33), (40, 40, 40))):
        part = [tokens[s, a:b] for s, (a, b) in enumerate(zip(lo, hi))]
        ragged_logits = ragged.forward(torch.cat(part), [len(p) for p in part])
    size = whole.std()
    for got, rows in ((logits, (0, 1, 2)), (ragged_logits, (2,))):
        for r in rows:
            off = float((got[r] - whole[r]).std() / size)
            print(f"row {r}: off by {off:.4f} of the logits' size", flush=True)
            assert off < 0.05
    assert torch.isfinite(logits).all()


def test_generation_repeats():
    prompt = torch.randint(0, VOCAB, (3, 21), dtype=torch.int32, device="cuda",
                           generator=torch.Generator(device="cuda").manual_seed(5))
    runs = [serve.generate(_model(), prompt, 9, generator=torch.Generator(device="cuda").manual_seed(7)) for _ in range(2)]
    assert torch.equal(*runs) and runs[0].shape == (3, 9)
    assert int(runs[0].min()) >= 0 and int(runs[0].max()) < VOCAB
    greedy = serve.generate(_model(), prompt, 2, temperature=0.0)
    model = _model()
    assert torch.equal(greedy[:, 0].long(), model.forward(prompt.flatten(), [21] * 3).argmax(-1))
