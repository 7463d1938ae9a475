"""A served decoder from embedding row to sampled token, with random weights.

    python examples/serve.py [--model 4B] [--layers 2] [--prompt 203] [--tokens 16] [--batch 4]

Every layer's projections are Tetra matrices (tetra_gemm for the prompt, tetra_gemv_grouped and tetra_gemv for
single tokens); keys and values go through kv_append into a paged 8-bit cache, kv_attend reads it, and sample draws
the tokens from the 4-bit head's logits.  torch does what is left between them: the norms over the hidden width,
SiLU and the residual sums.
"""

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_35465_amd as tt  # noqa: E402
from paper_2609_35465_amd import workloads  # noqa: E402

HEAD_DIM = 128


def _norm(x, weight):
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight).half()


class Matrix:
    def __init__(self, seed, rows, cols):
        words, sigma, tail = workloads.tetra_matrix(seed, rows, cols)
        self.codes = torch.from_numpy(tt.pack_rows(words, tail, rows, cols)).cuda()
        self.sigma, self.rows, self.cols = torch.from_numpy(sigma).cuda(), rows, cols


class Layer:
    def __init__(self, shape, seed, pages, page_tokens, table, lens):
        hidden, q, kv, inter = (shape[k] for k in ("hidden", "q", "kv", "inter"))
        sizes = [(q, hidden), (kv, hidden), (kv, hidden), (hidden, q), (inter, hidden), (inter, hidden), (hidden, inter)]
        self.q, self.k, self.v, self.o, self.gate, self.up, self.down = (Matrix(seed + i, *s) for i, s in enumerate(sizes))
        heads = kv // HEAD_DIM
        self.cache = tt.make_kv_cache(
            torch.zeros((pages, heads, page_tokens, HEAD_DIM), dtype=torch.int8, device="cuda"),
            torch.zeros((pages, heads, page_tokens // 16, HEAD_DIM, 16), dtype=torch.int8, device="cuda"),
            torch.zeros((pages, heads, 2), device="cuda"), table, lens)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.norms = [1 + 0.1 * torch.randn(n, device="cuda", generator=gen) for n in (hidden, hidden, HEAD_DIM, HEAD_DIM)]


class Model:
    """`seqs` sequences of up to `tokens` tokens each, their pages dealt out in turn."""

    def __init__(self, shape, layers, vocab, seqs, tokens, page_tokens=64, seed=workloads.SEED_BASE):
        self.hidden, self.vocab, self.seqs = shape["hidden"], vocab, seqs
        per_seq = -(-tokens // page_tokens)
        self.table = torch.arange(seqs * per_seq, dtype=torch.int32, device="cuda").view(per_seq, seqs).T.contiguous()
        self.lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.layers = [Layer(shape, seed + 16 * i, seqs * per_seq, page_tokens, self.table, self.lens)
                       for i in range(layers)]
        q, so, _ = workloads.emb4_table(seed, vocab, self.hidden)
        self.embedding = torch.from_numpy(q).cuda(), torch.from_numpy(so).cuda()
        self.norm = torch.ones(self.hidden, device="cuda")
        self.rope = tt.rope_table(per_seq * page_tokens, HEAD_DIM)
        self.product_space, self.attend_space = tt.gemm_workspace(), tt.kv_attend_workspace()
        self.sample_space = tt.sample_workspace(seqs, vocab)

    def _products(self, x, *matrices):
        """y [rows, M] of several matrices of one x: a prompt's rows, or up to eight single tokens."""
        rows = x.shape[0]
        out = [torch.empty((rows, m.rows), device="cuda") for m in matrices]
        if rows <= tt.MAX_BATCH:
            items = [(m.codes, m.sigma, x, y, m.rows, m.cols) for m, y in zip(matrices, out)]
            tt.gemv_grouped(tt.make_problems(items), rows)
        else:
            for m, y in zip(matrices, out):
                tt.gemm(m.codes, m.sigma, x, y, m.rows, m.cols, rows, self.product_space)
        return out

    def forward(self, tokens, counts):
        """Logits [seqs, vocab] after `counts` new tokens of every sequence (tokens int32, one after another)."""
        rows, counts_np = tokens.shape[0], np.asarray(counts)
        starts = torch.from_numpy(np.concatenate([[0], np.cumsum(counts_np)]).astype(np.int32)).cuda()
        self.lens += torch.from_numpy(counts_np.astype(np.int32)).cuda()
        x = torch.empty((rows, self.hidden), device="cuda")
        tt.emb4_gather(*self.embedding, self.vocab, self.hidden, tokens, x)
        most = int(counts_np.max())
        for layer in self.layers:
            q, k, v = self._products(_norm(x, layer.norms[0]), layer.q, layer.k, layer.v)
            rotated = torch.empty(q.shape, dtype=torch.float16, device="cuda")
            tt.kv_append(layer.cache, q, k, v, starts, most, self.rope, rotated, layer.norms[2], layer.norms[3])
            attended = torch.empty_like(rotated)
            tt.kv_attend(layer.cache, rotated, starts, most, attended, self.attend_space)
            x = x + self._products(attended, layer.o)[0]
            gate, up = self._products(_norm(x, layer.norms[1]), layer.gate, layer.up)
            x = x + self._products((torch.nn.functional.silu(gate) * up).half(), layer.down)[0]
        last = _norm(x[starts[1:].long() - 1], self.norm)
        logits = torch.empty((self.seqs, self.vocab), device="cuda")
        for i in range(0, self.seqs, tt.MAX_BATCH):
            part = last[i:i + tt.MAX_BATCH].contiguous()
            tt.head4_gemv(*self.embedding, part, logits[i:i + tt.MAX_BATCH], self.vocab, self.hidden, part.shape[0])
        return logits

    def sample(self, logits, temperature=0.7, top_k=20, top_p=0.95, min_p=0.0, generator=None):
        def full(value, dtype=torch.float32):
            return torch.full((self.seqs,), value, dtype=dtype, device="cuda")

        tokens = full(0, torch.int32)
        u = torch.rand(self.seqs, device="cuda", generator=generator)
        tt.sample(logits, full(temperature), full(top_k, torch.int32), full(top_p), full(min_p), u, tokens,
                  self.sample_space)
        return tokens


def generate(model, prompt, tokens, **settings):
    """[seqs, tokens] drawn after `prompt` [seqs, n] (int32)."""
    logits = model.forward(prompt.flatten(), [prompt.shape[1]] * model.seqs)
    out = []
    for i in range(tokens):
        out.append(model.sample(logits, **settings))
        if i + 1 < tokens:
            logits = model.forward(out[-1], [1] * model.seqs)
    return torch.stack(out, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", choices=sorted(workloads.QWEN3), default="4B")
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=203)
    ap.add_argument("--tokens", type=int, default=16)
    ap.add_argument("--batch", type=int, default=4)
    a = ap.parse_args()
    vocab = 151936
    model = Model(workloads.QWEN3[a.model], a.layers, vocab, a.batch, a.prompt + a.tokens)
    gen = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randint(0, vocab, (a.batch, a.prompt), dtype=torch.int32, device="cuda", generator=gen)
    print(generate(model, prompt, a.tokens, generator=gen).tolist())


if __name__ == "__main__":
    main()
