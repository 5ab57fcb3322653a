"""The choice of the next token (ftsample_choose) up to its largest vocabulary, 2^20: rows of more than 256 words of 16 bytes a lane, whose runs are of more than four words.
Against its definition in 64 bits.

Weights are whole multiples of 2^-42 there, each off by up to 2^-43 (and by 2^-46 of itself, the series' next term), sums by 2^20 * (2^-43 + 2^-46) < 2^-22 of the
largest weight, which is 1.  A probability w / all, all >= 1, is off by 2^-22 of itself for its sum, 2^-42 for its weight, and 2^-24 of itself for its rounding: 2^-21 p + 2^-42.  A
border between neighbouring tokens, and the goal u * all, are off by 2^-22 of the largest weight each: a token is right if the goal lies in its part of the sum, or within
2^-21 of it (parts of the least likely tokens are as short as that).
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftsample
from test_gpu_sample import TYPES

pytestmark = pytest.mark.gpu


def one(x, u, temperature, k, p, floor):
    """What is kept of one row x (float64): tokens in their order, their weights, the sums up to each; and the goal."""
    kept = np.argsort(-x, kind="stable")
    kept = kept[x[kept] > -np.inf]
    if temperature <= 0:
        kept, temperature = kept[:1], 1.0
    if k > 0:
        kept = kept[:k]
    w = np.exp((x[kept] - x[kept[0]]) / temperature)
    if p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        limit = p * w.sum()
        n = max(1, int((before < limit).sum()))
        assert n == len(w) or min(abs(before[n] - limit), abs(before[n - 1] - limit)) > 2.0 ** -22
        kept, w = kept[:n], w[:n]
    if floor > 0:
        n = max(1, int((w >= floor).sum()))
        kept, w = kept[:n], w[:n]
    order = np.argsort(kept)
    kept, w = kept[order], w[order]
    upto = np.cumsum(w)
    return kept, w, upto, u * upto[-1]


@pytest.mark.parametrize("dtype", [ftsample.F32, ftsample.F16, ftsample.BF16])
@pytest.mark.parametrize("vocab,offset", [(524288, 0), (524289, 0), (524285, 3), (700001, 1), (1 << 20, 0), (1 << 20, 1)])
def test_largest_vocabularies(vocab, offset, dtype):
    g = torch.Generator().manual_seed(vocab + offset)
    rows = 4
    x = torch.randn((rows, vocab), generator=g) * torch.tensor([[4.0], [1.0], [2.0], [0.1]])
    x[torch.rand((rows, vocab), generator=g) < 0.05] = -np.inf
    x = x.to(TYPES[dtype])
    flat = torch.full((rows * vocab + offset,), 50.0, dtype=TYPES[dtype], device="cuda")
    view = flat[offset:].view(rows, vocab)
    view.copy_(x)
    t, u = torch.tensor([1.0, 0.5, 2.0, 1.0]), torch.rand(rows, generator=g)
    k, p, m = torch.tensor([0, 5000, 300000, 600], dtype=torch.int32), torch.tensor([0.9, 0.6, 0.97, 0.8]), torch.tensor([0.0, 0.01, 0.0, 0.001])
    ctx = ftsample.FtSample(vocab, dtype, max_rows=rows)
    for rules in (dict(), dict(temperature=t), dict(temperature=t, top_p=p), dict(top_k=k), dict(temperature=t, top_k=k, top_p=p, min_p=m), dict(temperature=torch.zeros(rows))):
        tokens, chance = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), -7.0, device="cuda")
        ctx.choose(view, u.cuda(), tokens, probability=chance, stream=torch.cuda.current_stream().cuda_stream, **{n: r.cuda() for n, r in rules.items()})
        for r in range(rows):
            at = lambda name, otherwise: float(rules[name][r]) if name in rules else otherwise  # noqa: E731
            kept, w, upto, goal = one(x[r].double().numpy(), float(u[r]), at("temperature", 1.0), int(at("top_k", 0)), at("top_p", 1.0), at("min_p", 0.0))
            i = int(np.searchsorted(kept, int(tokens[r])))
            assert i < len(kept) and kept[i] == int(tokens[r]), (r, sorted(rules), int(tokens[r]))
            assert upto[i] - w[i] - 2.0 ** -21 <= goal <= upto[i] + 2.0 ** -21, (r, sorted(rules), int(tokens[r]))
            probability = w[i] / upto[-1]
            assert abs(float(chance[r]) - probability) <= 2.0 ** -21 * probability + 2.0 ** -42, (r, sorted(rules), float(chance[r]), probability)
