"""The choice of the next token (ftsample_choose) where few logits can be chosen: fewer than top_k, or most of them too far below the largest to have a weight.
Against its definition in 64 bits, as in test_gpu_sample.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftsample
from test_gpu_sample import TYPES, check

pytestmark = pytest.mark.gpu

ALL = [ftsample.F16, ftsample.BF16, ftsample.F32]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("masked", [0.5, 0.9, 0.95, 0.99])
@pytest.mark.parametrize("vocab", [3000, 6000, 50001])
def test_masked_rows_with_a_large_top_k(vocab, masked, dtype):
    g = torch.Generator().manual_seed(vocab + dtype)
    ks = [257, 290, 600, 1024, 1025, vocab // 2, vocab - 1]
    x = torch.randn((len(ks), vocab), generator=g) * 4
    x[5] *= 10
    x[torch.rand(x.shape, generator=g) < masked] = -np.inf
    x[:, 17] = 9.0
    x = x.to(TYPES[dtype])
    u, k, t = torch.rand(len(ks), generator=g), torch.tensor(ks, dtype=torch.int32), torch.full((len(ks),), 0.3)
    p, m = torch.tensor([0.9, 0.99, 0.5, 0.999, 0.7, 0.95, 0.8]), torch.tensor([0.01, 0.0, 0.2, 1e-6, 0.0, 1e-3, 0.0])
    check(x, u, t, k)
    check(x, u, t, k, p)
    check(x, u, t, k, None, m)
    check(x, u, t, k, p, m)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("far", [60.0, 3e4])
@pytest.mark.parametrize("k", [300, 700, 1500])
def test_top_k_at_the_number_of_logits_that_can_be_chosen(k, far, dtype):
    """As many as top_k, one fewer, one more; near the largest, or all but the largest more than 51 octaves below it."""
    g = torch.Generator().manual_seed(k)
    counts = [k, k - 1, k + 1, k, k - 1, k + 1, 1, 2]
    x = torch.full((len(counts), 4001), -np.inf)
    for r, n in enumerate(counts):
        at = torch.randperm(4001, generator=g)[:n]
        x[r, at] = torch.randn(n, generator=g) * (2 if r < 3 else 1) - (0 if r < 3 else far)
        x[r, at[n // 2]] = 6
    x, u, ks = x.to(TYPES[dtype]), torch.rand(len(counts), generator=g), torch.full((len(counts),), k, dtype=torch.int32)
    check(x, u, top_k=ks)
    check(x, u, top_k=ks, top_p=torch.full((len(counts),), 0.9))


@pytest.mark.parametrize("dtype", ALL)
def test_borders_just_below_zero(dtype):
    """Zeros of both signs and the smallest negative numbers beside larger ones: the border lies among the latter, whose keys end where those of zeros begin."""
    g = torch.Generator().manual_seed(9)
    vocab, zeros, small = 2000, 500, 700
    unit = {ftsample.F16: 2.0 ** -24, ftsample.BF16: 2.0 ** -133, ftsample.F32: 2.0 ** -149}[dtype]
    tops = [1.0, 0.8, 0.93, 1.1, 1.3, 2.0, 0.51, 0.7, 0.61, 1.7]
    rows = len(tops)
    x = np.full((rows, vocab), -np.inf)
    for r in range(rows):
        at = torch.randperm(vocab, generator=g).numpy()
        x[r, at[:zeros:2]], x[r, at[1:zeros:2]] = 0.0, -0.0
        x[r, at[zeros:zeros + small]] = -unit * torch.randint(1, 8, (small,), generator=g).numpy()
        x[r, at[zeros + small:zeros + small + 100]] = -0.6 + 0.5 * torch.rand(100, generator=g).numpy()
        x[r, at[-1]] = tops[r]
    x, u = torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype]), torch.rand(rows, generator=g)
    ks = torch.tensor([zeros + 1 + n for n in (1, 300, 500, 699, 650, 2, 400, 600, 100, 50)], dtype=torch.int32)
    check(x, u, top_k=ks)
    check(x, u, top_k=ks, top_p=torch.full((rows,), 0.95))
    check(x, u, top_p=0.5 + 0.4 * torch.rand(rows, generator=g))
