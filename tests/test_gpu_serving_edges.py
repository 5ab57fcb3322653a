"""Prompt and cache operators at the ends of their types' ranges: infinite values with weights that vanish, sums near the largest number."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftcache, ftprompt

TYPES = {ftprompt.F16: torch.float16, ftprompt.BF16: torch.bfloat16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def far_below(d, dtype, n, g):
    """Queries, and keys whose scores lie between -1 and 1, but for those that are set to -4: theirs lie below -100, and their weights below 2^-150."""
    q = torch.full((n, 2, d), 4.0, dtype=TYPES[dtype], device="cuda")
    k = (torch.randn((n, 1, d), generator=g, device="cuda") * 0.02).to(TYPES[dtype])
    return q, k


def infinite_ones(v, seen):
    """[query, D]: the sum of the values of v [key, D] that are not finite among the first seen[i] keys, 0 where there are none."""
    strange = torch.where(torch.isfinite(v), torch.zeros_like(v), v).double()
    return torch.stack([strange[:max(0, n)].sum(0) for n in seen])


def check_infinite(o, clean, v, seen):
    """o [query, head, D]: what is not finite comes through whatever its weight; all other elements are those of the finite values."""
    want = infinite_ones(v[:, 0].cpu(), seen)[:, None].expand(o.shape)
    o, clean = o.cpu(), clean.cpu()
    there = want != 0
    assert there.any() and torch.equal(torch.nan_to_num(o[there].double(), 7.0), torch.nan_to_num(want[there], 7.0))
    assert torch.equal(o[~there], clean[~there])


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(64, ftprompt.F16), (128, ftprompt.F16), (64, ftprompt.BF16), (128, ftprompt.BF16)])
def test_infinite_values_whose_weights_vanish(d, dtype):
    """In key tiles that every row of a workgroup sees whole, and in those that some do not."""
    n = 517
    q, k = far_below(d, dtype, n, generator(d))
    v = torch.randn((n, 1, d), generator=generator(1), device="cuda").to(TYPES[dtype])
    at = {3: (0, math.inf), 64: (7, -math.inf), 65: (8, math.nan), 130: (d - 1, math.inf), 255: (1, -math.inf), 300: (0, -math.inf), 511: (9, math.inf)}
    for j in at:
        k[j] = -4.0
    strange = v.clone()
    for j, (e, x) in at.items():
        strange[j, 0, e] = x
    ctx = ftprompt.FtPrompt(2, 1, d, dtype)
    clean, o = torch.empty_like(q), torch.empty_like(q)
    ctx.forward(q, k, v, clean, ints([0, n]))
    ctx.forward(q, k, strange, o, ints([0, n]))
    check_infinite(o, clean, strange, range(1, n + 1))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(64, ftprompt.F16), (128, ftprompt.BF16)])
def test_infinite_values_in_shares_whose_weights_vanish(d, dtype):
    """Few queries over many keys, which several workgroups share: the scores of a whole share lie far below the others'."""
    nq, nk = 40, 6000
    _, k = far_below(d, dtype, nk, generator(d))
    q = torch.full((nq, 2, d), 4.0, dtype=TYPES[dtype], device="cuda")
    v = torch.randn((nk, 1, d), generator=generator(2), device="cuda").to(TYPES[dtype])
    k[:3500] = -4.0
    k[5000:5980] = -4.0
    strange = v.clone()
    strange[100, 0, 3], strange[2000, 0, 5], strange[2001, 0, 5], strange[5500, 0, 6], strange[5975, 0, 11] = math.inf, math.inf, -math.inf, -math.inf, math.inf
    ctx = ftprompt.FtPrompt(2, 1, d, dtype)
    clean, o = torch.empty_like(q), torch.empty_like(q)
    ctx.forward(q, k, v, clean, ints([0, nq]), ints([0, nk]))
    ctx.forward(q, k, strange, o, ints([0, nq]), ints([0, nk]))
    check_infinite(o, clean, strange, range(nk - nq + 1, nk + 1))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [50, 400])
def test_scores_of_minus_infinity_with_infinite_values(n):
    """Queries that see only scores of -infinity give zeros, whatever the values."""
    d = 64
    q, k = far_below(d, ftprompt.F16, n, generator(0))
    v = torch.randn((n, 1, d), generator=generator(3), device="cuda").half()
    k[:, :, 0] = -math.inf
    v[3, 0, 5], v[n - 2, 0, 6], v[7, 0, 7] = math.inf, -math.inf, math.nan
    ctx = ftprompt.FtPrompt(2, 1, d, ftprompt.F16)
    o = torch.empty_like(q)
    ctx.forward(q, k, v, o, ints([0, n]))
    assert (o == 0).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_values_near_the_largest_number(d):
    """Sums of weights of at most 1 times values stay finite: 128 of 2e36.  Scores of the second half of the keys lie 7.2 powers of two above the first's."""
    n = 128
    q = torch.ones((n, 2, d), dtype=torch.bfloat16, device="cuda")
    k = (torch.randn((n, 1, d), generator=generator(d), device="cuda") * 0.02).bfloat16()
    k[64:] += 5.0 / math.sqrt(d)
    v = (torch.rand((n, 1, d), generator=generator(4), device="cuda") * 1e36 + 1e36).bfloat16()
    ctx = ftprompt.FtPrompt(2, 1, d, ftprompt.BF16)
    o = torch.empty_like(q)
    ctx.forward(q, k, v, o, ints([0, n]))
    s = (q[:, 0].double() @ k[:, 0].double().T / math.sqrt(d)).masked_fill(torch.ones(n, n, device="cuda").triu(1) > 0, -math.inf)
    want = s.softmax(1) @ v[:, 0].double()
    # weights rounded to bf16, divided by the sum of the rounded ones: u = 2^-8 of each and of their sum; the result's rounding another u; fp32 sums
    assert ((o.double() - want[:, None]).abs() <= (3 * 2.0 ** -8 + 2.0 ** -14) * 2e36).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", [(64, 100), (128, 100), (64, 5000)])
def test_cached_values_near_the_largest_number(d, n):
    """As many as let sums of weights of at most 1 times values stay finite."""
    top = 2.5e38 / n
    k = torch.randn((n, 1, d), generator=generator(d), device="cuda").bfloat16()
    v = ((torch.rand((n, 1, d), generator=generator(5), device="cuda") * 2 - 1) * top).bfloat16()
    q = torch.randn((1, 2, d), generator=generator(6), device="cuda").bfloat16()
    pages = (n + 15) // 16
    ctx = ftcache.FtCache(2, 1, d, pages, 16, ftcache.BF16)
    pool = torch.zeros(pages * ctx.page_bytes, dtype=torch.uint8, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    rotation = torch.from_numpy(ftcache.rotation_table(n, d)).cuda()
    ctx.append(pool, None, k, v, rotation, ints([0, n]), ints([0]), table, None, None)
    o = torch.empty_like(q)
    ctx.attend(pool, q, o, ints([n]), table)
    seen = [torch.empty_like(k) for _ in range(2)]
    ctx.read(pool, *seen, ints([0, n]), ints([0]), table)
    ks, vs = (x[:, 0].double() for x in seen)
    want = (q[0].double() @ ks.T / math.sqrt(d)).softmax(-1) @ vs
    # cached keys rounded to bf16 by read: a score is off by at most 2^-8 * sum |q k| / sqrt(d); the weight by twice as much, relatively; the weights'
    # rounding over codes 2 * 2^-8, read's rounding of values and the result's own 2^-8 each, fp32 sums
    scores = 2.0 ** -8 * (q[0].double().abs() @ ks.abs().T / math.sqrt(d)).max()
    assert ((o[0].double() - want).abs() <= (2 * scores + 4 * 2.0 ** -8 + 2.0 ** -14) * vs.abs().max()).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
def test_cached_values_beyond_the_largest_number(dtype):
    """A scale that was rounded up takes the largest code of the largest number beyond it: the result is held to the type's numbers as a value read back is."""
    d, top = 64, float(torch.finfo(TYPES[dtype]).max)
    v = torch.full((3, 1, d), top, device="cuda")
    v[:, 0, ::2] *= -1
    v = v.to(TYPES[dtype])
    k = torch.ones_like(v)
    q = torch.ones((1, 1, d), dtype=v.dtype, device="cuda")
    ctx = ftcache.FtCache(1, 1, d, 1, 16, dtype)
    pool = torch.zeros(ctx.page_bytes, dtype=torch.uint8, device="cuda")
    table, rotation = ints([[0]]), torch.from_numpy(ftcache.rotation_table(16, d)).cuda()
    ctx.append(pool, None, k, v, rotation, ints([0, 3]), ints([0]), table, None, None)
    o, seen = torch.empty_like(q), [torch.empty_like(k) for _ in range(2)]
    ctx.read(pool, *seen, ints([0, 3]), ints([0]), table)
    ctx.attend(pool, q, o, ints([1]), table)
    assert torch.isfinite(seen[1]).all() and torch.isfinite(o).all()
    # one token, weight 1: the same value, but for the rounding of weight times scale over 15 steps and that of the offset's sums
    assert ((o[0].double() - seen[1][0].double()).abs() <= (2 * 2.0 ** -8 + 2.0 ** -8) * top).all()
    ctx.close()
