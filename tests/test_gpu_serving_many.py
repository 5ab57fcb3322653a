"""Prompt and cache operators with more sequences than a wave has lanes, and with more than it finds in two steps of 64."""
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftcache, ftprompt

import test_gpu_cache as tc
import test_gpu_prompt as tp


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
@pytest.mark.parametrize("batch,interleaved", [(64, False), (65, True), (300, False), (4097, True)])
def test_append_and_read_of_many_sequences(batch, interleaved, dtype):
    """Bit by bit: new tokens of every sequence, none for some, behind different numbers of places; every other place of the pool as it was."""
    heads, hk, d, ps = 3, 1, 64, 16
    new, starts = [(5 * i) % 11 for i in range(batch)], [(7 * i) % 29 for i in range(batch)]
    new[batch - 1] = 9
    s = tc.Setup(batch, heads, hk, d, ps, dtype, [a + b for a, b in zip(new, starts)], interleaved=interleaved)
    total = sum(new)
    q, k, v = s.normal(total, heads, d), s.normal(total, hk, d), s.normal(total, hk, d)
    rotation = torch.from_numpy(ftcache.rotation_table(64, d)).cuda()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    m = s.model()
    s.ctx.append(s.pool, q, k, v, rotation, tc.bounds(new), tc.ints(starts), s.table_dev, q_out, k_out, torch.cuda.current_stream().cuda_stream)
    which = torch.tensor([b for b, n in enumerate(new) for _ in range(n)])
    place = torch.tensor([p for a, n in zip(starts, new) for p in range(a, a + n)])
    want_q, want_k = (tc.rotated(x.cpu(), rotation.cpu(), place, d, interleaved) for x in (q, k))
    assert torch.equal(q_out.cpu(), want_q) and torch.equal(k_out.cpu(), want_k)
    page, row = s.table[which, place // ps].long(), place % ps
    (kc, ks, kl), (vc, vs, vl) = tc.quantised(want_k), tc.quantised(v.cpu())
    m.k[page, :, row] = kc[..., 0::2] | kc[..., 1::2] << 4
    m.v[page, :, row // 8, :, row % 8] = (vc[..., 0::2] | vc[..., 1::2] << 4).unflatten(-1, (-1, 2))
    m.par[page, :, row // 8, :, row % 8] = torch.cat([ks, kl, vs, vl], -1).view(torch.uint8).unflatten(-1, (4, 2))
    assert torch.equal(s.pool.cpu(), m.raw)
    seen = [torch.empty_like(k) for _ in range(2)]
    s.ctx.read(s.pool, *seen, tc.bounds(new), tc.ints(starts), s.table_dev)
    for got, codes, scale, low in zip(seen, (kc, vc), (ks, vs), (kl, vl)):
        # product and sum in 32 bits, as read computes them
        assert torch.equal(got.cpu(), (codes.float() * scale.float() + low.float()).to(got.dtype))
    assert s.ctx.report() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [64, 65, 130])
def test_few_queries_of_many_sequences_over_long_prefixes(batch):
    """Row tiles that are divided by their keys (up to 64 sequences) and that are not: the formula's results, the same in every call."""
    nq, nk = [(3 * i) % 5 for i in range(batch)], [40 + (97 * i) % 900 for i in range(batch)]
    nq[7], nk[7], nq[batch - 1], nk[batch - 1] = 3, 4000, 2, 2900
    q, k, v = tp.made(batch, sum(nq), sum(nk), 2, 1, 64, ftprompt.BF16)
    ctx = ftprompt.FtPrompt(2, 1, 64, ftprompt.BF16)
    o, again = torch.empty_like(q), torch.empty_like(q)
    ctx.forward(q, k, v, o, tp.bounds(nq), tp.bounds(nk))
    tp.check(o, q, k, v, nq, nk, ftprompt.BF16)
    ctx.forward(q, k, v, again, tp.bounds(nq), tp.bounds(nk))
    assert torch.equal(o, again)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [ftprompt.F16, ftprompt.BF16])
@pytest.mark.parametrize("out", ["input", "32 bits"])
def test_the_bound_of_rounded_weights(d, dtype, out):
    """A row's weights w are rounded to w' = w (1 + e), |e| <= u = eps / 2 of the type, and divided by the sum of the rounded ones:
    o' - o = sum w e (v - o) / sum w', at most u / (1 - u) * max|v - o| <= 2 u max|v| (1 + 2 u).  A 16-bit result adds u of its own magnitude.
    Scores up to 64 carry a relative error of 2^-16 into the weights, twice that into the quotient: 2^-14 covers it and the fp32 sums."""
    lengths = [1, 130, 0, 257, 64]
    total = sum(lengths)
    q, k, v = tp.made(d, total, total, 6, 2, d, dtype)
    out_dtype = dtype if out == "input" else ftprompt.F32
    o = torch.empty(total, 6, d, dtype=tp.TYPES[out_dtype], device="cuda")
    ctx = ftprompt.FtPrompt(6, 2, d, dtype, out_dtype=out_dtype)
    ctx.forward(q, k, v, o, tp.bounds(lengths))
    want, most = tp.plain(q, k, v, lengths, lengths)
    u = float(torch.finfo(tp.TYPES[dtype]).eps) / 2
    bound = (2 * u * (1 + 2 * u) + 2.0 ** -14 + (u if out == "input" else 0.0)) * most
    assert ((o.cpu().double() - want).abs().amax(-1) <= bound).all()
    ctx.close()
