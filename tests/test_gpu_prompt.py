"""Attention over packed prompts (ftprompt_forward) against the formula in 64 bits.

Tolerance of a result, relative to the largest |v| that the row sees: the products q.k are exact in fp32 but for their sum (below
128 * 2^-24), the weights are rounded to the input type (half a step, u = eps / 2 each, and the weights of a row are >= 0 and divided by
their unrounded sum, so the result is off by at most u * max|v|), and the result is rounded to its type (u of its own magnitude, at most
max|v|).  Scores up to s in magnitude carry an fp32 error of about s * 2^-22, which the exponential turns into a relative one; s <= 64 here: 2^-16.
Together below (2 u + 2^-14) * max|v|, and 2 u of fp16 and bf16 are 2^-10 and 2^-7.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftprompt

TYPES = {ftprompt.F16: torch.float16, ftprompt.BF16: torch.bfloat16, ftprompt.F32: torch.float32}


def tolerance(dtype):
    return float(torch.finfo(TYPES[dtype]).eps) + 2.0 ** -14


def bounds(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def plain(q, k, v, nq, nk, scale=None):
    """The formula, sequence by sequence, in 64 bits on the host; and the largest |v| that each row sees."""
    q, k, v = (x.detach().cpu().double() for x in (q, k, v))
    heads, group, d = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    scale = d ** -0.5 if scale is None else scale
    out, most = torch.zeros(sum(nq), heads, d, dtype=torch.float64), torch.zeros(sum(nq), heads, dtype=torch.float64)
    at_q = at_k = 0
    for a, b in zip(nq, nk):
        for h in range(heads):
            ks, vs = k[at_k:at_k + b, h // group], v[at_k:at_k + b, h // group]
            s = scale * q[at_q:at_q + a, h] @ ks.T
            for i in range(a):
                n = b - a + i + 1
                if n > 0:
                    w = torch.softmax(s[i, :n], 0)
                    out[at_q + i, h] = w @ vs[:n]
                    most[at_q + i, h] = vs[:n].abs().max()
        at_q, at_k = at_q + a, at_k + b
    return out, most


def check(o, q, k, v, nq, nk, dtype, scale=None):
    want, most = plain(q, k, v, nq, nk, scale)
    got = o[:sum(nq)].cpu().double()
    assert torch.isfinite(got).all()
    off = (got - want).abs().amax(-1)
    assert (off <= tolerance(dtype) * most).all(), float((off / most.clamp(min=1e-30)).max())


def made(seed, total_q, total_k, heads, kv_heads, d, dtype, fused=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(TYPES[dtype])
    if fused:
        x = normal(total_q, heads + 2 * kv_heads, d)
        return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    return normal(total_q, heads, d), normal(total_k, kv_heads, d), normal(total_k, kv_heads, d)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftprompt.F16, ftprompt.BF16])
@pytest.mark.parametrize("heads,kv_heads,d,lengths", [
    (1, 1, 64, [1]), (1, 1, 128, [1]), (4, 2, 64, [5]), (8, 1, 128, [63, 64, 65]), (6, 6, 64, [0, 1, 127, 0, 129, 2]),
    (7, 1, 128, [33, 0, 200]), (12, 4, 64, [300, 17]), (5, 1, 64, [257]), (16, 2, 128, [130, 1, 1, 1, 70]), (71, 1, 64, [40, 3]),
    (2, 2, 128, [513]), (3, 1, 128, [1] * 130),
])
def test_packed_lengths(heads, kv_heads, d, lengths, dtype):
    total = sum(lengths)
    q, k, v = made(7 * heads + total, total, total, heads, kv_heads, d, dtype, fused=heads % 2 == 0)
    o = torch.empty(total, heads, d, dtype=TYPES[dtype], device="cuda")
    ctx = ftprompt.FtPrompt(heads, kv_heads, d, dtype)
    ctx.forward(q, k, v, o, bounds(lengths), stream=torch.cuda.current_stream().cuda_stream)
    check(o, q, k, v, lengths, lengths, dtype)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk", [([1, 5, 64], [400, 5, 90]), ([100, 3], [100, 1000]), ([7, 9, 4], [3, 0, 4]), ([0, 2], [50, 2])])
def test_keys_before_the_queries(d, nq, nk):
    """A chunk over its prefix; queries that stand before the first key see nothing and give zeros."""
    q, k, v = made(3, sum(nq), sum(nk), 8, 2, d, ftprompt.BF16)
    o = torch.full((sum(nq), 8, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx = ftprompt.FtPrompt(8, 2, d, ftprompt.BF16)
    ctx.forward(q, k, v, o, bounds(nq), bounds(nk))
    check(o, q, k, v, nq, nk, ftprompt.BF16)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftprompt.F16, ftprompt.BF16])
def test_result_in_32_bits_scale_and_padding(dtype):
    """An own scale; rows behind the last sequence stay as they are; queries, keys and values broadcast over heads and tokens."""
    lengths = [70, 0, 21]
    q, k, v = made(5, 100, 100, 4, 2, 64, dtype)
    v = v[:, :1].expand(-1, 2, -1)
    o = torch.full((100, 4, 64), 7.0, device="cuda")
    ctx = ftprompt.FtPrompt(4, 2, 64, dtype, out_dtype=ftprompt.F32, softmax_scale=0.3)
    ctx.forward(q, k, v, o, bounds(lengths))
    check(o, q, k, v, lengths, lengths, dtype, scale=0.3)
    assert (o[91:] == 7.0).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(64, ftprompt.F16), (128, ftprompt.BF16)])
def test_what_a_query_does_not_see_has_no_influence(d, dtype):
    """NaN and infinities in keys and values behind a query's place, of its own sequence and of others; the queries that see them get what the
    formula gives."""
    lengths = [90, 140]
    q, k, v = made(11, 230, 230, 6, 2, d, dtype)
    o, clean = (torch.empty(230, 6, d, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    ctx = ftprompt.FtPrompt(6, 2, d, dtype)
    ctx.forward(q, k, v, clean, bounds(lengths))
    k2, v2 = k.clone(), v.clone()
    k2[75], k2[89, 0, 3] = float("nan"), float("inf")
    v2[80, 1, 5], v2[85, 0], v2[89] = float("inf"), float("-inf"), float("nan")
    v2[90 + 100, 1, d - 1], k2[229] = float("nan"), float("nan")
    ctx.forward(q, k2, v2, o, bounds(lengths))
    seen = torch.zeros(230, dtype=torch.bool, device="cuda")
    seen[75:90], seen[190:] = True, True
    assert torch.equal(o[~seen], clean[~seen])
    # one value of head 1 is NaN from token 190 on: that element of its query heads only
    assert torch.isnan(o[190:229, 3:, d - 1]).all() and torch.equal(o[190:229, 3:, :d - 1], clean[190:229, 3:, :d - 1])
    assert torch.equal(o[190:229, :3], clean[190:229, :3]) and torch.isnan(o[229]).all()
    ctx.forward(q, k, v2, o, bounds(lengths))
    assert torch.equal(o[:80], clean[:80])
    assert (o[80:89, 3:, 5] == float("inf")).all() and torch.equal(o[80:85, :3], clean[80:85, :3])
    assert (o[85:89, :3] == float("-inf")).all() and torch.isnan(o[89]).all()
    ctx.close()


@pytest.mark.gpu
def test_scores_far_apart_and_without_end():
    """Scores that rise by far more than fp16 weights span, along the keys; infinite ones."""
    n, d = 300, 64
    q, k, v = made(2, n, n, 2, 2, d, ftprompt.F16)
    k *= torch.linspace(0.1, 20, n, device="cuda").view(-1, 1, 1).half()
    q = q.sign() * 2
    o = torch.empty(n, 2, d, dtype=torch.float16, device="cuda")
    ctx = ftprompt.FtPrompt(2, 2, d, ftprompt.F16)
    ctx.forward(q, k, v, o, bounds([n]))
    want, most = plain(q, k, v, [n], [n])
    # scores reach 500: their fp32 sums are off by up to 64 products of 40 at 2^-24 each, and the weights by as much, relatively
    off = (o.cpu().double() - want).abs().amax(-1)
    assert (off <= (tolerance(ftprompt.F16) + 64 * 40 * 2.0 ** -22) * most).all()
    k[:, :, 0] = float("-inf")
    q[:, :, 0] = 1.0
    ctx.forward(q, k, v, o, bounds([n]))
    assert (o == 0).all()
    ctx.close()


@pytest.mark.gpu
def test_on_its_own_stream_and_in_a_graph():
    lengths = [65, 130, 3]
    q, k, v = made(9, 198, 198, 8, 4, 128, ftprompt.BF16)
    ctx = ftprompt.FtPrompt(8, 4, 128, ftprompt.BF16)
    cu = bounds(lengths)
    want = torch.empty(198, 8, 128, dtype=torch.bfloat16, device="cuda")
    ctx.forward(q, k, v, want, cu)
    torch.cuda.synchronize()
    side, o = torch.cuda.Stream(), torch.zeros_like(want)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.forward(q, k, v, o, cu, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(o, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.forward(q, k, v, o, cu, stream=torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        q.copy_(made(20 + i, 198, 198, 8, 4, 128, ftprompt.BF16)[0])
        ctx.forward(q, k, v, want, cu)
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
    ctx.close()


@pytest.mark.gpu
def test_refusals_on_the_gpu():
    q, k, v = made(1, 10, 10, 4, 2, 64, ftprompt.F16)
    ctx = ftprompt.FtPrompt(4, 2, 64, ftprompt.F16)
    o, cu = torch.empty(10, 4, 64, dtype=torch.float16, device="cuda"), bounds([10])
    for bad in [dict(q=q[:, :3]), dict(k=k[:5]), dict(v=v.float()), dict(o=o.float()), dict(q=q.cpu()), dict(cu_q=cu.long()), dict(cu_k=bounds([5, 5])),
                dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(o=o[:1].expand(10, -1, -1)), dict(cu_q=cu[:1])]:
        with pytest.raises((ValueError, TypeError)):
            ctx.forward(**{**dict(q=q, k=k, v=v, o=o, cu_q=cu), **bad})
    with pytest.raises(ftprompt.FtPromptError):       # rows that do not begin at 16 bytes
        ctx.forward(torch.empty(4 * 64 * 10 + 8, dtype=torch.float16, device="cuda")[1:1 + 2560].view(10, 4, 64), k, v, o, cu)
    ctx.forward(q[:0], k[:0], v[:0], o[:0], bounds([0, 0]))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftprompt.F16, ftprompt.BF16])
@pytest.mark.parametrize("heads,kv_heads,d,nq,nk", [
    (4, 1, 64, [20, 0, 7], [6000, 50, 2500]), (2, 2, 128, [3, 130], [4500, 1800]), (8, 2, 128, [1500], [1500]), (1, 1, 64, [2, 1], [9000, 8999]),
])
def test_long_row_tiles_divided_among_workgroups(heads, kv_heads, d, nq, nk, dtype):
    """Few rows over many keys: the same result every time, and the formula's."""
    q, k, v = made(sum(nk), sum(nq), sum(nk), heads, kv_heads, d, dtype)
    ctx = ftprompt.FtPrompt(heads, kv_heads, d, dtype)
    o = torch.empty(sum(nq), heads, d, dtype=TYPES[dtype], device="cuda")
    args = (bounds(nq), bounds(nk))
    ctx.forward(q, k, v, o, *args)
    check(o, q, k, v, nq, nk, dtype)
    first = o.clone()
    for _ in range(5):
        ctx.forward(q, k, v, o.zero_(), *args)
        assert torch.equal(o, first)
    # captured, between eager calls of the same context
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.forward(q, k, v, o, *args, stream=torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        q.copy_(made(i, sum(nq), 1, heads, kv_heads, d, dtype)[0])
        ctx.forward(q, k, v, first, *args)
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, first)
    check(o, q, k, v, nq, nk, dtype)
    ctx.close()


@pytest.mark.gpu
def test_infinite_values_in_divided_row_tiles():
    """Values that only later queries see, at the end of a long row tile and inside one of its shares."""
    nk = 3000
    q, k, v = made(31, 100, nk, 2, 1, 64, ftprompt.BF16)
    ctx = ftprompt.FtPrompt(2, 1, 64, ftprompt.BF16)
    o, clean = (torch.empty(100, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.forward(q, k, v, clean, bounds([100]), bounds([nk]))
    v[nk - 40, 0, 9], v[nk - 1], k[nk - 20, 0, 0] = float("inf"), float("nan"), float("nan")
    ctx.forward(q, k, v, o, bounds([100]), bounds([nk]))
    assert torch.equal(o[:60], clean[:60])
    assert (o[60:80, :, 9] == float("inf")).all() and torch.isnan(o[80:]).all()
    keep = [e for e in range(64) if e != 9]
    assert torch.equal(o[60:80][..., keep], clean[60:80][..., keep])
    v[100, 0, 3] = float("-inf")
    ctx.forward(q, k, v, o, bounds([100]), bounds([nk]))
    assert (o[:80, :, 3] == float("-inf")).all() and torch.equal(o[:60][..., 4:], clean[:60][..., 4:])
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [65, 300])
def test_many_sequences(batch):
    """More sequences than a wave has lanes, one of them long."""
    lengths = [(7 * i) % 23 for i in range(batch)]
    lengths[batch // 2] = 1700
    total = sum(lengths)
    q, k, v = made(batch, total, total, 2, 1, 64, ftprompt.F16)
    o = torch.empty(total, 2, 64, dtype=torch.float16, device="cuda")
    ctx = ftprompt.FtPrompt(2, 1, 64, ftprompt.F16)
    ctx.forward(q, k, v, o, bounds(lengths))
    check(o, q, k, v, lengths, lengths, ftprompt.F16)
    ctx.close()


@pytest.mark.gpu
def test_the_result_in_place_of_the_queries_and_no_keys_at_all():
    lengths = [300, 40]
    q, k, v = made(77, 340, 340, 4, 4, 128, ftprompt.F16)
    ctx = ftprompt.FtPrompt(4, 4, 128, ftprompt.F16)
    o = torch.empty_like(q)
    ctx.forward(q, k, v, o, bounds(lengths))
    ctx.forward(q, k, v, q, bounds(lengths))
    assert torch.equal(q, o)
    o.fill_(7.0)
    ctx.forward(q, k[:0], v[:0], o, bounds(lengths), bounds([0, 0]))
    assert (o == 0).all()
    ctx.close()


@pytest.mark.gpu
def test_bounds_that_fall_leave_the_next_call_right():
    """Bounds that fall, lie beyond the tensors or below 0 read and write nothing out of range, and the calls behind them are as ever."""
    nq, nk = [20, 30], [5000, 3000]
    q, k, v = made(8, 50, 8000, 4, 1, 64, ftprompt.BF16)
    ctx = ftprompt.FtPrompt(4, 1, 64, ftprompt.BF16)
    o, want = (torch.empty(50, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.forward(q, k, v, want, bounds(nq), bounds(nk))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for bad_q, bad_k in [([0, 40, 10], [0, 5000, 8000]), ([0, 50, 90], [0, 9000, 20000]), ([-5, 20, 50], [-7, 6000, 100]), ([0, 20, 50], [0, 8000, 3000]),
                         ([50, 20, 0], [8000, 5000, 0]), ([2 ** 31 - 1, 0, 2 ** 31 - 1], [0, 2 ** 31 - 1, 0])]:
        ctx.forward(q, k, v, o, ints(bad_q), ints(bad_k))
        for _ in range(2):
            ctx.forward(q, k, v, o.zero_(), bounds(nq), bounds(nk))
            assert torch.equal(o, want)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_rows_far_apart(d):
    """Tokens 2^24 elements apart, the most that is allowed: 10 GB between the first row and the last."""
    lengths, stride = [170, 130], 2 ** 24
    whole = torch.empty(300 * stride, dtype=torch.bfloat16, device="cuda")
    view = lambda at, heads: torch.as_strided(whole, (300, heads, d), (stride, 2 * d, 1), at)
    q, k, v, o = view(0, 4), view(4096, 2), view(8192, 2), view(12288, 4)
    for x, y in zip((q, k, v), made(13, 300, 300, 4, 2, d, ftprompt.BF16)):
        x.copy_(y)
    ctx = ftprompt.FtPrompt(4, 2, d, ftprompt.BF16)
    ctx.forward(q, k, v, o, bounds(lengths))
    check(o, q, k, v, lengths, lengths, ftprompt.BF16)
    with pytest.raises(ftprompt.FtPromptError):
        ctx.forward(torch.as_strided(whole, (290, 4, d), (stride + 8, 2 * d, 1), 0), k[:290], v[:290], o[:290], bounds([290]))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftprompt.F16, ftprompt.BF16])
@pytest.mark.parametrize("heads,kv_heads,d", [(16, 4, 128), (12, 3, 64)])
def test_divided_row_tiles_many_times(heads, kv_heads, d, dtype):
    """Chunks behind prefixes, with the chip full and the states of many shares on their way at once: the same bits in every call and in every context."""
    nq, nk = [509, 60, 301, 77, 440, 130], [3509, 1060, 2301, 877, 2440, 3130]
    q, k, v = made(5, sum(nq), sum(nk), heads, kv_heads, d, dtype)
    o = torch.empty(40, sum(nq), heads, d, dtype=TYPES[dtype], device="cuda")
    args = (bounds(nq), bounds(nk))
    first = None
    for _ in range(8):
        ctx = ftprompt.FtPrompt(heads, kv_heads, d, dtype)
        o.zero_()
        for i in range(40):
            ctx.forward(q, k, v, o[i], *args, stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        ctx.close()
        first = o[0].clone() if first is None else first
        differ = (o != first).flatten(1).any(1)
        assert not differ.any(), differ.nonzero().flatten().tolist()
