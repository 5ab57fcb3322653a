"""The paged cache in 4 bits (ftcache_*) against its definition, spelled out here on the host.

Rotation and codes are defined in 32 bits, operation by operation, so what append writes is compared bit by bit.
Attention, relative to the largest |v| among a row's cached values: codes are exact operands; the query is exact (bf16) or exact but for
elements 2^-25 below the largest one (fp16); scores up to s carry an fp32 error of about s * 2^-21 (two sums of up to 128 products, codes
up to 15 against differences of a few of them), the weights as much, relatively: 2^-15 for s <= 64.  A weight times its value's scale is
rounded to bf16 (bf16: half a step, 2^-8; fp16: two words, 2^-16) and multiplied by codes and by the offset 128 that leaves again, exactly, in
fp32 sums: codes <= 15 of 15 steps that span at most twice max|v|: 2 * 2^-8 (2 * 2^-16) and 143 / 15 * 2 * 2^-22 for the sums.  Then the result's own rounding.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftcache, ftprompt

TYPES = {ftcache.F16: torch.float16, ftcache.BF16: torch.bfloat16, ftcache.F32: torch.float32}


def tolerance(dtype, out):
    weights = 2 * 2.0 ** -8 if dtype == ftcache.BF16 else 2 * 2.0 ** -16
    return weights + 2.0 ** -15 + 20 * 2.0 ** -22 + (0 if out == ftcache.F32 else float(torch.finfo(TYPES[out]).eps) / 2)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bounds(lengths):
    return ints(np.concatenate([[0], np.cumsum(lengths)]).tolist())


def rotated(x, table, places, rotary, interleaved):
    y, c, s = x.float(), table[places][:, None, :rotary // 2], table[places][:, None, rotary // 2:]
    a, b = (y[..., 0:rotary:2], y[..., 1:rotary:2]) if interleaved else (y[..., :rotary // 2], y[..., rotary // 2:rotary])
    u, v = a * c - b * s, b * c + a * s
    z = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([z, y[..., rotary:]], -1).to(x.dtype)


def quantised(x):
    """(codes, scale, minimum) of x [..., D]."""
    y = x.float()
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    scale = (hi / 15 - lo / 15).to(x.dtype)
    codes = ((y * 0.5 - lo * 0.5) / (scale.float() * 0.5)).round().clamp(0, 15)
    codes = torch.where(scale.float() == 0, 0.0, codes)
    fine = torch.isfinite(y).all(-1, keepdim=True)
    nan = torch.full_like(scale, float("nan"))
    return torch.where(fine, codes, 0.0).to(torch.uint8), torch.where(fine, scale, nan), torch.where(fine, lo.to(x.dtype), nan)


class Model:
    """The pool on the host, byte for byte."""

    def __init__(self, pool, kv_heads, d, page_size, dtype):
        self.raw, self.hk, self.d, self.ps, self.dtype = pool.cpu().clone(), kv_heads, d, page_size, TYPES[dtype]
        pages = self.raw.view(-1, kv_heads, page_size * (d + 8))
        self.k = pages[:, :, :page_size * d // 2].unflatten(-1, (page_size, d // 2))
        self.v = pages[:, :, page_size * d // 2:page_size * d].unflatten(-1, (page_size // 8, d // 4, 8, 2))
        self.par = pages[:, :, page_size * d:].unflatten(-1, (page_size // 8, 4, 8, 2))

    def put(self, page, row, k, v):
        """One token: k, v [kv_heads, D]."""
        (kc, ks, kl), (vc, vs, vl) = quantised(k), quantised(v)
        self.k[page, :, row] = kc[:, 0::2] | kc[:, 1::2] << 4
        self.v[page, :, row // 8, :, row % 8] = (vc[:, 0::2] | vc[:, 1::2] << 4).unflatten(-1, (-1, 2))
        self.par[page, :, row // 8, :, row % 8] = torch.cat([ks, kl, vs, vl], -1).view(torch.uint8).unflatten(-1, (4, 2))

    def get(self, page, row):
        """One token in 64 bits: k, v [kv_heads, D], before rounding."""
        kb, vb = self.k[page, :, row], self.v[page, :, row // 8, :, row % 8].flatten(-2)
        par = self.par[page, :, row // 8, :, row % 8].contiguous().view(self.dtype).squeeze(-1).double()
        k, v = (torch.stack([x & 15, x >> 4], -1).flatten(-2).double() for x in (kb, vb))
        return k * par[:, 0:1] + par[:, 1:2], v * par[:, 2:3] + par[:, 3:4]

    def sequence(self, table, first, n):
        rows = [self.get(int(table[p // self.ps]), p % self.ps) for p in range(first, first + n)]
        return torch.stack([r[0] for r in rows]), torch.stack([r[1] for r in rows])


class Setup:
    def __init__(self, seed, heads, kv_heads, d, page_size, dtype, whole, out=None, spare=2, **more):
        """Pages for sequences of `whole` tokens in shuffled order, pool of random bytes but sound parameters."""
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.heads, self.hk, self.d, self.ps, self.dtype, self.out = heads, kv_heads, d, page_size, dtype, dtype if out is None else out
        need = [(n + page_size - 1) // page_size for n in whole]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=self.g, device="cuda").tolist()
        self.table = torch.full((len(whole), max(1, max(need))), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.table_dev = self.table.cuda()
        self.ctx = ftcache.FtCache(heads, kv_heads, d, self.pages, page_size, dtype, out_dtype=self.out, max_batch=len(whole), **more)
        assert self.ctx.page_bytes == kv_heads * page_size * (d + 8)
        self.pool = torch.randint(0, 256, (self.pages * self.ctx.page_bytes,), dtype=torch.uint8, generator=self.g, device="cuda")
        par = self.pool.view(self.pages, kv_heads, -1)[:, :, page_size * d:].unflatten(-1, (page_size // 8, 4, 8, 2))
        n = torch.rand((self.pages, kv_heads, page_size // 8, 4, 8), generator=self.g, device="cuda") * 0.1 + 0.2
        n[:, :, :, 1::2] *= -8
        par.copy_(n.to(TYPES[dtype]).unsqueeze(-1).view(torch.uint8))

    def model(self):
        return Model(self.pool, self.hk, self.d, self.ps, self.dtype)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda").to(TYPES[self.dtype])

    def check_attend(self, o, q, lengths, scale=None):
        m, group = self.model(), self.heads // self.hk
        scale = self.d ** -0.5 if scale is None else scale
        for b, n in enumerate(lengths):
            if n == 0:
                assert (o[b] == 0).all()
                continue
            k, v = m.sequence(self.table[b].tolist(), 0, n)
            for h in range(self.heads):
                w = torch.softmax(scale * k[:, h // group] @ q[b, h].cpu().double(), 0)
                want, most = w @ v[:, h // group], v[:, h // group].abs().max()
                off = (o[b, h].cpu().double() - want).abs().max()
                assert off <= tolerance(self.dtype, self.out) * most, (b, h, float(off / most))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
@pytest.mark.parametrize("heads,kv_heads,d,page_size,rotary,interleaved,new,starts", [
    (4, 2, 64, 16, 64, False, [1, 1, 1], [0, 5, 31]), (8, 1, 128, 16, 128, False, [3, 0, 20, 1], [6, 3, 0, 16]),
    (3, 3, 64, 32, 32, True, [40, 1], [1, 31]), (5, 1, 128, 64, 96, False, [9, 70], [63, 0]), (6, 2, 128, 16, 128, True, [8, 16, 7], [8, 0, 9]),
    (2, 1, 64, 128, 16, False, [130], [100]), (1, 1, 128, 1024, 64, True, [1], [1023]),
])
def test_append_and_read_bit_by_bit(heads, kv_heads, d, page_size, rotary, interleaved, new, starts, dtype):
    s = Setup(heads + rotary, heads, kv_heads, d, page_size, dtype, [a + b for a, b in zip(new, starts)], rotary_dim=rotary, interleaved=interleaved)
    total, behind = sum(new), 3
    qkv = s.normal(total + behind, heads + 2 * kv_heads, d)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    table = torch.from_numpy(ftcache.rotation_table(max(a + b for a, b in zip(new, starts)), rotary))
    q_out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    m = s.model()
    s.ctx.append(s.pool, q, k, v, table.cuda(), bounds(new), ints(starts), s.table_dev, q_out, k_out, torch.cuda.current_stream().cuda_stream)
    places = torch.tensor([p for a, b in zip(starts, new) for p in range(a, a + b)], dtype=torch.long)
    want_q, want_k = (rotated(x[:total].cpu(), table, places, rotary, interleaved) for x in (q, k))
    assert torch.equal(q_out[:total].cpu(), want_q) and torch.equal(k_out[:total].cpu(), want_k)
    assert (q_out[total:] == 7.0).all() and (k_out[total:] == 7.0).all()
    t = 0
    for b, n in enumerate(new):
        for p in range(starts[b], starts[b] + n):
            m.put(int(s.table[b, p // page_size]), p % page_size, want_k[t], v[t].cpu())
            t += 1
    assert torch.equal(s.pool.cpu(), m.raw)
    # back: everything that the sequences hold
    whole = [a + b for a, b in zip(new, starts)]
    seen = [torch.full((sum(whole) + behind, kv_heads, d), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    s.ctx.read(s.pool, *seen, bounds(whole), ints([0] * len(new)), s.table_dev)
    parts = [m.sequence(s.table[b].tolist(), 0, n) for b, n in enumerate(whole) if n]
    for got, want in zip(seen, (torch.cat([p[i] for p in parts]) for i in range(2))):
        # product and sum in 32 bits, then rounded: the oracle's 64 bits can lie on the other side of a tie, one step off
        assert (got[:sum(whole)].cpu().double() - want).abs().max() <= torch.finfo(TYPES[dtype]).eps / 2 * want.abs().max() * (1 + 2.0 ** -10)
        assert (got[sum(whole):] == 7.0).all()
    # and only the new ones
    tail = [torch.empty(total, kv_heads, d, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    s.ctx.read(s.pool, *tail, bounds(new), ints(starts), s.table_dev)
    rows = torch.cat([torch.arange(sum(whole[:b]) + starts[b], sum(whole[:b + 1])) for b in range(len(new))]).cuda()
    assert all(torch.equal(a, c[rows]) for a, c in zip(tail, seen))
    assert s.ctx.report() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
def test_codes_of_flat_extreme_and_infinite_heads(dtype):
    """All elements equal; one apart; the type's largest numbers; subnormal ones; infinities and NaN."""
    d = 64
    s = Setup(1, 1, 1, d, 16, dtype, [9])
    top = float(torch.finfo(TYPES[dtype]).max)
    k = torch.full((9, 1, d), 1.25, dtype=TYPES[dtype], device="cuda")
    k[1, 0, 7] = 1.5
    k[2] = torch.where(torch.arange(d, device="cuda") % 2 == 0, top, -top).to(k.dtype)
    k[2, 0, 3] = top / 3
    k[3] = 2.0 ** -24 if dtype == ftcache.F16 else 2.0 ** -133
    k[3, 0, 0] = 0
    k[4, 0, 5], k[5, 0, 63], k[6] = float("nan"), float("-inf"), float("inf")
    k[7] = torch.arange(d, device="cuda").to(k.dtype)
    k[8] = 0
    table = torch.cat([torch.ones(9, d // 2), torch.zeros(9, d // 2)], 1).cuda()
    m = s.model()
    s.ctx.append(s.pool, None, k, k, table, bounds([9]), ints([0]), s.table_dev, None, None)
    for t in range(9):
        m.put(int(s.table[0, 0]), t, k[t].cpu(), k[t].cpu())
    # NaN parameters are compared as NaN: their bits are not specified
    new = s.model()
    assert torch.equal(new.k, m.k) and torch.equal(new.v, m.v)
    a, b = (x.par.contiguous().view(TYPES[dtype]).float() for x in (new, m))
    assert torch.equal(torch.nan_to_num(a, 1234.0), torch.nan_to_num(b, 1234.0))
    seen = [torch.empty_like(k) for _ in range(2)]
    s.ctx.read(s.pool, *seen, bounds([9]), ints([0]), s.table_dev)
    for x in seen:
        assert torch.isnan(x[4:7]).all() and torch.isfinite(x[[0, 1, 2, 3, 7, 8]]).all()
        assert torch.equal(x[0], k[0]) and torch.equal(x[8], k[8]) and torch.equal(x[1], k[1])


@pytest.mark.gpu
def test_append_in_place_and_keys_alone():
    """q_out may be q and k_out k; without queries the cache is the same."""
    s = Setup(4, 6, 2, 128, 16, ftcache.BF16, [20, 3])
    q, k, v = s.normal(23, 6, 128), s.normal(23, 2, 128), s.normal(23, 2, 128)
    table = torch.from_numpy(ftcache.rotation_table(64, 128)).cuda()
    args = (table, bounds([20, 3]), ints([0, 0]), s.table_dev)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    s.ctx.append(s.pool, q, k, v, *args, q_out, k_out)
    want = s.pool.clone()
    s.ctx.append(s.pool.zero_().copy_(want), None, k, v, *args, None, None)
    assert torch.equal(s.pool, want)
    s.ctx.append(s.pool, q, k, v, *args, q, k)
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(s.pool, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
@pytest.mark.parametrize("heads,kv_heads,d,page_size,lengths", [
    (1, 1, 64, 16, [1]), (1, 1, 128, 16, [1, 0, 2]), (8, 2, 128, 16, [31, 32, 33, 127, 128, 129]), (16, 1, 64, 32, [100, 7, 0]),
    (17, 1, 128, 64, [300]), (71, 1, 64, 16, [50, 129]), (12, 12, 64, 128, [200, 1]), (6, 3, 128, 1024, [1000]), (4, 4, 128, 16, [2000, 16]),
    (2, 1, 64, 16, [1, 2, 3, 5] * 20),
])
def test_attention_of_single_tokens(heads, kv_heads, d, page_size, lengths, dtype):
    for out in (dtype, ftcache.F32):
        s = Setup(heads + d, heads, kv_heads, d, page_size, dtype, lengths, out=out)
        q = s.normal(len(lengths), heads, d)
        o = torch.full((len(lengths), heads, d), 7.0, dtype=TYPES[out], device="cuda")
        for _ in range(2):
            s.ctx.attend(s.pool, q, o, ints(lengths), s.table_dev, torch.cuda.current_stream().cuda_stream)
            s.check_attend(o, q, lengths)
        assert s.ctx.report() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
def test_attention_of_one_long_sequence(dtype):
    """Divided among many workgroups, beside short ones; the same result every time."""
    lengths = [30000, 5, 0, 700]
    s = Setup(3, 8, 1, 128, 64, dtype, lengths)
    q = s.normal(4, 8, 128)
    o = torch.empty(4, 8, 128, dtype=TYPES[dtype], device="cuda")
    s.ctx.attend(s.pool, q, o, ints(lengths), s.table_dev)
    first = o.clone()
    for _ in range(5):
        s.ctx.attend(s.pool, q, o.zero_(), ints(lengths), s.table_dev)
        assert torch.equal(o, first)
    m = s.model()
    k, v = (x[:, 0].cuda() for x in m_sequence(s, m, 0, lengths[0]))
    w = torch.softmax(128 ** -0.5 * q[0].double() @ k.T, -1)
    assert ((first[0].double() - w @ v).abs() <= tolerance(dtype, dtype) * v.abs().max()).all()
    for b in (1, 3):
        k, v = (x[:, 0].cuda() for x in m_sequence(s, m, b, lengths[b]))
        w = torch.softmax(128 ** -0.5 * q[b].double() @ k.T, -1)
        assert ((first[b].double() - w @ v).abs() <= tolerance(dtype, dtype) * v.abs().max()).all()
    assert (first[2] == 0).all()


def m_sequence(s, m, b, n):
    """Model.sequence for long sequences, a page at a time."""
    out = []
    for x, first in ((m.k, 0), (m.v, 2)):
        pages = s.table[b].long()[:(n + s.ps - 1) // s.ps]
        codes = x[pages] if first == 0 else x[pages].transpose(3, 4).flatten(4).flatten(2, 3)
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
        par = m.par[pages].contiguous().view(m.dtype).squeeze(-1).double().transpose(3, 4).flatten(2, 3)
        out.append((codes * par[..., first:first + 1] + par[..., first + 1:first + 2]).transpose(1, 2).flatten(0, 1)[:n])
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
def test_what_lies_behind_a_sequence_has_no_influence(dtype):
    lengths = [37, 16, 1]
    s = Setup(8, 4, 2, 64, 16, dtype, lengths)
    q = s.normal(3, 4, 64)
    o, clean = (torch.empty(3, 4, 64, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    s.ctx.attend(s.pool, q, clean, ints(lengths), s.table_dev)
    m = s.model()
    nan = torch.full((2, 8), float("nan"), dtype=TYPES[dtype]).view(torch.uint8).unflatten(-1, (8, 2)).unsqueeze(1).expand(-1, 4, -1, -1)
    for b, n in enumerate(lengths):
        for p in range(n, (n + 15) // 16 * 16):
            m.par[int(s.table[b, p // 16]), :, p % 16 // 8, :, p % 8] = nan[:, :, 0]
    s.pool.copy_(m.raw)
    s.ctx.attend(s.pool, q, o, ints(lengths), s.table_dev)
    assert torch.equal(o, clean)
    # a NaN inside reaches the heads that read it, and no others
    m.par[int(s.table[0, 2]), 1, 0, 1, 3] = nan[0, 0, 0]
    s.pool.copy_(m.raw)
    s.ctx.attend(s.pool, q, o, ints(lengths), s.table_dev)
    assert torch.isnan(o[0, 2:]).all() and torch.equal(o[0, :2], clean[0, :2]) and torch.equal(o[1:], clean[1:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,power", [(ftcache.F16, -18), (ftcache.F16, 5), (ftcache.BF16, -100), (ftcache.BF16, 40)])
def test_queries_of_any_magnitude(dtype, power):
    """A query scaled by a power of two and a softmax scale that takes it back: the same result."""
    lengths = [77]
    a, b = Setup(6, 4, 1, 64, 16, dtype, lengths), Setup(6, 4, 1, 64, 16, dtype, lengths, softmax_scale=0.125 * 2.0 ** -power)
    q = (a.normal(1, 4, 64).float().clamp(-4, 4) * 16).round().div(16).to(TYPES[dtype])
    o, p = (torch.empty(1, 4, 64, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    a.ctx.attend(a.pool, q, o, ints(lengths), a.table_dev)
    b.ctx.attend(a.pool, (q.double() * 2.0 ** power).to(q.dtype), p, ints(lengths), a.table_dev)
    a.check_attend(o, q, lengths)
    assert torch.equal(o, p)


@pytest.mark.gpu
def test_pages_and_places_that_do_not_exist():
    """Counted, NaN in their place, nothing else touched; entries that no place needs may hold anything (-7 everywhere above)."""
    s = Setup(2, 4, 2, 64, 16, ftcache.BF16, [20, 20, 20])
    table = s.table_dev.clone()
    table[1, 1], table[2, 0] = s.pages, -1
    table_rot = torch.from_numpy(ftcache.rotation_table(18, 64)).cuda()      # places 18 and 19 have no rotation
    q, k, v = s.normal(60, 4, 64), s.normal(60, 2, 64), s.normal(60, 2, 64)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    before = s.model()
    s.ctx.append(s.pool, q, k, v, table_rot, bounds([20, 20, 20]), ints([0, 0, 0]), table, q_out, k_out)
    assert s.ctx.report() == (2 + 4 + 18, 0)      # places 18 and 19, 16 to 19, 0 to 15 and 18 and 19
    lost = torch.zeros(60, dtype=torch.bool, device="cuda")
    lost[[18, 19, 38, 39, 58, 59]] = True
    assert torch.isnan(q_out[lost]).all() and torch.isnan(k_out[lost]).all()
    assert torch.isfinite(q_out[~lost]).all() and torch.isfinite(k_out[~lost]).all()
    kept = [(int(s.table[0, p // 16]), p % 16) for p in range(18)] + [(int(s.table[1, 0]), p) for p in range(16)] + [(int(s.table[2, 1]), p) for p in range(2)]
    after = s.model()
    for page in range(s.pages):
        for row in range(16):
            if (page, row) not in kept:
                assert torch.equal(after.k[page, :, row], before.k[page, :, row])
                assert torch.equal(after.v[page, :, row // 8, :, row % 8], before.v[page, :, row // 8, :, row % 8])
    seen = [torch.zeros(60, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    s.ctx.read(s.pool, *seen, bounds([20, 20, 20]), ints([0, 0, 0]), table)
    gone = torch.zeros(60, dtype=torch.bool, device="cuda")
    gone[36:56] = True
    for x in seen:
        assert torch.isnan(x[gone]).all() and torch.isfinite(x[~gone]).all()
    assert s.ctx.report() == (20, 0)
    qq, o = s.normal(3, 4, 64), torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    s.ctx.attend(s.pool, qq, o, ints([20, 16, 20]), table)
    assert torch.isfinite(o[:2]).all() and torch.isnan(o[2]).all() and s.ctx.report() == (0, 1)
    s.ctx.attend(s.pool, qq, o, ints([-1, 33, 2 ** 31 - 1]), s.table_dev)
    assert torch.isnan(o).all() and s.ctx.report() == (0, 3)


@pytest.mark.gpu
def test_far_pages():
    """Pages whose bytes lie beyond 2^32 of a pool."""
    pages = 2 ** 32 // (8 * 1024 * 136) + 40
    d, ps, hk = 128, 1024, 8
    ctx = ftcache.FtCache(8, hk, d, pages, ps, ftcache.F16, max_batch=2)
    pool = torch.empty(pages * ctx.page_bytes, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    n = 1500
    q, k, v = (torch.randn(n, 8, d, generator=g, device="cuda").half() for _ in range(3))
    rotation = torch.from_numpy(ftcache.rotation_table(n, d)).cuda()
    results = []
    for table in (ints([[pages - 1, pages - 2]]), ints([[1, 0]])):
        k_out, q_out, seen = torch.empty_like(k), torch.empty_like(q), [torch.empty_like(k) for _ in range(2)]
        ctx.append(pool, q, k, v, rotation, bounds([n]), ints([0]), table, q_out, k_out)
        ctx.read(pool, *seen, bounds([n]), ints([0]), table)
        o = torch.empty(1, 8, d, dtype=torch.float16, device="cuda")
        ctx.attend(pool, q_out[-1:], o, ints([n]), table)
        results.append([q_out, k_out, *seen, o])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert (results[0][2].float() - results[0][1].float()).abs().max() < 0.5      # half of a step of 4 bits over about 9 sigma
    ctx.close()


@pytest.mark.gpu
def test_streams_and_graphs():
    """Steps in a captured graph, replayed with other inputs between other work of the same context."""
    s = Setup(5, 8, 2, 128, 16, ftcache.BF16, [400, 90, 33])
    rotation = torch.from_numpy(ftcache.rotation_table(512, 128)).cuda()
    q, k, v = s.normal(3, 8, 128), s.normal(3, 2, 128), s.normal(3, 2, 128)
    q_out, o = torch.empty_like(q), torch.empty_like(q)
    starts, lengths, cu = ints([399, 89, 32]), ints([400, 90, 33]), bounds([1, 1, 1])

    def step(out, stream):
        s.ctx.append(s.pool, q, k, v, rotation, cu, starts, s.table_dev, q_out, None, stream)
        s.ctx.attend(s.pool, q_out, out, lengths, s.table_dev, stream)

    step(o, 0)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.empty_like(o)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(other, side.cuda_stream)
    side.synchronize()
    assert torch.equal(o, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(other, torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(s.normal(*x.shape))
        lengths.copy_(ints([400 - i, 90, 33]))
        step(o, torch.cuda.current_stream().cuda_stream)
        other.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, other)
    s.check_attend(o, q_out, [397, 90, 33])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
def test_a_prompt_its_continuation_and_steps(dtype):
    """Prompts in two chunks and three tokens more, as a program runs them; the result of every stage against the formula over what the cache
    holds (steps) or the chunk and the prefix as read back (prompts)."""
    import test_gpu_prompt as tp
    heads, hk, d, ps = 8, 2, 64, 16
    first, second, steps = [40, 3, 17], [25, 60, 1], 3
    s = Setup(12, heads, hk, d, ps, dtype, [a + b + steps for a, b in zip(first, second)])
    prompt = ftprompt.FtPrompt(heads, hk, d, dtype)
    rotation = torch.from_numpy(ftcache.rotation_table(128, d)).cuda()
    stream = torch.cuda.current_stream().cuda_stream
    held = [0, 0, 0]
    for new in (first, second):
        total, whole = sum(new), [a + b for a, b in zip(held, new)]
        qkv = s.normal(total, heads + 2 * hk, d)
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + hk], qkv[:, heads + hk:]
        q_rot, k_rot, o = torch.empty(total, heads, d, dtype=q.dtype, device="cuda"), torch.empty(total, hk, d, dtype=q.dtype, device="cuda"), torch.empty(total, heads, d, dtype=q.dtype, device="cuda")
        s.ctx.append(s.pool, q, k, v, rotation, bounds(new), ints(held), s.table_dev, q_rot, k_rot, stream)
        keys, values = k_rot, v
        if sum(held):
            keys, values = (torch.empty(sum(whole), hk, d, dtype=q.dtype, device="cuda") for _ in range(2))
            s.ctx.read(s.pool, keys, values, bounds(whole), ints([0, 0, 0]), s.table_dev, stream)
        prompt.forward(q_rot, keys, values, o, bounds(new), bounds(whole), stream)
        tp.check(o, q_rot, keys, values, new, whole, dtype)
        held = whole
    for _ in range(steps):
        q, k, v = s.normal(3, heads, d), s.normal(3, hk, d), s.normal(3, hk, d)
        o = torch.empty_like(q)
        s.ctx.append(s.pool, q, k, v, rotation, bounds([1, 1, 1]), ints(held), s.table_dev, q, None, stream)
        held = [n + 1 for n in held]
        s.ctx.attend(s.pool, q, o, ints(held), s.table_dev, stream)
        s.check_attend(o, q, held)
    assert s.ctx.report() == (0, 0)


@pytest.mark.gpu
def test_refusals_on_the_gpu():
    s = Setup(1, 4, 2, 64, 16, ftcache.F16, [10, 20])
    q, k, v = s.normal(5, 4, 64), s.normal(5, 2, 64), s.normal(5, 2, 64)
    rotation = torch.from_numpy(ftcache.rotation_table(64, 64)).cuda()
    good = dict(pool=s.pool, q=q, k=k, v=v, rotation=rotation, cu_seqlens=bounds([2, 3]), starts=ints([0, 0]), page_table=s.table_dev, q_out=q, k_out=k)
    for bad in [dict(pool=s.pool[1:]), dict(pool=s.pool.cpu()), dict(q=None), dict(k=k[:, :1]), dict(v=v.float()), dict(rotation=rotation[:, ::2]),
                dict(rotation=rotation.double()), dict(starts=ints([0])), dict(page_table=s.table_dev[:1]), dict(page_table=s.table_dev.long()),
                dict(page_table=s.table_dev.t().contiguous().t()), dict(cu_seqlens=bounds([2, 3])[:1]), dict(q_out=q[:1].expand(5, -1, -1))]:
        with pytest.raises((ValueError, TypeError)):
            s.ctx.append(**{**good, **bad})
    good = dict(pool=s.pool, q=q[:2], o=q[:2].clone(), lengths=ints([1, 2]), page_table=s.table_dev)
    for bad in [dict(q=q[:1]), dict(o=k[:2]), dict(lengths=ints([1])), dict(lengths=bounds([1]).long())]:
        with pytest.raises((ValueError, TypeError)):
            s.ctx.attend(**{**good, **bad})
    three = s.table_dev[:1].expand(3, -1)
    with pytest.raises((ftcache.FtCacheError, ValueError)):       # more sequences than the context was made for
        s.ctx.attend(s.pool, q[:3], q[:3].clone(), ints([1, 1, 1]), three.contiguous())


@pytest.mark.gpu
def test_sequences_that_begin_before_their_first_place():
    s = Setup(2, 2, 1, 64, 16, ftcache.F16, [16, 16])
    rotation = torch.from_numpy(ftcache.rotation_table(16, 64)).cuda()
    q, k, v = s.normal(10, 2, 64), s.normal(10, 1, 64), s.normal(10, 1, 64)
    q_out, k_out, seen = torch.empty_like(q), torch.empty_like(k), [torch.empty_like(k) for _ in range(2)]
    before = s.pool.clone()
    s.ctx.append(s.pool, q, k, v, rotation, bounds([5, 5]), ints([-2, -2 ** 31]), s.table_dev, q_out, k_out)
    assert torch.equal(s.pool, before) and torch.isnan(q_out).all() and torch.isnan(k_out).all() and s.ctx.report() == (10, 0)
    s.ctx.read(s.pool, *seen, bounds([5, 5]), ints([-1, 2 ** 31 - 3]), s.table_dev)
    # (the second sequence's places pass the last one)
    assert all(torch.isnan(x).all() for x in seen) and s.ctx.report()[0] == 10


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [ftcache.F16, ftcache.BF16])
def test_one_head_of_a_very_long_sequence(dtype):
    """One key head: hundreds of parts, put together in three levels."""
    lengths = [400001, 900]
    s = Setup(9, 2, 1, 64, 64, dtype, lengths)
    q, m = s.normal(2, 2, 64), s.model()
    o = torch.empty(2, 2, 64, dtype=TYPES[dtype], device="cuda")
    s.ctx.attend(s.pool, q, o, ints(lengths), s.table_dev)
    first = o.clone()
    for _ in range(3):
        s.ctx.attend(s.pool, q, o.zero_(), ints(lengths), s.table_dev)
        assert torch.equal(o, first)
    for b, n in enumerate(lengths):
        k, v = (x[:, 0].cuda() for x in m_sequence(s, m, b, n))
        w = torch.softmax(64 ** -0.5 * q[b].double() @ k.T, -1)
        assert ((first[b].double() - w @ v).abs() <= tolerance(dtype, dtype) * v.abs().max()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [64, 65, 700])
def test_many_sequences(batch):
    lengths = [(13 * i) % 41 for i in range(batch)]
    lengths[batch - 2] = 5000
    s = Setup(batch, 2, 1, 64, 16, ftcache.F16, lengths)
    q = s.normal(batch, 2, 64)
    o = torch.empty_like(q)
    s.ctx.attend(s.pool, q, o, ints(lengths), s.table_dev)
    m = s.model()
    for b in list(range(0, batch, 29)) + [batch - 2, batch - 1]:
        n = lengths[b]
        if n == 0:
            assert (o[b] == 0).all()
            continue
        k, v = (x[:, 0].cuda() for x in m_sequence(s, m, b, n))
        w = torch.softmax(64 ** -0.5 * q[b].double() @ k.T, -1)
        assert ((o[b].double() - w @ v).abs() <= tolerance(ftcache.F16, ftcache.F16) * v.abs().max()).all()
    s.ctx.attend(s.pool, q, q, ints(lengths), s.table_dev)          # the result in place of the queries
    assert torch.equal(q, o)


@pytest.mark.gpu
def test_rows_apart_and_shared():
    """Results and queries as views, a page table that is part of a wider one, and sequences that read the same pages."""
    lengths = [50, 50, 33]
    s = Setup(21, 4, 2, 128, 16, ftcache.BF16, lengths)
    wide = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + s.table.shape[1]] = s.table_dev
    wide[1] = wide[0]
    table = wide[:, 2:2 + s.table.shape[1]]
    x = s.normal(3, 12, 128)
    q, o = x[:, 0:4], torch.full((3, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    s.ctx.attend(s.pool, q, o[:, 2:6], ints(lengths), table)
    s.table[1] = s.table[0]
    s.check_attend(o[:, 2:6], q, lengths)
    assert (o[:, :2] == 7.0).all() and (o[:, 6:] == 7.0).all()
    k, v = torch.zeros(2, 3, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 256, dtype=torch.bfloat16, device="cuda")
    s.ctx.read(s.pool, k[:, :2], v[:, :, 128:], bounds([1, 1, 0]), ints([7, 7, 0]), table)
    assert torch.equal(k[0], k[1]) and (k[:, 2] == 0).all() and (v[:, :, :128] == 0).all() and (k[:, :2] != 0).any()


@pytest.mark.gpu
def test_tokens_far_apart():
    """Rows of tokens 40 MB apart: 12 GB between the first and the last."""
    stride, n = 20 * 2 ** 20 + 8, 300
    whole = torch.empty(n * stride, dtype=torch.float16, device="cuda")
    view = lambda at, heads: torch.as_strided(whole, (n, heads, 64), (stride, 128, 1), at)
    q, k, v, q_out, k_out = view(0, 4), view(4096, 2), view(8192, 2), view(12288, 4), view(16384, 2)
    s = Setup(17, 4, 2, 64, 16, ftcache.F16, [n])
    near = [s.normal(n, h, 64) for h in (4, 2, 2)]
    for x, y in zip((q, k, v), near):
        x.copy_(y)
    args = (torch.from_numpy(ftcache.rotation_table(n, 64)).cuda(), bounds([n]), ints([0]), s.table_dev)
    want = [torch.empty_like(near[0]), torch.empty_like(near[1])]
    s.ctx.append(s.pool, *near, *args, *want)
    pool = s.pool.clone()
    s.ctx.append(s.pool, q, k, v, *args, q_out, k_out)
    assert torch.equal(s.pool, pool) and torch.equal(q_out, want[0]) and torch.equal(k_out, want[1])
    seen = [torch.empty_like(near[1]) for _ in range(2)]
    s.ctx.read(s.pool, *seen, *args[1:])
    s.ctx.read(s.pool, k, v, *args[1:])
    assert torch.equal(k, seen[0]) and torch.equal(v, seen[1])


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (40, 2)])
def test_a_bad_page_anywhere_in_a_long_sequence_counts_once(heads, kv_heads):
    """At its beginning, inside, in its last block, in several places; the calls behind it are as ever."""
    lengths = [20000, 300, 7]
    s = Setup(15, heads, kv_heads, 64, 16, ftcache.BF16, lengths)
    q = s.normal(3, heads, 64)
    o, want = torch.empty_like(q), torch.empty_like(q)
    s.ctx.attend(s.pool, q, want, ints(lengths), s.table_dev)
    for bad in [[(0, 0)], [(0, 700)], [(0, 1249)], [(0, 3), (0, 900), (0, 901)], [(1, 18)], [(0, 1200), (1, 9), (2, 0)]]:
        table = s.table_dev.clone()
        for b, entry in bad:
            table[b, entry] = s.pages if entry % 2 else -3
        s.ctx.attend(s.pool, q, o, ints(lengths), table)
        hit = sorted({b for b, _ in bad})
        assert s.ctx.report() == (0, len(hit))
        for b in range(3):
            assert torch.isnan(o[b]).all() if b in hit else torch.equal(o[b], want[b])
        s.ctx.attend(s.pool, q, o, ints(lengths), s.table_dev)
        assert torch.equal(o, want) and s.ctx.report() == (0, 0)


@pytest.mark.gpu
def test_places_behind_the_last_one():
    """Sequences that pass 2^31 - 16 places: what lies behind them is refused like any place without a page, and counted."""
    s = Setup(16, 2, 1, 64, 16, ftcache.F16, [16, 16])
    rotation = torch.from_numpy(ftcache.rotation_table(16, 64)).cuda()
    q, k, v = s.normal(40, 2, 64), s.normal(40, 1, 64), s.normal(40, 1, 64)
    q_out, k_out, seen = torch.empty_like(q), torch.empty_like(k), [torch.empty_like(k) for _ in range(2)]
    before = s.pool.clone()
    for starts in [[2 ** 31 - 1, 2 ** 31 - 20], [2 ** 31 - 17, 2 ** 31 - 8]]:
        for x in (q_out, k_out, *seen):
            x.zero_()
        s.ctx.append(s.pool, q, k, v, rotation, bounds([17, 23]), ints(starts), s.table_dev, q_out, k_out)
        assert torch.equal(s.pool, before) and torch.isnan(q_out).all() and torch.isnan(k_out).all() and s.ctx.report() == (40, 0)
        s.ctx.read(s.pool, *seen, bounds([17, 23]), ints(starts), s.table_dev)
        assert all(torch.isnan(x).all() for x in seen) and s.ctx.report() == (40, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads,d,dtype", [(32, 8, 128, ftcache.BF16), (12, 2, 64, ftcache.F16)])
def test_attention_many_times(heads, kv_heads, d, dtype):
    """Sequences divided among workgroups, with the chip full: the same bits in every call and in every context."""
    lengths = [9000, 0, 333, 4100, 17000, 1, 2500, 6400]
    s = Setup(17, heads, kv_heads, d, 32, dtype, lengths)
    q = s.normal(8, heads, d)
    o = torch.empty(60, 8, heads, d, dtype=q.dtype, device="cuda")
    at, first = ints(lengths), None
    for _ in range(6):
        ctx = ftcache.FtCache(heads, kv_heads, d, s.pages, 32, dtype, max_batch=8)
        o.zero_()
        for i in range(60):
            ctx.attend(s.pool, q, o[i], at, s.table_dev, stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        ctx.close()
        first = o[0].clone() if first is None else first
        differ = (o != first).flatten(1).any(1)
        assert not differ.any(), differ.nonzero().flatten().tolist()
