"""The linear layer on 8-bit integers (ftint8_*) against its definition, spelled out here on the host.

Codes and scales are defined in 32 bits, operation by operation; the sum over k is exact, and a result is that sum rounded to 32 bits times the
product of the scales, rounded, rounded once more to the result's type.  So everything is compared bit by bit.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftint8

pytestmark = pytest.mark.gpu

TYPES = {ftint8.F16: torch.float16, ftint8.BF16: torch.bfloat16, ftint8.F32: torch.float32}


def coded(x):
    """(codes, scales) of the rows of x (host, 16 bits)."""
    y = x.float().numpy()
    most = np.abs(y).max(axis=1)
    up = np.where(most < np.float32(2.0 ** -100), np.float32(2.0 ** 100), np.float32(1.0))
    fine = np.isfinite(most)
    with np.errstate(all="ignore"):
        inverse = np.where((most == 0) | ~fine, np.float32(0), np.float32(127) * (np.float32(1) / (most * up)))
        codes = np.rint(np.where(fine[:, None], y, 0) * up[:, None] * inverse[:, None])
        scales = np.where(fine, most / np.float32(127), np.float32("nan"))
    return codes.astype(np.int8), scales.astype(np.float32)


def product(cx, sx, cw, sw, dtype):
    sums = (cx.astype(np.float64) @ cw.astype(np.float64).T).astype(np.int64)          # (exact: below 2^53)
    y = sums.astype(np.float32) * (sx[:, None] * sw)
    return torch.from_numpy(y.astype(np.float32)).to(TYPES[dtype])


def bits(t):
    return t.cpu().view(torch.int32 if t.dtype is torch.float32 else torch.int16)


def same(got, want):
    """Equal bit by bit, NaN for NaN."""
    got = got.cpu()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(bits(torch.where(got.isnan(), 0.0, got)), bits(torch.where(want.isnan(), 0.0, want)))


def padded(codes, k_padded):
    out = np.zeros((codes.shape[0], k_padded), np.int8)
    out[:, :codes.shape[1]] = codes
    return torch.from_numpy(out).cuda()


def stream():
    return torch.cuda.current_stream().cuda_stream


def inputs(m, n, k, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((m, k), generator=g) * torch.where(torch.rand(k, generator=g) < 0.05, 8.0, 1.0)).to(TYPES[dtype])
    cw, sw = coded((torch.randn((n, k), generator=g) * k ** -0.5).to(TYPES[dtype]))
    return x, cw, sw


@pytest.mark.parametrize("dtype", [ftint8.F16, ftint8.BF16])
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 7), (5, 64), (2, 127), (70, 128), (9, 129), (33, 1000), (4, 8192), (2, 20011)])
def test_codes_and_scales(rows, k, dtype):
    x, _, _ = inputs(rows, 1, k, dtype, rows * 31 + k)
    ctx = ftint8.FtInt8(5, k, dtype)
    codes = torch.full((rows, ctx.k_padded), 77, dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, device="cuda")
    ctx.encode(x.cuda(), codes, scales, stream())
    want, want_scales = coded(x)
    assert ctx.k_padded % 128 == 0 and 0 <= ctx.k_padded - k < 128
    assert torch.equal(codes.cpu(), padded(want, ctx.k_padded).cpu())
    same(scales, torch.from_numpy(want_scales))


@pytest.mark.parametrize("dtype", [ftint8.F16, ftint8.BF16])
def test_rows_of_zeros_of_small_and_of_unbounded_numbers(dtype):
    k = 200
    x = torch.randn((9, k), generator=torch.Generator().manual_seed(5)).to(TYPES[dtype])
    x[0] = 0
    x[1] = x[1] * 0 - 0.0
    x[2, 17] = float("inf")
    x[3, 199] = float("-inf")
    x[4, 0] = float("nan")
    x[5] = torch.from_numpy(np.resize(np.array([1, 0x8001, 3, 0, 7], np.uint16), k).view(np.int16).copy()).view(TYPES[dtype])      # the smallest numbers
    x[6] = torch.finfo(TYPES[dtype]).max * torch.where(torch.arange(k) % 3 == 0, -1, 1).to(TYPES[dtype])
    x[7] = 0
    x[7, 63] = -1
    ctx = ftint8.FtInt8(40, k, dtype, ftint8.F32, max_tokens=9)
    codes, scales = torch.empty((9, ctx.k_padded), dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    ctx.encode(x.cuda(), codes, scales, stream())
    want, want_scales = coded(x)
    assert torch.equal(codes.cpu(), padded(want, ctx.k_padded).cpu())
    same(scales, torch.from_numpy(want_scales))
    cw, sw = coded(torch.randn((40, k), generator=torch.Generator().manual_seed(6)).to(TYPES[dtype]))
    y = torch.empty((9, 40), device="cuda")
    ctx.forward(x.cuda(), padded(cw, ctx.k_padded), torch.from_numpy(sw).cuda(), y, stream())
    same(y, product(want, want_scales, cw, sw, ftint8.F32))
    # (in bf16 the row of the largest numbers has sums beyond the largest number of 32 bits)
    assert y[2:5].isnan().all() and not y[5:].isnan().any() and (y[:2] == 0).all()


SHAPES = [(1, 1, 1), (1, 16, 64), (1, 515, 4096), (1, 2000, 9000), (2, 33, 65), (5, 4096, 512), (2, 4096, 4096), (3, 20, 4095), (4, 300, 200), (15, 100, 300), (16, 256, 128), (17, 257, 129), (31, 1000, 1000), (33, 48, 4096),
          (64, 64, 64), (65, 700, 260), (96, 512, 2048), (127, 129, 127), (128, 128, 256), (130, 96, 384), (200, 3, 77), (255, 300, 1024), (256, 256, 256), (300, 520, 900), (513, 257, 640),
          (700, 1030, 200), (1000, 96, 96), (1100, 2100, 512), (20, 70, 5001), (50, 200, 5001), (1, 33, 16385), (130, 500, 10000)]


@pytest.mark.parametrize("dtype,out", [(ftint8.F16, ftint8.F16), (ftint8.BF16, ftint8.BF16), (ftint8.F16, ftint8.F32), (ftint8.BF16, ftint8.F32)])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_layer(m, n, k, dtype, out):
    x, cw, sw = inputs(m, n, k, dtype, m + 7 * n + 13 * k)
    ctx = ftint8.FtInt8(n, k, dtype, out, max_tokens=m)
    y = torch.empty((m, n), dtype=TYPES[out], device="cuda")
    w, scales = padded(cw, ctx.k_padded), torch.from_numpy(sw).cuda()
    ctx.forward(x.cuda(), w, scales, y, stream())
    cx, sx = coded(x)
    want = product(cx, sx, cw, sw, out)
    same(y, want)
    y.fill_(7)
    ctx.product(padded(cx, ctx.k_padded), torch.from_numpy(sx).cuda(), w, scales, y, stream())
    same(y, want)


@pytest.mark.parametrize("m", [1, 3, 40, 300])
def test_longest_sums_of_the_largest_codes(m):
    """k = 130944 products of -128 and -128, and of 127 and -128: sums up to 2145386496."""
    k, n = 130944, 18
    ctx = ftint8.FtInt8(n, k, ftint8.BF16, ftint8.F32, max_tokens=1)
    cx, cw = np.full((m, k), -128, np.int8), np.full((n, k), -128, np.int8)
    cx[0] = 127
    cw[3] = 127
    cw[5, ::2] = 127
    sx, sw = np.linspace(0.5, 2, m, dtype=np.float32), np.linspace(1e-3, 1, n, dtype=np.float32)
    y = torch.empty((m, n), device="cuda")
    ctx.product(padded(cx, k), torch.from_numpy(sx).cuda(), padded(cw, k), torch.from_numpy(sw).cuda(), y, stream())
    same(y, product(cx, sx, cw, sw, ftint8.F32))


@pytest.mark.parametrize("m,n,k,x_pad,y_pad,offset", [(5, 33, 100, 3, 5, 1), (70, 130, 129, 7, 0, 0), (3, 64, 64, 8, 8, 8), (300, 257, 64, 0, 9, 3), (130, 256, 256, 8, 8, 0), (1, 100, 90, 0, 0, 5), (1, 100, 90, 0, 3, 8), (1, 50, 5000, 8, 1, 0),
                                                          (20, 100, 300, 8, 1, 0), (3, 100, 300, 4, 1, 0), (4, 4000, 4096, 8, 0, 0), (40, 130, 2100, 4, 3, 1)])
def test_views_of_larger_tensors(m, n, k, x_pad, y_pad, offset):
    """Rows apart and beginning anywhere; what lies between the rows of the result stays as it was."""
    x, cw, sw = inputs(m, n, k, ftint8.BF16, 3)
    ctx = ftint8.FtInt8(n, k, ftint8.BF16, max_tokens=m)
    xs = torch.full((m * (k + x_pad) + offset,), float("nan"), dtype=torch.bfloat16, device="cuda")
    xv = xs[offset:].view(m, k + x_pad)[:, :k]
    xv.copy_(x)
    ys = torch.full((m * (n + y_pad) + offset,), 5.0, dtype=torch.bfloat16, device="cuda")
    yv = ys[offset:].view(m, n + y_pad)[:, :n]
    ctx.forward(xv, padded(cw, ctx.k_padded), torch.from_numpy(sw).cuda(), yv, stream())
    cx, sx = coded(x)
    same(yv, product(cx, sx, cw, sw, ftint8.BF16))
    assert (ys[:offset] == 5).all() and (ys[offset:].view(m, n + y_pad)[:, n:] == 5).all()


def test_no_tokens():
    ctx = ftint8.FtInt8(8, 16, ftint8.F16, max_tokens=4)
    w, scales = torch.zeros((8, ctx.k_padded), dtype=torch.int8, device="cuda"), torch.zeros(8, device="cuda")
    ctx.forward(torch.empty((0, 16), dtype=torch.float16, device="cuda"), w, scales, torch.empty((0, 8), dtype=torch.float16, device="cuda"), stream())
    torch.cuda.synchronize()


@pytest.mark.parametrize("m,n,k", [(1, 600, 512), (40, 300, 700), (40, 300, 2100), (300, 260, 384)])
def test_on_another_stream_and_in_a_graph(m, n, k):
    sizes = inputs(m, n, k, ftint8.F16, 1)
    ctx = ftint8.FtInt8(n, k, ftint8.F16, max_tokens=m)
    x, w, scales = sizes[0].cuda(), padded(sizes[1], ctx.k_padded), torch.from_numpy(sizes[2]).cuda()
    y = torch.zeros((m, n), dtype=torch.float16, device="cuda")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    ctx.forward(x, w, scales, y, other.cuda_stream)
    other.synchronize()
    cx, sx = coded(sizes[0])
    same(y, product(cx, sx, sizes[1], sizes[2], ftint8.F16))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.forward(x, w, scales, y, stream())
    for seed in range(3):
        new, _, _ = inputs(m, n, k, ftint8.F16, seed + 10)
        x.copy_(new)
        y.fill_(3)
        graph.replay()
        cx, sx = coded(new)
        want = product(cx, sx, sizes[1], sizes[2], ftint8.F16)
        same(y, want)
        y.fill_(3)
        ctx.forward(x, w, scales, y, stream())
        same(y, want)
