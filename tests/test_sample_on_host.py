"""The choice of the next token (ftsample_choose), its kernels compiled for the host and run there, against its definition in 64 bits.

Rows on which the kernels' rarer paths depend: with few logits that can be chosen, with logits so far below the largest that they have no weight, with a top_k near to how
many there are.  LDS is filled with several patterns before each workgroup, and the waves run in several orders, so that a result may depend on neither.
"""
import os
import subprocess
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftsample
from test_gpu_sample import one

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2504_02211_amd")
CLANG = os.environ.get("ROCM_CLANG", "/opt/rocm/llvm/bin/clang++")
TYPES = {ftsample.F16: torch.float16, ftsample.BF16: torch.bfloat16, ftsample.F32: torch.float32}


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    path = tmp_path_factory.mktemp("host") / "libsample.so"
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-mf16c", "-shared", "-fPIC", "-w", "-I", os.path.join(ROOT, "tests", "workgroup_on_host"),
                    "-I", os.path.join(PKG, "include"), "-I", os.path.join(PKG, "csrc"), os.path.join(PKG, "csrc", "ftsample.hip"), "-o", str(path)], check=True)
    return str(path)


RUN = r"""
import ctypes as C, sys
import numpy as np
from paper_2504_02211_amd import ftsample
path, folder, dtype, rows, vocab = sys.argv[1], sys.argv[2], *[int(x) for x in sys.argv[3:6]]
lib, p = C.CDLL(path), lambda x: x.ctypes.data_as(C.c_void_p)
have = dict(np.load(folder + "/in.npz"))
cfg, handle = ftsample.Config(C.sizeof(ftsample.Config), vocab, rows, dtype, 0), C.c_void_p()
assert lib.ftsample_create(C.byref(cfg), C.byref(handle)) == 0
size = 4 if dtype == ftsample.F32 else 2
room = np.zeros(have["logits"].nbytes + 32, np.uint8)
at = -room.ctypes.data % 16 + int(have["skip"]) * size
room[at:at + have["logits"].nbytes] = have["logits"].view(np.uint8).ravel()
rules = (C.c_void_p * 4)(*[have[n].ctypes.data if n in have else None for n in ("temperature", "top_k", "top_p", "min_p")])
results = []
for order, filling in ((0, 0), (1, 255), (2, 0x3F)):
    tokens, chance = np.full(rows, -77, np.int32), np.full(rows, -77, np.float32)
    lib.host_order(order, filling)
    rc = lib.ftsample_choose(handle, C.c_void_p(room.ctypes.data + at), C.c_int64(vocab), rows, p(have["uniform"]), rules, p(tokens), p(chance), None)
    assert rc == 0
    results += [tokens, chance]
np.savez(folder + "/out.npz", *results)
"""


def check(library, folder, logits, dtype, uniform, skip=0, **rules):
    """logits: float32 [rows, vocab]; rules: lists of a number a row.  Every order and filling gives what the definition says."""
    x = torch.from_numpy(logits).to(TYPES[dtype])
    rows, vocab = x.shape
    have = {"temperature": np.float32, "top_k": np.int32, "top_p": np.float32, "min_p": np.float32}
    have = {n: np.asarray(v, have[n]) for n, v in rules.items()}
    np.savez(str(folder / "in.npz"), logits=x.view(torch.int32 if dtype == ftsample.F32 else torch.int16).numpy(), uniform=np.asarray(uniform, np.float32), skip=skip, **have)
    # (in a process of its own: a workgroup that never ends is a failure of one test)
    run = subprocess.run([sys.executable, "-c", RUN, library, str(folder), str(dtype), str(rows), str(vocab)], env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    with np.load(str(folder / "out.npz")) as f:
        results = [f[n] for n in f.files]
    at = lambda name, r, otherwise: have[name][r] if name in have else otherwise  # noqa: E731
    for r in range(rows):
        want, chance = one(x[r].double().numpy(), float(np.float32(uniform[r])), float(at("temperature", r, 1.0)), int(at("top_k", r, 0)), float(at("top_p", r, 1.0)),
                           float(at("min_p", r, 0.0)))
        for tokens, got in zip(results[::2], results[1::2]):
            # (probabilities: a rounding to 32 bits, 2^-24, and sums in whole multiples of 2^-42 or finer)
            assert tokens[r] == want and abs(float(got[r]) - chance) <= 2.0 ** -24 * chance + 2.0 ** -26, (r, int(tokens[r]), want, float(got[r]), chance)


ALL = [ftsample.F16, ftsample.BF16, ftsample.F32]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("vocab,skip", [(1, 0), (9, 1), (1000, 0), (6000, 3)])
def test_rows_like_any_other(library, tmp_path, dtype, vocab, skip):
    g = np.random.default_rng(vocab)
    rows = 6
    x = (g.standard_normal((rows, vocab)) * 3).astype(np.float32)
    check(library, tmp_path, x, dtype, g.random(rows), skip)
    check(library, tmp_path, x, dtype, g.random(rows), skip, temperature=[0.0, 0.3, 1.0, 2.0, 0.7, 1.3], top_k=[3, 0, 50, 300, 700, 1], top_p=[1.0, 0.9, 0.5, 0.99, 0.8, 0.3],
          min_p=[0, 0.1, 0, 0.01, 0, 0])


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("rule", ["top_k", "top_p", "min_p", "all"])
def test_fewer_logits_than_top_k_and_some_far_below(library, tmp_path, dtype, rule):
    """95 of 100 tokens masked, 512 or fewer left, most of them with no weight at a low temperature; and far more of them than fit a list."""
    g = np.random.default_rng(7)
    vocab, ks = 6000, [257, 290, 600, 1024, 5000, 5999]
    x = (g.standard_normal((len(ks), vocab)) * 4).astype(np.float32)
    x[g.random(x.shape) < 0.95] = -np.inf
    x[4] = g.standard_normal(vocab) * 40
    x[4, g.random(vocab) < 0.5] = -np.inf
    rules = {"top_k": ks, "temperature": [0.3] * len(ks)}
    if rule in ("top_p", "all"):
        rules["top_p"] = [0.9, 0.99, 0.5, 0.999, 0.95, 0.7]
    if rule in ("min_p", "all"):
        rules["min_p"] = [0.01, 0.0, 0.2, 1e-6, 0.0, 1e-3]
    check(library, tmp_path, x, dtype, g.random(len(ks)), **rules)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("far", [60.0, 3e4])
def test_top_k_at_the_number_of_logits_that_can_be_chosen(library, tmp_path, dtype, far):
    """As many as top_k, one fewer, one more; near the largest, or all but the largest more than 51 octaves below it."""
    g = np.random.default_rng(8)
    vocab, k = 3000, 400
    counts = [k, k - 1, k + 1, k, k - 1, k + 1, 1, 2]
    x = np.full((len(counts), vocab), -np.inf, np.float32)
    for r, n in enumerate(counts):
        at = g.permutation(vocab)[:n]
        x[r, at] = g.standard_normal(n) * (2 if r < 3 else 1) - (0 if r < 3 else far)
        x[r, at[n // 2]] = 6
    for top_p in (None, 0.9):
        rules = {} if top_p is None else {"top_p": [top_p] * len(counts)}
        check(library, tmp_path, x, dtype, g.random(len(counts)), top_k=[k] * len(counts), **rules)


@pytest.mark.parametrize("dtype", ALL)
def test_borders_just_below_zero(library, tmp_path, dtype):
    """Zeros of both signs and the smallest negative numbers beside larger ones: the border lies among the latter, whose keys end where those of zeros begin."""
    g = np.random.default_rng(9)
    vocab, zeros, small = 2000, 500, 700
    unit = {ftsample.F16: 2.0 ** -24, ftsample.BF16: 2.0 ** -133, ftsample.F32: 2.0 ** -149}[dtype]
    tops = [1.0, 0.8, 0.93, 1.1, 1.3, 2.0, 0.51, 0.7, 0.61, 1.7]
    rows = len(tops)
    x = np.full((rows, vocab), -np.inf)
    for r in range(rows):
        at = g.permutation(vocab)
        x[r, at[:zeros]] = np.where(g.random(zeros) < 0.5, 0.0, -0.0)
        x[r, at[zeros:zeros + small]] = -unit * g.integers(1, 8, small)
        x[r, at[zeros + small:zeros + small + 100]] = -0.5 * g.random(100) - 0.1
        x[r, at[-1]] = tops[r]
    with np.errstate(under="ignore"):
        x = x.astype(np.float32)
    ks = [zeros + 1 + n for n in (1, 300, 500, 699, 650, 2, 400, 600, 100, 50)]
    check(library, tmp_path, x, dtype, g.random(rows), top_k=ks)
    check(library, tmp_path, x, dtype, g.random(rows), top_k=ks, top_p=[0.95] * rows)
    check(library, tmp_path, x, dtype, g.random(rows), top_p=list(0.5 + 0.4 * g.random(rows)))
