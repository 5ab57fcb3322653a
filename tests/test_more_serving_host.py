"""The linear layer on 8-bit integers, linear attention with a decay and the choice of the next token without a GPU: the C ABI's own checks, the
layout of its structures, what the bindings refuse."""
import ctypes as C
import os
import re

import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftdecay, ftint8, ftprompt, ftsample
from paper_2504_02211_amd.ftattn import LIB_PATH
from test_kernel_registers import built_kernels
from test_serving_host import create

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

INT8 = dict(n=64, k=128, in_dtype=0, out_dtype=0, max_tokens=4, device=0)
DECAY = dict(heads=8, kv_heads=2, head_dim=64, in_dtype=0, scale=0.0, device=0)
SAMPLE = dict(vocab=1000, max_rows=4, in_dtype=2, device=0)


@pytest.mark.parametrize("bad,code,word", [
    (dict(n=0), -1, "n and k"), (dict(k=0), -1, "n and k"), (dict(k=130945), -2, "130944"), (dict(n=2 ** 24 + 1), -2, "2^24"), (dict(in_dtype=2), -1, "in_dtype"),
    (dict(out_dtype=1), -1, "out_dtype"), (dict(max_tokens=0), -1, "max_tokens"), (dict(max_tokens=2 ** 22 + 1), -1, "max_tokens")])
def test_int8_configurations_that_are_refused(bad, code, word):
    rc, message = create(ftint8, "ftint8", {**INT8, **bad})
    assert rc == code and word in message


@pytest.mark.parametrize("bad,code,word", [
    (dict(heads=0), -1, "kv_heads"), (dict(kv_heads=3), -1, "multiple"), (dict(kv_heads=0), -1, "kv_heads"), (dict(heads=2 ** 20, kv_heads=1), -2, "65536"),
    (dict(head_dim=96), -2, "head_dim"), (dict(in_dtype=2), -1, "in_dtype"), (dict(scale=float("nan")), -1, "scale"), (dict(scale=float("-inf")), -1, "scale")])
def test_decay_configurations_that_are_refused(bad, code, word):
    rc, message = create(ftdecay, "ftdecay", {**DECAY, **bad})
    assert rc == code and word in message


@pytest.mark.parametrize("bad,code,word", [
    (dict(vocab=0), -1, "vocab"), (dict(vocab=2 ** 20 + 1), -2, "vocab"), (dict(max_rows=0), -1, "max_rows"), (dict(max_rows=65537), -1, "max_rows"), (dict(in_dtype=3), -1, "in_dtype"),
    (dict(in_dtype=-1), -1, "in_dtype")])
def test_sample_configurations_that_are_refused(bad, code, word):
    rc, message = create(ftsample, "ftsample", {**SAMPLE, **bad})
    assert rc == code and word in message


def test_structures_of_another_size_and_null():
    for module, name, fields in ((ftint8, "ftint8", INT8), (ftdecay, "ftdecay", DECAY), (ftsample, "ftsample", SAMPLE)):
        lib = module.load_library()
        cfg, handle = module.Config(struct_size=4, **fields), C.c_void_p()
        assert getattr(lib, name + "_create")(C.byref(cfg), C.byref(handle)) == -1
        assert getattr(lib, name + "_create")(None, C.byref(handle)) == -1
        assert getattr(lib, name + "_get_config")(None, None) == -1
        assert getattr(lib, name + "_destroy")(None) == 0
    lib = ftint8.load_library()
    assert lib.ftint8_k_padded(None) == -1 and lib.ftint8_encode(None, None, 1, None, None, None) == -1
    assert lib.ftint8_product(None, None, None, 1, None, None, None, None) == -1 and lib.ftint8_forward(None, None, 1, None, None, None, None) == -1
    lib = ftdecay.load_library()
    assert lib.ftdecay_forward(*[None] * 7, 0, None, None, None, 1, 1, None) == -1 and lib.ftdecay_step(*[None] * 7, 0, None, 1, None) == -1
    assert ftsample.load_library().ftsample_choose(None, None, 0, 1, None, None, None, None, None) == -1


def test_a_sound_configuration_without_a_gpu_is_an_error_of_the_device():
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    for module, name, fields in ((ftint8, "ftint8", INT8), (ftdecay, "ftdecay", DECAY), (ftsample, "ftsample", SAMPLE)):
        assert create(module, name, fields)[0] == -3
    with pytest.raises(ftint8.FtInt8Error):
        ftint8.FtInt8(8, 8, ftint8.F16)
    with pytest.raises(ftdecay.FtDecayError):
        ftdecay.FtDecay(8, 2, 64, ftdecay.F16)
    with pytest.raises(ftsample.FtSampleError):
        ftsample.FtSample(100, ftsample.F32)


@pytest.mark.parametrize("header,module", [("ftint8.h", ftint8), ("ftdecay.h", ftdecay), ("ftsample.h", ftsample)])
def test_bindings_name_what_the_headers_declare(header, module):
    with open(os.path.join(ROOT, "paper_2504_02211_amd", "include", header)) as f:
        text = f.read()
    name = header[:-2]
    declared = set(re.findall(r"\b(%s_\w+)\(" % name, re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert declared == set(module.EXPORTS)
    lib = module.load_library()
    assert all(hasattr(lib, n) for n in declared)
    config = re.search(r"typedef struct \{([^{}]*?)\} %s_config;" % name, re.sub(r"/\*.*?\*/", "", text, flags=re.S), re.S).group(1)
    assert [x for line in re.findall(r"\w+\s+([\w, ]+);", config) for x in re.split(r",\s*", line)] == [n for n, _ in module.Config._fields_]


def test_tensors_that_the_bindings_refuse():
    ftint8.load_library(), ftdecay.load_library(), ftsample.load_library()
    x = torch.zeros((4, 64), dtype=torch.float16)
    with pytest.raises(TypeError):
        ftint8.matrix(5, "x", 64, 0, 0)
    for bad in (x[:, :63], x[0], x.bfloat16(), x):          # (the last one: not on a GPU)
        with pytest.raises(ValueError):
            ftint8.matrix(bad, "x", 64, 0, 0)
    for bad in (torch.zeros(5), torch.zeros(4, dtype=torch.int32), torch.zeros(4)):
        with pytest.raises(ValueError):
            ftprompt.array(bad, "scales", 4, torch.float32, 0)
    with pytest.raises(TypeError):
        ftprompt.array([1.0] * 4, "scales", 4, torch.float32, 0)


def test_kernels_spill_no_vector_registers():
    kernels = {n: k for n, k in built_kernels(LIB_PATH).items() if any(name in n for name in ("ftint8_", "ftdecay_", "ftsample_"))}
    assert len(kernels) >= 10
    assert {n for n, k in kernels.items() if k[".vgpr_spill_count"]} == set()
