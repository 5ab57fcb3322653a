"""Prompt and cache operators without a GPU: the C ABI's own checks, the layout of its structures, the rotation table."""
import ctypes as C
import os
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftcache, ftprompt
from test_kernel_registers import built_kernels
from paper_2504_02211_amd.ftattn import LIB_PATH

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROMPT = dict(heads=8, kv_heads=2, head_dim=64, in_dtype=0, out_dtype=0, softmax_scale=0.0, device=0)
CACHE = dict(heads=8, kv_heads=2, head_dim=64, pages=4, page_size=16, in_dtype=1, out_dtype=1, rotary_dim=0, interleaved=0, softmax_scale=0.0,
             max_batch=4, device=0)


def create(module, name, fields):
    lib = module.load_library()
    cfg = module.Config(struct_size=C.sizeof(module.Config), **fields)
    handle = C.c_void_p()
    rc = getattr(lib, name + "_create")(C.byref(cfg), C.byref(handle))
    assert rc != 0 and not handle
    return rc, getattr(lib, name + "_last_error")(None).decode()


@pytest.mark.parametrize("bad,code,word", [
    (dict(heads=0), -1, "kv_heads"), (dict(kv_heads=3), -1, "multiple"), (dict(kv_heads=0), -1, "kv_heads"), (dict(heads=2 ** 20, kv_heads=1), -2, "65536"),
    (dict(head_dim=96), -2, "head_dim"), (dict(in_dtype=2), -1, "in_dtype"), (dict(out_dtype=1), -1, "out_dtype"), (dict(softmax_scale=float("nan")), -1, "softmax"),
    (dict(softmax_scale=float("inf")), -1, "softmax")])
def test_prompt_configurations_that_are_refused(bad, code, word):
    rc, message = create(ftprompt, "ftprompt", {**PROMPT, **bad})
    assert rc == code and word in message


@pytest.mark.parametrize("bad,code,word", [
    (dict(heads=7), -1, "multiple"), (dict(heads=8192, kv_heads=1), -2, "4096"), (dict(head_dim=32), -2, "head_dim"), (dict(pages=0), -1, "pages"),
    (dict(page_size=8), -2, "page_size"), (dict(page_size=48), -2, "page_size"), (dict(page_size=2048), -2, "page_size"), (dict(in_dtype=2), -1, "in_dtype"),
    (dict(out_dtype=0), -1, "out_dtype"), (dict(rotary_dim=24), -2, "rotary"), (dict(rotary_dim=80), -2, "rotary"), (dict(rotary_dim=-16), -2, "rotary"),
    (dict(interleaved=2), -1, "interleaved"), (dict(max_batch=0), -1, "max_batch"), (dict(max_batch=65537), -1, "max_batch"),
    (dict(softmax_scale=float("-inf")), -1, "softmax")])
def test_cache_configurations_that_are_refused(bad, code, word):
    rc, message = create(ftcache, "ftcache", {**CACHE, **bad})
    assert rc == code and word in message


def test_structures_of_another_size_and_null():
    for module, name, fields in ((ftprompt, "ftprompt", PROMPT), (ftcache, "ftcache", CACHE)):
        lib = module.load_library()
        cfg, handle = module.Config(struct_size=4, **fields), C.c_void_p()
        assert getattr(lib, name + "_create")(C.byref(cfg), C.byref(handle)) == -1
        assert getattr(lib, name + "_create")(None, C.byref(handle)) == -1
        assert getattr(lib, name + "_get_config")(None, None) == -1
        assert getattr(lib, name + "_destroy")(None) == 0
    lib = ftcache.load_library()
    assert lib.ftcache_page_bytes(None) == -1
    assert lib.ftcache_attend(None, None, 1, None, None, 1, 1, None, None, None) == -1
    assert lib.ftcache_append(None, None, None, None, 1, None, None, None, None, None, None) == -1
    assert lib.ftcache_read(None, None, None, None, None, None) == -1 and lib.ftcache_report(None, None) == -1
    assert ftprompt.load_library().ftprompt_forward(None, None, None, None, None, None, None, 1, 1, 1, None) == -1


def test_a_sound_configuration_without_a_gpu_is_an_error_of_the_device():
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    assert create(ftprompt, "ftprompt", PROMPT)[0] == -3
    assert create(ftcache, "ftcache", CACHE)[0] in (-3, -4)
    with pytest.raises(ftprompt.FtPromptError):
        ftprompt.FtPrompt(8, 2, 64, ftprompt.F16)
    with pytest.raises(ftcache.FtCacheError):
        ftcache.FtCache(8, 2, 64, 4, 16, ftcache.F16)


@pytest.mark.parametrize("header,module", [("ftprompt.h", ftprompt), ("ftcache.h", ftcache)])
def test_bindings_name_what_the_headers_declare(header, module):
    with open(os.path.join(ROOT, "paper_2504_02211_amd", "include", header)) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    name = header[:-2]
    declared = set(re.findall(r"\b(%s_\w+)\(" % name, text))
    assert declared == set(module.EXPORTS)
    lib = module.load_library()
    assert all(hasattr(lib, n) for n in declared)
    body = re.search(r"typedef struct \{([^}]*)\} %s_config;" % name, text).group(1)
    fields = [n.strip() for line in re.findall(r"(?:u?int32_t|float)\s+([^;]+);", body) for n in line.split(",")]
    assert fields == [n for n, _ in module.Config._fields_]
    assert ftcache._PLACES.size == 48 and ftprompt._ROWS.size == 24


def test_tensors_that_the_bindings_refuse():
    ftcache.load_library()
    x = torch.zeros(4, 8, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="not on a GPU"):
        ftprompt.rows(x, "x", 4, 8, 64, ftprompt.F16, 0)
    with pytest.raises(ValueError, match="expected"):
        ftprompt.rows(x, "x", 5, 8, 64, ftprompt.F16, 0)
    with pytest.raises(ValueError, match="float16"):
        ftprompt.rows(x, "x", 4, 8, 64, ftprompt.BF16, 0)
    with pytest.raises(TypeError):
        ftprompt.rows([1], "x", 4, 8, 64, ftprompt.F16, 0)
    with pytest.raises(ValueError, match="int32"):
        ftprompt.ints(torch.zeros(3), "x", 3, 0)
    with pytest.raises(ValueError, match="not on a GPU"):
        ftprompt.ints(torch.zeros(3, dtype=torch.int32), "x", 3, 0)


def test_rotation_table():
    """Angles in 64 bits: a far position's cosine is the exact one, rounded."""
    t = ftcache.rotation_table(70001, 64, 10000.0)
    assert t.dtype == np.float32 and t.shape == (70001, 64)
    for p in (0, 1, 4095, 70000):
        for i in (0, 1, 17, 31):
            angle = p * 10000.0 ** (-2 * i / 64)
            # the angle's own rounding, 2^-53 of at most 70000, and the result's to 32 bits
            assert abs(t[p, i] - np.cos(angle)) <= 2.0 ** -24 and abs(t[p, 32 + i] - np.sin(angle)) <= 2.0 ** -24
    assert (t[0, :32] == 1).all() and (t[0, 32:] == 0).all()


def test_kernels_spill_no_vector_registers():
    mine = {n: k for n, k in built_kernels(LIB_PATH).items() if "ftprompt_main" in n or "ftcache_" in n}
    assert len(mine) == 8 + 8 + 4 + 8
    assert {n for n, k in mine.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]} == set()


@pytest.mark.parametrize("scale", [2.4e38, 2.9e38])
def test_softmax_scales_beyond_what_the_kernels_hold(scale):
    """The kernels multiply by log2(e) first: a scale above 3.4e38 / log2(e) would be infinite there, and a score of 0 NaN."""
    for module, name, fields in ((ftprompt, "ftprompt", PROMPT), (ftcache, "ftcache", CACHE)):
        rc, message = create(module, name, {**fields, "softmax_scale": scale})
        assert rc == -1 and "softmax" in message
