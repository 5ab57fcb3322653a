"""Sizes at which calls of ftint8, ftdecay and ftsample need more workgroups than a launch has: refused on the host, before the first launch; and what the largest launch.

A launch has fewer than 2^32 threads in a dimension.  The library runs in a process of its own whose HIP runtime is a stand-in that keeps no device and only
notes launches, so both sides of each limit can be called without a GPU."""
import os
import subprocess
import sys

import pytest

pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_IN = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
extern "C" {
struct dim { uint32_t x, y, z; };
static dim grid, block;
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipSetDevice(int) { return 0; }
int hipMalloc(void** p, size_t n) { std::printf("memory %zu\n", n); *p = std::aligned_alloc(256, 4096); return 0; }
int hipFree(void* p) { std::free(p); return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetLastError() { return 0; }
int __hipPushCallConfiguration(dim g, dim b, size_t, void*) { grid = g; block = b; return 0; }
int __hipPopCallConfiguration(dim* g, dim* b, size_t* shared, void** stream) { *g = grid; *b = block; *shared = 0; *stream = nullptr; return 0; }
int hipLaunchKernel(const void*, dim g, dim b, void**, size_t, void*) { std::printf("launch %u %u %u\n", g.x, g.y, b.x); std::fflush(stdout); return 0; }
}
"""

CALLS = r"""
import ctypes as C, sys
from paper_2504_02211_amd import ftdecay, ftint8, ftprompt, ftsample
row, P = ftprompt._ROWS.pack(0x1000, 1024, 64), 0x1000

def create(module, name, **fields):
    cfg, handle = module.Config(struct_size=C.sizeof(module.Config), in_dtype=0, device=0, **fields), C.c_void_p()
    assert getattr(module.load_library(), name + "_create")(C.byref(cfg), C.byref(handle)) == 0
    return module.load_library(), handle

def int8(n, k):
    lib, h = create(ftint8, "ftint8", n=n, k=k, out_dtype=0, max_tokens=1 << 22)
    x, y = ftint8._MATRIX.pack(P, max(k, 8)), ftint8._MATRIX.pack(P, n)
    return dict(encode=lambda m: lib.ftint8_encode(h, x, m, P, P, None), product=lambda m: lib.ftint8_product(h, P, P, m, P, P, y, None),
                forward=lambda m: lib.ftint8_forward(h, x, m, P, P, y, None))

def decay(dim):
    lib, h = create(ftdecay, "ftdecay", heads=4, kv_heads=2, head_dim=dim, scale=0.0)
    return dict(prompt=lambda total, batch: lib.ftdecay_forward(h, row, row, row, row, P, None, 0, None, P, None, batch, total, None),
                step=lambda batch: lib.ftdecay_step(h, row, row, row, row, P, P, 1 << 30, None, batch, None))

lib, h = create(ftsample, "ftsample", vocab=9, max_rows=65536)
sample = dict(choose=lambda rows: lib.ftsample_choose(h, P, 16, rows, P, None, P, None, None))
made = {}
for call in sys.argv[1:]:
    module, sizes, name, *numbers = call.split(",")
    if (module, sizes) not in made:
        made[module, sizes] = sample if module == "sample" else {"int8": int8, "decay": decay}[module](*[int(x) for x in sizes.split("x")])
    print(call, "gives", made[module, sizes][name](*[int(x) for x in numbers]), flush=True)
"""

# tiles of 256 x 256, 512 threads each; a workgroup of 256 threads a row of more than 2048 elements, four rows of fewer; four heads a sequence
FITS = ["int8,16777216x8,product,32512", "int8,16777216x8,forward,32512", "int8,16777216x8,forward,1", "int8,16777216x8,product,32", "int8,8x4000,encode,16777215", "int8,8x8,encode,16777215",
        "int8,2000x130944,product,4194304", "decay,128,prompt,0,4190000", "decay,128,prompt,257,262143", "decay,64,prompt,2147483647,1000", "decay,128,step,4194303",
        "sample,9,choose,65536"]
DOES_NOT = ["int8,16777216x8,product,32513", "int8,16777216x8,forward,32513", "int8,16777216x8,product,4194304", "int8,8x4000,encode,16777216", "int8,8x8,product,4194305",
            "decay,128,prompt,0,4194304", "decay,128,prompt,257,262144", "decay,128,prompt,2147483647,2147483647", "decay,128,step,4194304", "decay,64,step,1073741824"]


# tokens x (features, columns): columns are divided among workgroups, whose shares lie in the context
DIVIDED = ["int8,%dx%d,product,%d" % (n, k, m) for n in (1, 128, 500, 2000, 4096, 8192, 16384, 16385, 100000) for k in (100, 2000, 2048, 4096, 8191, 10000, 20000, 130944)
           for m in (1, 17, 33, 64, 65, 200, 1000, 5000)]


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    """What each call gave, its launches and the memory of its context."""
    folder = tmp_path_factory.mktemp("stand_in")
    (folder / "hip.cpp").write_text(STAND_IN)
    (folder / "calls.py").write_text(CALLS)
    subprocess.run(["g++", "-shared", "-fPIC", "-o", str(folder / "hip.so"), str(folder / "hip.cpp")], check=True)
    env = dict(os.environ, PYTHONPATH=ROOT, LD_PRELOAD=" ".join([str(folder / "hip.so"), os.environ.get("LD_PRELOAD", "")]).strip())
    run = subprocess.run([sys.executable, str(folder / "calls.py"), *FITS, *DOES_NOT, *DIVIDED], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    said, memory, launches, held = {}, {}, [], 0
    for line in run.stdout.splitlines():
        words = line.split()
        if words[:1] == ["launch"]:
            launches.append(tuple(int(x) for x in words[1:]))
        elif words[:1] == ["memory"]:
            held = int(words[1])
        elif len(words) == 3 and words[1] == "gives":
            context = words[0].rsplit(",", 2 if words[0].startswith("int8") else 3)[0]
            memory.setdefault(context, held)
            said[words[0]], launches = (int(words[2]), launches), []
    said["memory"] = memory
    return said


def test_shares_of_divided_columns_fit_into_the_context(calls):
    divided = 0
    for call in DIVIDED:
        context = call.rsplit(",", 2)[0]
        k = int(context.split("x")[1])
        codes = (1 << 22) * ((k + 127) // 128 * 128 + 4)
        code, launches = calls[call]
        assert code == 0
        x, y, _ = launches[0]
        assert len(launches) == (2 if y > 1 else 1)
        if y > 1:
            divided += 1
            assert x * y * 64 * 128 * 4 + codes <= calls["memory"][context], call
            assert y <= (k + 127) // 128 // 8
        assert calls["memory"][context] <= codes + (8 << 20)
    assert 20 < divided < len(DIVIDED)


@pytest.mark.parametrize("call", FITS)
def test_the_largest_calls_are_launched(calls, call):
    code, launches = calls[call]
    assert code == 0 and launches
    for x, y, threads in launches:
        assert 0 < x * threads < 2 ** 32 and 0 < y < 65536


@pytest.mark.parametrize("call", DOES_NOT)
def test_larger_calls_are_refused_without_a_launch(calls, call):
    assert calls[call] == (-2, [])
