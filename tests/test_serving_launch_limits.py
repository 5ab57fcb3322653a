"""Sizes at which the serving operators' calls need more workgroups than a launch has: refused on the host.

A launch has fewer than 2^32 threads in a dimension, 2^24 - 1 workgroups of 256.  The library runs in a process of its own whose HIP runtime is a
stand-in that keeps no device and only notes launches, so both sides of each limit can be called without a GPU."""
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
int hipMalloc(void** p, size_t) { *p = std::aligned_alloc(256, 4096); return 0; }
int hipFree(void* p) { std::free(p); return 0; }
int hipMemset(void*, int, size_t) { return 0; }
int hipDeviceSynchronize() { return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetLastError() { return 0; }
int __hipPushCallConfiguration(dim g, dim b, size_t, void*) { grid = g; block = b; return 0; }
int __hipPopCallConfiguration(dim* g, dim* b, size_t* shared, void** stream) { *g = grid; *b = block; *shared = 0; *stream = nullptr; return 0; }
int hipLaunchKernel(const void*, dim g, dim b, void**, size_t, void*) { std::printf("launch %u %u %u\n", g.x, g.y, b.x); std::fflush(stdout); return 0; }
}
"""

CALLS = r"""
import ctypes as C, sys
from paper_2504_02211_amd import ftcache, ftprompt
row = ftprompt._ROWS.pack(0x1000, 1024, 64)

def create(module, name, **fields):
    cfg, handle = module.Config(struct_size=C.sizeof(module.Config), head_dim=64, in_dtype=0, out_dtype=0, softmax_scale=0.0, device=0, **fields), C.c_void_p()
    assert getattr(module.load_library(), name + "_create")(C.byref(cfg), C.byref(handle)) == 0
    return module.load_library(), handle

lib, h = create(ftprompt, "ftprompt", heads=4, kv_heads=4)
forward = lambda tokens, batch: lib.ftprompt_forward(h, row, row, row, row, 0x1000, 0x1000, batch, tokens, 64, None)
lib, hc = create(ftcache, "ftcache", heads=512, kv_heads=256, pages=4, page_size=16, rotary_dim=0, interleaved=0, max_batch=65536)
places = lambda tokens, batch: ftcache._PLACES.pack(batch, tokens, 0x1000, 0x1000, 0x1000, 4, 4)
append = lambda tokens, batch: lib.ftcache_append(hc, 0x1000, places(tokens, batch), 0x1000, 16, row, row, row, row, row, None)
read = lambda tokens, batch: lib.ftcache_read(hc, 0x1000, places(tokens, batch), row, row, None)
attend = lambda batch, width: lib.ftcache_attend(hc, 0x1000, batch, 0x1000, 0x1000, width, width, row, row, None)
for name, a, b in [x.split(",") for x in sys.argv[1:]]:
    print(name, a, b, "gives", {"forward": forward, "append": append, "read": read, "attend": attend}[name](int(a), int(b)), flush=True)
"""

# row tiles of 128 rows and one more a sequence, times 4 key heads; blocks of 8 places and two more a sequence; sequences of up to 64 tokens, times 256 key heads
FITS = ["forward,536870656,1", "forward,10,4194302", "append,134217704,1", "append,7,8388607", "read,134217704,1", "read,7,8388607", "attend,65535,4"]
DOES_NOT = ["forward,536870784,1", "forward,10,4194304", "forward,2147483647,1", "append,134217712,1", "append,8,8388608", "append,2147483647,2147483647",
            "read,134217712,1", "read,8,8388608", "attend,65536,4"]


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    folder = tmp_path_factory.mktemp("stand_in")
    (folder / "hip.cpp").write_text(STAND_IN)
    (folder / "calls.py").write_text(CALLS)
    subprocess.run(["g++", "-shared", "-fPIC", "-o", str(folder / "hip.so"), str(folder / "hip.cpp")], check=True)
    env = dict(os.environ, PYTHONPATH=ROOT, LD_PRELOAD=" ".join([str(folder / "hip.so"), os.environ.get("LD_PRELOAD", "")]).strip())
    run = subprocess.run([sys.executable, str(folder / "calls.py"), *FITS, *DOES_NOT], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    said, launch = {}, None
    for line in run.stdout.splitlines():
        words = line.split()
        if words[:1] == ["launch"]:
            launch = tuple(int(x) for x in words[1:])
        elif len(words) == 5 and words[3] == "gives":
            said[",".join(words[:3])], launch = (int(words[4]), launch), None
    return said


@pytest.mark.parametrize("call", FITS)
def test_the_largest_calls_are_launched(calls, call):
    code, (x, y, threads) = calls[call]
    assert code == 0 and threads == 256 and 2 ** 23 < x < 2 ** 24 and y == 1


@pytest.mark.parametrize("call", DOES_NOT)
def test_larger_calls_are_refused_without_a_launch(calls, call):
    assert calls[call] == (-2, None)
