"""Which workgroups of a call read a state that another one of the same launch writes: none may, as nothing orders them.  And where states lie between launches.

The lines of ftdecay.hip that choose where a segment's state comes from and where it goes are compiled for the host, as they stand, and asked for every segment of a call.
"""
import os
import random
import re
import subprocess

import pytest

pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "paper_2504_02211_amd", "csrc", "ftdecay.hip")

HARNESS = r"""
#include <cstdint>
#include <cstdio>
#include <vector>
constexpr int D = 1;      // (a state is one number: addresses count states)
struct Segment { int b, h, number, tokens, first; bool last; int64_t before; };
struct Args { const int32_t* starts; float* between; int heads; };
%(constants)s
struct Chunk { const float* from = nullptr; float* to = nullptr; };
int main() {
  static float pool[1], workspace[1 << 14];
  for (int starts = 0; starts < 2; ++starts)
    for (int there = 0; there < 2; ++there)
      for (int segments = 1; segments < 5; ++segments)
        for (int number = 0; number < segments; ++number) {
          int32_t s = starts;
          const Args a{&s, workspace, 2};
          const Segment g{0, 1, number, 10, 0, number == segments - 1, 3};
          float* const state = there ? pool : nullptr;
          float* to = nullptr;
          struct { void put(int, float* x, float = 1.f) { *at = x; } float power(int) { return 1.f; } float** at; } c{&to};
          const int S = 0, lifted = 0;
          %(from)s
          %(to)s
          auto place = [&](const float* x) { return x == nullptr ? -1L : x == pool ? -2L : (long)(x - workspace); };
          std::printf("%%d %%d %%d %%d %%ld %%ld\n", starts, there, segments, number, place(from), place(to));
        }
}
"""


def source():
    with open(SOURCE) as f:
        return f.read()


@pytest.fixture(scope="module")
def segments(tmp_path_factory):
    """{(continues, has a place in the pool, segments, number): (where from, where to)}; -1: nowhere, -2: the pool, else a place in the workspace."""
    text = source()
    kernel = text[text.index("void ftdecay_chunks("):]
    begin = re.search(r"const float\* from = nullptr;.*?(?=\n  const Loader)", kernel, re.S).group(0)
    end = re.search(r"if \([^;\n]*\) c\.put\(S, [^;\n]*\);", kernel).group(0)
    folder = tmp_path_factory.mktemp("segments")
    constants = re.search(r"constexpr int STATES = [^;]*;", text).group(0)
    (folder / "s.cpp").write_text(HARNESS % {"constants": constants, "from": begin, "to": end})
    subprocess.run(["g++", "-std=c++17", "-w", "-o", str(folder / "s"), str(folder / "s.cpp")], check=True)
    lines = subprocess.run([str(folder / "s")], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    rows = [tuple(int(x) for x in line.split()) for line in lines]
    return {r[:4]: r[4:] for r in rows}


def test_no_segment_reads_a_state_that_another_one_writes(segments):
    assert len(segments) == 2 * 2 * (1 + 2 + 3 + 4)
    for (starts, there, n, number), (begins, ends) in segments.items():
        written = [segments[starts, there, n, other][1] for other in range(n) if other != number]
        assert begins == -1 or begins not in written, (starts, there, n, number, begins)


def test_every_segment_begins_with_what_it_continues(segments):
    for (starts, there, n, number), (begins, ends) in segments.items():
        assert ends == (-2 if there and number == n - 1 else -1)
        if number == 0:
            assert (begins != -1) == bool(starts and there)
        else:
            assert begins == (3 + number - 1) * 2 + 1      # (the state behind the segment before it)


def test_places_in_the_workspace_belong_to_one_state_each(segments):
    """Divided sequences of any lengths: what they keep between launches lies in the room that a context has, at places of their own."""
    text = source()
    states = int(re.search(r"constexpr int STATES = (\d+)", text).group(1))
    rooms = int(re.search(r"hipMalloc\(\(void\*\*\)&c->between, \(size_t\)(?:(\d+) \* )?STATES", text).group(1) or 1)
    rng = random.Random(5)
    first = segments[1, 1, 2, 0][0]          # of (before 3, 2 heads, head 1)
    for _ in range(300):
        heads, batch = rng.choice([1, 2, 3, 4, 8, 12, 32]), rng.randint(1, 40)
        lengths = [rng.choice([0, 1, 191, 192, 193, rng.randint(0, 2000)]) for _ in range(batch)]
        total = sum(lengths)
        per = max(192, (total * heads + 511) // 512, -(-total * heads // states))
        per = -(-per // 64) * 64
        at, used = 0, set()
        for n in lengths:
            pieces = max(1, -(-n // per))
            if pieces > 1:
                before = at // per
                places = [(before + i) * heads + h for i in range(pieces - 1) for h in range(heads)]
                places += [first - (3 * 2 + 1) + before * heads + h for h in range(heads)]
                assert not used.intersection(places) and max(places) < rooms * states
                used.update(places)
            at += n
