"""CPU checks of which keys a query of the attention sees, as its kernels count them: the
header's arithmetic compiled for the host, against its definition."""
import os
import subprocess

import numpy as np

from oracle import step_operators as O
from paper_2609_15160_amd import build

NONE = (1 << 31) - 1  # no window

MAIN = """
#include <cstdio>
#include "visible.h"
int main() {
  int p, window, sinks;
  while (std::scanf("%d %d %d", &p, &window, &sinks) == 3) {
    const tlf::VisibleKeys k(p, window, sinks);
    std::printf("%d %d %d", k.near, k.sinks, k.count);
    for (int i = 0; i < k.count && i < 200; ++i) std::printf(" %d", k[i]);
    std::printf("\\n");
  }
}
"""


def _keys(tmp_path, cases):
    """The lines of the header's answers.  -ftrapv: arithmetic that leaves 32 bits ends the program."""
    (tmp_path / "t.cpp").write_text(MAIN)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-ftrapv", "-I", build.CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")])
    text = "".join(" ".join(map(str, c)) + "\n" for c in cases)
    out = subprocess.run([str(tmp_path / "t")], input=text, capture_output=True, text=True, check=True).stdout
    return [[int(v) for v in line.split()] for line in out.splitlines()]


def test_visible_keys_are_the_definitions(tmp_path):
    cases = [(p, w, s) for p in (-40, -4, -3, -2, -1, 0, 1, 2, 5, 39, 63, 64, 65, 130) for w in (1, 2, 40, 64, 500, NONE)
             for s in ((0, 1, 3, 64) if w != NONE else (0,))]
    n = 131
    for (p, w, s), got in zip(cases, _keys(tmp_path, cases)):
        want = np.flatnonzero(O.visible(n, n, None if w == NONE else w, s)[p]) if p >= 0 else []
        assert got[3:] == list(want) and got[2] == len(want), (p, w, s, got)


def test_positions_at_the_ends_of_their_range(tmp_path):
    """Queries far before the first key, which see none, and far behind it."""
    far = 1 << 29
    cases = [(p, w, s) for p in (-far, -3, far - 1) for w in (1, 40, far - 2, far - 1, far, NONE) for s in ((0, 64) if w != NONE else (0,))]
    for (p, w, s), got in zip(cases, _keys(tmp_path, cases)):
        if p < 0:
            assert got[2] == 0 and len(got) == 3, (p, w, s, got)
            continue
        near = max(0, p - w + 1)
        first = min(s, near)
        assert got[:3] == [near, first, first + p - near + 1], (p, w, s, got)
        assert got[3:] == [i if i < first else near + i - first for i in range(min(got[2], 200))]
