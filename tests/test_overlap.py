"""The entry points' check for arrays that share memory, compiled for the host, against marking every byte."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_11857_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "overlap.h"
int main() {   // pairs of (base, rows, groups, row stride, group stride, columns, bytes per element)
    long long v[14];
    for (;;) {
        for (long long &x : v) if (scanf("%lld", &x) != 1) return 0;
        auto rows = [](const long long *w) { return liec::rows_of((const void *)w[0], w[1], w[2], w[3], w[4], w[5], w[6]); };
        printf("%d\n", (int)liec::overlap(rows(v), rows(v + 7)));
    }
}
"""


@pytest.fixture(scope="module")
def judge(tmp_path_factory):
    where = tmp_path_factory.mktemp("overlap")
    (where / "overlap.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-I", CSRC, str(where / "overlap.cpp"), "-o", str(where / "overlap")], check=True)

    def ask(pairs):
        text = "\n".join(" ".join(str(x) for x in a + b) for a, b in pairs)
        out = subprocess.run([str(where / "overlap")], input=text, capture_output=True, text=True, check=True).stdout
        return [line == "1" for line in out.split()]
    return ask


def touched(a):
    base, rows, groups, row, group, cols, size = a
    return {base + (g * group + r * row) * size + q for g in range(groups) for r in range(rows) for q in range(cols * size)}


def dense(a):
    n = touched(a)
    return max(n) - min(n) + 1 == len(n)


def draw(rng, nested):
    rows, groups, cols, size = rng.randint(1, 5), rng.randint(1, 4), rng.randint(1, 6), rng.choice([2, 4])
    if nested:
        row = cols + rng.choice([0, 0, 1, 4])
        group = (rows - 1) * row + cols + rng.choice([0, row - cols, 3, 11])
        if rng.random() < 0.3:
            group = cols + rng.choice([0, 1, 4])
            row = (groups - 1) * group + cols + rng.choice([0, group - cols, 5])
    else:
        row, group = rng.randint(0, 12), rng.randint(0, 30)
    return (1024 + size * rng.randint(0, 120), rows, groups, row, group, cols, size)


def test_slices_of_one_buffer_and_blocks(judge):
    """Equal strides, as two slices of one buffer have, or one array without gaps: the answer is exact."""
    rng = random.Random(1)
    pairs = []
    while len(pairs) < 20000:
        a = draw(rng, rng.random() < 0.7)
        if rng.random() < 0.5:
            b = (1024 + a[6] * rng.randint(0, 120),) + a[1:]
        else:
            b = draw(rng, rng.random() < 0.5)
            if not (dense(a) or dense(b)):
                continue
            blocks = [c for c in (a, b) if c[1] == 1 or c[3] in (0, c[5])]
            if not any(c[2] == 1 or c[4] in (0, c[5] if c[1] == 1 or c[3] == 0 else c[1] * c[3]) for c in blocks):
                continue   # (without gaps, but folded over itself: not taken for a block)
        pairs.append((a, b))
    want = [bool(touched(a) & touched(b)) for a, b in pairs]
    assert 4000 < sum(want) < 16000
    wrong = [(p, w) for p, w, got in zip(pairs, want, judge(pairs)) if got != w]
    assert not wrong, wrong[:3]


def test_nothing_apart_is_refused(judge):
    """Any pair at all: what is called an overlap is one."""
    rng = random.Random(2)
    pairs = [(draw(rng, rng.random() < 0.5), draw(rng, rng.random() < 0.5)) for _ in range(20000)]
    wrong = [p for p, got in zip(pairs, judge(pairs)) if got and not touched(p[0]) & touched(p[1])]
    assert not wrong, wrong[:3]


def test_large_offsets(judge):
    """Slices of a buffer beyond 2^32 elements."""
    h, rows, groups = 1000, 1 << 21, 8
    wide = (1 << 20, rows, groups, 3 * h, 3 * h * rows, h, 4)
    at = lambda shift: ((1 << 20) + 4 * shift,) + wide[1:]
    pairs = [(wide, at(h)), (wide, at(h - 1)), (wide, at(2 * h)), (wide, at(2 * h + 1)), (wide, at(3 * h * rows * 3 + h)), (wide, at(3 * h * rows * 3 + 1)),
             (wide, at(3 * h * rows * groups))]
    assert judge(pairs) == [False, True, False, True, False, True, False]
