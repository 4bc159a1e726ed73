"""Host arithmetic of the operators on activations, compiled for the host: the weight gradient's share-out covers the work
exactly once, and arrays of three axes that share memory are told apart byte by byte."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_11857_b200", "csrc")

PLAN = r"""
#include <cstdio>
#include <map>
#include <set>
#include <vector>
#include "weight_grad_plan.h"
using namespace liec;
int main() {   // workers, rows, in, out, dtype -> 0, or the number of the check that failed
    long long w, rows, in, out, dtype;
    while (scanf("%lld %lld %lld %lld %lld", &w, &rows, &in, &out, &dtype) == 5) {
        const WgPlan p = wg_plan((int)w, rows, (int)in, (int)out, (int)dtype);
        const long long slabs = wg_slabs((int)dtype), c_tiles = (in + 255) / 256, slabs_all = (out + 255) / 256, o_tiles = (slabs_all + slabs - 1) / slabs;
        int bad = 0;
        if (p.stages != (rows + 31) / 32 || p.pairs < 1 || p.pairs > WG_PAIRS || p.pairs > p.items) bad = 1;
        std::map<std::vector<int>, std::vector<char>> seen;   // tile -> stages done
        std::map<std::vector<int>, std::vector<long long>> slots;
        std::set<std::pair<long long, long long>> used;
        for (long long i = 0; i < p.items && !bad; ++i) {
            const WgItem t = p.item(i);
            std::vector<int> key = {t.worker, t.c_tile, t.o_tile};
            if (t.worker < 0 || t.worker >= w || t.c_tile < 0 || t.c_tile >= c_tiles || t.o_tile < 0 || t.o_tile >= o_tiles) { bad = 2; break; }
            if (t.slabs != std::min(slabs, slabs_all - t.o_tile * slabs) || t.stages < 1) { bad = 3; break; }
            auto &s = seen[key];
            s.resize(p.stages);
            if (t.stage < 0 || t.stage + t.stages > p.stages) { bad = 4; break; }
            for (int k = t.stage; k < t.stage + t.stages; ++k) bad = s[k]++ ? 5 : bad;
            const bool whole = t.stages == p.stages;
            if (whole != (t.slot < 0)) bad = 6;                       // whole tiles go to the gradient, others to the workspace
            if (t.slot >= 0) {
                const long long size = (long long)t.slabs * 256 * 256;
                if (t.slot % 4 || t.slot + size > p.slots()) bad = 7;
                if (!used.insert({t.slot, t.slot + size}).second) bad = 8;
                slots[key].push_back(t.slot);
            }
        }
        long long end = 0;
        for (auto &u : used) { if (u.first < end) bad = 9; end = u.second; }
        if (!bad && (long long)seen.size() != w * c_tiles * o_tiles) bad = 10;
        for (auto &s : seen) for (char c : s.second) if (c != 1) bad = bad ? bad : 11;
        // the joining kernel's places: cut tile `index` has its runs tiles * size apart
        const long long cut = p.runs > 1 ? p.full - p.whole : 0;
        for (long long y = 0; y < cut + (p.last_runs > 1 ? p.last : 0) && !bad; ++y) {
            const bool last = y >= cut;
            const long long index = last ? y - cut : y, tiles = last ? p.last : cut, size = p.slot_size(last);
            const WgItem t = p.tile_of((last ? p.full : p.whole) + index);
            auto &list = slots[{t.worker, t.c_tile, t.o_tile}];
            if ((long long)list.size() != (last ? p.last_runs : p.runs)) { bad = 12; break; }
            for (size_t r = 0; r < list.size(); ++r)
                if (list[r] != index * size + (last ? cut * p.runs * p.slot_size(false) : 0) + (long long)r * tiles * size) bad = 13;
        }
        printf("%d\n", bad);
    }
}
"""

AXES = r"""
#include <cstdio>
#include "axes.h"
using namespace liec;
int main() {   // pairs of (base, columns, bytes, n0, n1, n2, s0, s1, s2), outer to inner -> meet(a, b), disjoint(a)
    long long v[18];
    for (;;) {
        for (long long &x : v) if (scanf("%lld", &x) != 1) return 0;
        auto axes = [](const long long *w) { return axes_of((const void *)w[0], w[1], (int)w[2], {w[3], w[4], w[5]}, {w[6], w[7], w[8]}); };
        printf("%d %d\n", (int)meet(axes(v), axes(v + 9)), (int)disjoint(v[1], {v[3], v[4], v[5]}, {v[6], v[7], v[8]}));
    }
}
"""


def compiled(tmp_path_factory, name, text):
    where = tmp_path_factory.mktemp(name)
    (where / "p.cpp").write_text(text)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, str(where / "p.cpp"), "-o", str(where / "p")], check=True)
    return lambda rows: subprocess.run([str(where / "p")], input="\n".join(" ".join(str(x) for x in r) for r in rows), capture_output=True, text=True,
                                       check=True).stdout.split("\n")[:-1]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return compiled(tmp_path_factory, "plan", PLAN)


@pytest.fixture(scope="module")
def axes(tmp_path_factory):
    return compiled(tmp_path_factory, "axes", AXES)


def test_every_stage_of_every_tile_once(plan):
    rng = random.Random(1)
    log = lambda lo, hi: max(lo, min(hi, int(lo * (hi / lo) ** rng.random())))
    cases = [(8, 8192, 768, 2304, 1), (16, 3136, 512, 2048, 1), (3, 1501, 1333, 515, 1), (4, 32, 256, 256, 0), (148, 4096, 256, 256, 0), (1, 1, 1, 1, 0),
             (1, 1, 1, 1, 1), (74, 33, 256, 512, 1), (75, 33, 256, 512, 1), (1, 1 << 20, 64, 64, 1), (200, 5, 300, 700, 1), (1, 100, 65536, 300, 0)]
    cases += [(log(1, 300), log(1, 20000), log(1, 4096), log(1, 4096), rng.randrange(2)) for _ in range(600)]
    bad = [(c, r) for c, r in zip(cases, plan(cases)) if r != "0"]
    assert not bad, bad[:5]


def touched(a):
    base, cols, size, n0, n1, n2, s0, s1, s2 = a
    return [base + (i * s0 + j * s1 + k * s2) * size + q for i in range(n0) for j in range(n1) for k in range(n2) for q in range(cols * size)]


def test_three_axes(axes):
    rng = random.Random(2)

    def nested():
        cols, size = rng.randint(1, 5), rng.choice([2, 4])
        order, n, s, reach = rng.sample(range(3), 3), [0] * 3, [0] * 3, cols
        for axis in order:
            n[axis] = rng.randint(1, 4)
            s[axis] = reach + rng.choice([0, 0, 1, 3])
            reach = s[axis] * (n[axis] - 1) + reach
        return cols, size, *n, *s

    pairs = []
    for _ in range(20000):
        a = nested()
        b = a if rng.random() < 0.6 else nested()
        if rng.random() < 0.2:
            b = b[:5] + (0,) + b[6:] if b[5] > 1 else b
        pairs.append(((1024 + a[1] * rng.randint(0, 150),) + a, (1024 + b[1] * rng.randint(0, 150),) + b))
    pairs = [(a, tuple(max(1, v) if 3 <= i <= 5 else v for i, v in enumerate(b))) for a, b in pairs]
    hits = 0
    for (a, b), line in zip(pairs, axes([a + b for a, b in pairs])):
        met, apart = line.split()
        ta, tb = touched(a), touched(b)
        share = bool(set(ta) & set(tb))
        assert apart == "1" and len(set(ta)) == len(ta), a       # nested steps never overlap themselves
        assert met == "0" or share, (a, b)                        # what is called an overlap is one
        if a[1:] == b[1:]:                                        # slices of one buffer: exact
            assert (met == "1") == share, (a, b)
            hits += share
    assert hits > 2000


def test_arrays_that_overlap_themselves_are_told(axes):
    rng = random.Random(3)
    rows = [(1024, rng.randint(1, 4), 2) + tuple(rng.randint(1, 4) for _ in range(3)) + tuple(rng.randint(0, 20) for _ in range(3)) for _ in range(5000)]
    for a, line in zip(rows, axes([a + a for a in rows])):
        if line.split()[1] == "1":
            t = touched(a)
            assert len(set(t)) == len(t), a
