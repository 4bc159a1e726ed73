"""The weight gradient's share-out where a bfloat16 gradient takes several sums: every tile goes through the workspace, in one run or
in several, and none takes another's place.  (Compiled for the host.)"""
import random

from test_activation_plans import PLAN, compiled


def changed(text, old, new):
    assert text.count(old) == 1
    return text.replace(old, new)


def test_every_tile_has_a_place(tmp_path_factory):
    text = changed(PLAN, "(int)out, (int)dtype);", "(int)out, (int)dtype, true);")
    text = changed(text, "whole != (t.slot < 0)", "(whole && p.stages <= WG_SUM_STAGES_BF16) != (t.slot < 0)")
    text = changed(text, "const long long cut = p.runs > 1 ? p.full - p.whole : 0;", "const long long cut = p.cut_joins() ? p.full - p.whole : 0;")
    text = changed(text, "(p.last_runs > 1 ? p.last : 0)", "(p.last_joins() ? p.last : 0)")
    plan = compiled(tmp_path_factory, "long_plan", text)
    rng = random.Random(4)
    log = lambda lo, hi: max(lo, min(hi, int(lo * (hi / lo) ** rng.random())))
    cases = [(74, 16384, 256, 512, 1), (74, 16385, 256, 512, 1), (74, 1 << 20, 32, 8, 1), (300, 20000, 300, 700, 1), (1, 1 << 21, 64, 64, 0), (75, 16500, 33, 520, 1)]
    cases += [(log(1, 300), log(1000, 200000), log(1, 2048), log(1, 2048), rng.randrange(2)) for _ in range(300)]
    bad = [(c, r) for c, r in zip(cases, plan(cases)) if r != "0"]
    assert not bad, bad[:5]
