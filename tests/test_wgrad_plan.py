"""The weight gradient's plan on the CPU: the forms of the calls that the GPU
tests make, the workspace, and that every token falls into one run."""
import random

import pytest

import paper_2507_07114_amd as ll
import wgrad_plans as wp

FORMS = {"256 whole", "256 both", "256 runs", "128 whole", "128 both", "128 runs", "light whole"}


def test_every_form_of_both_types_is_among_the_cases():
    # (fp32 dy has no light form; 128 x 128 tiles, whole and in runs of bf16 dy are in
    # further cases of test_gpu_local.py)
    bf16 = {c[-2] for c in wp.CASES}
    f32 = {c[-1] for c in wp.CASES}
    assert bf16 >= {"light whole", "128 runs", "256 whole", "256 both", "256 runs"}
    assert f32 >= FORMS - {"light whole"}
    for form in ("256 whole", "256 both", "256 runs"):
        assert {c[2] % 8 == 0 and c[3] % 8 == 0 for c in wp.CASES if c[-2] == form} == {True, False}


@pytest.mark.parametrize("case", wp.CASES, ids=lambda c: "x".join(map(str, c[:4])))
def test_forms(case):
    n, t, o, h = case[:4]
    plans = [wp.plan(bf16, n, t, o, h) for bf16 in (True, False)]
    assert tuple(p.form for p in plans) == case[-2:]
    # one workspace serves either type
    assert ll.ll_act_wgrad_workspace_bytes(n, t, o, h) == max(p.part for p in plans)


def test_tiles_and_runs_cover_any_call():
    rng = random.Random(5)
    size = lambda top: int(round(2 ** rng.uniform(0, top)))
    seen = set()
    for _ in range(3000):
        n, t, o, h = size(7), size(15), size(13), size(13)
        bf16 = rng.random() < 0.5
        p = wp.plan(bf16, n, t, o, h)
        seen.add(p.form)
        assert p.whole + p.rest == n * -(-o // p.edge) * -(-h // p.edge)
        if p.runs == 1:
            assert p.rest == 0 and p.part == 0
        else:
            # every run has tokens, the last one ends the batch
            assert p.rest > 0 and p.run_t % 32 == 0
            assert (p.runs - 1) * p.run_t < t <= p.runs * p.run_t
            assert p.part == p.rest * p.runs * p.edge ** 2 * 4 <= 1 << 28
        assert not p.light or (bf16 and p.runs == 1)
    assert seen == FORMS
    assert wp.plan(True, 3, 0, 40, 50).runs == 1  # no tokens
