"""Every way that attention of trees may go is run against 64 bits: the cases of test_gpu_tree_paths.py are asked of the plan itself, so that
a rule that is moved cannot leave a kernel without one (host code, on the CPU)."""
import math
import random

import pytest

import tree_paths as P


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    return P.build_driver(tmp_path_factory.mktemp("tree"))


def some_shapes(count, seed):
    rng = random.Random(seed)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    for _ in range(count):
        hk, page = rng.choice((1, 1, 2, 3, 4, 8, 16)), rng.choice((1, 4, 16, 32, 64, 256))
        width = 0 if rng.random() < 0.05 else max(1, log(1, 20000) // page)
        yield (log(1, 600), log(1, 64), hk * log(1, 20), hk, rng.choice((16, 64, 96, 128, 192, 256)), log(1, 20000) if rng.random() < 0.55 else 0, width, page,
               rng.choice(("bf16", "fp16")), rng.random() < 0.5)


def test_every_way_of_the_plan_has_a_case(driver):
    ran = P.ways_of(driver, P.CASES)
    assert None not in ran
    joined, formats = set(ran), {(w[:4], c[9]) for w, c in zip(ran, P.CASES)}
    shapes = list(some_shapes(60000, 1))
    found = [(w, c) for w, c in zip(P.ways_of(driver, shapes), shapes) if w]
    assert len(found) > 50000
    missing = {w: c for w, c in found if w not in joined}
    assert not missing, missing
    missing = {(w[:4], c[9]): c for w, c in found if (w[:4], c[9]) not in formats}
    assert not missing, missing


def test_every_form_of_a_workgroup_has_a_case(driver):
    """Those that treeattn_unit.hip picks from, for each padded head: a prefix's form with a sequence's in one launch, or a sequence's behind a prefix."""
    ran = {w[:4] for w in P.ways_of(driver, P.CASES)}
    forms = {64: ("64", "128"), 128: ("64", "128", "256"), 256: ("128",)}
    for dp, many in forms.items():
        few = "few8" if dp == 256 else "few"
        assert {(dp, "-", f, "inline") for f in (*many, "few8", few)} <= ran
        assert {(dp, "-", f, how) for f in (*many, few) for how in ("whole", "cut")} <= ran
        assert {(dp, p, s, "cut") for i, p in enumerate(many) for s in ("few", *many[:i + 1])} <= ran
        assert {(dp, p, "-", "none") for p in (*many, few)} <= ran and {(dp, few, few, "cut"), (dp, "-", "few8", "whole")} <= ran
        assert {w[2] for w in ran if w[0] == dp and w[1] in many and w[3] == "whole"} >= {many[0], many[-1]}


def test_sequences_without_keys_have_no_order(driver):
    """Lengths are not there then: a call that sorted by them would read at address 0."""
    shapes = [c[:6] + (0,) + c[7:] for c in some_shapes(20000, 2)] + P.WITHOUT_OWN
    plans = [p for p in P.plans_of(driver, shapes) if p]
    assert len(plans) > 15000 and all(p[5] == "0" and p[3] in ("inline", "none") for p in plans)
    ordered = [p for p in P.plans_of(driver, [c[:6] + (1,) + c[7:] for c in P.WITHOUT_OWN])]
    assert all(p[3] == "inline" and p[5] == "1" for p in ordered)
