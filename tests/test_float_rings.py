"""Rings of the products on tensor memory: nobody waits for a round of a place without knowing that the round before is through.

A barrier tells a round by its parity, so a wait for round r returns at once while round r - 1 is still under way.  The model below walks a group of converter warps through its stages and keeps what the group can know - what it has
waited for itself, and what follows from that because stages are emptied in order and units are fetched in order - with copies that
land in any order.  Host arithmetic on the library's own plans; no GPU.
"""
from __future__ import annotations

import itertools

import pytest

from paper_2011_10680_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()


def unsafe_wait(stages, units, unit_stages, groups, steps, turns=40):
    """The first wait of a group that may return a round too early, or None.  `steps`: stages of a tile."""
    padded = -(-steps // unit_stages) * unit_stages
    per_tile = padded // unit_stages                                  # units
    last_stage = {}                                                   # of a unit: the last stage that is converted
    for unit in range(turns * groups // unit_stages + 2):
        tile, at = divmod(unit, per_tile)
        last_stage[unit] = tile * steps + min((at + 1) * unit_stages, steps) - 1

    def unit_of(stage):
        tile, at = divmod(stage, steps)
        return tile * per_tile + at // unit_stages

    for group in range(groups):
        landed, landed_to = set(), -1                                 # units this group has seen; all units up to that one
        emptied_to = -1                                               # stages up to that one have been multiplied
        for v in range(group, turns * groups, groups):
            tile, at = divmod(v, padded)
            unit = v // unit_stages
            if unit >= units and not (unit - units in landed or unit - units <= landed_to):
                return "raw", group, v
            landed.add(unit)
            # this unit was fetched once the unit before in its place was through: all earlier fetches had landed for that, and every stage
            # of it had found its place empty
            landed_to = max(landed_to, unit - units)
            if unit >= units:
                emptied_to = max(emptied_to, last_stage[unit - units] - stages)
            if at < steps:
                stage = tile * steps + at
                if stage >= 2 * stages and emptied_to < stage - 2 * stages:
                    return "stage", group, v
                emptied_to = max(emptied_to, stage - stages)
            if emptied_to >= 0:
                landed_to = max(landed_to, unit_of(emptied_to))
    return None


def plans():
    seen = {}
    for product, m, n, k in itertools.product(("linear", "dgrad", "wgrad"), (17, 40, 100, 120, 300, 513, 600, 1000, 2500, 4000, 8192),
                                              (16, 96, 200, 520, 1032, 2048, 4096, 8200, 20000), (32, 96, 160, 352, 1056, 4096, 8224)):
        plan = binding.linear_plan(product, m, n, k, 64)
        if plan["kernel"] == "tensor_memory":
            seen.setdefault((product, plan["columns"]), set()).add(tuple(plan[name] for name in ("stages", "units", "unit_stages", "groups")))
    return seen


def test_no_wait_returns_a_round_early():
    seen = plans()
    assert set(seen) == set(itertools.product(("linear", "dgrad", "wgrad"), (32, 64, 128, 256)))
    for (product, columns), rings in seen.items():
        assert len(rings) == 1
        (stages, units, unit_stages, groups), = rings
        for steps in range(1, 70):
            assert unsafe_wait(stages, units, unit_stages, groups, steps) is None, (product, columns, steps)


@pytest.mark.parametrize("rings,steps", [
    ((6, 6, 1, 4), 40),       # four groups in a ring of six units: group 2 meets unit 6 without having seen unit 0
    ((6, 8, 1, 6), 40),       # six in a ring of eight
    ((6, 2, 4, 6), 40),       # units of four stages: the same, by stages
    ((6, 2, 4, 4), 11),       # the units fit; the filled-up stages of a tile's last unit leave a group without a recent stage
    ((6, 9, 1, 9), 40),       # more groups than stages
])
def test_the_model_tells_rings_that_do_not_hold(rings, steps):
    assert unsafe_wait(*rings, steps) is not None


def test_plan_refuses_what_it_cannot_plan():
    import ctypes as C
    plan = binding.hq_product_plan()
    L = binding.lib()
    for bad in ((3, 1, 8, 32, 32, 148), (-1, 1, 8, 32, 32, 148), (0, 0, 8, 32, 32, 148), (0, 1, 0, 32, 32, 148), (0, 1, 8, 31, 32, 148), (0, 1, 8, 32, 48, 148),
                (0, 1, 8, 32, 32, 0)):
        assert L.hq_linear_plan(*bad, C.byref(plan)) == binding.HQ_ERR_INVALID_ARG
    assert L.hq_linear_plan(0, 1, 8, 32, 32, 148, None) == binding.HQ_ERR_INVALID_ARG
    assert binding.linear_plan("dgrad", 10, 33, 64, 32)["kernel"] == "cuda_cores"
    assert binding.linear_plan("linear", 1, 4096, 4096, 128)["kernel"] == "few_rows"


def test_launchers_take_the_number_of_sms_from_the_handle():
    import os
    import re
    for name in sorted(os.listdir(build.CSRC_FLOAT)):
        with open(os.path.join(build.CSRC_FLOAT, name)) as f:
            code = re.sub(r"//[^\n]*", "", f.read())
        assert not re.search(r"\b148(ll|u|ull)?\b", code), name
