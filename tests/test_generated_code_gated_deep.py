"""The machine code around the LDS loads of the gated pairs' kernel for deep ranks and ragged widths, under the rules of the other products'
(test_generated_code.py); and that none of the gated pairs' kernels spills."""
import os

import pytest
import test_generated_code as rules

from paper_2309_03824_amd import build


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    obj = os.path.join(build.OBJ, "gated.hip.o")
    if not os.path.exists(obj):
        os.makedirs(build.OBJ, exist_ok=True)
        build._compile(os.path.join(build.CSRC, "gated.hip"))
    patch = pytest.MonkeyPatch()
    patch.setattr(rules, "OBJ", obj)
    try:
        return rules.listing(tmp_path_factory.mktemp("code"))
    finally:
        patch.undo()


@pytest.fixture(scope="module")
def deep(listing):
    kernels = {k: rows for k, rows in listing.items() if "gated_deep" in k}
    assert len(kernels) == 6                # three activations, both directions
    return kernels


def test_descriptors_are_settled(deep):
    assert not {k: [hex(a) for a in rules.faults(rows)] for k, rows in deep.items() if rules.faults(rows)}


def test_m0_belongs_to_the_loads(deep):
    loads = [sum(op.startswith("buffer_load") and args.endswith(" lds") for _, op, args, _ in rows) for rows in deep.values()]
    assert min(loads) > 0 and rules.m0_writes(deep) == sum(loads)


def test_a_stage_is_there_before_it_is_read(deep):
    # in the loop over stages every LDS load is waited for (all of them: vmcnt(0)) ahead of the barrier behind which the stage is read
    for k, rows in deep.items():
        barriers = [i for i, r in enumerate(rows) if r[1] == "s_barrier"]
        assert barriers, k
        for at in barriers:
            before = [r for r in rows[max(0, at - 12):at] if r[1] == "s_waitcnt"]
            assert any("vmcnt(0)" in r[2] for r in before) and "lgkmcnt(0)" in rows[at - 1][2], (k, hex(rows[at][0]))


def test_no_kernel_spills(listing):
    gated = {k: rows for k, rows in listing.items() if "gated_" in k}
    assert len(gated) > 102 and not [k for k, rows in gated.items() if any(op.startswith("scratch_") for _, op, _, _ in rows)]
