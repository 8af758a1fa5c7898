"""The sizes of operator_plans reach every kernel that there is; no GPU call is made."""
import ctypes as C

import pytest

import paper_1906_12043_amd as P
from tests import operator_plans as op
from tests.operator_plans import DEEP, DIRECT, LARGE, MEDIUM, REGISTERS, SMALL, SQUARE, TALL

BOTH = (False, True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_products_of_16_bits(dtype):
    want = {(kind, tile, split, DIRECT) for kind in op.DIRECTIONS for tile in (LARGE, MEDIUM, SMALL, DEEP, TALL) for split in BOTH
            if kind != "weight_grad" or tile != TALL}
    want |= {(kind, tile, split, REGISTERS) for kind in op.DIRECTIONS for tile in (MEDIUM, SMALL) for split in BOTH}
    assert op.of_products(dtype) == want
    assert op.of_codes(dtype) == {(LARGE, s, True) for s in BOTH} | {(tile, s, d) for tile in (MEDIUM, SMALL) for s in BOTH for d in BOTH}


def test_products_of_32_bits():
    assert op.of_products("fp32") == {(kind, tile, split, REGISTERS) for kind in op.DIRECTIONS for tile in (MEDIUM, SMALL, SQUARE) for split in BOTH}
    assert op.of_codes("fp32") == {(tile, s, False) for tile in (MEDIUM, SMALL, SQUARE) for s in BOTH}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_losses_of_16_bits(dtype):
    want = {(kind, tile, DIRECT) for kind in ("logits", "slopes") for tile in (LARGE, MEDIUM, SMALL, DEEP)}
    want |= {(kind, tile, REGISTERS) for kind in ("logits", "slopes") for tile in (MEDIUM, SMALL)}
    want |= {("dh", tile, split, pieces, DIRECT) for tile in (LARGE, MEDIUM, SMALL, DEEP, TALL) for split in BOTH for pieces in BOTH}
    want |= {("dh", tile, split, pieces, REGISTERS) for tile in (MEDIUM, SMALL) for split in BOTH for pieces in BOTH}
    want |= {("de", tile, split) for tile in (LARGE, MEDIUM, SMALL, DEEP) for split in BOTH}
    assert op.of_losses(dtype) == want


def test_losses_of_32_bits():
    tiles = (MEDIUM, SMALL, SQUARE)
    want = {(kind, tile, REGISTERS) for kind in ("logits", "slopes") for tile in tiles}
    want |= {("dh", tile, split, pieces, REGISTERS) for tile in tiles for split in BOTH for pieces in BOTH} | {("de", tile, split) for tile in tiles for split in BOTH}
    assert op.of_losses("fp32") == want


def test_a_plan_follows_the_addresses():
    """What cannot go to LDS directly passes through registers, in a tile that does; without a workspace no sum is split."""
    call = op.product_call("bf16", 1, 700, 136, 16392)
    assert P.debug_grouped_plan(call, P.GROUPED_FORWARD) == (LARGE, 1, DIRECT)
    call.set(x=2 * op.A + 2)
    assert P.debug_grouped_plan(call, P.GROUPED_FORWARD) == (MEDIUM, 1, REGISTERS)
    call = op.product_call("bf16", 1, 700, 8200, 136)
    assert P.debug_grouped_plan(call, P.GROUPED_FORWARD)[1] > 1
    call.set(workspace=None)
    assert P.debug_grouped_plan(call, P.GROUPED_FORWARD)[1] == 1


def test_plans_refuse_what_the_calls_refuse():
    call = op.product_call("bf16", 1, 700, 136, 136)
    call.set(ldx=135)
    for bad, direction, text in ((call, P.GROUPED_FORWARD, "rows of x"), (op.product_call("bf16", 1, 7, 8, 8), 3, "direction"),
                                 (op.product_call("bf16", 0, 7, 8, 8), 0, "groups")):
        with pytest.raises(P.CocodError, match=text):
            P.debug_grouped_plan(bad, direction)
    loss = op.loss_call("bf16", 1, 16, 64, 700, 0)
    loss.set(flags=2)
    with pytest.raises(P.CocodError, match="flag"):
        P.debug_cross_entropy_plan(loss)
    lib = P.lib()
    assert lib.cocod_debug_grouped_plan(C.byref(call), 0, None) == P.ERR_INVALID
    assert lib.cocod_debug_grouped_plan(None, 0, None) == P.ERR_INVALID
    assert lib.cocod_debug_cross_entropy_plan(None, None, None) == P.ERR_INVALID
