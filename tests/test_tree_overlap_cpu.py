"""Outputs of the tree calls that share bytes with what their workgroups read are
refused on the host (no call passes validation, so nothing reaches a GPU)."""

import ctypes

import pytest

import paper_2609_32663_amd as d

POOL = ctypes.c_void_p(0x90000000)
FIRST, PATH, N_PATH, TABLE, NEW_LEN, KEEP = (0x10000 * i for i in range(1, 7))
N, B, HKV, MOST, PPS = 4, 2, 2, 8, 5
# bytes of each: int32 [N], int32 [B][MOST], int32 [B], int32 [N * HKV][PPS], int32 [N], uint8 [N * HKV][PPS]
BYTES = {"first": 4 * N, "path": 4 * B * MOST, "n_path": 4 * B, "table": 4 * N * HKV * PPS, "new_len": 4 * N,
         "keep": N * HKV * PPS}
AT = {"first": FIRST, "path": PATH, "n_path": N_PATH, "table": TABLE, "new_len": NEW_LEN, "keep": KEEP}


def accept(**kw):
    a = {**AT, **kw}
    p = {k: None if v is None else ctypes.c_void_p(v) for k, v in a.items()}
    return d.library().dkv_paged_accept(d.DKV_CACHE_F8, N, B, HKV, 128, p["first"], p["path"], p["n_path"], MOST, p["table"],
                                        PPS, 128, POOL, POOL, POOL, 9, p["new_len"], p["keep"], None)


@pytest.mark.parametrize("out", ["new_len", "keep"])
@pytest.mark.parametrize("other", ["first", "path", "n_path", "table", "new_len", "keep"])
def test_accept_refuses_outputs_over_its_inputs(out, other):
    """The first and the last byte of one in the other, from either side: a unit's first segment writes what another
    segment, or another layer's unit, has still to read."""
    if out == other:
        return
    unit = 1 if out == "keep" else 4
    for at in (AT[other], AT[other] + BYTES[other] - unit, AT[other] - BYTES[out] + unit):
        assert accept(**{out: at}) == d.DKV_ERR_INVALID_ARG, hex(at - AT[other])


PLAN_BYTES = {"off": 4 * 3, "first": 4 * 2, "parent": 4 * 80, "pos": 4 * 80, "mask": 8 * 80 * 2}
PLAN_AT = {name: 0x10000 * i for i, name in enumerate(PLAN_BYTES, 1)}


def plan(**kw):
    p = {k: ctypes.c_void_p(v) for k, v in {**PLAN_AT, **kw}.items()}
    return d.library().dkv_tree_plan(2, 80, 70, p["off"], p["first"], p["parent"], p["pos"], p["mask"], 2, None)


@pytest.mark.parametrize("out", ["pos", "mask"])
@pytest.mark.parametrize("other", list(PLAN_BYTES))
def test_plan_refuses_outputs_over_its_inputs(out, other):
    """One sequence's workgroup writes its rows while another's reads offsets and parents.  Positions in the very place of
    the parents are the exception: a workgroup holds its own parents by then."""
    if out == other:
        return
    unit = 8  # of the mask, whose alignment is checked first
    for at in (PLAN_AT[other], PLAN_AT[other] + (PLAN_BYTES[other] - 1) // unit * unit, PLAN_AT[other] - PLAN_BYTES[out] + unit):
        if (out, other) == ("pos", "parent") and at == PLAN_AT[other]:
            continue
        assert plan(**{out: at}) == d.DKV_ERR_INVALID_ARG, hex(at - PLAN_AT[other])
