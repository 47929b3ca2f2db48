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
