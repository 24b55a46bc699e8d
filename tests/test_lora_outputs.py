"""Outputs of the adapters' calls that are another array of the same call are
refused, before anything is enqueued (no GPU is needed)."""
import ctypes

import pytest

import paper_2105_14713_amd as onexn

ARG = onexn._STATUS_NAMES.index("ONEXN_ERR_ARG")
buf = (ctypes.c_double * 256)()
at = [ctypes.addressof(buf) + 64 * (k + 1) for k in range(16)]      # addresses that are looked at only
at = [a // 16 * 16 for a in at]

FWD = dict(x=at[0], xdt=0, xs=8, rows=1, m=8, A=at[1], B=at[2], n=8, r=4, L=2, scale=at[3], ids=at[4], base=at[5],
           bs=8, y=at[6], ydt=0, ys=8, u=at[7], stream=None)
BWD = dict(x=at[0], xdt=0, xs=8, rows=1, m=8, A=at[1], B=at[2], n=8, r=4, L=2, scale=at[3], ids=at[4], u=at[7],
           dy=at[8], dys=8, base=at[5], bs=8, dx=at[9], dxdt=0, dxs=8, dA=at[10], dB=at[11], ws=at[12], wsb=1 << 20,
           stream=None)


@pytest.mark.parametrize("out,other", [("y", k) for k in ("x", "A", "B", "scale", "ids", "u")] +
                         [("u", k) for k in ("x", "A", "B", "scale", "ids", "base", "y")])
def test_forward(out, other):
    lib = onexn.load_library()
    assert lib.onexn_fc_lora_fwd(*dict(FWD, **{out: FWD[other]}).values()) == ARG
    assert "must not overlap" in onexn.last_error()


@pytest.mark.parametrize("out,other", [("dx", k) for k in ("x", "A", "B", "scale", "ids", "u", "dy")] +
                         [(o, k) for o in ("dA", "dB") for k in ("x", "A", "B", "scale", "ids", "u", "dy", "base", "dx")] +
                         [("dA", "dB")])
def test_backward(out, other):
    lib = onexn.load_library()
    assert lib.onexn_fc_lora_bwd(*dict(BWD, **{out: BWD[other]}).values()) == ARG
    assert "must not overlap" in onexn.last_error()


def test_in_place_needs_the_same_stride():
    lib = onexn.load_library()
    assert lib.onexn_fc_lora_fwd(*dict(FWD, y=FWD["base"], ys=9).values()) == ARG
    assert lib.onexn_fc_lora_bwd(*dict(BWD, dx=BWD["base"], dxs=9).values()) == ARG
