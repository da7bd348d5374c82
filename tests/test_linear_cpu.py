"""CPU checks of the linear layers' entry points: what they refuse, they refuse on the host, before anything is launched; and the
oracle itself on small cases worked out by hand."""
import ctypes

import numpy as np
import pytest

from oracle import linear as ol
from paper_2208_00763_b200 import binding as hk
from paper_2208_00763_b200 import build as lib_build


@pytest.fixture(scope="module", autouse=True)
def built_library():
    lib_build.build()
    return hk.lib()


# addresses that no call here may follow, far enough apart that nothing overlaps
X, W, OUT, SCALE, SCALE2, BIAS, RES, OFF = (0x100000000000 + (i << 40) for i in range(8))
WS = 0x900000000000
GOOD = dict(ws_ptr=None, ws_bytes=0, x=X, x_row=64, w=W, store=8, M=4, N=32, K=64, p=8, q=8, xs=1, ws=1, out=OUT, out_row=32, ep=dict(out_type=hk.OUT_BF16))


def call(grouped=False, offsets=OFF, E=3, **change):
    a = {**GOOD, **change}
    ep = None if a["ep"] is None else ctypes.byref(hk.EpilogueT(**a["ep"]))
    sizes = (a["M"], a["N"], a["K"], a["p"], a["q"], a["xs"], a["ws"], a["out"], a["out_row"], ep, a["ws_ptr"], a["ws_bytes"],
             None)
    if grouped:
        return hk.lib().hikonv_grouped_linear(a["x"], a["x_row"], a["w"], a["store"], offsets, E, *sizes)
    return hk.lib().hikonv_linear(a["x"], a["x_row"], a["w"], a["store"], *sizes)


F, C, S = (dict(out_type=t) for t in (hk.OUT_BF16, hk.OUT_CODES, hk.OUT_SUMS))
REFUSED = [
    (hk.ERR_INVALID_ARG, dict(ep=None)),
    (hk.ERR_INVALID_ARG, dict(M=-1)), (hk.ERR_INVALID_ARG, dict(N=0)), (hk.ERR_INVALID_ARG, dict(K=0)),
    (hk.ERR_INVALID_ARG, dict(p=0)), (hk.ERR_INVALID_ARG, dict(p=9)), (hk.ERR_INVALID_ARG, dict(q=0)), (hk.ERR_INVALID_ARG, dict(q=9)),
    (hk.ERR_INVALID_ARG, dict(x=None)), (hk.ERR_INVALID_ARG, dict(w=None)), (hk.ERR_INVALID_ARG, dict(out=None)),
    (hk.ERR_INVALID_ARG, dict(x_row=63)), (hk.ERR_INVALID_ARG, dict(out_row=31)), (hk.ERR_INVALID_ARG, dict(x_row=-64)),
    (hk.ERR_UNSUPPORTED, dict(M=(1 << 30) + 1)), (hk.ERR_UNSUPPORTED, dict(N=(1 << 30) + 1, out_row=1 << 31)),
    (hk.ERR_INVALID_ARG, dict(x_row=1 << 40)), (hk.ERR_INVALID_ARG, dict(x_row=1 << 50)), (hk.ERR_INVALID_ARG, dict(out_row=1 << 50)),
    (hk.ERR_INVALID_ARG, dict(store=4)), (hk.ERR_INVALID_ARG, dict(store=3, q=3)), (hk.ERR_INVALID_ARG, dict(store=0)),
    (hk.ERR_UNSUPPORTED, dict(store=4, q=4, K=63)), (hk.ERR_UNSUPPORTED, dict(store=1, q=1, K=60)),
    (hk.ERR_NO_FIT, dict(K=131072, x_row=131072)), (hk.ERR_NO_FIT, dict(K=33026, x_row=33026, xs=0, ws=0)),
    (hk.ERR_NO_FIT, dict(K=131072, x_row=131072, store=4, q=4)), (hk.ERR_NO_FIT, dict(K=2 ** 31 - 8, x_row=2 ** 31)),
    (hk.ERR_INVALID_ARG, dict(ep=dict(out_type=5))), (hk.ERR_INVALID_ARG, dict(ep=dict(out_type=-1))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(F, activation=4))), (hk.ERR_INVALID_ARG, dict(ep=dict(F, activation=-1))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(F, shift=1))), (hk.ERR_INVALID_ARG, dict(ep=dict(S, hi=1))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(S, activation=1))), (hk.ERR_INVALID_ARG, dict(ep=dict(S, d_bias=BIAS))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(S, d_x_scale=SCALE))), (hk.ERR_INVALID_ARG, dict(ep=dict(C, d_w_scale=SCALE))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(C, d_residual=RES, residual_row_stride=32))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(C, shift=32, hi=1))), (hk.ERR_INVALID_ARG, dict(ep=dict(C, shift=-1, hi=1))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(C, lo=2, hi=1))), (hk.ERR_INVALID_ARG, dict(ep=dict(C, lo=-129))), (hk.ERR_INVALID_ARG, dict(ep=dict(C, hi=256))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(F, d_residual=RES, residual_row_stride=31))),
    # addresses that are not aligned to their elements
    (hk.ERR_INVALID_ARG, dict(out=OUT + 1)), (hk.ERR_INVALID_ARG, dict(out=OUT + 2, ep=S)), (hk.ERR_INVALID_ARG, dict(ep=dict(F, d_x_scale=SCALE + 2))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(F, d_bias=BIAS + 1))), (hk.ERR_INVALID_ARG, dict(ep=dict(F, d_residual=RES + 1, residual_row_stride=32))),
    # outputs that share memory with an input
    (hk.ERR_INVALID_ARG, dict(out=X + 254)), (hk.ERR_INVALID_ARG, dict(out=W + 2)), (hk.ERR_INVALID_ARG, dict(out=X - 254)),
    (hk.ERR_INVALID_ARG, dict(ep=dict(F, d_x_scale=OUT + 4))), (hk.ERR_INVALID_ARG, dict(ep=dict(F, d_bias=OUT))),
    (hk.ERR_INVALID_ARG, dict(ep=dict(F, d_residual=OUT + 2, residual_row_stride=32))),
    (hk.ERR_INVALID_ARG, dict(out_row=40, ep=dict(F, d_residual=OUT, residual_row_stride=32))),
]


@pytest.mark.parametrize("status,change", REFUSED)
def test_refusals(status, change):
    assert call(**change) == status
    assert call(grouped=True, **change) == status


def test_refusals_of_groups():
    assert call(grouped=True, offsets=None) == hk.ERR_INVALID_ARG
    assert call(grouped=True, offsets=OFF + 2) == hk.ERR_INVALID_ARG
    assert call(grouped=True, E=0) == hk.ERR_INVALID_ARG
    assert call(grouped=True, E=hk.MAX_GROUPS + 1) == hk.ERR_UNSUPPORTED
    assert call(grouped=True, offsets=OUT + 8) == hk.ERR_INVALID_ARG
    assert call(grouped=True, E=3, out=W + 3 * 32 * 64 - 2) == hk.ERR_INVALID_ARG


def space(**change):
    a = {**GOOD, **change}
    return hk.lib().hikonv_linear_workspace_bytes(a["x"], a["x_row"], a["w"], a["store"], a.get("E", 0), a["M"], a["N"], a["K"])


def test_workspace():
    # what is aligned needs none, nor do a few rows; else both operands or either, their rows rounded up to 16 bytes
    assert space() == 0 and space(M=100, K=60, x_row=64, E=3) == 3 * 32 * 64
    big = dict(M=100, K=60, x_row=60)
    assert space(**big) == 100 * 64 + 32 * 64
    assert space(M=100, x_row=65) == 100 * 64 and space(M=100, x=X + 1) == 100 * 64 and space(M=100, w=W + 4) == 32 * 64
    assert space(M=100, K=60, x_row=64, store=4) == 32 * 32
    assert space(M=1, K=60) == 0 and space(M=0) == 0 and space(store=3) == 0
    need = space(**big)
    for ptr, size in ((None, 0), (WS, need - 1), (WS + 8, need)):
        assert call(**big, ws_ptr=ptr, ws_bytes=size) == hk.ERR_WORKSPACE
    for ptr in (X + 16, W, OUT):
        assert call(**big, ws_ptr=ptr, ws_bytes=need) == hk.ERR_INVALID_ARG


def test_no_rows_is_fine_without_memory():
    assert call(M=0, x=None, w=None, out=None) == hk.OK
    assert call(grouped=True, M=0, x=None, w=None, out=None, offsets=None) == hk.OK


def quantize(x=X, x_type=hk.OUT_BF16, row=64, M=4, K=64, bits=8, signed=1, codes=OUT, scale=SCALE):
    return hk.lib().hikonv_quantize_rows(x, x_type, row, M, K, bits, signed, codes, scale, None)


@pytest.mark.parametrize("change", [dict(x=None), dict(codes=None), dict(scale=None), dict(x_type=hk.OUT_SUMS), dict(x_type=5), dict(M=-1), dict(K=0),
                                    dict(bits=0), dict(bits=9), dict(bits=1, signed=1), dict(row=-1), dict(row=1 << 50), dict(x=X + 1),
                                    dict(x=X + 2, x_type=hk.OUT_F32), dict(scale=SCALE + 1), dict(codes=X + 500), dict(scale=X), dict(scale=OUT + 128)])
def test_refusals_of_quantize(change):
    assert quantize(**change) == hk.ERR_INVALID_ARG


def test_quantize_of_no_rows():
    assert quantize(M=0, x=None, codes=None, scale=None) == hk.OK


def test_oracle_by_hand():
    x, w = np.array([[1, -2, 3], [0, 4, -1]]), np.array([[2, 1, 0], [-3, 5, 7]])
    s = ol.sums(x, w)
    assert s.tolist() == [[0, 8], [4, 13]]
    assert ol.codes(s, np.array([-1, 4]), 1, -1, 7).tolist() == [[-1, 6], [1, 7]]
    y, bound = ol.floats(s, [0.5, 2.0], [1.0, 0.25], [1.0, -2.0], ol.RELU, np.array([[0.5, 0.0], [0.0, 1.0]]))
    assert y.tolist() == [[1.5, 0.0], [9.0, 5.5]] and (bound < 1e-5).all()
    c, t = ol.quantize(np.array([[1.0, -2.0, 0.5], [0.0, 0.0, 0.0]]), 2, True)
    assert c.tolist() == [[0, -1, 0], [0, 0, 0]] and t.tolist() == [2.0, 0.0]
    c, t = ol.quantize(np.array([[-5.0, 3.0, 1.5]]), 2, False)
    assert c.tolist() == [[0, 3, 2]] and t.tolist() == [1.0]
