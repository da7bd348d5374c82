"""CPU checks of the calls of a mixture of experts: what they refuse, they refuse on the host, before anything is launched; and the
oracle on small cases worked out by hand."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import experts as oe
from paper_2208_00763_b200 import binding as hk
from paper_2208_00763_b200 import build as lib_build


@pytest.fixture(scope="module", autouse=True)
def built_library():
    lib_build.build()
    return hk.lib()


# addresses that no call here may follow, far enough apart that nothing overlaps
A, B, C, D, E, F, G = (0x100000000000 + (i << 40) for i in range(7))

SORT = dict(experts=A, index=4, row=3, T=10, k=3, E=4, offsets=B, slots=C, ws=None, ws_bytes=0)
TO = dict(x=A, size=2, x_row=64, slots=B, T=5, k=3, H=64, out=C, out_row=64, R=15)
FROM = dict(y=A, type=hk.OUT_BF16, y_row=64, R=15, slots=B, weights=C, T=5, k=3, H=64, residual=D, res_row=64, out=E, out_row=64)
GRAD = dict(grad=A, type=hk.OUT_BF16, grad_row=64, y=B, y_row=64, R=15, slots=C, weights=D, T=5, k=3, H=64, grad_y=E, grad_y_row=64, grad_w=F)
QUANT = dict(x=A, type=hk.OUT_BF16, x_row=200, M=5, K=200, f8=0, slots=B, k=3, R=15, values=C, values_row=208, scale=D, scale_row=15)
TILES = dict(w=A, type=hk.OUT_BF16, w_row=200, E=2, N=130, K=200, f8=0, values=B, values_row=208, scale=C)
LINEAR = dict(x=A, xt=0, x_row=208, w=B, wt=0, w_row=208, M=5, N=130, K=200, xs=C, xs_row=5, ws=D, out=E, out_row=136, ep=dict(out_type=hk.OUT_BF16))
GROUPED = dict(x=A, xt=0, x_row=208, w=B, wt=0, w_row=208, off=F, E=3, M=5, N=130, K=200, xs=C, xs_row=5, ws=D, out=E, out_row=136, ep=dict(out_type=hk.OUT_BF16))
CALLS = {"sort": ("hikonv_sort_by_expert", SORT), "to": ("hikonv_rows_to_experts", TO), "from": ("hikonv_rows_from_experts", FROM),
         "grad": ("hikonv_rows_from_experts_grad", GRAD), "quantize": ("hikonv_quantize_blocks", QUANT), "tiles": ("hikonv_quantize_tiles", TILES),
         "linear": ("hikonv_linear_f8", LINEAR), "grouped": ("hikonv_grouped_linear_f8", GROUPED)}


def call(which, **change):
    name, good = CALLS[which]
    a = {**good, **change}
    if "ep" in a:
        a["ep"] = None if a["ep"] is None else ctypes.byref(hk.EpilogueT(**a["ep"]))
    return getattr(hk.lib(), name)(*a.values(), None)


BAD, NOT, SPACE = hk.ERR_INVALID_ARG, hk.ERR_UNSUPPORTED, hk.ERR_WORKSPACE
REFUSED = [
    ("sort", BAD, dict(index=2)), ("sort", BAD, dict(T=-1)), ("sort", BAD, dict(k=0)), ("sort", BAD, dict(E=0)), ("sort", NOT, dict(E=1025)),
    ("sort", NOT, dict(T=1 << 30)), ("sort", BAD, dict(experts=None)), ("sort", BAD, dict(offsets=None)), ("sort", BAD, dict(slots=None)),
    ("sort", BAD, dict(row=-1)), ("sort", BAD, dict(experts=A + 2)), ("sort", BAD, dict(experts=A + 4, index=8)), ("sort", BAD, dict(offsets=B + 1)),
    ("sort", BAD, dict(slots=C + 2)), ("sort", BAD, dict(slots=A + 4)), ("sort", BAD, dict(offsets=A + 116)), ("sort", BAD, dict(offsets=C + 4)),
    ("sort", SPACE, dict(T=5000)), ("sort", SPACE, dict(T=5000, ws=D, ws_bytes=16)), ("sort", BAD, dict(T=5000, ws=C, ws_bytes=1 << 20)),
    ("sort", SPACE, dict(T=5000, ws=D + 2, ws_bytes=1 << 20)), ("sort", BAD, dict(T=5000, ws=A + 59996, ws_bytes=1 << 20)),
    ("to", BAD, dict(size=3)), ("to", BAD, dict(size=8)), ("to", BAD, dict(T=-1)), ("to", BAD, dict(k=0)), ("to", BAD, dict(H=0)), ("to", BAD, dict(R=-1)),
    ("to", NOT, dict(H=(1 << 23) + 1, x_row=1 << 24, out_row=1 << 24)), ("to", NOT, dict(T=1 << 29)), ("to", BAD, dict(x=None)), ("to", BAD, dict(slots=None)),
    ("to", BAD, dict(out=None)), ("to", BAD, dict(x_row=-1)), ("to", BAD, dict(out_row=63)), ("to", BAD, dict(out_row=1 << 50)), ("to", BAD, dict(x=A + 1)),
    ("to", BAD, dict(out=C + 1)), ("to", BAD, dict(slots=B + 2)), ("to", BAD, dict(out=A + 638)), ("to", BAD, dict(slots=C)),
    ("from", BAD, dict(type=hk.OUT_SUMS)), ("from", BAD, dict(type=hk.OUT_CODES)), ("from", BAD, dict(type=7)), ("from", BAD, dict(T=-1)), ("from", BAD, dict(k=0)),
    ("from", BAD, dict(H=0)), ("from", BAD, dict(R=-1)), ("from", NOT, dict(H=(1 << 23) + 1)), ("from", BAD, dict(y=None)), ("from", BAD, dict(slots=None)),
    ("from", BAD, dict(out=None)), ("from", BAD, dict(y_row=-2)), ("from", BAD, dict(out_row=63)), ("from", BAD, dict(res_row=63)), ("from", BAD, dict(y=A + 1)),
    ("from", BAD, dict(out=E + 1)), ("from", BAD, dict(residual=D + 1)), ("from", BAD, dict(weights=C + 2)), ("from", BAD, dict(out=A)), ("from", BAD, dict(out=B + 4)),
    ("from", BAD, dict(out=C + 8)), ("from", BAD, dict(residual=E + 2)), ("from", BAD, dict(residual=E, res_row=72)),
    ("grad", BAD, dict(type=hk.OUT_SUMS)), ("grad", BAD, dict(weights=None)), ("grad", BAD, dict(grad_w=None)), ("grad", BAD, dict(grad=None)),
    ("grad", BAD, dict(y=None)), ("grad", BAD, dict(slots=None)), ("grad", BAD, dict(grad_y=None)), ("grad", BAD, dict(grad_y_row=63)),
    ("grad", BAD, dict(grad_row=-1)), ("grad", BAD, dict(y_row=-1)), ("grad", BAD, dict(k=0)), ("grad", NOT, dict(H=(1 << 23) + 1)), ("grad", BAD, dict(grad_y=A + 2)),
    ("grad", BAD, dict(grad_y=B)), ("grad", BAD, dict(grad_y=C)), ("grad", BAD, dict(grad_w=D)), ("grad", BAD, dict(grad_w=E)), ("grad", BAD, dict(grad_w=C + 56)),
    ("grad", BAD, dict(grad_w=A)), ("grad", BAD, dict(grad_w=B)), ("grad", BAD, dict(grad_w=F + 2)),
    ("quantize", BAD, dict(type=hk.OUT_SUMS)), ("quantize", BAD, dict(f8=2)), ("quantize", BAD, dict(M=-1)), ("quantize", BAD, dict(K=0)), ("quantize", BAD, dict(k=0)),
    ("quantize", BAD, dict(slots=None)), ("quantize", BAD, dict(x=None)), ("quantize", BAD, dict(values=None)), ("quantize", BAD, dict(scale=None)),
    ("quantize", BAD, dict(x_row=-1)), ("quantize", BAD, dict(values_row=192)), ("quantize", NOT, dict(values_row=204)), ("quantize", NOT, dict(values=C + 8)),
    ("quantize", BAD, dict(scale_row=14)), ("quantize", BAD, dict(x=A + 1)), ("quantize", BAD, dict(scale=D + 2)), ("quantize", BAD, dict(slots=B + 1)),
    ("quantize", BAD, dict(values=A)), ("quantize", BAD, dict(scale=A)), ("quantize", BAD, dict(scale=C)), ("quantize", BAD, dict(slots=C + 16)),
    ("quantize", BAD, dict(slots=D)), ("quantize", NOT, dict(K=(1 << 26) + 1)), ("quantize", NOT, dict(M=1 << 29)),
    ("tiles", BAD, dict(type=0)), ("tiles", BAD, dict(f8=-1)), ("tiles", BAD, dict(E=0)), ("tiles", BAD, dict(N=0)), ("tiles", BAD, dict(K=0)), ("tiles", BAD, dict(w=None)),
    ("tiles", BAD, dict(values=None)), ("tiles", BAD, dict(scale=None)), ("tiles", NOT, dict(values_row=201)), ("tiles", NOT, dict(values=B + 4)),
    ("tiles", BAD, dict(values=A)), ("tiles", BAD, dict(scale=A)), ("tiles", BAD, dict(scale=B)), ("tiles", NOT, dict(E=1 << 20, N=1 << 12)),
]
for which in ("linear", "grouped"):
    REFUSED += [(which, s, c) for s, c in [
        (BAD, dict(ep=None)), (BAD, dict(M=-1)), (BAD, dict(N=0)), (BAD, dict(K=0)), (BAD, dict(xt=2)), (BAD, dict(wt=-1)), (BAD, dict(ep=dict(out_type=hk.OUT_SUMS))),
        (BAD, dict(ep=dict(out_type=hk.OUT_CODES))), (BAD, dict(ep=dict(out_type=hk.OUT_F32, activation=4))), (BAD, dict(ep=dict(out_type=hk.OUT_F32, d_x_scale=C))),
        (BAD, dict(ep=dict(out_type=hk.OUT_F32, d_w_scale=C))), (BAD, dict(ep=dict(out_type=hk.OUT_F32, shift=1))), (NOT, dict(M=(1 << 30) + 1)),
        (BAD, dict(x=None)), (BAD, dict(w=None)), (BAD, dict(xs=None)), (BAD, dict(ws=None)), (BAD, dict(out=None)), (BAD, dict(x_row=192)), (BAD, dict(w_row=192)),
        (BAD, dict(xs_row=4)), (BAD, dict(out_row=129)), (NOT, dict(x_row=200)), (NOT, dict(w_row=200)), (NOT, dict(x=A + 8)), (NOT, dict(w=B + 1)),
        (BAD, dict(out=E + 1)), (BAD, dict(xs=C + 2)), (BAD, dict(ws=D + 1)), (BAD, dict(ep=dict(out_type=hk.OUT_BF16, d_bias=F + 2))), (BAD, dict(out=A)),
        (BAD, dict(out=B)), (BAD, dict(out=C)), (BAD, dict(out=D)), (BAD, dict(ep=dict(out_type=hk.OUT_BF16, d_bias=E + 4))),
        (BAD, dict(ep=dict(out_type=hk.OUT_BF16, d_residual=E + 2, residual_row_stride=136))),
        (BAD, dict(ep=dict(out_type=hk.OUT_BF16, d_residual=E, residual_row_stride=144))), (BAD, dict(ep=dict(out_type=hk.OUT_BF16, d_residual=G, residual_row_stride=129))),
        (BAD, dict(out_row=1 << 45)), (BAD, dict(x_row=1 << 45))]]
REFUSED += [("grouped", BAD, dict(off=None)), ("grouped", BAD, dict(E=0)), ("grouped", NOT, dict(E=1025)), ("grouped", BAD, dict(off=F + 2)),
            ("grouped", BAD, dict(off=E + 4)), ("grouped", NOT, dict(E=1024, N=1 << 22, out_row=1 << 22))]


@pytest.mark.parametrize("which,status,change", REFUSED)
def test_refusals(which, status, change):
    assert call(which, **change) == status


NOTHING = [("to", dict(T=0)), ("to", dict(R=0)), ("from", dict(T=0)), ("grad", dict(T=0)), ("quantize", dict(M=0)), ("quantize", dict(R=0)),
           ("linear", dict(M=0)), ("grouped", dict(M=0))]


@pytest.mark.parametrize("which,change", NOTHING)
def test_nothing_to_do(which, change):
    assert call(which, **change) == hk.OK


@pytest.mark.parametrize("which", ["to", "from", "grad", "quantize", "tiles", "linear", "grouped"])
@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not to be followed")
def test_good_calls_reach_the_launch(which):
    assert call(which) == hk.ERR_CUDA


# outputs that may lie between the rows of another matrix
@pytest.mark.parametrize("which,change", [("from", dict(residual=E + 128, res_row=128, out_row=128)), ("from", dict(residual=E, res_row=64)),
                                          ("to", dict(x=C + 128, x_row=128, out_row=128)),
                                          ("linear", dict(out_row=272, ep=dict(out_type=hk.OUT_BF16, d_residual=E + 272, residual_row_stride=272)))])
@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not to be followed")
def test_columns_of_one_buffer_are_taken(which, change):
    assert call(which, **change) == hk.ERR_CUDA


def test_workspace_of_the_sort():
    assert hk.sort_by_expert_workspace_bytes(512, 8, 64) == 0
    assert hk.sort_by_expert_workspace_bytes(513, 8, 64) == 3 * 65 * 4
    assert hk.sort_by_expert_workspace_bytes(1 << 27, 8, 1024) == 128 * 1025 * 4
    assert hk.sort_by_expert_workspace_bytes(32768, 8, 256) == 128 * 257 * 4
    assert hk.sort_by_expert_workspace_bytes(0, 8, 64) == 0


def test_cpu_tensors_are_refused():
    x, slots = torch.zeros(2, 8), torch.zeros(2, 1, dtype=torch.int32)
    f8, one = torch.zeros(2, 16, dtype=torch.float8_e4m3fn), torch.zeros(1, 2)
    for f in (lambda: hk.sort_by_expert(slots, 4), lambda: hk.rows_to_experts(x, slots), lambda: hk.rows_from_experts(x, slots),
              lambda: hk.rows_from_experts_grad(x, None, slots), lambda: hk.quantize_blocks(x), lambda: hk.quantize_tiles(x),
              lambda: hk.linear_f8(f8, f8, one, torch.zeros(1, 1)), lambda: hk.grouped_linear_f8(f8, f8[None], slots[0], one, torch.zeros(1, 1, 1))):
        with pytest.raises(ValueError):
            f()


# ---- the oracle

def test_oracle_sort_by_hand():
    offsets, slots = oe.sort([[2, 0], [-1, 2], [0, 0], [9, 1]], 3)
    assert offsets.tolist() == [0, 3, 4, 6]
    assert slots.tolist() == [[4, 0], [-2 - 6, 5], [1, 2], [-2 - 7, 3]]


@pytest.mark.parametrize("exponent,dtype", [(4, torch.float8_e4m3fn), (5, torch.float8_e5m2)])
def test_oracle_f8_numbers_are_torchs(exponent, dtype):
    table = torch.arange(256, dtype=torch.uint8).view(dtype).double().numpy()
    assert np.array_equal(oe.f8_table(exponent), table, equal_nan=True)
    g = np.random.default_rng(1)
    v = np.concatenate([g.normal(size=4000) * oe.MOST[exponent] / 4, table[np.isfinite(table)], g.normal(size=2000) * 2.0 ** -6, [0.0, -0.0, np.nan]])
    finite = np.sort(table[np.isfinite(table)])
    v = np.concatenate([v, (finite[1:] + finite[:-1]) / 2]).astype(np.float32).astype(np.float64)
    v = v.clip(-oe.MOST[exponent], oe.MOST[exponent])
    want = torch.from_numpy(v).float().to(dtype).view(torch.uint8).numpy()
    got = oe.f8_round(v, exponent)
    nan = np.isnan(v)
    assert np.array_equal(got[~nan], want[~nan]) and np.isnan(oe.f8_table(exponent)[got[nan]]).all()


def test_oracle_blocks_by_hand():
    x = np.zeros((2, 130))
    x[0, 0], x[0, 1], x[0, 129], x[1, 5] = 896.0, -3.0, 7.0, -448.0
    codes, scale = oe.quantize_blocks(x, 4)
    assert scale.shape == (2, 2) and scale.tolist() == [[2.0, 1.0], [7.0 / 448, 0.0]]
    v = oe.f8_table(4)[codes]
    assert (v[0, 0], v[0, 1], v[0, 129], v[1, 5], v[1, 129]) == (448.0, -1.5, 448.0, -448.0, 0.0)


def test_oracle_gradient_by_differences():
    g = np.random.default_rng(0)
    _, slots = oe.sort(g.integers(-1, 3, (5, 2)), 3)
    y, w, up = g.normal(size=(10, 4)), g.normal(size=(5, 2)), g.normal(size=(5, 4))
    gy, gw = oe.rows_from_grad(up, y, slots, w, np.full((10, 4), 9.0))
    loss = lambda yy, ww: (oe.rows_from(yy, slots, ww) * up).sum()  # noqa: E731  (linear in each: differences are exact up to rounding)
    for i in np.ndindex(y.shape):
        d = np.zeros_like(y)
        d[i] = 1.0
        assert abs(loss(y + d, w) - loss(y, w) - gy[i]) < 1e-12
    for i in np.ndindex(w.shape):
        d = np.zeros_like(w)
        d[i] = 1.0
        assert abs(loss(y, w + d) - loss(y, w) - gw[i]) < 1e-12
