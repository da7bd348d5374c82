"""GPU parity of the linear layers on codes: exact sums and codes, float results within the bound of their arithmetic."""
import numpy as np
import pytest
import torch

from gpu_util import assert_exact
from oracle import linear as ol
from paper_2208_00763_b200 import binding as hk
from paper_2208_00763_b200 import inputs

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = [hk.ACT_NONE, hk.ACT_RELU, hk.ACT_SILU, hk.ACT_GELU]


def rows_on_device(values, gap=0, lead=0):
    """Codes one per byte, rows `gap` bytes further apart than they are long, the first `lead` bytes into its buffer."""
    M, K = values.shape
    stored = inputs.to_storage(values)
    buf = torch.full((lead + M * (K + gap) + 64,), 77, dtype=torch.int8, device="cuda")
    view = buf[lead:lead + M * (K + gap)].view(M, K + gap)[:, :K]
    view.copy_(torch.from_numpy(stored).view(M, K))
    return view


def weights_on_device(values, store_bits):
    if store_bits == 8:
        return torch.from_numpy(inputs.to_storage(values)).cuda()
    K = values.shape[-1]
    dense = inputs.to_dense(values, store_bits)
    return torch.from_numpy(dense).view(*values.shape[:-1], K * store_bits // 8).cuda()


def draw(shape_x, shape_w, p, q, xs, ws, seed, kind="uniform"):
    rng = np.random.default_rng(seed)
    if kind == "uniform":
        return inputs.uniform_codes(rng, shape_x, p, xs), inputs.uniform_codes(rng, shape_w, q, ws)
    (xl, xh), (wl, wh) = inputs.code_range(p, xs), inputs.code_range(q, ws)
    pick = {"min": (xl, wl), "max": (xh, wh), "mixed": (xl, wh)}[kind]
    return np.full(shape_x, pick[0], dtype=np.int64), np.full(shape_w, pick[1], dtype=np.int64)


def assert_floats(got, value, bound, what=""):
    """Within the bound of the 32-bit arithmetic and half a step of the output's type (at least half its smallest subnormal)."""
    torch.cuda.synchronize()
    info = torch.finfo(got.dtype)
    half = info.eps / 2
    y = got.detach().cpu().to(torch.float64).numpy()
    over = np.abs(value) + bound >= float(info.max)
    tol = bound + half * (np.abs(value) + bound) + info.smallest_normal * half
    err = np.abs(y - value)
    bad = (err > tol) & ~over
    assert not bad.any() and np.isfinite(y[~over]).all(), "%s: %d values off, worst %.3g of its tolerance, at %s" % (
        what, bad.sum(), np.nanmax(np.where(over, 0, err / tol)), np.argwhere(bad)[:1])


# rows, depth, columns: one of each, sizes below, at and behind the tiles' edges, depths whose rows start anywhere
SIZES = [(1, 1, 1), (1, 16, 7), (2, 33, 3), (3, 17, 130), (5, 64, 128), (8, 512, 64), (16, 128, 256), (17, 130, 129), (31, 96, 40),
         (33, 1000, 65), (48, 272, 200), (64, 128, 128), (65, 384, 300), (100, 4096, 33), (127, 160, 127), (128, 256, 384),
         (129, 1001, 257), (255, 48, 256), (256, 640, 130), (300, 144, 513), (513, 2048, 129)]
CODES = [(8, 8, True, True), (8, 8, False, True), (8, 8, True, False), (8, 8, False, False), (4, 4, True, True), (4, 4, False, True),
         (1, 1, True, True), (7, 3, False, True)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_sums_of_bytes(M, K, N):
    for i, (p, q, xs, ws) in enumerate(CODES):
        x, w = draw((M, K), (N, K), p, q, xs, ws, seed=1000 * i + M + K + N)
        got = hk.linear(rows_on_device(x), weights_on_device(w, 8), p, q, xs, ws)
        assert got.dtype == torch.int32
        assert_exact(got, ol.sums(x, w), "%s" % ((M, K, N, p, q, xs, ws),))


@pytest.mark.parametrize("q", [1, 2, 4])
@pytest.mark.parametrize("ws", [False, True])
def test_sums_of_dense_weights(q, ws):
    for i, (M, K, N) in enumerate(SIZES):
        K = -(-K * q // 8) * 8 // q                      # whole bytes per row
        for p, xs in ((8, True), (8, False), (4, True)):
            x, w = draw((M, K), (N, K), p, q, xs, ws, seed=i)
            got = hk.linear(rows_on_device(x), weights_on_device(w, q), p, q, xs, ws, w_store_bits=q)
            assert_exact(got, ol.sums(x, w), "%s" % ((M, K, N, p, q, xs, ws),))


def test_dense_weights_over_many_stages_and_tiles():
    # long walks through the rings of the unpacking warps: several tiles per CTA, depths that end inside a step, flipped activations
    for M, K, N in ((400, 4128, 256), (2100, 1056, 1300), (200, 6144, 512)):
        for q, xs, ws in ((4, True, True), (4, False, True), (2, True, False), (1, True, True)):
            x, w = draw((M, K), (N, K), 8, q, xs, ws, seed=K)
            got = hk.linear(rows_on_device(x), weights_on_device(w, q), 8, q, xs, ws, w_store_bits=q)
            assert_exact(got, ol.sums(x, w), "%s" % ((M, K, N, q, xs, ws),))


def test_bytes_over_many_tiles():
    # more tiles than SMs, operands of every pair of types, rows that start on 16-byte boundaries and rows that do not
    for M, K, N in ((2100, 272, 1300), (1500, 333, 1700)):
        for xs, ws in ((True, True), (False, True), (True, False), (False, False)):
            x, w = draw((M, K), (N, K), 8, 8, xs, ws, seed=K)
            assert_exact(hk.linear(rows_on_device(x), weights_on_device(w, 8), 8, 8, xs, ws), ol.sums(x, w), "%s" % ((M, K, N, xs, ws),))


@pytest.mark.parametrize("kind", ["min", "max", "mixed"])
def test_extreme_codes_at_the_largest_depth(kind):
    for p, q, xs, ws, store in ((8, 8, True, True, 8), (8, 8, False, True, 8), (8, 8, False, False, 8), (8, 8, True, False, 8), (8, 4, True, True, 4), (8, 1, True, True, 1),
                                (8, 2, False, True, 2), (4, 4, False, False, 4)):
        per = (128 if xs else (1 << p) - 1) * (128 if ws else (1 << q) - 1)
        K = min((2 ** 31 - 1) // per, 140000) // 16 * 16
        for M, N in ((3, 5), (40, 130)):
            x, w = draw((M, K), (N, K), p, q, xs, ws, seed=0, kind=kind)
            got = hk.linear(rows_on_device(x), weights_on_device(w, store), p, q, xs, ws, w_store_bits=store)
            assert_exact(got, ol.sums(x, w), "%s" % ((p, q, xs, ws, store, M),))


def _terms(M, N, out, seed, lead=()):
    rng = np.random.default_rng(seed)
    t = {"x_scale": rng.uniform(0.5, 1.5, M).astype(np.float32) / 64, "w_scale": rng.uniform(0.5, 1.5, lead + (N,)).astype(np.float32) / 128,
         "bias": rng.normal(size=lead + (N,)).astype(np.float32)}
    res = torch.from_numpy(rng.normal(size=(M, N)).astype(np.float32)).to(TYPES[out])
    return t, res


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
def test_float_results(out, act):
    for i, (M, K, N) in enumerate([(1, 64, 40), (4, 100, 33), (16, 256, 128), (20, 128, 131), (70, 512, 260), (200, 96, 129), (257, 160, 48)]):
        for store, p, q, xs in ((8, 8, 8, True), (4, 8, 4, True), (8, 8, 8, False)):
            x, w = draw((M, K), (N, K), p, q, xs, True, seed=i)
            t, res = _terms(M, N, out, i)
            d = {k: torch.from_numpy(v).cuda() for k, v in t.items()}
            s = ol.sums(x, w)
            dx, dw = rows_on_device(x), weights_on_device(w, store)
            # everything, then one term after the other left out
            for left in ((), ("bias",), ("x_scale",), ("w_scale", "bias"), ("residual",), ("x_scale", "w_scale", "bias", "residual")):
                use = {k: v for k, v in d.items() if k not in left}
                ref = {k: v for k, v in t.items() if k not in left}
                r = None if "residual" in left else res
                got = hk.linear(dx, dw, p, q, xs, True, w_store_bits=store, activation=act, residual=None if r is None else r.cuda(),
                                out_dtype=TYPES[out], **use)
                value, bound = ol.floats(s, act=act, residual=None if r is None else r.double().numpy(), **ref)
                assert_floats(got, value, bound, "%s without %s" % ((M, K, N, store, xs), left))


def test_codes():
    for i, (M, K, N) in enumerate([(1, 64, 40), (9, 77, 33), (16, 256, 128), (70, 512, 260), (130, 96, 129)]):
        for p, q, xs, ws, rq, dtype in ((8, 8, True, True, (9, -128, 127), None), (4, 4, False, True, (4, 0, 15), torch.uint8),
                                        (8, 8, False, False, (12, 0, 255), torch.uint8), (8, 4, True, True, (0, -8, 7), torch.int8),
                                        (8, 8, True, True, (31, -1, 0), None)):
            x, w = draw((M, K), (N, K), p, q, xs, ws, seed=i)
            for bias in (None, np.random.default_rng(i).integers(-2 ** 31, 2 ** 31, N), np.random.default_rng(i).integers(-500, 500, N)):
                got = hk.linear(rows_on_device(x), weights_on_device(w, 8), p, q, xs, ws, requant=rq, out_dtype=dtype,
                                bias=None if bias is None else torch.from_numpy(bias.astype(np.int32)).cuda())
                assert got.dtype == (dtype or torch.int8)
                assert_exact(got.view(torch.uint8), ol.codes(ol.sums(x, w), bias, *rq) & 255, "%s" % ((M, K, N, rq),))


@pytest.mark.parametrize("M,K,N", [(1, 100, 50), (6, 256, 140), (40, 130, 129), (150, 512, 200)])
def test_rows_apart(M, K, N):
    x, w = draw((M, K), (N, K), 8, 8, True, True, seed=3)
    t, res = _terms(M, N, "bf16", 4)
    d = {k: torch.from_numpy(v).cuda() for k, v in t.items()}
    value, bound = ol.floats(ol.sums(x, w), residual=res.double().numpy(), **t)
    for gap, lead, out_gap in ((0, 0, 3), (16, 0, 0), (-K % 16, 0, 8), (5, 3, 1), (-K % 16 + 16, 32, 0)):
        buf = torch.full((M + 2, N + out_gap), 7.0, dtype=torch.bfloat16, device="cuda")
        out = buf[1:M + 1, :N]
        got = hk.linear(rows_on_device(x, gap, lead), weights_on_device(w, 8), 8, 8, True, True, residual=res.cuda(), out=out, **d)
        assert got.data_ptr() == out.data_ptr()
        assert_floats(out, value, bound, "gap %d lead %d" % (gap, lead))
        assert (buf[0] == 7).all() and (buf[M + 1] == 7).all() and (buf[:, N:] == 7).all()
        # the residual in place
        out.copy_(res)
        hk.linear(rows_on_device(x, gap, lead), weights_on_device(w, 8), 8, 8, True, True, residual=out, out=out, **d)
        assert_floats(out, value, bound, "in place, gap %d" % gap)
        assert (buf[0] == 7).all() and (buf[M + 1] == 7).all() and (buf[:, N:] == 7).all()


def test_weights_that_start_anywhere():
    M, K, N = 20, 48, 70
    for store, q in ((8, 8), (4, 4)):
        x, w = draw((M, K), (N, K), 8, q, True, True, seed=6)
        dw = weights_on_device(w, store)
        for lead in (1, 4, 8, 15):
            buf = torch.zeros(dw.numel() + 64, dtype=dw.dtype, device="cuda")
            view = buf[lead:lead + dw.numel()].view(dw.shape)
            view.copy_(dw)
            for rows in (M, 2):
                assert_exact(hk.linear(rows_on_device(x[:rows]), view, 8, q, True, True, w_store_bits=store), ol.sums(x[:rows], w), "lead %d" % lead)


def test_given_workspaces():
    x, w = draw((70, 333), (90, 333), 8, 8, True, True, seed=9)
    dx, dw = rows_on_device(x), weights_on_device(w, 8)
    need = hk.linear_workspace_bytes(dx, dw)
    assert need == (70 + 90) * 336
    buf = torch.full((need + 64,), 3, dtype=torch.uint8, device="cuda")
    got = hk.linear(dx, dw, 8, 8, True, True, workspace=buf[32:need + 32])
    assert_exact(got, ol.sums(x, w))
    assert (buf[:32] == 3).all() and (buf[need + 32:] == 3).all()
    with pytest.raises(hk.HikonvError):
        hk.linear(dx, dw, 8, 8, True, True, workspace=buf[:16])
    with pytest.raises(ValueError):
        hk.linear(dx, dw, 8, 8, True, True, workspace=torch.empty(need, dtype=torch.uint8))
    # made by the call, on a stream of the caller's
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [hk.linear(dx, dw, 8, 8, True, True, stream=side) for _ in range(20)]
    torch.cuda.synchronize()
    for y in got:
        assert_exact(y, ol.sums(x, w))


def test_no_rows_and_one_value():
    w = torch.ones((5, 16), dtype=torch.int8, device="cuda")
    out = hk.linear(torch.empty((0, 16), dtype=torch.int8, device="cuda"), w, 8, 8, True, True)
    assert out.shape == (0, 5)
    out = hk.linear(torch.full((1, 1), -7, dtype=torch.int8, device="cuda"), torch.full((1, 1), 9, dtype=torch.int8, device="cuda"), 8, 8, True, True)
    assert out.item() == -63


def test_values_that_are_not_finite():
    # an infinite or undefined scale or bias reaches just its own rows and columns
    M, K, N = 20, 64, 40
    x, w = draw((M, K), (N, K), 8, 8, True, True, seed=8)
    x[4] = 0
    for act in ACTS:
        xs = torch.full((M,), 0.01, device="cuda")
        ws = torch.full((N,), 0.01, device="cuda")
        b = torch.zeros(N, device="cuda")
        xs[3], xs[4], ws[5], b[6] = float("nan"), float("inf"), float("nan"), float("nan")
        got = hk.linear(rows_on_device(x), weights_on_device(w, 8), 8, 8, True, True, x_scale=xs, w_scale=ws, bias=b, activation=act,
                        out_dtype=torch.float32).isnan().cpu()
        want = torch.zeros((M, N), dtype=torch.bool)
        want[3], want[4], want[:, 5], want[:, 6] = True, True, True, True
        assert torch.equal(got, want)


# ------------------------------------------------------------------ groups

def _grouped_reference(x, w, offsets, before, f):
    """f(rows, e) of every group in place of `before`."""
    want = before.copy()
    for e in range(len(offsets) - 1):
        at = slice(offsets[e], offsets[e + 1])
        if offsets[e + 1] > offsets[e]:
            want[at] = f(at, e)
    return want


GROUPS = {"even": [0, 4, 8, 12, 16], "empty ones": [0, 0, 9, 9, 9, 10, 10], "one": [0, 23], "all empty": [0, 0, 0], "lead and tail": [3, 5, 40, 41],
          "large": [0, 1, 130, 300, 301, 600], "many": list(range(0, 130, 2)), "one of many": [0] * 40 + [50] * 25,
          "ragged": [0, 17, 17, 50, 191, 192, 448, 449]}


@pytest.mark.parametrize("name", list(GROUPS))
def test_groups(name):
    offsets = GROUPS[name]
    E, T = len(offsets) - 1, offsets[-1] + 4
    d_off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    for i, (K, N, p, q, xs, store) in enumerate([(64, 130, 8, 8, True, 8), (100, 33, 8, 8, True, 8), (256, 128, 8, 4, True, 4),
                                                 (128, 140, 8, 8, False, 8), (640, 257, 4, 2, False, 2)]):
        x, w = draw((T, K), (E, N, K), p, q, xs, True, seed=i)
        dx, dw = rows_on_device(x), weights_on_device(w, store)
        out = torch.full((T, N), 123456, dtype=torch.int32, device="cuda")
        hk.grouped_linear(dx, dw, d_off, p, q, xs, True, w_store_bits=store, out=out)
        want = _grouped_reference(x, w, offsets, np.full((T, N), 123456, dtype=np.int64), lambda at, e: ol.sums(x[at], w[e]))
        assert_exact(out, want, "%s %s" % (name, (K, N, p, q, xs, store)))
        # floats with every term
        t, res = _terms(T, N, "bf16", i, (E,))
        d = {k: torch.from_numpy(v).cuda() for k, v in t.items()}
        out = res.cuda()
        hk.grouped_linear(dx, dw, d_off, p, q, xs, True, w_store_bits=store, activation=hk.ACT_SILU, residual=out, out=out, **d)
        value, bound = np.zeros((T, N)), np.zeros((T, N))
        for e in range(E):
            at = slice(offsets[e], offsets[e + 1])
            if offsets[e + 1] > offsets[e]:
                value[at], bound[at] = ol.floats(ol.sums(x[at], w[e]), t["x_scale"][at], t["w_scale"][e], t["bias"][e], ol.SILU,
                                                 res[at].double().numpy())
        inside = np.zeros(T, dtype=bool)
        inside[offsets[0]:offsets[-1]] = True
        assert_floats(out[torch.from_numpy(inside).cuda()], value[inside], bound[inside], name)
        assert torch.equal(out.cpu()[~inside], res[~inside])
        # codes
        rq = (7, 0, 15)
        out = torch.full((T, N), 99, dtype=torch.uint8, device="cuda")
        hk.grouped_linear(dx, dw, d_off, p, q, xs, True, w_store_bits=store, requant=rq, out=out)
        want = _grouped_reference(x, w, offsets, np.full((T, N), 99, dtype=np.int64), lambda at, e: ol.codes(ol.sums(x[at], w[e]), None, *rq))
        assert_exact(out, want, name)


def test_the_most_groups():
    E, K, N = hk.MAX_GROUPS, 32, 16
    rng = np.random.default_rng(0)
    offsets = np.concatenate([[0], np.cumsum(rng.integers(0, 3, E))])
    T = int(offsets[-1])
    x, w = draw((T, K), (E, N, K), 4, 4, True, True, seed=1)
    got = hk.grouped_linear(rows_on_device(x), weights_on_device(w, 4), torch.tensor(offsets, dtype=torch.int32, device="cuda"), 4, 4, True,
                            True, w_store_bits=4)
    assert_exact(got, _grouped_reference(x, w, offsets.tolist(), np.zeros((T, N), dtype=np.int64), lambda at, e: ol.sums(x[at], w[e])))


def test_offsets_that_are_wrong_touch_nothing_else():
    # bounds outside the rows are taken as the nearest one, groups that end before they begin as empty
    K, N, T = 64, 70, 30
    x, w = draw((T, K), (4, N, K), 8, 8, True, True, seed=2)
    for offsets, taken in (([-5, 10, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], [(0, 10, 0), (10, 30, 1)]),
                           ([20, 10, 5, 5, -2 ** 31], []), ([-9, -3, 4, 31, 8], [(0, 4, 1), (4, 30, 2)])):
        buf = torch.full((T + 2, N), 5, dtype=torch.int32, device="cuda")
        hk.grouped_linear(rows_on_device(x), weights_on_device(w, 8), torch.tensor(offsets, dtype=torch.int32, device="cuda"), 8, 8, True, True,
                          out=buf[1:T + 1])
        want = np.full((T + 2, N), 5, dtype=np.int64)
        for a, b, e in taken:
            want[a + 1:b + 1] = ol.sums(x[a:b], w[e])
        assert_exact(buf, want, str(offsets))


# ------------------------------------------------------------------ as they are used

@pytest.mark.parametrize("M,store", [(1, 4), (5, 8), (40, 4), (150, 8)])
def test_mlp_block_of_the_calls_together(M, store):
    # floats -> codes -> product with GELU -> codes -> product plus the residual stream; each call against its oracle on what it was given
    H, F = 192, 512
    rng = np.random.default_rng(M)
    q = 4 if store == 4 else 8
    w1, w2 = inputs.uniform_codes(rng, (F, H), q, True), inputs.uniform_codes(rng, (H, F), q, True)
    s1, s2 = (rng.uniform(0.5, 1.5, n).astype(np.float32) / (20 << q) for n in (F, H))
    b1 = rng.normal(size=F).astype(np.float32)
    h = torch.from_numpy(rng.normal(size=(M, H)).astype(np.float32)).to(torch.bfloat16).cuda()
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    c1, t1 = hk.quantize_rows(h, 8)
    u = hk.linear(c1, weights_on_device(w1, store), 8, q, True, True, w_store_bits=store, x_scale=t1, w_scale=dev(s1), bias=dev(b1), activation=hk.ACT_GELU)
    c2, t2 = hk.quantize_rows(u, 8)
    y = hk.linear(c2, weights_on_device(w2, store), 8, q, True, True, w_store_bits=store, x_scale=t2, w_scale=dev(s2), residual=h)
    for floats, got_c, got_t in ((h, c1, t1), (u, c2, t2)):
        want_c, want_t = ol.quantize(floats.double().cpu().numpy(), 8, True)
        assert_exact(got_c, want_c)
        assert np.array_equal(got_t.cpu().numpy(), want_t)
    value, bound = ol.floats(ol.sums(c1.cpu().numpy(), w1), t1.cpu().numpy(), s1, b1, ol.GELU)
    assert_floats(u, value, bound)
    value, bound = ol.floats(ol.sums(c2.cpu().numpy(), w2), t2.cpu().numpy(), s2, residual=h.double().cpu().numpy())
    assert_floats(y, value, bound)


def test_captured_and_replayed_with_other_inputs_and_groups():
    E, K, N, T = 6, 128, 200, 60
    x, w = draw((T, K), (E, N, K), 8, 8, True, True, seed=5)
    dx, dw = rows_on_device(x), weights_on_device(w, 8)
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    out = torch.zeros((T, N), dtype=torch.int32, device="cuda")
    plain = torch.zeros((T, N), dtype=torch.int32, device="cuda")
    hk.grouped_linear(dx, dw, off, 8, 8, True, True, out=out)
    hk.linear(dx, dw[2], 8, 8, True, True, out=plain)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hk.grouped_linear(dx, dw, off, 8, 8, True, True, out=out)
        hk.linear(dx, dw[2], 8, 8, True, True, out=plain)
    for i, offsets in enumerate(([0, 10, 20, 30, 40, 50, 60], [0, 0, 60, 60, 60, 60, 60], [2, 3, 3, 4, 50, 51, 51])):
        x2, _ = draw((T, K), (1, 1, K), 8, 8, True, True, seed=50 + i)
        dx.copy_(torch.from_numpy(inputs.to_storage(x2)))
        off.copy_(torch.tensor(offsets, dtype=torch.int32))
        out.fill_(3)
        graph.replay()
        want = _grouped_reference(x2, w, offsets, np.full((T, N), 3, dtype=np.int64), lambda at, e: ol.sums(x2[at], w[e]))
        assert_exact(out, want, "replay %d" % i)
        assert_exact(plain, ol.sums(x2, w[2]))


def test_two_streams_at_once():
    # calls of several sizes side by side on two streams, again and again, each with its own result
    shapes = [(1, 512, 300), (16, 256, 256), (200, 512, 384), (64, 1024, 512)]
    cases = []
    for i, (M, K, N) in enumerate(shapes):
        x, w = draw((M, K), (N, K), 8, 4, True, True, seed=i)
        cases.append((rows_on_device(x), weights_on_device(w, 4), torch.from_numpy(ol.sums(x, w)).to(torch.int32).cuda()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for rep in range(10):
        for i, (dx, dw, want) in enumerate(cases):
            s = streams[(rep + i) % 2]
            with torch.cuda.stream(s):
                got.append((hk.linear(dx, dw, 8, 4, True, True, w_store_bits=4), want))
            got.append((hk.linear(dx, dw, 8, 4, True, True, w_store_bits=4, stream=streams[rep % 2]), want))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y, want in got)


def test_refusals_of_the_binding():
    x = torch.zeros((4, 16), dtype=torch.int8, device="cuda")
    w = torch.zeros((8, 16), dtype=torch.int8, device="cuda")
    v = torch.ones(8, device="cuda")
    ok = dict(x_scale=torch.ones(4, device="cuda"), w_scale=v)
    hk.linear(x, w, 8, 8, True, True, **ok)
    bad = [dict(x_scale=torch.ones(5, device="cuda")), dict(w_scale=v.double()), dict(w_scale=v.cpu()),
           dict(bias=v.to(torch.int32), x_scale=ok["x_scale"]), dict(requant=(1, 0, 1), x_scale=ok["x_scale"]),
           dict(requant=(1, 0, 1), out_dtype=torch.float16), dict(residual=torch.zeros((4, 8), device="cuda"), out_dtype=torch.bfloat16),
           dict(out=torch.zeros((4, 9), dtype=torch.int32, device="cuda")), dict(out=torch.zeros((8, 4), dtype=torch.int32, device="cuda").t()),
           dict(out_dtype=torch.float64), dict(out_dtype=torch.int64), dict(w_store_bits=4), dict(out=torch.zeros((4, 8), dtype=torch.int32))]
    for kw in bad:
        with pytest.raises(ValueError):
            hk.linear(x, w, 8, 8, True, True, **kw)
    for args, kw in (((x, w, 9, 8, True, True), {}), ((x, w, 8, 8, True, True), dict(activation=1)), ((x, w, 8, 8, True, True), dict(bias=v)),
                     ((x, w, 8, 8, True, True), dict(activation=9, x_scale=ok["x_scale"])), ((x, w, 8, 8, True, True), dict(requant=(32, 0, 1))),
                     ((x, w, 8, 8, True, True), dict(requant=(1, 2, 1)))):
        with pytest.raises(hk.HikonvError):
            hk.linear(*args, **kw)
    for t in (x.cpu(), x.to(torch.int32), x[0], x.t()):
        with pytest.raises(ValueError):
            hk.linear(t, w, 8, 8, True, True)
    with pytest.raises(ValueError):
        hk.linear(x, w[:, :8], 8, 8, True, True)
    w3 = torch.zeros((2, 8, 16), dtype=torch.int8, device="cuda")
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    hk.grouped_linear(x, w3, off, 8, 8, True, True)
    for o in (off.long(), off[:2], off.cpu()):
        with pytest.raises(ValueError):
            hk.grouped_linear(x, w3, o, 8, 8, True, True)
    with pytest.raises(hk.HikonvError):
        hk.grouped_linear(x, w3, None, 8, 8, True, True)
    with pytest.raises(ValueError):
        hk.grouped_linear(x, w, off, 8, 8, True, True)
    # memory shared between the output and an input
    both = torch.zeros(4 * 16 * 4, dtype=torch.int8, device="cuda")
    with pytest.raises(hk.HikonvError):
        hk.linear(both[:64].view(4, 16), w, 8, 8, True, True, out=both[:128].view(torch.int32).view(4, 8))
    line = torch.zeros(64, dtype=torch.float32, device="cuda")
    with pytest.raises(hk.HikonvError):
        hk.linear(x, w, 8, 8, True, True, residual=line[8:40].view(4, 8), out=line[:32].view(4, 8))


def test_no_wait_has_run_out_and_those_that_do_are_counted():
    assert hk.linear_wait_timeouts() == 0                # over all tests of this process so far
    side = torch.cuda.Stream()
    for n in (1, 2):
        for _ in range(n):
            hk.linear_wait_check(2000000, stream=side)
        assert hk.linear_wait_timeouts() == n
        assert hk.linear_wait_timeouts() == 0
    with pytest.raises(hk.HikonvError):
        hk.linear_wait_check(1 << 40)
