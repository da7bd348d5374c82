"""GPU parity of a mixture of experts: sorting, rows to experts and back with gradients, blocks of 8-bit floating point numbers, against
the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import experts as oe
from paper_2208_00763_b200 import binding as hk

pytestmark = pytest.mark.gpu

FLOATS = [torch.float32, torch.float16, torch.bfloat16]
F8 = {torch.float8_e4m3fn: 4, torch.float8_e5m2: 5}


def route(T, k, E, seed, dropped=0.1):
    g = np.random.default_rng(seed)
    experts = g.integers(0, E, (T, k))
    return np.where(g.random((T, k)) < dropped, g.choice([-1, E, -7, 2 ** 31 - 1], (T, k)), experts)


def places(T, k, E, seed, dropped=0.1):
    offsets, slots = oe.sort(route(T, k, E, seed, dropped), E)
    return offsets, slots, torch.tensor(slots, dtype=torch.int32, device="cuda").reshape(T, k)


def wide(t, extra, offset=0):
    """The same values with rows that lie apart."""
    buf = torch.full((t.shape[0], t.shape[1] + extra + offset), 7, dtype=torch.float32, device=t.device).to(t.dtype)
    view = buf[:, offset:offset + t.shape[1]]
    view.copy_(t)
    return view


def f64(t):
    return t.double().cpu().numpy()


# ---- sorting

def check_sort(experts, E, dtype=torch.int32, **kw):
    offsets, slots = hk.sort_by_expert(torch.tensor(experts, dtype=dtype, device="cuda"), E, **kw)
    want_offsets, want_slots = oe.sort(experts, E)
    assert offsets.dtype == slots.dtype == torch.int32
    assert np.array_equal(offsets.cpu().numpy(), want_offsets) and np.array_equal(slots.cpu().numpy(), want_slots)


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 64), (3, 2, 5), (31, 1, 4), (64, 8, 64), (100, 7, 33), (512, 8, 256), (4096, 1, 1024), (4097, 1, 16),
                                   (513, 8, 1024), (1000, 6, 511), (1024, 8, 300), (1025, 8, 300), (8193, 1, 1024), (9000, 3, 1024), (2048, 8, 512), (20000, 8, 256), (70001, 8, 20)])
def test_sort(T, k, E, dtype):
    check_sort(route(T, k, E, T + E), E, dtype)


@pytest.mark.parametrize("T", [1, 33, 4096, 9000])
@pytest.mark.parametrize("what", ["one", "none", "last", "runs"])
def test_sort_of_lopsided_choices(T, what):
    experts = {"one": np.full((T, 2), 3), "none": np.full((T, 2), -1), "last": np.full((T, 2), 7), "runs": np.arange(2 * T).reshape(T, 2) * 8 // (2 * T)}[what]
    check_sort(experts, 8)


def test_sort_of_nothing():
    offsets, slots = hk.sort_by_expert(torch.empty(0, 4, dtype=torch.int64, device="cuda"), 5, offsets=torch.full((6,), 9, dtype=torch.int32, device="cuda"))
    assert offsets.tolist() == [0] * 6 and slots.shape == (0, 4)


def test_sort_of_far_indices():
    experts = torch.tensor([[2 ** 32 + 1, 1], [-(2 ** 40), 2 ** 31], [0, 1 - 2 ** 32]], device="cuda")
    offsets, slots = hk.sort_by_expert(experts, 3)
    assert offsets.tolist() == [0, 1, 2, 2] and slots.tolist() == [[-4, 1], [-5, -6], [0, -7]]


@pytest.mark.parametrize("T", [40, 6000])
def test_sort_of_columns_of_a_wider_matrix(T):
    experts = route(T, 9, 16, 3)
    e = torch.tensor(experts, device="cuda")[:, 2:5]
    offsets, slots = hk.sort_by_expert(e, 16)
    want = oe.sort(experts[:, 2:5], 16)
    assert np.array_equal(offsets.cpu().numpy(), want[0]) and np.array_equal(slots.cpu().numpy(), want[1])
    one = torch.tensor(experts[:1], device="cuda").expand(T, 9)             # every token chooses the same
    assert np.array_equal(hk.sort_by_expert(one, 16)[1].cpu().numpy(), oe.sort(np.repeat(experts[:1], T, 0), 16)[1])


def test_sort_of_many_blocks_per_cta():
    T = 200000                                           # two blocks a CTA
    check_sort(route(T, 8, 77, 5), 77, torch.int32)


# ---- rows

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("T,k,H", [(1, 1, 1), (3, 2, 5), (5, 3, 64), (7, 8, 129), (33, 2, 1003), (2, 5, 4096), (300, 1, 16), (4, 2, 70001)])
def test_rows_to(T, k, H, dtype):
    _, slots, d_slots = places(T, k, 6, T + H)
    x = torch.randint(0, 100, (T, H), device="cuda").to(torch.float32).to(dtype)
    before = torch.randint(0, 100, (T * k, H), device="cuda").to(torch.float32).to(dtype)
    want = oe.rows_to(f64(x.float()), slots, f64(before.float()))
    out = before.clone()
    assert hk.rows_to_experts(x, d_slots, out=out) is out
    assert np.array_equal(f64(out.float()), want)
    # rows that lie apart, at any address
    apart = wide(before, 3, 1)
    hk.rows_to_experts(wide(x, 5), d_slots, out=apart)
    assert np.array_equal(f64(apart.float()), want)
    fresh = hk.rows_to_experts(x, d_slots)
    named = slots[slots >= 0]
    assert fresh.shape == (T * k, H) and np.array_equal(f64(fresh.float())[named], want[named])


def test_rows_to_a_longer_and_a_shorter_matrix():
    _, slots, d_slots = places(6, 2, 3, 0)
    x = torch.arange(48, dtype=torch.float32, device="cuda").reshape(6, 8)
    for rows in (20, 5):
        out = torch.full((rows, 8), -1.0, device="cuda")
        hk.rows_to_experts(x, d_slots, out=out)
        assert np.array_equal(f64(out), oe.rows_to(f64(x), slots, np.full((rows, 8), -1.0)))
    same = hk.rows_to_experts(x[:1].expand(6, 8), d_slots, out=torch.zeros(12, 8, device="cuda"))
    assert np.array_equal(f64(same), oe.rows_to(np.repeat(f64(x)[:1], 6, 0), slots, np.zeros((12, 8))))


def sums_are_near(got, terms, want):
    """k + 1 additions and products of 32 bits, half a step each of what has been added up, and one rounding."""
    eps = torch.finfo(got.dtype).eps
    n = terms.shape[0] + 2
    bound = n * 2.0 ** -24 * np.abs(terms).sum(0) + (eps / 2) * np.abs(want) * (1 + n * 2.0 ** -24) + float(torch.finfo(got.dtype).smallest_normal) * eps
    assert (np.abs(f64(got) - want) <= bound).all(), np.abs(f64(got) - want).max()


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("T,k,H", [(1, 1, 1), (3, 2, 5), (5, 3, 64), (7, 8, 129), (33, 9, 1003), (2, 5, 4096), (300, 1, 16), (2, 2, 70001)])
def test_rows_from(T, k, H, dtype):
    _, slots, d_slots = places(T, k, 6, T + H, 0.3)
    g = torch.Generator("cuda").manual_seed(H)
    y = torch.randn(T * k, H, generator=g, device="cuda").to(dtype)
    w = torch.rand(T, k, generator=g, device="cuda") * 2 - 0.5
    r = torch.randn(T, H, generator=g, device="cuda").to(dtype)
    w[d_slots < 0] = float("nan")                          # counts for nothing
    y[-1] = y[-1] if slots.max() == T * k - 1 else float("nan")
    for weights in (w, None):
        for residual in (r, None):
            want = oe.rows_from(f64(y), slots, None if weights is None else f64(w), None if residual is None else f64(r))
            terms = [np.abs(f64(r))] if residual is not None else []
            for j in range(k):
                one = slots[:, j:j + 1]
                terms.append(np.abs(oe.rows_from(f64(y), one, None if weights is None else f64(w)[:, j:j + 1])))
            terms = np.stack(terms)
            sums_are_near(hk.rows_from_experts(y, d_slots, weights, residual), terms, want)
            out = wide(torch.zeros_like(r), 3, 1)
            hk.rows_from_experts(wide(y, 1), d_slots, weights, None if residual is None else wide(r, 2), out=out)
            sums_are_near(out, terms, want)
            if residual is not None:
                both = r.clone()
                assert hk.rows_from_experts(y, d_slots, weights, both, out=both) is both
                sums_are_near(both, terms, want)


def test_rows_from_keeps_to_the_rows_there_are():
    _, slots, d_slots = places(6, 2, 3, 0)
    y = torch.randn(5, 8, device="cuda")
    want = oe.rows_from(f64(y), slots)
    assert np.allclose(f64(hk.rows_from_experts(y, d_slots)), want, atol=1e-6)
    assert not hk.rows_from_experts(y[:0], d_slots).any()
    assert hk.rows_from_experts(y, d_slots[:0]).shape == (0, 8)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("T,k,H", [(1, 1, 1), (3, 2, 5), (5, 3, 64), (7, 8, 129), (33, 9, 1003), (2, 5, 4096), (300, 1, 16), (40, 17, 72)])
def test_rows_from_grad(T, k, H, dtype):
    _, slots, d_slots = places(T, k, 6, T + H, 0.3)
    g = torch.Generator("cuda").manual_seed(H)
    grad = torch.randn(T, H, generator=g, device="cuda").to(dtype)
    y = torch.randn(T * k, H, generator=g, device="cuda").to(dtype)
    w = torch.rand(T, k, generator=g, device="cuda") * 2 - 0.5
    for weights in (w, None):
        want_y, want_w = oe.rows_from_grad(f64(grad), f64(y), slots, None if weights is None else f64(w), np.full((T * k, H), np.nan))
        eps = torch.finfo(dtype).eps
        mass = np.abs(f64(grad)) @ np.abs(f64(y)).T
        mass = np.where((slots >= 0), np.take_along_axis(mass, slots.clip(min=0), 1), 0.0)

        def check(got_y, got_w):
            # one product of 32 bits, one rounding
            assert (np.abs(f64(got_y) - want_y) <= (eps / 2 + 2.0 ** -24) * np.abs(want_y) * (1 + eps) + float(torch.finfo(dtype).smallest_normal) * eps).all()
            if weights is None:
                assert got_w is None
            else:
                # H products, added in any order: half a step of all for each
                assert (np.abs(f64(got_w) - want_w) <= H * 2.0 ** -24 * mass).all()

        check(*hk.rows_from_experts_grad(grad, y, d_slots, weights))
        gy, gw = wide(torch.full_like(y, float("nan")), 3, 1), torch.full_like(w, float("nan"))
        got = hk.rows_from_experts_grad(wide(grad, 1), None if weights is None else wide(y, 2), d_slots, weights, grad_y=gy,
                                        grad_weights=None if weights is None else gw)
        assert got[0] is gy
        check(*got)
        if k * T > 2 and weights is not None:
            again = hk.rows_from_experts_grad(grad, y, d_slots, weights)
            assert torch.equal(again[1], hk.rows_from_experts_grad(grad, y, d_slots, weights)[1])


def test_rows_to_and_from_are_each_others_gradient():
    # <rows_to(x), u> = <x, rows_from(u)> in whole numbers
    _, slots, d_slots = places(50, 3, 7, 1)
    x, u = (torch.randint(-8, 9, (n, 24), device="cuda").float() for n in (50, 150))
    y = hk.rows_to_experts(x, d_slots, out=torch.zeros(150, 24, device="cuda"))
    assert (y * u).sum().item() == (x * hk.rows_from_experts(u, d_slots)).sum().item()


# ---- blocks of 8-bit floating point numbers

def same_f8(got, want, exponent):
    got = got.view(torch.uint8).cpu().numpy()
    table = oe.f8_table(exponent)
    assert got.shape == want.shape
    bad = (got != want) & ~(np.isnan(table[got]) & np.isnan(table[want]))
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


def hidden(M, K, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(M, K, generator=g, device="cuda") * (torch.rand(M, 1, generator=g, device="cuda") * 8 + 0.01)).to(dtype)


@pytest.mark.parametrize("f8", list(F8))
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("M,K", [(1, 1), (1, 128), (3, 127), (5, 129), (2, 4096), (33, 520), (7, 1003), (130, 256), (2, 20001)])
def test_quantize_blocks(M, K, dtype, f8):
    x = hidden(M, K, dtype, M + K)
    want, want_scale = oe.quantize_blocks(f64(x), F8[f8])
    values, scale = hk.quantize_blocks(x, f8)
    assert values.dtype == f8 and values.stride(0) % 16 == 0 or M == 1
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    same_f8(values, want, F8[f8])
    values, scale = hk.quantize_blocks(wide(x, 3, 1), f8)
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    same_f8(values, want, F8[f8])


@pytest.mark.parametrize("f8", list(F8))
@pytest.mark.parametrize("T,k,K", [(1, 1, 5), (3, 2, 128), (40, 3, 300), (9, 8, 4096)])
def test_quantize_blocks_to_experts(T, k, K, f8):
    _, slots, d_slots = places(T, k, 5, T + K, 0.3)
    x = hidden(T, K, torch.bfloat16, K)
    codes, one = oe.quantize_blocks(f64(x), F8[f8])
    R = T * k + 2
    buf = torch.full((R, (K + 15) // 16 * 16 + 16), 0x33, dtype=torch.uint8, device="cuda")
    values, scale = buf.view(f8)[:, :K], torch.full((-(-K // 128), R + 5), -1.0, device="cuda")[:, :R]
    got = hk.quantize_blocks(x, f8, d_slots, values, scale)
    assert got[0] is values and got[1] is scale
    assert np.array_equal(values.view(torch.uint8).cpu().numpy(), oe.rows_to(codes, slots, np.full((R, K), 0x33, np.uint8)))
    assert np.array_equal(scale.cpu().numpy().T, oe.rows_to(one.T, slots, np.full((R, one.shape[0]), -1.0, np.float32)))
    assert (buf[:, K:] == 0x33).all()                      # behind a row's end
    fresh, fresh_scale = hk.quantize_blocks(x, f8, d_slots)
    named = torch.tensor(slots[slots >= 0], device="cuda")
    assert torch.equal(fresh.view(torch.uint8)[named], values.view(torch.uint8)[named]) and torch.equal(fresh_scale[:, named], scale[:, named])


@pytest.mark.parametrize("f8", list(F8))
@pytest.mark.parametrize("dtype", FLOATS)
def test_quantize_blocks_of_special_values(dtype, f8):
    most = oe.MOST[F8[f8]]
    finite = oe.f8_table(F8[f8])
    finite = np.sort(finite[np.isfinite(finite)])
    x = torch.zeros(10, 256, dtype=torch.float64)
    x[1, 5] = -3.0
    x[2] = torch.finfo(dtype).tiny * 0.25 * (torch.arange(256) % 5)          # subnormal
    x[3] = torch.finfo(dtype).max * ((torch.arange(256) % 3) - 1)
    x[4, :128] = torch.arange(128) - 64
    ties = (finite[1:] + finite[:-1]) / 2                                     # a scale of one: quotients are the values themselves
    x[5, 1:128], x[5, 0] = torch.tensor(ties[:127]), most
    x[6, 1:128], x[6, 0] = torch.tensor(ties[-127:]), -most
    x[7, 0], x[7, 1] = most, most * 2.0 ** -20
    x[8] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps        # the smallest subnormal
    x[9] = -0.0
    x = x.to(dtype)
    want, want_scale = oe.quantize_blocks(f64(x), F8[f8])
    values, scale = hk.quantize_blocks(x.cuda(), f8)
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    got = values.view(torch.uint8).cpu().numpy()
    zero = (want & 127) == 0
    assert np.array_equal(got[~zero], want[~zero]) and ((got[zero] & 127) == 0).all()


@pytest.mark.parametrize("f8", list(F8))
def test_quantize_blocks_of_infinities_and_nan(f8):
    x = torch.ones(3, 384, device="cuda")
    x[0, 3], x[1, 130] = float("nan"), float("-inf")
    values, scale = hk.quantize_blocks(x, f8)
    v, s = values.float(), scale.T
    assert torch.isnan(s[0, 0]) and torch.isnan(v[0, :128]).all() and torch.isfinite(s[0, 1:]).all() and torch.isfinite(v[0, 128:]).all()
    assert torch.isinf(s[1, 1]) and torch.isnan(v[1, 130]) and (v[1, 131:256] == 0).all() and torch.isfinite(s[1, [0, 2]]).all()
    assert torch.isfinite(v[2]).all() and torch.isnan(v[1, 128:256] * s[1, 1]).all()


@pytest.mark.parametrize("f8", list(F8))
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("shape", [(1, 1), (3, 130), (128, 128), (129, 257), (2, 200, 300), (3, 128, 64)])
def test_quantize_tiles(shape, dtype, f8):
    w = hidden(int(np.prod(shape[:-1])), shape[-1], dtype, shape[-1]).reshape(shape)
    values, scale = hk.quantize_tiles(w, f8)
    for e, one in enumerate(w if w.dim() == 3 else [w]):
        want, want_scale = oe.quantize_tiles(f64(one), F8[f8])
        same_f8(values[e] if w.dim() == 3 else values, want, F8[f8])
        assert np.array_equal((scale[e] if w.dim() == 3 else scale).cpu().numpy(), want_scale)


def test_shapes_that_do_not_fit_are_refused():
    x, f8 = torch.zeros(4, 32, device="cuda"), torch.zeros(4, 32, dtype=torch.float8_e4m3fn, device="cuda")
    slots = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    for f in (lambda: hk.sort_by_expert(x, 4), lambda: hk.sort_by_expert(slots, 4, offsets=slots[0]), lambda: hk.rows_to_experts(x, slots[:3]),
              lambda: hk.rows_to_experts(x, slots.long()), lambda: hk.rows_to_experts(x.double(), slots), lambda: hk.rows_to_experts(x, slots, out=x.half()),
              lambda: hk.rows_to_experts(x, slots, out=torch.zeros(8, 31, device="cuda")), lambda: hk.rows_to_experts(x.t(), slots),
              lambda: hk.rows_from_experts(x.double(), slots), lambda: hk.rows_from_experts(x, slots, torch.ones(4, 1, device="cuda")),
              lambda: hk.rows_from_experts(x, slots, torch.ones(4, 2, device="cuda").half()), lambda: hk.rows_from_experts(x, slots, residual=x[:3]),
              lambda: hk.rows_from_experts(x, slots, residual=x.half()), lambda: hk.rows_from_experts(x, slots.cpu()),
              lambda: hk.rows_from_experts_grad(x, None, slots, torch.ones(4, 2, device="cuda")), lambda: hk.rows_from_experts_grad(x, x.half(), slots, torch.ones(4, 2, device="cuda")),
              lambda: hk.rows_from_experts_grad(x, x, slots, None, grad_weights=torch.ones(4, 2, device="cuda")), lambda: hk.rows_from_experts_grad(x[:3], x, slots),
              lambda: hk.quantize_blocks(x.double()), lambda: hk.quantize_blocks(x, torch.float16), lambda: hk.quantize_blocks(x, values=f8[:3]),
              lambda: hk.quantize_blocks(x, scale=torch.ones(4, 1, device="cuda")), lambda: hk.quantize_blocks(x, slots=slots[:3]),
              lambda: hk.quantize_tiles(x[0]), lambda: hk.quantize_tiles(x, scale=torch.ones(1, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(hk.HikonvError):
        hk.quantize_blocks(x[:, :20], values=torch.zeros(4, 20, dtype=torch.float8_e4m3fn, device="cuda"))
    with pytest.raises(hk.HikonvError):
        hk.rows_to_experts(x, slots, out=x)


def test_in_a_graph_replayed_with_other_choices():
    T, k, E, H = 900, 8, 16, 72                            # two launches of the sort
    experts = torch.randint(-1, E, (T, k), device="cuda")
    x, grad = torch.randn(T, H, device="cuda"), torch.randn(T, H, device="cuda")
    w = torch.rand(T, k, device="cuda")

    def step():
        offsets, slots = hk.sort_by_expert(experts, E)
        y = hk.rows_to_experts(x, slots, out=torch.zeros(T * k, H, device="cuda"))
        return (offsets, slots, y, hk.rows_from_experts(y, slots, w), *hk.rows_from_experts_grad(grad, y, slots, w), *hk.quantize_blocks(x))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2):
        torch.manual_seed(seed)
        experts.copy_(torch.randint(-1, E, (T, k), device="cuda")), x.normal_(), w.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) if a.element_size() == 1 else torch.equal(a, b)


def test_a_sort_on_several_streams():
    cases = [torch.randint(-1, 64, (T, 8), device="cuda") for T in (40, 3000, 700)]
    want = [hk.sort_by_expert(c, 64) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for _ in range(20):
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(hk.sort_by_expert(c, 64))
    torch.cuda.synchronize()
    for i, (o, s) in enumerate(got):
        assert torch.equal(o, want[i % 3][0]) and torch.equal(s, want[i % 3][1])


# ---- offsets beyond 32 bits

def far(t, stride):
    """The same rows, `stride` elements apart, behind one another in memory of their own."""
    buf = torch.empty((t.shape[0] - 1) * stride + t.shape[1], dtype=t.dtype, device="cuda")
    view = buf.as_strided(t.shape, (stride, 1))
    view.copy_(t)
    return view


@pytest.mark.parametrize("H", [64, 37])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_far_apart(dtype, H):
    T, k = 3, 2
    _, slots, d_slots = places(T, k, 4, 5, 0.2)
    g = torch.Generator("cuda").manual_seed(H)
    x, r = (torch.randn(T, H, generator=g, device="cuda").to(dtype) for _ in range(2))
    y = torch.randn(T * k, H, generator=g, device="cuda").to(dtype)
    w = torch.rand(T, k, generator=g, device="cuda")
    by_token, by_pair = (1 << 30) + 64, (1 << 29) - 64                 # the last rows lie 2^31 elements and more behind the first
    zero = torch.zeros_like(y)
    named = torch.tensor(slots[slots >= 0], device="cuda")
    assert torch.equal(hk.rows_to_experts(far(x, by_token), d_slots, out=far(zero, by_pair))[named], hk.rows_to_experts(x, d_slots)[named])
    want = hk.rows_from_experts(y, d_slots, w, r)
    assert torch.equal(hk.rows_from_experts(far(y, by_pair), d_slots, w, far(r, by_token)), want)
    assert torch.equal(hk.rows_from_experts(y, d_slots, w, r, out=far(torch.zeros_like(r), by_token)), want)
    grad_y, grad_w = hk.rows_from_experts_grad(x, y, d_slots, w)
    far_y, far_w = hk.rows_from_experts_grad(far(x, by_token), far(y, by_pair), d_slots, w, grad_y=far(zero, by_pair))
    assert torch.equal(far_y, grad_y)
    # products in another order where rows begin elsewhere
    assert torch.allclose(far_w, grad_w, rtol=0, atol=H * 2.0 ** -24 * (x.float().abs() @ y.float().abs().T).max().item() * 2)


def test_blocks_far_apart():
    T, k, K = 3, 2, 300
    _, slots, d_slots = places(T, k, 4, 5, 0.2)
    x = hidden(T, K, torch.bfloat16, 0)
    named = torch.tensor(slots[slots >= 0], device="cuda")
    values, scale = hk.quantize_blocks(x, slots=d_slots)
    row = 1 << 30
    out = torch.empty(5 * row + K, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).as_strided((T * k, K), (row, 1))
    out_scale = torch.empty(2 * row + T * k, device="cuda").as_strided((3, T * k), (row, 1))
    hk.quantize_blocks(far(x, row + 64), slots=d_slots, values=out, scale=out_scale)
    assert torch.equal(out.view(torch.uint8)[named], values.view(torch.uint8)[named]) and torch.equal(out_scale[:, named], scale[:, named])
    w = hidden(131, K, torch.float32, 1)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(hk.quantize_tiles(far(w, 1 << 25)), hk.quantize_tiles(w)))


# ---- rows at every address

@pytest.mark.parametrize("dtype", [torch.int8, torch.float16])
@pytest.mark.parametrize("H", [1, 2, 3, 4, 5, 6, 7, 8, 9, 31, 33, 127, 530, 1333])
def test_rows_to_from_and_to_every_address(dtype, H):
    T, k = 5, 3
    _, slots, d_slots = places(T, k, 4, H, 0.2)
    x = torch.randint(-100, 100, (T, H), device="cuda").to(dtype)
    for shift in range(4):
        for pitch in (H, H + 1, H + 2, H + 3):
            source = torch.full((shift + T * pitch + 4,), 55, device="cuda").to(dtype)
            rows = source[shift:shift + T * pitch].view(T, pitch)[:, :H]
            rows.copy_(x)
            for out_shift in range(4):
                for out_pitch in (H, H + 1, H + 3):
                    buf = torch.full((out_shift + T * k * out_pitch + 4,), 77, device="cuda").to(dtype)
                    want = buf.clone()
                    view = lambda b: b[out_shift:out_shift + T * k * out_pitch].view(T * k, out_pitch)[:, :H]
                    named = d_slots >= 0
                    view(want)[d_slots[named].long()] = x[:, None].expand(T, k, H)[named]
                    hk.rows_to_experts(rows, d_slots, out=view(buf))
                    assert torch.equal(buf, want), (shift, pitch, out_shift, out_pitch)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("T,k,H", [(9, 3, 1333), (6, 2, 264), (5, 2, 700), (11, 3, 2600), (3, 9, 4104)])
def test_rows_of_widths_between_powers_of_two(T, k, H, dtype):
    test_rows_to(T, k, H, torch.bfloat16 if dtype != torch.float32 else torch.float32)
    test_rows_from(T, k, H, dtype)
    test_rows_from_grad(T, k, H, dtype)
