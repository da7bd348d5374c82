"""GPU parity of matrix products of 8-bit floating point numbers with a scale for each block of 128, against the definition in 64 bits, and
a mixture of experts as it is used."""
import numpy as np
import pytest
import torch

from oracle import experts as oe
from paper_2208_00763_b200 import binding as hk

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
ACTS = [hk.ACT_NONE, hk.ACT_RELU, hk.ACT_SILU, hk.ACT_GELU]
SLOPE = {hk.ACT_NONE: 1.0, hk.ACT_RELU: 1.0, hk.ACT_SILU: 1.1, hk.ACT_GELU: 1.13}


def spread(scale, size, dim):
    return scale.double().repeat_interleave(128, dim).narrow(dim, 0, size)


def act64(v, act):
    return {hk.ACT_NONE: lambda: v, hk.ACT_RELU: lambda: v.clamp(min=0), hk.ACT_SILU: lambda: v * torch.sigmoid(v),
            hk.ACT_GELU: lambda: v * 0.5 * torch.erfc(-v / 2 ** 0.5)}[act]()


def reference(x, w, xs, ws, bias, act, residual):
    """(result, bound of the 32-bit arithmetic in front of the last rounding), float64."""
    K, N = x.shape[1], w.shape[0]
    xv = x.double() * spread(xs.T, K, 1)
    wv = w.double() * spread(spread(ws, N, 0), K, 1)
    v = xv @ wv.T
    # A block's 128 products are exact in 32 bits and added up by the tensor cores in 32-bit arithmetic of unknown rounding and order: a whole
    # step, 2^-23, of the sum of magnitudes for each.  Blocks: a product of scales and an addition, half a step each; eight parts at most on top.
    off = (xv.abs() @ wv.abs().T) * (128 * 2.0 ** -23 + (K // 128 + 12) * 2.0 ** -24)
    if bias is not None:
        v = v + bias.double()
        off = off + 2.0 ** -24 * v.abs()
    off = SLOPE[act] * off + 2.0 ** -21 * v.abs() * (act >= hk.ACT_SILU)
    v = act64(v, act)
    if residual is not None:
        v = v + residual.double()
        off = off + 2.0 ** -24 * v.abs()
    return v, off


def near(got, want, off):
    eps, small = torch.finfo(got.dtype).eps, torch.finfo(got.dtype).smallest_normal
    bound = off + (eps / 2) * (want.abs() + off) + small * eps
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (bad.sum().item(), bad.nonzero()[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist(), bound[bad][:3].tolist())


def f8_rows(rows, K, f8, g, lead=()):
    most = torch.finfo(f8).max
    v = torch.randn(*lead, rows, (K + 15) // 16 * 16, generator=g, device="cuda") * most / 4
    return v.clamp(-most, most).to(f8)[..., :K]


def operands(M, N, K, seed, xt=E4M3, wt=E4M3, E=0):
    g = torch.Generator("cuda").manual_seed(seed)
    lead = (E,) if E else ()
    x, w = f8_rows(M, K, xt, g), f8_rows(N, K, wt, g, lead)
    kb, nb = -(-K // 128), -(-N // 128)
    xs = (torch.rand(kb, M, generator=g, device="cuda") + 0.1) / torch.finfo(xt).max
    ws = (torch.rand(*lead, nb, kb, generator=g, device="cuda") + 0.1) / torch.finfo(wt).max / K ** 0.5 * 8
    return x, w, xs, ws, g


SIZES = [(1, 1, 1), (1, 128, 128), (3, 5, 7), (16, 64, 128), (17, 130, 200), (2, 4096, 4096), (31, 257, 1000), (33, 96, 2048), (64, 128, 8192), (65, 1001, 300),
         (128, 128, 128), (129, 255, 129), (200, 512, 384), (257, 384, 640), (500, 1501, 1001), (1024, 1024, 512), (3000, 520, 260), (1, 20000, 512), (130, 33, 6000), (8, 4096, 4096), (9, 300, 700), (3, 5000, 6000), (8, 17, 20000),
         (300, 256, 128), (700, 2304, 1920)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(M, N, K):
    x, w, xs, ws, g = operands(M, N, K, M + N + K)
    want, off = reference(x, w, xs, ws, None, hk.ACT_NONE, None)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        near(hk.linear_f8(x, w, xs, ws, out_dtype=dtype), want, off)
    assert hk.linear_wait_timeouts() == 0


@pytest.mark.parametrize("xt,wt", [(E4M3, E5M2), (E5M2, E4M3), (E5M2, E5M2)])
@pytest.mark.parametrize("M,N,K", [(5, 130, 300), (100, 256, 512), (700, 384, 256)])
def test_types(M, N, K, xt, wt):
    x, w, xs, ws, _ = operands(M, N, K, M, xt, wt)
    near(hk.linear_f8(x, w, xs, ws, out_dtype=torch.float32), *reference(x, w, xs, ws, None, hk.ACT_NONE, None))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N,K", [(3, 200, 256), (40, 131, 128), (600, 256, 256), (600, 259, 128), (300, 2048, 384)])
def test_epilogues(M, N, K, act, dtype):
    x, w, xs, ws, g = operands(M, N, K, M + act)
    bias = torch.randn(N, generator=g, device="cuda")
    residual = torch.randn(M, N, generator=g, device="cuda").to(dtype)
    want, off = reference(x, w, xs, ws, bias, act, residual)
    near(hk.linear_f8(x, w, xs, ws, bias, act, residual, out=torch.empty(M, N, dtype=dtype, device="cuda")), want, off)
    near(hk.linear_f8(x, w, xs, ws, bias, act, out_dtype=dtype), *reference(x, w, xs, ws, bias, act, None))
    # the residual itself, and rows that lie apart
    both = residual.clone()
    assert hk.linear_f8(x, w, xs, ws, bias, act, both, out=both) is both
    near(both, want, off)
    buf = torch.full((M, 2 * N + 3), 5.0, dtype=dtype, device="cuda")
    buf[:, 1:N + 1] = residual
    wide_scale = torch.full((xs.shape[0], M + 9), float("nan"), device="cuda")
    wide_scale[:, 4:M + 4] = xs
    hk.linear_f8(x, w, wide_scale[:, 4:M + 4], ws, bias, act, buf[:, 1:N + 1], out=buf[:, N + 2:2 * N + 2])
    near(buf[:, N + 2:2 * N + 2], want, off)
    assert torch.equal(buf[:, 1:N + 1], residual) and (buf[:, [0, N + 1, 2 * N + 2]] == 5.0).all()


def test_strided_operands():
    M, N, K = 70, 140, 256
    x, w, xs, ws, _ = operands(M, N, K, 0)
    xw, ww = (torch.zeros(r, 3 * K, dtype=E4M3, device="cuda") for r in (M, N))
    xw[:, 128:128 + K], ww[:, 16:16 + K] = x, w
    want = hk.linear_f8(x, w, xs, ws)
    assert torch.equal(hk.linear_f8(xw[:, 128:128 + K], ww[:, 16:16 + K], xs, ws), want)
    one = hk.linear_f8(x[:1].expand(1, K), w, xs[:, :1], ws)
    near(one, *reference(x[:1], w, xs[:, :1], ws, None, 0, None))


def groups(counts, first=0, tail=0):
    off = first + np.concatenate([[0], np.cumsum(counts)])
    return off, torch.tensor(off, dtype=torch.int32, device="cuda"), int(off[-1]) + tail


@pytest.mark.parametrize("N,K", [(128, 128), (200, 300), (1024, 512), (257, 129)])
@pytest.mark.parametrize("counts,first,tail", [([3], 0, 0), ([0, 5, 0, 1], 2, 3), ([0, 0, 0], 0, 4), ([200, 0, 17, 128, 1], 0, 5), ([1] * 40, 0, 0),
                                               ([700, 300, 650], 1, 2), ([2, 0, 1000] + [0] * 61, 0, 0),
                                               ([0] * 30 + [50] + [1] * 9, 0, 3), ([0, 300, 0, 0, 257, 0, 0, 130], 5, 5)])
def test_groups(counts, first, tail, N, K):
    off, offsets, M = groups(counts, first, tail)
    x, w, xs, ws, g = operands(M, N, K, sum(counts), E=len(counts))
    bias = torch.randn(len(counts), N, generator=g, device="cuda")
    out = torch.full((M, N), 3.0, dtype=torch.bfloat16, device="cuda")
    # what lies outside the groups counts for nothing
    x.view(torch.uint8)[:first], x.view(torch.uint8)[off[-1]:] = 0x7F, 0x7F
    assert hk.grouped_linear_f8(x, w, offsets, xs, ws, bias, hk.ACT_SILU, out=out) is out
    assert (out[:first] == 3).all() and (out[off[-1]:] == 3).all()
    for e in range(len(counts)):
        at = slice(off[e], off[e + 1])
        if counts[e]:
            near(out[at], *reference(x[at], w[e], xs[:, at], ws[e], bias[e], hk.ACT_SILU, None))
    assert hk.linear_wait_timeouts() == 0


@pytest.mark.parametrize("xt,wt", [(E4M3, E4M3), (E5M2, E4M3)])
@pytest.mark.parametrize("N,K", [(64, 128), (259, 300), (512, 513), (1024, 2048)])
@pytest.mark.parametrize("counts,first,tail", [([1], 0, 0), ([0, 5, 0, 1], 1, 1), ([1] * 8, 0, 0), ([0] * 5 + [8], 0, 0), ([0] * 5 + [9], 0, 0), ([0, 0, 0], 0, 8),
                                               ([3, 0, 0, 0, 0, 0, 4], 1, 0)])
def test_few_rows_however_they_fall_to_groups(counts, first, tail, N, K, xt, wt):
    off, offsets, M = groups(counts, first, tail)
    x, w, xs, ws, g = operands(M, N, K, sum(counts) + N, xt, wt, E=len(counts))
    bias = torch.randn(len(counts), N, generator=g, device="cuda")
    out = torch.full((M, N), 3.0, dtype=torch.float32, device="cuda")
    x.view(torch.uint8)[:first], x.view(torch.uint8)[off[-1]:] = 0x7F, 0x7F
    hk.grouped_linear_f8(x, w, offsets, xs, ws, bias, out=out)
    assert (out[:first] == 3).all() and (out[off[-1]:] == 3).all()
    for e in range(len(counts)):
        at = slice(off[e], off[e + 1])
        if counts[e]:
            near(out[at], *reference(x[at], w[e], xs[:, at], ws[e], bias[e], hk.ACT_NONE, None))


def test_few_rows_with_offsets_that_are_not_in_order_stay_in_bounds():
    M, N, K = 8, 130, 256
    x, w, xs, ws, _ = operands(M, N, K, 3, E=3)
    guard = torch.full((M + 20, N), 3.0, dtype=torch.bfloat16, device="cuda")
    for off in ([-5, 1, 3, 2000], [6, 2, 4, 8], [8, 0, 8, 0]):
        guard.fill_(3.0)
        hk.grouped_linear_f8(x, w, torch.tensor(off, dtype=torch.int32, device="cuda"), xs, ws, out=guard[10:M + 10])
        assert (guard[:10] == 3).all() and (guard[M + 10:] == 3).all()


def test_offsets_that_are_not_in_order_stay_in_bounds():
    M, N, K = 64, 128, 128
    x, w, xs, ws, _ = operands(M, N, K, 3, E=3)
    guard = torch.full((M + 20, N), 3.0, dtype=torch.bfloat16, device="cuda")
    for off in ([-5, 10, 30, 2000], [60, 20, 40, 64], [64, 0, 64, 0]):
        guard.fill_(3.0)
        hk.grouped_linear_f8(x, w, torch.tensor(off, dtype=torch.int32, device="cuda"), xs, ws, out=guard[10:M + 10])
        assert (guard[:10] == 3).all() and (guard[M + 10:] == 3).all()
    assert hk.linear_wait_timeouts() == 0


def test_infinities_and_nan_stay_in_their_rows_and_columns():
    for M in (4, 300):
        x, w, xs, ws, _ = operands(M, 256, 256, 9)
        clean = hk.linear_f8(x, w, xs, ws)
        x, xs = x.clone(), xs.clone()
        x.view(torch.uint8)[1, 7] = 0x7F                   # NaN
        xs[1, 2] = float("inf")
        got = hk.linear_f8(x, w, xs, ws)
        keep = torch.ones(M, dtype=torch.bool, device="cuda")
        keep[[1, 2]] = False
        assert torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any() and torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("act", [hk.ACT_RELU, hk.ACT_SILU, hk.ACT_GELU])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("M", [3, 40, 300])
def test_activations_at_the_ends_of_their_range(M, dtype, act):
    # sums of a power of two each: one value of x, one of w
    N, K = 256, 128
    x, w = torch.zeros(M, K, device="cuda").to(E4M3), torch.zeros(N, K, device="cuda").to(E4M3)
    x[:, 0], w[:, 0] = 1.0, 1.0
    scale = torch.linspace(-95, 95, M, device="cuda")
    scale[0], scale[1] = float("nan"), 1e-30
    bias = torch.zeros(N, device="cuda")
    bias[1::2] = -1.0                                      # neighbours of other size
    bias[7] = float("inf")
    got = hk.linear_f8(x, w, scale[None], torch.ones(2, 1, device="cuda"), bias, act, out_dtype=dtype)
    v = (scale[:, None] + bias).double()
    want = act64(v, act)
    assert torch.isnan(got[0]).all() and torch.isinf(got[1:, 7]).all()
    rows = torch.ones(M, N, dtype=torch.bool, device="cuda")
    rows[0], rows[:, 7] = False, False
    # SiLU: every normal result to 2^-16 of itself, and the rounding; GELU is 2^-21 |v| off at most; both after an addition in 32 bits.
    # For outputs in 32 bits SiLU multiplies v by exp(-|v|), which is a multiple of 2^-149 where it is subnormal: half of that off, |v| 2^-150 in the product.
    eps, tiny = torch.finfo(dtype).eps, torch.finfo(dtype).smallest_normal
    bound = want.abs() * (eps / 2 + (2.0 ** -16 if act == hk.ACT_SILU else 2.0 ** -24)) + tiny * eps + (2.0 ** -21 * v.abs() if act == hk.ACT_GELU else 0.0)
    bound = bound + (v.abs() * 2.0 ** -150 if act == hk.ACT_SILU and dtype == torch.float32 else 0.0)
    assert ((got.double() - want).abs() <= bound)[rows & (want.abs() < torch.finfo(dtype).max)].all()


def test_zero_scales_and_rows_of_nothing():
    x, w, xs, ws, _ = operands(5, 130, 256, 4)
    assert not hk.linear_f8(x, w, torch.zeros_like(xs), ws).any()
    assert hk.linear_f8(x[:0], w, xs[:, :0], ws).shape == (0, 130)


def test_results_repeat_bit_for_bit():
    for M, N, K in ((2, 512, 4096), (900, 512, 512)):
        x, w, xs, ws, _ = operands(M, N, K, M)
        first = hk.linear_f8(x, w, xs, ws, out_dtype=torch.float32)
        for _ in range(5):
            assert torch.equal(hk.linear_f8(x, w, xs, ws, out_dtype=torch.float32), first)


def test_refusals():
    x, w, xs, ws, _ = operands(4, 130, 200, 0)
    out = torch.empty(4, 130, device="cuda")
    for f in (lambda: hk.linear_f8(x.float(), w, xs, ws), lambda: hk.linear_f8(x, w.float(), xs, ws), lambda: hk.linear_f8(x, w[:, :64], xs, ws),
              lambda: hk.linear_f8(x, w, xs.T, ws), lambda: hk.linear_f8(x, w, xs, ws.T), lambda: hk.linear_f8(x, w, xs.double(), ws),
              lambda: hk.linear_f8(x, w, xs, ws, out_dtype=torch.float64), lambda: hk.linear_f8(x, w, xs, ws, out=out[:3]),
              lambda: hk.linear_f8(x, w, xs, ws, bias=out[0, :5]), lambda: hk.linear_f8(x, w, xs, ws, residual=out[:2]),
              lambda: hk.linear_f8(x, w[None], xs, ws), lambda: hk.grouped_linear_f8(x, w, torch.zeros(2, dtype=torch.int32, device="cuda"), xs, ws),
              lambda: hk.grouped_linear_f8(x, w[None], torch.zeros(3, dtype=torch.int32, device="cuda"), xs, ws[None]),
              lambda: hk.linear_f8(x, w, xs, ws, residual=out, out_dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(hk.HikonvError) as err:
        hk.linear_f8(torch.zeros(4, 200, dtype=E4M3, device="cuda"), w, xs, ws)      # rows 200 bytes apart
    assert err.value.status == hk.ERR_UNSUPPORTED
    with pytest.raises(hk.HikonvError):
        hk.linear_f8(x, w, xs, ws, activation=9)
    with pytest.raises(hk.HikonvError):
        hk.grouped_linear_f8(x, w[None], None, xs, ws[None])


# ---- together

class Layer:
    """Experts on 8-bit floating point numbers: two products with an activation between."""

    def __init__(self, E, H, I, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.E = E
        w1, w2 = (torch.randn(E, *s, generator=g, device="cuda") / s[1] ** 0.5 for s in ((I, H), (H, I)))
        (self.w1, self.s1), (self.w2, self.s2) = hk.quantize_tiles(w1.bfloat16()), hk.quantize_tiles(w2.bfloat16())

    def __call__(self, h, experts, weights, stream=None):
        offsets, slots = hk.sort_by_expert(experts, self.E, stream=stream)
        x, xs = hk.quantize_blocks(h, slots=slots, stream=stream)
        u = hk.grouped_linear_f8(x, self.w1, offsets, xs, self.s1, activation=hk.ACT_SILU, stream=stream)
        x, xs = hk.quantize_blocks(u, stream=stream)
        y = hk.grouped_linear_f8(x, self.w2, offsets, xs, self.s2, stream=stream)
        return hk.rows_from_experts(y, slots, weights, residual=h, stream=stream)

    def plain(self, h, experts, weights):
        """The same in 64 bits from the same 8-bit weights; activations are not quantised."""
        w1 = self.w1.double() * spread(spread(self.s1, self.w1.shape[1], 1), self.w1.shape[2], 2)
        w2 = self.w2.double() * spread(spread(self.s2, self.w2.shape[1], 1), self.w2.shape[2], 2)
        out = h.double()
        for e in range(self.E):
            t, j = (experts == e).nonzero(as_tuple=True)
            v = h[t].double() @ w1[e].T
            out.index_add_(0, t, (v * torch.sigmoid(v)) @ w2[e].T * weights[t, j].double()[:, None])
        return out


def tokens(T, E, k, H, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    h = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    top, experts = torch.topk(torch.randn(T, E, generator=g, device="cuda"), k, dim=1)
    experts[::7, 0] = -1
    return h, experts, torch.softmax(top, 1)


@pytest.mark.parametrize("T,E,k,H,I", [(1, 8, 2, 256, 384), (30, 16, 4, 512, 256), (900, 8, 2, 384, 520)])
def test_a_mixture_of_experts(T, E, k, H, I):
    layer = Layer(E, H, I, T)
    h, experts, weights = tokens(T, E, k, H, T)
    got, want = layer(h, experts, weights), layer.plain(h, experts, weights)
    # Two quantisations round by half a step of 2^-3 at most, 2^-4 of each value (uniformly: 0.58 of that as a deviation); an output is a sum of H or I
    # products of independent roundings, so the deviation is below 2^-4 of the deviation that the products themselves make, twice; with
    # SiLU's slope of 1.1 at most, and bf16's roundings: below 0.16 of what the experts add.
    added = (want - h.double())
    off = (got.double() - want).square().mean().sqrt() / added.square().mean().sqrt()
    assert off < 0.16, off.item()


def test_a_mixture_in_a_graph_replayed_with_other_tokens():
    layer = Layer(8, 256, 384, 0)
    h, experts, weights = tokens(40, 8, 2, 256, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(h, experts, weights)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(h, experts, weights)
    for seed in (2, 3):
        h2, experts2, weights2 = tokens(40, 8, 2, 256, seed)
        h.copy_(h2), experts.copy_(experts2), weights.copy_(weights2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, layer(h2, experts2, weights2))
    assert hk.linear_wait_timeouts() == 0


def test_on_another_stream():
    layer = Layer(8, 256, 384, 0)
    h, experts, weights = tokens(300, 8, 2, 256, 1)
    want = layer(h, experts, weights)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [layer(h, experts, weights, stream=side) for _ in range(3)]
    with torch.cuda.stream(side):
        got.append(layer(h, experts, weights))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    # the same as the call without the native path
    assert torch.equal(hk.linear_f8(*operands(5, 200, 256, 0)[:4], stream=side).cpu(), hk.linear_f8(*operands(5, 200, 256, 0)[:4]).cpu())


def test_two_calls_at_once():
    one, two = Layer(8, 256, 384, 0), Layer(8, 256, 384, 5)
    a, b = tokens(600, 8, 2, 256, 1), tokens(3, 8, 2, 256, 2)
    want = one(*a), two(*b)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(10):
        for s, layer, args in zip(streams, (one, two), (a, b)):
            with torch.cuda.stream(s):
                got.append(layer(*args))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % 2])


def test_training_step_of_experts():
    """Forward and backward of experts on float32 rows, by these calls around plain products, against automatic differentiation in 64 bits."""
    T, E, k, H = 60, 5, 2, 48
    g = torch.Generator("cuda").manual_seed(0)
    x, up = (torch.randn(T, H, generator=g, device="cuda") for _ in range(2))
    w = torch.randn(E, H, H, generator=g, device="cuda") / H ** 0.5
    top, experts = torch.topk(torch.randn(T, E, generator=g, device="cuda"), k, dim=1)
    experts[3, 1] = experts[7, 0] = experts[7, 1] = -1
    weights = torch.softmax(top, 1)
    offsets, slots = hk.sort_by_expert(experts, E)
    ends = offsets.tolist()
    rows = hk.rows_to_experts(x, slots, out=torch.zeros(T * k, H, device="cuda"))
    y = torch.zeros_like(rows)
    for e in range(E):
        y[ends[e]:ends[e + 1]] = rows[ends[e]:ends[e + 1]] @ w[e].T
    out = hk.rows_from_experts(y, slots, weights, residual=x)
    grad_y, grad_weights = hk.rows_from_experts_grad(up, y, slots, weights)
    grad_rows, grad_w = torch.zeros_like(rows), torch.zeros_like(w)
    for e in range(E):
        at = slice(ends[e], ends[e + 1])
        grad_rows[at], grad_w[e] = grad_y[at] @ w[e], grad_y[at].T @ rows[at]
    grad_x = hk.rows_from_experts(grad_rows, slots, residual=up)
    x64, w64, r64 = (t.double().requires_grad_() for t in (x, w, weights))
    want = x64
    for j in range(k):
        there = (experts[:, j] >= 0)[:, None]
        want = want + torch.where(there, torch.einsum("th,tnh->tn", x64, w64[experts[:, j].clamp(min=0)]) * r64[:, j:j + 1], 0.0)
    (want * up.double()).sum().backward()
    # sums of H = 48 products and of some dozens of rows in 32 bits, of values of order one: 2^-24 times a few hundred
    for got, ref in ((out, want), (grad_x, x64.grad), (grad_w, w64.grad), (grad_weights, torch.where(experts >= 0, r64.grad, 0.0))):
        assert (got.double() - ref).abs().max() < 400 * 2.0 ** -24 * max(1.0, ref.abs().max().item())


def test_clusters_at_once_on_two_streams():
    # layers whose depth is shared by clusters, many at once
    cases = [operands(M, N, 4096, M) for M, N in ((9, 512), (100, 1024), (12, 2048), (60, 640))]
    want = [hk.linear_f8(*c[:4]) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(4)], []
    for _ in range(50):
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(hk.linear_f8(*c[:4]))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 4]) for i, y in enumerate(got)) and hk.linear_wait_timeouts() == 0


@pytest.mark.parametrize("M,N", [(3, 40), (40, 140), (300, 130), (300, 2048), (2048, 2048), (4096, 2048)])
def test_operands_far_apart(M, N):
    # rows of x, w, the scales and the output reach beyond 2^32 bytes
    K = 384
    x, w, xs, ws, g = operands(M, N, K, M)
    residual = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    want = hk.linear_f8(x, w, xs, ws, residual=residual)

    def far(t, span):
        step = span // (t.shape[0] - 1) // 16 * 16 + 16
        view = torch.empty((t.shape[0] - 1) * step + (t.shape[1] + 15) // 16 * 16, dtype=t.dtype, device="cuda").as_strided(t.shape, (step, 1))
        view.copy_(t)
        return view

    out = far(torch.zeros_like(residual), 1 << 31)
    hk.linear_f8(far(x, 1 << 32), far(w, 1 << 32), far(xs, 1 << 31), ws, residual=far(residual, 1 << 31), out=out)
    assert torch.equal(out, want)


def test_weights_of_many_bytes():
    # the last matrices begin 2^32 bytes and more behind the first
    E, N, K = 33, 8192, 16384
    w = torch.zeros(E, N, K, dtype=torch.uint8, device="cuda").view(E4M3)
    ws = torch.ones(E, N // 128, K // 128, device="cuda")
    for counts in ([0] * 31 + [3, 4], [0] * 31 + [40, 300], [1] * 33):
        off, offsets, M = groups(counts)
        x, small, xs, small_ws, _ = operands(M, N, 128, len(counts) + M, E=2)
        w[31:, :, -128:].view(torch.uint8).copy_(small.view(torch.uint8))
        ws[31:, :, -1] = small_ws[..., 0]
        wide_x, wide_xs = torch.zeros(M, K, dtype=torch.uint8, device="cuda").view(E4M3), torch.zeros(K // 128, M, device="cuda")
        wide_x[:, -128:].view(torch.uint8).copy_(x.view(torch.uint8))
        wide_xs[-1] = xs[0]
        got = hk.grouped_linear_f8(wide_x, w, offsets, wide_xs, ws, out_dtype=torch.float32)
        assert not got[:off[31]].any()
        for i in range(2):
            at = slice(off[31 + i], off[32 + i])
            near(got[at], *reference(x[at], small[i], xs[:, at], small_ws[i], None, hk.ACT_NONE, None))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,N,K,act", [(4096, 2048, 384, hk.ACT_SILU), (4096, 2049, 384, hk.ACT_NONE), (4100, 2064, 300, hk.ACT_GELU), (4096, 2200, 200, hk.ACT_SILU),
                                       (500, 1501, 256, hk.ACT_NONE), (500, 1536, 256, hk.ACT_RELU), (130, 1009, 640, hk.ACT_SILU)])
def test_bias_and_residual_of_large_outputs(M, N, K, act, dtype):
    x, w, xs, ws, g = operands(M, N, K, N)
    bias = torch.randn(N, generator=g, device="cuda")
    residual = torch.randn(M, N, generator=g, device="cuda").to(dtype)
    for b, r in ((bias, None), (None, residual), (bias, residual)):
        want, off = reference(x, w, xs, ws, b, act, r)
        near(hk.linear_f8(x, w, xs, ws, b, act, r, out_dtype=dtype), want, off)
    both = residual.clone()                                # in place
    hk.linear_f8(x, w, xs, ws, bias, act, both, out=both)
    near(both, want, off)
    assert hk.linear_wait_timeouts() == 0
