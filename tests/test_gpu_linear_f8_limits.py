"""GPU: products of 8-bit floating point numbers where it is the last bits that count."""
import pytest
import torch

from paper_2208_00763_b200 import binding as hk

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def ones(rows, K, lead=()):
    """Matrices whose rows are a one in the first place and zeros: sums are the scales' products."""
    t = torch.zeros(*lead, rows, (K + 15) // 16 * 16, device="cuda")
    t[..., 0] = 1.0
    return t.to(E4M3)[..., :K]


def silu(v):
    return torch.where(v < 0, v * v.exp() / (1 + v.exp()), v / (1 + (-v).exp()))


@pytest.mark.parametrize("dtype,most", [(torch.bfloat16, 80.0), (torch.float16, 4.0)])
@pytest.mark.parametrize("N", [128, 130, 2048])
@pytest.mark.parametrize("M", [3, 12, 40, 100, 300, 4096])
def test_silu_less_a_residual_that_cancels_it(M, N, dtype, most):
    # values whose SiLU is next to a number of the output's type, which the residual takes away: what is left shows the bits behind
    g = torch.Generator("cuda").manual_seed(M)
    v = (torch.rand(1 << 20, generator=g, device="cuda") * 2 - 1) * most
    want = silu(v.double())
    v = v[(want + (-want).to(dtype).double()).abs() <= 2.0 ** -15 * want.abs()][:M]
    assert len(v) == M
    want = silu(v.double())[:, None].expand(M, N)
    residual = (-want).to(dtype)
    got = hk.linear_f8(ones(M, 128), ones(N, 128), v[None], torch.ones(-(-N // 128), 1, device="cuda"), None, hk.ACT_SILU, residual, out_dtype=dtype)
    # SiLU to 2^-21 of itself, of a sum that is exact; what the residual leaves is exact in 32 bits and rounded to the output's type, whose steps
    # end at tiny * eps
    left = want + residual.double()
    bound = 2.0 ** -21 * want.abs()
    bound = bound + torch.finfo(dtype).eps / 2 * (left.abs() + bound) + torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2
    assert ((got.double() - left).abs() <= bound).all(), ((got.double() - left).abs() / bound).max().item()
    assert hk.linear_wait_timeouts() == 0


@pytest.mark.parametrize("N", [2048, 2176])                # the last tile of 256 columns whole, and half of one
@pytest.mark.parametrize("K", [16, 128, 640, 768, 896, 1500])    # fewer steps than there are stages, as many, and more
def test_pairs_of_ctas_one_call_after_the_other(K, N):
    # each call's CTAs come to where the ones of the call before have just left
    g = torch.Generator("cuda").manual_seed(K)
    M = 4096
    x, w = (torch.randn(r, (K + 15) // 16 * 16, generator=g, device="cuda").mul_(100).clamp_(-448, 448).to(E4M3)[:, :K] for r in (M, N))
    xs, ws = torch.rand(-(-K // 128), M, generator=g, device="cuda"), torch.rand(-(-N // 128), -(-K // 128), generator=g, device="cuda")
    out = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    for i in range(64):
        hk.linear_f8(x, w, xs, ws, out=out[i % 8])
        if i % 3 == 0:
            hk.linear_f8(x[: 40 * (i % 5) + 1], w, xs[:, : 40 * (i % 5) + 1], ws)
    xv = x.float() * xs.T.repeat_interleave(128, 1)[:, :K]
    wv = w.float() * ws.repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    want, size = xv.double() @ wv.double().T, xv.double().abs() @ wv.double().abs().T
    # a block's sum by the tensor cores, 2^-23 of its magnitudes each; the scales' products and the blocks, half a step each; and the rounding
    bound = size * (128 * 2.0 ** -23 + (K // 128 + 8) * 2.0 ** -24)
    assert ((out[0].double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all()
    assert all(torch.equal(o, out[0]) for o in out) and hk.linear_wait_timeouts() == 0


def test_waits_that_run_out_are_counted():
    assert hk.linear_wait_timeouts() == 0
    side = torch.cuda.Stream()
    for n in (1, 2):
        for _ in range(n):
            hk.linear_f8_wait_check(2000000, stream=side)
        assert hk.linear_wait_timeouts() == n
        assert hk.linear_wait_timeouts() == 0
    hk.linear_f8_wait_check(2000000)
    hk.linear_wait_check(2000000)
    assert hk.linear_wait_timeouts() == 2 and hk.linear_wait_timeouts() == 0
    for cycles in (1 << 40, -1):
        with pytest.raises(hk.HikonvError):
            hk.linear_f8_wait_check(cycles)


@pytest.mark.parametrize("M,N", [(3, 130), (12, 128), (40, 130), (100, 256), (300, 257), (4096, 2048)])
def test_scales_whose_product_leaves_the_normal_numbers(M, N):
    # two blocks: a sum of 128 * 64 each
    x, w = torch.full((M, 256), 8.0, device="cuda").to(E4M3), torch.full((N, 256), 8.0, device="cuda").to(E4M3)
    xs, ws = torch.full((2, M), 1.3 * 2.0 ** -80, device="cuda"), torch.full((-(-N // 128), 2), 1.7 * 2.0 ** -66, device="cuda")
    got = hk.linear_f8(x, w, xs, ws, out_dtype=torch.float32).double()
    want = 2 * 128 * 64 * xs[0, 0].double() * ws[0, 0].double()
    # each product of scales is a multiple of 2^-149, half of that off; the sum of two terms is rounded once
    assert ((got - want).abs() <= 2 * 128 * 64 * 2.0 ** -150 + 2.0 ** -24 * want).all()
    xs.fill_(2.0 ** 70), ws.fill_(2.0 ** 60)
    assert torch.isinf(hk.linear_f8(x, w, xs, ws, out_dtype=torch.float32)).all()
    x[:, :] = torch.zeros_like(x)
    assert torch.isnan(hk.linear_f8(x, w, xs, ws, out_dtype=torch.float32)).all()


@pytest.mark.parametrize("f8,most", [(E4M3, 448.0), (torch.float8_e5m2, 57344.0)])
@pytest.mark.parametrize("K", [128, 200])
def test_blocks_of_the_smallest_numbers(f8, most, K):
    def blocks(v):
        v = torch.tensor(v, dtype=torch.float64).float()   # subnormal numbers on the host, kept by a copy
        x = torch.zeros(1, K)
        x[0, : len(v)] = v
        values, scale = hk.quantize_blocks(x.cuda(), f8)
        return values.float().cpu()[0, : len(v)].tolist(), scale.cpu()[0, 0].item()

    # a scale that rounds to one step of 2^-149 for up to one and a half: quotients above the largest number saturate
    step = 2.0 ** -149
    values, scale = blocks([1.4 * most * step, -1.4 * most * step, most * step / 2])
    assert scale == step and values == [most, -most, most / 2]
    # half a step and less: zeros, as for a block of zeros
    for top in (most * step / 2, step, 0.0):
        values, scale = blocks([top, -top])
        assert scale == 0.0 and values == [0.0, 0.0]
    # -0 is a zero of either sign
    values, scale = blocks([-0.0, most])
    assert scale == 1.0 and values == [0.0, most]
