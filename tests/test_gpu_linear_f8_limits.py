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
