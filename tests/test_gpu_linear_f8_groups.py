"""GPU: products of 8-bit floating point numbers by group with a residual, and sums to the last bits.

The values are small whole numbers, so that a block's sum is exact in any order of its 128 products: what is left are the scales and the blocks' additions,
whose bound is some steps of 2^-24."""
import numpy as np
import pytest
import torch

from paper_2208_00763_b200 import binding as hk

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


def whole_numbers(rows, K, f8, g, lead=()):
    """-8 .. 8, what either type holds of them (e5m2: not 5 and 7)."""
    v = torch.randint(-8, 9, (*lead, rows, (K + 15) // 16 * 16), generator=g, device="cuda")
    if f8 == E5M2:
        v = torch.where((v.abs() == 5) | (v.abs() == 7), v.sign() * 6, v)
    return v.float().to(f8)[..., :K]


def operands(M, N, K, seed, E=0, xt=E4M3, wt=E4M3):
    g = torch.Generator("cuda").manual_seed(seed)
    lead = (E,) if E else ()
    x, w = whole_numbers(M, K, xt, g), whole_numbers(N, K, wt, g, lead)
    xs = torch.rand(-(-K // 128), M, generator=g, device="cuda") + 0.1
    ws = (torch.rand(*lead, -(-N // 128), -(-K // 128), generator=g, device="cuda") + 0.1) / 64
    return x, w, xs, ws, g


def exactly(x, w, xs, ws, bias=None, residual=None):
    """(result in 64 bits, bound of the 32-bit arithmetic in front of the last rounding)."""
    K, N = x.shape[1], w.shape[0]
    v, size = 0.0, 0.0
    for b in range(xs.shape[0]):
        at = slice(128 * b, min(128 * b + 128, K))
        term = (x[:, at].double() @ w[:, at].double().T) * xs[b].double()[:, None] * ws[:, b].double().repeat_interleave(128)[:N]
        v, size = v + term, size + term.abs()
    # half a step of 2^-23 for the product of two scales, for each block's multiply and add, and for each of up to eight parts of a depth
    off = size * (xs.shape[0] + 9) * 2.0 ** -24
    if bias is not None:
        v = v + bias.double()
        off = off + 2.0 ** -24 * (v.abs() + off)
    if residual is not None:
        v = v + residual.double()
        off = off + 2.0 ** -24 * (v.abs() + off)
    return v, off


def near(got, want, off):
    bound = off + torch.finfo(got.dtype).eps / 2 * (want.abs() + off) + torch.finfo(got.dtype).tiny
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (bad.sum().item(), bad.nonzero()[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist())


@pytest.mark.parametrize("M,N,K", [(1, 128, 4096), (3, 130, 300), (8, 512, 8192), (9, 300, 700), (16, 1024, 8192), (40, 140, 5000), (100, 2048, 4096), (128, 128, 128),
                                   (200, 513, 384), (257, 384, 2100), (1024, 1024, 512), (4096, 2048, 1024), (4099, 2056, 700)])
@pytest.mark.parametrize("xt,wt", [(E4M3, E4M3), (E5M2, E4M3), (E4M3, E5M2), (E5M2, E5M2)])
def test_sums_to_the_last_bits(M, N, K, xt, wt):
    x, w, xs, ws, _ = operands(M, N, K, M + N, 0, xt, wt)
    near(hk.linear_f8(x, w, xs, ws, out_dtype=torch.float32), *exactly(x, w, xs, ws))


COUNTS = [([1], 0, 0), ([3, 0, 0, 0, 4], 1, 0), ([0, 0, 8], 0, 3), ([0, 5, 0, 1], 2, 3), ([9, 7, 0, 20], 3, 0), ([200, 0, 17, 128, 1], 0, 5), ([1] * 40, 0, 0),
          ([700, 300, 650], 1, 2), ([0] * 30 + [50] + [1] * 9, 0, 3), ([1500, 0, 700, 1, 129, 257], 5, 7), ([5] * 64, 1, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("N,K", [(128, 128), (200, 300), (1024, 512), (257, 129), (2048, 1024)])
@pytest.mark.parametrize("counts,first,tail", COUNTS)
def test_groups_with_a_residual(counts, first, tail, N, K, dtype):
    ends = first + np.concatenate([[0], np.cumsum(counts)])
    offsets, M = torch.tensor(ends, dtype=torch.int32, device="cuda"), int(ends[-1]) + tail
    x, w, xs, ws, g = operands(M, N, K, sum(counts) + N, len(counts))
    bias = torch.randn(len(counts), N, generator=g, device="cuda")
    # what lies outside the groups counts for nothing
    x.view(torch.uint8)[:first], x.view(torch.uint8)[ends[-1]:] = 0x7F, 0x7F
    outside = torch.ones(M, dtype=torch.bool, device="cuda")
    outside[ends[0]:ends[-1]] = False
    residual = torch.randn(M, N, generator=g, device="cuda").to(dtype)
    out = torch.full((M, N), 3.0, dtype=dtype, device="cuda")
    hk.grouped_linear_f8(x, w, offsets, xs, ws, bias, residual=residual, out=out)
    both = residual.clone()                                # in place
    hk.grouped_linear_f8(x, w, offsets, xs, ws, bias, residual=both, out=both)
    # columns of one buffer, rows on no boundary
    buf = torch.full((M, 2 * N + 5), 5.0, dtype=dtype, device="cuda")
    buf[:, 1:N + 1] = residual
    hk.grouped_linear_f8(x, w, offsets, xs, ws, bias, residual=buf[:, 1:N + 1], out=buf[:, N + 3:2 * N + 3])
    assert (out[outside] == 3).all() and torch.equal(both[outside], residual[outside]) and (buf[:, N + 3:2 * N + 3][outside] == 5).all()
    assert torch.equal(buf[:, 1:N + 1], residual) and (buf[:, [0, N + 1, N + 2, 2 * N + 3, 2 * N + 4]] == 5).all()
    for e in range(len(counts)):
        at = slice(ends[e], ends[e + 1])
        if counts[e]:
            want, off = exactly(x[at], w[e], xs[:, at], ws[e], bias[e], residual[at])
            for got in (out, both, buf[:, N + 3:2 * N + 3]):
                near(got[at], want, off)
    assert hk.linear_wait_timeouts() == 0


@pytest.mark.parametrize("ends", [[0, 30, 20, 64], [10, 40, 25, 60], [64, 0, 64, 0], [-5, 10, 30, 2000], [60, 20, 40, 64], [0, 4, 2, 8], [8, 0, 8, 0], [-5, 1, 3, 2000], [6, 2, 4, 8]])
@pytest.mark.parametrize("M", [8, 64, 400])
def test_rows_that_one_group_alone_claims(M, ends):
    # offsets out of order: such a row has its group's result, one that none claims stays; what two claim is undefined
    N, K = 200, 256
    ends = [e * (M // 8 if max(ends) <= 8 else max(M // 64, 1)) for e in ends]
    x, w, xs, ws, _ = operands(M, N, K, 7, 3)
    out = torch.full((M, N), 3.0, device="cuda")
    hk.grouped_linear_f8(x, w, torch.tensor(ends, dtype=torch.int32, device="cuda"), xs, ws, out=out)
    claimed = [[] for _ in range(M)]
    for e in range(3):
        for m in range(min(max(ends[e], 0), M), min(max(ends[e + 1], 0), M)):
            claimed[m].append(e)
    assert all((out[m] == 3).all() for m in range(M) if not claimed[m])
    for e in range(3):
        rows = [m for m in range(M) if claimed[m] == [e]]
        if rows:
            near(out[rows], *exactly(x[rows], w[e], xs[:, rows], ws[e]))
    assert hk.linear_wait_timeouts() == 0
