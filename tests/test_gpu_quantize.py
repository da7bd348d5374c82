"""GPU parity of the quantisation of rows: codes and scales equal the definition's, bit for bit."""
import numpy as np
import pytest
import torch

from gpu_util import assert_exact
from oracle import linear as ol
from paper_2208_00763_b200 import binding as hk

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
WIDTHS = [(8, True), (4, True), (2, True), (7, True), (8, False), (4, False), (1, False), (3, False)]


def check(x, bits, signed, **kw):
    codes, scale = hk.quantize_rows(x, bits, signed, **kw)
    torch.cuda.synchronize()
    want, want_scale = ol.quantize(x.double().cpu().numpy(), bits, signed)
    got = codes.cpu().numpy().view(np.int8 if signed else np.uint8).astype(np.int64)
    assert codes.dtype == (torch.int8 if signed else torch.uint8)
    assert np.array_equal(scale.cpu().numpy(), want_scale, equal_nan=True)
    assert got.shape == want.shape and np.array_equal(got, want), np.argwhere(got != want)[:3]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(1, 1), (1, 4096), (3, 7), (5, 32), (2, 255), (9, 256), (4, 257), (33, 128), (2, 1000), (130, 520), (3, 5003),
                                 (2, 8192), (3, 16384), (2, 16392), (1, 40000), (2, 33001), (700, 64)])
def test_sizes(dtype, M, K):
    g = torch.Generator().manual_seed(M * 100 + K)
    x = (torch.randn(M, K, generator=g) * (torch.rand(M, 1, generator=g) * 10 + 0.01)).to(dtype).cuda()
    for bits, signed in WIDTHS:
        check(x, bits, signed)


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_and_rows_that_are_special(dtype):
    x = torch.zeros(12, 96, dtype=torch.float64)
    x[1, 5] = 3.0
    x[2] = torch.arange(96) - 48                         # quotients that are halves for some widths
    x[3] = (torch.arange(96) % 31 - 15) * 0.5
    x[4, :10] = -1.0
    x[5, 3], x[5, 4] = float("inf"), 1.0
    x[6, 2], x[6, 3] = float("nan"), 2.0
    x[7, 0] = float("-inf")
    x[8] = torch.finfo(dtype).tiny * 0.25 * (torch.arange(96) % 5)          # subnormal
    x[9] = torch.finfo(dtype).max * ((torch.arange(96) % 3) - 1)
    x[10, 95] = -2.5
    x[11] = 127 * torch.sign(torch.arange(96) - 40) + torch.arange(96) % 2 * 0.5
    for bits, signed in WIDTHS:
        check(x.to(dtype).cuda(), bits, signed)


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_to_even(dtype):
    # a scale of one: quotients are the values themselves
    x = torch.arange(-127, 128, dtype=torch.float64) * 0.5
    x[0] = 127.0
    x = x.to(dtype).cuda()[None]
    check(x, 8, True)
    check(x.abs() + x.abs(), 8, False)


@pytest.mark.parametrize("repeat", [1, 34])             # 34: rows longer than the registers hold
@pytest.mark.parametrize("bits,signed", WIDTHS)
def test_quotients_next_to_halves(bits, signed, repeat):
    """Values a few floats to either side of (n + 1/2) scale, for scales of many mantissas (those next to 1 and 2 among them) and sizes."""
    rng = np.random.default_rng(bits)
    hi = (1 << (bits - 1)) - 1 if signed else (1 << bits) - 1
    mantissas = np.concatenate([np.arange(24), (1 << 23) - 1 - np.arange(24), rng.integers(0, 1 << 23, 200)])
    exponents = np.concatenate([[0, -64, 63, -63, 64, -100, 110], rng.integers(-60, 60, len(mantissas) - 7)])
    scale = (np.ldexp(1.0 + mantissas / 2.0**23, rng.permutation(exponents))).astype(np.float32)
    top = (scale.astype(np.float64) * hi).astype(np.float32)
    scale = (top / np.float32(hi)).astype(np.float32)               # the definition's, which need not be the one wished for
    n = rng.integers(0, hi, (len(scale), 997)) + 0.5
    x = (n * scale[:, None].astype(np.float64)).astype(np.float32)
    x = (x.view(np.int32) + rng.integers(-3, 4, x.shape, dtype=np.int32)).view(np.float32)
    x *= rng.choice(np.float32([-1, 1]), x.shape) if signed else np.float32(1)
    x = np.minimum(np.maximum(x, -top[:, None]), top[:, None])
    x[:, 0] = top
    check(torch.from_numpy(np.tile(x, (1, repeat))).cuda(), bits, signed)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart_and_rows_that_are_one(dtype):
    g = torch.Generator().manual_seed(5)
    base = torch.randn(20, 700, generator=g).to(dtype).cuda()
    for view in (base[:, :512], base[:, 3:260], base[::3, 8:520], base[4:5, 1:2], base[:1].expand(6, 700), base[:, 1:601]):
        check(view, 8, True)
        check(view, 4, False)


def test_given_outputs_and_what_lies_around_them():
    x = torch.randn(7, 130, device="cuda")
    codes = torch.full((9, 130), 55, dtype=torch.int8, device="cuda")
    scale = torch.full((9,), -1.0, device="cuda")
    c, s = hk.quantize_rows(x, 8, codes=codes[1:8], scale=scale[1:8])
    assert c.data_ptr() == codes[1:].data_ptr() and s.data_ptr() == scale[1:].data_ptr()
    assert (codes[0] == 55).all() and (codes[8] == 55).all() and scale[0] == -1 and scale[8] == -1
    check(x, 8, True, codes=codes[1:8], scale=scale[1:8])
    c, s = hk.quantize_rows(torch.empty((0, 16), device="cuda"), 8)
    assert c.shape == (0, 16) and s.shape == (0,)


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_that_start_on_any_byte(dtype):
    for K in (1, 3, 9, 77, 520, 1001, 8190):
        x = torch.randn(6, K, generator=torch.Generator().manual_seed(K)).to(dtype).cuda()
        for lead in range(5):
            buf = torch.full((6 * K + 16,), 55, dtype=torch.int8, device="cuda")
            check(x, 8, True, codes=buf[lead:lead + 6 * K].view(6, K))
            assert (buf[:lead] == 55).all() and (buf[lead + 6 * K:] == 55).all()


def test_captured_and_other_streams():
    x = torch.randn(40, 256, device="cuda").bfloat16()
    codes = torch.zeros((40, 256), dtype=torch.int8, device="cuda")
    scale = torch.zeros(40, device="cuda")
    hk.quantize_rows(x, 8, codes=codes, scale=scale)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hk.quantize_rows(x, 8, codes=codes, scale=scale)
    for seed in range(3):
        x.copy_(torch.randn(40, 256, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        want, want_scale = ol.quantize(x.double().cpu().numpy(), 8, True)
        assert_exact(codes, want)
        assert np.array_equal(scale.cpu().numpy(), want_scale)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    c, t = hk.quantize_rows(x, 8, stream=s)
    with torch.cuda.stream(s):
        c2, t2 = hk.quantize_rows(x, 8)
    torch.cuda.synchronize()
    assert torch.equal(c, codes) and torch.equal(t, scale) and torch.equal(c2, codes) and torch.equal(t2, scale)


def test_refusals_of_the_binding():
    x = torch.zeros((4, 16), device="cuda")
    for t in (x.double(), x.cpu(), x[0], x.t(), x.to(torch.int8)):
        with pytest.raises(ValueError):
            hk.quantize_rows(t, 8)
    for kw in (dict(codes=torch.zeros((4, 15), dtype=torch.int8, device="cuda")), dict(codes=torch.zeros((4, 16), dtype=torch.int32, device="cuda")),
               dict(scale=torch.zeros(5, device="cuda")), dict(scale=torch.zeros(4, device="cuda").half()), dict(codes=torch.zeros((4, 16), dtype=torch.int8))):
        with pytest.raises(ValueError):
            hk.quantize_rows(x, 8, **kw)
    for bits, signed in ((0, True), (1, True), (9, True), (0, False), (9, False)):
        with pytest.raises(hk.HikonvError):
            hk.quantize_rows(x, bits, signed)
    with pytest.raises(hk.HikonvError):
        hk.quantize_rows(x, 8, codes=x.view(torch.int8).view(-1)[:64].view(4, 16))
