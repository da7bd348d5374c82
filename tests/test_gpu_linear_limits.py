"""GPU parity of the linear layers at the ends of what their documentation allows."""
import numpy as np
import pytest
import torch

from oracle import linear as ol
from paper_2208_00763_b200 import binding as hk
from test_gpu_linear import draw, rows_on_device, weights_on_device

pytestmark = pytest.mark.gpu


def _claims(offsets, T):
    """The groups that claim each row: bounds outside 0 .. T are the nearest one, groups that end before they begin are empty."""
    b = np.clip(np.asarray(offsets, dtype=np.int64), 0, T)
    return [[e for e in range(len(b) - 1) if b[e] <= m < b[e + 1]] for m in range(T)]


WRONG = {
    "two alternate": [0, 64, 300, 64, 300, 64, 300, 64, 300],
    "one holds all": [0, 300, 10, 20, 40, 50, 290, 299, 300],
    "the last holds all": [250, 260, 100, 130, 20, 60, 50, 0, 300],
    "out of bounds": [-5, 200, 2 ** 31 - 1, 100, 150, -2 ** 31, 250, 90, 400],
    "random": np.random.default_rng(3).integers(-40, 340, 41).tolist(),
}


# an 8-bit layer deep enough that clusters share its tiles, dense ones of one and of many steps, flipped activations, and a few rows
@pytest.mark.parametrize("name", list(WRONG))
@pytest.mark.parametrize("T,K,N,q,xs,store", [(300, 4096, 128, 8, True, 8), (300, 128, 128, 4, True, 4), (300, 1024, 200, 4, False, 4),
                                              (300, 640, 130, 8, False, 8), (30, 256, 70, 4, True, 4)])
def test_offsets_that_decrease_spoil_no_row_of_one_group(name, T, K, N, q, xs, store):
    offsets = WRONG[name]
    E = len(offsets) - 1
    x, w = draw((T, K), (E, N, K), 8, q, xs, True, seed=T + K)
    buf = torch.full((T + 2, N), 123456789, dtype=torch.int32, device="cuda")
    for _ in range(2):
        hk.grouped_linear(rows_on_device(x), weights_on_device(w, store), torch.tensor(offsets, dtype=torch.int32, device="cuda"), 8, q, xs, True,
                          w_store_bits=store, out=buf[1:T + 1])
    torch.cuda.synchronize()
    assert hk.linear_wait_timeouts() == 0
    got = buf.cpu().numpy().astype(np.int64)
    assert (got[[0, T + 1]] == 123456789).all()
    every = [ol.sums(x, w[e]) for e in range(E)]
    for m, groups in enumerate(_claims(offsets, T)):
        if not groups:
            assert (got[m + 1] == 123456789).all(), m
        elif len(groups) == 1:
            assert np.array_equal(got[m + 1], every[groups[0]][m]), m
        else:                                            # one of the groups that claim it, value by value
            assert (np.stack([every[e][m] for e in groups]) == got[m + 1]).any(axis=0).all(), m


@pytest.mark.parametrize("store", [8, 1])
def test_the_largest_depths(store):
    # one-bit codes: the last multiple of 16 below 2^31, whose steps do not fit a rounded-up count
    M, N, K = 2, 2, 2 ** 31 - 16
    x = torch.randint(0, 2, (M, K), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(store))
    w = torch.randint(0, 2, (N, K), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(9))
    x[1], w[1] = 1, 1                                    # the largest sum
    stored = w
    if store == 1:
        stored = torch.zeros((N, K // 8), dtype=torch.uint8, device="cuda")
        for i in range(8):
            stored |= w[:, i::8] << i
    got = hk.linear(x, stored, 1, 1, False, False, w_store_bits=store)
    part = 1 << 26
    want = torch.stack([torch.stack([sum((x[m, k:k + part] & w[n, k:k + part]).sum(dtype=torch.int64) for k in range(0, K, part))
                                     for n in range(N)]) for m in range(M)])
    assert torch.equal(got.to(torch.int64), want) and want[1, 1] == K
    assert hk.linear_wait_timeouts() == 0


def _quantized_as_defined(x, codes, scale, part=1 << 26):
    """Signed 8-bit codes and scales of the rows of x against the definition, by parts; divisions by tensors on the device are IEEE's."""
    M, K = x.shape
    hi = torch.tensor(127.0, device="cuda")
    if K == 1:
        for m in range(0, M, part):
            v = x[m:m + part, 0].float()
            assert torch.equal(scale[m:m + part], v.abs() / hi)
            want = torch.where(v == 0, torch.zeros_like(v), v / scale[m:m + part]).round()
            assert torch.equal(codes[m:m + part, 0].float(), want)
    else:
        for m in range(M):
            top = max(x[m, k:k + part].abs().max().item() for k in range(0, K, part))
            assert scale[m] == torch.tensor(top, device="cuda") / hi
            for k in range(0, K, part):
                assert torch.equal(codes[m, k:k + part].float(), (x[m, k:k + part].float() / scale[m]).round())


@pytest.mark.parametrize("M,K", [(1, 2 ** 31 - 1), (2 ** 31 - 1, 1), (2 ** 31 - 7, 1)])
def test_the_longest_and_the_most_rows_to_quantise(M, K):
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    x[-1, -1] = 9.5                                      # the last value counts
    codes, scale = hk.quantize_rows(x, 8)
    _quantized_as_defined(x, codes, scale)
    assert codes[-1, -1] == 127


@pytest.mark.parametrize("M", [3, 12, 40, 700])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_silu_over_its_whole_range(M, dtype):
    """Sums of zero, so that the activation's argument is the bias, exactly.  exp(-|v|) is off by 2 steps, 4 U (U = 2^-24) of its value, which
    v < 0 passes on to the result once at most; a product, a sum and a quotient (half a step and 2^-20 of one) add U each: 7 U.  Where the exponential is
    subnormal (v below -87.3) its steps are 2^-149, times |v|; the product's and the quotient's are half of one such step each."""
    K = 64
    v = torch.cat([torch.linspace(-112, -84, 2001), torch.linspace(-84, 112, 1500), torch.tensor([0.0, -0.0, 1e-40, -1e-40, 3e38, -3e38, float("inf")])])
    N = len(v)
    w = torch.ones((N, K), dtype=torch.int8, device="cuda")
    got = hk.linear(torch.zeros((M, K), dtype=torch.int8, device="cuda"), w, 8, 8, True, True, bias=v.cuda(), activation=hk.ACT_SILU, out_dtype=dtype)
    y = got.cpu().double()
    assert torch.equal(y, y[:1].expand_as(y))            # all rows alike, bit for bit but for signs of zero
    exact = v.double()
    exact = torch.where(exact < -700, torch.zeros_like(exact), exact / (1 + torch.exp(-exact.clamp(min=-700))))
    u = 2.0 ** -24
    tol = 1.01 * 7 * u * exact.abs() + (2 * v.double().abs().clamp(max=112) + 1) * 2.0 ** -149
    info = torch.finfo(dtype)
    if dtype != torch.float32:
        tol = tol + info.eps / 2 * (exact.abs() + tol) + info.smallest_normal * info.eps / 2
    over = exact.abs() >= info.max                       # the infinite one, and for float16 what exceeds it
    assert torch.equal(y[0][over], torch.full_like(y[0][over], float("inf")))
    err = (y[0] - exact).abs()
    assert (err[~over] <= tol[~over]).all(), [(v[i].item(), y[0][i].item(), exact[i].item()) for i in torch.nonzero(~over & (err > tol))[:3, 0]]
    normal = ~over & (exact.abs() >= info.smallest_normal)
    assert (y[0][normal] != 0).all()                     # no normal result is lost


def test_groups_without_offsets_are_refused():
    # whatever the weights' shape: a call by groups is never taken for a plain one
    x = torch.zeros((4, 16), dtype=torch.int8, device="cuda")
    for stream in (None, torch.cuda.current_stream()):
        with pytest.raises(ValueError):
            hk.grouped_linear(x, torch.zeros((8, 16), dtype=torch.int8, device="cuda"), None, 8, 8, True, True, stream=stream)
        with pytest.raises(hk.HikonvError):
            hk.grouped_linear(x, torch.zeros((1, 8, 16), dtype=torch.int8, device="cuda"), None, 8, 8, True, True, stream=stream)


@pytest.mark.parametrize("M,K,N", [(1, 64, 40), (5, 64, 40), (14, 33, 70), (70, 512, 130), (300, 100, 257)])
def test_columns_of_one_buffer(M, K, N):
    x, w = draw((M, K), (N, K), 8, 8, True, True, seed=M)
    s, dw = ol.sums(x, w), weights_on_device(w, 8)
    # the output beside the residual, on either side, with room in front, between and behind
    res = np.random.default_rng(M).integers(-1000, 1000, (M, N)).astype(np.float32)
    for at_res, at_out in ((0, N), (N, 0), (3, N + 5), (N + 4, 1)):
        buf = torch.full((M, 2 * N + 8), 7.0, device="cuda")
        buf[:, at_res:at_res + N] = torch.from_numpy(res).cuda()
        want = buf.clone()
        want[:, at_out:at_out + N] = torch.from_numpy((s + res).astype(np.float32)).cuda()      # whole numbers below 2^24: exact
        hk.linear(rows_on_device(x), dw, 8, 8, True, True, residual=buf[:, at_res:at_res + N], out=buf[:, at_out:at_out + N])
        assert torch.equal(buf, want)
    # codes beside the codes that they come from
    for at_x, at_out in ((0, K), (N, 0), (5, K + 6), (N + 16, 3), (16, K + 16)):
        buf = torch.full((M, K + N + 32), 5, dtype=torch.uint8, device="cuda")
        buf[:, at_x:at_x + K] = torch.from_numpy(x.astype(np.uint8)).cuda()
        want = buf.clone()
        want[:, at_out:at_out + N] = torch.from_numpy(ol.codes(s, None, 9, 0, 255).astype(np.uint8)).cuda()
        hk.linear(buf[:, at_x:at_x + K], dw, 8, 8, True, True, requant=(9, 0, 255), out=buf[:, at_out:at_out + N])
        assert torch.equal(buf, want)
