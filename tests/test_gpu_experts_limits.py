"""GPU: rows to experts and back where slots name only some of the rows."""
import numpy as np
import pytest
import torch

from oracle import experts as oe
from paper_2208_00763_b200 import binding as hk

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def nan_behind(rows, H, dtype, stream=None):
    """Memory of this size that was written with NaN and then freed, which the next call's output gets."""
    with torch.cuda.stream(stream):
        some = [torch.full((rows, H), float("nan"), dtype=dtype, device="cuda") for _ in range(3)]
        del some


def some_slots(T, k, R, g):
    """Distinct places below R, all but a few of them: some pairs have none (-1, and beyond the last row), some are without expert (-2 - place)."""
    slots = torch.randperm(R, generator=g)[: T * k].reshape(T, k).int()
    slots[T // 2, 0] = -1
    slots[T // 3, k - 1] = R + 3
    slots[T - 1, 0] = -2 - slots[T - 1, 0]
    return slots


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_weights", [True, False])
@pytest.mark.parametrize("T,k,R,H", [(5, 2, 10, 64), (7, 3, 40, 133), (60, 4, 240, 256), (60, 4, 300, 257), (1, 1, 1, 8), (1, 1, 5, 8)])
@pytest.mark.parametrize("own_stream", [False, True])
def test_gradient_of_rows_that_no_slot_names_is_zero(T, k, R, H, dtype, with_weights, own_stream):
    g = torch.Generator().manual_seed(T + R)
    slots = some_slots(T, k, R, g) if T > 2 else torch.full((T, k), -1, dtype=torch.int32)
    grad, y, weights = torch.randn(T, H, generator=g).to(dtype), torch.randn(R, H, generator=g).to(dtype), torch.rand(T, k, generator=g)
    if not with_weights:
        weights = None
    want, want_w = oe.rows_from_grad(grad.double().numpy(), y.double().numpy(), slots.numpy(), None if weights is None else weights.double().numpy(), np.zeros((R, H)))
    stream = torch.cuda.Stream() if own_stream else None
    args = grad.cuda(), y.cuda(), slots.cuda(), None if weights is None else weights.cuda()
    torch.cuda.synchronize()
    nan_behind(R, H, dtype, stream)
    got, got_w = hk.rows_from_experts_grad(*args, stream=stream)
    torch.cuda.synchronize()
    assert got.shape == (R, H)
    # one product, rounded once to 32 bits and once to the type; weights: sums of H products in 32 bits
    want = torch.from_numpy(want)
    assert ((got.cpu().double() - want).abs() <= want.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -23) + torch.finfo(dtype).tiny).all()
    if with_weights:
        off = grad.double().abs() @ y.double().abs().T
        want_w = torch.from_numpy(want_w)
        assert ((got_w.cpu().double() - want_w).abs() <= (H + 2) * 2.0 ** -24 * off.max()).all()
    else:
        assert got_w is None


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_without_tokens_is_zero(dtype):
    H, k, R = 64, 3, 50
    y = torch.randn(R, H, device="cuda").to(dtype)
    nothing = torch.empty(0, H, dtype=dtype, device="cuda"), y, torch.empty(0, k, dtype=torch.int32, device="cuda"), torch.empty(0, k, device="cuda")
    for stream in (None, torch.cuda.Stream()):
        nan_behind(R, H, dtype, stream)
        got, got_w = hk.rows_from_experts_grad(*nothing, stream=stream)
        torch.cuda.synchronize()
        assert got.shape == (R, H) and got_w.shape == (0, k) and not got.any()


def test_gradient_without_rows_made_for_pairs_that_have_none():
    # without y: a row per pair, of which some get nothing
    T, k, H = 9, 2, 40
    grad = torch.randn(T, H, device="cuda")
    slots = torch.arange(T * k, dtype=torch.int32, device="cuda").reshape(T, k)
    slots[3, 1] = slots[8, 0] = -1
    nan_behind(T * k, H, torch.float32)
    got, _ = hk.rows_from_experts_grad(grad, None, slots)
    want = grad.repeat_interleave(k, 0)
    want[[7, 16]] = 0.0
    assert torch.equal(got, want)


def test_gradient_in_a_graph_replayed_with_other_slots():
    T, k, R, H = 20, 2, 50, 96
    g = torch.Generator().manual_seed(0)
    grad, y, weights = torch.randn(T, H, device="cuda"), torch.randn(R, H, device="cuda"), torch.rand(T, k, device="cuda")
    slots = some_slots(T, k, R, g).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hk.rows_from_experts_grad(grad, y, slots, weights)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, got_w = hk.rows_from_experts_grad(grad, y, slots, weights)
    for _ in range(3):
        slots.copy_(some_slots(T, k, R, g))
        graph.replay()
        want, want_w = hk.rows_from_experts_grad(grad, y, slots, weights, grad_y=torch.zeros_like(y))
        assert torch.equal(got, want) and torch.equal(got_w, want_w)


def test_rows_of_a_given_gradient_that_no_slot_names_stay():
    T, k, R, H = 20, 2, 50, 96
    slots = some_slots(T, k, R, torch.Generator().manual_seed(1)).cuda()
    grad, y = torch.randn(T, H, device="cuda"), torch.randn(R, H, device="cuda")
    given = torch.full((R, H), 7.0, device="cuda")
    hk.rows_from_experts_grad(grad, y, slots, grad_y=given)
    named = torch.where(slots >= 0, slots, -2 - slots).flatten()
    named = named[(named >= 0) & (named < R)].long()
    rest = torch.ones(R, dtype=torch.bool, device="cuda")
    rest[named] = False
    assert (given[rest] == 7.0).all() and not (given[~rest] == 7.0).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,R,H", [(300, 4, 1200, 4096), (300, 4, 1300, 4001), (1, 1, 9, 1 << 20), (2000, 2, 100000, 50), (70000, 2, 140000, 33), (0, 2, 3000, 2048), (500, 1, 100000, 133)])
@pytest.mark.parametrize("own_stream", [False, True])
def test_gradient_of_large_rows_that_no_slot_names_is_zero(T, k, R, H, dtype, own_stream):
    # beyond 8 MB the rows that no slot names are found
    g = torch.Generator().manual_seed(T + R)
    slots = torch.randperm(R, generator=g)[: T * k].reshape(T, k).int()
    if T > 1:
        slots[T // 2, 0], slots[T // 3, k - 1], slots[T - 1, 0] = -1, R + 3, -2 - slots[T - 1, 0]
        slots[5:9, 0] = torch.tensor([-(1 << 31), (1 << 31) - 1, -2 - R, R], dtype=torch.int32)
    slots, stream = slots.cuda(), torch.cuda.Stream() if own_stream else None
    grad, y = torch.randn(T, H, device="cuda").to(dtype), torch.randn(R, H, device="cuda").to(dtype)
    want, _ = hk.rows_from_experts_grad(grad, y, slots, grad_y=torch.zeros_like(y))
    torch.cuda.synchronize()
    nan_behind(R, H, dtype, stream)
    for _ in range(2):
        got, _ = hk.rows_from_experts_grad(grad, y, slots, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        got.fill_(float("nan"))
        del got


def test_large_gradient_in_a_graph_replayed_with_other_slots():
    T, k, R, H = 400, 2, 1000, 4100
    g = torch.Generator().manual_seed(0)
    grad, y, weights = torch.randn(T, H, device="cuda"), torch.randn(R, H, device="cuda"), torch.rand(T, k, device="cuda")
    slots = some_slots(T, k, R, g).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hk.rows_from_experts_grad(grad, y, slots, weights)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, got_w = hk.rows_from_experts_grad(grad, y, slots, weights)
    for _ in range(3):
        slots.copy_(some_slots(T, k, R, g))
        graph.replay()
        want, want_w = hk.rows_from_experts_grad(grad, y, slots, weights, grad_y=torch.zeros_like(y))
        assert torch.equal(got, want) and torch.equal(got_w, want_w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,row,first", [(1, 1, 0), (3, 5, 1), (7, 7, 1), (8, 8, 0), (9, 24, 3), (64, 64, 0), (133, 140, 5), (4096, 4096, 1)])
def test_zeros_in_other_rows_alone(H, row, first, dtype):
    T, k, R = 50, 3, 400
    slots = some_slots(T, k, R, torch.Generator().manual_seed(H)).cuda()
    buf = torch.full((R * row + first + 8,), 7.0, dtype=dtype, device="cuda")
    rows = buf[first:first + R * row].view(R, row)[:, :H]
    space = torch.full((R + 1,), 1, dtype=torch.uint8, device="cuda")[1:]
    status = hk.lib().hikonv_zero_other_rows(slots.data_ptr(), T, k, rows.data_ptr(), buf.element_size(), row, R, H, space.data_ptr(), R,
                                             torch.cuda.current_stream().cuda_stream)
    assert status == hk.OK
    named = torch.where(slots >= 0, slots, -2 - slots).flatten()
    named = named[(named >= 0) & (named < R)].long()
    want = torch.full_like(buf, 7.0)
    inner = want[first:first + R * row].view(R, row)
    rest = torch.ones(R, dtype=torch.bool, device="cuda")
    rest[named] = False
    inner[:, :H][rest] = 0.0
    assert torch.equal(buf, want)
