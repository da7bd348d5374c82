"""CPU: sizes beyond the C interface's 32 bits are refused, not cut off."""
import pytest
import torch

from paper_2208_00763_b200 import binding as hk
from paper_2208_00763_b200 import build as lib_build

BIG = (1 << 32) + 5


@pytest.fixture(scope="module", autouse=True)
def built_library():
    lib_build.build()
    return hk.lib()


class Matrix:
    """Looks like a CUDA matrix of any size, of which all rows are one."""
    is_cuda, layout, device = True, torch.strided, torch.device("cuda:0")

    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, shape

    def dim(self):
        return len(self.shape)

    def stride(self, d):
        return 1 if d in (-1, len(self.shape) - 1) else 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        raise AssertionError("an address was taken")

    def numel(self):
        return 1

    def element_size(self):
        return self.dtype.itemsize


def test_workspace_of_a_sort():
    assert hk.sort_by_expert_workspace_bytes(5000, 1, 8) > 0
    for sizes in ((BIG, 1, 8), (5000, BIG, 8), (5000, 1, BIG), (1 << 31, 1, 8)):
        with pytest.raises(ValueError):
            hk.sort_by_expert_workspace_bytes(*sizes)


@pytest.mark.parametrize("call", [
    lambda m: hk.sort_by_expert(m(torch.int64, BIG, 1), 8),
    lambda m: hk.sort_by_expert(m(torch.int64, 4, BIG), 8),
    lambda m: hk.sort_by_expert(m(torch.int64, 4, 1), BIG),
    lambda m: hk.rows_to_experts(m(torch.uint8, BIG, 16), m(torch.int32, BIG, 1)),
    lambda m: hk.rows_from_experts(m(torch.float32, BIG, 16), m(torch.int32, 4, 1)),
    lambda m: hk.rows_from_experts(m(torch.float32, 4, 16), m(torch.int32, BIG, 1)),
    lambda m: hk.rows_from_experts_grad(m(torch.float32, BIG, 16), None, m(torch.int32, BIG, 1)),
    lambda m: hk.quantize_blocks(m(torch.float32, BIG, 16)),
    lambda m: hk.quantize_blocks(m(torch.float32, 4, BIG)),
    lambda m: hk.quantize_tiles(m(torch.float32, BIG, 16)),
    lambda m: hk.quantize_tiles(m(torch.float32, BIG, 4, 16)),
    lambda m: hk.linear_f8(m(torch.float8_e4m3fn, BIG, 16), m(torch.float8_e4m3fn, 4, 16), m(torch.float32, 1, BIG), m(torch.float32, 1, 1)),
    lambda m: hk.linear_f8(m(torch.float8_e4m3fn, 4, 16), m(torch.float8_e4m3fn, BIG, 16), m(torch.float32, 1, 4), m(torch.float32, 1, 1)),
])
def test_sizes_beyond_32_bits(call):
    with pytest.raises(ValueError, match="2\\^31"):
        call(Matrix)


A, B, C = (0x100000000000 + (i << 40) for i in range(3))
OTHER = dict(slots=A, T=5, k=3, rows=B, size=2, row=64, R=15, H=64, ws=C, ws_bytes=15)


@pytest.mark.parametrize("status,change", [
    (hk.ERR_INVALID_ARG, dict(T=-1)), (hk.ERR_INVALID_ARG, dict(k=0)), (hk.ERR_INVALID_ARG, dict(size=1)), (hk.ERR_INVALID_ARG, dict(size=8)),
    (hk.ERR_INVALID_ARG, dict(H=0)), (hk.ERR_INVALID_ARG, dict(R=-1)), (hk.ERR_INVALID_ARG, dict(slots=None)), (hk.ERR_INVALID_ARG, dict(rows=None)),
    (hk.ERR_INVALID_ARG, dict(row=63)), (hk.ERR_INVALID_ARG, dict(row=1 << 50)), (hk.ERR_INVALID_ARG, dict(rows=B + 1)), (hk.ERR_INVALID_ARG, dict(slots=A + 2)),
    (hk.ERR_UNSUPPORTED, dict(T=1 << 29)), (hk.ERR_UNSUPPORTED, dict(H=(1 << 23) + 1, row=1 << 24)), (hk.ERR_WORKSPACE, dict(ws=None)),
    (hk.ERR_WORKSPACE, dict(ws_bytes=14)), (hk.ERR_INVALID_ARG, dict(ws=A + 59)), (hk.ERR_INVALID_ARG, dict(ws=B - 14)), (hk.ERR_INVALID_ARG, dict(rows=A + 8)),
    (hk.OK, dict(R=0))])
def test_refusals_of_zeros_in_other_rows(status, change):
    assert hk.lib().hikonv_zero_other_rows(*{**OTHER, **change}.values(), None) == status
