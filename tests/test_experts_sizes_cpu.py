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
