"""What the low-bit calls refuse or allow, on shapes and addresses alone: stand-ins for CUDA tensors, no device."""
import pytest
import torch

import paper_2408_10746_b200 as pac
from paper_2408_10746_b200 import binding


class Shape:
    """A CUDA tensor's shape and place; reading its address says that the call went on to the kernel."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, shape, dtype=torch.bfloat16, stride=None, at=None):
        self.shape, self.dtype, self.at = tuple(shape), dtype, at
        self._stride = stride or tuple(torch.empty(shape, device="meta").stride())

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self._stride

    def numel(self):
        return int(torch.Size(self.shape).numel())

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        assert self.at is not None, "went on to the kernel"
        return self.at


def matrix(rows, cols):
    return tuple(Shape(s, torch.uint8) for s in pac.mxfp_shapes(rows, cols))


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1])
def test_sizes_beyond_32_bits_are_refused_and_not_cut(n):
    small = matrix(64, 64)
    for call in (lambda: pac.mxfp_linear(Shape((n, 64)), *small), lambda: pac.mxfp_linear(Shape((4, n)), *matrix(64, n)), lambda: pac.mxfp_linear(Shape((4, 64)), *matrix(n, 64)),
                 lambda: pac.mxfp_linear_grad(Shape((n, 64)), *small, 64), lambda: pac.mxfp_linear_grad(Shape((4, n)), *matrix(n, 64), 64),
                 lambda: pac.mxfp_linear_grad(Shape((4, 64)), *matrix(64, n), n), lambda: pac.mxfp_product(*matrix(n, 64), *small, 64),
                 lambda: pac.mxfp_product(*small, *matrix(n, 64), 64), lambda: pac.mxfp_product(*matrix(4, n), *matrix(4, n), n),
                 lambda: pac.quantize_mxfp(Shape((4, n))), lambda: pac.quantize_mxfp(Shape((n, 64))), lambda: pac.dequantize_mxfp(*matrix(4, n), n),
                 lambda: pac.dequantize_mxfp(*matrix(n, 64), 64)):
        with pytest.raises(pac.PacError) as e:
            call()
        assert e.value.status_name == "PAC_ERR_INVALID_ARG"
