"""What the low-bit calls refuse or allow, on shapes and addresses alone: stand-ins for CUDA tensors, no device."""
import pytest
import torch

import paper_2408_10746_b200 as pac
from paper_2408_10746_b200 import binding


class Shape:
    """A CUDA tensor's shape and place; reading its address says that the call went on to the kernel."""
    is_cuda, device, requires_grad = True, torch.device("cuda", 0), False

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


def view(at, rows, cols, pitch, dtype=torch.bfloat16):
    return Shape((rows, cols), dtype, (pitch, 1), at)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_columns_of_one_buffer_beside_each_other_lie_apart(dtype):
    """A result and an input as column slices of the same rows: their spans cross, their elements do not."""
    e, P = dtype.itemsize, 200
    x = view(4096, 6, 64, P, dtype)
    fine = [(64, 6, 136), (64, 6, 40), (100, 6, 40), (100, 3, 40), (264, 5, 100), (P * 3 + 64, 2, 136), (64, 1, 136), (P * 5 + 64, 9, 136), (6 * P - 136, 4, 136)]
    for first, rows, cols in fine:
        binding._apart(view(4096 + e * first, rows, cols, P, dtype), x)
        binding._apart(x, view(4096 + e * first, rows, cols, P, dtype))
    for first, rows, cols in [(0, 6, 64), (63, 6, 40), (40, 1, 10), (100, 6, 101), (P - 10, 3, 11), (P * 2, 1, 1), (P * 5 + 63, 1, 1)]:
        for a, b in ((view(4096 + e * first, rows, cols, P, dtype), x), (x, view(4096 + e * first, rows, cols, P, dtype))):
            with pytest.raises(pac.PacError):
                binding._apart(a, b)


def test_overlaps_are_those_of_the_elements():
    """Against the sets of elements, over places, widths and pitches."""
    import random
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(4000):
        P = rng.randint(4, 12)
        a = (rng.randint(0, 40), rng.randint(0, 4), rng.randint(1, P), P)
        Q = P if rng.random() < 0.7 else rng.randint(4, 12)
        b = (rng.randint(0, 40), rng.randint(0, 4), rng.randint(1, Q), Q)
        cells = [{at + r * p + c for r in range(rows) for c in range(cols)} for at, rows, cols, p in (a, b)]
        meet = bool(cells[0] & cells[1])
        args = [view(4096 + 2 * at, rows, cols, p) for at, rows, cols, p in (a, b)]
        try:
            binding._apart(*args)
            refused = False
        except pac.PacError:
            refused = True
        assert refused or not meet                               # never an overlap let through
        if P == Q or min(a[1], b[1]) <= 1:
            assert refused == meet, (a, b)                       # rows of one buffer: exactly the overlaps (others: when their spans cross)
        seen[refused] += 1
    assert min(seen) > 400


@pytest.mark.parametrize("call", [lambda x, m, out: pac.mxfp_linear(x, *m, out=out), lambda x, m, out: pac.mxfp_linear_grad(x, *m, 64, out=out)])
def test_a_gradient_is_not_lost_in_silence(call):
    """The calls record no graph: under grad mode they refuse what requires a gradient, and go on with it without."""
    m = matrix(64, 64)
    needs, plain = Shape((4, 64)), Shape((4, 64))
    needs.requires_grad = True
    for x, out in ((needs, None), (plain, needs)):
        with pytest.raises(pac.PacError) as e:
            call(x, m, out)
        assert e.value.status_name == "PAC_ERR_INVALID_ARG" and "gradient" in str(e.value)
    with torch.no_grad(), pytest.raises(AssertionError, match="went on"):
        call(needs, m, None)
    with pytest.raises(AssertionError, match="went on"):
        call(plain, m, None)
