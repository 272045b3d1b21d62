"""MXFP4 products where tiles, lists and index ranges end."""
import numpy as np
import pytest
import torch

from tests.test_mxfp_gpu import TYPES, bound, host, matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,cols,red", [(1, 44, 4096), (1, 300, 4096), (2, 172, 2100), (3, 129, 4096), (20, 4, 4096), (40, 260, 2048), (100, 133, 1030)])
@pytest.mark.parametrize("what", ["linear", "grad", "product"])
def test_split_reductions_whose_last_ranks_have_nothing_to_store(what, M, cols, red):
    """A cluster shares out a tile's columns; past the last one its CTAs leave without having read each other's sums."""
    import paper_2408_10746_b200 as pac
    codes, scales, w = matrix(*((red, cols) if what == "grad" else (cols, red)), 5)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(M, red, generator=g).bfloat16().cuda()
    op, adds = (w if what == "grad" else w.T), red / 16 + 16
    if what == "linear":
        call = lambda: pac.mxfp_linear(x, codes, scales, torch.float32)  # noqa: E731
    elif what == "grad":
        call = lambda: pac.mxfp_linear_grad(x, codes, scales, cols, torch.float32)  # noqa: E731
    else:
        a = pac.quantize_mxfp(x)
        x = pac.dequantize_mxfp(*a, red)
        call = lambda: pac.mxfp_product(*a, codes, scales, red, torch.float32)  # noqa: E731
    ref, size = host(x) @ op, np.abs(host(x)) @ np.abs(op)
    first = call()
    assert (np.abs(host(first) - ref) <= bound(ref, size, adds, TYPES["f32"])).all()
    for _ in range(50):
        assert torch.equal(call(), first)


def test_few_tokens_of_more_than_32_bits_of_values():
    """16 tokens of 2^28 + 512 columns: the last 8192 of the last token are beyond 2^32 values of x."""
    import paper_2408_10746_b200 as pac
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    M, N, K = 16, 4, 2 ** 28 + 512
    codes = torch.full((N, K // 2), 0x22, dtype=torch.uint8, device="cuda")          # 1 everywhere
    codes[1] = 0x44                                              # 2
    scales = torch.full(pac.mxfp_shapes(N, K)[1], 127, dtype=torch.uint8, device="cuda")
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    x[15, -8192:] = (torch.arange(8192, device="cuda") % 64).bfloat16()              # whole numbers: every sum is exact
    x[3, :64] = 1
    x[15, 0] = 5
    y = pac.mxfp_linear(x, codes, scales, torch.float32)
    want = torch.zeros(M, N, device="cuda")
    want[3], want[15] = 64, 5 + 128 * 2016
    want[:, 1] *= 2
    same = torch.equal(y, want)
    del x, codes
    torch.cuda.empty_cache()                                     # 35 GB that other tests may want
    assert same


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 5, 40, 700])
def test_results_beside_their_inputs_in_one_buffer(M, dtype):
    """x in the first columns of a buffer, y, dx and values read back in others; what lies between stays as it was."""
    import paper_2408_10746_b200 as pac
    N, K = 300, 520
    codes, scales, w = matrix(N, K, 8)
    g = torch.Generator().manual_seed(2)
    buf = torch.randn(M, 2600, generator=g).to(dtype).cuda()
    before, apart = buf.clone(), buf[:, :K].clone()
    x, y, dx, back = buf[:, :K], buf[:, 600:600 + N], buf[:, 1000:1000 + K], buf[:, 2000:2000 + K]
    want_y = pac.mxfp_linear(apart, codes, scales)
    want_dx = pac.mxfp_linear_grad(want_y, codes, scales, K)
    pac.mxfp_linear(x, codes, scales, out=y)
    pac.mxfp_linear_grad(y, codes, scales, K, out=dx)
    held = pac.quantize_mxfp(x)
    pac.dequantize_mxfp(*held, K, out=back)
    assert torch.equal(y, want_y) and torch.equal(dx, want_dx) and torch.equal(back, pac.dequantize_mxfp(*pac.quantize_mxfp(apart), K, dtype))
    for t in (y, dx, back):
        first = t.storage_offset()
        t.copy_(before[:, first:first + t.shape[1]])
    assert torch.equal(buf, before)


def test_as_an_autograd_function():
    """How a graph is recorded: the forward call runs without grad mode inside a Function, whose backward pass is the gradient's call."""
    import paper_2408_10746_b200 as pac
    codes, scales, w = matrix(300, 200, 3)

    class Frozen(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return pac.mxfp_linear(x, codes, scales)

        @staticmethod
        def backward(ctx, dy):
            return pac.mxfp_linear_grad(dy.contiguous(), codes, scales, 200)

    x = torch.randn(20, 200, device="cuda", requires_grad=True)
    with pytest.raises(pac.PacError):
        pac.mxfp_linear(x, codes, scales)
    y = Frozen.apply(x)
    dy = torch.randn(20, 300, device="cuda")
    y.backward(dy)
    ref, size = host(dy) @ w, np.abs(host(dy)) @ np.abs(w)
    assert (np.abs(host(x.grad) - ref) <= bound(ref, size, 300 / 16 + 16, torch.float32)).all()
    held = pac.quantize_mxfp(torch.nn.Parameter(torch.randn(40, 64, device="cuda")))          # codes have no gradient: nothing is lost
    assert held[0].shape == (40, 32)
