"""MXFP4 codec and products on the GPU against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import lowbit_oracle as lo

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def strided(rows, cols, dtype, ld, offset, seed):
    """A matrix whose rows are `ld` elements apart and begin `offset` elements into its storage."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))
    flat = torch.full((rows * ld + offset + 8,), 7.0, dtype=dtype, device="cuda")
    view = flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(x)
    return view, flat


def host(t):
    return t.detach().cpu().double().numpy()


def matrix(rows, cols, seed, spread=8):
    """(codes, scales) on the GPU and the values they stand for, from the oracle's packing; filling bytes are large scales."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    scales = rng.integers(127 - spread, 127 + spread + 1, (rows, (cols + 31) // 32)).astype(np.uint8)
    packed, tiled = lo.pack(codes, scales, pad_scale=254)
    return torch.from_numpy(packed).cuda(), torch.from_numpy(tiled).cuda(), lo.values(codes, scales)


def bound(ref, size, adds, dtype):
    """One rounding of the result, and for every addition of the accumulation a cut of at most 2^-22 of the sum of magnitudes (the
    tensor core drops bits below the fp32 sum instead of rounding: up to 2^-23, twice for the alignment within a product)."""
    return HALF_STEP[dtype] * np.abs(ref) + adds * 2.0 ** -22 * size + 1e-37


# ---------------------------------------------------------------- codec
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 32, 0, 0), (3, 33, 0, 0), (5, 31, 3, 1), (130, 257, 0, 0), (128, 256, 0, 0), (127, 1000, 8, 0),
                                                  (257, 96, 5, 3), (64, 4096, 0, 0), (2, 770, 0, 0), (600, 48, 16, 16)])
def test_codes_scales_and_values_are_the_oracles(rows, cols, pad, offset, dtype):
    import paper_2408_10746_b200 as pac
    x, _ = strided(rows, cols, TYPES[dtype], cols + pad, offset, rows + cols)
    if cols > 40:
        x[rows // 2, 32:40] = 0
    codes, scales = pac.quantize_mxfp(x)
    ref = lo.quantize(host(x))
    packed, tiled = lo.pack(*ref)
    assert np.array_equal(codes.cpu().numpy(), packed)
    assert np.array_equal(scales.cpu().numpy(), tiled)
    for out in TYPES.values():
        y = pac.dequantize_mxfp(codes, scales, cols, out)
        assert y.dtype == out and np.array_equal(host(y), lo.values(*ref))


def test_borders_zeros_subnormals_and_values_that_are_not_finite():
    import paper_2408_10746_b200 as pac
    x = torch.zeros(12, 64)
    x[0, :32] = torch.arange(32) / 4.0                           # every tie of the grid
    x[1, :32] = -torch.arange(32) / 4.0
    x[2, 5] = float("inf")
    x[3, 40] = float("nan")
    x[4] = torch.randn(64) * 2.0 ** -146                         # subnormal, below the smallest scale
    x[5] = torch.randn(64).clamp(-1, 1) * 3e38
    x[6] = torch.tensor(2.0) ** -torch.arange(64)
    x[7, 0] = torch.finfo(torch.float32).max
    x[8] = 7.0                                                   # beyond 6: 6
    x[9, :32] = torch.nextafter(torch.tensor(2.5), torch.tensor(9.0))
    x[10, 63] = -float("inf")
    x[11] = -0.0
    codes, scales = pac.quantize_mxfp(x.cuda())
    ref = lo.quantize(x.double().numpy())
    packed, tiled = lo.pack(*ref)
    assert np.array_equal(scales.cpu().numpy(), tiled)
    got, want = host(pac.dequantize_mxfp(codes, scales, 64, torch.float32)), lo.values(*ref)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[2, :32]).all() and np.isnan(got[3, 32:]).all() and np.isnan(got[10, 32:]).all() and np.isfinite(got[2, 32:]).all()


def test_rows_around_the_result_stay_as_they_were():
    import paper_2408_10746_b200 as pac
    codes, scales, v = matrix(5, 70, 3)
    for dtype in TYPES.values():
        view, flat = strided(5, 70, dtype, 83, 5, 1)
        before = flat.clone()
        pac.dequantize_mxfp(codes, scales, 70, out=view)
        assert np.array_equal(host(view), v)
        view.copy_(before[5:5 + 5 * 83].view(5, 83)[:, :70])
        assert torch.equal(flat, before)


# ---------------------------------------------------------------- products with x as it is
SHAPES = [(1, 1, 1), (1, 4100, 2100), (2, 2500, 1000), (2, 64, 1500), (1, 40000, 300), (3, 300, 100), (16, 23000, 520), (5, 24321, 250), (12, 1100, 4100), (1, 128, 128), (1, 130, 32), (2, 17, 33), (16, 128, 256), (17, 300, 770), (33, 129, 1000), (64, 1, 64), (65, 500, 129), (128, 128, 512),
          (130, 257, 96), (256, 256, 1024), (257, 384, 640), (300, 1000, 250), (7, 64, 4096), (1, 2500, 1030)]


def check_linear(grad, M, N, K, xt, yt, pad=0, offset=0, out_pad=0):
    import paper_2408_10746_b200 as pac
    codes, scales, w = matrix(N, K, M + N + K)
    red, cols = (N, K) if grad else (K, N)
    x, _ = strided(M, red, TYPES[xt], red + pad, offset, M)
    call = (lambda **k: pac.mxfp_linear_grad(x, codes, scales, K, **k)) if grad else (lambda **k: pac.mxfp_linear(x, codes, scales, **k))
    op = w if grad else w.T
    ref, size = host(x) @ op, np.abs(host(x)) @ np.abs(op)
    dtype = TYPES[yt]
    if out_pad:
        view, flat = strided(M, cols, dtype, cols + out_pad, 1, 2)
        before = flat.clone()
        y = call(out=view)
        assert y is view
        keep = torch.ones_like(flat, dtype=torch.bool)
        keep[1:1 + M * (cols + out_pad)].view(M, -1)[:, :cols] = False
        assert torch.equal(flat[keep], before[keep])
    else:
        y = call(dtype=dtype)
    off = np.abs(host(y) - ref)
    assert (off <= bound(ref, size, red / 16 + 16, dtype)).all(), (off / size).max()


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_linear_and_its_gradient_against_64_bits(grad, M, N, K, xt, yt):
    check_linear(grad, M, N, K, xt, yt)


@pytest.mark.parametrize("M,N,K", [(1000, 3000, 136), (520, 8200, 300), (2049, 1300, 520), (700, 2600, 128)])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_many_tokens(grad, M, N, K, xt, yt):
    """Tiles of pairs of CTAs: several to a pair, odd ones at every edge."""
    check_linear(grad, M, *((K, N) if grad else (N, K)), xt, yt)
    check_linear(grad, M, *((K, N) if grad else (N, K)), xt, yt, pad=5, offset=1, out_pad=3)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("xt,yt,pad,offset,out_pad", [("bf16", "f32", 8, 0, 3), ("bf16", "bf16", 3, 0, 8), ("bf16", "bf16", 8, 1, 0), ("f32", "bf16", 4, 0, 5),
                                                      ("f32", "f32", 0, 1, 0), ("f32", "f32", 3, 3, 7)])
def test_pitches_and_alignments(grad, xt, yt, pad, offset, out_pad):
    check_linear(grad, 37, 200, 328, xt, yt, pad, offset, out_pad)
    check_linear(grad, 1, 328, 200, xt, yt, pad, offset, out_pad)


def test_gradient_against_differences():
    """<dy, y(x + h) - y(x - h)> / 2h = <dx, direction>: the product is linear, so the two agree to rounding."""
    import paper_2408_10746_b200 as pac
    codes, scales, _ = matrix(200, 330, 5)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, d = (torch.randn(40, 330, device="cuda", generator=g) for _ in range(2))
    dy = torch.randn(40, 200, device="cuda", generator=g)
    up, down = (pac.mxfp_linear(x + s * d, codes, scales).double() for s in (0.5, -0.5))
    dx = pac.mxfp_linear_grad(dy, codes, scales, 330).double()
    left, right = (dy.double() * (up - down)).sum(), (dx * d.double()).sum()
    # errors of 8000 and 13200 terms of either sum, each below 2^-18 of sum |x||w|: sizes about 330 * 2^8 * 4
    assert abs(left - right) < 2.0 ** -18 * 330 * 2.0 ** 8 * 4 * 8000 ** 0.5 * 4


@pytest.mark.parametrize("which", ["scale", "x"])
def test_not_a_number_stays_in_its_row_or_column(which):
    import paper_2408_10746_b200 as pac
    codes, scales, w = matrix(150, 200, 9)
    x = torch.randn(20, 200, device="cuda").bfloat16()
    if which == "scale":
        scales[1, 0, 3, 0, 2] = 255                              # row 131, columns 64..95
        y = pac.mxfp_linear(x, codes, scales)
        assert y[:, 131].isnan().all() and y.isnan().sum() == 20
        dx = pac.mxfp_linear_grad(torch.randn(20, 150, device="cuda").bfloat16(), codes, scales, 200)
        assert dx[:, 64:96].isnan().all() and dx.isnan().sum() == 20 * 32
        a = pac.quantize_mxfp(x)
        y = pac.mxfp_product(*a, codes, scales, 200)
        assert y[:, 131].isnan().all() and y.isnan().sum() == 20
    else:
        x[7, 11] = float("nan")
        x[9, 12] = float("inf")
        for x_ in (x, x.float()):
            got, want = host(pac.mxfp_linear(x_, codes, scales)), (host(x)[:, None, :] * w[None]).sum(2)
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want)) and np.isinf(want).any()
        y = pac.mxfp_product(*pac.quantize_mxfp(x), codes, scales, 200)
        assert y[[7, 9]].isnan().all() and y[:7].isfinite().all() and y[10:].isfinite().all()


@pytest.mark.parametrize("n", [300, 4000])                        # W converted; x as terms
@pytest.mark.parametrize("xt", ["bf16", "f32"])
def test_few_tokens_with_values_that_are_not_finite_and_of_all_sizes(xt, n):
    """Up to 16 tokens x is a sum of twelve 4-bit matrices: to 2^-23 of the largest of 32 neighbours; infinities and NaN as ever."""
    import paper_2408_10746_b200 as pac
    codes, scales, w = matrix(n, 1100, 21)
    g = torch.Generator().manual_seed(3)
    x = (torch.randn(16, 1100, generator=g) * torch.exp2(torch.randint(-30, 30, (16, 1100), generator=g).float())).to(TYPES[xt]).cuda()
    x[3] = 0
    x[5, 7:40] = 0
    near = host(x)
    top = np.abs(np.pad(near, ((0, 0), (0, 20)))).reshape(16, 35, 32).max(2).repeat(32, 1)[:, :1100]
    y = pac.mxfp_linear(x, codes, scales, torch.float32)
    tol = bound(near @ w.T, np.abs(near) @ np.abs(w.T), 1100 / 16 + 16, torch.float32) + 2.0 ** -23 * (top @ np.abs(w.T))
    assert (np.abs(host(y) - near @ w.T) <= tol).all()
    for m in (1, 2):                                             # the terms are made in the product's kernel there
        assert (np.abs(host(pac.mxfp_linear(x[4:4 + m], codes, scales, torch.float32)) - near[4:4 + m] @ w.T) <= tol[4:4 + m]).all()
    x[2, 500], x[7, 0], x[9, 1099] = float("inf"), float("nan"), -float("inf")
    x[9, 3] = float("inf")
    got, want = host(pac.mxfp_linear(x, codes, scales, torch.float32)), np.stack([(row * w).sum(1) for row in host(x)])
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    assert np.array_equal(np.sign(got[np.isinf(got)]), np.sign(want[np.isinf(want)]))
    for m in (2, 7, 8):
        two, need = host(pac.mxfp_linear(x[m:m + 2], codes, scales, torch.float32)), want[m:m + 2]
        assert np.array_equal(np.isnan(two), np.isnan(need)) and np.array_equal(np.isinf(two), np.isinf(need))
    assert np.array_equal(got[[0, 1, 3, 4, 5, 6, 8]], host(y)[[0, 1, 3, 4, 5, 6, 8]])


def test_filling_bytes_of_the_scales_do_not_matter_to_linear():
    import paper_2408_10746_b200 as pac
    codes, scales, w = matrix(100, 72, 4)
    x, dy = torch.randn(9, 72, device="cuda"), torch.randn(9, 100, device="cuda")
    want = pac.mxfp_linear(x, codes, scales), pac.mxfp_linear_grad(dy, codes, scales, 72)
    row = 32 * torch.arange(4, device="cuda")[None, :, None] + torch.arange(32, device="cuda")[:, None, None]
    block = torch.arange(4, device="cuda")[None, None, :]
    scales[0, 0] = torch.where((row >= 100) | (block >= 3), 255, scales[0, 0])
    scales[0, 1] = 255
    # (few tokens: a sum that a filling byte has made NaN is formed again, by 72 fused operations in fp32: 72 roundings of 2^-24
    # of the sum of magnitudes, less than the (72 / 16 + 16) 2^-22 of bound())
    ref, size = host(x) @ w.T, np.abs(host(x)) @ np.abs(w.T)
    for y in (want[0], pac.mxfp_linear(x, codes, scales)):
        assert (np.abs(host(y) - ref) <= bound(ref, size, 72 / 16 + 16, torch.float32)).all()
    assert torch.equal(pac.mxfp_linear_grad(dy, codes, scales, 72), want[1])
    more = torch.randn(20, 72, device="cuda")
    got = pac.mxfp_linear(more, codes, scales)
    scales[0, 1] = 0
    assert torch.equal(pac.mxfp_linear(more, codes, scales), got) and got.isfinite().all()


@pytest.mark.parametrize("M", [1, 20])
def test_largest_fp32_values(M):
    """The largest fp32 is beyond the largest bf16: its terms are finite all the same."""
    import paper_2408_10746_b200 as pac
    codes = np.full((128, 64), 1, np.uint8)                      # 0.5 everywhere, scale 1
    packed, tiled = lo.pack(codes, np.full((128, 2), 127, np.uint8))
    x = torch.zeros(M, 64, device="cuda")
    x[0, 3], x[M - 1, 40] = torch.finfo(torch.float32).max, -torch.finfo(torch.float32).max
    y = pac.mxfp_linear(x, torch.from_numpy(packed).cuda(), torch.from_numpy(tiled).cuda())
    want = host(x).sum(1) / 2
    assert (np.abs(host(y) - want[:, None]) <= 2.0 ** -22 * 2 * np.abs(host(x)).max() / 2).all()


@pytest.mark.parametrize("s", [0, 1, 60, 200, 240])
def test_extreme_scales_are_exact(s):
    """x = 1 at one column: the result is the value itself, from subnormal powers of two to large ones."""
    import paper_2408_10746_b200 as pac
    codes = np.tile(np.arange(16, dtype=np.uint8), (128, 2))
    packed, tiled = lo.pack(codes, np.full((128, 1), s, np.uint8))
    x = torch.zeros(1, 32)
    x[0, 5] = 1.0 if s else 2.0 ** 20                            # keeps the result among the normal numbers
    y = pac.mxfp_linear(x.cuda(), torch.from_numpy(packed).cuda(), torch.from_numpy(tiled).cuda())
    want = float(lo.values(codes, np.full((128, 1), s, np.uint8))[0, 5]) * float(x[0, 5])
    assert (host(y) == want).all()


# ---------------------------------------------------------------- both operands in 4 bits
@pytest.mark.parametrize("yt", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", SHAPES + [(513, 130, 300), (1, 64, 257), (1000, 3000, 136), (520, 8200, 300), (2049, 1300, 520), (700, 2600, 1280)])
def test_product_of_two_matrices_in_four_bits(M, N, K, yt):
    import paper_2408_10746_b200 as pac
    a, b = matrix(M, K, M + 1), matrix(N, K, N + 2)
    y = pac.mxfp_product(a[0], a[1], b[0], b[1], K, TYPES[yt])
    ref, size = a[2] @ b[2].T, np.abs(a[2]) @ np.abs(b[2].T)
    off = np.abs(host(y) - ref)
    assert (off <= bound(ref, size, K / 64 + 16, TYPES[yt])).all(), (off / size).max()


@pytest.mark.parametrize("n", [256, 5000])
def test_every_scale_and_every_pair_of_codes_in_the_block_scaled_product(n):
    """Row i of A has code i % 16 in column i and 0 elsewhere, so y[i][j] is one product: all pairs, all positions, all scales."""
    import paper_2408_10746_b200 as pac
    K, N = 512, n
    codes = np.zeros((K, K), np.uint8)
    codes[np.arange(K), np.arange(K)] = np.arange(K) % 16
    rng = np.random.default_rng(0)
    sa = rng.integers(90, 165, (K, K // 32)).astype(np.uint8)
    cb, sb = rng.integers(0, 16, (N, K)).astype(np.uint8), rng.integers(90, 165, (N, K // 32)).astype(np.uint8)
    A, B = lo.pack(codes, sa), lo.pack(cb, sb)
    y = pac.mxfp_product(*(torch.from_numpy(t).cuda() for t in (*A, *B)), K, torch.float32)
    assert np.array_equal(host(y), lo.values(codes, sa) @ lo.values(cb, sb).T)


# ---------------------------------------------------------------- the calls themselves
@pytest.mark.parametrize("M,N,dtype", [(50, 700, torch.bfloat16), (50, 700, torch.float32), (1, 700, torch.bfloat16), (7, 5000, torch.bfloat16), (600, 5000, torch.float32)])
def test_calls_repeat_bit_for_bit_and_are_captured(M, N, dtype):
    import paper_2408_10746_b200 as pac
    codes, scales, w = matrix(N, 900, 6)
    x = torch.randn(M, 900, device="cuda").to(dtype)
    dy = torch.randn(M, N, device="cuda").to(dtype)
    y, dx, q = (torch.empty(s, device="cuda") for s in ((M, N), (M, 900), (M, N)))
    xc, xs = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in pac.mxfp_shapes(M, 900))

    def calls():
        pac.mxfp_linear(x, codes, scales, out=y)
        pac.mxfp_linear_grad(dy, codes, scales, 900, out=dx)
        pac.quantize_mxfp(x, xc, xs)
        pac.mxfp_product(xc, xs, codes, scales, 900, out=q)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (1, 2):
        torch.manual_seed(seed)
        x.copy_(torch.randn(M, 900))
        dy.copy_(torch.randn(M, N))
        calls()
        want = [t.clone() for t in (y, dx, q)]
        for t in (y, dx, q):
            t.fill_(float("nan"))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, q), want))


def test_two_streams_at_once():
    import paper_2408_10746_b200 as pac
    mats = [matrix(n, 512, i) for i, n in enumerate((300, 9000))]
    xs = [torch.randn(m, 512, device="cuda").bfloat16() for m in (30, 9)]
    want = [pac.mxfp_linear(x, m[0], m[1]) for x, m in zip(xs, mats)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(pac.mxfp_linear(xs[i], mats[i][0], mats[i][1]))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i]) for i in range(2) for g in got[i])


def test_no_rows():
    import paper_2408_10746_b200 as pac
    codes, scales, _ = matrix(40, 64, 1)
    x = torch.empty(0, 64, device="cuda")
    assert pac.mxfp_linear(x, codes, scales).shape == (0, 40)
    assert pac.mxfp_linear_grad(torch.empty(0, 40, device="cuda"), codes, scales, 64).shape == (0, 64)
    c, s = pac.quantize_mxfp(x)
    assert c.shape == (0, 32) and s.shape == (0, 2, 32, 4, 4)
    assert pac.dequantize_mxfp(c, s, 64).shape == (0, 64)
    assert pac.mxfp_product(c, s, codes, scales, 64).shape == (0, 40)


def test_refusals():
    import paper_2408_10746_b200 as pac
    codes, scales, _ = matrix(40, 64, 1)
    x, wide = torch.randn(4, 64, device="cuda"), torch.randn(4, 200, device="cuda")
    bad = [lambda: pac.mxfp_linear(x[:, :32], codes, scales), lambda: pac.mxfp_linear(x.half(), codes, scales), lambda: pac.mxfp_linear(x.t(), codes, scales),
           lambda: pac.mxfp_linear(x[0], codes, scales), lambda: pac.mxfp_linear(x, codes[:, :16], scales), lambda: pac.mxfp_linear(x, codes, scales[:, :1]),
           lambda: pac.mxfp_linear(x, codes.float(), scales), lambda: pac.mxfp_linear(x, codes, scales.cpu()), lambda: pac.mxfp_linear(x, codes, scales, torch.float16),
           lambda: pac.mxfp_linear(x, codes, scales, out=torch.empty(4, 41, device="cuda")), lambda: pac.mxfp_linear(x[:1].expand(4, 64), codes, scales),
           lambda: pac.mxfp_linear_grad(x, codes, scales, 64), lambda: pac.mxfp_linear_grad(x[:, :40], codes, scales, 96),
           lambda: pac.mxfp_product(codes, scales, codes, scales, 96), lambda: pac.quantize_mxfp(x.half()), lambda: pac.quantize_mxfp(x, codes=codes),
           lambda: pac.dequantize_mxfp(codes, scales, 64, torch.float16), lambda: pac.quantize_mxfp(x.t()),
           lambda: pac.mxfp_linear(wide[:, :64], codes, scales, out=wide[:, 30:70]), lambda: pac.mxfp_linear_grad(wide[:, :40], codes, scales, 64, out=wide[:, :64]),
           lambda: pac.mxfp_product(codes[:4], scales, codes, scales, 64, out=codes.view(torch.bfloat16)[:4])]
    for i, call in enumerate(bad):
        with pytest.raises(pac.PacError) as e:
            call()
        assert e.value.status_name == "PAC_ERR_INVALID_ARG", i
