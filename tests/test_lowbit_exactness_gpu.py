"""What the low-bit calls promise beyond a rounding error's size: operands that enter exactly, the limits of an accumulator on both sides
of every route, and what 8-bit moments hold after many steps."""
import numpy as np
import pytest
import torch

from tests.test_mxfp_gpu import HALF_STEP, TYPES, host, matrix

pytestmark = pytest.mark.gpu


def ones(rows, cols):
    """A matrix of 1: code 2 and scale 127 everywhere."""
    import paper_2408_10746_b200 as pac
    codes, scales = (torch.zeros(s, dtype=torch.uint8, device="cuda") for s in pac.mxfp_shapes(rows, cols))
    full = torch.zeros(rows, codes.shape[1] * 2, dtype=torch.uint8, device="cuda")
    full[:, :cols] = 2
    return full[:, 0::2] | (full[:, 1::2] << 4), scales + 127


def identity(n):
    import paper_2408_10746_b200 as pac
    codes, scales = (torch.zeros(s, dtype=torch.uint8, device="cuda") for s in pac.mxfp_shapes(n, n))
    k = torch.arange(n, device="cuda")
    codes[k, k // 2] = (2 << (4 * (k % 2))).to(torch.uint8)
    return codes, scales + 127


def full_numbers(n, seed):
    """fp32 numbers with all 24 significant bits in use, of many sizes; the first eight bits not all ones, so that the bf16 next to a
    number is of its binade and the number's last bit within the 24 bits of a sum that begins there."""
    g = torch.Generator().manual_seed(seed)
    low = torch.randint(0, 1 << 15, (n,), generator=g) * 2 + 1
    high = torch.randint(0, 127, (n,), generator=g)
    bits = (torch.randint(127 - 60, 127 + 60, (n,), generator=g) << 23) | (high << 16) | low
    return (bits.to(torch.int32).view(torch.float32) * torch.where(torch.rand(n, generator=g) < 0.5, -1.0, 1.0)).cuda()


@pytest.mark.parametrize("M,N,K", [(20, 300, 770), (130, 140, 520), (300, 5000, 400), (700, 2600, 200)])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1)])
def test_fp32_tokens_enter_with_all_their_bits(grad, M, N, K, pad, offset):
    """One number in every row and a matrix of ones: the result is the number, bit for bit."""
    import paper_2408_10746_b200 as pac
    rows, cols = (K, N) if grad else (N, K)                      # the tiles of y are the same in both directions
    codes, scales = ones(rows, cols)
    red = rows if grad else cols
    flat = torch.zeros(M * (red + pad) + offset + 8, device="cuda")
    x = flat[offset:offset + M * (red + pad)].view(M, red + pad)[:, :red]
    v = full_numbers(M, M)
    m = torch.arange(M, device="cuda")
    x[m, (m * 37 + 5) % red] = v
    y = pac.mxfp_linear_grad(x, codes, scales, cols) if grad else pac.mxfp_linear(x, codes, scales)
    assert torch.equal(y, v[:, None].expand(M, N))


@pytest.mark.parametrize("M", [1, 2, 3, 16])
def test_few_tokens_enter_as_the_sum_of_their_terms(M):
    """Through an identity: bf16 values within 2^14 of each other come out as they are, fp32 ones to 2^-23 of the largest of their 32."""
    import paper_2408_10746_b200 as pac
    n = 2048                                                     # 4 M values: few tokens are a sum of terms there
    codes, scales = identity(n)
    g = torch.Generator().manual_seed(M)
    block = torch.exp2(torch.randint(-60, 60, (M, n // 32), generator=g).float()).repeat_interleave(32, 1)
    x = (1 + torch.rand(M, n, generator=g)) * torch.exp2(-torch.randint(0, 14, (M, n), generator=g).float()) * torch.where(torch.rand(M, n, generator=g) < 0.5, -1, 1) * block
    exact = x.bfloat16().cuda()
    assert torch.equal(pac.mxfp_linear(exact, codes, scales, torch.float32), exact.float())
    x = x.cuda()
    top = x.abs().view(M, -1, 32).amax(2).repeat_interleave(32, 1)
    off = (pac.mxfp_linear(x, codes, scales) - x).abs()
    assert (off <= 2.0 ** -23 * top).all() and (off > 0).any()


# one accumulator takes at most 128 additions for an fp32 result and 512 for a bf16 one (64 products each in a block-scaled one, else
# 16), each of which cuts at most 2^-22 of the sum of magnitudes; an fp32 x adds 256 of its smaller terms, 2^-8 of the sizes, which
# is one addition's worth; and at most 16 sums of parts, accumulators or CTAs are rounded
def bound(ref, size, dtype):
    return HALF_STEP[dtype] * np.abs(ref) + ((128 if dtype == torch.float32 else 512) + 1 + 16) * 2.0 ** -22 * size


@pytest.mark.parametrize("red", [4096, 4200, 8192, 16500])
@pytest.mark.parametrize("M,out", [(300, 5000), (150, 400)])
@pytest.mark.parametrize("grad", [False, True])
def test_long_reductions_on_both_sides_of_every_limit(grad, M, out, red):
    import paper_2408_10746_b200 as pac
    rng = np.random.default_rng(red)
    rows, cols = (red, out) if grad else (out, red)
    codes, scales, values = matrix(rows, cols, 7, spread=3)
    x = torch.from_numpy(rng.standard_normal((M, red)).astype(np.float32)).cuda()
    op = values if grad else values.T
    for xt in TYPES.values():
        xs = x.to(xt)
        ref, size = host(xs) @ op, np.abs(host(xs)) @ np.abs(op)
        for yt in TYPES.values():
            y = pac.mxfp_linear_grad(xs, codes, scales, cols, yt) if grad else pac.mxfp_linear(xs, codes, scales, yt)
            off = np.abs(host(y) - ref)
            assert (off <= bound(ref, size, yt)).all(), (xt, yt, (off / size).max())


@pytest.mark.parametrize("K", [8192, 8300, 33000])
@pytest.mark.parametrize("M,N", [(300, 5000), (150, 400)])
def test_long_block_scaled_products_on_both_sides_of_every_limit(M, N, K):
    import paper_2408_10746_b200 as pac
    a, b = matrix(M, K, 1, spread=3), matrix(N, K, 2, spread=3)
    ref, size = a[2] @ b[2].T, np.abs(a[2]) @ np.abs(b[2].T)
    for yt in TYPES.values():
        off = np.abs(host(pac.mxfp_product(a[0], a[1], b[0], b[1], K, yt)) - ref)
        assert (off <= bound(ref, size, yt)).all(), (yt, (off / size).max())


def test_eight_bits_move_as_far_as_32_and_to_the_same_place():
    """60 noisy steps on |p|^2 / 2.  m is off by at most half a code's gap (1/16) times (1 - 0.81)^-1/2: 14 % of itself, v by
    1/8 ((1/60)^2 + .. + 1)^(1/2) / .. : at most 56 %, the root 28 %.  So the way differs by less than 0.14 + 0.28 of its length, and
    along it, where the errors of 65536 elements average out, by the mean of 1 / root: some 0.28^2."""
    import paper_2408_10746_b200 as pac
    ways = []
    for bits in (32, 8):
        g = torch.Generator(device="cuda").manual_seed(0)
        p = torch.randn(65536, device="cuda", generator=g)
        start, grad = p.clone(), torch.empty_like(p)
        opt = pac.AdamWTensors([p], [grad], bits=bits, seed=1)
        for _ in range(60):
            grad.copy_(p + 0.1 * torch.randn(65536, device="cuda", generator=g))
            opt.step(pac.AdamW(lr=1e-2))
        ways.append((p - start).double())
    length = ways[0].norm()
    assert length > 0.2 * 256                                    # 60 steps of up to 0.01 each for 256^2 elements
    assert (ways[1] - ways[0]).norm() < 0.42 * length
    assert abs(float(ways[1] @ ways[0] / length ** 2) - 1) < 0.28 ** 2


@pytest.mark.parametrize("sigma", [0.0, 2.0])
def test_what_second_moments_hold_after_many_steps(sigma):
    """The root's code is rounded without bias, so its square has the rounding's variance on top.  With gaps h of 1/16 to 1/8 of a root
    and moves of (1 - beta2) / 2 |g^2 / v - 1|, some 4.8e-4 of it, a step adds a variance of 4.8e-4 h, and moments forget at
    1 - beta2 = 1e-3: the root has 12 to 17 % of noise and v is 3 to 6 % too large; twice over the exact sum's own spread."""
    import paper_2408_10746_b200 as pac
    n = 65536
    g = torch.Generator(device="cuda").manual_seed(3)
    size = torch.exp(sigma * torch.randn(n, device="cuda", generator=g)) * 1e-3
    p, grad = torch.zeros(n, device="cuda"), torch.empty(n, device="cuda")
    opt = pac.AdamWTensors([p], [grad], bits=8, seed=2)
    exact = torch.zeros(n, dtype=torch.float64, device="cuda")
    state, ratios = opt.state_lists(), []
    for t in range(4000):
        grad.copy_(size * torch.randn(n, device="cuda", generator=g))
        opt.step(pac.AdamW())
        exact.mul_(0.999).add_(grad.double() ** 2, alpha=1e-3)
        if t >= 2000 and t % 200 == 0:
            root = state["v"][0].double() * state["v_scale"][0].double().repeat_interleave(256)
            ratios.append(root ** 2 / exact)
    r = torch.stack(ratios)
    assert 1.0 < float(r.mean()) < 1.10
    assert 0.10 < float(r.sqrt().std()) < 0.20


def test_what_lies_far_below_a_blocks_largest_moment_is_held_too_large():
    """A block holds roots from its largest down to 1 / 229376 of it; those below are held as the smallest code and not as 0."""
    import paper_2408_10746_b200 as pac
    p, grad = torch.zeros(256, device="cuda"), torch.full((256,), 1e-9, device="cuda")
    grad[0] = 1.0
    opt = pac.AdamWTensors([p], [grad], bits=8, decay=[False])
    opt.step(pac.AdamW())
    s = opt.state_lists()
    held = s["v"][0].float() * s["v_scale"][0]
    assert (s["v"][0].view(torch.uint8)[1:] == 1).all()
    assert abs(float(held[0] / held[1]) - 229376) < 1 and float(held[1]) > 1e2 * 1e-9 * 0.001 ** 0.5


@pytest.mark.parametrize("M", [1, 2, 16, 20, 130])
def test_tokens_near_the_end_of_fp32s_range(M):
    """The smallest scale is 2^-127 and the smallest bf16 2^-133: few tokens enter to 2^-23 of the largest of 32 or to 2^-129, fp32 ones of
    more tokens to 2^-134, and exactly from 2^-110 on.  W is 2^60 times an identity, so that the results are normal numbers."""
    import paper_2408_10746_b200 as pac
    n = 2048
    codes, scales = identity(n)
    scales += 60
    g = torch.Generator().manual_seed(M)
    size = torch.exp2(torch.randint(-140, -90, (M, n // 32), generator=g).float()).repeat_interleave(32, 1)
    x = (torch.randn(M, n, generator=g) * size).cuda()
    y = pac.mxfp_linear(x, codes, scales).double()
    want = x.double() * 2.0 ** 60
    if M <= 16:
        top = x.double().abs().view(M, -1, 32).amax(2).repeat_interleave(32, 1)
        off = (2.0 ** -23 * top).clamp(min=2.0 ** -129)
    else:
        off = torch.where(x.abs() < 2.0 ** -110, 2.0 ** -134, 0.0).double()
    # a cut of 2^-22 of the sum for each of the three or twelve terms
    assert ((y - want).abs() <= 2.0 ** 60 * off + 12 * 2.0 ** -22 * want.abs()).all(), ((y - want).abs() / 2.0 ** 60).max()
