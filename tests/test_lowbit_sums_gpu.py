"""Long reductions with MXFP4 matrices: what the tensor core cuts off its sums must not add up."""
import pytest
import torch

pytestmark = pytest.mark.gpu
ADDS = 512                                                       # into one accumulator, for a bf16 result


GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def positive(rows, cols, seed, spread=0, top=None):
    """Codes and scales on the GPU of values 0.5 .. 6 (in row r up to code top[r]) times 1 .. 2^-spread, block by block; and rows of the
    values in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks = (cols + 31) // 32
    nib = torch.randint(1, 8, (rows, 32 * blocks), generator=g, device="cuda", dtype=torch.uint8)
    if top is not None:
        nib = nib.clamp(max=top[:, None])
    nib[:, cols:] = 0
    codes = nib[:, 0::2] | (nib[:, 1::2] << 4)
    scales = torch.randint(127 - spread, 128, ((rows + 127) // 128, 2 * ((cols + 255) // 256), 32, 4, 4), generator=g, device="cuda", dtype=torch.uint8)
    grid = torch.tensor(GRID, device="cuda")

    def values(a, b):
        row, block = torch.arange(a, min(b, rows), device="cuda")[:, None], torch.arange(blocks, device="cuda")
        factor = torch.exp2(scales[row // 128, block // 4, row % 32, row % 128 // 32, block % 4].double() - 127)
        return (grid[nib[a:b].int()].double().view(-1, blocks, 32) * factor[:, :, None]).view(-1, 32 * blocks)[:, :cols]
    return codes, scales, values


def mean_cut(y, ref):
    """Mean relative distance of y to the rounded exact result.  Rows are spread evenly over a binade, so a shift of d moves the share
    d / step of the values by one step and the mean by d."""
    best = ref.to(torch.bfloat16)
    return float(((y.double() - best.double()) / ref).mean())


def tolerance(parts):
    """Sums of numbers above 0 grow evenly: the cut after addition n of a part is at most 2^-22 (2^-23, twice for the alignment within
    a product) of n / ADDS of the part's sum, in all 2^-22 (ADDS + 1) / 2 of it; a rounding of 2^-24 for every part added; and the
    mean over 2000 rows of what steps of 2^-7 leave where a share of 1 in 20 moves: 2^-7 (1 / 20 / 2000)^(1/2)."""
    return 2.0 ** -22 * (ADDS + 1) / 2 + parts * 2.0 ** -24 + 2.0 ** -7 * (1 / 20 / 2000) ** 0.5


def spread(rows, cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.rand(rows, cols, generator=g, device="cuda") + 0.5) * (1 + torch.arange(rows, device="cuda") / rows)[:, None]


@pytest.mark.parametrize("grad", [False, True])
def test_bf16_results_of_long_reductions(grad):
    import paper_2408_10746_b200 as pac
    M, out, red = 2000, 1280, 200010
    codes, scales, values = positive(*((red, out) if grad else (out, red)), 1)
    x = spread(M, red, 2).bfloat16()
    y = pac.mxfp_linear_grad(x, codes, scales, out) if grad else pac.mxfp_linear(x, codes, scales)
    ref = torch.zeros(M, out, dtype=torch.float64, device="cuda")
    if grad:
        for a in range(0, red, 40000):
            ref += x[:, a:a + 40000].double() @ values(a, min(red, a + 40000))
    else:
        for a in range(0, out, 256):
            w = values(a, a + 256)
            for b in range(0, red, 40000):
                ref[:, a:a + 256] += x[:, b:b + 40000].double() @ w[:, b:b + 40000].T
    cut = mean_cut(y, ref)
    assert abs(cut) <= tolerance(25), cut


def test_bf16_results_of_long_block_scaled_products():
    import paper_2408_10746_b200 as pac
    M, N, K = 2560, 1024, 600010
    b, bs, bv = positive(N, K, 3, spread=12)
    a, as_, av = positive(M, K, 4, spread=12, top=(1 + 7 * torch.arange(M, device="cuda") // M).to(torch.uint8))
    y = pac.mxfp_product(a, as_, b, bs, K)
    ref = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for r in range(0, N, 512):
        w = bv(r, r + 512)
        for c in range(0, M, 256):
            ref[c:c + 256, r:r + 512] = av(c, c + 256) @ w.T
    cut = mean_cut(y, ref)
    assert abs(cut) <= tolerance(19), cut
