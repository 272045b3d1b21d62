"""AdamW with 8-bit moments at both ends of what fp32 holds."""
import numpy as np
import pytest
import torch

from oracle import lowbit_oracle as lo

pytestmark = pytest.mark.gpu
f = np.float32


def decode(codes, scale):
    sign = np.where(codes >= 128, f(-1), f(1))
    return sign * lo.e4m3_values().astype(f)[codes & 127] * np.repeat(scale, 256)[:codes.size]


def host(t):
    return t.detach().float().cpu().numpy()


def codes_of(t):
    return t.view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("eps", [1e-8, 1e-13, 0.0])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_second_moments_that_are_subnormal(dtype, offset, eps):
    """Blocks of gradients from 2^-75 to 2^-40 in size, alone and beside larger ones: v = (1 - beta2) g^2 is subnormal for most."""
    import paper_2408_10746_b200 as pac
    hp = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": eps, "weight_decay": 0.01}
    n = 256 * 36 + 100
    rng = np.random.default_rng(1)
    size = np.exp2(-75.0 + np.arange(n) // 256)
    mixed = rng.random(n) < 0.05
    size = np.where(mixed & (np.arange(n) // 256 % 3 == 0), np.exp2(rng.uniform(-75, -10, n)), size)
    flat_p, flat_g = torch.randn(n + 8, device="cuda").to(dtype), torch.zeros(n + 8, device="cuda").to(dtype)
    p, g = flat_p[offset:offset + n], flat_g[offset:offset + n]
    opt = pac.AdamWTensors([p], [g], bits=8, seed=5)
    state = opt.state_lists()
    for step in (1, 2, 3):
        g.copy_(torch.from_numpy((rng.standard_normal(n) + 3) * size * rng.choice([-1, 1], n)))
        before = host(p).astype(np.float64)
        m, root = (decode(codes_of(state[k][0]), host(state[k + "_scale"][0])) for k in ("m", "v"))
        grad = host(g)
        m = f(0.9) * m + (f(1) - f(0.9)) * grad
        v = f(0.999) * (root * root) + ((f(1) - f(0.999)) * grad) * grad
        assert ((v > 0) & (v < 2.0 ** -126)).sum() > 2000
        opt.step(pac.AdamW(**hp))
        bits = lo.random_bits(5, step, 0, n)
        for key, value, u, keep in (("m", m, bits & np.uint64(0xFFFF), False), ("v", np.sqrt(v), bits >> np.uint64(16), True)):
            codes, scale = lo.encode_e4m3(np.abs(value), u, keep)
            assert np.array_equal(host(state[key + "_scale"][0]), scale), (key, step)
            assert np.array_equal(codes_of(state[key][0]), codes + 128 * (value < 0)), (key, step)
        b1, b2, lr, wd = (float(f(hp[k])) for k in ("beta1", "beta2", "lr", "weight_decay"))
        bc1, bc2 = float(f(1 - b1 ** step)), float(f(1 - b2 ** step))
        with np.errstate(all="ignore"):
            move = lr * (m.astype(np.float64) / bc1) / (np.sqrt(v.astype(np.float64) / bc2) + float(f(eps)))
        # (eps 0 and a v of 0 have no step: 0.001 g^2 rounds to 0 below 2^-150, for g below 2^-70, which are 3 to 2^73 .. 2^75 below 1:
        # the first four of 37 blocks, some 11 %)
        fine = np.isfinite(move)
        assert fine.mean() > 0.8
        want = before - float(f(lr) * f(wd)) * before - move
        # nine fp32 operations of at most 2 ulp each in the step, four roundings of the parameter, and its own type's
        tol = 18 * 2.0 ** -23 * (np.abs(move) + 1e-5 * np.abs(before)) + 4 * 2.0 ** -24 * np.abs(want) + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0)
        off = np.abs(host(p) - want)
        assert (off[fine] <= tol[fine]).all(), (step, (off / tol)[fine].max())
        p.copy_(torch.where(torch.from_numpy(fine).cuda(), p, 1.0))


@pytest.mark.parametrize("offset", [0, 1])
def test_second_moment_that_overflows_from_a_finite_gradient(offset):
    """v is infinite and the step m / infinity nothing, as with 32 bits; the block's constant says that its moment is not finite."""
    import paper_2408_10746_b200 as pac
    flat = torch.zeros(1032, device="cuda")
    g = flat[offset:offset + 1024]
    g.fill_(1e-3)
    g[300], g[301] = 1e21, -3e22
    ends = []
    for bits in (32, 8):
        store = torch.ones(1032, device="cuda")
        p = store[offset:offset + 1024]
        opt = pac.AdamWTensors([p], [g], bits=bits)
        opt.step(pac.AdamW(lr=1e-3, weight_decay=0.01))
        ends.append(p)
        if bits == 8:
            s = opt.state_lists()
            assert s["v_scale"][0].isnan().tolist() == [False, True, False, False] and s["m_scale"][0].isfinite().all()
    assert ends[1].isfinite().all()
    # steps of 1e-3 by nine operations of at most 2 ulp, four roundings of the parameter
    assert ((ends[0] - ends[1]).abs() <= 18 * 2.0 ** -23 * 1.1e-3 + 4 * 2.0 ** -24).all()
    assert (ends[1][300:302] > 0.9999).all()
