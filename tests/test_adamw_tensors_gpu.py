"""AdamW over lists of tensors against the oracle, and against pac_adam_step."""
import numpy as np
import pytest
import torch

from oracle import lowbit_oracle as lo

pytestmark = pytest.mark.gpu
HP = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [1, 3, 12, 255, 256, 257, 512, 2048, 5000, 70001]


def tensors(sizes, dtype, gap, scale, seed):
    """Views of one flat tensor, `gap` elements between them (so their alignments differ)."""
    g = torch.Generator().manual_seed(seed)
    flat = (torch.randn(sum(sizes) + gap * len(sizes) + gap, generator=g) * scale).to(dtype).cuda()
    at, out = gap, []
    for n in sizes:
        out.append(flat[at:at + n])
        at += n + gap
    return out, flat


def f32(t):
    return t.detach().float().cpu().numpy()


@pytest.mark.parametrize("gap", [0, 1, 256])
@pytest.mark.parametrize("pt,gt", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_against_the_oracle(bits, pt, gt, gap):
    import paper_2408_10746_b200 as pac
    params, flat = tensors(SIZES, TYPES[pt], gap, 0.1, 1)
    grads, _ = tensors(SIZES, TYPES[gt], gap, 1e-3, 2)
    decay = [i % 3 != 0 for i in range(len(SIZES))]
    opt = pac.AdamWTensors(params, grads, bits=bits, decay=decay, seed=9)
    state, hp = opt.state_lists(), pac.AdamW(**HP)
    e4m3 = lo.e4m3_values().astype(np.float32)
    dec = lambda c, s: np.where(c >= 128, np.float32(-1), np.float32(1)) * e4m3[c & 127] * np.repeat(s, 256)[:c.size]  # noqa: E731
    for step in (1, 2, 3):
        before = []
        for i in range(len(SIZES)):
            m, v = state["m"][i], state["v"][i]
            if bits == 8:
                m, root = (dec(t.view(torch.uint8).cpu().numpy(), f32(s[i])) for t, s in ((m, state["m_scale"]), (v, state["v_scale"])))
                v = root * root
            else:
                m, v = f32(m), f32(v)
            before.append((f32(params[i]), m, v))
        opt.step(hp, grad_scale=0.5)
        for i, n in enumerate(SIZES):
            p, m, v = lo.adamw(before[i][0], f32(grads[i]), before[i][1], before[i][2], HP, step, decay[i], 0.5)
            if bits == 32:
                assert np.array_equal(f32(state["m"][i]), m) and np.array_equal(f32(state["v"][i]), v), (step, i)
                want = torch.from_numpy(p).to(TYPES[pt])
                assert torch.equal(params[i].cpu(), want), (step, i)
                continue
            rnd = lo.random_bits(9, step, i, n)
            codes, consts = lo.encode_e4m3(np.abs(m), rnd & np.uint64(0xFFFF), False)
            assert np.array_equal(f32(state["m_scale"][i]), consts)
            assert np.array_equal(state["m"][i].view(torch.uint8).cpu().numpy(), codes + 128 * (m < 0))
            codes, consts = lo.encode_e4m3(np.sqrt(v), rnd >> np.uint64(16), True)
            assert np.array_equal(f32(state["v_scale"][i]), consts)
            assert np.array_equal(state["v"][i].view(torch.uint8).cpu().numpy(), codes)
            # the update itself is a chain of nine fp32 operations of at most 2 ulp each, the parameter another four
            step_size = np.abs(before[i][0] - p) + 1e-3 * 1e-2 * np.abs(p)
            off = np.abs(f32(params[i]).astype(np.float64) - p)
            tol = 18 * 2.0 ** -23 * step_size + 4 * 2.0 ** -24 * np.abs(p)
            assert (off <= tol + (2.0 ** -8 * np.abs(p) if pt == "bf16" else 0)).all(), (step, i)
        opt_between = flat.clone()
    keep = torch.ones_like(flat, dtype=torch.bool)
    at = gap
    for n in SIZES:
        keep[at:at + n] = False
        at += n + gap
    assert torch.equal(flat[keep], tensors(SIZES, TYPES[pt], gap, 0.1, 1)[1][keep]) and torch.equal(flat, opt_between)


def test_32_bits_is_the_frameworks_own_step():
    """The adapters of a small trainer, stepped by pac_adam_step and as a list of tensors: the same bits."""
    import pac_inputs as pi
    import paper_2408_10746_b200 as pac
    spec = pi.CONFIGS["tiny_fp32"]
    ctx = pac.PacContext(0)
    ctx.cache_register(pi.cache_full(spec, 0, "cuda"), pi.labels(spec, 0, "cuda"))
    ctx.adapter_init(r=spec.r, n_out=spec.n_out, max_batch=spec.B)
    ctx.set_params(pi.random_params(spec, 3))
    L, d, r, c = spec.L, spec.d, spec.r, spec.n_out
    sizes, decay = [L * d * r, L, r * d, d * c, c], [True, False, True, True, False]
    p = torch.from_numpy(ctx.get_params()).cuda()
    g = torch.zeros_like(p)
    opt = pac.AdamWTensors(list(p.split(sizes)), list(g.split(sizes)), decay=decay)
    for step in range(3):
        ctx.train_step(list(range(step, step + spec.B)))
        g.copy_(torch.from_numpy(ctx.get_grads()))
        ctx.adam_step(pac.AdamW())
        opt.step(pac.AdamW())
        ctx.sync()
        assert np.array_equal(ctx.get_params(), p.cpu().numpy())
    m, v, t = ctx.get_opt_state()
    assert t == opt.steps and np.array_equal(m, torch.cat(opt.state_lists()["m"]).cpu().numpy()) and np.array_equal(v, torch.cat(opt.state_lists()["v"]).cpu().numpy())
    ctx.close()


@pytest.mark.parametrize("count", [48, 49, 480, 481, 1000])
@pytest.mark.parametrize("bits", [32, 8])
def test_long_lists_with_empty_tensors(count, bits):
    import paper_2408_10746_b200 as pac
    rng = np.random.default_rng(count)
    sizes = [int(n) for n in rng.integers(0, 700, count)]
    sizes[0] = sizes[-1] = 0
    params, _ = tensors(sizes, torch.float32, 0, 0.1, 1)
    grads, _ = tensors(sizes, torch.float32, 0, 1e-2, 2)
    before = [f32(t) for t in params]
    opt = pac.AdamWTensors(params, grads, bits=bits, seed=3)
    opt.step(pac.AdamW(**HP))
    e4m3 = lo.e4m3_values()
    for i, n in enumerate(sizes):
        p, m, v = lo.adamw(before[i], f32(grads[i]), np.zeros(n, np.float32), np.zeros(n, np.float32), HP, 1, True)
        assert np.allclose(f32(params[i]), p, rtol=4 * 2.0 ** -24, atol=18 * 2.0 ** -23 * 1.1e-3)
        if bits == 8 and n:
            codes, consts = lo.encode_e4m3(np.abs(m), lo.random_bits(3, 1, i, n) & np.uint64(0xFFFF), False)
            assert np.array_equal(state_codes(opt, "m", i), codes + 128 * (m < 0))
    assert e4m3.size == 128


def state_codes(opt, name, i):
    return opt.state_lists()[name][i].view(torch.uint8).cpu().numpy()


def test_gradients_that_are_not_finite():
    import paper_2408_10746_b200 as pac
    p = torch.ones(1024, device="cuda")
    g = torch.full((1024,), 1e-3, device="cuda")
    g[300], g[800] = float("inf"), float("nan")
    for bits in (32, 8):
        q = p.clone()
        opt = pac.AdamWTensors([q], [g], bits=bits)
        opt.step(pac.AdamW(**HP))
        bad = torch.zeros(1024, dtype=torch.bool, device="cuda")
        bad[300] = bad[800] = True
        assert torch.equal(~q.isfinite(), bad)
        s = opt.state_lists()
        if bits == 8:
            for k in ("m_scale", "v_scale"):
                assert s[k][0].isnan().tolist() == [False, True, False, True]
            assert not s["m"][0].view(torch.uint8)[256:512].any()
        else:
            assert torch.equal(~s["m"][0].isfinite(), bad)


def test_moments_of_zero_and_roots_that_must_not_vanish():
    import paper_2408_10746_b200 as pac
    p, g = torch.ones(512, device="cuda"), torch.zeros(512, device="cuda")
    g[0] = 1.0
    g[1] = 1e-7                                                  # its root is far below the smallest code of the block
    opt = pac.AdamWTensors([p], [g], bits=8, decay=[False])
    opt.step(pac.AdamW(**HP))
    codes = opt.state_lists()["v"][0].view(torch.uint8)
    assert codes[0] == 126 and codes[1] >= 1 and not codes[2:].any() and (p[2:] == 1).all()
    g.zero_()
    for _ in range(20):
        opt.step(pac.AdamW(**HP))
    assert p.isfinite().all() and (p - 1).abs().max() < 0.05 and (p[2:] == 1).all()


def test_eight_bits_follow_32_on_a_quadratic():
    """Steps on |p|^2 / 2 with noise: both walk to the same place at the same pace."""
    import paper_2408_10746_b200 as pac
    ends = []
    for bits in (32, 8):
        torch.manual_seed(0)
        p = torch.randn(4096, device="cuda")
        g = torch.empty_like(p)
        opt = pac.AdamWTensors([p], [g], bits=bits, seed=1)
        for _ in range(60):
            g.copy_(p + 0.1 * torch.randn(4096, device="cuda"))
            opt.step(pac.AdamW(lr=1e-2))
        ends.append(p)
    assert ends[1].isfinite().all() and not torch.equal(*ends)


def test_captured_steps_take_their_number_from_the_device():
    import paper_2408_10746_b200 as pac
    for bits in (32, 8):
        params, _ = tensors(SIZES, torch.float32, 0, 0.1, 1)
        grads, flat = tensors(SIZES, torch.float32, 0, 1e-3, 2)
        copies = [p.clone() for p in params]
        eager = pac.AdamWTensors(copies, grads, bits=bits, seed=4)
        opt = pac.AdamWTensors(params, grads, bits=bits, seed=4)
        number = torch.zeros(1, dtype=torch.int64, device="cuda")
        hp = pac.AdamW(**HP)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            number.add_(1)
            opt.step(hp, step=number)
        for _ in range(3):
            flat.mul_(1.3)
            graph.replay()
            eager.step(hp)
        assert number.item() == 3 and eager.steps == 3 and opt.steps == 0
        assert all(torch.equal(a, b) for a, b in zip(params, copies))
        for k, lists in opt.state_lists().items():
            for a, b in zip(lists, eager.state_lists()[k]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), k
        failed = None
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            number.add_(1)
            try:
                opt.step(hp)
            except pac.PacError as e:
                failed = e
        assert failed is not None and failed.status_name == "PAC_ERR_BAD_STATE"


def test_refusals():
    import paper_2408_10746_b200 as pac
    p, g = torch.zeros(600, device="cuda"), torch.zeros(600, device="cuda")
    s8 = pac.AdamWTensors([p], [g], bits=8).state_lists()
    bad = [lambda: pac.AdamWTensors([p], [g[:599]]), lambda: pac.AdamWTensors([p, p], [g, g]), lambda: pac.AdamWTensors([p, p[10:20]], [g, g[:10]]),
           lambda: pac.AdamWTensors([p], [p]), lambda: pac.AdamWTensors([p.half()], [g.half()]), lambda: pac.AdamWTensors([p[::2]], [g[::2]]),
           lambda: pac.AdamWTensors([p], [g], state=s8), lambda: pac.AdamWTensors([p], [g], bits=8, state={**s8, "m_scale": [torch.zeros(2, device="cuda")]}),
           lambda: pac.AdamWTensors([p], [g], decay=[]), lambda: pac.AdamWTensors([p], [g.cpu()]),
           lambda: pac.AdamWTensors([p], [g]).step(pac.AdamW(), step=torch.ones(1, device="cuda"))]
    for i, call in enumerate(bad):
        with pytest.raises(pac.PacError) as e:
            call()
        assert e.value.status_name == "PAC_ERR_INVALID_ARG", i
    pac.AdamWTensors([], []).step(pac.AdamW())
    pac.AdamWTensors([p[:0]], [g[:0]]).step(pac.AdamW())
