"""The low-bit operators together, as a trainer beside a frozen matrix uses them: hidden states kept in 4 bits, a frozen LM head in
4 bits, the gradient through it, and the adapter's update with 8-bit moments."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_adapter_under_a_frozen_head_in_four_bits():
    import paper_2408_10746_b200 as pac
    torch.manual_seed(0)
    M, d, V, r = 120, 256, 1000, 16
    head = torch.randn(V, d, device="cuda") / d ** 0.5
    codes, scales = pac.quantize_mxfp(head)
    W = pac.dequantize_mxfp(codes, scales, d, torch.float32).double()
    held = pac.quantize_mxfp(torch.randn(M, d, device="cuda").bfloat16())
    h = pac.dequantize_mxfp(*held, d, torch.float32)
    target = torch.randint(0, V, (M,), device="cuda")
    down = torch.randn(d, r, device="cuda") / d ** 0.5
    up = torch.randn(r, d, device="cuda") / r ** 0.5
    params = [down, up]
    grads = [torch.zeros_like(p) for p in params]
    opt = pac.AdamWTensors(params, grads, bits=8)
    for _ in range(4):
        a = h @ down
        y = h + a @ up
        logits = pac.mxfp_linear(y, codes, scales)
        p = torch.softmax(logits, 1)
        dlogits = (p - torch.nn.functional.one_hot(target, V)) / M
        dy = pac.mxfp_linear_grad(dlogits, codes, scales, d)
        grads[1].copy_(a.T @ dy)
        grads[0].copy_(h.T @ (dy @ up.T))
        # the same in 64 bits
        q = [t.double().requires_grad_() for t in params]
        loss = torch.nn.functional.cross_entropy((h.double() + h.double() @ q[0] @ q[1]) @ W.T, target)
        for g, want in zip(grads, torch.autograd.grad(loss, q)):
            assert (g - want).norm() <= 2e-5 * want.norm()       # fp32 sums of up to 1000 terms, twice, and torch's own products
        before = [t.clone() for t in params]
        opt.step(pac.AdamW())
        assert all(t.isfinite().all() and not torch.equal(t, b) for t, b in zip(params, before))
    # the frozen matrix with the states as they are held: the block-scaled product is that of the values
    logits4 = pac.mxfp_product(*held, codes, scales, d, torch.float32)
    want = h.double() @ W.T
    size = h.double().abs() @ W.T.abs()
    assert ((logits4 - want).abs() <= 2.0 ** -24 * want.abs() + (d / 64 + 16) * 2.0 ** -22 * size).all()
