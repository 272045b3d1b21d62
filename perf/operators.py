"""Operators around what a trainer keeps in few bits, as a user's program runs them.

A frozen matrix in microscaled 4-bit floating point (MXFP4: values of E2M1, one power of two for every 32 of them),
the products with it, and the optimizer's moments in 8 bits or in 32.  A case is a dict of plain values with an "op":

    codec     quantize_mxfp of x [rows][cols] and dequantize_mxfp of the result
    linear    mxfp_linear: y [M][N] = x [M][K] W^T, W [N][K] in 4 bits, x as it is
    grad      mxfp_linear_grad: dx [M][K] = dy [M][N] W
    product   quantize_mxfp of x, then mxfp_product: both operands of y = x W^T in 4 bits
    adamw     one AdamW step over all tensors of a list (AdamWTensors)

Layouts.  codes: uint8 [rows][16 * ceil(cols / 32)], two values to a byte, the even column in the low half; a value is a
sign bit and three bits that number 0, 0.5, 1, 1.5, 2, 3, 4, 6.  scales: uint8 [ceil(rows / 128)][2 * ceil(cols / 256)][32][4][4];
byte [R][C][i][j][b] belongs to row 128 R + 32 j + i and to the columns 32 (4 C + b) and following; e stands for 2^(e - 127).
Eight-bit moments: one float8 (E4M3) per element times an fp32 constant per 256 elements; the second moment is held as its root.
"""
import math

import numpy as np
import torch

own = False

HP = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FLOP_MOST = 2.0 * 8192 * 11008 * 4096          # the largest listed product
ADAM_SEED = 17

# tensors of the adapters (W_down of every layer, lambda, W_up, head) and of whole layers that are trained in full
ADAPTERS_T5_BASE = [768 * 64] * 12 + [12, 64 * 768, 768 * 3, 3]
ADAPTERS_7B = [4096 * 64] * 32 + [32, 64 * 4096, 4096 * 2, 2]
LAYER_7B = [4096 * 4096] * 4 + [11008 * 4096] * 3 + [4096] * 2


def listed():
    return [
        # one feed-forward matrix of a 7B backbone put into 4 bits and read back in bf16, as when a checkpoint is loaded
        {"name": "codec_ffn_matrix", "op": "codec", "rows": 11008, "cols": 4096, "x": "f32", "y": "bf16"},
        # hidden states of 20 short samples of 30 tokens, kept in 4 bits and read back: the smallest call
        {"name": "codec_hidden_states", "op": "codec", "rows": 600, "cols": 768, "x": "bf16", "y": "bf16"},
        # one token through a square projection of a 7B layer: the call whose latency counts
        {"name": "linear_one_token", "op": "linear", "M": 1, "N": 4096, "K": 4096, "x": "bf16", "y": "bf16"},
        # the last tokens of 16 samples through a frozen LM head
        {"name": "linear_head_16_tokens", "op": "linear", "M": 16, "N": 32000, "K": 4096, "x": "bf16", "y": "f32"},
        # the first epoch's forward, 16 samples of 512 tokens through a feed-forward matrix
        {"name": "linear_ffn_8192_tokens", "op": "linear", "M": 8192, "N": 11008, "K": 4096, "x": "bf16", "y": "bf16"},
        # gradient through a frozen LM head, four samples of 512 tokens
        {"name": "grad_head_2048_tokens", "op": "grad", "M": 2048, "N": 32000, "K": 4096, "x": "bf16", "y": "bf16"},
        # fp32 gradients of 10 samples of 30 tokens through a head of 1000 classes on an odd width
        {"name": "grad_ragged_f32", "op": "grad", "M": 300, "N": 1000, "K": 770, "x": "f32", "y": "f32"},
        # activations quantised on the way: short samples through a fused query, key, value projection
        {"name": "product_short_samples", "op": "product", "M": 600, "N": 2304, "K": 768, "x": "bf16", "y": "f32"},
        # the first epoch's forward with both operands in 4 bits
        {"name": "product_ffn_8192_tokens", "op": "product", "M": 8192, "N": 11008, "K": 4096, "x": "bf16", "y": "bf16"},
        # the adapters of a T5-Base-shaped stack, one flat fp32 vector whose tensors begin where the last one ends
        {"name": "adamw32_adapters_t5_base", "op": "adamw", "bits": 32, "tensors": "adapters_t5_base", "p": "f32", "g": "f32", "packed": True},
        # the adapters of a 7B-shaped stack with their moments in 8 bits
        {"name": "adamw8_adapters_7b", "op": "adamw", "bits": 8, "tensors": "adapters_7b", "p": "f32", "g": "f32", "packed": False},
        # one whole 7B layer in bf16, moments in 8 bits: the largest update
        {"name": "adamw8_layer_7b", "op": "adamw", "bits": 8, "tensors": "layer_7b", "p": "bf16", "g": "bf16", "packed": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["codec", "linear", "linear", "grad", "product", "adamw"])
    x, y = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "f32"])
    if op == "codec":
        return {"op": op, "rows": _log(rng, 1, 11008), "cols": _log(rng, 32, 4096), "x": x, "y": y}
    if op == "adamw":
        count = rng.randint(1, 120)
        sizes = ",".join(str(_log(rng, 1, 20000000 // count)) for _ in range(count))
        return {"op": op, "bits": rng.choice([8, 32]), "tensors": sizes, "p": x, "g": rng.choice([x, "f32"]), "packed": rng.random() < 0.5}
    while True:
        case = {"op": op, "M": _log(rng, 1, 8192), "N": _log(rng, 16, 32000), "K": _log(rng, 32, 11008), "x": x, "y": y}
        if 2.0 * case["M"] * case["N"] * case["K"] * (6 if x == "f32" else 1) <= FLOP_MOST:
            return case


def _sizes(case):
    known = {"adapters_t5_base": ADAPTERS_T5_BASE, "adapters_7b": ADAPTERS_7B, "layer_7b": LAYER_7B}
    return known[case["tensors"]] if case["tensors"] in known else [int(s) for s in case["tensors"].split(",")]


# --------------------------------------------------------------------------- inputs
# bytes of two codes each, as rounding a normal variable gives them: its largest of 32 lies between 4 and 8
_NORMAL_NIBBLES = None


def _nibbles(device):
    global _NORMAL_NIBBLES
    if _NORMAL_NIBBLES is None:
        u = (torch.arange(256, dtype=torch.float64) + 0.5) / 256
        v = torch.erfinv(2 * u - 1) * math.sqrt(2) * 2.4
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
        mag = (v.abs()[:, None] - grid).abs().argmin(1)
        _NORMAL_NIBBLES = (mag + 8 * (v < 0)).to(torch.uint8)
    return _NORMAL_NIBBLES.to(device)


def _weights(rows, cols, gen):
    """Codes and scales of a frozen matrix whose entries are about 1 / sqrt(cols) in size; zeros past the last column."""
    table, blocks = _nibbles("cuda"), (cols + 31) // 32
    draw_ = lambda: torch.randint(0, 256, (rows, 16 * blocks), generator=gen, device="cuda", dtype=torch.uint8)  # noqa: E731
    lo, hi = table[draw_().int()], table[draw_().int()]
    first = 2 * torch.arange(16 * blocks, device="cuda")
    codes = torch.where(first < cols, lo, 0) + 16 * torch.where(first + 1 < cols, hi, 0)
    middle = 127 - round(math.log2(2.4 * math.sqrt(cols)))
    shape = ((rows + 127) // 128, 2 * ((cols + 255) // 256), 32, 4, 4)
    scales = torch.randint(middle - 1, middle + 2, shape, generator=gen, device="cuda", dtype=torch.uint8)
    return codes.to(torch.uint8), scales


def _layout(sizes, packed):
    at, offsets = 0, []
    for n in sizes:
        offsets.append(at)
        at += n if packed else (n + 255) // 256 * 256
    return offsets, at


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    op = case["op"]
    if op == "adamw":
        sizes = _sizes(case)
        offsets, total = _layout(sizes, case["packed"])
        blocks = [(n + 255) // 256 for n in sizes]
        boff = [sum(blocks[:i]) for i in range(len(blocks))]
        # gradients whose size differs from part to part of the vector, moments as after some hundred steps of them
        size = torch.exp(rand(total // 512 + 1)).repeat_interleave(512)[:total] * 1e-3
        p, g, steps = (rand(total) * 0.02).to(TYPES[case["p"]]), (rand(total) * size).to(TYPES[case["g"]]), 400
        s = {"case": case, "p": p, "g": g, "steps": steps, "offsets": offsets, "sizes": sizes, "blocks": blocks, "boff": boff}
        if case["bits"] == 32:
            s["m"], s["v"] = rand(total) * size * 0.23, size * size * 0.33 * (1 + 0.1 * torch.rand(total, generator=gen, device="cuda"))
        else:
            # codes of the two moments, and the blocks' constants (the largest of a block is code 126 times its constant)
            nb = sum(blocks)
            m = torch.randint(40, 127, (total,), generator=gen, device="cuda", dtype=torch.uint8)
            sign = torch.randint(0, 2, (total,), generator=gen, device="cuda", dtype=torch.uint8) * 128
            s["m"] = (m + sign).view(torch.float8_e4m3fn)
            s["v"] = torch.randint(90, 127, (total,), generator=gen, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
            c = torch.exp(0.3 * rand(nb)) * 1e-3 / 448
            s["m_scale"], s["v_scale"] = 0.6 * c, 1.4 * c
        return s
    if op == "codec":
        x = rand(case["rows"], case["cols"]) * torch.exp(rand(case["rows"], 1)) * 0.05
        x[:, ::97] *= 8                                     # outlier channels
        return {"case": case, "x": x.to(TYPES[case["x"]])}
    codes, scales = _weights(case["N"], case["K"], gen)
    x = rand(case["M"], case["N"] if op == "grad" else case["K"])
    if op != "grad":
        x[:, ::97] *= 8
    return {"case": case, "x": x.to(TYPES[case["x"]]), "codes": codes, "scales": scales}


# --------------------------------------------------------------------------- plain forms
def _values(codes, scales, cols):
    """What codes and scales stand for, in fp32 (exact)."""
    rows = codes.shape[0]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    nib = torch.stack((codes & 15, codes >> 4), dim=2).reshape(rows, -1)[:, :cols]
    e = scales.permute(0, 3, 2, 1, 4).reshape(scales.shape[0] * 128, -1)[:rows, :(cols + 31) // 32]
    factor = torch.pow(2.0, e.double() - 127).float().repeat_interleave(32, dim=1)[:, :cols]
    return grid[nib.int()] * factor


def _rounded(x):
    """x [rows][cols] as MXFP4 holds it, in fp32: the largest of 32 values lands in [4, 8), larger than 6 becomes 6, ties to even."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    v = torch.zeros(rows, blocks * 32, device=x.device)
    v[:, :cols] = x.float()
    v = v.reshape(rows, blocks, 32)
    top = v.abs().amax(dim=2, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(min=-127).double()
    a = v.double() * torch.pow(2.0, -e)
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0)).double()
    q = (torch.round(a / step) * step).clamp(-6, 6)
    return (q * torch.pow(2.0, e)).float().reshape(rows, -1)[:, :cols]


def _mix(x):
    """The finaliser of a 32-bit multiply and xor-shift hash, on int64 tensors or numbers below 2^32."""
    x = (x ^ (x >> 16)) * 0x85EBCA6B & 0xFFFFFFFF
    x = (x ^ (x >> 13)) * 0xC2B2AE35 & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(seed, step, tensor):
    k = _mix((seed + 0x9E3779B9 * step) & 0xFFFFFFFF)
    return _mix((_mix((k + 0x9E3779B9 * (tensor + 1)) & 0xFFFFFFFF) + 0) & 0xFFFFFFFF)


def _decoded(code, scale):
    n = code.numel()
    return code.float() * scale.repeat_interleave(256)[:n]


def _encoded(x, rand16, positive):
    """E4M3 codes and constants of x >= 0 in blocks of 256, rounded up or down by 16 random bits; `positive`: what is not 0 stays so."""
    n, nb = x.numel(), (x.numel() + 255) // 256
    top = torch.zeros(nb * 256, device=x.device)
    top[:n] = x
    top = top.reshape(nb, 256).amax(dim=1)
    big = torch.full_like(top, 448.0)
    none = top < 2.0 ** -100
    scale = torch.where(none, 0.0, top / big)
    r = x * torch.where(none, 0.0, big / top).repeat_interleave(256)[:n]
    r = torch.minimum(r, torch.full_like(r, 448.0))
    add = rand16 << 4
    normal = (((r.view(torch.int32).long() + add) >> 20) - 960)
    small = ((r * 2.0 ** 29).long() + add) >> 20
    code = torch.where(r < 2.0 ** -6, small, normal)
    if positive:
        code = torch.where((r > 0) & (code == 0), 1, code)
    return code.to(torch.uint8), scale


def _adamw_plain(s):
    case, f = s["case"], np.float32
    lr, b1, b2, eps, wd = (f(HP[k]) for k in ("lr", "beta1", "beta2", "eps", "weight_decay"))
    s["steps"] += 1
    device = s["p"].device
    bc1 = torch.tensor(1 - float(b1) ** s["steps"], dtype=torch.float32, device=device)
    bc2 = torch.tensor(1 - float(b2) ** s["steps"], dtype=torch.float32, device=device)
    for t, (n, at, nb, bat) in enumerate(zip(s["sizes"], s["offsets"], s["blocks"], s["boff"])):
        p, g = s["p"][at:at + n], s["g"][at:at + n].float()
        m_held, v_held = s["m"][at:at + n], s["v"][at:at + n]
        if case["bits"] == 8:
            m = _decoded(m_held, s["m_scale"][bat:bat + nb])
            root = _decoded(v_held, s["v_scale"][bat:bat + nb])
            v = root * root
        else:
            m, v = m_held, v_held
        m = m * float(b1) + g * float(f(1) - b1)
        v = v * float(b2) + (g * float(f(1) - b2)) * g
        th = p.float()
        th = (th - th * float(lr * wd)) if n > 64 else th - th * 0.0       # vectors of 64 and less (lambda, biases) do not decay
        p.copy_(th - ((m / bc1) * float(lr)) / (torch.sqrt(v / bc2) + float(eps)))
        if case["bits"] == 8:
            h = _mix(torch.arange(n, device=device) ^ _key(ADAM_SEED, s["steps"], t))
            code, scale = _encoded(m.abs(), h & 0xFFFF, False)
            m_held.view(torch.uint8).copy_(code + 128 * (m < 0).to(torch.uint8))
            s["m_scale"][bat:bat + nb] = scale
            code, scale = _encoded(torch.sqrt(v), h >> 16, True)
            v_held.view(torch.uint8).copy_(code)
            s["v_scale"][bat:bat + nb] = scale
        else:
            m_held.copy_(m)
            v_held.copy_(v)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale") if k in s}


# --------------------------------------------------------------------------- the framework's calls
def _adamw_own(s):
    import paper_2408_10746_b200 as pac
    if "opt" not in s:
        cut = lambda flat, at, n: [flat[a:a + k] for a, k in zip(at, n)]  # noqa: E731
        state = {"m": cut(s["m"], s["offsets"], s["sizes"]), "v": cut(s["v"], s["offsets"], s["sizes"])}
        if s["case"]["bits"] == 8:
            state.update(m_scale=cut(s["m_scale"], s["boff"], s["blocks"]), v_scale=cut(s["v_scale"], s["boff"], s["blocks"]))
        s["opt"] = pac.AdamWTensors(cut(s["p"], s["offsets"], s["sizes"]), cut(s["g"], s["offsets"], s["sizes"]), bits=s["case"]["bits"],
                                    state=state, decay=[n > 64 for n in s["sizes"]], steps=s["steps"], seed=ADAM_SEED)
        s["hp"] = pac.AdamW(**HP)
    s["opt"].step(s["hp"])
    return _adamw_outputs(s)


def run(state):
    case = state["case"]
    op = case["op"]
    if op == "adamw":
        return _adamw_own(state) if own else _adamw_plain(state)
    x, out = state["x"], TYPES[case["y"]]
    if own:
        import paper_2408_10746_b200 as pac
        if op == "codec":
            return pac.dequantize_mxfp(*pac.quantize_mxfp(x), case["cols"], out)
        if op == "linear":
            return pac.mxfp_linear(x, state["codes"], state["scales"], out)
        if op == "grad":
            return pac.mxfp_linear_grad(x, state["codes"], state["scales"], case["K"], out)
        return pac.mxfp_product(*pac.quantize_mxfp(x), state["codes"], state["scales"], case["K"], out)
    if op == "codec":
        return _rounded(x).to(out)
    w = _values(state["codes"], state["scales"], case["K"])
    if op == "linear":
        return (x.float() @ w.T).to(out)
    if op == "grad":
        return (x.float() @ w).to(out)
    return (_rounded(x) @ w.T).to(out)


def work(case):
    size = {"f32": 4, "bf16": 2}
    op = case["op"]
    if op == "adamw":
        n, nb = sum(_sizes(case)), sum((k + 255) // 256 for k in _sizes(case))
        held = 16 * n if case["bits"] == 32 else 4 * n + 16 * nb
        return {"bytes": n * (2 * size[case["p"]] + size[case["g"]]) + held, "flops": 0}
    if op == "codec":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["x"]] + size[case["y"]]) + 2 * n * 17 / 32, "flops": 0}
    M, N, K = case["M"], case["N"], case["K"]
    xs, ys = (N, K) if op == "grad" else (K, N)
    held = N * K * 17 / 32 + (2 * M * K * 17 / 32 if op == "product" else 0)
    return {"bytes": M * xs * size[case["x"]] + held + M * ys * size[case["y"]], "flops": 2.0 * M * N * K}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _exact_matrix(codes, scales, cols):
    rows = codes.shape[0]
    col = torch.arange(cols, device=codes.device)
    row = torch.arange(rows, device=codes.device)[:, None]
    nib = (codes.long()[:, col // 2] >> (4 * (col % 2))) & 15
    e = scales[row // 128, col // 128, row % 32, row % 128 // 32, col % 128 // 32].double() - 127
    ex, man = (nib >> 1) & 3, nib & 1
    mag = torch.where(ex == 0, 0.5 * man, (1 + 0.5 * man) * torch.exp2((ex - 1).double()))
    return torch.where(nib >= 8, -mag, mag) * torch.exp2(e)


def _exact_rounded(x):
    """The nearest value of the grid, one after another, ties to the even code."""
    rows, cols = x.shape
    pad = torch.nn.functional.pad(x.double(), (0, -cols % 32)).reshape(rows, -1, 32)
    top = pad.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -149)))
    e = e - (torch.exp2(e) > top).double() + (torch.exp2(e + 1) <= top).double()      # a logarithm next to a whole number
    unit = torch.exp2((e - 2).clamp(min=-127))
    a = (pad / unit).abs()
    q = torch.zeros_like(a)
    for value, border, up in ((0.5, 0.25, False), (1, 0.75, True), (1.5, 1.25, False), (2, 1.75, True), (3, 2.5, False), (4, 3.5, True), (6, 5, False)):
        q = torch.where((a >= border) if up else (a > border), torch.full_like(a, value), q)
    return (torch.copysign(q, pad) * unit).reshape(rows, -1)[:, :cols]


def _exact_adamw(s):
    case = s["case"]
    f32 = lambda v: float(np.float32(v))  # noqa: E731
    lr, b1, b2, eps, wd = (f32(HP[k]) for k in ("lr", "beta1", "beta2", "eps", "weight_decay"))
    t = s["steps"] + 1
    out = {k: torch.zeros_like(s[k], dtype=torch.float64) for k in ("p", "m", "v", "m_scale", "v_scale") if k in s}
    for k in ("p", "m", "v"):
        out[k] += s[k].double()
    for i, n in enumerate(s["sizes"]):
        at = slice(s["offsets"][i], s["offsets"][i] + n)
        bl = slice(s["boff"][i], s["boff"][i] + s["blocks"][i])
        g, m, v = s["g"][at].double(), s["m"][at].double(), s["v"][at].double()
        which = torch.arange(n, device=g.device) // 256
        if case["bits"] == 8:
            m, v = m * s["m_scale"][bl].double()[which], (v * s["v_scale"][bl].double()[which]) ** 2
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        p = s["p"][at].double()
        out["p"][at] = p * (1 - lr * wd * (n > 64)) - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + eps)
        if case["bits"] == 32:
            out["m"][at], out["v"][at] = m, v
            continue
        bits = torch.arange(n, device=g.device)
        k = 0
        for word in ((ADAM_SEED + 0x9E3779B9 * t), 0x9E3779B9 * (i + 1), 0):
            k = _exact_mix((k + word) % 2 ** 32)
        bits = _exact_mix(bits ^ k)
        for name, value, u in (("m", m, bits % 2 ** 16), ("v", torch.sqrt(v), bits // 2 ** 16)):
            top = torch.zeros(s["blocks"][i], dtype=torch.float64, device=g.device).scatter_reduce(0, which, value.abs(), "amax")
            out[name + "_scale"][bl] = top / 448
            r = value.abs() / top.clamp(min=1e-300)[which] * 448
            # distance of neighbouring values of E4M3 at r; up with the probability of the remainder
            gap = torch.exp2(torch.floor(torch.log2(r.clamp(min=2.0 ** -6))) - 3)
            q = torch.floor(r / gap + u.double() / 65536) * gap
            if name == "v":
                q = torch.where((r > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q)
            out[name][at] = torch.copysign(q, value)
    return out


def _exact_mix(x):
    for shift, factor in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
        x = x ^ (x // 2 ** shift)
        # the low 32 bits of a product, the factor in two halves
        x = (x * (factor % 65536) + (x * (factor // 65536) % 65536) * 65536) % 2 ** 32
    return x ^ (x // 65536)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    if case["op"] == "codec":
        return _exact_rounded(s["x"])
    w = _exact_matrix(s["codes"], s["scales"], case["K"])
    if case["op"] == "grad":
        return s["x"].double() @ w
    return (_exact_rounded(s["x"]) if case["op"] == "product" else s["x"].double()) @ w.T
