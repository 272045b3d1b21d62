"""Pins of the MXFP4 and 8-bit-moment oracle that need no GPU: torch's own float8 type, hand-made blocks, moments of the
rounding, and the shapes and refusals of the binding."""
import numpy as np
import pytest
import torch

from oracle import lowbit_oracle as lo


def test_nearest_value_is_nearest_and_ties_are_even():
    a = np.linspace(0, 9, 3601)
    c = lo.nearest_e2m1(a)
    best = np.abs(a[:, None] - lo.GRID).min(1)
    assert np.allclose(np.abs(a - lo.GRID[c]), best)
    for tie, code in ((0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (7.9, 7)):
        assert lo.nearest_e2m1(np.array([tie]))[0] == code


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -140, 2.0 ** 120])
def test_largest_of_a_block_lands_between_four_and_eight(scale):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((7, 65)) * scale
    codes, s = lo.quantize(x)
    v = lo.values(codes, s)
    for b in range(3):
        part, q = x[:, 32 * b:32 * b + 32], v[:, 32 * b:32 * b + 32]
        unit = np.exp2(s[:, b].astype(float) - 127)
        top = np.abs(part).max(1) / unit
        assert ((top < 8) & ((top >= 4) | (s[:, b] == 0))).all()
        # half the largest gap (2) below 6; up to 2 beyond it
        assert (np.abs(q - part) <= np.where(np.abs(part) / unit[:, None] <= 6, 1, 2) * unit[:, None]).all()


def test_blocks_that_are_not_finite_and_blocks_of_zeros():
    x = np.zeros((3, 64))
    x[1, 3], x[2, 40] = np.inf, np.nan
    codes, s = lo.quantize(x)
    assert s.tolist() == [[0, 0], [255, 0], [0, 255]] and not codes.any()
    assert np.isnan(lo.values(codes, s)[1, :32]).all() and (lo.values(codes, s)[1, 32:] == 0).all()


def test_e4m3_table_is_torchs():
    t = torch.arange(128, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, lo.e4m3_values(), equal_nan=True)


def test_rounding_is_unbiased_and_keeps_what_is_not_zero():
    n = 1 << 16
    x = np.full(n, 0.3, np.float32)
    x[::256] = 1.0
    codes, c = lo.encode_e4m3(x, lo.random_bits(5, 3, 0, n) & 0xFFFF, False)
    got = lo.e4m3_values()[codes] * np.repeat(c.astype(np.float64), 256)
    # neighbours of 0.3 * 448 = 134.4 are 128 and 144: sd of one 16 / 448 * sqrt(0.4 * 0.6), of the mean 1/256 of it; five of them
    assert abs(got[x < 1].mean() - 0.3) < 5 * 16 / 448 * 0.49 / 256 * 1.01
    x[:] = 1e-9
    x[0] = 1.0
    assert (lo.encode_e4m3(x, np.zeros(n, np.uint64), True)[0] > 0).all()


def test_random_bits_differ_by_seed_step_and_place():
    a = [lo.random_bits(*k, 4096) for k in ((1, 2, 3), (2, 2, 3), (1, 3, 3), (1, 2, 4))]
    for i in range(4):
        for j in range(i):
            assert (a[i] == a[j]).mean() < 0.01
    assert abs(np.mean((a[0] & 0xFFFF).astype(float)) / 65536 - 0.5) < 5 * 0.29 / 64


def test_shapes_and_refusals_without_a_device():
    import paper_2408_10746_b200 as pac
    assert pac.mxfp_shapes(1, 1) == ((1, 16), (1, 2, 32, 4, 4))
    assert pac.mxfp_shapes(129, 257) == ((129, 144), (2, 4, 32, 4, 4))
    x = torch.zeros(4, 64)
    codes, scales = (torch.zeros(s, dtype=torch.uint8) for s in pac.mxfp_shapes(4, 64))
    for call in (lambda: pac.quantize_mxfp(x), lambda: pac.dequantize_mxfp(codes, scales, 64), lambda: pac.mxfp_linear(x, codes, scales),
                 lambda: pac.mxfp_linear_grad(x[:, :4], codes, scales, 64), lambda: pac.mxfp_product(codes, scales, codes, scales, 64),
                 lambda: pac.AdamWTensors([x], [x.clone()]), lambda: pac.AdamWTensors([x], [x.clone()], bits=16), lambda: pac.AdamWTensors([x], [])):
        with pytest.raises(pac.PacError) as e:
            call()
        assert e.value.status_name == "PAC_ERR_INVALID_ARG"


def test_bad_arguments_of_the_c_calls_are_refused_before_any_device_is_touched():
    import ctypes as C

    import paper_2408_10746_b200 as pac
    from paper_2408_10746_b200 import binding as b
    lib = pac.load_library()
    ok = 4096                                                  # never followed: every call below is refused on the host
    assert lib.pac_quantize_mxfp(0, None, None, 0, 4, 64, 64, ok, ok) == 1
    assert lib.pac_quantize_mxfp(0, None, ok, 2, 4, 64, 64, ok, ok) == 1
    assert lib.pac_quantize_mxfp(0, None, ok, 0, 4, 64, 63, ok, ok) == 1
    assert lib.pac_quantize_mxfp(0, None, ok, 0, 4, 0, 64, ok, ok) == 1
    assert lib.pac_quantize_mxfp(0, None, ok, 0, -1, 64, 64, ok, ok) == 1
    assert lib.pac_quantize_mxfp(0, None, ok + 2, 0, 4, 64, 64, ok, ok) == 1
    assert lib.pac_quantize_mxfp(0, None, ok, 0, 4, 64, 64, ok + 8, ok) == 1
    assert lib.pac_quantize_mxfp(0, None, ok, 0, 0, 64, 64, ok, ok) == 0
    assert lib.pac_dequantize_mxfp(0, None, ok, ok + 4, 4, 64, ok, 0, 64) == 1
    assert lib.pac_dequantize_mxfp(0, None, ok, ok, 4, 64, ok, 0, 63) == 1
    for f in (lambda *a: lib.pac_mxfp_linear(*a, ok, 1 << 20), lambda *a: lib.pac_mxfp_linear_grad(*a, ok, 1 << 20)):
        assert f(0, None, ok, 0, 4, 64, ok, ok, 64, 64, ok, 0, 63) == 1
        assert f(0, None, ok, 0, 4, 63, ok, ok, 64, 64, ok, 0, 64) == 1
        assert f(0, None, ok, 0, 4, 64, ok, ok, 0, 64, ok, 0, 64) == 1
        assert f(0, None, ok, 3, 4, 64, ok, ok, 64, 64, ok, 0, 64) == 1
        assert f(0, None, ok + 1, 1, 4, 64, ok, ok, 64, 64, ok, 0, 64) == 1
        assert f(0, None, None, 0, 0, 64, ok, ok, 64, 64, None, 0, 64) == 0
    # workspaces: terms of few tokens, packed copies of what boxes cannot read, none for aligned bf16
    assert lib.pac_mxfp_linear_workspace(ok, 1, 17, 64, 64, 64, 0) == 0 == lib.pac_mxfp_linear_workspace(ok, 1, 3, 64, 64, 64, 1)
    assert lib.pac_mxfp_linear_workspace(ok, 1, 17, 65, 64, 64, 0) == 17 * 128 * 2 == lib.pac_mxfp_linear_workspace(ok + 2, 1, 17, 64, 64, 64, 1)
    assert lib.pac_mxfp_linear_workspace(ok, 0, 17, 64, 130, 64, 1) == 17 * 256 * 6 and lib.pac_mxfp_linear_workspace(ok, 1, 3, 4096, 4096, 4096, 0) > 0
    assert lib.pac_mxfp_linear_workspace(ok, 1, 1, 64, 64, 64, 0) == 0 == lib.pac_mxfp_linear_workspace(ok, 1, 3, 64, 64, 64, 0) and lib.pac_mxfp_linear_workspace(ok, 1, 1, 4096, 32000, 4096, 0) > 0
    for space, n in ((None, 0), (ok, 17 * 128 * 6 - 1), (ok + 16, 1 << 20)):
        assert lib.pac_mxfp_linear(0, None, ok, 0, 17, 64, ok, ok, 64, 64, ok, 0, 64, space, n) == 1
    assert lib.pac_mxfp_product(0, None, ok, ok, 4, ok, ok + 1, 64, 64, ok, 0, 64) == 1
    assert lib.pac_mxfp_product(0, None, ok, None, 4, ok, ok, 64, 64, ok, 0, 64) == 1
    hp = pac.AdamW()._c()
    t = (b._AdamWTensor * 1)(b._AdamWTensor(ok, ok, ok, ok, ok, ok, 5, 0, 0, 1))
    call = lambda count=1, bits=32, step=1, lst=t: lib.pac_adamw_tensors(0, None, lst, count, bits, C.byref(hp), step, None, 1.0, 0)  # noqa: E731
    assert call(bits=16) == 1 and call(step=0) == 1 and call(count=-1) == 1 and call(lst=None) == 1
    for field, bad in (("p", None), ("g", ok + 2), ("m", None), ("n", -1), ("p_dtype", 2), ("m", ok + 1)):
        u = (b._AdamWTensor * 1)(t[0])
        setattr(u[0], field, bad)
        assert call(lst=u) == 1, field
    u = (b._AdamWTensor * 1)(t[0])
    u[0].v_scale = None
    assert call(lst=u, bits=8) == 1
