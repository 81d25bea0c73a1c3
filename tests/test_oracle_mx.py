"""Pins of the microscaled oracle: grids, scales, rounding, layout, rotation, gradients."""
import numpy as np
import pytest

from oracle import mx


def test_grids_are_those_of_the_element_types():
    assert list(mx.E2M1) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert len(mx.E4M3) == 127 and mx.E4M3[-1] == 448 and mx.E4M3[1] == 2.0 ** -9 and mx.E4M3[8] == 2.0 ** -6
    assert np.all(np.diff(mx.E4M3) > 0)
    import torch
    every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(every, mx.E4M3)


@pytest.mark.parametrize("bits", [4, 8])
def test_scale_puts_the_largest_element_into_the_top_binade(bits):
    rng = np.random.default_rng(bits)
    x = (rng.standard_normal((6, 96)) * np.exp(rng.uniform(-40, 40, (6, 1)))).astype(np.float32)
    codes, scales = mx.quantize(x, bits)
    t = np.abs(x.reshape(6, 3, 32)).max(2) / 2.0 ** (scales.astype(float) - 127)
    assert np.all(t >= 2.0 ** mx.EMAX[bits]) and np.all(t < 2.0 ** (mx.EMAX[bits] + 1))
    # nearest or saturated
    v, q = x.astype(np.float64), mx.values(codes, scales, bits)
    step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)
    top = mx.GRID[bits].max() * step
    near = np.min(np.abs(np.abs(v)[:, :, None] / step[:, :, None] - mx.GRID[bits]), axis=2) * step
    assert np.allclose(np.abs(v - q), near, rtol=0, atol=0)
    assert np.all(np.abs(q) <= top)


def test_ties_go_to_the_even_code_and_signs_stay():
    x = np.zeros((1, 32), np.float32)
    x[0, :10] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, 7.9]
    codes, scales = mx.quantize(x, 4)
    assert scales[0, 0] == 127
    assert list(mx.E2M1[codes[0, :8] & 7]) == [4, 0, 1, 1, 2, 2, 4, 4] and codes[0, 8] == 8 and codes[0, 9] == 7
    x[0, :4] = [256, 1.0625, 1.1875, 511]
    codes, scales = mx.quantize(x, 8)
    assert scales[0, 0] == 127 and list(mx.E4M3[codes[0, :4]]) == [256, 1.0, 1.25, 448]


def test_zeros_smallest_and_largest_scales_and_blocks_that_are_not_finite():
    x = np.zeros((1, 160), np.float32)
    x[0, 32], x[0, 64], x[0, 96], x[0, 130] = 1e-45, 3.4e38, np.nan, -np.inf
    for bits in (4, 8):
        codes, scales = mx.quantize(x, bits)
        assert list(scales[0]) == [0, 0, 254 - mx.EMAX[bits], 255, 255]
        assert not codes[0, 96:].any()
        assert np.isnan(mx.values(codes, scales, bits)[0, 96:]).all()


def test_layout():
    rng = np.random.default_rng(0)
    s = rng.integers(0, 255, (300, 5)).astype(np.uint8)
    t = mx.tile(s)
    assert len(t) == 3 * 2 * 512
    assert t[0] == s[0, 0] and t[3] == s[0, 3] and t[16] == s[1, 0] and t[4] == s[32, 0] and t[512] == s[0, 4] and t[1024] == s[128, 0]
    c = rng.integers(0, 16, (3, 64)).astype(np.uint8)
    assert np.array_equal(mx.unpack(mx.pack(c, 4), 4), c) and mx.pack(c, 4)[0, 0] == c[0, 0] + 16 * c[0, 1]


def test_package_helpers_lay_scales_out_alike():
    import torch

    import paper_2502_05003_b200 as quest
    s = torch.from_numpy(np.random.default_rng(1).integers(0, 255, (130, 9)).astype(np.uint8))
    t = quest.mx_scales_tiled(s)
    assert np.array_equal(t.numpy(), mx.tile(s.numpy()))
    assert torch.equal(quest.mx_scales_rows(t, 130, 9 * 32), s)
    assert quest.quest_mx_scales_bytes(130, 9 * 32) == t.numel()


def test_rotation_is_the_orthonormal_transform_and_cancels():
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((4, 64)).astype(np.float32), rng.standard_normal((3, 64)).astype(np.float32)
    h = mx.hadamard(32)
    assert np.allclose(h @ h.T, np.eye(32), atol=1e-14)
    r = mx.rotate(x, 32)
    assert np.allclose(r, mx.inverse(x.astype(np.float64), 32), atol=1e-6)
    assert np.allclose(r.astype(np.float64) @ mx.rotate(w, 32).astype(np.float64).T, x.astype(np.float64) @ w.T, atol=1e-5)
    assert np.allclose(mx.inverse(mx.inverse(x.astype(np.float64), 32), 32), x, atol=1e-12)


@pytest.mark.parametrize("g", [1, 32])
def test_gradients_against_differences(g):
    # straight through the rounding: the gradient of the linear map whose operands are the rounded tensors
    rng = np.random.default_rng(3)
    xv, wv = rng.standard_normal((3, 64)), rng.standard_normal((5, 64))
    dy = rng.standard_normal((3, 5))
    dx, dw, bx, bw = mx.backward(dy, xv, wv, g)
    loss = lambda a, b: np.sum(dy * ((xv + mx.inverse(a, g)) @ (wv + mx.inverse(b, g)).T))  # noqa: E731
    zx, zw = np.zeros((3, 64)), np.zeros((5, 64))
    for i, j in ((0, 0), (2, 63), (1, 17)):
        a = zx.copy()
        a[i, j] = 1e-6
        assert abs((loss(a, zw) - loss(-a, zw)) / 2e-6 - dx[i, j]) < 1e-7 * (1 + abs(dx[i, j])) + 1e-7
        b = zw.copy()
        b[i, j] = 1e-6
        assert abs((loss(zx, b) - loss(zx, -b)) / 2e-6 - dw[i, j]) < 1e-7 * (1 + abs(dw[i, j])) + 1e-7
    assert np.all(np.abs(dx) <= bx * (1 + 1e-12)) and np.all(np.abs(dw) <= bw * (1 + 1e-12))
