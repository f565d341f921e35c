"""Pins of the oracle of the operators around attention: its formats against torch's, closed forms, brute force."""
import math

import numpy as np
import pytest
import torch

from oracle import layer as L


def test_e4m3_is_torchs():
    every = torch.arange(256, dtype=torch.uint8)
    finite = (every & 127) != 127
    want = every.view(torch.float8_e4m3fn).float().numpy()[finite.numpy()]
    np.testing.assert_array_equal(L.e4m3_values(every.numpy()[finite.numpy()]), want)
    g = torch.Generator().manual_seed(1)
    y = torch.cat([torch.randn(5000, generator=g) * s for s in (1e-3, 0.1, 1.0, 100.0)]).clamp(-448, 448)
    mid = torch.from_numpy((L.E4M3[1:] + L.E4M3[:-1]) / 2).float()                 # ties
    y = torch.cat([y, mid, -mid, torch.zeros(1)])
    np.testing.assert_array_equal(L.e4m3_bytes(y.double().numpy()), y.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert L.e4m3_bytes(np.array([1e9, -1e9])).tolist() == [126, 254]              # saturating


def test_e2m1_ties_go_to_the_even_code():
    assert L.E2M1.tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6]
    assert L.encode(np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 100.0]), L.E2M1).tolist() == [0, 2, 2, 4, 4, 6, 6, 7]


def test_linear_of_exact_codes():
    """Integers up to 16 times powers of two survive the codes, so the product is the plain one."""
    rng = np.random.default_rng(2)
    x, w = rng.integers(-7, 8, (5, 300)).astype(float), rng.integers(-7, 8, (130, 300)).astype(float)
    x[:, ::128], w[:, ::128] = 7.0, 7.0
    x *= 448.0 / 7.0 / 64.0
    w *= 448.0 / 7.0 / 64.0
    out, _ = L.linear(*L.quantize_rows(x), *L.quantize_tiles(w))
    np.testing.assert_allclose(out, x @ w.T, rtol=1e-12)


def test_activations():
    y = np.array([-50.0, -3.0, -0.5, 0.0, 0.1, 1.0, 4.0, 60.0])
    np.testing.assert_allclose(L.activation(y, "gelu"), 0.5 * y * (1 + np.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))), atol=1e-14)
    np.testing.assert_allclose(L.activation(y, "silu"), y / (1 + np.exp(-y)), rtol=1e-14)
    assert (L.activation(y, "none") == y).all()


def test_zero_rows_have_scale_one():
    codes, scale = L.quantize_rows(np.zeros((2, 130)))
    assert (codes == 0).all() and (scale == 1.0).all() and scale.shape == (2, 2)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_is_a_rotation_and_its_inverse_undoes_it(layout):
    rng = np.random.default_rng(3)
    x, g = rng.standard_normal((2, 3, 5, 16)), rng.standard_normal((2, 3, 5, 16))
    theta = L.frequencies([3, 1, 2], 100.0)
    pos = [rng.integers(0, 9, (1, 5)) for _ in range(3)]
    args = (theta, pos, [3, 1, 2], 12, layout)
    y = L.rope(x, *args)
    np.testing.assert_allclose(L.rope(y, *args, inverse=True), x, atol=1e-12)
    np.testing.assert_array_equal(y[..., 12:], x[..., 12:])
    # the gradient of <g, R x> is the inverse rotation of g: by differences
    grad, h = L.rope(g, *args, inverse=True), 1e-5
    for at in [(0, 0, 0, 0), (1, 2, 4, 7), (0, 1, 3, 11), (1, 0, 2, 14)]:
        e = np.zeros_like(x)
        e[at] = h
        diff = ((g * L.rope(x + e, *args)).sum() - (g * L.rope(x - e, *args)).sum()) / (2 * h)
        assert abs(diff - grad[at]) < 1e-8
    # relative positions: the product of two rotated rows depends on the distance alone
    one = [np.array([[4]]), np.array([[0]]), np.array([[0]])]
    two = [np.array([[11]]), np.array([[0]]), np.array([[0]])]
    q, k = x[:1, :1, :1], g[:1, :1, :1]
    a = (L.rope(q, theta, one, *args[2:]) * L.rope(k, theta, two, *args[2:])).sum()
    one[0], two[0] = one[0] + 100, two[0] + 100
    assert abs(a - (L.rope(q, theta, one, *args[2:]) * L.rope(k, theta, two, *args[2:])).sum()) < 1e-10


def test_frequency_rules():
    plain = L.frequencies([8], 10000.0)
    assert plain[0] == 1.0 and math.isclose(plain[4], 0.01)
    np.testing.assert_allclose(L.frequencies([8], 10000.0, "linear", 4.0), plain / 4)
    ntk = L.frequencies([8], 10000.0, "ntk", 4.0)
    assert ntk[0] == 1.0 and math.isclose(ntk[-1], plain[-1] / 4)                   # the slowest pair is slowed down by the factor
    parts = L.frequencies([8], 10000.0, "parts", 4.0, 4096)
    assert parts[0] == plain[0] and math.isclose(parts[-1], plain[-1] / 4)


@pytest.mark.parametrize("form,worst", [("e4m3", 2.0 ** -4), ("fp4", 0.25)])
def test_cache_rows_come_back_near(form, worst):
    x = np.random.default_rng(4).standard_normal((20, 64))
    for row in x:
        _, scale, sf, values = L.cache_row(row, form)
        # half a step of the format's coarsest binade, relative to the largest value a scale stands for
        assert np.abs(values - row).max() <= worst * np.abs(row).max()
    codes, scale, sf, values = L.cache_row(np.zeros(64), form)
    assert (codes == 0).all() and scale == 1.0 and (values == 0).all()


def test_nan_and_infinities():
    nan, inf = float("nan"), float("inf")
    x = np.tile(np.linspace(-1, 1, 128), (4, 1))
    x[1, 5], x[2, 5], x[3] = nan, inf, nan
    codes, scale = L.quantize_rows(x)
    assert (codes[1] == 127).sum() == (codes[2] == 127).sum() == 1 and (codes[3] == 127).all()
    assert scale[0].tolist() == [float(L.f32(1 / 448)), float(L.f32(1 / 448)), inf, 1.0]
    assert np.isnan(L.e4m3_values(L.quantize_tiles(x[1:2])[0])).sum() == 1
    for form in ("e4m3", "fp4"):
        values = [L.cache_row(row, form)[3] for row in x]
        assert np.isfinite(values[0]).all() and np.isnan(values[2]).all() and np.isnan(values[3]).all()
        assert np.isnan(values[1]).sum() == (1 if form == "e4m3" else 128)
