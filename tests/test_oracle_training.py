"""The 64-bit restatement of the training-step operators against what their definitions fix."""
import numpy as np
import pytest

from oracle import training as T


def test_format():
    v = T.e4m3_values()
    assert v[0x7E] == 448 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0xB8] == -1.0
    assert np.isnan(v[[0x7F, 0xFF]]).all() and np.isfinite(np.delete(v, [0x7F, 0xFF])).all()
    pos = v[:0x7F]
    assert (np.diff(pos) > 0).all()
    assert np.array_equal(T.spacing(pos[:-1]), np.diff(pos))          # spacing() is the distance to the next code up


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0000001, 1), (224.0, -1), (1.0, -8), (0.875, -9), (0.8750001, -8), (3e38, 100), (1e-40, -100)])
def test_scale(amax, e):
    assert T.scale_of(amax) == 2.0 ** e
    assert T.scale_of(0.0) == 1.0


@pytest.mark.parametrize("rows,cols", [(1, 128), (128, 1), (128, 128)])
def test_quantize_keeps_what_the_format_can_hold(rows, cols):
    rng = np.random.default_rng(0)
    q0, s0 = rng.choice(np.delete(T.e4m3_values(), [0x7F, 0xFF]), (300, 200)), None
    q0[::rows if rows > 1 else 1, ::cols if cols > 1 else 1] = 448.0   # every block reaches the top: its scale is 1
    q, s = T.quantize(q0, rows, cols)
    assert np.array_equal(q, q0) and (s == 1).all()
    x = rng.standard_normal((300, 200)) * 10.0 ** rng.uniform(-6, 6, (1, 200))
    q, s = T.quantize(x, rows, cols)
    wide = np.repeat(np.repeat(s, rows, 0), cols, 1)[:300, :200]
    assert (np.abs(q * wide - x) <= T.spacing(x / wide) * wide / 2).all()
    assert np.isin(q, T.e4m3_values()).all()


def test_random_rounding_is_right_on_average():
    """The mean over many seeds of the kept value is the value: standard error sqrt(f (1 - f) / n) of a spacing."""
    y = np.array([0.001, 0.3, 1.03, 17.9, 300.0])
    n = 20000
    got = np.zeros_like(y)
    for i, x in enumerate(y):
        bits = T.random_bits(7 + i, n, 12345, 0) >> np.uint64(16)
        got[i] = (np.floor(T.random_round(np.full(n, x), bits)) * T.spacing(x)).mean()
    assert (np.abs(got - y) <= 5 * 0.5 / np.sqrt(n) * T.spacing(y)).all()


def test_random_bits_look_uniform():
    b = T.random_bits(0, 1 << 18, 1, 0)
    for shift in (0, 8, 16, 24):
        h = np.bincount((b >> np.uint64(shift) & np.uint64(255)).astype(int), minlength=256)
        assert ((h - 1024) ** 2 / 1024).sum() < 256 + 6 * np.sqrt(2 * 256)           # chi squared, 6 sigma
    assert not np.array_equal(b, T.random_bits(0, 1 << 18, 2, 0)) and not np.array_equal(b, T.random_bits(0, 1 << 18, 1, 1))
    assert np.array_equal(b[256:], T.random_bits(1, (1 << 18) - 256, 1, 0))         # by place, not by launch


def test_adamw_against_a_scalar_loop():
    rng = np.random.default_rng(1)
    p, m, v = rng.standard_normal(5), np.zeros(5), np.zeros(5)
    q, mm, vv = p.copy(), [0.0] * 5, [0.0] * 5
    for step in range(1, 4):
        g = rng.standard_normal(5)
        p, m, v, _ = T.adamw(p, g, m, v, lr=0.1, beta1=0.9, beta2=0.95, eps=1e-8, decay=0.1, step=step, coef=0.5)
        for i in range(5):
            gi = 0.5 * g[i]
            mm[i] = 0.9 * mm[i] + (1 - 0.9) * gi
            vv[i] = 0.95 * vv[i] + (1 - 0.95) * gi * gi
            q[i] = q[i] * (1 - 0.1 * 0.1) - 0.1 * (mm[i] / (1 - 0.9 ** step)) / ((vv[i] / (1 - 0.95 ** step)) ** 0.5 + 1e-8)
    assert np.allclose(p, q, rtol=1e-13, atol=0)


def test_norm():
    assert T.grad_norm([np.array([3.0]), np.array([4.0])], 1.0) == (5.0, 1.0 / (5 + 1e-6), 1.0)
    assert T.grad_norm([np.array([3.0, np.inf])], 1.0)[1:] == (0.0, 0.0)
    assert T.grad_norm([], 1.0) == (0.0, 1.0, 1.0)
