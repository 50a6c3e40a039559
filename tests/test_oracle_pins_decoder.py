"""Pins for the oracle of the norm, the 4-bit rows, the rotation and attention:
closed forms, independent computations, and planted mistakes that they catch."""
from __future__ import annotations

import types

import numpy as np
import pytest

import oracle

REAL = types.SimpleNamespace(rms_norm_block=oracle.rms_norm_block, rotate=oracle.rotate, quant_rows=oracle.quant_rows,
                             cached_rows=oracle.cached_rows, attend=oracle.attend)


def check_norm(ns):
    """Rows of equal magnitude have rms 1 / |value|; the sum, gate and scale by hand."""
    x = np.array([[3.0, -3.0, 3.0, 3.0], [0.5, 0.5, -0.5, 0.5]])
    y, r = ns.rms_norm_block(x, weight=np.array([1.0, 2.0, 4.0, 8.0]), eps=0.0)
    np.testing.assert_allclose(y, np.sign(x) * [1, 2, 4, 8], rtol=1e-15)
    np.testing.assert_array_equal(r, x)
    _, r = ns.rms_norm_block(x, residual=10 * np.ones((2, 4)), post=np.zeros(4), gate=np.array([1.0, 2.0, 0.0, 1.0]),
                             scale=0.5, offset=3.0, eps=0.0)
    np.testing.assert_allclose(r, 10 + 0.5 * 3 * np.sign(x) * [1, 2, 0, 1], rtol=1e-15)
    y, _ = ns.rms_norm_block(np.ones((1, 4)), weight=np.ones(4), eps=3.0)
    np.testing.assert_allclose(y, 0.5, rtol=1e-15)


def check_rotation(ns):
    """A complex product: pairs (i, i + D/2) turn by the angle; a quarter turn by hand."""
    rng = np.random.default_rng(0)
    x, a = rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 4))
    z = (x[..., :4] + 1j * x[..., 4:]) * np.exp(1j * a)[:, None]
    np.testing.assert_allclose(ns.rotate(x, np.cos(a), np.sin(a)), np.concatenate([z.real, z.imag], -1), atol=1e-14)
    np.testing.assert_array_equal(ns.rotate(np.array([[[1.0, 0.0]]]), np.zeros((1, 1)), np.ones((1, 1))), [[[0.0, 1.0]]])


def check_rows(ns):
    """A ramp of 16 steps is stored exactly; every row is within half a step (and
    the rounding of its scale) of what it stands for; constants and rows that are
    not finite as documented."""
    ramp = np.arange(16) * 0.25 - 1.5
    q, s, z = ns.quant_rows(ramp, "f16")
    np.testing.assert_array_equal(q, np.arange(16))
    assert (s, z) == (0.25, 6.0)
    rng = np.random.default_rng(1)
    for dt, u in (("f16", 2.0 ** -11), ("bf16", 2.0 ** -8)):
        x = (rng.standard_normal((200, 64)) * np.exp(2 * rng.standard_normal((200, 1))) + rng.standard_normal((200, 1)))
        step = np.ptp(x, -1, keepdims=True) / 15
        # half a step, 15 steps of a rounded scale, the rounding of a zero-point
        z = np.abs(x.min(-1, keepdims=True)) / step
        assert (np.abs(ns.cached_rows(x, dt) - x) <= step * (0.5 + 16 * u + z * u + 1e-4) * (1 + u)).all()
        np.testing.assert_array_equal(ns.cached_rows(np.full((1, 8), 2.5), dt), 2.5)
        np.testing.assert_array_equal(ns.cached_rows(np.zeros((1, 8)), dt), 0.0)
        assert np.isnan(ns.cached_rows(np.array([[1.0, np.inf], [np.nan, 2.0]]), dt)).all()


def check_attention(ns):
    """Equal scores average; a far score takes all; a query that sees none gives
    zeros; against scipy's softmax."""
    from scipy.special import softmax
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((4, 8)), rng.standard_normal((6, 8)), rng.standard_normal((6, 8))
    np.testing.assert_allclose(ns.attend(0 * q, k, v, 1.0, [5, 2, 0, -1]),
                               [v.mean(0), v[:3].mean(0), v[0], np.zeros(8)], atol=1e-15)
    got = ns.attend(q, k, v, 0.3, [5] * 4)
    np.testing.assert_allclose(got, softmax(0.3 * q @ k.T, axis=1) @ v, atol=1e-14)
    big = 1e4 * k[3:4]
    np.testing.assert_allclose(ns.attend(big, k, v, 1.0, [5]), v[[np.argmax(k @ k[3])]], atol=1e-12)


CHECKS = [check_norm, check_rotation, check_rows, check_attention]


@pytest.mark.parametrize("check", CHECKS, ids=lambda c: c.__name__)
def test_pins(check):
    check(REAL)


MISTAKES = {
    "norm before the sum": (check_norm, "rms_norm_block",
                            lambda x, weight=None, **kw: (REAL.rms_norm_block(x, weight=weight, **kw)[0], x)),
    "eps outside the root": (check_norm, "rms_norm_block", lambda x, weight=None, eps=0.0, **kw: (
        None if weight is None else x / (np.sqrt((x * x).mean(-1, keepdims=True)) + eps) * weight,
        REAL.rms_norm_block(x, eps=eps, **kw)[1])),
    "interleaved pairs": (check_rotation, "rotate", lambda x, c, s: np.stack(
        [x[..., ::2] * c[:, None] - x[..., 1::2] * s[:, None], x[..., 1::2] * c[:, None] + x[..., ::2] * s[:, None]],
        -1).reshape(x.shape)),
    "turned backwards": (check_rotation, "rotate", lambda x, c, s: REAL.rotate(x, c, -s)),
    "16 steps": (check_rows, "quant_rows", lambda x, dt: tuple(
        f(t) for f, t in zip((lambda q: q, lambda s: s * 15 / 16, lambda z: z), REAL.quant_rows(x, dt)))),
    "truncated codes": (check_rows, "cached_rows", lambda x, dt: (
        lambda q, s, z: s * (np.clip(np.floor(x / np.where(s == 0, 1, s) + z), 0, 15) - z))(*REAL.quant_rows(x, dt))),
    "one key more": (check_attention, "attend", lambda q, k, v, s, last: REAL.attend(q, k, v, s, np.asarray(last) + 1)),
    "no maximum, no scale": (check_attention, "attend", lambda q, k, v, s, last: REAL.attend(q, k, v, 1.0, last)),
}


@pytest.mark.parametrize("name", MISTAKES)
def test_planted_mistakes_are_caught(name):
    check, attr, wrong = MISTAKES[name]
    ns = types.SimpleNamespace(**vars(REAL))
    setattr(ns, attr, wrong)
    with pytest.raises(Exception):
        with np.errstate(all="ignore"):
            check(ns)
