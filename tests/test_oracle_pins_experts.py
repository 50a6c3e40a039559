"""Pins for the oracle of 8-bit linear layers and layers made of experts: closed
forms, independent computations, and planted mistakes that they catch."""
from __future__ import annotations

import fractions
import types

import numpy as np
import pytest

import oracle

NAMES = ("gated_rows", "row_codes", "w8a8", "route", "expert_order", "expert_products", "combine")
REAL = types.SimpleNamespace(**{n: getattr(oracle, n) for n in NAMES})


def check_codes(ns):
    """A ramp to 127 is its own codes; a row times 2 has the same codes and twice the
    scale; silu by hand; rows that are tiny or not finite."""
    ramp = np.arange(-127.0, 128.0)[None]
    v, s = ns.row_codes(ramp)
    np.testing.assert_array_equal(v, ramp)
    assert s[0] == 1.0
    v2, s2 = ns.row_codes(-2 * ramp)
    np.testing.assert_array_equal(v2, -ramp)
    assert s2[0] == 2.0
    v, s = ns.row_codes(np.array([[1.0, np.inf], [np.nan, 1.0], [0.0, 0.0], [2.0 ** -101, 0.0], [4.0, 2.0]]))
    np.testing.assert_array_equal(v, [[0, 0], [0, 0], [0, 0], [0, 0], [127, 63.5]])
    np.testing.assert_array_equal(s, [np.nan, np.nan, 0, 0, 4 / 127])
    np.testing.assert_allclose(ns.gated_rows(np.array([[0.0, np.log(3.0), 5.0, 2.0]])), [[0.0, 2 * 0.75 * np.log(3.0)]],
                               rtol=1e-15)


def check_product(ns):
    """Against whole numbers and exact fractions, -128 included."""
    rng = np.random.default_rng(0)
    q, w = rng.integers(-128, 128, (3, 40)).astype(np.int8), rng.integers(-128, 128, (40, 5)).astype(np.int8)
    s, ws = 2.0 ** -rng.integers(0, 9, 3), 2.0 ** -rng.integers(0, 9, 5)
    got = ns.w8a8(q, s, w, ws)
    for m in range(3):
        for n in range(5):
            total = sum(int(q[m, k]) * int(w[k, n]) for k in range(40))
            assert got[m, n] == float(total * fractions.Fraction(s[m]) * fractions.Fraction(ws[n]))


def check_routing(ns):
    """Weights by hand; ties, bias, groups, masked experts."""
    w, e = ns.route(np.log([[1.0, 4.0, 2.0, 1.0]]), 3)
    np.testing.assert_array_equal(e, [[1, 2, 0]])
    np.testing.assert_allclose(w, [[0.5, 0.25, 0.125]], rtol=1e-15)
    w, _ = ns.route(np.log([[1.0, 4.0, 2.0, 1.0]]), 2, renormalize=True, scale=3.0)
    np.testing.assert_allclose(w, [[2.0, 1.0]], rtol=1e-15)
    # the bias moves the choice and not the weight
    w, e = ns.route(np.log([[1.0, 3.0, 1 / 3]]), 1, bias=np.array([0.3, 0.0, 0.0]), scoring="sigmoid")
    assert e[0, 0] == 0 and abs(w[0, 0] - 0.5) < 1e-15
    # groups (0 1)(2 3)(4 5): by the sum of two the middle one, by the largest the last
    x = np.array([[0.0, 0.0, 2.0, 2.0, 3.0, -9.0]])
    assert ns.route(x, 1, scoring="sigmoid", groups=3, top_groups=1)[1][0, 0] == 2
    assert ns.route(x, 1, scoring="sigmoid", groups=3, top_groups=1, group_score="max")[1][0, 0] == 4
    # a group of one open expert before one of none; equal groups by index
    x = np.array([[-np.inf, -np.inf, np.nan, -5.0, 1.0, 1.0, 1.0, 1.0]])
    assert ns.route(x, 4, groups=4, top_groups=3)[1].tolist() == [[4, 5, 6, 7]]
    w, e = ns.route(np.array([[-np.inf, 0.0, np.nan, -np.inf]]), 3, renormalize=True)
    assert e.tolist() == [[1, 0, 2]] and w.tolist() == [[1.0, 0.0, 0.0]]
    w, e = ns.route(np.zeros((1, 3)), 3, bias=np.array([-np.inf, 0.0, np.nan]))
    assert e.tolist() == [[1, 0, 2]] and w.tolist() == [[1 / 3, 0.0, 0.0]]
    w, e = ns.route(np.full((1, 3), -np.inf), 2, renormalize=True)
    assert e.tolist() == [[0, 1]] and w.tolist() == [[0.0, 0.0]]
    w, e = ns.route(np.array([[np.inf, 0.0, np.inf, 5.0]]), 3)
    assert e.tolist() == [[0, 2, 1]] and w.tolist() == [[0.5, 0.5, 0.0]]


def check_order(ns):
    """A hand-made order; every slot belongs to the choice that points to it."""
    o, t, p = ns.expert_order(np.array([[2, 0], [0, 3], [2, 3]]), 5)
    assert o.tolist() == [0, 2, 2, 4, 6, 6] and t.tolist() == [0, 1, 0, 2, 1, 2]
    assert p.tolist() == [[2, 0], [1, 4], [3, 5]]


def check_experts(ns):
    """Each slot alone as a dense product; sums by hand."""
    rng = np.random.default_rng(1)
    q, w = rng.integers(-9, 9, (4, 16)).astype(np.int8), rng.integers(-9, 9, (3, 16, 8)).astype(np.int8)
    s, ws = rng.random(4), rng.random((3, 8))
    out = ns.expert_products(q, s, w, ws, [0, 2, 2, 4], [3, 1, 0, 7, 0])
    for i, (r, e) in enumerate([(3, 0), (1, 0), (0, 2)]):
        np.testing.assert_allclose(out[i], s[r] * ws[e] * (q[r].astype(int) @ w[e].astype(int)), rtol=1e-14)
    assert (out[3] == 0).all() and np.isnan(out[4]).all()
    y = np.array([[1.0, 2.0], [10.0, 20.0], [np.nan, np.nan]])
    got = ns.combine(y, np.array([[0.5, 0.25], [2.0, 0.0]]), np.array([[1, 0], [9, 2]]), add=np.array([[100.0, 0.0], [7.0, 8.0]]))
    np.testing.assert_allclose(got, [[105.25, 10.5], [7.0, 8.0]], rtol=1e-15)


CHECKS = [check_codes, check_product, check_routing, check_order, check_experts]


@pytest.mark.parametrize("check", CHECKS, ids=lambda f: f.__name__)
def test_pins(check):
    check(REAL)


def with_(**kw):
    return types.SimpleNamespace(**{**vars(REAL), **kw})


MISTAKES = {
    "scale of 128": (check_codes, with_(row_codes=lambda x: (REAL.row_codes(x)[0], REAL.row_codes(x)[1] * 127 / 128))),
    "halves swapped": (check_codes, with_(gated_rows=lambda x: REAL.gated_rows(np.roll(x, x.shape[-1] // 2, -1)))),
    "unsigned codes": (check_product, with_(w8a8=lambda q, s, w, ws: REAL.w8a8(q.view(np.uint8), s, w, ws))),
    "sums of 16 bits": (check_product, with_(w8a8=lambda q, s, w, ws: (q.astype(np.int16) @ w.astype(np.int16)) * s[:, None] * ws)),
    "bias in the weight": (check_routing, with_(route=lambda x, k, bias=None, **kw: REAL.route(
        x, k, bias=bias, **kw) if bias is None else (REAL.route(x, k, bias=bias, **kw)[0] + bias[0], REAL.route(x, k, bias=bias, **kw)[1]))),
    "largest of a group": (check_routing, with_(route=lambda x, k, group_score="top2", **kw: REAL.route(x, k, group_score="max", **kw))),
    "scores of all experts": (check_routing, with_(route=lambda x, k, renormalize=False, **kw: REAL.route(x, k, **kw))),
    "tokens not in order": (check_order, with_(expert_order=lambda e, E: (
        REAL.expert_order(e, E)[0], REAL.expert_order(e, E)[1][::-1], REAL.expert_order(e, E)[2]))),
    "weights of the next expert": (check_experts, with_(expert_products=lambda q, s, w, ws, o, r: REAL.expert_products(
        q, s, np.roll(w, -1, 0), ws, o, r))),
    "add left out": (check_experts, with_(combine=lambda y, w, p, add=None: REAL.combine(y, w, p))),
}


@pytest.mark.parametrize("name", MISTAKES)
def test_pins_catch(name):
    check, ns = MISTAKES[name]
    with pytest.raises((AssertionError, ValueError)):
        check(ns)
