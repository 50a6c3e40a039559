"""Every form of the 8-bit product, dense and by expert, with and without gathered rows,
against whole sums in 64 bits: ragged rows and columns, K of several passes of the
loop and not whole pairs of its steps, one tile a workgroup and several.

Tolerances as in test_gpu_experts.py: the sums are exact, an output carries their
conversion, two fp32 products and its rounding.  test_plan_choice_w8a8.py holds that
each size runs the form it is listed for."""
from __future__ import annotations

import pytest

from test_gpu_experts import DT, E32, TINY, U, tf  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DIRECT = "16 x 16"
# (rows and columns a tile, M, K, N): the second of a form has more tiles than workgroups
DENSE = [
    (DIRECT, 5, 1040, 264), (DIRECT, 16, 4112, 4104), (DIRECT, 45, 2064, 1032),
    ("64 x 64", 100, 1040, 520), ("64 x 64", 128, 208, 16392), ("64 x 64", 60, 1040, 65528),
    ("64 x 128", 333, 1040, 4104), ("64 x 128", 100, 208, 32776), ("64 x 128", 700, 2064, 2056),
    ("128 x 128", 333, 2064, 6152), ("128 x 128", 2100, 1040, 4104), ("128 x 128", 1500, 208, 6152),
    ("128 x 256", 700, 1040, 6152), ("128 x 256", 3000, 1040, 6152), ("128 x 256", 3000, 2064, 6152),
    ("256 x 256", 2100, 2064, 4104), ("256 x 256", 4200, 2064, 6152), ("256 x 256", 3000, 4000, 4120)]
# (rows and columns a tile, experts, slots, K, N)
EXPERTS = [
    (DIRECT, 3, 40, 1040, 264), (DIRECT, 8, 150, 2064, 264),
    ("64 x 64", 5, 150, 1040, 2056), ("64 x 64", 64, 1000, 1040, 4104),
    ("64 x 128", 5, 1000, 1040, 1032), ("64 x 128", 64, 3000, 1040, 2056),
    ("128 x 128", 5, 1000, 1040, 2056), ("128 x 128", 8, 2000, 1040, 4104),
    ("128 x 256", 3, 2000, 1040, 2056), ("128 x 256", 8, 3000, 2064, 4104),
    ("256 x 256", 3, 2000, 2064, 4104), ("256 x 256", 20, 5000, 2064, 4104)]
# slots past the last row of A
PAST = [(DIRECT, 8, 150, 2064, 264), ("64 x 64", 5, 150, 1040, 2056), ("256 x 256", 3, 2000, 2064, 4104)]


def ints(*shape):
    return torch.randint(-128, 128, shape, dtype=torch.int8, device="cuda")


def operands(seed, rows, K, weights, N):
    torch.manual_seed(seed)
    q, s = ints(rows, K), 0.5 + torch.rand(rows, device="cuda")
    w, ws = ints(weights, K, N), (0.5 + torch.rand(weights, N, device="cuda")) / (5500 * K ** 0.5)
    return q, s, w, ws


def product(q, s, w, ws):
    """In float64: the sums are whole numbers under 2^53."""
    return (q.double() @ w.double()) * s.double()[:, None] * ws.double()


def check(got, want, dt):
    assert ((got.double() - want).abs() <= (U[dt] + 4 * E32) * want.abs() + TINY[dt]).all()


@pytest.mark.parametrize("form,M,K,N", DENSE)
def test_dense(tf, form, M, K, N):
    q, s, w, ws = operands(M + N, M, K, 1, N)
    packed = tf.pack_w8a8(w[0], ws[0])
    want = product(q, s, w[0], ws[0])
    for dt in ("f16", "bf16"):
        out = torch.full((M + 3, N), 7.0, dtype=DT[dt], device="cuda")
        tf.w8a8_gemm(q, s, packed, K, N, out=out[:M])
        check(out[:M], want, dt)
        assert (out[M:] == 7).all()


def offsets_of(kind, E, S):
    """Ends of the experts' slots; the first and last slots are no expert's."""
    if kind == "even":
        ends = [2 + (S - 5) * e // E for e in range(E + 1)]
    elif kind == "one":                                 # all to one expert in the middle
        ends = [2 if e <= E // 2 else S - 3 for e in range(E + 1)]
    else:                                               # ragged, some of none and of one
        cuts = sorted(torch.randint(2, S - 2, (E - 1,)).tolist())
        if E > 2:
            cuts[1] = cuts[0]
        if E > 4:
            cuts[3] = min(cuts[2] + 1, S - 3)
            cuts[4:] = [max(c, cuts[3]) for c in cuts[4:]]
        ends = [2] + cuts + [S - 3]
    return ends


def check_experts(out, dt, q, s, w, ws, ends, rows):
    S = out.shape[0] - 2
    owned = torch.zeros(S + 2, dtype=torch.bool, device="cuda")
    for e in range(len(ends) - 1):
        a, b = ends[e], ends[e + 1]
        owned[a:b] = True
        at = rows[a:b].long()
        there = (at >= 0) & (at < len(q))
        at = at.clamp(0, len(q) - 1)
        want = torch.where(there[:, None], product(q[at], s[at], w[e], ws[e]), 0.0)
        check(out[a:b], want, dt)
        assert (out[a:b][~there] == 0).all()
    assert (out[~owned] == 7).all()


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("kind", ["even", "one", "ragged"])
@pytest.mark.parametrize("form,E,S,K,N", EXPERTS)
def test_experts(tf, form, kind, gather, E, S, K, N):
    A = S // 3 if gather else S
    q, s, w, ws = operands(E + S + K, A, K, E, N)
    packed, ends = tf.pack_w8a8(w, ws), offsets_of(kind, E, S)
    rows = torch.randint(0, A, (S,), device="cuda") if gather else torch.arange(S, device="cuda")
    if gather:
        rows[3], rows[S // 2], rows[S - 5] = -1, A, 2 ** 31 - 1
    rows, offsets = rows.to(torch.int32), torch.tensor(ends, dtype=torch.int32, device="cuda")
    for dt in ("f16", "bf16"):
        out = torch.full((S + 2, N), 7.0, dtype=DT[dt], device="cuda")
        tf.w8a8_expert_gemm(q, s, packed, K, N, offsets, rows if gather else None, out=out[:S])
        check_experts(out, dt, q, s, w, ws, ends, rows)


@pytest.mark.parametrize("a_rows", [1, 5, 149])
@pytest.mark.parametrize("form,E,S,K,N", PAST)
def test_slots_past_the_last_row(tf, form, E, S, K, N, a_rows):
    """Without rows, slots past the last row of A are rows that do not exist (the C
    entry; the binding has a slot for each row)."""
    q, s, w, ws = operands(E + a_rows, a_rows, K, E, N)
    packed, ends = tf.pack_w8a8(w, ws), offsets_of("even", E, S)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    out = torch.full((S + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    tf._launch("tf_w8a8_expert_gemm", out.device, tf.TF_BF16, tf._ptr(q), tf._ptr(s), a_rows, tf._ptr(packed),
               tf._ptr(offsets), None, tf._ptr(out), S, K, N, E)
    check_experts(out, "bf16", q, s, w, ws, ends, torch.arange(S, device="cuda"))
