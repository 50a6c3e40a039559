"""8-bit codes and products at the ends of their types' ranges, against the CPU oracle
in float64."""
from __future__ import annotations

import numpy as np
import pytest

import oracle
from test_gpu_experts import DT, E32, TINY, U, down, tf  # noqa: F401
from test_gpu_w8a8_forms import ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def gated_codes(x):
    with np.errstate(over="ignore", invalid="ignore"):
        return oracle.row_codes(oracle.gated_rows(x))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("N", [16, 528, 2064, 14336])
def test_gated_codes_of_extreme_gates(tf, dt, N):
    """Gates at which e^-g leaves fp32, up to the type's lowest and highest values,
    in rows of ordinary ones and alone, beside factors that are as large.

    h = g u e^g there: an exponential of g / 2 twice (two units in the last place, 4
    roundings, each) and three products, 11 roundings; elsewhere fewer.  Twice that
    (h and its row's maximum), then 127 / max and the product."""
    rng = np.random.default_rng(N)
    most = float(torch.finfo(DT[dt]).max)
    rows = [  # (gates, factors) put over the first places of an ordinary row
        ([-most], [1.0]), ([-most, most], [1.0, 0.0]), ([most], [0.25]), ([-100.0, -90.0], [1.0, most]),
        ([-88.0, -87.5, -87.0, -80.0], [most, most, most, -most]), ([-95.0, -104.0, -120.0], [most, -most, most]),
        ([-64.0, -64.5, -63.5, -65.0], [most] * 4), ([-most, -most / 2], [most, -most]), ([-np.inf], [1.0]),
        ([np.inf], [1.0]), ([np.nan], [0.0]), ([-most], [np.inf]), ([-100.0], [-np.inf])]
    x = np.zeros((len(rows) + 4, 2 * N))
    x[:, :N], x[:, N:] = rng.standard_normal((2, len(x), N))
    for r, (g, u) in enumerate(rows):
        x[r, N - len(g):N], x[r, 2 * N - len(g):] = g, u
    # whole rows of them
    x[-4, :N], x[-4, N:] = -most, most
    x[-3, :N], x[-3, N:] = np.linspace(-110, -55, N), most / 2
    x[-2, :N] = np.linspace(-66, -60, N)
    x[-1, :N], x[-1, N:] = np.linspace(-150, -100, N), 1.0
    t = torch.from_numpy(x).to(DT[dt])
    v, unit = gated_codes(t.double().numpy())
    q, s = tf.quantize_rows(t.cuda(), gated=True)
    s, q = down(s), down(q)
    np.testing.assert_array_equal(np.isnan(s), np.isnan(unit))
    ok = ~np.isnan(unit)
    assert ok.sum() == len(x) - 5
    assert (np.abs(s - unit)[ok] <= (11 + 1) * E32 * unit[ok]).all()
    assert (np.abs(q - v) <= 0.5 + (2 * 11 + 2) * E32 * 127).all()
    assert (q[-4] == 0).all() and s[-4] == 0 and (q[-1] == 0).all() and s[-1] == 0


def far_scales(n):
    """Powers of two over all that fp32 holds, subnormal ones too, times 1 to 2."""
    e = torch.randint(-149, 128, (n,), device="cuda")
    return torch.ldexp(1 + torch.rand(n, dtype=torch.float64, device="cuda"), e).clamp_max(3.4e38).float()


def check_far(got, want, dt):
    """Outputs past the type's highest value are infinite, others as ever; under the
    lowest normal fp32 value one more rounding to a multiple of 2^-149."""
    most, got = float(torch.finfo(DT[dt]).max), got.double()
    over, within = want.abs() > most * (1 + 2 * U[dt]), want.abs() < most
    assert torch.equal(got[over], want[over].sign() * np.inf)
    tiny = {"f16": TINY["f16"], "bf16": 2.0 ** -134}[dt] + 2.0 ** -150
    assert ((got - want).abs() <= (U[dt] + 4 * E32) * want.abs() + tiny)[within].all()
    assert within.any() and over.any() and (want[within].abs() > 2.0 ** -20).any()


# direct, 64 x 64, K split, 128 x 128 (several tiles a workgroup), 256 x 256
@pytest.mark.parametrize("M,K,N", [(5, 1040, 264), (100, 1040, 520), (64, 8208, 264), (2100, 1040, 4104), (2100, 2064, 4104)])
def test_products_of_far_scales(tf, M, K, N):
    """Scales whose product leaves fp32 where the output does not."""
    torch.manual_seed(M + K)
    q, w = ints(M, K), ints(K, N)
    q[0] = 0
    s, ws = far_scales(M), far_scales(N)
    s[0], s[1], s[2] = 3e38, 0.0, 1.0
    ws[0], ws[1], ws[2] = 3e38, 0.0, 1.0
    packed = tf.pack_w8a8(w, ws)
    want = (q.double() @ w.double()) * s.double()[:, None] * ws.double()
    for dt in ("f16", "bf16"):
        out = tf.w8a8_gemm(q, s, packed, K, N, dtype=DT[dt])
        check_far(out, want, dt)
        assert (out[0] == 0).all() and (out[1] == 0).all() and (out[:, 1] == 0).all()


def test_far_scales_leave_the_others(tf):
    """Rows and columns of ordinary scales have the same bits beside far ones as alone."""
    M, K, N = 300, 1040, 520
    q, w = ints(M, K), ints(K, N)
    s, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda") * 1e-4
    want = tf.w8a8_gemm(q, s, tf.pack_w8a8(w, ws), K, N, dtype=torch.bfloat16)
    s[::7], ws[::5] = 1e-38, 1e38
    got = tf.w8a8_gemm(q, s, tf.pack_w8a8(w, ws), K, N, dtype=torch.bfloat16)
    rows, cols = torch.arange(M, device="cuda") % 7 != 0, torch.arange(N, device="cuda") % 5 != 0
    assert torch.equal(got[rows][:, cols], want[rows][:, cols])


# direct, 64 x 64, 64 x 128, 256 x 256
@pytest.mark.parametrize("E,S,K,N", [(8, 150, 2064, 264), (5, 150, 1040, 2056), (5, 1000, 1040, 1032), (3, 2000, 2064, 4104)])
@pytest.mark.parametrize("gather", [False, True])
def test_experts_of_far_scales(tf, gather, E, S, K, N):
    """The same by expert; rows that do not exist are zeros by columns of any scale."""
    torch.manual_seed(E + S)
    A = S // 2 if gather else S - S // 5
    q, w = ints(A, K), ints(E, K, N)
    s, ws = far_scales(A), far_scales(E * N).view(E, N)
    ws[:, 3], ws[:, 4], ws[:, 5] = float("inf"), float("nan"), 3.4e38
    packed = tf.pack_w8a8(w, ws)
    rows = torch.randint(0, A, (S,), device="cuda") if gather else torch.arange(S, device="cuda")
    if gather:
        rows[::9], rows[4::11] = -1, A
    rows32 = rows.to(torch.int32)
    ends = [S * e // E for e in range(E + 1)]
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    there = (rows >= 0) & (rows < A)
    at = rows.clamp(0, A - 1)
    finite = torch.isfinite(ws).all(0)
    for dt in ("f16", "bf16"):
        out = torch.full((S, N), 7.0, dtype=DT[dt], device="cuda")
        tf._launch("tf_w8a8_expert_gemm", out.device, tf._dtype_code(DT[dt], "dt"), tf._ptr(q), tf._ptr(s), A, tf._ptr(packed),
                   tf._ptr(offsets), tf._ptr(rows32) if gather else None, tf._ptr(out), S, K, N, E)
        assert (out[~there] == 0).all()
        for e in range(E):
            mine = torch.arange(ends[e], ends[e + 1], device="cuda")
            mine = mine[there[mine]]
            if not len(mine):
                continue
            sums = q[at[mine]].double() @ w[e].double()
            check_far(out[mine][:, finite], (sums * s[at[mine]].double()[:, None] * ws[e].double())[:, finite], dt)
            assert torch.isnan(out[mine][:, 4]).all() and (~torch.isfinite(out[mine][:, 3])).all()
