"""8-bit codes and products at the ends of their types' ranges, against the CPU oracle
in float64."""
from __future__ import annotations

import numpy as np
import pytest

import oracle
from test_gpu_experts import DT, E32, down, put, tf  # noqa: F401

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
