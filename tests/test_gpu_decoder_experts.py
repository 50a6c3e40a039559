"""MLPs of any number of experts in a decoder layer (the router's product takes columns
by the eight)."""
from __future__ import annotations

import numpy as np
import pytest

import oracle
from test_gpu_experts import DT, E32, U, down, tf, up  # noqa: F401
from test_gpu_experts_layer import dec, layer_of  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("E,k", [(1, 1), (3, 2), (6, 6), (60, 4)])
def test_any_number_of_experts(tf, dec, dt, T, E, k):
    """The choice as the router's weights make it, and the sum over the chosen experts of
    what each alone gives."""
    cfg, w = layer_of(dec, dt, experts=E, top_k=k)
    layer = dec.Layer(cfg, w)
    x, _ = up(np.random.default_rng(T).standard_normal((T, cfg.hidden)), dt)
    out = layer._mlp(x)
    q, s = tf.quantize_rows(x)
    exact = oracle.w8a8(q.cpu().numpy(), down(s), w["router"][0].cpu().numpy(), down(w["router"][1]))
    # the logits' own rounding: the sum's conversion, two fp32 products, the output's
    logits = tf.w8a8_gemm(q, s, layer.router, cfg.hidden, layer.router_columns, dtype=DT[dt])[:, :E]
    assert logits.shape == (T, E)
    assert (np.abs(down(logits) - exact) <= (U[dt] + 4 * E32) * np.abs(exact) + 2.0 ** -25).all()
    weights, experts = oracle.route(down(logits), k, renormalize=True)
    ys, terms = np.zeros((T, cfg.hidden)), np.zeros((T, cfg.hidden))
    for e in range(E):
        one = [tf.pack_w8a8(w[n][0][e].contiguous(), w[n][1][e].contiguous()) for n in ("gate_up", "down")]
        g = tf.w8a8_gemm(q, s, one[0], *cfg.linears()["gate_up"], dtype=DT[dt])
        y = down(tf.w8a8_gemm(*tf.quantize_rows(g, gated=True), one[1], *cfg.linears()["down"], dtype=DT[dt]))
        mine = ((experts == e) * weights).sum(1)[:, None]
        ys += mine * y
        terms += np.abs(mine * y)
    # a weight's rounding and a partial sum's a term, the output's
    assert (np.abs(down(out) - ys) <= U[dt] * np.abs(ys) + (k + 3) * E32 * terms + 2.0 ** -25).all()


def test_command_runs(dec, capsys):
    dec.main(["--layers", "1", "--prompt", "40", "--batch", "2", "--steps", "3", "--eight-bit", "--experts", "3"])
    assert "us a step" in capsys.readouterr().out
