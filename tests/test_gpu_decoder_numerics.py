"""Attention where softmax weights are of very different sizes: one key that takes
most of a row's weight and whose value is near nothing (so that the result is what
all the others add up to), and values whose sizes differ by powers of two.

Tolerances are those of test_gpu_decoder_ops: relative to sum p |v|, which the key
that takes most has no part in.
"""
from __future__ import annotations

import numpy as np
import pytest

import oracle
from test_gpu_decoder_ops import DT, check_decode, down, i32, offsets, table_for, tf, up  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def sink_inputs(rng, heads, n, batch, new, size, margin):
    """Queries that score about `margin` above all other keys on key 0, whose value is
    a hundredth of the others' size."""
    Hq, Hk, D = heads
    d = rng.choice([-1.0, 1.0], D)
    k = 0.05 * rng.standard_normal((n, Hk, D))
    k[0] = d * margin / D ** 0.5
    v = size * (rng.standard_normal((n, Hk, D)) + 0.5)
    v[0] *= 0.01
    q = d + 0.1 * rng.standard_normal((batch, new, Hq, D))
    return q, k, v


def cached(tf, dt, k, v, lens, page, rng):
    (k, kv), (v, vv) = up(k, dt), up(v, dt)
    table, pages = table_for(lens, page, rng)
    cache = tf.kv4_cache(pages, page, k.shape[1], k.shape[2], dtype=DT[dt])
    cache.data.fill_(0xFF)
    tf.kv4_append(cache, table, i32(offsets(lens)), i32([0] * len(lens)), k, v)
    return cache, table, *(oracle.cached_rows(x.astype(np.float32), dt) for x in (kv, vv))


SINKS = [((8, 2, 128), 8192, 1, 0.1, 11.3), ((8, 2, 128), 16384, 1, 0.02, 12.4), ((4, 1, 64), 32768, 3, 0.02, 12.0),
         ((8, 1, 256), 20000, 1, 0.05, 12.0), ((8, 1, 256), 65537, 4, 0.05, 13.3), ((16, 1, 128), 9000, 2, 2e-3, 11.0)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("batch", [1, 1100])
@pytest.mark.parametrize("heads,n,new,size,margin", SINKS, ids=str)
def test_decode_beside_a_key_that_takes_most(tf, dt, batch, heads, n, new, size, margin):
    """One sequence, whose keys many workgroups share, and many on the same pages, of
    which a workgroup takes one whole."""
    rng = np.random.default_rng(n)
    q, k, v = sink_inputs(rng, heads, n, batch, new, size, margin)
    cache, table, k, v = cached(tf, dt, k, v, [n], 64, rng)
    q, qv = up(q, dt)
    got = down(tf.kv4_attention(q, cache, table.expand(batch, -1).contiguous(), i32([n] * batch)))
    assert np.isfinite(got).all()
    for b in {0, batch // 2, batch - 1}:
        check_decode(dt, got[b:b + 1], qv[b:b + 1], k, v, [n], heads, new)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
@pytest.mark.parametrize("heads,new", [((8, 2, 128), 1), ((8, 1, 256), 4), ((4, 2, 64), 2)], ids=str)
def test_decode_of_values_of_all_sizes(tf, dt, order, heads, new):
    """Values from 2^-20 (scales that fp16 holds as subnormals) to 2^15."""
    lens = [3000, 700]
    rng = np.random.default_rng(len(order))
    size = np.concatenate([2.0 ** np.linspace(-20, 14, n) for n in lens])
    size = {"rising": size, "falling": size[::-1], "mixed": rng.permutation(size)}[order]
    shape = (sum(lens), heads[1], heads[2])
    k, v = rng.standard_normal(shape), size[:, None, None] * np.clip(rng.standard_normal(shape), -1.9, 1.9)
    cache, table, k, v = cached(tf, dt, k, v, lens, 64, rng)
    q, qv = up(rng.standard_normal((2, new, heads[0], heads[2])), dt)
    check_decode(dt, down(tf.kv4_attention(q, cache, table, i32(lens))), qv, k, v, lens, heads, new)


@pytest.mark.parametrize("new", [1, 4])
def test_decode_of_hidden_large_values(tf, new):
    """Values of 2^14 that a row does not see leave its bits as they are."""
    heads, n = (8, 2, 128), 333
    rng = np.random.default_rng(7)
    k, v = 0.3 * rng.standard_normal((n + 1, 2, 128)), 1e-3 * rng.standard_normal((n + 1, 2, 128))
    q, _ = up(rng.standard_normal((1, new, 8, 128)), "f16")
    out = []
    for size in (1.0, 2.0 ** 24):
        v[-1] *= size                     # of the last token: past the length, or seen by the last row alone
        cache, table, *_ = cached(tf, "f16", k, v, [n + 1], 64, np.random.default_rng(8))
        out.append(tf.kv4_attention(q, cache, table, i32([n + 1 if new > 1 else n])))
    seen = new - 1 if new > 1 else 1
    assert torch.equal(out[0][:, :seen], out[1][:, :seen])


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("split", [False, None], ids=["whole", "split"])
@pytest.mark.parametrize("heads,n_q,n_k,margin", [((4, 1, 128), 9, 30000, 16.23), ((2, 2, 64), 3, 65536, 16.23),
                                                  ((2, 1, 256), 5, 20000, 15.5), ((2, 1, 128), 130, 4000, 12.0)], ids=str)
def test_prompt_beside_a_key_that_takes_most(tf, dt, split, heads, n_q, n_k, margin):
    """Per query: u for the output, u sum p |v| for the rounded weights (fp16: those
    under 2^-21 of the largest lose at most 2^-32 each), the scores' fp32 error e as in
    check_prompt."""
    Hq, Hk, D = heads
    rng = np.random.default_rng(n_k)
    d = rng.choice([-1.0, 1.0], D)
    k = 0.01 * rng.standard_normal((n_k, Hk, D))
    k[0] = d * margin / D ** 0.5
    v = rng.standard_normal((n_k, Hk, D)) + 0.5
    v[0] *= 0.01
    (q, qv), (k, kv), (v, vv) = (up(t, dt) for t in (np.broadcast_to(d, (n_q, Hq, D)), k, v))
    got = down(tf.prompt_attention(q, k, v, i32([0, n_q]), i32([0, n_k]), workspace=split))
    u, least = (2.0 ** -11, 2.0 ** -32) if dt == "f16" else (2.0 ** -8, 0.0)
    for h in range(Hq):
        one = (qv[:, h], kv[:, h * Hk // Hq], vv[:, h * Hk // Hq], D ** -0.5, n_k - n_q + np.arange(n_q))
        want, bound = oracle.attend(*one), oracle.attend_bound(*one)
        e = 2.0 ** -21 * D ** -0.5 * D * np.abs(kv).max()
        tol = u * np.abs(want) + (u + 2 * e + 2.0 ** -20) * bound + least * (n_k * np.abs(vv).max() + 128)
        assert (np.abs(got[:, h] - want) <= tol).all(), (h, np.abs(got[:, h] - want).max(), tol.min())
