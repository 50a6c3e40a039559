"""A decoder layer of the library's operators against the same layer in float64
from the oracle: prompts, a chunk after cached tokens, and decode steps, one
after the other on one cache.

The reference keeps the 16-bit rounding of every tensor that the layer stores,
which is part of what the layer defines (and decides the codes of keys and
values near a tie).  What is left are the operators' own errors: some ten
tensors that differ by a rounding in places, and a code in some hundred by one,
a step of range / 15; 3e-2 (bf16) and 1e-2 (fp16) of the output's norm.
"""
from __future__ import annotations

import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
TOL = {"f16": 1e-2, "bf16": 3e-2}


@pytest.fixture(scope="module")
def dec():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_11357_amd import decoder
    return decoder


def dequant(w, group):
    """AWQ tensors -> float64 weights."""
    q, z, s = (t.cpu() for t in w)
    shift = torch.arange(0, 32, 4, dtype=torch.int32)
    nib = lambda t: ((t[:, :, None] >> shift) & 15).reshape(t.shape[0], -1).double()  # noqa: E731
    rep = lambda t: t.repeat_interleave(group, 0)  # noqa: E731
    return ((nib(q) - rep(nib(z))) * rep(s.double())).numpy()


class Reference:
    """The layer in float64; caches[b] the cached keys and values of sequence b."""

    def __init__(self, cfg, weights, dt, batch):
        self.cfg, self.dt = cfg, dt
        self.w = {n: dequant(weights[n], cfg.group) for n in cfg.linears()}
        self.norms = [weights[n].double().cpu().numpy() for n in ("norm_in", "norm_mlp")]
        c = cfg
        self.k = [np.zeros((0, c.kv_heads, c.head_dim)) for _ in range(batch)]
        self.v = [np.zeros((0, c.kv_heads, c.head_dim)) for _ in range(batch)]

    def __call__(self, x, lens, mode, cos, sin):
        c, out = self.cfg, []
        r16 = lambda t: oracle.round16(t, self.dt)  # noqa: E731
        n, r = oracle.rms_norm_block(x, weight=self.norms[0], eps=c.eps)
        qkv = r16(r16(n) @ self.w["qkv"]).reshape(len(x), -1, c.head_dim)
        at = 0
        for b, m in enumerate(lens):
            past = len(self.k[b])
            pos = past + np.arange(m)
            turn = lambda t: oracle.rotate(t, cos[pos], sin[pos])  # noqa: E731
            part = qkv[at:at + m]
            q, k, v = turn(part[:, :c.q_heads]), turn(part[:, c.q_heads:-c.kv_heads]), part[:, -c.kv_heads:]
            cached = lambda t: oracle.cached_rows(t.astype(np.float32), self.dt)  # noqa: E731
            self.k[b], self.v[b] = np.concatenate([self.k[b], cached(k)]), np.concatenate([self.v[b], cached(v)])
            q, k = r16(q), r16(k)
            ks, vs = (k, v) if mode == "prompt" else (self.k[b], self.v[b])
            if mode == "chunk":                   # read back as 16-bit values
                ks, vs = r16(ks), r16(vs)
            o = np.stack([oracle.attend(q[:, h], ks[:, h * c.kv_heads // c.q_heads], vs[:, h * c.kv_heads // c.q_heads],
                                        c.head_dim ** -0.5, len(ks) - m + np.arange(m)) for h in range(c.q_heads)], 1)
            out.append(o.reshape(m, -1))
            at += m
        n, r = oracle.rms_norm_block(r16(r16(np.concatenate(out)) @ self.w["o"]), r, self.norms[1], eps=c.eps)
        gu = r16(r16(n) @ self.w["gate_up"])
        g, u = gu[:, :c.mlp], gu[:, c.mlp:]
        return r16(oracle.silu(g) * u) @ self.w["down"], r


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 1, 128)], ids=str)
def test_layer(dec, dt, heads):
    cfg = dec.Config(hidden=256, q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], mlp=512, theta=10000.0)
    weights = dec.random_weights(cfg, DT[dt], 1)
    layer, page = dec.Layer(cfg, weights), 32
    tf = dec.tf
    cache = tf.kv4_cache(14, page, cfg.kv_heads, cfg.head_dim, dtype=DT[dt])
    table = torch.randperm(14, device="cuda").to(torch.int32).view(2, 7)
    cos, sin = dec.rotation(cfg, 224)
    ref = Reference(cfg, weights, dt, 2)
    cn, sn = cos.double().cpu().numpy(), sin.double().cpu().numpy()
    i32 = lambda a: torch.tensor(list(a), dtype=torch.int32).cuda()  # noqa: E731
    done = np.zeros(2, int)
    torch.manual_seed(5)
    for lens, mode in (([70, 33], "prompt"), ([20, 45], "chunk"), ([1, 1], "decode"), ([1, 1], "decode"),
                       ([3, 3], "decode")):
        x = torch.randn(sum(lens), cfg.hidden, device="cuda").to(DT[dt])
        args = [cache, table, i32([0, lens[0], sum(lens)]), i32(done), cos, sin]
        after = done + lens
        if mode == "decode":
            args.append(i32(after))
        elif mode == "chunk":
            args += [None, (i32([0, after[0], after.sum()]), i32([0, 0]), int(after.sum()))]
        y, r = layer(x, None, *args)
        want, want_r = ref(x.double().cpu().numpy(), lens, mode, cn, sn)
        for got, w in ((y, want), (r, want_r)):
            got = got.double().cpu().numpy()
            assert np.linalg.norm(got - w) <= TOL[dt] * np.linalg.norm(w), (mode, np.linalg.norm(got - w) / np.linalg.norm(w))
        done = after


def test_command_runs(dec, capsys):
    dec.main(["--layers", "1", "--prompt", "200", "--batch", "2", "--steps", "3"])
    assert "us a step" in capsys.readouterr().out
