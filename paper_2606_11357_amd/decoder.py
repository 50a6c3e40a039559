"""Decoder layers of the library's operators: 4-bit linear layers, norms with the
residual sum, rotation and a 4-bit paged key/value cache, attention over prompts
and over the cache.

    python -m paper_2606_11357_amd.decoder [--layers 2 --prompt 2048 --batch 8 --steps 16]

runs a prompt for each sequence, then decode steps (one captured graph, replayed),
on layers of the Llama-3-8B shape with random weights, and prints what each took.

A layer (pre-norm, as Llama's):

    n, r   = add_rms_norm(x, r, w_in)              r: the residual stream
    q,k,v  = w4a16(n, W_qkv)                       one packed projection
    q, k   = kv4_append(...)                       rotate, quantize into the cache
    o      = prompt_attention(q, k, v)             a prompt's own tokens in 16 bits
           | prompt_attention(q, *kv4_read(...))   a chunk after cached ones
           | kv4_attention(q, cache)               single tokens
    n, r   = add_rms_norm(w4a16(o, W_o), r, w_mlp)
    x      = w4a16(silu_mul(w4a16(n, W_gate_up)), W_down)
"""
from __future__ import annotations

import argparse
import dataclasses

from . import tilefuse as tf


@dataclasses.dataclass(frozen=True)
class Config:
    """The shape of a layer; the defaults are Llama-3-8B's."""
    hidden: int = 4096
    q_heads: int = 32
    kv_heads: int = 8
    head_dim: int = 128
    mlp: int = 14336
    group: int = 128
    eps: float = 1e-5
    theta: float = 500000.0

    @property
    def qkv(self):
        return (self.q_heads + 2 * self.kv_heads) * self.head_dim

    def linears(self):
        """(K, N) of the linear layers by name."""
        return {"qkv": (self.hidden, self.qkv), "o": (self.q_heads * self.head_dim, self.hidden),
                "gate_up": (self.hidden, 2 * self.mlp), "down": (self.mlp, self.hidden)}


def rotation(cfg: Config, positions: int, device="cuda"):
    """cos and sin of the rotation, fp32 [positions, head_dim / 2] each."""
    import torch
    half = torch.arange(cfg.head_dim // 2, device=device, dtype=torch.float64)
    a = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * cfg.theta ** (-2 * half / cfg.head_dim)
    return a.cos().float().contiguous(), a.sin().float().contiguous()


class Layer:
    """One decoder layer.  weights: for each linear layer the AWQ tensors
    (qweight, qzeros, scales), packed here once, and the norm weights "norm_in"
    and "norm_mlp"; the scales' type (fp16 or bf16) is the layer's."""

    def __init__(self, cfg: Config, weights: dict):
        self.cfg = cfg
        self.packed = {n: tf.pack_w4(*weights[n], K, N, cfg.group) for n, (K, N) in cfg.linears().items()}
        self.norm_in, self.norm_mlp = weights["norm_in"], weights["norm_mlp"]

    def _linear(self, name, x):
        K, N = self.cfg.linears()[name]
        f = tf.w4a16_gemv if x.shape[0] == 1 else tf.w4a16_gemm
        return f(x, self.packed[name], K, N, self.cfg.group)

    def __call__(self, x, residual, cache, table, cu, starts, cos, sin, lens=None, prefix=None):
        """x, residual: [tokens, hidden] (residual None before the first layer), the
        packed tokens of the sequences as cu says, from position starts[b] on.

        lens given: single tokens (as many of each sequence, up to 8) that attend
        over the cache, lens counting them.  Otherwise prompts, whose tokens attend
        over each other, or, with prefix = (cu_k, zeros, keys), over the keys that
        kv4_read gives for those offsets: all of their sequence so far.
        Returns (x, residual) for the next layer."""
        c = self.cfg
        T = x.shape[0]
        n, residual = tf.add_rms_norm(x, residual, self.norm_in, eps=c.eps)
        qkv = self._linear("qkv", n).view(T, -1, c.head_dim)
        q, k, v = qkv[:, :c.q_heads], qkv[:, c.q_heads:c.q_heads + c.kv_heads], qkv[:, c.q_heads + c.kv_heads:]
        own = lens is None and prefix is None
        q, k = tf.kv4_append(cache, table, cu, starts, k, v, cos, sin, q=q, keys=own)
        if lens is not None:
            o = tf.kv4_attention(q.view(lens.shape[0], -1, c.q_heads, c.head_dim), cache, table, lens)
        elif own:
            o = tf.prompt_attention(q, k, v, cu)
        else:
            cu_k, first, keys = prefix
            o = tf.prompt_attention(q, *tf.kv4_read(cache, table, cu_k, first, keys), cu, cu_k)
        n, residual = tf.add_rms_norm(self._linear("o", o.view(T, -1)), residual, self.norm_mlp, eps=c.eps)
        return self._linear("down", tf.silu_mul(self._linear("gate_up", n))), residual


class Stack:
    """Layers one after the other with a cache each, and a final norm."""

    def __init__(self, layers, final_norm, pages: int, page_size: int, positions: int, dtype):
        self.layers, self.final_norm = layers, final_norm
        c = self.cfg = layers[0].cfg
        self.caches = [tf.kv4_cache(pages, page_size, c.kv_heads, c.head_dim, dtype=dtype) for _ in layers]
        self.cos, self.sin = rotation(c, positions)

    def __call__(self, x, table, cu, starts, lens=None, prefix=None):
        residual = None
        for layer, cache in zip(self.layers, self.caches):
            x, residual = layer(x, residual, cache, table, cu, starts, self.cos, self.sin, lens, prefix)
        return tf.add_rms_norm(x, residual, self.final_norm, eps=self.cfg.eps)[0]


def random_weights(cfg: Config, dtype, seed: int, device="cuda") -> dict:
    """Random AWQ tensors of a layer; scales that keep its outputs near those of a
    trained one (each linear layer's output of the size of its input)."""
    import torch
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    word = lambda *shape: torch.randint(-2 ** 31, 2 ** 31, shape, dtype=torch.int32, device=device, generator=gen)  # noqa: E731
    w = {}
    for name, (K, N) in cfg.linears().items():
        step = (12 * K) ** -0.5 / 3         # codes minus zero-points spread over about 6.5 of 16 steps
        s = step * (1 + torch.rand((K // cfg.group, N), device=device, generator=gen))
        w[name] = (word(K, N // 8), word(K // cfg.group, N // 8), s.to(dtype))
    for name in ("norm_in", "norm_mlp"):
        w[name] = (1 + 0.1 * torch.randn(cfg.hidden, device=device, generator=gen)).to(dtype)
    return w


def main(argv=None):
    import time

    import torch
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=2048, help="tokens of each prompt")
    ap.add_argument("--batch", type=int, default=8, help="sequences")
    ap.add_argument("--steps", type=int, default=16, help="decode steps")
    ap.add_argument("--dtype", choices=("f16", "bf16"), default="bf16")
    a = ap.parse_args(argv)
    cfg, page = Config(), 64
    dtype = torch.float16 if a.dtype == "f16" else torch.bfloat16
    layers = [Layer(cfg, random_weights(cfg, dtype, i)) for i in range(a.layers)]
    per_seq = -(-(a.prompt + a.steps + 1) // page)
    ones = torch.ones(cfg.hidden, device="cuda", dtype=dtype)
    stack = Stack(layers, ones, a.batch * per_seq, page, a.prompt + a.steps + 1, dtype)
    table = torch.randperm(a.batch * per_seq, device="cuda").to(torch.int32).view(a.batch, per_seq)
    cu = torch.arange(a.batch + 1, device="cuda", dtype=torch.int32) * a.prompt
    starts = torch.zeros(a.batch, device="cuda", dtype=torch.int32)
    x = torch.randn(a.batch * a.prompt, cfg.hidden, device="cuda").to(dtype)

    def timed(f, n):
        f()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(n):
            f()
        torch.cuda.synchronize()
        return (time.perf_counter() - t) / n

    t = timed(lambda: stack(x, table, cu, starts), 3)
    print(f"prompts: {a.batch} x {a.prompt} tokens, {a.layers} layers: {1e3 * t:.3f} ms "
          f"({a.batch * a.prompt / t:.0f} tokens/s a stack of {a.layers})")

    # decode: positions and lengths advance on the device, so one graph serves every step
    one = torch.arange(a.batch + 1, device="cuda", dtype=torch.int32)
    pos = torch.full((a.batch,), a.prompt, device="cuda", dtype=torch.int32)
    lens = pos + 1
    token = torch.randn(a.batch, cfg.hidden, device="cuda").to(dtype)
    stack(token, table, one, pos, lens)          # once outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = stack(token, table, one, pos, lens)
        token.copy_(out)
        pos.add_(1)
        lens.add_(1)
    t = timed(graph.replay, a.steps - 1)
    print(f"decode: {a.batch} sequences from {a.prompt} cached tokens, {a.layers} layers: {1e6 * t:.1f} us a step "
          f"({1e6 * t / a.layers:.1f} us a layer)")
    assert torch.isfinite(out).all()


if __name__ == "__main__":
    main()
