"""The operators of 8-bit layers and experts together, as a decoder layer runs them:
the MLP against the same in float64, on streams, on other calls' heels, captured into
graphs that are replayed with new inputs, and two at once; the native and the general
path of the binding."""
from __future__ import annotations

import numpy as np
import pytest

import oracle
from test_gpu_experts import DT, E32, U, down, put, tf, up, weight  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec(tf):
    from paper_2606_11357_amd import decoder
    return decoder


def layer_of(dec, dt, **kw):
    cfg = dec.Config(hidden=256, q_heads=4, kv_heads=2, head_dim=64, mlp=272, theta=10000.0, **kw)
    return cfg, dec.random_weights(cfg, DT[dt], 1, eight_bit=True)


def codes_within(got_q, got_s, x):
    """Codes and scales of rows x (float64 of what the kernel read)."""
    v, unit = oracle.row_codes(x)
    assert (np.abs(down(got_s) - unit) <= 8 * E32 * unit).all()
    assert (np.abs(down(got_q) - v) <= 0.5 + 16 * E32 * 127).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 64, 700])
@pytest.mark.parametrize("E,k", [(8, 2), (16, 5)])
def test_mlp_of_experts(tf, dec, dt, T, E, k):
    """Every stage from what the one before gave, by the oracle's definition, and the
    whole as the layer runs it, bit for bit."""
    cfg, w = layer_of(dec, dt, experts=E, top_k=k)
    layer = dec.Layer(cfg, w)
    x, xv = up(np.random.default_rng(T).standard_normal((T, cfg.hidden)), dt)
    (K1, N1), (K2, N2) = cfg.linears()["gate_up"], cfg.linears()["down"]
    int8 = {n: (w[n][0].cpu().numpy(), down(w[n][1])) for n in ("router", "gate_up", "down")}
    near = lambda got, want: (np.abs(down(got) - want) <= (U[dt] + 4 * E32) * np.abs(want) + 2.0 ** -25).all()  # noqa: E731

    q, s = tf.quantize_rows(x)
    codes_within(q, s, xv)
    qn, sn = q.cpu().numpy(), down(s)
    logits = tf.w8a8_gemm(q, s, layer.router, cfg.hidden, E, dtype=DT[dt])
    assert near(logits, oracle.w8a8(qn, sn, *int8["router"]))
    r = tf.route_experts(logits, k, renormalize=True)
    weights, experts = oracle.route(down(logits), k, renormalize=True)
    offsets, tokens, places = oracle.expert_order(experts, E)
    for got, want in zip(r[1:], (experts, offsets, tokens, places)):
        np.testing.assert_array_equal(got.cpu().numpy(), want)
    g = tf.w8a8_expert_gemm(q, s, layer.packed["gate_up"], K1, N1, r.offsets, r.tokens, dtype=DT[dt])
    assert near(g, oracle.expert_products(qn, sn, *int8["gate_up"], offsets, tokens))
    h, hs = tf.quantize_rows(g, gated=True)
    codes_within(h, hs, oracle.gated_rows(down(g)))
    y = tf.w8a8_expert_gemm(h, hs, layer.packed["down"], K2, N2, r.offsets, dtype=DT[dt])
    assert near(y, oracle.expert_products(h.cpu().numpy(), down(hs), *int8["down"], offsets, np.arange(T * k)))
    out = tf.combine_experts(y, r.weights, r.places)
    want = oracle.combine(down(y), down(r.weights), places)
    terms = oracle.combine(np.abs(down(y)), down(r.weights), places)
    assert (np.abs(down(out) - want) <= U[dt] * np.abs(want) + (k + 2) * E32 * terms + 2.0 ** -25).all()
    assert torch.equal(layer._mlp(x), out)

    # and against the layer of unquantized activations: a code is off by half a step of
    # its row's maximum over 127 at most, some 3 standard deviations over it, so by 1 / 150 of
    # the row's norm on average in each of two products, and 16-bit outputs between
    wf = {n: int8[n][0] * int8[n][1][..., None, :] for n in int8}
    gu = np.stack([xv[t] @ wf["gate_up"][e] for e, t in zip(np.repeat(np.arange(E), np.diff(offsets)), tokens)])
    yf = np.stack([row @ wf["down"][e] for e, row in zip(np.repeat(np.arange(E), np.diff(offsets)), oracle.gated_rows(gu))])
    want = oracle.combine(yf, weights, places)
    assert np.linalg.norm(down(out) - want) <= 0.05 * np.linalg.norm(want)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_eight_bit_mlp(tf, dec, dt):
    cfg, w = layer_of(dec, dt)
    layer = dec.Layer(cfg, w)
    x, xv = up(np.random.default_rng(2).standard_normal((37, cfg.hidden)), dt)
    wf = {n: w[n][0].double().cpu().numpy() * down(w[n][1]) for n in ("gate_up", "down")}
    want = oracle.gated_rows(xv @ wf["gate_up"]) @ wf["down"]
    assert np.linalg.norm(down(layer._mlp(x)) - want) <= 0.05 * np.linalg.norm(want)


@pytest.mark.parametrize("T", [3, 200])
def test_captured_and_replayed(tf, dec, T):
    """Two graphs of the MLP, replayed in turn with new inputs, eager calls between: the
    routing, and with it every expert's rows, changes from replay to replay."""
    cfg, w = layer_of(dec, "bf16", experts=8, top_k=2)
    layer = dec.Layer(cfg, w)
    xs = [torch.randn(T, cfg.hidden, device="cuda").bfloat16() for _ in range(2)]
    layer._mlp(xs[0])
    graphs = []
    for x in xs:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layer._mlp(x)
        graphs.append((g, x, out))
    for i in range(4):
        for g, x, out in graphs:
            x.copy_(torch.randn(T, cfg.hidden, device="cuda").bfloat16() * (i + 1))
            g.replay()
            got = out.clone()
            assert torch.equal(got, layer._mlp(x))


def test_on_two_streams_at_once(tf, dec):
    cfg, w = layer_of(dec, "bf16", experts=8, top_k=2)
    layer = dec.Layer(cfg, w)
    xs = [torch.randn(300 + 100 * i, cfg.hidden, device="cuda").bfloat16() for i in range(2)]
    want = [layer._mlp(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(layer._mlp(xs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i]) for i in range(2) for g in got[i])


def test_same_bits_every_time(tf):
    """Tiles, routing and sums do not depend on which workgroup is first."""
    q = torch.randint(-128, 128, (900, 1040), device="cuda").to(torch.int8)
    packed = tf.pack_w8a8(torch.randint(-128, 128, (1040, 1288), device="cuda").to(torch.int8), torch.rand(1288, device="cuda"))
    s, x = torch.rand(900, device="cuda") * 1e-4, torch.randn(2000, 64, device="cuda").half()
    want, r = tf.w8a8_gemm(q, s, packed, 1040, 1288), tf.route_experts(x, 6)
    for _ in range(5):
        assert torch.equal(tf.w8a8_gemm(q, s, packed, 1040, 1288), want)
        assert all(torch.equal(a, b) for a, b in zip(tf.route_experts(x, 6), r))


def test_rows_of_many_sizes_agree(tf):
    """A row's product does not depend on how many others there are, and so on which
    kernel they run: the sums are whole numbers."""
    K, N = 1072, 264
    q = torch.randint(-128, 128, (1500, K), device="cuda").to(torch.int8)
    s = torch.rand(1500, device="cuda") * 1e-4
    packed = tf.pack_w8a8(torch.randint(-128, 128, (K, N), device="cuda").to(torch.int8), torch.rand(N, device="cuda"))
    want = tf.w8a8_gemm(q, s, packed, K, N, dtype=torch.bfloat16)
    for M in (1, 2, 15, 16, 17, 31, 48, 49, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 384, 640, 1023, 1025):
        assert torch.equal(tf.w8a8_gemm(q[:M], s[:M], packed, K, N, dtype=torch.bfloat16), want[:M]), M


@pytest.mark.parametrize("path", ["native", "general"])
@pytest.mark.parametrize("M,K,N", [(17, 14336, 4096), (49, 14336, 1032), (64, 8208, 264), (70, 14336, 4096), (128, 16384, 520)])
def test_split_over_k(tf, monkeypatch, path, M, K, N):
    """With the cached workspace, one of the caller's that starts as noise, and none: the
    same bits; rows behind the output stay as they are."""
    if path == "general":
        monkeypatch.setattr(tf, "_experts", {"gemm": lambda *call: NotImplemented})
    q = torch.randint(-128, 128, (M, K), device="cuda").to(torch.int8)
    w, ws = torch.randint(-128, 128, (K, N), device="cuda").to(torch.int8), torch.rand(N, device="cuda")
    s, packed = torch.rand(M, device="cuda") * 1e-5, tf.pack_w8a8(w, ws)
    need = tf.w8a8_workspace_bytes(M, K, N)
    assert need > 0
    big = torch.full((M + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    one = tf.w8a8_gemm(q, s, packed, K, N, out=big[:M], workspace=False)
    own = torch.randint(-2 ** 31, 2 ** 31, (need // 4 + 16,), dtype=torch.int32, device="cuda")
    keep = own[need // 4:].clone()
    for ws in (None, own, None, own[:need // 4]):
        out = torch.full((M + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
        tf.w8a8_gemm(q, s, packed, K, N, out=out[:M], workspace=ws)
        assert torch.equal(out, big)
    assert (big[M:] == 7).all() and torch.equal(own[need // 4:], keep)
    got = down(one)
    want = oracle.w8a8(q.cpu().numpy(), down(s), w.cpu().numpy(), packed_scales(tf, packed, K, N))
    assert (np.abs(got - want) <= (U["bf16"] + 4 * E32) * np.abs(want)).all()
    with pytest.raises(tf.TileFuseError) as err:
        tf.w8a8_gemm(q, s, packed, K, N, workspace=own[:8])
    assert err.value.status == tf.TF_ERR_ARG


def packed_scales(tf, packed, K, N):
    """The columns' scales at the end of a packed weight."""
    at = (N + 15) // 16 * ((K + 127) // 128 * 2) * 1024
    return packed[at:at + 4 * N].view(torch.float32).double().cpu().numpy()


def test_split_over_k_in_graphs(tf):
    """Two graphs and eager calls, larger ones too, between their replays: each has a
    workspace of its own."""
    K, N = 14336, 1024
    packed = tf.pack_w8a8(torch.randint(-127, 128, (K, N), device="cuda").to(torch.int8), torch.rand(N, device="cuda"))
    make = lambda M: torch.randint(-127, 128, (M, K), device="cuda").to(torch.int8)  # noqa: E731
    s, graphs = torch.rand(128, device="cuda") * 1e-5, []
    assert all(tf.w8a8_workspace_bytes(M, K, N) for M in (50, 64, 128))
    for M in (50, 64):
        q = make(M)
        tf.w8a8_gemm(q, s[:M], packed, K, N)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = tf.w8a8_gemm(q, s[:M], packed, K, N)
        graphs.append((g, q, out, M))
    side = torch.cuda.Stream()
    for _ in range(4):
        with torch.cuda.stream(side):
            other = make(128)
            got = tf.w8a8_gemm(other, s, packed, K, N)
        for g, q, out, M in graphs:
            q.copy_(make(M))
            g.replay()
            assert torch.equal(out, tf.w8a8_gemm(q, s[:M], packed, K, N, workspace=False))
        side.synchronize()
        assert torch.equal(got, tf.w8a8_gemm(other, s, packed, K, N, workspace=False))


@pytest.fixture(params=["native", "general"])
def path(request, tf, monkeypatch):
    if request.param == "general":
        monkeypatch.setattr(tf, "_experts", dict.fromkeys(("quantize", "gemm", "route", "expert_gemm", "combine"),
                                                          lambda *call: NotImplemented))


def test_forms_of_the_arguments(tf, path):
    """What the documentation allows, and what it refuses, on both paths."""
    x = torch.randn(6, 64, device="cuda").half()
    q, s = tf.quantize_rows(x)
    w, ws = torch.randint(-127, 128, (2, 64, 32), device="cuda").to(torch.int8), torch.rand(2, 32, device="cuda") * 1e-2
    packed, one = tf.pack_w8a8(w, ws), tf.pack_w8a8(w[0].contiguous(), ws[0])
    y = tf.w8a8_gemm(q, s, one, 64, 32)
    assert y.dtype == torch.float16 and torch.equal(tf.w8a8_gemm(q, s, one, 64, 32, out=torch.empty_like(y)), y)
    assert tf.w8a8_gemm(q, s, one, 64, 32, dtype=torch.bfloat16).dtype == torch.bfloat16
    assert tf.w8a8_gemm(q[:0], s[:0], one, 64, 32).shape == (0, 32)
    r = tf.route_experts(x[:, :2], 1, scale=2)
    assert isinstance(r, tf.Routing) and r.weights.shape == (6, 1)
    e = tf.w8a8_expert_gemm(q, s, packed, 64, 32, r.offsets, r.tokens)
    for i in range(2):
        mine = r.experts[:, 0] == i
        assert torch.equal(e[r.places[:, 0].long()][mine], tf.w8a8_gemm(q, s, tf.pack_w8a8(w[i].contiguous(), ws[i]), 64, 32)[mine])
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert tf.w8a8_expert_gemm(q, s, packed, 64, 32, r.offsets, none).shape == (0, 32)
    assert (tf.w8a8_expert_gemm(q[:0], s[:0], packed, 64, 32, r.offsets, r.tokens) == 0).all()
    assert torch.equal(tf.combine_experts(e, torch.ones(6, 1, device="cuda"), r.places), e[r.places[:, 0].long()])
    assert tf.quantize_rows(torch.empty(0, 64, device="cuda").half(), gated=True)[0].shape == (0, 32)
    i32 = torch.zeros(3, dtype=torch.int32, device="cuda")
    for call in (lambda: tf.quantize_rows(x.float()), lambda: tf.quantize_rows(x.t()), lambda: tf.quantize_rows(x[:, :3], gated=True),
                 lambda: tf.quantize_rows(x, codes=q[:3]), lambda: tf.w8a8_gemm(q.short(), s, one, 64, 32),
                 lambda: tf.w8a8_gemm(q, s.half(), one, 64, 32), lambda: tf.w8a8_gemm(q, s[:5], one, 64, 32),
                 lambda: tf.w8a8_gemm(q, s, one[:100], 64, 32), lambda: tf.w8a8_gemm(q, s, one, 64, 32, dtype=torch.float32),
                 lambda: tf.w8a8_gemm(q, s, one, 64, 32, out=y[:3]), lambda: tf.w8a8_gemm(q, s, one, 64, 32, dtype=torch.bfloat16, out=y),
                 lambda: tf.w8a8_gemm(q[:, ::2], s, one, 32, 32),
                 lambda: tf.w8a8_expert_gemm(q, s, one, 64, 32, i32), lambda: tf.w8a8_expert_gemm(q, s, packed, 64, 32, i32.long()),
                 lambda: tf.w8a8_expert_gemm(q, s, packed, 64, 32, i32[:1]),
                 lambda: tf.w8a8_expert_gemm(q, s, packed, 64, 32, i32, r.tokens.long()),
                 lambda: tf.route_experts(x[0], 1), lambda: tf.route_experts(x.double(), 1), lambda: tf.route_experts(x, 1, bias=s.half()),
                 lambda: tf.route_experts(x, 1, scoring="max"), lambda: tf.route_experts(x, 1, group_score="sum"),
                 lambda: tf.combine_experts(e, torch.ones(6, 2, device="cuda"), r.places),
                 lambda: tf.combine_experts(e.float(), torch.ones(6, 1, device="cuda"), r.places),
                 lambda: tf.combine_experts(e, torch.ones(6, 1, device="cuda"), r.places, add=e[:3]),
                 lambda: tf.pack_w8a8(w.short(), ws), lambda: tf.pack_w8a8(w, ws[0]), lambda: tf.pack_w8a8(w, ws, out=one)):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: tf.quantize_rows(x[:, :24]), tf.TF_ERR_SHAPE), (lambda: tf.route_experts(x, 65), tf.TF_ERR_SHAPE),
                         (lambda: tf.quantize_rows(x[:, 1:33]), tf.TF_ERR_ALIGN), (lambda: tf.route_experts(x, 0), tf.TF_ERR_SHAPE),
                         (lambda: tf.route_experts(x, 2, groups=3), tf.TF_ERR_SHAPE), (lambda: tf.route_experts(x, 2, scale=0.0), tf.TF_ERR_ARG),
                         (lambda: tf.w8a8_gemm(q[:, :40].contiguous(), s, one, 40, 32), tf.TF_ERR_SHAPE)):
        with pytest.raises(tf.TileFuseError) as err:
            call()
        assert err.value.status == status


def test_inputs_with_gradients_are_read(tf, path):
    """Inference calls take tensors that record gradients and return ones that do not."""
    x = torch.randn(4, 64, device="cuda").half().requires_grad_()
    q, s = tf.quantize_rows(x)
    r = tf.route_experts(x, 3)
    assert not q.requires_grad and not s.requires_grad and not r.weights.requires_grad
    with torch.inference_mode():
        assert torch.equal(tf.quantize_rows(x.detach())[0], q)


@pytest.mark.parametrize("args", [["--eight-bit"], ["--experts", "8"], ["--eight-bit", "--experts", "16", "--top-k", "3"]], ids=str)
def test_command_runs(dec, capsys, args):
    dec.main(["--layers", "1", "--prompt", "100", "--batch", "2", "--steps", "3", *args])
    assert "us a step" in capsys.readouterr().out
