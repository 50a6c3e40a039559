"""Cached workspaces of the binding: each stream has its own, a captured graph's
are the graph's, and no call takes away what another may still use."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from paper_2606_11357_amd import tilefuse as tf  # noqa: E402


class Caller:
    """A caller's device, stream and capture, as the binding is told them."""

    def __init__(self, monkeypatch):
        self.at = (0, 7, 0)
        monkeypatch.setattr(tf, "_place", lambda device: self.at, raising=False)

    def __call__(self, make, nbytes, stream, capture=0):
        self.at = (0, stream, capture)
        return make(nbytes)


def decode_ws(cache):
    return lambda n: tf._cached_workspace(cache, torch.device("cpu", 0), n)


def check_cached(caller, make, cache):
    a = caller(make, 20000, 7)
    assert caller(make, 100, 7) is a and (a == 0).all()
    b = caller(make, 20000, 8)                    # another stream: another buffer
    assert b is not a
    assert caller(make, 20000, 7) is a and caller(make, 20000, 8) is b
    # a capture takes neither, and an eager call that needs more leaves its buffer alone
    c = caller(make, 20000, 7, capture=3)
    assert c is not a and c is not b
    assert (c[:8192] == 0).all()
    assert caller(make, 20000, 7) is a
    d = caller(make, 3 << 20, 7)
    assert d.numel() >= 3 << 20 and (d == 0).all()
    assert caller(make, 20000, 7, capture=3) is c
    # the first call of all under capture leaves none behind for eager calls
    e = caller(make, 20000, 9, capture=3)
    f = caller(make, 20000, 9)
    assert e is not f and (f == 0).all()
    # the next capture has its own; the last one's are given back to their graph
    g = caller(make, 20000, 7, capture=4)
    assert g is not c and all(h is not c for h in cache.values())
    assert caller(make, 20000, 7) is d and caller(make, 20000, 9) is f


def test_attention_workspaces(monkeypatch):
    cache = {}
    check_cached(Caller(monkeypatch), decode_ws(cache), cache)


def test_matmul_workspaces(monkeypatch):
    monkeypatch.setattr(tf, "_default_ws", {})
    check_cached(Caller(monkeypatch), lambda n: tf.default_workspace(torch.device("cpu", 0), n), tf._default_ws)


# ---------------------------------------------------------------------------
# on the GPU
# ---------------------------------------------------------------------------
def i32(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def decode_case(lens, new):
    """Long sequences of one head of 256, whose parts go through the workspace."""
    torch.manual_seed(3)
    per = -(-max(lens) // 64)
    cache = tf.kv4_cache(len(lens) * per, 64, 1, 256, dtype=torch.bfloat16)
    table = torch.randperm(len(lens) * per, device="cuda").to(torch.int32).view(len(lens), per)
    kv = torch.randn(sum(lens), 1, 256, device="cuda").bfloat16()
    cu = torch.cat([i32(0), i32(*lens).cumsum(0).to(torch.int32)])
    tf.kv4_append(cache, table, cu, i32(*[0] * len(lens)), kv, kv)
    q = torch.randn(len(lens), new, 8, 256, device="cuda").bfloat16()
    n = i32(*lens)
    return lambda: tf.kv4_attention(q, cache, table, n)


def chunk_case(n, past):
    """Few queries on many keys, whose parts go through the workspace."""
    torch.manual_seed(4)
    q, k = torch.randn(n, 16, 128, device="cuda").bfloat16(), torch.randn(n + past, 2, 128, device="cuda").bfloat16()
    cu, ck = i32(0, n), i32(0, n + past)
    return lambda: tf.prompt_attention(q, k, k, cu, ck)


def matmul_case(M, K, N, kind):
    """A matmul whose K is split over workgroups."""
    torch.manual_seed(5)
    word = lambda *shape: torch.randint(-2 ** 31, 2 ** 31, shape, dtype=torch.int32, device="cuda")  # noqa: E731
    s = (0.01 * torch.rand((K // 128, N), device="cuda")).half()
    packed = tf.pack_w4(word(K, N // 8), word(K // 128, N // 8), s, K, N)
    x = torch.randn(M, K, device="cuda").half()
    assert tf.workspace_bytes(4, M, K, N) > 0
    return lambda: getattr(tf, f"w4a16_{kind}")(x, packed, K, N)


def captured(call):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    return g, out


@pytest.mark.gpu
def test_captures_are_told_apart():
    at = lambda: tf._capture_of(torch.cuda.current_stream().cuda_stream)  # noqa: E731
    x = torch.zeros(8, device="cuda")
    assert at() == 0
    with torch.cuda.stream(torch.cuda.Stream()):
        assert at() == 0
    seen, graphs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.add_(1)
            seen.append(at())
            x.add_(1)
            assert at() == seen[-1]
        graphs.append(g)
    assert 0 < seen[0] != seen[1] > 0 and at() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("small,large", [(lambda: decode_case([9000, 50], 1), lambda: decode_case([9000, 50], 4)),
                                         (lambda: chunk_case(200, 3000), lambda: chunk_case(500, 7000)),
                                         (lambda: matmul_case(1, 14336, 4096, "gemv"),
                                          lambda: matmul_case(200, 12288, 4096, "gemm"))],
                         ids=["decode", "prompt", "matmul"])
def test_graph_on_the_default_workspace(small, large):
    """Captured, then a call that needs more and tensors of every size, then replays:
    each as the eager call, with eager calls in between, and no tensor touched."""
    small, large = small(), large()
    want = small()
    torch.cuda.synchronize()
    g, out = captured(small)
    large()
    torch.cuda.synchronize()
    others = [torch.full((1 << n,), 0x5A, dtype=torch.uint8, device="cuda") for n in range(9, 26) for _ in range(3)]
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(small(), want)
    assert all(bool((t == 0x5A).all()) for t in others)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [lambda: decode_case([9000, 50], 1), lambda: matmul_case(1, 14336, 4096, "gemv")],
                         ids=["decode", "matmul"])
def test_first_call_on_a_stream_is_a_captured_one(case):
    """Eager calls on the stream of a capture, before any replay of its graph."""
    call = case()
    want = call()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        out = call()
    with torch.cuda.stream(s):
        first = call()
    s.synchronize()
    assert torch.equal(first, want)
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_streams_side_by_side():
    """The default workspace on two streams at once."""
    a, b = decode_case([9000, 50], 1), decode_case([7000, 5000], 1)
    c, d = matmul_case(1, 14336, 4096, "gemv"), matmul_case(2, 14336, 4096, "gemv")
    calls = a, b, c, d
    want = [f() for f in calls]
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(20):
        for i, f in enumerate(calls):
            with torch.cuda.stream(streams[i % 2]):
                got.append(f())
    torch.cuda.synchronize()
    for i, t in enumerate(got):
        assert torch.equal(t, want[i % 4])
