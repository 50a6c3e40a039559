"""Threads that share the default stream, and with it the cached workspaces: every
output has the bits of the same call alone."""
from __future__ import annotations

import threading

import pytest

from test_gpu_experts import tf  # noqa: F401
from test_workspaces import chunk_case, decode_case, matmul_case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def w8a8_case(tf, M, K, N):
    torch.manual_seed(M)
    q = torch.randint(-128, 128, (M, K), device="cuda").to(torch.int8)
    s = torch.rand(M, device="cuda") * 1e-5
    packed = tf.pack_w8a8(torch.randint(-128, 128, (K, N), device="cuda").to(torch.int8), torch.rand(N, device="cuda"))
    assert tf.w8a8_workspace_bytes(M, K, N) > 0
    return lambda: tf.w8a8_gemm(q, s, packed, K, N)


CASES = {"w8a8": lambda tf: [w8a8_case(tf, 64, 14336, 1024), w8a8_case(tf, 100, 14336, 520), w8a8_case(tf, 17, 14336, 4096)],
         "matmul": lambda tf: [matmul_case(100, 14336, 2048, "gemm"), matmul_case(40, 8192, 1024, "gemm"), matmul_case(1, 14336, 4096, "gemv")],
         "prompt": lambda tf: [chunk_case(200, 3000), chunk_case(500, 7000)],
         "decode": lambda tf: [decode_case([9000, 50], 1), decode_case([70000], 8)]}


@pytest.mark.parametrize("kind", CASES)
def test_threads_on_one_stream(tf, kind):
    calls = CASES[kind](tf)
    want = [call() for call in calls]
    torch.cuda.synchronize()
    got, errors, go = [[] for _ in calls], [], threading.Barrier(len(calls))

    def work(i):
        try:
            go.wait(30)
            for _ in range(40):
                got[i].append(calls[i]())
        except Exception as e:   # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    torch.cuda.synchronize()
    assert not errors and all(len(g) == 40 for g in got)
    assert all(torch.equal(t, want[i]) for i, g in enumerate(got) for t in g)
