"""Calls of several threads that share a stream and its workspace (CPU only): a call of
several launches hands parts from one to the next through the workspace, so no other
call's launch may come between them.

The calls run in a child process whose launches go to a stand-in that notes which
thread made each, after a pause that lets the other thread come first if it can."""
from __future__ import annotations

import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_IN = r"""
#include <atomic>
#include <unistd.h>
static std::atomic<int> n;
static long who[4096];
static thread_local long me;
extern "C" void i_am(long id) { me = id; }
extern "C" int made(long* out) {
    const int k = n.exchange(0);
    for (int i = 0; i < k; ++i) out[i] = who[i];
    return k;
}
extern "C" int hipLaunchKernel(const void*) {
    usleep(3000);
    const int i = n++;
    if (i < 4096) who[i] = me;
    return 0;
}
"""

CHILD = r"""
import ctypes, json, sys, threading
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # before the library's own
from paper_2606_11357_amd import tilefuse as tf
lib = tf.load()
P, WS, BIG = ctypes.c_void_p(0x10000), [ctypes.c_void_p(0x20000), ctypes.c_void_p(0x30000)], 1 << 40
def matmul(kind, bits, M, K, N):
    f = getattr(lib, f"tf_w{bits}a16_{kind}")
    return lambda ws: f(P, P, P, M, K, N, 128, ws, BIG, None)
def w8a8(M, K, N):
    return lambda ws: lib.tf_w8a8_gemm(1, P, P, P, P, M, K, N, ws, BIG, None)
def prompt(n, past):
    return lambda ws: lib.tf_prompt_attention(1, P, 2048, P, 256, P, 256, P, P, 1, n, n + past, 16, 2, 128, 0.1, 1, P, ws, BIG, None)
def decode(q_len):
    cache = tf._Kv4Struct(0x10000, 1024, 64, 1, 256, 1, 0x10000, 1024, 1024)
    return lambda ws: lib.tf_kv4_attention(ctypes.byref(cache), P, 8 * 256, P, 1, q_len, 8, 0.1, P, ws, BIG, None)
makers = dict(matmul=matmul, w8a8=w8a8, prompt=prompt, decode=decode)
out = (ctypes.c_long * 4096)()
def launches():
    return list(out[:stand_in.made(out)])
got = []
for pair, same in json.load(sys.stdin):
    calls = [makers[name](*args) for name, *args in pair]
    alone = []
    for i, call in enumerate(calls):
        assert call(WS[0]) == 0, pair[i]
        alone.append(len(launches()))
    go = threading.Barrier(2)
    def work(i):
        stand_in.i_am(i + 1)
        go.wait()
        for _ in range(6):
            assert calls[i](WS[0 if same else i]) == 0
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads], [t.join() for t in threads]
    got.append((alone, launches()))
json.dump(got, sys.stdout)
"""

# two launches a call: the product of codes with K split, the tiles of a matmul with K
# split, stream-K, prompts and decode steps whose keys are split; one: a decode matmul
SPLIT = ["w8a8", 64, 14336, 4096]
TILES, STREAM_K = ["matmul", "gemm", 4, 100, 14336, 2048], ["matmul", "gemm", 4, 2048, 14336, 4096]
ONE = ["matmul", "gemv", 4, 1, 14336, 4096]
PROMPT, DECODE = ["prompt", 200, 3000], ["decode", 8]


@pytest.fixture(scope="module")
def order(tmp_path_factory):
    import torch
    d = tmp_path_factory.mktemp("turns")
    src, lib = d / "stand_in.cpp", d / "stand_in.so"
    src.write_text(STAND_IN)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", str(lib), str(src)], check=True)
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1",
               LD_LIBRARY_PATH=os.pathsep.join([os.path.join(os.path.dirname(torch.__file__), "lib"),
                                                "/opt/rocm/lib", os.environ.get("LD_LIBRARY_PATH", "")]))

    def run(*pairs):
        r = subprocess.run([sys.executable, "-c", CHILD, str(lib)], cwd=ROOT, env=env, input=json.dumps(pairs), text=True,
                           capture_output=True, timeout=120)
        assert r.returncode == 0, r.stderr[-3000:]
        return json.loads(r.stdout)
    return run


@pytest.mark.parametrize("a,b", [(SPLIT, SPLIT), (SPLIT, ["w8a8", 100, 14336, 1032]), (TILES, TILES), (TILES, ONE),
                                 (STREAM_K, TILES), (STREAM_K, ONE), (PROMPT, PROMPT), (DECODE, DECODE)], ids=str)
def test_calls_take_turns(order, a, b):
    (alone, made), = order(([a, b], True))
    assert alone[0] == 2 and alone[1] == (1 if b is ONE else 2)
    assert sorted(made) == [1] * (6 * alone[0]) + [2] * (6 * alone[1])
    at = 0
    while at < len(made):
        n = alone[made[at] - 1]
        assert made[at:at + n] == [made[at]] * n, made
        at += n


def test_other_workspaces_do_not_wait(order):
    """Calls on workspaces of their own go on side by side."""
    (alone, made), = order(([SPLIT, SPLIT], False))
    assert sorted(made) == [1] * 12 + [2] * 12
    assert any(made[i] != made[i + 1] for i in range(0, len(made), 2)), made
