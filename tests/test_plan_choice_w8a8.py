"""Which form an 8-bit product takes, read from the plan log (CPU only), in a child
process that sees no GPU, as in test_plan_choice.py: that the tests named for a form
run it, and that they leave none out."""
from __future__ import annotations

import json
import os
import subprocess
import sys

import pytest

from test_plan_choice import ROOT, _skip_with_gpu

torch = pytest.importorskip("torch")

CHILD = r"""
import ctypes, json, sys
hip = ctypes.CDLL("libamdhip64.so")
n = ctypes.c_int(0)
if hip.hipGetDeviceCount(ctypes.byref(n)) == 0 and n.value > 0:
    sys.exit("a GPU is visible: the calls below must not reach one")
from paper_2606_11357_amd import tilefuse as tf
lib = tf.load()
P = ctypes.c_void_p(0x10000)
for dtype, experts, M, K, N, rows in json.load(sys.stdin):
    print("call", file=sys.stderr, flush=True)
    if experts:
        rc = lib.tf_w8a8_expert_gemm(dtype, P, P, 1, P, P, P if rows else None, P, M, K, N, experts, None)
    else:
        rc = lib.tf_w8a8_gemm(dtype, P, P, P, P, M, K, N, P if rows else None, 1 << 40, None)
    assert rc == tf.TF_ERR_HIP
"""


def plans(calls):
    """The plan of each (dtype, experts or 0, rows of C, K, N, gathered or with a workspace) call."""
    env = dict(os.environ, TF_LOG="1", HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1",
               LD_LIBRARY_PATH=os.pathsep.join([os.path.join(os.path.dirname(torch.__file__), "lib"),
                                                "/opt/rocm/lib", os.environ.get("LD_LIBRARY_PATH", "")]))
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=env, input=json.dumps(calls), text=True,
                       capture_output=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    got = [part.split("[tilefuse] ")[1].splitlines()[0] for part in r.stderr.split("call\n")[1:]]
    assert len(got) == len(calls)
    return got


FORMS = ["16 x 16", "64 x 64", "64 x 128", "128 x 128", "128 x 256", "256 x 256"]


def many(form, rows, N):
    """More tiles than workgroups run at a time (rows of experts have as many at least)."""
    bm, bn = (int(v) for v in form.split(" x "))
    return -(-rows // bm) * -(-N // bn) > 256 * (2 if bm == 64 else 1)


def test_forms_of_the_gpu_tests():
    _skip_with_gpu()
    import test_gpu_w8a8_forms as t
    calls = [(dt, 0, M, K, N, False) for _, M, K, N in t.DENSE for dt in (1, 3)]
    forms = [form for form, *_ in t.DENSE for _ in range(2)]
    calls += [(dt, E, S, K, N, rows) for _, E, S, K, N in t.EXPERTS + t.PAST for dt in (1, 3) for rows in (False, True)]
    forms += [form for form, *_ in t.EXPERTS + t.PAST for _ in range(4)]
    for c, form, line in zip(calls, forms, plans(calls)):
        kernel = "w8a8_direct_kernel" if form == t.DIRECT else "w8a8_tile_kernel"
        assert f": {kernel}, {form} tiles, K in 1," in line, (c, line)
        assert (" gathered" in line) == bool(c[1] and c[5]), line
    for cases in ([(f, M, N) for f, M, _, N in t.DENSE], [(f, S - 5, N) for f, _, S, _, N in t.EXPERTS]):
        assert {f for f, *_ in cases} == set(FORMS)
        assert {f for f, rows, N in cases if f != t.DIRECT and many(f, rows, N)} == set(FORMS) - {t.DIRECT}
    assert all(K % 128 and K > 64 * 8 for _, _, K, _ in t.DENSE if K > 208)


def test_split_over_k():
    """The sizes of the test of products with K split run split, with a workspace alone."""
    _skip_with_gpu()
    for M, K, N, parts in ((17, 14336, 4096, 4), (49, 14336, 1032, 4), (64, 8208, 264, 4), (70, 14336, 4096, 2),
                           (128, 16384, 520, 4)):
        with_ws, without = plans([(1, 0, M, K, N, True), (1, 0, M, K, N, False)])
        assert f"64 x 64 tiles, K in {parts}," in with_ws and "K in 1," in without
