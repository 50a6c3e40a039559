"""C-ABI checks of the 8-bit linear layers and the layers made of experts that need
no GPU: sizes, and refusals made before any HIP call; refusals of the binding."""
from __future__ import annotations

import ctypes

import pytest

from paper_2606_11357_amd import tilefuse as tfb

P = ctypes.c_void_p(0x10000)          # never dereferenced: validation fails first
P_16 = ctypes.c_void_p(0x10010)
P_8 = ctypes.c_void_p(0x10008)
P_2 = ctypes.c_void_p(0x10002)
P_1 = ctypes.c_void_p(0x10001)
NULL = None
NONE, SHAPE, ARG, ALIGN = tfb.TF_ERR_NULL, tfb.TF_ERR_SHAPE, tfb.TF_ERR_ARG, tfb.TF_ERR_ALIGN


@pytest.fixture(scope="module")
def lib():
    return tfb.load()


@pytest.mark.parametrize("K,N,want", [
    (16, 8, 2 * 1024 + 256), (128, 16, 2 * 1024 + 256), (144, 24, 2 * 4 * 1024 + 256), (4096, 4096, 4096 * 4096 + 16384),
    (65536, 65536, 65536 * 65536 + 262144), (0, 8, SHAPE), (24, 8, SHAPE), (16, 12, SHAPE), (65552, 8, SHAPE),
    (16, 65544, SHAPE), (-16, 8, SHAPE)])
def test_packed_bytes(lib, K, N, want):
    assert lib.tf_w8a8_packed_bytes(K, N) == want


QUANT = dict(dtype=1, X=P, stride=64, M=4, N=64, gated=0, codes=P, scales=P)


@pytest.mark.parametrize("kw,want", [
    (dict(X=NULL), NONE), (dict(codes=NULL), NONE), (dict(scales=NULL), NONE), (dict(dtype=2), ARG), (dict(M=0), SHAPE),
    (dict(N=0), SHAPE), (dict(N=56), SHAPE), (dict(N=65552, stride=65552), SHAPE), (dict(stride=56), SHAPE),
    (dict(stride=68), SHAPE), (dict(gated=1), SHAPE), (dict(M=1 << 22, N=65536, stride=65536), SHAPE),
    (dict(X=P_8), ALIGN), (dict(codes=P_8), ALIGN), (dict(scales=P_2), ALIGN)], ids=str)
def test_quantize_rejects(lib, kw, want):
    assert lib.tf_quantize_rows(*(QUANT | kw).values(), NULL) == want


PACK = dict(w=P, scales=P, dtype=1, K=64, N=64, experts=2, packed=P)


@pytest.mark.parametrize("kw,want", [
    (dict(w=NULL), NONE), (dict(scales=NULL), NONE), (dict(packed=NULL), NONE), (dict(dtype=0), ARG), (dict(dtype=4), ARG),
    (dict(K=8), SHAPE), (dict(N=4), SHAPE), (dict(experts=0), SHAPE), (dict(experts=1025), SHAPE), (dict(packed=P_16), ALIGN),
    (dict(w=P_8), ALIGN)], ids=str)
def test_pack_rejects(lib, kw, want):
    assert lib.tf_pack_w8a8(*(PACK | kw).values(), NULL) == want


GEMM = dict(dtype=1, A=P, scales=P, packed=P, C=P, M=4, K=64, N=64, ws=NULL, ws_bytes=0)


@pytest.mark.parametrize("kw,want", [
    (dict(A=NULL), NONE), (dict(scales=NULL), NONE), (dict(packed=NULL), NONE), (dict(C=NULL), NONE), (dict(dtype=2), ARG),
    (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(K=72), SHAPE), (dict(N=68), SHAPE), (dict(A=P_8), ALIGN),
    (dict(C=P_8), ALIGN), (dict(packed=P_16), ALIGN), (dict(scales=P_2), ALIGN), (dict(ws=P_8, ws_bytes=1 << 30), ALIGN),
    (dict(M=64, K=14336, N=4096, ws=P, ws_bytes=64), ARG)], ids=str)
def test_gemm_rejects(lib, kw, want):
    assert lib.tf_w8a8_gemm(*(GEMM | kw).values(), NULL) == want


@pytest.mark.parametrize("M,K,N,want", [
    (64, 14336, 4096, 4 * 64 * 4096 * 4), (1, 14336, 4096, 0), (64, 4096, 4096, 0), (2048, 14336, 4096, 0),
    (0, 64, 64, SHAPE), (1, 24, 64, SHAPE), (1, 64, 4, SHAPE), ((1 << 20) + 1, 64, 64, SHAPE)])
def test_gemm_workspace(lib, M, K, N, want):
    assert lib.tf_w8a8_workspace_bytes(M, K, N) == want


ROUTE = dict(dtype=1, logits=P, stride=8, bias=NULL, T=4, experts=8, top_k=2, scoring=0, groups=1, top_groups=1,
             group_score=1, renormalize=0, scale=1.0, weights=P, chosen=P, offsets=P, tokens=P, places=P)


@pytest.mark.parametrize("kw,want", [
    *((dict([(n, NULL)]), NONE) for n in ("logits", "weights", "chosen", "offsets", "tokens", "places")),
    (dict(dtype=0), ARG), (dict(scoring=2), ARG), (dict(group_score=-1), ARG), (dict(scale=0.0), ARG),
    (dict(scale=float("nan")), ARG), (dict(T=0), SHAPE), (dict(experts=0, stride=0), SHAPE),
    (dict(experts=1025, stride=1025), SHAPE), (dict(stride=7), SHAPE), (dict(groups=3), SHAPE), (dict(groups=0), SHAPE),
    (dict(groups=2, top_groups=3), SHAPE), (dict(groups=2, top_groups=0), SHAPE), (dict(top_k=0), SHAPE),
    (dict(top_k=9), SHAPE), (dict(groups=4, top_groups=1, top_k=3), SHAPE), (dict(experts=128, stride=128, groups=128), SHAPE),
    (dict(experts=64, stride=64, top_k=33), SHAPE), (dict(logits=P_1), ALIGN), (dict(dtype=2, logits=P_2), ALIGN),
    (dict(bias=P_2), ALIGN), (dict(places=P_2), ALIGN)], ids=str)
def test_route_rejects(lib, kw, want):
    assert lib.tf_route_experts(*(ROUTE | kw).values(), NULL) == want


EXPERTS = dict(dtype=1, A=P, scales=P, a_rows=4, packed=P, offsets=P, rows=P, C=P, slots=8, K=64, N=64, experts=2)


@pytest.mark.parametrize("kw,want", [
    *((dict([(n, NULL)]), NONE) for n in ("A", "scales", "packed", "offsets", "C")), (dict(dtype=2), ARG),
    (dict(a_rows=0), SHAPE), (dict(slots=0), SHAPE), (dict(slots=(1 << 25) + 1), SHAPE), (dict(K=40), SHAPE),
    (dict(N=4), SHAPE), (dict(experts=0), SHAPE), (dict(experts=1025), SHAPE), (dict(a_rows=1 << 20, K=4096), SHAPE),
    (dict(offsets=P_2), ALIGN), (dict(rows=P_2), ALIGN), (dict(A=P_8), ALIGN)], ids=str)
def test_expert_gemm_rejects(lib, kw, want):
    assert lib.tf_w8a8_expert_gemm(*(EXPERTS | kw).values(), NULL) == want


COMBINE = dict(dtype=1, Y=P, slots=8, weights=P, places=P, add=NULL, T=4, top_k=2, N=64, out=P)


@pytest.mark.parametrize("kw,want", [
    *((dict([(n, NULL)]), NONE) for n in ("Y", "weights", "places", "out")), (dict(dtype=2), ARG), (dict(T=0), SHAPE),
    (dict(slots=0), SHAPE), (dict(top_k=0), SHAPE), (dict(top_k=33), SHAPE), (dict(N=4), SHAPE), (dict(N=65544), SHAPE),
    (dict(T=1 << 20, N=65536), SHAPE), (dict(add=P_8), ALIGN), (dict(Y=P_8), ALIGN), (dict(weights=P_2), ALIGN)], ids=str)
def test_combine_rejects(lib, kw, want):
    assert lib.tf_combine_experts(*(COMBINE | kw).values(), NULL) == want


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    x, q, s = torch.zeros(2, 64).half(), torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    i = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: tfb.quantize_rows(x), lambda: tfb.pack_w8a8(q, s), lambda: tfb.w8a8_gemm(q, s, q, 64, 64),
                 lambda: tfb.route_experts(x, 2), lambda: tfb.w8a8_expert_gemm(q, s, q, 64, 64, i),
                 lambda: tfb.combine_experts(x, s[:, None], i[:2, None])):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
