"""C-ABI checks of the operators around the linear layers that need no GPU:
sizes, and refusals made before any HIP call."""
from __future__ import annotations

import ctypes

import pytest

from paper_2606_11357_amd import tilefuse as tfb

P = ctypes.c_void_p(0x10000)          # never dereferenced: validation fails first
P_ODD = ctypes.c_void_p(0x10008)
P_2 = ctypes.c_void_p(0x10002)
NULL = None


@pytest.fixture(scope="module")
def lib():
    return tfb.load()


NORM = dict(dtype=1, X=P, residual=P, post=NULL, gate=NULL, gate_stride=0, scale=1.0, weight=P, offset=0.0, eps=1e-5,
            M=4, N=64, r_out=P, Y=P)


@pytest.mark.parametrize("kw,want", [
    (dict(X=NULL), tfb.TF_ERR_NULL), (dict(r_out=NULL, Y=NULL), tfb.TF_ERR_NULL), (dict(weight=NULL), tfb.TF_ERR_NULL),
    (dict(dtype=2), tfb.TF_ERR_ARG), (dict(eps=-1.0), tfb.TF_ERR_ARG), (dict(eps=float("nan")), tfb.TF_ERR_ARG),
    (dict(M=0), tfb.TF_ERR_SHAPE), (dict(N=60), tfb.TF_ERR_SHAPE), (dict(N=65544), tfb.TF_ERR_SHAPE),
    (dict(gate=P, gate_stride=32), tfb.TF_ERR_SHAPE), (dict(gate=P, gate_stride=68), tfb.TF_ERR_SHAPE),
    (dict(Y=P_ODD), tfb.TF_ERR_ALIGN), (dict(gate=P_ODD), tfb.TF_ERR_ALIGN)], ids=str)
def test_norm_rejects(lib, kw, want):
    assert lib.tf_add_rms_norm(*(NORM | kw).values(), NULL) == want


@pytest.mark.parametrize("args,want", [
    ((1, 32, 1, 64), 32 * (32 + 32) + 256), ((10, 64, 8, 128), 10 * 8 * 2 * (32 * 128 + 256)),
    ((3, 96, 2, 256), 3 * 2 * 3 * (32 * 256 + 256)),
    ((1 << 20, 256, 8, 128), (1 << 20) * 8 * 8 * (32 * 128 + 256)),          # beyond 32 bits
    ((0, 32, 1, 64), tfb.TF_ERR_SHAPE), ((1, 48, 1, 64), tfb.TF_ERR_SHAPE), ((1, 0, 1, 64), tfb.TF_ERR_SHAPE),
    ((1, 32, 0, 64), tfb.TF_ERR_SHAPE), ((1, 32, 1, 96), tfb.TF_ERR_SHAPE)])
def test_cache_bytes(lib, args, want):
    assert lib.tf_kv4_cache_bytes(*args) == want


def cache(**kw):
    d = dict(data=0x10000, pages=8, page_size=64, kv_heads=2, head_dim=128, dtype=1, table=0x10000, table_stride=4,
             max_pages=4) | kw
    return tfb._Kv4Struct(*d.values())


BAD_CACHE = [(dict(data=0), tfb.TF_ERR_NULL), (dict(table=0), tfb.TF_ERR_NULL), (dict(dtype=2), tfb.TF_ERR_ARG),
             (dict(pages=0), tfb.TF_ERR_SHAPE), (dict(page_size=40), tfb.TF_ERR_SHAPE),
             (dict(kv_heads=0), tfb.TF_ERR_SHAPE), (dict(head_dim=80), tfb.TF_ERR_SHAPE),
             (dict(max_pages=0), tfb.TF_ERR_SHAPE), (dict(table_stride=3), tfb.TF_ERR_SHAPE),
             (dict(max_pages=1 << 26, table_stride=1 << 26), tfb.TF_ERR_SHAPE),      # positions beyond 31 bits
             (dict(data=0x10010), tfb.TF_ERR_ALIGN), (dict(table=0x10002), tfb.TF_ERR_ALIGN)]
APPEND = dict(Q=P, q_stride=1024, K=P, k_stride=256, V=P, v_stride=256, cos=P, sin=P, positions=9, cu=P, starts=P,
              batch=2, tokens=5, q_heads=8, Q_out=P, K_out=NULL)
READ = dict(cu=P, starts=P, batch=2, tokens=5, K_out=P, V_out=P)
DECODE = dict(Q=P, q_stride=1024, lens=P, batch=2, q_len=1, q_heads=8, scale=0.1, O=P, ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("kw,want", BAD_CACHE, ids=str)
def test_cache_rejects(lib, kw, want):
    c = cache(**kw)
    assert lib.tf_kv4_append(c, *APPEND.values(), NULL) == want
    assert lib.tf_kv4_read(c, *READ.values(), NULL) == want
    assert lib.tf_kv4_attention(c, *DECODE.values(), NULL) == want


@pytest.mark.parametrize("kw,want", [
    (dict(K=NULL), tfb.TF_ERR_NULL), (dict(V=NULL), tfb.TF_ERR_NULL), (dict(cu=NULL), tfb.TF_ERR_NULL),
    (dict(starts=NULL), tfb.TF_ERR_NULL), (dict(cos=NULL), tfb.TF_ERR_NULL), (dict(Q_out=NULL), tfb.TF_ERR_NULL),
    (dict(batch=0), tfb.TF_ERR_SHAPE), (dict(batch=65537), tfb.TF_ERR_SHAPE), (dict(tokens=0), tfb.TF_ERR_SHAPE),
    (dict(q_heads=0), tfb.TF_ERR_SHAPE), (dict(Q=NULL, Q_out=NULL), tfb.TF_ERR_SHAPE),
    (dict(k_stride=248), tfb.TF_ERR_SHAPE), (dict(v_stride=260), tfb.TF_ERR_SHAPE),
    (dict(positions=0), tfb.TF_ERR_SHAPE), (dict(K=P_ODD), tfb.TF_ERR_ALIGN), (dict(K_out=P_ODD), tfb.TF_ERR_ALIGN),
    (dict(cu=P_2), tfb.TF_ERR_ALIGN)], ids=str)
def test_append_rejects(lib, kw, want):
    assert lib.tf_kv4_append(cache(), *(APPEND | kw).values(), NULL) == want


@pytest.mark.parametrize("kw,want", [
    (dict(cu=NULL), tfb.TF_ERR_NULL), (dict(K_out=NULL), tfb.TF_ERR_NULL), (dict(tokens=0), tfb.TF_ERR_SHAPE),
    (dict(V_out=P_ODD), tfb.TF_ERR_ALIGN), (dict(starts=P_2), tfb.TF_ERR_ALIGN)], ids=str)
def test_read_rejects(lib, kw, want):
    assert lib.tf_kv4_read(cache(), *(READ | kw).values(), NULL) == want


@pytest.mark.parametrize("kw,want", [
    (dict(Q=NULL), tfb.TF_ERR_NULL), (dict(lens=NULL), tfb.TF_ERR_NULL), (dict(ws=NULL), tfb.TF_ERR_NULL),
    (dict(q_len=0), tfb.TF_ERR_ARG), (dict(q_len=9), tfb.TF_ERR_ARG), (dict(q_heads=7), tfb.TF_ERR_SHAPE),
    (dict(q_stride=1016), tfb.TF_ERR_SHAPE), (dict(scale=0.0), tfb.TF_ERR_ARG), (dict(scale=float("nan")), tfb.TF_ERR_ARG),
    (dict(ws_bytes=64), tfb.TF_ERR_ARG), (dict(O=P_ODD), tfb.TF_ERR_ALIGN), (dict(ws=P_ODD), tfb.TF_ERR_ALIGN),
    (dict(lens=P_2), tfb.TF_ERR_ALIGN)], ids=str)
def test_decode_rejects(lib, kw, want):
    assert lib.tf_kv4_attention(cache(), *(DECODE | kw).values(), NULL) == want


def test_decode_rejects_more_pieces_than_32_bits_count(lib):
    c = cache(max_pages=1 << 20, table_stride=1 << 20)
    assert lib.tf_kv4_attention(c, *(DECODE | dict(batch=65536)).values(), NULL) == tfb.TF_ERR_SHAPE


PROMPT = dict(dtype=3, Q=P, q_stride=1024, K=P, k_stride=256, V=P, v_stride=256, cu_q=P, cu_k=P, batch=2, tokens_q=9,
              tokens_k=9, q_heads=8, kv_heads=2, head_dim=128, scale=0.1, causal=1, O=P, ws=NULL, ws_bytes=0)


@pytest.mark.parametrize("kw,want", [
    (dict(Q=NULL), tfb.TF_ERR_NULL), (dict(cu_k=NULL), tfb.TF_ERR_NULL), (dict(O=NULL), tfb.TF_ERR_NULL),
    (dict(dtype=2), tfb.TF_ERR_ARG), (dict(scale=-1.0), tfb.TF_ERR_ARG), (dict(head_dim=32), tfb.TF_ERR_SHAPE),
    (dict(q_heads=9), tfb.TF_ERR_SHAPE), (dict(batch=0), tfb.TF_ERR_SHAPE), (dict(tokens_k=0), tfb.TF_ERR_SHAPE),
    (dict(tokens_q=(1 << 20) + 1), tfb.TF_ERR_SHAPE), (dict(k_stride=128), tfb.TF_ERR_SHAPE),
    (dict(V=P_ODD), tfb.TF_ERR_ALIGN), (dict(ws=P_ODD), tfb.TF_ERR_ALIGN),
    (dict(tokens_k=9000, batch=1, ws=P, ws_bytes=64), tfb.TF_ERR_ARG)], ids=str)
def test_prompt_rejects(lib, kw, want):
    assert lib.tf_prompt_attention(*(PROMPT | kw).values(), NULL) == want


def test_calls_of_more_threads_than_a_launch_has(lib):
    """Sizes that each pass their own limit and together ask for 2^32 threads."""
    big = dict(tokens=1 << 20)
    c = cache(kv_heads=1024, head_dim=256)
    wide = dict(q_stride=1024 * 256, k_stride=1024 * 256, v_stride=1024 * 256, q_heads=1024)
    assert lib.tf_kv4_append(c, *(APPEND | wide | big).values(), NULL) == tfb.TF_ERR_SHAPE
    assert lib.tf_kv4_read(c, *(READ | big).values(), NULL) == tfb.TF_ERR_SHAPE
    assert lib.tf_prompt_attention(*(PROMPT | wide | dict(tokens_q=1 << 20, batch=65536, kv_heads=1024, head_dim=256)).values(),
                                   NULL) == tfb.TF_ERR_SHAPE
    assert lib.tf_prompt_attention_workspace_bytes(1, 1 << 20, 1 << 20, 1024, 1, 128) == 0      # 2^31: fits


def test_workspace_queries(lib):
    """Decode: at least what one call's parts and counters take, the same region
    of counters for every shape.  Prompts: none where blocks fill the chip."""
    n = lib.tf_kv4_attention_workspace_bytes(1, 1, 32, 8, 128)
    assert n > 0 and n % 256 == 0
    assert lib.tf_kv4_attention_workspace_bytes(64, 1, 32, 8, 128) == n
    # 32 rows a workgroup: twice the parts' rows, of as many workgroups (heads of
    # 256) or of half as many (128, where the rows' sums halve what a unit holds)
    assert lib.tf_kv4_attention_workspace_bytes(1, 8, 32, 8, 128) == n
    assert lib.tf_kv4_attention_workspace_bytes(1, 4, 8, 1, 256) > lib.tf_kv4_attention_workspace_bytes(1, 1, 8, 1, 256)
    assert lib.tf_kv4_attention_workspace_bytes(1, 9, 32, 8, 128) == tfb.TF_ERR_ARG
    assert lib.tf_kv4_attention_workspace_bytes(1, 1, 30, 8, 128) == tfb.TF_ERR_SHAPE
    assert lib.tf_prompt_attention_workspace_bytes(1, 8192, 8192, 32, 8, 128) == 0
    assert lib.tf_prompt_attention_workspace_bytes(1, 100, 100, 8, 8, 128) == 0
    assert lib.tf_prompt_attention_workspace_bytes(1, 500, 7500, 16, 2, 128) > 0
    assert lib.tf_prompt_attention_workspace_bytes(1, 500, 7500, 16, 3, 128) == tfb.TF_ERR_SHAPE


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64).half()
    kv, cu = torch.zeros(4, 1, 64).half(), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        tfb.add_rms_norm(x, x, x[0])
    with pytest.raises(ValueError):
        tfb.prompt_attention(kv, kv, kv, cu)
    with pytest.raises(ValueError):
        tfb.KV4Cache(torch.zeros(1 << 20, dtype=torch.uint8), 2, 32, 1, 64, torch.float16)
