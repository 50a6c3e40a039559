"""Python binding of libtilefuse (ctypes; argument marshalling only).

Every computation runs in the library's HIP kernels; torch supplies device
memory and the current stream.  The names mirror the C ABI in
``include/tilefuse.h``.  The library has no fallback: if it is not built, the
first call fails with an error that says how to build it.  The native half of
the matmul calls only saves host time; without it they run through ctypes.
"""
from __future__ import annotations

import collections
import ctypes
import os
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
# TILEFUSE_LIB names another build of the same library to load instead (the
# host-sanitizer build the CPU tests run the argument checks under).
LIB_PATH = os.environ.get("TILEFUSE_LIB") or os.path.join(PKG, "libtilefuse.so")

TF_OK = 0
TF_ERR_NULL = -1
TF_ERR_SHAPE = -2
TF_ERR_GROUP = -3
TF_ERR_ALIGN = -4
TF_ERR_ARG = -5
TF_ERR_HIP = -6
TF_F16 = 1
TF_F32 = 2
TF_BF16 = 3
GEMV_MAX_M = 8

EXPORTS = (
    "tf_layout_version", "tf_status_str", "tf_packed_bytes", "tf_pack_w4", "tf_pack_w8",
    "tf_pack_w8_sym", "tf_workspace_bytes", "tf_gemm_workspace_bytes", "tf_w4a16_gemm",
    "tf_w8a16_gemm", "tf_w4a16_gemv", "tf_w8a16_gemv", "tf_w4a16_gemv_noalloc", "tf_w4a16_gemm_bf16", "tf_w8a16_gemm_bf16", "tf_w4a16_gemv_bf16",
    "tf_w8a16_gemv_bf16", "tf_unpack", "tf_dequant", "tf_silu_mul", "tf_silu_mul_bf16",
    "tf_add_rms_norm", "tf_kv4_cache_bytes", "tf_kv4_append", "tf_kv4_read",
    "tf_kv4_attention_workspace_bytes", "tf_kv4_attention", "tf_prompt_attention_workspace_bytes",
    "tf_prompt_attention", "tf_quantize_rows", "tf_w8a8_packed_bytes", "tf_pack_w8a8", "tf_w8a8_workspace_bytes",
    "tf_w8a8_gemm", "tf_route_experts", "tf_w8a8_expert_gemm", "tf_combine_experts",
)


class _Kv4Struct(ctypes.Structure):
    """tf_kv4_cache"""
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("max_pages", ctypes.c_int64)]


class TileFuseError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} (status {status})")


_lib = None


def load() -> ctypes.CDLL:
    """Load libtilefuse.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing; build it with "
                          "`python -m paper_2606_11357_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    P, I64, I, SZ, F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
    C = ctypes.POINTER(_Kv4Struct)
    sig = {
        "tf_layout_version": (I, []),
        "tf_status_str": (ctypes.c_char_p, [I]),
        "tf_packed_bytes": (I64, [I, I64, I64, I]),
        "tf_pack_w4": (I, [P, P, P, I64, I64, I, P, P]),
        "tf_pack_w8": (I, [P, P, P, I64, I64, I, P, P]),
        "tf_pack_w8_sym": (I, [P, P, I64, I64, I, P, P]),
        "tf_workspace_bytes": (I64, [I, I64, I64, I64, I]),
        "tf_gemm_workspace_bytes": (I64, [I, I64, I64, I64, I]),
        "tf_w4a16_gemm": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_w8a16_gemm": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_w4a16_gemv": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_w8a16_gemv": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_w4a16_gemv_noalloc": (I, [P, P, P, I64, I64, I64, I, P]),
        "tf_w4a16_gemm_bf16": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_w8a16_gemm_bf16": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_w4a16_gemv_bf16": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_w8a16_gemv_bf16": (I, [P, P, P, I64, I64, I64, I, P, SZ, P]),
        "tf_unpack": (I, [I, P, I64, I64, I, P, P, P]),
        "tf_dequant": (I, [I, P, I64, I64, I, I, P, P]),
        "tf_silu_mul": (I, [P, I64, I64, P, P]),
        "tf_silu_mul_bf16": (I, [P, I64, I64, P, P]),
        "tf_add_rms_norm": (I, [I, P, P, P, P, I64, F, P, F, F, I64, I64, P, P, P]),
        "tf_kv4_cache_bytes": (I64, [I64, I, I, I]),
        "tf_kv4_append": (I, [C, P, I64, P, I64, P, I64, P, P, I64, P, P, I64, I64, I, P, P, P]),
        "tf_kv4_read": (I, [C, P, P, I64, I64, P, P, P]),
        "tf_kv4_attention_workspace_bytes": (I64, [I64, I, I, I, I]),
        "tf_kv4_attention": (I, [C, P, I64, P, I64, I, I, F, P, P, SZ, P]),
        "tf_prompt_attention": (I, [I, P, I64, P, I64, P, I64, P, P, I64, I64, I64, I, I, I, F, I, P, P, SZ, P]),
        "tf_prompt_attention_workspace_bytes": (I64, [I64, I64, I64, I, I, I]),
        "tf_quantize_rows": (I, [I, P, I64, I64, I64, I, P, P, P]),
        "tf_w8a8_packed_bytes": (I64, [I64, I64]),
        "tf_pack_w8a8": (I, [P, P, I, I64, I64, I64, P, P]),
        "tf_w8a8_workspace_bytes": (I64, [I64, I64, I64]),
        "tf_w8a8_gemm": (I, [I, P, P, P, P, I64, I64, I64, P, SZ, P]),
        "tf_route_experts": (I, [I, P, I64, P, I64, I, I, I, I, I, I, I, F, P, P, P, P, P, P]),
        "tf_w8a8_expert_gemm": (I, [I, P, P, I64, P, P, P, P, I64, I64, I64, I64, P]),
        "tf_combine_experts": (I, [I, P, I64, P, P, P, I64, I, I64, P, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def status_str(status: int) -> str:
    return load().tf_status_str(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != TF_OK:
        raise TileFuseError(status, where)


# ---------------------------------------------------------------------------
# torch-facing wrappers
# ---------------------------------------------------------------------------
def _torch():
    import torch
    return torch


def _launch(name, device, *args):
    """One call of the library on the device's current stream, with the device current
    (a launch goes to the current one, whatever its stream is)."""
    torch = _torch()
    if device.index != torch._C._cuda_getDevice():
        with torch.cuda.device(device):
            return _launch(name, device, *args)
    _check(getattr(load(), name)(*args, ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(device.index))), name)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _need_cuda(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("tensors must be on the GPU (the library has no CPU path)")
        if t is not None and not t.is_contiguous():
            raise ValueError("tensors must be contiguous")


def packed_bytes(bits: int, K: int, N: int, group: int = 128) -> int:
    n = load().tf_packed_bytes(bits, K, N, group)
    if n < 0:
        raise TileFuseError(int(n), "tf_packed_bytes")
    return int(n)


def workspace_bytes(bits: int, M: int, K: int, N: int, group: int = 128) -> int:
    n = load().tf_workspace_bytes(bits, M, K, N, group)
    if n < 0:
        raise TileFuseError(int(n), "tf_workspace_bytes")
    return int(n)


# Arrival counters are in the first bytes of every workspace; nothing else in one
# needs an initial value.
_COUNTER_BYTES = 8192


def _capture_of(stream: int) -> int:
    """The graph capture that the stream of that handle is in: a number that no other
    capture has, or 0 where it is in none."""
    if stream == 0:                      # the default stream cannot be captured
        return 0
    state, number = ctypes.c_int(0), ctypes.c_ulonglong(0)
    if load().hipStreamGetCaptureInfo(ctypes.c_void_p(stream), ctypes.byref(state), ctypes.byref(number)) != 0:
        raise TileFuseError(TF_ERR_HIP, "hipStreamGetCaptureInfo")
    return number.value + 1 if state.value else 0


def _place(device):
    """What a cached workspace is kept under: device, current stream, its capture."""
    torch = _torch()
    device = torch.device(device)
    index = torch.cuda.current_device() if device.index is None else device.index
    stream = torch.cuda.current_stream(index).cuda_stream
    return index, stream, _capture_of(stream)


def _stream_workspace(cache, device, nbytes, counters=True):
    """A workspace of at least nbytes for calls on the current stream, cached.

    Each stream has its own, made, used and (where a call needs more) given back in
    that stream's order.  A call under capture takes one of the graph's: from the
    memory of the graph (torch.cuda.graph's), its counters cleared by a captured
    fill, so that neither a replay nor an eager call ever meets what the other
    left.  It serves the calls of that capture; the next capture gives it back."""
    torch = _torch()
    key = _place(device)
    buf = cache.get(key)
    if buf is None or buf.numel() < nbytes:
        if key[2]:
            for old in [k for k in list(cache) if k[2] not in (0, key[2])]:
                cache.pop(old, None)
            buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
            if counters:
                buf[:_COUNTER_BYTES].zero_()
        else:
            buf = (torch.zeros if counters else torch.empty)(nbytes, dtype=torch.uint8, device=device)
        cache[key] = buf
    return buf


_default_ws = {}


def default_workspace(device, nbytes: int):
    """A zero-filled workspace of at least `nbytes`, cached per device and stream
    (and, under capture, per capture: _stream_workspace).

    Every call returns the workspace's arrival counters to zero, so the cached
    buffer serves later calls of any shape on its stream without clearing; it must
    not be shared by calls running concurrently on different streams.
    """
    return _stream_workspace(_default_ws, device, max(nbytes, 1 << 20))


def pack_w4(qweight, qzeros, scales, K: int, N: int, group: int = 128, out=None):
    """Pre-tile an AWQ 4-bit weight (int32 [K, N/8], int32 [K/G, N/8], fp16 or bf16
    [K/G, N]; the scale bits are copied as they are)."""
    torch = _torch()
    _need_cuda(qweight, qzeros, scales)
    if out is None:
        out = torch.empty(packed_bytes(4, K, N, group), dtype=torch.uint8, device=qweight.device)
    _launch("tf_pack_w4", qweight.device, _ptr(qweight), _ptr(qzeros), _ptr(scales), K, N, group, _ptr(out))
    return out


def pack_w8(qweight, zeros, scales, K: int, N: int, group: int = 128, out=None):
    """Pre-tile an 8-bit weight (uint8 [K, N], uint8 [K/G, N], fp16 or bf16 [K/G, N])."""
    torch = _torch()
    _need_cuda(qweight, zeros, scales)
    if out is None:
        out = torch.empty(packed_bytes(8, K, N, group), dtype=torch.uint8, device=qweight.device)
    _launch("tf_pack_w8", qweight.device, _ptr(qweight), _ptr(zeros), _ptr(scales), K, N, group, _ptr(out))
    return out


def pack_w8_sym(qweight, scales, K: int, N: int, group: int = 128, out=None):
    """Pre-tile a signed INT8 weight with one scale per output channel
    (int8 [K, N], fp16 or bf16 [N]); use it with the 8-bit matmul calls and `group`."""
    torch = _torch()
    _need_cuda(qweight, scales)
    if out is None:
        out = torch.empty(packed_bytes(8, K, N, group), dtype=torch.uint8, device=qweight.device)
    _launch("tf_pack_w8_sym", qweight.device, _ptr(qweight), _ptr(scales), K, N, group, _ptr(out))
    return out


_bound = None


def _native():
    """The native module's matmul, bound to the loaded library's functions;
    where the module is missing or does not load (another Python or torch than
    it was built for), a stand-in that leaves every call to the general path,
    which needs the library alone."""
    global _bound
    if _bound is None:
        torch = _torch()
        lib = load()
        try:
            from . import _tf_binding
        except ImportError as e:
            _bound = lambda *call: NotImplemented  # noqa: E731
            warnings.warn(f"the native binding does not load ({e}): matmul calls take about 5 us more on the host; "
                          "build it with `python -m paper_2606_11357_amd.build`", RuntimeWarning, stacklevel=4)
            return _bound
        at = lambda name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value  # noqa: E731
        fns = tuple(at(f"tf_w{bits}a16_{kind}{dt}") for bits in (4, 8) for kind in ("gemm", "gemv")
                    for dt in ("", "_bf16"))
        stream = torch._C._cuda_getCurrentRawStream
        _tf_binding.bind(fns, at("tf_workspace_bytes"), stream, _default_ws, default_workspace,
                         at("hipStreamGetCaptureInfo"))
        _bound = _tf_binding.matmul
    return _bound


def _matmul(bits, kind, A, packed, K, N, group, out, workspace):
    # The common form in one native call (a decode loop would otherwise wait
    # for the steps below); any other form, and every refusal, comes back as
    # NotImplemented and takes them.
    got = (_bound or _native())(bits, kind == "gemv", A, packed, K, N, group, out, workspace)
    if type(got) is int:
        _check(got, f"tf_w{bits}a16_{kind}" + ("_bf16" if A.dtype == _torch().bfloat16 else ""))
    if got is not NotImplemented:
        return got
    return _matmul_general(bits, kind, A, packed, K, N, group, out, workspace)


def _matmul_general(bits, kind, A, packed, K, N, group, out, workspace):
    """A fp16 or bfloat16 [M, K] selects the entry point (the packed scales must
    hold the same dtype's bits); the output has A's dtype.
    workspace: None -> the current stream's cached default, False -> none (single-pass
    kernels), or a caller tensor (zero-filled before its first use)."""
    torch = _torch()
    _need_cuda(A, packed, out)
    M = A.shape[0]
    if A.dtype not in (torch.float16, torch.bfloat16) or A.dim() != 2 or A.shape[1] != K:
        raise ValueError("A must be fp16 or bf16 [M, K]")
    if out is None:
        out = torch.empty((M, N), dtype=A.dtype, device=A.device)
    elif out.dtype != A.dtype or tuple(out.shape) != (M, N):
        raise ValueError("out must have A's dtype and shape [M, N]")
    if workspace is None:
        need = workspace_bytes(bits, M, K, N, group)
        workspace = default_workspace(A.device, need) if need else False
    if workspace is False:
        ws_ptr, ws_bytes = None, 0
    else:
        _need_cuda(workspace)
        ws_ptr, ws_bytes = _ptr(workspace), workspace.numel() * workspace.element_size()
    name = f"tf_w{bits}a16_{kind}" + ("_bf16" if A.dtype == torch.bfloat16 else "")
    _launch(name, A.device, _ptr(A), _ptr(packed), _ptr(out), M, K, N, group, ws_ptr, ws_bytes)
    return out


def w4a16_gemm(A, packed, K: int, N: int, group: int = 128, out=None, workspace=None):
    return _matmul(4, "gemm", A, packed, K, N, group, out, workspace)


def w8a16_gemm(A, packed, K: int, N: int, group: int = 128, out=None, workspace=None):
    return _matmul(8, "gemm", A, packed, K, N, group, out, workspace)


def w4a16_gemv(A, packed, K: int, N: int, group: int = 128, out=None, workspace=None):
    return _matmul(4, "gemv", A, packed, K, N, group, out, workspace)


def w8a16_gemv(A, packed, K: int, N: int, group: int = 128, out=None, workspace=None):
    return _matmul(8, "gemv", A, packed, K, N, group, out, workspace)


def w4a16_gemv_noalloc(A, packed, K: int, N: int, group: int = 128, out=None):
    """The decode GEMV through tf_w4a16_gemv_noalloc: no workspace argument, the
    library's static per-device scratch instead (A fp16 [M, K], 1 <= M <= 8)."""
    torch = _torch()
    _need_cuda(A, packed, out)
    M = A.shape[0]
    if A.dtype != torch.float16 or A.dim() != 2 or A.shape[1] != K:
        raise ValueError("A must be fp16 [M, K]")
    if out is None:
        out = torch.empty((M, N), dtype=A.dtype, device=A.device)
    elif out.dtype != A.dtype or tuple(out.shape) != (M, N):
        raise ValueError("out must have A's dtype and shape [M, N]")
    _launch("tf_w4a16_gemv_noalloc", A.device, _ptr(A), _ptr(packed), _ptr(out), M, K, N, group)
    return out


def unpack(bits: int, packed, K: int, N: int, group: int = 128):
    """Codes q [K, N] and zero-points z [K/G, N] read back from a packed buffer."""
    torch = _torch()
    _need_cuda(packed)
    q = torch.empty((K, N), dtype=torch.uint8, device=packed.device)
    z = torch.empty((K // group, N), dtype=torch.uint8, device=packed.device)
    _launch("tf_unpack", packed.device, bits, _ptr(packed), K, N, group, _ptr(q), _ptr(z))
    return q, z


def dequant(bits: int, packed, K: int, N: int, group: int = 128, dtype=None):
    """Dequantized weights [K, N]: fp16 rounded once or exact fp32 (fp16 scales),
    or bfloat16 rounded once (bfloat16 scales)."""
    torch = _torch()
    dtype = dtype or torch.float16
    _need_cuda(packed)
    code = {torch.float16: TF_F16, torch.float32: TF_F32, torch.bfloat16: TF_BF16}[dtype]
    w = torch.empty((K, N), dtype=dtype, device=packed.device)
    _launch("tf_dequant", packed.device, bits, _ptr(packed), K, N, group, code, _ptr(w))
    return w


def silu_mul(gu, out=None):
    """H = silu(gu[:, :N]) * gu[:, N:] for an fp16 or bfloat16 [M, 2N] CUDA
    tensor (the gate and up halves side by side); returns [M, N] of gu's dtype."""
    torch = _torch()
    _need_cuda(gu, out)
    if gu.dtype not in (torch.float16, torch.bfloat16) or gu.dim() != 2 or gu.shape[1] % 2 != 0:
        raise ValueError("gu must be fp16 or bf16 [M, 2N]")
    M, N = gu.shape[0], gu.shape[1] // 2
    if out is None:
        out = torch.empty((M, N), dtype=gu.dtype, device=gu.device)
    elif out.dtype != gu.dtype:
        raise ValueError("out must have gu's dtype")
    name = "tf_silu_mul_bf16" if gu.dtype == torch.bfloat16 else "tf_silu_mul"
    _launch(name, gu.device, _ptr(gu), M, N, _ptr(out))
    return out


# ---------------------------------------------------------------------------
# the rest of a decoder layer: norm, 4-bit paged cache, attention
# ---------------------------------------------------------------------------
def _dtype_code(dtype, what):
    torch = _torch()
    if dtype == torch.float16:
        return TF_F16
    if dtype == torch.bfloat16:
        return TF_BF16
    raise ValueError(f"{what} must be fp16 or bf16")


def _same(t, dtype, device, shape, what):
    if t.dtype != dtype or t.device != device or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be {dtype} {list(shape)} on {device}")


def _heads_of(t, what):
    """Checks a [tokens, heads, head_dim] operand whose tokens may be strided;
    its token stride."""
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU (the library has no CPU path)")
    if t.dim() != 3:
        raise ValueError(f"{what} must be [tokens, heads, head_dim]")
    T, H, D = t.shape
    if t.is_contiguous():                # (one without elements whatever its strides are)
        return H * D
    if (D > 1 and t.stride(2) != 1) or (H > 1 and t.stride(1) != D):
        raise ValueError(f"the heads of {what} must be contiguous")
    return t.stride(0) if T > 1 else H * D


def _int32(t, shape, device, what):
    torch = _torch()
    _need_cuda(t)
    _same(t, torch.int32, device, shape, what)


_ops = None


def _native_ops():
    """The native module's calls of these operators, bound to the loaded library's
    functions, or stand-ins that leave every call to the general paths (as for the
    matmuls, _native)."""
    global _ops
    if _ops is None:
        torch = _torch()
        lib = load()
        names = ("norm", "append", "read", "decode", "prompt")
        try:
            from . import _tf_binding_ops as native
        except ImportError as e:
            _ops = dict.fromkeys(names, lambda *call: NotImplemented)
            warnings.warn(f"the native binding does not load ({e}): norm, cache and attention calls take some 8 us more "
                          "on the host; build it with `python -m paper_2606_11357_amd.build`", RuntimeWarning, stacklevel=4)
            return _ops
        at = lambda name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value  # noqa: E731
        native.bind(tuple(at(n) for n in ("tf_add_rms_norm", "tf_kv4_append", "tf_kv4_read",
                                              "tf_kv4_attention_workspace_bytes", "tf_kv4_attention",
                                              "tf_prompt_attention_workspace_bytes", "tf_prompt_attention",
                                              "hipStreamGetCaptureInfo")),
                        torch._C._cuda_getCurrentRawStream, _attention_ws, _prompt_ws, _cached_workspace)
        _ops = {n: getattr(native, n) for n in names}
    return _ops


def _call(name, where, *args):
    """One native call: its result, NotImplemented (for the general path), or the
    library's refusal raised."""
    got = (_ops or _native_ops())[name](*args)
    if type(got) is int:
        _check(got, where)
    return got


def add_rms_norm(x, residual=None, weight=None, *, post_weight=None, gate=None, scale=1.0, offset=0.0, eps=1e-6,
                 out=None, residual_out=None):
    """The residual sum and the norms around it, for fp16 or bf16 [M, N]:

        y = x, or rms(x) * (post_weight + offset)
        r = residual + scale * gate * y
        out = rms(r) * (weight + offset)

    in fp32, each output rounded once.  gate is [N] or [M, N].  Returns (out, r);
    without a weight out is None, and with nothing that changes x (no residual,
    post_weight, gate or scale) r is x.  residual_out may be residual itself and
    out may be x: both are then updated in place."""
    got = _call("norm", "tf_add_rms_norm", x, residual, weight, post_weight, gate, scale, offset, eps, out, residual_out)
    if got is not NotImplemented:
        return got
    torch = _torch()
    _need_cuda(x, residual, weight, post_weight, out, residual_out)
    if x.dim() != 2:
        raise ValueError("x must be fp16 or bf16 [M, N]")
    code = _dtype_code(x.dtype, "x")
    M, N = x.shape
    for t, shape, what in ((residual, (M, N), "residual"), (weight, (N,), "weight"),
                           (post_weight, (N,), "post_weight"), (out, (M, N), "out"),
                           (residual_out, (M, N), "residual_out")):
        if t is not None:
            _same(t, x.dtype, x.device, shape, what)
    gate_stride = 0
    if gate is not None:
        if gate.dtype != x.dtype or gate.device != x.device or tuple(gate.shape) not in ((N,), (M, N)):
            raise ValueError(f"gate must be {x.dtype} [{N}] or [{M}, {N}] on {x.device}")
        if N > 1 and gate.stride(-1) != 1:
            raise ValueError("the rows of gate must be contiguous")
        gate_stride = gate.stride(0) if gate.dim() == 2 and M > 1 else 0
    if weight is None and out is not None:
        raise ValueError("out needs a weight")
    keep = residual is None and post_weight is None and gate is None and scale == 1.0 and residual_out is None
    if keep and weight is None:
        return None, x
    if out is None and weight is not None:
        out = torch.empty_like(x)
    if residual_out is None and not keep:
        residual_out = torch.empty_like(x)
    if M > 0:
        _launch("tf_add_rms_norm", x.device, code, _ptr(x), _ptr(residual), _ptr(post_weight), _ptr(gate),
                gate_stride, scale, _ptr(weight), offset, eps, M, N, _ptr(residual_out), _ptr(out))
    return out, x if keep else residual_out


def kv4_cache_bytes(pages: int, page_size: int, kv_heads: int, head_dim: int) -> int:
    n = load().tf_kv4_cache_bytes(pages, page_size, kv_heads, head_dim)
    if n < 0:
        raise TileFuseError(int(n), "tf_kv4_cache_bytes")
    return int(n)


class KV4Cache:
    """A pool of pages of 4-bit keys and values (made by kv4_cache): `data` in the
    library's layout, and the sizes it was made for."""
    __slots__ = ("data", "pages", "page_size", "kv_heads", "head_dim", "dtype", "_sizes")

    def __init__(self, data, pages, page_size, kv_heads, head_dim, dtype):
        self._sizes = (pages, page_size, kv_heads, head_dim, _dtype_code(dtype, "dtype"))
        if not data.is_cuda or not data.is_contiguous() or data.nbytes < kv4_cache_bytes(*self._sizes[:4]):
            raise ValueError("data must be contiguous GPU memory of kv4_cache_bytes(...) bytes")
        self.data, self.pages, self.page_size = data, pages, page_size
        self.kv_heads, self.head_dim, self.dtype = kv_heads, head_dim, dtype

    def _with(self, table, batch):
        torch = _torch()
        if not table.is_cuda or table.device != self.data.device:
            raise ValueError("the page table must be on the cache's GPU")
        if table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != batch:
            raise ValueError(f"the page table must be int32 [{batch}, pages]")
        if table.shape[1] > 1 and table.stride(1) != 1:
            raise ValueError("the rows of the page table must be contiguous")
        n = table.shape[1]
        return _Kv4Struct(self.data.data_ptr(), *self._sizes, table.data_ptr(), table.stride(0) if batch > 1 else n, n)


def kv4_cache(pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=None, device="cuda"):
    """A 4-bit cache of `pages` pages of page_size positions (a multiple of 32)
    for keys and values of `dtype` (fp16 or bf16); uninitialised."""
    torch = _torch()
    dtype = dtype or torch.float16
    _dtype_code(dtype, "dtype")
    data = torch.empty(kv4_cache_bytes(pages, page_size, kv_heads, head_dim), dtype=torch.uint8, device=device)
    return KV4Cache(data, pages, page_size, kv_heads, head_dim, dtype)


def kv4_append(cache, table, cu, starts, k, v, cos=None, sin=None, q=None, keys=False, q_out=None, k_out=None):
    """Rotates q and k by their positions and appends k and v to the cache.

    k, v: [tokens, kv_heads, head_dim], q: [tokens, q_heads, head_dim] (parts of
    one packed projection are fine), cu: int32 [batch + 1] offsets of the
    sequences' tokens, starts: int32 [batch] position of each sequence's first
    token, table: int32 [batch, pages].  cos, sin: fp32 [positions, head_dim / 2],
    or None for no rotation.  Returns (q, k) rotated, as new tensors or in q_out
    and k_out; q is None where it is not given, k unless keys is true or k_out
    is given."""
    got = _call("append", "tf_kv4_append", cache, table, cu, starts, k, v, cos, sin, q, keys, q_out, k_out)
    if got is not NotImplemented:
        return got
    torch = _torch()
    dev = cache.data.device
    k_stride, v_stride = _heads_of(k, "k"), _heads_of(v, "v")
    T, B = k.shape[0], starts.shape[0]
    shape = (T, cache.kv_heads, cache.head_dim)
    _same(k, cache.dtype, dev, shape, "k")
    _same(v, cache.dtype, dev, shape, "v")
    _int32(cu, (B + 1,), dev, "cu")
    _int32(starts, (B,), dev, "starts")
    st = cache._with(table, B)
    q_stride = q_heads = positions = 0
    if q is not None:
        q_stride, q_heads = _heads_of(q, "q"), q.shape[1]
        _same(q, cache.dtype, dev, (T, q_heads, cache.head_dim), "q")
        if q_out is None:
            q_out = torch.empty((T, q_heads, cache.head_dim), dtype=q.dtype, device=dev)
    elif q_out is not None:
        raise ValueError("q_out needs q")
    if keys and k_out is None:
        k_out = torch.empty(shape, dtype=k.dtype, device=dev)
    for t, n, what in ((q_out, q_heads, "q_out"), (k_out, cache.kv_heads, "k_out")):
        if t is not None:
            _need_cuda(t)
            _same(t, cache.dtype, dev, (T, n, cache.head_dim), what)
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        _need_cuda(cos, sin)
        positions = cos.shape[0]
        for t, what in ((cos, "cos"), (sin, "sin")):
            _same(t, torch.float32, dev, (positions, cache.head_dim // 2), what)
    if T > 0:
        _launch("tf_kv4_append", dev, st, _ptr(q), q_stride, _ptr(k), k_stride, _ptr(v), v_stride, _ptr(cos),
                _ptr(sin), positions, _ptr(cu), _ptr(starts), B, T, q_heads, _ptr(q_out), _ptr(k_out))
    return q_out, k_out


def kv4_read(cache, table, cu, starts, tokens: int, k_out=None, v_out=None):
    """The cached keys and values of positions starts[b] .. as [tokens, kv_heads,
    head_dim] each, packed as cu (int32 [batch + 1], cu[-1] == tokens) says."""
    got = _call("read", "tf_kv4_read", cache, table, cu, starts, tokens, k_out, v_out)
    if got is not NotImplemented:
        return got
    torch = _torch()
    dev = cache.data.device
    B = starts.shape[0]
    _int32(cu, (B + 1,), dev, "cu")
    _int32(starts, (B,), dev, "starts")
    st = cache._with(table, B)
    shape = (tokens, cache.kv_heads, cache.head_dim)
    k_out = torch.empty(shape, dtype=cache.dtype, device=dev) if k_out is None else k_out
    v_out = torch.empty(shape, dtype=cache.dtype, device=dev) if v_out is None else v_out
    for t, what in ((k_out, "k_out"), (v_out, "v_out")):
        _need_cuda(t)
        _same(t, cache.dtype, dev, shape, what)
    if tokens > 0:
        _launch("tf_kv4_read", dev, st, _ptr(cu), _ptr(starts), B, tokens, _ptr(k_out), _ptr(v_out))
    return k_out, v_out


def kv4_attention_workspace_bytes(batch: int, q_len: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    n = load().tf_kv4_attention_workspace_bytes(batch, q_len, q_heads, kv_heads, head_dim)
    if n < 0:
        raise TileFuseError(int(n), "tf_kv4_attention_workspace_bytes")
    return int(n)


_attention_ws, _prompt_ws = {}, {}


def _cached_workspace(cache, device, nbytes):
    """The attention calls' workspace (decode and prompt attention have one each), of
    which prompts need no counters."""
    return _stream_workspace(cache, device, nbytes, cache is not _prompt_ws)


def kv4_attention(q, cache, table, lens, scale=None, out=None, workspace=None):
    """Attention of each sequence's last tokens over its cached keys and values.

    q: [batch, q_heads, head_dim] or [batch, q_len, q_heads, head_dim] (q_len up
    to 8), lens: int32 [batch], the cached tokens with the asking ones; token i
    sees the positions up to lens - q_len + i.  scale: 1 / sqrt(head_dim) unless
    given.  workspace: None for a cached one of the current stream (under
    torch.cuda.graph one of the graph's), or zero-filled bytes
    (kv4_attention_workspace_bytes) of the caller's, which calls that may run
    concurrently must not share.  Returns a tensor of q's shape."""
    got = _call("decode", "tf_kv4_attention", q, cache, table, lens, scale, out, workspace)
    if got is not NotImplemented:
        return got
    torch = _torch()
    dev = cache.data.device
    if q.dim() not in (3, 4):
        raise ValueError("q must be [batch, q_heads, head_dim] or [batch, q_len, q_heads, head_dim]")
    B, q_len = q.shape[0], 1 if q.dim() == 3 else q.shape[1]
    q_heads, D = q.shape[-2:]
    _same(q, cache.dtype, dev, (*q.shape[:-1], cache.head_dim), "q")
    if q_len > 1 and B > 1 and q.stride(0) != q_len * q.stride(1):
        raise ValueError("the tokens of q must be equally spaced")
    if q.dim() == 3:
        rows = q
    elif q_len == 1:
        rows = q[:, 0]
    else:
        rows = q.as_strided((B * q_len, q_heads, D), q.stride()[1:])
    stride = _heads_of(rows, "q")
    _int32(lens, (B,), dev, "lens")
    st = cache._with(table, B)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    else:
        _need_cuda(out)
        _same(out, q.dtype, dev, q.shape, "out")
    if B == 0:
        return out
    if workspace is None:
        workspace = _cached_workspace(_attention_ws, dev, kv4_attention_workspace_bytes(B, q_len, q_heads, cache.kv_heads, D))
    elif workspace is False:
        raise ValueError("decode attention needs a workspace")
    else:
        _need_cuda(workspace)
    _launch("tf_kv4_attention", dev, st, _ptr(q), stride, _ptr(lens), B, q_len, q_heads,
            D ** -0.5 if scale is None else scale, _ptr(out), _ptr(workspace),
            workspace.numel() * workspace.element_size())
    return out


def prompt_attention_workspace_bytes(batch: int, tokens_q: int, tokens_k: int, q_heads: int, kv_heads: int,
                                     head_dim: int) -> int:
    n = load().tf_prompt_attention_workspace_bytes(batch, tokens_q, tokens_k, q_heads, kv_heads, head_dim)
    if n < 0:
        raise TileFuseError(int(n), "tf_prompt_attention_workspace_bytes")
    return int(n)


def prompt_attention(q, k, v, cu_q, cu_k=None, scale=None, causal=True, out=None, workspace=None):
    """Attention over packed prompts: q [tokens, q_heads, head_dim], k and v
    [keys, kv_heads, head_dim] (parts of one packed projection are fine), cu_q and
    cu_k int32 [batch + 1] (cu_k is cu_q unless given).  causal: the queries are
    the last of their sequence's keys.  workspace: None for a cached one of the
    current stream (under torch.cuda.graph one of the graph's), False for none
    (keys are then never split over workgroups), or bytes
    (prompt_attention_workspace_bytes) of the caller's, which calls that may run
    concurrently must not share.  Returns [tokens, q_heads, head_dim]: zeros for a
    query that sees no key; rows that no sequence owns are not written."""
    got = _call("prompt", "tf_prompt_attention", q, k, v, cu_q, cu_k, scale, causal, out, workspace)
    if got is not NotImplemented:
        return got
    torch = _torch()
    strides = [_heads_of(t, what) for t, what in ((q, "q"), (k, "k"), (v, "v"))]
    code = _dtype_code(q.dtype, "q")
    T, q_heads, D = q.shape
    Tk, kv_heads, _ = k.shape
    _same(k, q.dtype, q.device, (Tk, kv_heads, D), "k")
    _same(v, q.dtype, q.device, (Tk, kv_heads, D), "v")
    B = cu_q.shape[0] - 1
    cu_k = cu_q if cu_k is None else cu_k
    _int32(cu_q, (B + 1,), q.device, "cu_q")
    _int32(cu_k, (B + 1,), q.device, "cu_k")
    if out is None:
        out = torch.empty((T, q_heads, D), dtype=q.dtype, device=q.device)
    else:
        _need_cuda(out)
        _same(out, q.dtype, q.device, (T, q_heads, D), "out")
    if T > 0 and Tk == 0:                # one key that no sequence owns, for the call's checks and rows
        k = v = torch.zeros((1, kv_heads, D), dtype=q.dtype, device=q.device)
        Tk, strides[1:] = 1, [kv_heads * D] * 2
    if T > 0:
        if workspace is None:
            need = prompt_attention_workspace_bytes(B, T, Tk, q_heads, kv_heads, D)
            workspace = _cached_workspace(_prompt_ws, q.device, need) if need else False
        ws_bytes = 0
        if workspace is False:
            workspace = None
        else:
            _need_cuda(workspace)
            ws_bytes = workspace.numel() * workspace.element_size()
        _launch("tf_prompt_attention", q.device, code, _ptr(q), strides[0], _ptr(k), strides[1], _ptr(v),
                strides[2], _ptr(cu_q), _ptr(cu_k), B, T, Tk, q_heads, kv_heads, D,
                D ** -0.5 if scale is None else scale, int(causal), _ptr(out), _ptr(workspace), ws_bytes)
    return out


# ---------------------------------------------------------------------------
# 8-bit activations, and layers made of experts
# ---------------------------------------------------------------------------
_experts = None


def _native_experts():
    """The native module's calls of these operators (as for the norm, cache and
    attention, _native_ops)."""
    global _experts
    if _experts is None:
        torch = _torch()
        lib = load()
        names = ("quantize", "gemm", "route", "expert_gemm", "combine")
        try:
            from . import _tf_binding_experts as native
        except ImportError as e:
            _experts = dict.fromkeys(names, lambda *call: NotImplemented)
            warnings.warn(f"the native binding does not load ({e}): calls of 8-bit layers and experts take some 5 us more "
                          "on the host; build it with `python -m paper_2606_11357_amd.build`", RuntimeWarning, stacklevel=4)
            return _experts
        at = lambda name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value  # noqa: E731
        native.bind(tuple(at(n) for n in ("tf_quantize_rows", "tf_w8a8_packed_bytes", "tf_w8a8_workspace_bytes",
                                          "tf_w8a8_gemm", "tf_route_experts", "tf_w8a8_expert_gemm",
                                          "tf_combine_experts", "hipStreamGetCaptureInfo")),
                    torch._C._cuda_getCurrentRawStream, _w8a8_ws, _w8a8_workspace)
        _experts = {n: getattr(native, n) for n in names}
    return _experts


def _expert_call(name, where, *args):
    """One native call: its result, NotImplemented (for the general path), or the
    library's refusal raised."""
    got = (_experts or _native_experts())[name](*args)
    if type(got) is int:
        _check(got, where)
    return got


def _refuse(name, *args):
    """The library's refusals of a call's sizes, before memory is made for them and for
    calls without rows: one without pointers, which it refuses last."""
    status = getattr(load(), name)(*args, None)
    if status != TF_ERR_NULL:
        _check(status, name)


def quantize_rows(x, gated=False, codes=None, scales=None):
    """Codes (int8 [M, N]) and scales (fp32 [M]) of the rows of a fp16 or bf16 [M, N]
    matrix: scale = max|row| / 127, codes = round(row * 127 / max|row|).  gated: x
    is [M, 2N] and the rows are silu(x[:, :N]) * x[:, N:].  Rows may be strided (by a
    multiple of 8 elements).  A row with a value that is not finite has the scale NaN."""
    got = _expert_call("quantize", "tf_quantize_rows", x, gated, codes, scales)
    if got is not NotImplemented:
        return got
    torch = _torch()
    if not x.is_cuda:
        raise ValueError("tensors must be on the GPU (the library has no CPU path)")
    code = _dtype_code(x.dtype, "x")
    if x.dim() != 2 or (gated and x.shape[1] % 2 != 0):
        raise ValueError("x must be fp16 or bf16 [M, N], gated [M, 2N]")
    M, N = x.shape[0], x.shape[1] // (2 if gated else 1)
    if x.shape[1] > 1 and x.stride(1) != 1 and not x.is_contiguous():
        raise ValueError("the rows of x must be contiguous")
    if M == 0:
        _refuse("tf_quantize_rows", code, None, x.shape[1], 1, N, int(gated), None, None)
    codes = torch.empty((M, N), dtype=torch.int8, device=x.device) if codes is None else codes
    scales = torch.empty((M,), dtype=torch.float32, device=x.device) if scales is None else scales
    _need_cuda(codes, scales)
    _same(codes, torch.int8, x.device, (M, N), "codes")
    _same(scales, torch.float32, x.device, (M,), "scales")
    if M > 0:
        _launch("tf_quantize_rows", x.device, code, _ptr(x), x.stride(0) if M > 1 else x.shape[1], M, N, int(gated),
                _ptr(codes), _ptr(scales))
    return codes, scales


def w8a8_packed_bytes(K: int, N: int) -> int:
    """Bytes of one packed weight (of each expert's)."""
    n = load().tf_w8a8_packed_bytes(K, N)
    if n < 0:
        raise TileFuseError(int(n), "tf_w8a8_packed_bytes")
    return int(n)


def pack_w8a8(qweight, scales, out=None):
    """Pre-tile signed INT8 weights for w8a8_gemm (int8 [K, N], scales fp16, bf16 or
    fp32 [N]) or for w8a8_expert_gemm (int8 [experts, K, N], scales [experts, N])."""
    torch = _torch()
    _need_cuda(qweight, scales, out)
    if qweight.dtype != torch.int8 or qweight.dim() not in (2, 3):
        raise ValueError("qweight must be int8 [K, N] or [experts, K, N]")
    if scales.dtype not in (torch.float16, torch.bfloat16, torch.float32):
        raise ValueError("scales must be fp16, bf16 or fp32")
    _same(scales, scales.dtype, qweight.device, (*qweight.shape[:-2], qweight.shape[-1]), "scales")
    (K, N), E = qweight.shape[-2:], qweight.shape[0] if qweight.dim() == 3 else 1
    need = E * w8a8_packed_bytes(K, N)
    if out is None:
        out = torch.empty(need, dtype=torch.uint8, device=qweight.device)
    elif out.device != qweight.device or out.nbytes < need:
        raise ValueError(f"out must hold {need} bytes on {qweight.device}")
    code = TF_F32 if scales.dtype == torch.float32 else _dtype_code(scales.dtype, "scales")
    _launch("tf_pack_w8a8", qweight.device, _ptr(qweight), _ptr(scales), code, K, N, E, _ptr(out))
    return out


def _codes_of(a, scales, packed, K, N, weights, dtype):
    """Checks the operands of an 8-bit matmul; the output's type and its code."""
    torch = _torch()
    _need_cuda(a, scales, packed)
    if a.dtype != torch.int8 or a.dim() != 2 or a.shape[1] != K:
        raise ValueError("the codes must be int8 [M, K]")
    _same(scales, torch.float32, a.device, (a.shape[0],), "scales")
    if packed.device != a.device or packed.nbytes < weights * w8a8_packed_bytes(K, N):
        raise ValueError("packed must be what pack_w8a8 made for this K and N, on the codes' GPU")
    dtype = dtype or torch.float16
    return dtype, _dtype_code(dtype, "dtype")


def _product_out(out, dtype, device, shape):
    if out is None:
        return _torch().empty(shape, dtype=dtype, device=device)
    _need_cuda(out)
    _same(out, dtype, device, shape, "out")
    return out


def w8a8_workspace_bytes(M: int, K: int, N: int) -> int:
    n = load().tf_w8a8_workspace_bytes(M, K, N)
    if n < 0:
        raise TileFuseError(int(n), "tf_w8a8_workspace_bytes")
    return int(n)


_w8a8_ws = {}


def _w8a8_workspace(device, nbytes):
    """The 8-bit products' workspace for the current stream (or its capture), which
    needs no counters."""
    return _stream_workspace(_w8a8_ws, device, nbytes, False)


def w8a8_gemm(codes, scales, packed, K: int, N: int, dtype=None, out=None, workspace=None):
    """The product of int8 codes [M, K] with a scale a row (quantize_rows) and a packed
    weight (pack_w8a8): [M, N] of dtype (fp16 unless given, or bf16).  Sums are exact.
    workspace: None for a cached one of the current stream (under torch.cuda.graph one
    of the graph's), False for none (K is then never split over workgroups), or bytes
    (w8a8_workspace_bytes) of the caller's, which calls that may run concurrently must
    not share."""
    got = _expert_call("gemm", "tf_w8a8_gemm", codes, scales, packed, K, N, dtype, out, workspace)
    if got is not NotImplemented:
        return got
    dtype, code = _codes_of(codes, scales, packed, K, N, 1, dtype if out is None else dtype or out.dtype)
    M = codes.shape[0]
    out = _product_out(out, dtype, codes.device, (M, N))
    if M > 0:
        if workspace is None:
            need = w8a8_workspace_bytes(M, K, N)
            workspace = _w8a8_workspace(codes.device, need) if need else False
        ws_bytes = 0
        if workspace is False:
            workspace = None
        else:
            _need_cuda(workspace)
            if workspace.device != codes.device:
                raise ValueError(f"the workspace must be on {codes.device}")
            ws_bytes = workspace.numel() * workspace.element_size()
        _launch("tf_w8a8_gemm", codes.device, code, _ptr(codes), _ptr(scales), _ptr(packed), _ptr(out), M, K, N,
                _ptr(workspace), ws_bytes)
    return out


Routing = collections.namedtuple("Routing", "weights experts offsets tokens places")
Routing.__doc__ = """What route_experts gives: weights fp32 and experts int32 [T, top_k]; offsets int32
[experts + 1] of the experts' slots; tokens int32 [T * top_k], the token of each slot; places int32
[T, top_k], the slot of each choice."""


def route_experts(logits, top_k: int, *, bias=None, scoring="softmax", groups=1, top_groups=None, group_score="top2",
                  renormalize=False, scale=1.0):
    """Chooses top_k of the experts for each token of logits [T, experts] (fp16, bf16
    or fp32) and orders the choices by expert.

    score = softmax or sigmoid of the logits; the choice is by score + bias (fp32
    [experts]), within the top_groups best of `groups` neighbouring groups where
    given, a group's value being the sum of its two largest choices ("top2") or the
    largest ("max"); ties go to the lower index.  weights = score, divided by the sum
    of the chosen ones with renormalize, times scale.  An expert whose logit or choice
    is -infinity or NaN comes last, with weight 0.  Returns a Routing."""
    if scoring not in ("softmax", "sigmoid"):
        raise ValueError("scoring must be softmax or sigmoid")
    if group_score not in ("top2", "max"):
        raise ValueError("group_score must be top2 or max")
    by = int(scoring == "sigmoid"), groups, groups if top_groups is None else top_groups, int(group_score == "top2")
    got = _expert_call("route", "tf_route_experts", logits, top_k, bias, *by, renormalize, scale)
    if got is not NotImplemented:
        return Routing(*got)
    torch = _torch()
    if not logits.is_cuda:
        raise ValueError("tensors must be on the GPU (the library has no CPU path)")
    if logits.dim() != 2:
        raise ValueError("logits must be [T, experts]")
    dev = logits.device
    code = TF_F32 if logits.dtype == torch.float32 else _dtype_code(logits.dtype, "logits of other types than fp32")
    T, E = logits.shape
    if E > 1 and logits.stride(1) != 1 and not logits.is_contiguous():
        raise ValueError("the rows of logits must be contiguous")
    if bias is not None:
        _need_cuda(bias)
        _same(bias, torch.float32, dev, (E,), "bias")
    if max(map(abs, (top_k, *by))) >= 2 ** 31:           # (more than the library's integers hold)
        raise TileFuseError(TF_ERR_SHAPE, "tf_route_experts")
    _refuse("tf_route_experts", code, None, E, None, 1, E, top_k, *by, int(renormalize), scale, *[None] * 5)
    make = lambda n, dt=torch.int32: torch.empty(n, dtype=dt, device=dev)  # noqa: E731
    r = Routing(make((T, top_k), torch.float32), make((T, top_k)), make(E + 1), make(T * top_k), make((T, top_k)))
    if T == 0:
        r.offsets.zero_()
        return r
    _launch("tf_route_experts", dev, code, _ptr(logits), logits.stride(0) if T > 1 else E, _ptr(bias), T, E, top_k,
            *by, int(renormalize), scale, *(_ptr(t) for t in r))
    return r


def w8a8_expert_gemm(codes, scales, packed, K: int, N: int, offsets, rows=None, dtype=None, out=None):
    """The experts' products: slot i of expert e (offsets[e] <= i < offsets[e + 1],
    int32 [experts + 1] on the device) is row rows[i] (int32 [slots]; i without rows)
    of the codes times weight e.  Returns [slots, N] of dtype (fp16 unless given):
    rows that no expert has are not written, one whose row of the codes does not
    exist is zeros."""
    got = _expert_call("expert_gemm", "tf_w8a8_expert_gemm", codes, scales, packed, K, N, offsets, rows, dtype, out)
    if got is not NotImplemented:
        return got
    torch = _torch()
    _need_cuda(offsets, rows)
    E = offsets.shape[0] - 1 if offsets.dim() == 1 else -1
    if E < 1:
        raise ValueError("offsets must be int32 [experts + 1]")
    dtype, code = _codes_of(codes, scales, packed, K, N, E, dtype if out is None else dtype or out.dtype)
    _int32(offsets, (E + 1,), codes.device, "offsets")
    slots = codes.shape[0]
    if rows is not None:
        slots = rows.numel()
        _int32(rows, (slots,), codes.device, "rows")
    if slots == 0:
        _refuse("tf_w8a8_expert_gemm", code, None, None, 1, None, None, None, None, 1, K, N, E)
    out = _product_out(out, dtype, codes.device, (slots, N))
    if slots > 0 and codes.shape[0] == 0:        # no row exists: one that none asks for, for the call's checks
        codes = torch.zeros((1, K), dtype=torch.int8, device=out.device)
        scales = torch.zeros(1, dtype=torch.float32, device=out.device)
        rows = torch.full_like(rows, -1)
    if slots > 0:
        _launch("tf_w8a8_expert_gemm", codes.device, code, _ptr(codes), _ptr(scales), codes.shape[0], _ptr(packed),
                _ptr(offsets), _ptr(rows), _ptr(out), slots, K, N, E)
    return out


def combine_experts(y, weights, places, add=None, out=None):
    """out[t] = add[t] + sum_j weights[t, j] * y[places[t, j]] for y [slots, N] (fp16 or
    bf16), weights fp32 and places int32 [T, top_k], add [T, N] or None; sums in fp32.
    A choice of weight 0 or of a place outside y adds nothing.  out may be add."""
    got = _expert_call("combine", "tf_combine_experts", y, weights, places, add, out)
    if got is not NotImplemented:
        return got
    torch = _torch()
    _need_cuda(y, weights, places, add, out)
    code = _dtype_code(y.dtype, "y")
    if y.dim() != 2 or places.dim() != 2:
        raise ValueError("y must be [slots, N] and places int32 [T, top_k]")
    (T, k), N, dev = places.shape, y.shape[1], y.device
    _int32(places, (T, k), dev, "places")
    _same(weights, torch.float32, dev, (T, k), "weights")
    if add is not None:
        _same(add, y.dtype, dev, (T, N), "add")
    if T == 0:
        _refuse("tf_combine_experts", code, None, 1, None, None, None, 1, k, N, None)
    out = _product_out(out, y.dtype, dev, (T, N))
    if T > 0 and y.shape[0] == 0:                # no row exists: one that none asks for, for the call's checks
        y, places = torch.zeros((1, N), dtype=y.dtype, device=dev), torch.full_like(places, -1)
    if T > 0:
        _launch("tf_combine_experts", dev, code, _ptr(y), y.shape[0], _ptr(weights), _ptr(places), _ptr(add), T, k, N,
                _ptr(out))
    return out
