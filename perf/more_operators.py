"""Linear layers whose activations are 8-bit integers too, and layers made of
experts, as cases that can be timed and checked: the matrix product of int8
codes with a scale for each token and each channel (with the making of a token's
codes before it), the choice of experts, the experts' products over the tokens
sent to them, and the weighted sum of their outputs.

Every case computes one operator once, either in its plain form (elementary
torch operations in 32 bits, 64 where scores are compared, rounded once at the
end) or, where ``own`` is true, by the library's calls.  The layers' sizes are
those of the Llama-3-8B shape that the repository's workloads name (hidden 4096,
MLP 14336, packed q, k, v projection 6144) and generic ones.

A row x of activations stands as codes q = round(x 127 / max|x|) with a scale
s = max|x| / 127, a weight's column as codes with a scale of its own.
"""
from __future__ import annotations

import math

import torch

own = False


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _product(name, kind, dtype, M, K, N, gated=False):
    """kind linear: 16-bit activations [M, K] (gated: [M, 2 K], whose halves make
    silu(gate) * up) are turned into codes, then multiplied; product: the codes are there."""
    c = {"kind": kind, "dtype": dtype, "M": M, "K": K, "N": N, "gated": gated}
    return {"name": name, **c} if name else c


def _route(name, dtype, T, E, k, scoring="softmax", groups=1, top_groups=1, bias=False, renormalize=True):
    c = {"kind": "route", "dtype": dtype, "T": T, "E": E, "k": k, "scoring": scoring, "groups": groups,
         "top_groups": top_groups, "bias": bias, "renormalize": renormalize}
    return {"name": name, **c} if name else c


def _experts(name, dtype, T, E, k, K, N, gather):
    """T tokens, k of E experts each.  gather: the rows are the tokens', read by each
    expert that they go to (the first product); otherwise one row a choice (the second)."""
    c = {"kind": "experts", "dtype": dtype, "T": T, "E": E, "k": k, "K": K, "N": N, "gather": gather}
    return {"name": name, **c} if name else c


def _combine(name, dtype, T, k, N, add=False):
    c = {"kind": "combine", "dtype": dtype, "T": T, "k": k, "N": N, "add": add}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token through the attention block's output projection: latency
        _product("linear_m1", "linear", "fp16", 1, 4096, 4096),
        # a decode step of 16 sequences through the down projection, its input the gated activation
        _product("linear_m16_gated", "linear", "bf16", 16, 14336, 4096, True),
        # a ragged chunk of a prompt through the packed q, k, v projection
        _product("linear_m333", "linear", "bf16", 333, 4096, 6144),
        # 2048 tokens through the down projection, their codes made before
        _product("product_m2048", "product", "fp16", 2048, 14336, 4096),
        # prompts of 8192 tokens through the packed gate and up projection: the largest piece of a prefill
        _product("linear_m8192", "linear", "bf16", 8192, 4096, 28672),
        # a decode step of 64 sequences, 2 of 8 experts each
        _route("route_t64_e8", "bf16", 64, 8, 2),
        # prompts of 8192 tokens, 8 of 256 experts in 4 of 8 groups, chosen with a bias for balance
        _route("route_t8192_e256", "fp32", 8192, 256, 8, "sigmoid", 8, 4, True),
        # a decode step of 16 sequences through the experts' gate and up projections: every expert's weight, few rows
        _experts("experts_t16_e8", "bf16", 16, 8, 2, 4096, 28672, True),
        # a middle batch over many small experts
        _experts("experts_t500_e64", "fp16", 500, 64, 6, 2048, 2000, True),
        # a prompt of 4096 tokens through the experts' down projections
        _experts("experts_t4096_e8", "bf16", 4096, 8, 2, 14336, 4096, False),
        # the outputs of a decode step summed for each token
        _combine("combine_t16", "bf16", 16, 2, 4096),
        # those of a prompt, with the output of a shared expert
        _combine("combine_t8192", "bf16", 8192, 8, 4096, True),
    ]


_MOST = 8192 * 4096 * 28672


def _log_int(rng, lo, hi):
    """A power of two or an odd number between lo and hi, spread over the logarithm."""
    hi = max(lo, hi)
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, 1 << (n.bit_length() - 1) if rng.random() < 0.3 else n | 1))


def draw(rng):
    kind = rng.choice(["linear", "linear", "product", "route", "experts", "experts", "combine"])
    dtype = rng.choice(["fp16", "bf16"])
    if kind in ("linear", "product"):
        K, N = rng.choice([(4096, 4096), (4096, 6144), (4096, 28672), (14336, 4096), (2048, 2048),
                           (16 * (2 * rng.randint(8, 250) + 1), 8 * (2 * rng.randint(8, 500) + 1))])
        M = _log_int(rng, 1, min(8192, _MOST // (K * N)))
        return _product("", kind, dtype, M, K, N, kind == "linear" and rng.random() < 0.4)
    if kind == "route":
        E = rng.choice([4, 8, 16, 60, 64, 128, 256])
        groups = rng.choice([1, 1, 2, 4, 8]) if E % 16 == 0 else 1
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(8, E // groups * top_groups))
        return _route("", rng.choice(["fp16", "bf16", "fp32"]), _log_int(rng, 1, 8192), E, k,
                      rng.choice(["softmax", "sigmoid"]), groups, top_groups, rng.random() < 0.5, rng.random() < 0.7)
    if kind == "combine":
        k = rng.randint(1, 8)
        N = rng.choice([2048, 4096, 8 * (2 * rng.randint(8, 500) + 1)])
        return _combine("", dtype, _log_int(rng, 1, 8192), k, N, rng.random() < 0.5)
    E = rng.choice([4, 8, 16, 60, 64, 128])
    k = rng.randint(1, min(8, E))
    K, N = rng.choice([(4096, 28672), (14336, 4096), (4096, 4096), (2048, 2000), (1024, 4096),
                       (16 * (2 * rng.randint(8, 60) + 1), 8 * (2 * rng.randint(8, 250) + 1))])
    while E * K * N > 8 * 4096 * 28672:
        E //= 2
    k = min(k, E)
    return _experts("", dtype, _log_int(rng, 1, min(4096, _MOST // (2 * k * K * N))), E, k, K, N, rng.random() < 0.5)


def work(case):
    if case["kind"] in ("linear", "product"):
        M, K, N = case["M"], case["K"], case["N"]
        row = K + 4 if case["kind"] == "product" else (4 if case["gated"] else 2) * K
        return {"bytes": M * row + K * N + 2 * N + 2 * M * N, "flops": 2 * M * K * N}
    T, k = case["T"], case["k"]
    if case["kind"] == "route":
        E = case["E"]
        return {"bytes": T * E * (4 if case["dtype"] == "fp32" else 2) + 16 * T * k + 4 * (E + 1),
                "flops": T * E * 8}
    N = case["N"]
    if case["kind"] == "combine":
        return {"bytes": 2 * T * k * N + 8 * T * k + 2 * T * N * (2 if case["add"] else 1), "flops": 2 * T * k * N}
    E, K = case["E"], case["K"]
    rows = T if case["gather"] else T * k
    return {"bytes": rows * (K + 4) + min(E, T * k) * (K * N + 2 * N) + 2 * T * k * N, "flops": 2 * T * k * K * N}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _dt(case):
    return {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}[case["dtype"]]


def _activations(gen, M, K, dtype):
    """Activations with a few large channels, as trained models have them."""
    amp = torch.exp(0.7 * torch.randn((1, K), device="cuda", generator=gen))
    return (torch.randn((M, K), device="cuda", generator=gen) * amp).to(dtype)


def _weight(gen, shape, dtype):
    """int8 codes and a scale a column that keep outputs near the size of the inputs."""
    q = torch.empty(shape, dtype=torch.int8, device="cuda")
    for i in range(shape[0]):             # one expert's at a time: the draws are in 32 bits
        q[i] = (torch.randn(shape[1:], device="cuda", generator=gen) * 32).round().clamp(-127, 127).to(torch.int8)
    s = (0.5 + torch.rand((shape[0], shape[2]), device="cuda", generator=gen)) / (32 * shape[1] ** 0.5)
    return q, s.to(dtype)


def _codes(x):
    """The codes and scales of rows given in 32 bits."""
    top = x.abs().amax(-1, keepdim=True)
    return (x * (127.0 / top)).round().to(torch.int8), top[:, 0] / 127.0


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    gen, dt = torch.Generator(device="cuda"), _dt(case)
    gen.manual_seed(seed)
    s = {}
    if case["kind"] in ("linear", "product"):
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = _activations(gen, M, 2 * K if case["gated"] else K, dt)
        q, scales = _weight(gen, (1, K, N), dt)
        s["w"], s["ws"] = q[0], scales[0]
        if case["kind"] == "product":
            s["q"], s["s"] = _codes(s.pop("x").float())
        return s
    T, k = case["T"], case["k"]
    if case["kind"] == "combine":
        N = case["N"]
        s["y"] = torch.randn((T * k, N), device="cuda", generator=gen).to(dt)
        w = torch.rand((T, k), device="cuda", generator=gen) + 0.05
        s["weights"] = w / w.sum(-1, keepdim=True)
        s["places"] = torch.randperm(T * k, device="cuda", generator=gen).to(torch.int32).view(T, k)
        if case["add"]:
            s["add"] = torch.randn((T, N), device="cuda", generator=gen).to(dt)
        return s
    E = case["E"]
    # some experts are asked for more often than others
    logits = 1.5 * torch.randn((T, E), device="cuda", generator=gen)
    logits = logits + 0.7 * torch.randn(E, device="cuda", generator=gen)
    if case["kind"] == "route":
        s["logits"] = logits.to(dt)
        s["bias"] = 0.05 * torch.randn(E, device="cuda", generator=gen) if case["bias"] else None
        return s
    flat = logits.topk(k, dim=-1).indices.flatten()
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=E)
    s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    s["rows"] = (order // k).to(torch.int32) if case["gather"] else None
    s["most"] = int(counts.max())
    s["q"], s["s"] = _codes(_activations(gen, T if case["gather"] else T * k, case["K"], dt).float())
    s["w"], s["ws"] = _weight(gen, (E, case["K"], case["N"]), dt)
    return s


def prepare(case, seed):
    """What a serving program holds before the call.  The weights are in the form in
    which each side keeps them: the library's packed buffer, or codes and scales."""
    s = {"case": case, **_inputs(case, seed)}
    if own and "w" in s:
        from paper_2606_11357_amd import tilefuse as tf
        s["packed"] = tf.pack_w8a8(s.pop("w"), s.pop("ws"))
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_product(s):
    case = s["case"]
    if case["kind"] == "linear":
        x = s["x"].float()
        if case["gated"]:
            gate, up = x.chunk(2, -1)
            x = gate / (1 + torch.exp(-gate)) * up
        top = x.abs().amax(-1, keepdim=True)
        q, scale = (x * (127.0 / top)).round(), top / 127.0
    else:
        q, scale = s["q"].float(), s["s"][:, None]
    return (torch.matmul(q, s["w"].float()) * (scale * s["ws"].float())).to(_dt(case))


def _plain_route(s):
    case = s["case"]
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    x = s["logits"].double()                       # scores are compared: 64 bits
    if case["scoring"] == "softmax":
        e = torch.exp(x - x.amax(-1, keepdim=True))
        score = e / e.sum(-1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-x))
    choice = score if s["bias"] is None else score + s["bias"].double()
    if G > 1:
        by_group = choice.view(T, G, E // G)
        best = by_group.sort(dim=-1, descending=True).values[..., :2].sum(-1)
        taken = best.sort(dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device="cuda").scatter_(1, taken, True)
        choice = torch.where(keep[:, :, None], by_group, -math.inf).view(T, E)
    experts = choice.sort(dim=-1, descending=True, stable=True).indices[:, :k]
    weights = score.gather(1, experts)
    if case["renormalize"]:
        weights = weights / weights.sum(-1, keepdim=True)
    flat = experts.flatten()
    order = flat.sort(dim=0, stable=True).indices
    places = torch.empty_like(order).scatter_(0, order, torch.arange(T * k, device="cuda"))
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").scatter_add_(0, flat + 1, torch.ones_like(flat))
    return (weights.float(), experts.to(torch.int32), counts.cumsum(0).to(torch.int32),
            (order // k).to(torch.int32), places.view(T, k).to(torch.int32))


def _plain_experts(s):
    """Each expert's rows beside each other, as many as the largest has, in one batched product."""
    S = s["case"]["T"] * s["case"]["k"]
    slot = torch.arange(S, device="cuda")
    expert = torch.searchsorted(s["offsets"], slot.to(torch.int32), right=True) - 1
    row = slot if s["rows"] is None else s["rows"].long()
    at = slot - s["offsets"][expert]
    x = torch.zeros((s["w"].shape[0], s["most"], s["q"].shape[1]), device="cuda")
    x[expert, at] = s["q"][row].float()
    y = torch.matmul(x, s["w"].float())[expert, at]
    return (y * (s["s"][row][:, None] * s["ws"][expert].float())).to(_dt(s["case"]))


def _plain_combine(s):
    y = (s["y"][s["places"].long()].float() * s["weights"][..., None]).sum(1)
    return (y + s["add"].float() if "add" in s else y).to(_dt(s["case"]))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _own_run(s):
    from paper_2606_11357_amd import tilefuse as tf
    case = s["case"]
    kind = case["kind"]
    if kind in ("linear", "product"):
        q, scale = tf.quantize_rows(s["x"], gated=case["gated"]) if kind == "linear" else (s["q"], s["s"])
        return tf.w8a8_gemm(q, scale, s["packed"], case["K"], case["N"], dtype=_dt(case))
    if kind == "route":
        return tuple(tf.route_experts(s["logits"], case["k"], bias=s["bias"], scoring=case["scoring"],
                                      groups=case["groups"], top_groups=case["top_groups"],
                                      renormalize=case["renormalize"]))
    if kind == "experts":
        return tf.w8a8_expert_gemm(s["q"], s["s"], s["packed"], case["K"], case["N"], s["offsets"], s["rows"],
                                   dtype=_dt(case))
    return tf.combine_experts(s["y"], s["weights"], s["places"], add=s.get("add"))


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    if kind in ("linear", "product"):
        return _plain_product(state)
    if kind == "route":
        return _plain_route(state)
    return _plain_experts(state) if kind == "experts" else _plain_combine(state)


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------
def _exact_row_codes(x):
    """Rows in 64 bits as codes (whole numbers) and what one code stands for."""
    unit = x.abs().max(1, keepdim=True).values / 127
    return torch.round(x / unit), unit


def _exact_route(case, s):
    import numpy as np
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    x = s["logits"].double().cpu().numpy()
    if case["scoring"] == "softmax":
        score = np.exp(x - x.max(1, keepdims=True))
        score /= score.sum(1, keepdims=True)
    else:
        score = 1.0 / (1.0 + np.exp(-x))
    left = score.copy()
    if s["bias"] is not None:
        left += s["bias"].double().cpu().numpy()
    if G > 1:
        parts = np.sort(left.reshape(T, G, -1), axis=2)
        value = parts[:, :, -1] + (parts[:, :, -2] if parts.shape[2] > 1 else 0.0)
        for _ in range(G - case["top_groups"]):      # the worst group leaves, the highest index of equal ones
            worst = G - 1 - np.argmin(value[:, ::-1], axis=1)
            value[np.arange(T), worst] = np.inf
            left.reshape(T, G, -1)[np.arange(T), worst] = -np.inf
    chosen = np.zeros((T, k), np.int64)
    for j in range(k):
        chosen[:, j] = left.argmax(1)
        left[np.arange(T), chosen[:, j]] = -np.inf
    w = np.take_along_axis(score, chosen, 1)
    if case["renormalize"]:
        w = w / w.sum(1, keepdims=True)
    slots = np.lexsort((np.arange(T * k), chosen.ravel()))
    places = np.zeros(T * k, np.int32)
    places[slots] = np.arange(T * k)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(chosen.ravel(), minlength=E))]).astype(np.int32)
    return w, chosen.astype(np.int32), offsets, (slots // k).astype(np.int32), places.reshape(T, k)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "route":
        return _exact_route(case, s)
    if kind == "combine":
        out = s["add"].double() if case["add"] else torch.zeros((case["T"], case["N"]), dtype=torch.float64, device="cuda")
        for j in range(case["k"]):
            out += s["weights"][:, j, None].double() * s["y"][s["places"][:, j].long()].double()
        return out
    if kind == "experts":
        out = torch.zeros((case["T"] * case["k"], case["N"]), dtype=torch.float64, device="cuda")
        ends = s["offsets"].tolist()
        for e in range(case["E"]):
            a, b = ends[e], ends[e + 1]
            rows = s["rows"][a:b].long() if case["gather"] else slice(a, b)
            x = s["q"][rows].double() * s["s"][rows].double()[:, None]
            out[a:b] = x @ (s["w"][e].double() * s["ws"][e].double())
        return out
    if kind == "product":
        codes, unit = s["q"].double(), s["s"].double()[:, None]
    else:
        x = s["x"].double()
        if case["gated"]:
            x = x[:, :case["K"]] * torch.sigmoid(x[:, :case["K"]]) * x[:, case["K"]:]
        codes, unit = _exact_row_codes(x)
    return (codes @ s["w"].double()) * unit * s["ws"].double()
