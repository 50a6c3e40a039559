"""8-bit linear layers and layers made of experts against the CPU oracle in float64,
at the sizes, masks and layouts where they can go wrong.

Tolerances, from the formats: u = 2^-11 (fp16) or 2^-8 (bf16) bounds the relative
error of one rounding; e = 2^-24 that of one in fp32.  A matmul's sums are exact;
its output carries the conversion of the sum, two fp32 products and the output's
rounding: u + 3 e, and e u more.
"""
from __future__ import annotations

import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f16": 2.0 ** -25, "bf16": 0.0}            # half the smallest subnormal step
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
E32 = 2.0 ** -24


@pytest.fixture(scope="module")
def tf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_11357_amd import tilefuse
    tilefuse.load()
    return tilefuse


def up(a, dt):
    """float64 -> (GPU tensor of dt, its values as float64)."""
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DT[dt])
    return t.cuda(), t.double().numpy()


def put(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def down(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------------------
# codes of rows
# ---------------------------------------------------------------------------
ROWS = [(1, 16), (1, 4096), (3, 512), (5, 528), (2, 1040), (9, 2048), (4, 2064), (3, 4112), (2, 8208), (1, 16400),
        (2, 65536), (130, 14336)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N", ROWS)
def test_quantize(tf, dt, gated, M, N):
    rng = np.random.default_rng(M * 7 + N)
    x, xv = up(rng.standard_normal((M, 2 * N if gated else N)) * np.exp(rng.standard_normal((M, 1))), dt)
    q, s = tf.quantize_rows(x, gated=gated)
    assert q.dtype == torch.int8 and s.dtype == torch.float32 and q.shape == (M, N)
    v, unit = oracle.row_codes(oracle.gated_rows(xv) if gated else xv)
    # of h and of its maximum: exp (two units in the last place and half one of its argument's sign change,
    # none), 1 + exp, the quotient, the product: 2 * 2 + 3 roundings; then 127 / max and the product
    off = (2 * 7 if gated else 0) + 2
    assert (np.abs(down(s) - unit) <= (off // 2 + 1) * E32 * unit).all()
    assert (np.abs(down(q) - v) <= 0.5 + off * E32 * 127).all()


def test_quantize_strides_and_outputs(tf):
    """Parts of a wider matrix; given outputs; one row with any stride."""
    x = torch.randn(7, 96, device="cuda").half()
    want = tf.quantize_rows(x[:, 16:80].contiguous())
    got = tf.quantize_rows(x[:, 16:80], codes=torch.empty(7, 64, dtype=torch.int8, device="cuda"), scales=torch.empty(7, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    one = tf.quantize_rows(x[2:3, 16:80])
    assert torch.equal(one[0], want[0][2:3]) and torch.equal(one[1], want[1][2:3])
    assert tf.quantize_rows(x[:0])[0].shape == (0, 96)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_quantize_rows_that_are_odd(tf, dt):
    """Rows that are zero, tiny or not finite; one value far over the others; halves
    of codes (max 127) go to the even one."""
    x = torch.randn(8, 1040, device="cuda").to(DT[dt])
    x[0], x[1, 5], x[2, 7], x[3, 1039] = 0.0, float("nan"), float("inf"), -float("inf")
    x[4, 3] = 30000.0
    x[5] = torch.arange(1040, device="cuda") % 128 - 0.5
    x[5, 0] = 127.0
    if dt == "bf16":
        x[6] = 2.0 ** -101
        x[7] = 2.0 ** -101
        x[7, 9] = 2.0 ** -99
    q, s = tf.quantize_rows(x)
    v, unit = oracle.row_codes(down(x))
    np.testing.assert_array_equal(np.isnan(down(s)), np.isnan(unit))
    ok = ~np.isnan(unit)
    assert (np.abs(down(s) - unit)[ok] <= 2 * E32 * unit[ok]).all()
    assert (np.abs(down(q) - v) <= 0.5 + 2 * E32 * 127).all()
    assert (q[1:4] == 0).all() and (q[0] == 0).all() and s[0] == 0
    np.testing.assert_array_equal(down(q)[5], np.round(v[5]))


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def weight(rng, shape):
    return rng.integers(-128, 128, shape).astype(np.int8)


def check_product(got, want, dt):
    assert (np.abs(got - want) <= (U[dt] + 4 * E32) * np.abs(want) + TINY[dt]).all()


SIZES = [(1, 16, 8), (1, 4096, 4096), (3, 144, 24), (15, 80, 40), (16, 128, 16), (17, 272, 136), (32, 1040, 200),
         (33, 208, 72), (64, 512, 264), (65, 64, 64), (100, 4112, 520), (128, 256, 256), (129, 192, 48), (200, 2048, 1000),
         (256, 128, 256), (257, 336, 264), (300, 1024, 776), (511, 640, 512), (512, 4096, 768), (700, 272, 1032),
         (1024, 1024, 2048), (1100, 512, 1288)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_gemm(tf, dt, M, K, N):
    """Random codes in the whole range of 8 bits; the scales keep fp16 from its limits."""
    rng = np.random.default_rng(M * 31 + K * 7 + N)
    q, w = weight(rng, (M, K)), weight(rng, (K, N))
    s, sv = (0.5 + rng.random(M)).astype(np.float32), None
    ws, wsv = up((0.5 + rng.random(N)) / (5500 * K ** 0.5), dt)
    packed = tf.pack_w8a8(put(w), ws)
    out = tf.w8a8_gemm(put(q), put(s), packed, K, N, dtype=DT[dt])
    assert out.shape == (M, N) and out.dtype == DT[dt]
    check_product(down(out), oracle.w8a8(q, s, w, wsv), dt)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_gemm_extremes(tf, M):
    """The largest sums: 65536 products of 128 squared; rows beside a matrix of noise."""
    K, N = 65536, 24
    q, w = torch.full((M, K), -128, dtype=torch.int8), torch.full((K, N), -128, dtype=torch.int8)
    q[0, ::2] = 127
    packed = tf.pack_w8a8(w.cuda(), torch.full((N,), 2.0 ** -20, device="cuda"))
    out = tf.w8a8_gemm(q.cuda(), torch.ones(M, device="cuda"), packed, K, N, dtype=torch.bfloat16)
    sums = (q.double().sum(1) * -128)[:, None].expand(M, N)
    assert torch.equal(out.cpu(), (sums * 2.0 ** -20).to(torch.bfloat16))


def test_gemm_rows_that_are_not_finite(tf):
    """A scale that is NaN makes its own row NaN and no other."""
    q = torch.randint(-127, 128, (70, 128), device="cuda").to(torch.int8)
    s = torch.ones(70, device="cuda")
    s[3] = float("nan")
    packed = tf.pack_w8a8(torch.randint(-127, 128, (128, 64), device="cuda").to(torch.int8), torch.ones(64, device="cuda") * 1e-3)
    out = tf.w8a8_gemm(q, s, packed, 128, 64, dtype=torch.bfloat16)
    assert torch.isnan(out[3]).all() and torch.isfinite(out[torch.arange(70) != 3]).all()


def test_gemm_leaves_its_neighbours(tf):
    """Rows and columns past the output stay as they are."""
    for M, K, N in ((5, 80, 24), (70, 144, 72), (300, 144, 264)):
        big = torch.full((M + 4, N), 7.0, device="cuda", dtype=torch.float16)
        w = torch.ones(K, N, dtype=torch.int8, device="cuda")
        packed = tf.pack_w8a8(w, torch.ones(N, device="cuda"))
        out = tf.w8a8_gemm(torch.ones(M, K, dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda"), packed, K, N,
                           out=big[2:M + 2])
        assert (out == K).all() and (big[:2] == 7).all() and (big[M + 2:] == 7).all()


def test_scales_of_each_type(tf):
    w = torch.randint(-127, 128, (64, 40), device="cuda").to(torch.int8)
    s = (0.01 + torch.rand(40, device="cuda")).bfloat16()
    want = tf.pack_w8a8(w, s.float())
    assert torch.equal(tf.pack_w8a8(w, s), want)
    h = s.half()
    assert torch.equal(tf.pack_w8a8(w, h), tf.pack_w8a8(w, h.float()))


# ---------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------
ROUTES = [
    dict(T=1, E=1, k=1), dict(T=1, E=8, k=2), dict(T=64, E=8, k=2, renormalize=True), dict(T=5, E=60, k=4, scoring="sigmoid"),
    dict(T=33, E=64, k=8, scale=2.5), dict(T=7, E=65, k=32, renormalize=True), dict(T=100, E=128, k=6, bias=True),
    dict(T=130, E=256, k=8, scoring="sigmoid", groups=8, top_groups=4, bias=True, renormalize=True, scale=2.5),
    dict(T=40, E=256, k=8, groups=8, top_groups=3, group_score="max"), dict(T=21, E=60, k=5, groups=4, top_groups=2),
    dict(T=11, E=64, k=3, groups=64, top_groups=5), dict(T=9, E=512, k=10, groups=2, top_groups=1, scoring="sigmoid"),
    dict(T=6, E=1000, k=12, groups=40, top_groups=7), dict(T=17, E=1024, k=1), dict(T=3, E=24, k=24, renormalize=True),
    dict(T=700, E=16, k=3, bias=True, scoring="sigmoid", renormalize=True), dict(T=1100, E=4, k=2)]


def check_routing(tf, logits, values, k, bias=None, **kw):
    T, E = values.shape
    r = tf.route_experts(logits, k, bias=None if bias is None else put(bias, torch.float32), **kw)
    w, e = oracle.route(values, k, bias=bias, **kw)
    np.testing.assert_array_equal(r.experts.cpu().numpy(), e)
    # one rounding to 32 bits; 64-bit ones far below it
    assert (np.abs(down(r.weights) - w) <= (E32 + 1e-12) * np.abs(w) + 2.0 ** -150).all()
    offsets, tokens, places = oracle.expert_order(e, E)
    np.testing.assert_array_equal(r.offsets.cpu().numpy(), offsets)
    np.testing.assert_array_equal(r.tokens.cpu().numpy(), tokens)
    np.testing.assert_array_equal(r.places.cpu().numpy(), places)


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("case", ROUTES, ids=str)
def test_route(tf, dt, case):
    case = dict(case)
    T, E, k = (case.pop(n) for n in ("T", "E", "k"))
    rng = np.random.default_rng(T * 31 + E)
    x = rng.standard_normal((T, E)) * 2
    logits = put(x, DT.get(dt, torch.float32))
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32) if case.pop("bias", False) else None
    check_routing(tf, logits, down(logits), k, bias=bias, **case)


@pytest.mark.parametrize("kw", [dict(), dict(scoring="sigmoid", renormalize=True), dict(groups=4, top_groups=2),
                                dict(groups=8, top_groups=3, group_score="max", scoring="sigmoid")], ids=str)
def test_route_ties(tf, kw):
    """Few different logits, so that most choices and groups are equal to others."""
    rng = np.random.default_rng(3)
    x = rng.integers(0, 3, (60, 64)).astype(np.float32)
    check_routing(tf, put(x), x.astype(np.float64), 6, **kw)


@pytest.mark.parametrize("kw", [dict(), dict(scoring="sigmoid"), dict(renormalize=True, bias=True), dict(groups=8, top_groups=2),
                                dict(groups=8, top_groups=2, group_score="max", scoring="sigmoid", bias=True)], ids=str)
@pytest.mark.parametrize("share", [0.3, 0.9, 1.0])
def test_route_masked(tf, share, kw):
    """-infinity and NaN in most places, rows with nothing else among them, and
    infinite logits; a bias that is not finite."""
    kw = dict(kw)
    rng = np.random.default_rng(int(share * 10))
    x = rng.standard_normal((50, 64)).astype(np.float32)
    x[rng.random(x.shape) < share] = -np.inf
    x[rng.random(x.shape) < 0.1] = np.nan
    x[::7] = -np.inf
    if "bias" not in kw:
        x[3, 5] = x[3, 9] = x[5, 60] = np.inf
    bias = None
    if kw.pop("bias", False):
        bias = rng.standard_normal(64).astype(np.float32)
        bias[4], bias[11], bias[20] = np.nan, -np.inf, np.inf
    check_routing(tf, put(x), x.astype(np.float64), 5, bias=bias, **kw)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_bias_that_masks(tf, scoring):
    """Experts that a bias takes out are chosen for want of others only, with weight 0."""
    x = np.random.default_rng(4).standard_normal((20, 6)).astype(np.float32)
    bias = np.array([-np.inf, 0.1, np.nan, -np.inf, 0.0, -0.1], np.float32)
    for k in (2, 3, 4, 6):
        check_routing(tf, put(x), x.astype(np.float64), k, bias=bias, scoring=scoring, renormalize=True)


def test_route_large_logits(tf):
    """The type's lowest and highest values, and differences that underflow."""
    big = float(np.finfo(np.float32).max)
    x = np.array([[-big, big, 0.0, 1.0], [-big] * 4, [big] * 4, [1e4, -1e4, 9e3, 9999.0], [-800.0, -700.0, -1e30, -900.0]], np.float32)
    for scoring in ("softmax", "sigmoid"):
        check_routing(tf, put(x), x.astype(np.float64), 3, scoring=scoring, renormalize=True)


def test_order_of_many_choices(tf):
    """Whole blocks of choices for every wave, a few more, and several times as many."""
    for T, E, k in ((8192, 16, 8), (8200, 16, 8), (70000, 5, 3)):
        x = torch.randn(T, E, device="cuda")
        r = tf.route_experts(x, k)
        assert torch.equal(r.experts.long(), x.double().sort(dim=1, descending=True, stable=True).indices[:, :k])
        flat = r.experts.flatten().long()
        order = torch.argsort(flat, stable=True)
        assert torch.equal(r.tokens.long(), order // k)
        assert torch.equal(r.places.flatten().long()[order], torch.arange(T * k, device="cuda"))
        assert r.offsets.tolist() == [0] + torch.bincount(flat, minlength=E).cumsum(0).tolist()


def test_route_strided_and_empty(tf):
    wide = torch.randn(9, 40, device="cuda")
    a, b = tf.route_experts(wide[:, 3:27], 4), tf.route_experts(wide[:, 3:27].contiguous(), 4)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    r = tf.route_experts(wide[:0], 4)
    assert r.weights.shape == (0, 4) and r.offsets.tolist() == [0] * 41 and r.tokens.numel() == 0


# ---------------------------------------------------------------------------
# the experts' products and their sum
# ---------------------------------------------------------------------------
def counts_of(kind, E, S, rng):
    if kind == "even":
        return [S // E + (e < S % E) for e in range(E)]
    if kind == "one":                                   # all to one expert in the middle
        return [S if e == E // 2 else 0 for e in range(E)]
    cuts = np.sort(rng.integers(0, S + 1, E - 1)) if E > 1 else np.array([], int)
    return np.diff(np.concatenate([[0], cuts, [S]])).tolist()


EXPERTS = [(1, 1, 16, 8), (4, 3, 80, 24), (8, 32, 512, 264), (60, 70, 144, 40), (8, 300, 272, 200), (3, 400, 128, 520),
           (5, 1200, 208, 136), (2, 1500, 512, 512), (128, 40, 64, 64), (8, 4000, 256, 272)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["even", "one", "ragged"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("E,S,K,N", EXPERTS)
def test_expert_gemm(tf, dt, kind, gather, E, S, K, N):
    rng = np.random.default_rng(E * 31 + S + K)
    A = max(1, S // 3) if gather else S
    q, w = weight(rng, (A, K)), weight(rng, (E, K, N))
    s = (0.5 + rng.random(A)).astype(np.float32)
    ws, wsv = up((0.5 + rng.random((E, N))) / (5500 * K ** 0.5), dt)
    offsets = np.concatenate([[0], np.cumsum(counts_of(kind, E, S, rng))]).astype(np.int32)
    rows = rng.integers(0, A, S).astype(np.int32) if gather else np.arange(S, dtype=np.int32)
    out = tf.w8a8_expert_gemm(put(q), put(s), tf.pack_w8a8(put(w), ws), K, N, put(offsets), put(rows) if gather else None,
                              dtype=DT[dt])
    want = np.concatenate([oracle.w8a8(q[rows[a:b]], s[rows[a:b]], w[e], wsv[e])
                           for e, (a, b) in enumerate(zip(offsets, offsets[1:]))])
    check_product(down(out), want, dt)


@pytest.mark.parametrize("S", [50, 1000])
def test_expert_gemm_rows_of_no_expert(tf, S):
    """Rows before the first and behind the last expert's stay as they are; rows of A
    that do not exist give zeros; offsets outside the output and falling ones are
    taken within it."""
    rng = np.random.default_rng(S)
    E, K, N = 4, 144, 72
    q, w = weight(rng, (S, K)), weight(rng, (E, K, N))
    packed = tf.pack_w8a8(put(w), torch.full((E, N), 2.0 ** -12, device="cuda"))
    s = np.ones(S, np.float32)
    rows = rng.integers(0, S, S).astype(np.int32)
    rows[5], rows[6], rows[20] = -1, S, 2 ** 31 - 1
    offsets = np.array([3, S // 2, S // 2, S // 2 + 7, S - 4], np.int32)
    out = torch.full((S, N), 9.0, dtype=torch.bfloat16, device="cuda")
    tf.w8a8_expert_gemm(put(q), put(s), packed, K, N, put(offsets), put(rows), out=out)
    want = oracle.expert_products(q, s, w, np.full((E, N), 2.0 ** -12), offsets, rows)
    mine = ~np.isnan(want).any(1)
    check_product(down(out)[mine], want[mine], "bf16")
    assert (down(out)[~mine] == 9).all() and not mine[:3].any() and not mine[S - 4:].any()
    for wild in ([-5, S, S + 9, 2 ** 31 - 1, S + 1], [0, S, -7, 5, 4]):
        got = tf.w8a8_expert_gemm(put(q), put(s), packed, K, N, put(np.array(wild, np.int32)), dtype=torch.bfloat16)
        check_product(down(got), oracle.w8a8(q, s, w[0], np.full(N, 2.0 ** -12)), "bf16")


@pytest.mark.parametrize("slots,a_rows", [(40, 5), (40, 1), (600, 300), (3000, 2), (3000, 2600)])
def test_expert_gemm_more_slots_than_rows(tf, slots, a_rows):
    """Slots past the last row of A, without rows, are rows that do not exist: zeros (the
    C entry; the binding has a slot for each row)."""
    rng = np.random.default_rng(slots)
    E, K, N = 2, 272, 72
    q, w = weight(rng, (a_rows, K)), weight(rng, (E, K, N))
    s, packed = np.ones(a_rows, np.float32), tf.pack_w8a8(put(w), torch.full((E, N), 2.0 ** -12, device="cuda"))
    offsets = np.array([0, slots // 2, slots], np.int32)
    out = torch.full((slots + 1, N), 9.0, dtype=torch.bfloat16, device="cuda")
    qd, sd, od = put(q), put(s), put(offsets)
    tf._launch("tf_w8a8_expert_gemm", out.device, tf.TF_BF16, tf._ptr(qd), tf._ptr(sd), a_rows, tf._ptr(packed),
               tf._ptr(od), None, tf._ptr(out), slots, K, N, E)
    want = oracle.expert_products(q, s, w, np.full((E, N), 2.0 ** -12), offsets, np.arange(slots))
    check_product(down(out)[:slots], want, "bf16")
    assert (out[slots:] == 9).all() and (out[a_rows:slots] == 0).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("T,k,N", [(1, 1, 8), (1, 2, 4096), (7, 3, 264), (50, 8, 2048), (33, 32, 40), (300, 9, 520), (4, 6, 65536)])
def test_combine(tf, dt, add, T, k, N):
    rng = np.random.default_rng(T + k + N)
    S = T * k
    y, yv = up(rng.standard_normal((S, N)), dt)
    w = rng.random((T, k)).astype(np.float32)
    places = rng.permutation(S).astype(np.int32).reshape(T, k)
    a, av = up(rng.standard_normal((T, N)), dt) if add else (None, None)
    out = tf.combine_experts(y, put(w), put(places), add=a)
    want = oracle.combine(yv, w, places, av)
    terms = oracle.combine(np.abs(yv), w, places, None if av is None else np.abs(av))
    # one rounding of every partial sum (an fma each, one more for add)
    assert (np.abs(down(out) - want) <= U[dt] * np.abs(want) + (k + 2) * E32 * terms + TINY[dt]).all()


def test_combine_leaves_out(tf):
    """Weight 0 and places that do not exist add nothing, whatever is there; in place."""
    y = torch.ones(4, 64, device="cuda").half()
    y[1], y[2] = float("nan"), float("inf")
    w = put(np.array([[1.0, 0.0, 0.0], [2.0, 3.0, 1.0], [0.0, 0.0, 0.0]], np.float32))
    places = put(np.array([[0, 1, 2], [-1, 4, 3], [1, 2, 2 ** 31 - 1]], np.int32))
    add = torch.full((3, 64), 0.5, device="cuda").half()
    got = tf.combine_experts(y, w, places, add=add, out=add)
    assert got is add and (got[0] == 1.5).all() and (got[1] == 1.5).all() and (got[2] == 0.5).all()
    assert (tf.combine_experts(y[:0], w, places) == 0).all()
