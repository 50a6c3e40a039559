"""The operators around the linear layers (norm, 4-bit paged cache, attention of
single tokens over it, attention over prompts) against the CPU oracle in
float64, at the sizes, masks and layouts where they can go wrong.

Tolerances, from the formats: u = 2^-11 (fp16) or 2^-8 (bf16) bounds the
relative error of one rounding.  An output carries one rounding; the attention
kernels round each softmax weight once more (u times sum p |v| at most, twice
that where the weight times the value's scale is what is rounded and summed).
fp32 sums add terms of a few 2^-24 of what they add up, stated at each test.
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


def down(t):
    return t.double().cpu().numpy()


def i32(a):
    return torch.tensor(list(a), dtype=torch.int32).cuda()


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(int)


# ---------------------------------------------------------------------------
# norm
# ---------------------------------------------------------------------------
NORMS = [(1, 8), (1, 4096), (3, 512), (5, 520), (2, 1032), (7, 2048), (4, 2056), (3, 4104), (2, 8200), (1, 16392),
         (2, 65536), (130, 4096)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("form", ["plain", "residual", "sandwich", "rows"])
@pytest.mark.parametrize("M,N", NORMS)
def test_norm(tf, dt, form, M, N):
    rng = np.random.default_rng(M * 7 + N)
    x, xv = up(rng.standard_normal((M, N)) * 3, dt)
    w, wv = up(1 + 0.3 * rng.standard_normal(N), dt)
    kw, ov = {}, {}
    if form != "plain":
        kw["residual"], ov["residual"] = up(rng.standard_normal((M, N)) * 5, dt)
    if form in ("sandwich", "rows"):
        kw["post_weight"], ov["post"] = up(0.3 * rng.standard_normal(N), dt)
        # a gate per row is a strided part of a wider matrix
        g, gv = up(rng.random((M, 2 * N) if form == "rows" else N), dt)
        kw["gate"], ov["gate"] = (g[:, N:], gv[:, N:]) if form == "rows" else (g, gv)
        kw.update(scale=0.5, offset=1.0)
        ov.update(scale=0.5, offset=1.0)
    y, r = tf.add_rms_norm(x, weight=w, eps=1e-5, **kw)
    want, want_r = oracle.rms_norm_block(xv, weight=wv, eps=1e-5, **ov)
    # the output's rounding, and some ten fp32 roundings of 2^-24 of the terms of r
    terms = np.abs(want_r) + (np.abs(ov["residual"]) if "residual" in ov else 0)
    rms = np.sqrt((want_r ** 2).mean(-1, keepdims=True) + 1e-5)
    slack = 2.0 ** -20 * terms / rms * np.abs(wv + ov.get("offset", 0.0)) + 2.0 ** -20 * np.abs(want)
    assert (np.abs(down(y) - want) <= U[dt] * np.abs(want) + slack + TINY[dt]).all()
    if form == "plain":
        assert r is x
    else:
        assert (np.abs(down(r) - want_r) <= U[dt] * np.abs(want_r) + 2.0 ** -20 * terms + TINY[dt]).all()


def test_norm_of_many_rows_is_that_of_few(tf):
    """More than 2^24 elements: the same bits as in calls of fewer."""
    x, res = (torch.randn(4100, 4104, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(4104, device="cuda").bfloat16()
    y, r = tf.add_rms_norm(x, res, w)
    for i in range(0, 4100, 1025):
        y_part, r_part = tf.add_rms_norm(x[i:i + 1025], res[i:i + 1025], w)
        assert torch.equal(y[i:i + 1025], y_part) and torch.equal(r[i:i + 1025], r_part)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_norm_in_place_and_parts(tf, dt):
    """residual_out may be residual and out may be x; either output alone."""
    rng = np.random.default_rng(5)
    x, _ = up(rng.standard_normal((9, 2048)), dt)
    res, _ = up(rng.standard_normal((9, 2048)), dt)
    w, _ = up(rng.standard_normal(2048), dt)
    y, r = tf.add_rms_norm(x, res, w)
    none, r2 = tf.add_rms_norm(x, res)
    assert none is None and torch.equal(r, r2)
    x2, res2 = x.clone(), res.clone()
    tf.add_rms_norm(x2, res2, w, out=x2, residual_out=res2)
    assert torch.equal(x2, y) and torch.equal(res2, r)


def test_norm_values_that_are_not_finite(tf):
    """NaN and inf stay in their rows; a row of zeros gives zeros (eps > 0)."""
    x = torch.randn(4, 1024, device="cuda").half()
    x[1, 3], x[2, 5], x[3] = float("nan"), float("inf"), 0.0
    y, _ = tf.add_rms_norm(x, weight=torch.ones(1024, device="cuda").half())
    assert torch.isfinite(y[0]).all() and torch.isnan(y[1]).all() and not torch.isfinite(y[2, 5])
    assert (y[3] == 0).all()


# ---------------------------------------------------------------------------
# the cache
# ---------------------------------------------------------------------------
HEADS = [(8, 2, 128), (3, 3, 64), (8, 1, 256), (5, 1, 128)]


def table_for(lens, page, rng, spare=2, width=0):
    """Random pages, each sequence's row padded with -1."""
    need = [-(-int(n) // page) for n in lens]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    t = -np.ones((len(lens), max([1, width, *need])), dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(t).cuda(), pages


def angles(n, D):
    inv = 10000.0 ** (-np.arange(0, D // 2) * 2 / D)
    a = np.arange(n)[:, None] * inv
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("turn", [True, False], ids=["rotated", "as is"])
def test_append_and_read(tf, dt, heads, turn):
    """Packed sequences of 0, 1 and more tokens that begin anywhere in a tile,
    from strided parts of one projection: the rotated rows, and the cached ones
    exactly (a code is the outcome of float32 roundings that the oracle makes
    too)."""
    Hq, Hk, D = heads
    rng = np.random.default_rng(Hq + D)
    lens, starts = [1, 0, 37, 64, 5, 130], [0, 7, 31, 32, 95, 1]
    T, cu = sum(lens), offsets(lens)
    qkv, val = up(rng.standard_normal((T, Hq + 2 * Hk, D)) * np.exp(rng.standard_normal((1, 1, D))), dt)
    cos, sin = angles(300, D)
    pos = np.concatenate([s + np.arange(n) for s, n in zip(starts, lens)])
    table, pages = table_for([s + n for s, n in zip(starts, lens)], 64, rng)
    cache = tf.kv4_cache(pages, 64, Hk, D, dtype=DT[dt])
    q, k = tf.kv4_append(cache, table, i32(cu), i32(starts), qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:],
                         *([torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()] if turn else []),
                         q=qkv[:, :Hq], keys=True)
    rk, rv = tf.kv4_read(cache, table, i32(cu), i32(starts), T)
    turned = oracle.rotate(val[:, :Hq + Hk], cos[pos].astype(np.float64), sin[pos].astype(np.float64)) if turn else val
    for got, want in ((q, turned[:, :Hq]), (k, turned[:, Hq:Hq + Hk])):
        # two products and a sum in fp32
        big = np.abs(want) + 2 * np.abs(val).max(-1, keepdims=True)[:, :1]
        assert (np.abs(down(got) - want) <= U[dt] * np.abs(want) + 2.0 ** -22 * big + TINY[dt]).all()
    k32 = val[:, Hq:Hq + Hk].astype(np.float32)
    if turn:
        k32 = oracle.rotate(k32, cos[pos], sin[pos])
    for got, x in ((rk, k32), (rv, val[:, Hq + Hk:].astype(np.float32))):
        codes, s, z = oracle.quant_rows(x, dt)
        want = ((codes.astype(np.float32) - z.astype(np.float32)) * s.astype(np.float32)).astype(np.float64)
        np.testing.assert_array_equal(down(got), oracle.round16(want, dt))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_cached_rows_at_the_edges(tf, dt):
    """Constant rows, rows of one sign far from zero, tiny and huge ranges, and
    rows that are not finite."""
    D = 64
    rng = np.random.default_rng(3)
    big = 60000.0 if dt == "f16" else 3e38
    rows = [np.zeros(D), np.full(D, 3.25), np.full(D, -7.0), 100 + rng.random(D), -100 - rng.random(D),
            1e-6 * rng.standard_normal(D), np.where(rng.random(D) < 0.5, big, -big), np.r_[big, np.zeros(D - 1)],
            np.r_[np.nan, rng.standard_normal(D - 1)], np.r_[rng.standard_normal(D - 1), np.inf],
            np.r_[-np.inf, rng.standard_normal(D - 1)], 1e-38 * rng.standard_normal(D)]
    x, val = up(np.array(rows)[:, None], dt)
    T = len(rows)
    cache = tf.kv4_cache(1, 32, 1, D, dtype=DT[dt])
    args = (cache, i32([0]).view(1, 1), i32([0, T]), i32([0]))
    tf.kv4_append(*args, x, x)
    k, v = tf.kv4_read(*args, T)
    with np.errstate(all="ignore"):
        codes, s, z = oracle.quant_rows(val.astype(np.float32), dt)
        want = ((codes.astype(np.float32) - z.astype(np.float32)) * s.astype(np.float32)).astype(np.float64)
        want = oracle.round16(np.nan_to_num(want, nan=0.0, posinf=np.inf, neginf=-np.inf), dt)
    want[8:11] = np.nan
    np.testing.assert_array_equal(down(k), want)
    np.testing.assert_array_equal(down(v), want)


def test_append_out_of_place(tf):
    """Tokens past the angles, past the table or on no page: NaN rows or nothing
    cached, and the neighbours untouched."""
    D, Hk = 64, 2
    cache = tf.kv4_cache(2, 32, Hk, D)
    table = torch.tensor([[1, -1], [5, 0]], dtype=torch.int32).cuda()     # 5 is outside the pool
    x = torch.randn(100, Hk, D, device="cuda").half()
    cu, starts = i32([0, 50, 90]), i32([0, -3])                            # ten tokens that no sequence owns
    cos, sin = (torch.from_numpy(t).cuda() for t in angles(45, D))
    q, k = tf.kv4_append(cache, table, cu, starts, x, x, cos, sin, q=x, keys=True)
    bad = torch.zeros(100, dtype=torch.bool)
    bad[45:53], bad[90:] = True, True                                      # positions 45.. and below 0; unowned
    for t in (q, k):
        assert torch.equal(torch.isnan(t).all(-1).all(-1).cpu(), bad)
        assert torch.isfinite(t[~bad.cuda()]).all()
    rk, rv = tf.kv4_read(cache, table, cu, starts, 100)
    nowhere = bad.clone()
    nowhere[32:90] = True                                                  # no page; page 5
    nowhere[85:90] = False                                                 # positions 32..36 of sequence 1: page 0
    for t in (rk, rv):
        assert torch.equal(torch.isnan(t).all(-1).all(-1).cpu(), nowhere)


@pytest.mark.parametrize("heads", [(8, 64), (5, 128), (2, 256)], ids=str)
def test_reads_of_many_tokens_are_those_of_few(tf, heads):
    """4 M values and more are read tile by tile, fewer row by row: the same
    bits, from sequences that begin anywhere in a tile, empty ones, missing
    pages, positions below 0 and tokens that no sequence owns."""
    Hk, D = heads
    rng = np.random.default_rng(D)
    lens, starts = [4000, 0, 1, 37, 2500, 64, 90], [13, 5, 31, 32, 95, 0, -40]
    lens[0] += max(0, -(-(1 << 22) // (Hk * D)) - sum(lens))
    first, T = 3, sum(lens) + 3 + 45                    # unowned: 3 before the first, 45 behind the last
    table, pages = table_for([max(0, s + n) for s, n in zip(starts, lens)], 64, rng)
    table[0, 7], table[4, 1] = -1, pages                # missing; outside the pool
    cache = tf.kv4_cache(pages, 64, Hk, D)
    cu = i32(first + offsets(lens))
    k, v = (torch.randn(T, Hk, D, device="cuda").half() for _ in range(2))
    tf.kv4_append(cache, table, cu, i32(starts), k, v)
    assert T * Hk * D >= 1 << 22
    many = tf.kv4_read(cache, table, cu, i32(starts), T)
    few = [torch.full_like(t, float("nan")) for t in many]
    at = first
    for b, n in enumerate(lens):
        for i in range(0, n, 900):
            m = min(900, n - i)
            part = tf.kv4_read(cache, table[b:b + 1].contiguous(), i32([0, m]), i32([starts[b] + i]), m)
            for whole, piece in zip(few, part):
                whole[at + i:at + i + m] = piece
        at += n
    for a, b in zip(many, few):
        assert torch.equal(torch.isnan(a), torch.isnan(b))
        assert torch.equal(a.nan_to_num(), b.nan_to_num())
    # unowned; page 7 of sequence 0; the 33 positions from 95 on page 1 of sequence 4; below 0
    assert torch.isnan(many[0]).all(-1).all(-1).sum().item() == 3 + 45 + 64 + 33 + 40


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_append_and_read_of_many_sequences(tf, dt):
    """More sequences than a workgroup keeps the offsets of (1100)."""
    Hk, D = 2, 64
    rng = np.random.default_rng(11)
    lens, starts = rng.integers(0, 4, 1100).tolist(), rng.integers(0, 40, 1100).tolist()
    T, cu = sum(lens), offsets(lens)
    k, kv = up(rng.standard_normal((T, Hk, D)), dt)
    v, vv = up(rng.standard_normal((T, Hk, D)), dt)
    table, pages = table_for([s + n for s, n in zip(starts, lens)], 32, rng)
    cache = tf.kv4_cache(pages, 32, Hk, D, dtype=DT[dt])
    tf.kv4_append(cache, table, i32(cu), i32(starts), k, v)
    for got, x in zip(tf.kv4_read(cache, table, i32(cu), i32(starts), T), (kv, vv)):
        np.testing.assert_array_equal(down(got), oracle.round16(oracle.cached_rows(x.astype(np.float32), dt), dt))


# ---------------------------------------------------------------------------
# attention over the cache
# ---------------------------------------------------------------------------
def filled(tf, dt, heads, lens, page, seed, width=0):
    Hq, Hk, D = heads
    rng = np.random.default_rng(seed)
    T = int(sum(lens))
    k, kv = up(rng.standard_normal((T, Hk, D)) * np.exp(0.5 * rng.standard_normal((1, Hk, D))), dt)
    v, vv = up(rng.standard_normal((T, Hk, D)) + 0.5, dt)
    table, pages = table_for(lens, page, rng, width=width)
    cache = tf.kv4_cache(pages, page, Hk, D, dtype=DT[dt])
    cache.data.fill_(0xFF)                          # NaN scales wherever nothing is appended
    if T:
        tf.kv4_append(cache, table, i32(offsets(lens)), i32([0] * len(lens)), k, v)
    return cache, table, oracle.cached_rows(kv.astype(np.float32), dt), oracle.cached_rows(vv.astype(np.float32), dt), rng


def check_decode(dt, got, q, k, v, lens, heads, new, scale=None):
    """Per query: u for the output; 2 u sum p |v| for the rounded weights; the
    scores' fp32 error e (offset, zero-point and code products, 2^-22 of their
    size) as 2 e sum p |v|; the value offsets' 2^-24 of up to 1039 (fp16) or
    143 (bf16) code steps, over sums of up to 64 tiles a wave."""
    Hq, Hk, D = heads
    scale = D ** -0.5 if scale is None else scale
    off, cu, r = (1039 if dt == "f16" else 143), offsets(lens), Hq // Hk
    for b, n in enumerate(lens):
        for h in range(Hq):
            kb, vb = k[cu[b]:cu[b] + n, h // r], v[cu[b]:cu[b] + n, h // r]
            last = n - new + np.arange(new)
            want = oracle.attend(q[b, :, h], kb, vb, scale, last)
            bound = oracle.attend_bound(q[b, :, h], kb, vb, scale, last)
            step = (np.ptp(kb, -1).max() / 15, np.ptp(vb, -1).max() / 15) if n else (0, 0)
            e = 2.0 ** -22 * scale * np.abs(q[b, :, h]).sum(-1, keepdims=True) * step[0] * (off + 30)
            tol = U[dt] * np.abs(want) + (2 * U[dt] + 2 * e) * bound + 2.0 ** -21 * off * step[1] + TINY[dt]
            bad = ~(np.abs(got[b, :, h] - want) <= tol)      # NaN is bad too
            assert not bad.any(), (b, n, h, np.abs(got[b, :, h] - want).max(), tol.min())


DECODES = [((8, 2, 128), [1], 32, 1), ((8, 2, 128), [0, 1, 31, 32, 33, 129, 500], 32, 1),
           ((3, 3, 64), [5, 700, 64], 64, 1), ((8, 1, 256), [1000, 3], 128, 1),
           ((32, 8, 128), [127, 128, 2049], 64, 1), ((8, 2, 128), [2, 300, 0, 7], 96, 4),
           ((8, 1, 256), [77, 400], 64, 4), ((5, 1, 128), [260, 8], 64, 8), ((16, 1, 64), [90, 1], 32, 3),
           ((6, 6, 64), [350] * 70, 32, 1), ((2, 1, 128), [9000, 11], 256, 2)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,lens,page,new", DECODES, ids=str)
def test_decode(tf, dt, heads, lens, page, new):
    cache, table, k, v, rng = filled(tf, dt, heads, lens, page, len(lens) + new)
    q, qv = up(rng.standard_normal((len(lens), new, heads[0], heads[2])), dt)
    got = tf.kv4_attention(q, cache, table, i32(lens))
    check_decode(dt, down(got), qv, k, v, lens, heads, new)
    # the same from run to run, on the workspace that the first call left
    assert torch.equal(got, tf.kv4_attention(q, cache, table, i32(lens)))


# many items (512 and more: workgroups of four waves), of many sequences
MANY = [((6, 6, 64), 90, 1), ((8, 4, 128), 130, 1), ((16, 2, 128), 260, 4), ((8, 1, 256), 520, 1),
        ((8, 1, 256), 515, 4), ((16, 1, 64), 600, 2), ((5, 1, 128), 300, 8)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,batch,new", MANY, ids=str)
def test_decode_of_many_sequences(tf, dt, heads, batch, new):
    lens = np.random.default_rng(batch).integers(0, 120, batch).tolist()
    lens[1], lens[batch // 2], lens[-1] = 0, 1300, 200
    cache, table, k, v, rng = filled(tf, dt, heads, lens, 32, batch)
    q, qv = up(rng.standard_normal((batch, new, heads[0], heads[2])), dt)
    got = tf.kv4_attention(q, cache, table, i32(lens))
    check_decode(dt, down(got), qv, k, v, lens, heads, new)
    assert torch.equal(got, tf.kv4_attention(q, cache, table, i32(lens)))


# long sequences whose parts are added by a launch of their own
JOINED = [((8, 1, 256), [9000, 5], 4), ((16, 1, 64), [20000, 100], 2), ((16, 1, 128), [0, 9000, 40], 1),
          ((32, 2, 128), [300, 9000], 1), ((5, 1, 256), [12, 4000, 9000], 8),
          ((16, 1, 128), [40] * 300 + [6000] + [3] * 300, 1)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,lens,new", JOINED, ids=["256x4", "64x2", "128", "two heads", "40 rows", "many"])
def test_decode_of_long_sequences(tf, dt, heads, lens, new):
    cache, table, k, v, rng = filled(tf, dt, heads, lens, 64, len(lens) + new)
    q, qv = up(rng.standard_normal((len(lens), new, heads[0], heads[2])), dt)
    got = tf.kv4_attention(q, cache, table, i32(lens))
    check_decode(dt, down(got), qv, k, v, lens, heads, new)
    assert torch.equal(got, tf.kv4_attention(q, cache, table, i32(lens)))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_decode_strided_queries_scale_and_sharp_softmax(tf, dt):
    """Queries as a part of a wider projection, a scale of the caller's, and
    scores so far apart that one key takes nearly everything."""
    heads, lens = (8, 2, 128), [333, 90]
    cache, table, k, v, rng = filled(tf, dt, heads, lens, 64, 9)
    wide, wv = up(4 * rng.standard_normal((2, 12, 128)), dt)
    got = tf.kv4_attention(wide[:, :8], cache, table, i32(lens), scale=0.7)
    check_decode(dt, down(got)[:, None], wv[:, None, :8], k, v, lens, heads, 1, 0.7)


@pytest.mark.parametrize("new", [1, 4])
def test_decode_sees_nothing_of_what_is_hidden(tf, new):
    """Rows that are not finite behind a query's last position, pages missing
    from the table, and lengths beyond it."""
    heads, lens, page = (4, 2, 64), [40, 70], 32
    cache, table, k, v, rng = filled(tf, "f16", heads, lens, page, 21, width=4)
    q, qv = up(rng.standard_normal((2, new, 4, 64)), "f16")
    want = tf.kv4_attention(q, cache, table, i32(lens))
    # three positions appended beyond the lengths, not finite
    bad = torch.full((6, 2, 64), float("nan"), device="cuda").half()
    tf.kv4_append(cache, table, i32([0, 3, 6]), i32(lens), bad, bad)
    assert torch.equal(tf.kv4_attention(q, cache, table, i32(lens)), want)
    if new > 1:                                     # the last position is seen by the last query alone
        one = torch.full((2, 2, 64), float("nan"), device="cuda").half()
        tf.kv4_append(cache, table, i32([0, 1, 2]), i32([n - 1 for n in lens]), one, one)
        got = tf.kv4_attention(q, cache, table, i32(lens))
        assert torch.equal(got[:, :-1], want[:, :-1]) and torch.isnan(got[:, -1]).all()
        return
    gone = table.clone()
    gone[1, 0] = -1                                 # positions 0..31 of sequence 1 leave
    got = tf.kv4_attention(q, cache, gone, i32(lens))
    assert torch.equal(got[0], want[0])
    check_decode("f16", down(got[1:]), qv[1:], k[40 + 32:], v[40 + 32:], [38], heads, 1)
    gone[1] = 99
    assert (tf.kv4_attention(q, cache, gone, i32(lens))[1] == 0).all()
    # lengths past the table's width, or negative
    full = tf.kv4_attention(q, cache, table[:, :1].contiguous(), i32([32, -5]))
    assert torch.equal(tf.kv4_attention(q, cache, table[:, :1].contiguous(), i32([10 ** 9, 0]))[0], full[0])
    assert (full[1] == 0).all()


def test_decode_pool_beyond_32_bits(tf):
    """Pages whose byte offsets pass 2^32 (a pool of 4.6 GiB)."""
    heads, page = (8, 8, 128), 256
    per_page = tf.kv4_cache_bytes(1, page, 8, 128)
    pages = int(4.6 * 2 ** 30) // per_page
    cache = tf.kv4_cache(pages, page, 8, 128)
    rng = np.random.default_rng(1)
    k, kv = up(rng.standard_normal((600, 8, 128)), "f16")
    v, vv = up(rng.standard_normal((600, 8, 128)), "f16")
    table = i32([pages - 1, 3, pages - 2]).view(1, 3)
    tf.kv4_append(cache, table, i32([0, 600]), i32([0]), k, v)
    q, qv = up(rng.standard_normal((1, 1, 8, 128)), "f16")
    got = tf.kv4_attention(q, cache, table, i32([600]))
    check_decode("f16", down(got), qv, oracle.cached_rows(kv.astype(np.float32), "f16"),
                 oracle.cached_rows(vv.astype(np.float32), "f16"), [600], heads, 1)


def test_decode_after_many_tokens_one_by_one(tf):
    """Tokens appended one at a time give the cache that one append gives."""
    heads, D = (4, 2, 64), 64
    rng = np.random.default_rng(2)
    k, _ = up(rng.standard_normal((75, 2, D)), "bf16")
    v, _ = up(rng.standard_normal((75, 2, D)), "bf16")
    table = i32([2, 0, 1]).view(1, 3)
    one, all_ = (tf.kv4_cache(3, 32, 2, D, dtype=torch.bfloat16) for _ in range(2))
    tf.kv4_append(all_, table, i32([0, 75]), i32([0]), k, v)
    for i in range(75):
        tf.kv4_append(one, table, i32([0, 1]), i32([i]), k[i:i + 1], v[i:i + 1])
    a = (i32([0, 75]), i32([0]), 75)
    for x, y in zip(tf.kv4_read(one, table, *a), tf.kv4_read(all_, table, *a)):
        assert torch.equal(x, y)


# ---------------------------------------------------------------------------
# attention over prompts
# ---------------------------------------------------------------------------
def check_prompt(dt, got, q, k, v, n_q, n_k, causal=True, scale=None):
    """Per query: u for the output, u sum p |v| for the rounded weights (fp16:
    those under 2^-14 of the largest lose at most 2^-25 each), and the scores'
    fp32 error e = 2^-21 scale |q| |k| as 2 e sum p |v|."""
    Hq, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    scale = D ** -0.5 if scale is None else scale
    cq, ck = offsets(n_q), offsets(n_k)
    for b in range(len(n_q)):
        for h in range(Hq):
            qb = q[cq[b]:cq[b + 1], h]
            kb, vb = (t[ck[b]:ck[b + 1], h * Hk // Hq] for t in (k, v))
            last = n_k[b] - n_q[b] + np.arange(n_q[b]) if causal else np.full(n_q[b], n_k[b])
            want = oracle.attend(qb, kb, vb, scale, last)
            bound = oracle.attend_bound(qb, kb, vb, scale, last)
            e = 2.0 ** -21 * scale * (np.abs(qb).sum(-1, keepdims=True) * np.abs(kb).max() if kb.size else 0)
            small = TINY[dt] * n_k[b] * (np.abs(vb).max() if vb.size else 0)
            tol = U[dt] * np.abs(want) + (U[dt] + 2 * e + 2.0 ** -20) * bound + small + TINY[dt]
            bad = ~(np.abs(got[cq[b]:cq[b + 1], h] - want) <= tol)      # NaN is bad too
            assert not bad.any(), (b, h, np.abs(got[cq[b]:cq[b + 1], h] - want).max())


PROMPTS = [((8, 2, 128), [1], [1]), ((8, 2, 128), [0, 1, 31, 64, 65, 129, 200], None), ((3, 3, 64), [300, 17], None),
           ((4, 1, 256), [130, 3], None), ((8, 2, 128), [5, 100, 1], [500, 163, 70]),
           ((5, 1, 128), [100, 40, 6, 2], [30, 40, 0, 1]), ((2, 2, 64), [257], [321]), ((4, 4, 256), [33, 140], [97, 141])]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("heads,n_q,n_k", PROMPTS, ids=str)
def test_prompt(tf, dt, causal, heads, n_q, n_k):
    """Packed lengths of 0, 1 and across tile edges; prompts that follow earlier
    keys; more queries than keys (rows that see nothing give zeros)."""
    Hq, Hk, D = heads
    n_k = n_q if n_k is None else n_k
    rng = np.random.default_rng(sum(n_q) + D)
    q, qv = up(rng.standard_normal((sum(n_q), Hq, D)), dt)
    k, kv = up(rng.standard_normal((sum(n_k), Hk, D)) * np.exp(0.5 * rng.standard_normal((1, Hk, D))), dt)
    v, vv = up(rng.standard_normal((sum(n_k), Hk, D)) + 0.5, dt)
    got = tf.prompt_attention(q, k, v, i32(offsets(n_q)), i32(offsets(n_k)), causal=causal)
    check_prompt(dt, down(got), qv, kv, vv, n_q, n_k, causal)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_prompt_of_many_sequences(tf, dt):
    """More sequences than a workgroup has threads."""
    heads = Hq, Hk, D = (2, 1, 64)
    rng = np.random.default_rng(6)
    n_q = rng.integers(0, 9, 700).tolist()
    n_q[350] = 200
    n_k = [n + int(p) for n, p in zip(n_q, rng.integers(0, 20, 700))]
    q, qv = up(rng.standard_normal((sum(n_q), Hq, D)), dt)
    k, kv = up(rng.standard_normal((sum(n_k), Hk, D)), dt)
    v, vv = up(rng.standard_normal((sum(n_k), Hk, D)) + 0.5, dt)
    got = tf.prompt_attention(q, k, v, i32(offsets(n_q)), i32(offsets(n_k)))
    check_prompt(dt, down(got), qv, kv, vv, n_q, n_k)


SPLITS = [((4, 1, 128), [70], [3000]), ((2, 2, 64), [1], [2049]), ((2, 1, 256), [40, 0, 129], [5000, 7, 1300]),
          ((3, 3, 64), [200, 33], [190, 4200]), ((8, 1, 256), [500], [3500])]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("heads,n_q,n_k", SPLITS, ids=str)
def test_prompt_split_over_keys(tf, dt, causal, heads, n_q, n_k):
    """Few queries on many keys: the keys in parts, with and without a workspace."""
    Hq, Hk, D = heads
    assert tf.prompt_attention_workspace_bytes(len(n_q), sum(n_q), sum(n_k), Hq, Hk, D) > 0
    rng = np.random.default_rng(sum(n_q) + D)
    q, qv = up(rng.standard_normal((sum(n_q), Hq, D)), dt)
    k, kv = up(rng.standard_normal((sum(n_k), Hk, D)) * np.exp(0.5 * rng.standard_normal((1, Hk, D))), dt)
    v, vv = up(rng.standard_normal((sum(n_k), Hk, D)) + 0.5, dt)
    args = (q, k, v, i32(offsets(n_q)), i32(offsets(n_k)))
    got = tf.prompt_attention(*args, causal=causal)
    check_prompt(dt, down(got), qv, kv, vv, n_q, n_k, causal)
    assert torch.equal(got, tf.prompt_attention(*args, causal=causal))
    check_prompt(dt, down(tf.prompt_attention(*args, causal=causal, workspace=False)), qv, kv, vv, n_q, n_k, causal)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_prompt_strided_scale_and_sharp_softmax(tf, dt):
    """Parts of one projection as they are, a scale of the caller's, scores far apart."""
    rng = np.random.default_rng(4)
    qkv, val = up(4 * rng.standard_normal((190, 12, 128)), dt)
    got = tf.prompt_attention(qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], i32([0, 90, 190]), scale=0.3)
    check_prompt(dt, down(got), val[:, :8], val[:, 8:10], val[:, 10:], [90, 100], [90, 100], True, 0.3)


def test_prompt_hidden_keys_do_not_act(tf):
    """Keys and values behind a query's last key may be NaN or inf."""
    q, k, v = (torch.randn(150, 4, 128, device="cuda").half() for _ in range(3))
    cu = i32([0, 150])
    want = tf.prompt_attention(q, k, v, cu)
    k[149], v[148] = float("nan"), float("inf")
    got = tf.prompt_attention(q, k, v, cu)
    assert torch.equal(got[:128], want[:128])
    finite = tf.prompt_attention(q[:148].contiguous(), k[:148].contiguous(), v[:148].contiguous(), i32([0, 148]))
    assert torch.isfinite(finite).all()
    assert not torch.isfinite(got[148:]).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,n_q,n_k", [((4, 2, 64), [97, 150], [97, 190]), ((4, 4, 128), [150], [150]),
                                           ((4, 1, 128), [70, 9], [3000, 300]), ((2, 1, 256), [200, 3], [140, 3])],
                         ids=["64", "128", "128 after earlier keys", "256, more queries than keys"])
def test_prompt_values_that_are_not_finite_act_where_seen(tf, dt, heads, n_q, n_k):
    """A value that is not finite changes its dim of the queries that see it and
    nothing else, wherever its tile is shared with queries that do not; a key
    of NaN changes the queries that see it alone (the others' sums may move to a
    new maximum at another step: two results, each within u |o| + u sum p |v| and
    a fifth of that of fp32 error, so 5 u max |v| apart at most)."""
    Hq, Hk, D = heads
    q, k, v = (torch.randn(sum(n), h, D, device="cuda").to(DT[dt])
               for n, h in ((n_q, Hq), (n_k, Hk), (n_k, Hk)))
    cq, ck = offsets(n_q), offsets(n_k)
    for causal in (True, False):
        args = (i32(cq), i32(ck))
        want = tf.prompt_attention(q, k, v, *args, causal=causal)
        assert torch.isfinite(want).all()
        for b in range(len(n_q)):
            for back, bad in ((1, float("inf")), (2, float("-inf")), (33, float("nan")), (66, float("nan")),
                              (90, float("inf"))):
                j = n_k[b] - back
                if j < 0:
                    continue
                sees = torch.zeros(sum(n_q), dtype=torch.bool, device="cuda")
                i0 = max(0, j - (n_k[b] - n_q[b])) if causal else 0
                sees[cq[b] + i0:cq[b + 1]] = True
                w, h, d = v.clone(), back % Hk, (7 * back) % D
                w[ck[b] + j, h, d] = bad
                heads_of = slice(h * Hq // Hk, (h + 1) * Hq // Hk)
                got = tf.prompt_attention(q, k, w, *args, causal=causal)
                hit = got[sees][:, heads_of, d]
                assert (torch.isnan(hit) if bad != bad else hit == bad).all(), (b, back, causal)
                got[cq[b] + i0:cq[b + 1], heads_of, d] = want[cq[b] + i0:cq[b + 1], heads_of, d]
                # a tile's other values are those it had, to the bit
                assert torch.equal(got, want), (b, back, causal)
                w = k.clone()
                w[ck[b] + j, h, d] = float("nan")
                got = tf.prompt_attention(q, w, v, *args, causal=causal)
                assert torch.isnan(got[sees][:, heads_of]).all()
                got[cq[b] + i0:cq[b + 1], heads_of] = want[cq[b] + i0:cq[b + 1], heads_of]
                apart = (got.double() - want.double()).abs().max()
                assert apart <= 5 * U[dt] * v.abs().max().double(), (b, back, causal)


def test_prompt_offsets_that_do_not_fit(tf):
    """Sequences whose offsets leave the tensors or run backwards are left out."""
    q, k, v = (torch.randn(64, 2, 64, device="cuda").half() for _ in range(3))
    out = torch.full((64, 2, 64), 7.0, device="cuda").half()
    tf.prompt_attention(q, k, v, i32([0, 20, 10, 500]), out=out)
    want = tf.prompt_attention(q[:20].contiguous(), k[:20].contiguous(), v[:20].contiguous(), i32([0, 20]))
    assert torch.equal(out[:20], want) and (out[20:] == 7).all()


# ---------------------------------------------------------------------------
# graphs and streams
# ---------------------------------------------------------------------------
def test_graph_replays_match_eager(tf):
    """A decode step of all four operators captured and replayed, with eager
    work between the replays."""
    heads, lens = (8, 2, 128), [700, 33, 260]
    Hq, Hk, D = heads
    cache, table, *_ = filled(tf, "bf16", heads, lens, 64, 31, width=13)
    x = torch.randn(3, (Hq + 2 * Hk) * D, device="cuda").bfloat16()
    w = torch.ones(x.shape[1], device="cuda").bfloat16()
    cos, sin = (torch.from_numpy(t).cuda() for t in angles(1000, D))
    cu, starts, after = i32(range(4)), i32(lens), i32([n + 1 for n in lens])
    ws = torch.zeros(tf.kv4_attention_workspace_bytes(3, 1, Hq, Hk, D), dtype=torch.uint8, device="cuda")
    bufs = {n: torch.empty(3, h, D, dtype=x.dtype, device="cuda") for n, h in (("q", Hq), ("o", Hq), ("p", Hq))}
    normed = torch.empty_like(x)

    def step():
        tf.add_rms_norm(x, weight=w, out=normed)
        y = normed.view(3, Hq + 2 * Hk, D)
        tf.kv4_append(cache, table, cu, starts, y[:, Hq:Hq + Hk], y[:, Hq + Hk:], cos, sin, q=y[:, :Hq],
                      q_out=bufs["q"])
        tf.kv4_attention(bufs["q"], cache, table, after, out=bufs["o"], workspace=ws)
        tf.prompt_attention(bufs["q"], y[:, Hq:Hq + Hk], y[:, Hq + Hk:], cu, out=bufs["p"])

    step()
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in bufs.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for t in bufs.values():
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for n, t in bufs.items():
            assert torch.equal(t, want[n]), n


def test_another_stream(tf):
    """Calls go to the current stream; each stream with a workspace of its own."""
    heads, lens = (8, 2, 128), [900, 90]
    cache, table, *_ = filled(tf, "f16", heads, lens, 64, 8)
    q = torch.randn(2, 8, 128, device="cuda").half()
    want = tf.kv4_attention(q, cache, table, i32(lens))
    s = torch.cuda.Stream()
    ws = torch.zeros(tf.kv4_attention_workspace_bytes(2, 1, 8, 2, 128), dtype=torch.uint8, device="cuda")
    n = i32(lens)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = tf.kv4_attention(q * 1, cache, table, n, workspace=ws)
    s.synchronize()
    assert torch.equal(got, want)


def test_native_and_general_paths_agree(tf, monkeypatch):
    """The native module's calls and the general paths that stand behind them."""
    heads, lens = (8, 2, 128), [300, 41]
    cache, table, *_ = filled(tf, "bf16", heads, lens, 64, 12, width=6)
    x = torch.randn(2, 12, 128, device="cuda").bfloat16()
    w = torch.randn(1536, device="cuda").bfloat16()
    cos, sin = (torch.from_numpy(t).cuda() for t in angles(400, 128))
    cu, starts, after = i32(range(3)), i32(lens), i32([n + 1 for n in lens])
    flat = x.view(2, 1536)

    def all_calls():
        return [*tf.add_rms_norm(flat, flat, w), *tf.add_rms_norm(flat, None, w, gate=flat, scale=2),
                *tf.kv4_append(cache, table, cu, starts, x[:, 8:10], x[:, 10:], cos, sin, q=x[:, :8], keys=True),
                *tf.kv4_read(cache, table, cu, starts, 2), tf.kv4_attention(x[:, :8], cache, table, after, scale=0.1),
                tf.prompt_attention(x[:, :8], x[:, 8:10], x[:, 10:], cu)]

    assert tf._native_ops()["norm"](flat, flat, w, None, None, 1.0, 0.0, 1e-6, None, None) is not NotImplemented
    native = all_calls()
    monkeypatch.setattr(tf, "_ops", dict.fromkeys(("norm", "append", "read", "decode", "prompt"),
                                                  lambda *call: NotImplemented))
    for a, b in zip(native, all_calls()):
        assert torch.equal(a, b)


def test_refusals(tf):
    """What the binding and the library refuse, on either path."""
    x = torch.zeros(4, 64, device="cuda").half()
    with pytest.raises(ValueError):
        tf.add_rms_norm(x, x.bfloat16(), x[0])
    with pytest.raises(ValueError):
        tf.add_rms_norm(x, x[:2], x[0])
    with pytest.raises(ValueError):
        tf.add_rms_norm(x.float())
    with pytest.raises(tf.TileFuseError) as e:
        tf.add_rms_norm(x[:, :60].contiguous(), weight=x[0, :60].contiguous())
    assert e.value.status == tf.TF_ERR_SHAPE
    cache = tf.kv4_cache(2, 32, 1, 64)
    table, cu, starts = i32([0, 1]).view(1, 2), i32([0, 4]), i32([0])
    kv = torch.zeros(4, 1, 64, device="cuda").half()
    for bad in (dict(k=kv.bfloat16()), dict(k=kv[:3]), dict(cu=i32([0, 2, 4])), dict(starts=starts.long()),
                dict(table=table.view(2, 1)), dict(cos=torch.zeros(9, 32, device="cuda")), dict(k=kv.cpu()),
                dict(k=torch.zeros(4, 1, 128, device="cuda").half()[:, :, ::2])):
        a = dict(table=table, cu=cu, starts=starts, k=kv, v=kv) | bad
        with pytest.raises(ValueError):
            tf.kv4_append(cache, **a)
    with pytest.raises(ValueError):
        tf.kv4_attention(kv[:, :, :32], cache, table, starts)
    q = torch.zeros(1, 9, 1, 64, device="cuda").half()
    with pytest.raises(tf.TileFuseError) as e:
        tf.kv4_attention(q, cache, table, starts)                  # nine tokens
    assert e.value.status == tf.TF_ERR_ARG
    with pytest.raises(tf.TileFuseError) as e:
        tf.kv4_attention(kv[:1], cache, table, starts, scale=0.0)
    assert e.value.status == tf.TF_ERR_ARG
    with pytest.raises(tf.TileFuseError) as e:
        tf.kv4_attention(kv[:1], cache, table, starts, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == tf.TF_ERR_ARG
    with pytest.raises(ValueError):
        tf.prompt_attention(kv, kv, kv.bfloat16(), cu)
    with pytest.raises(tf.TileFuseError) as e:
        tf.prompt_attention(kv.expand(4, 3, 64).contiguous(), kv.expand(4, 2, 64).contiguous(),
                            kv.expand(4, 2, 64).contiguous(), cu)
    assert e.value.status == tf.TF_ERR_SHAPE
    with pytest.raises(tf.TileFuseError):
        tf.kv4_cache(2, 48, 1, 64)


def test_nothing_to_do(tf):
    """Calls without tokens return empty tensors."""
    e = torch.empty(0, 2, 64, device="cuda").half()
    cache = tf.kv4_cache(1, 32, 2, 64)
    table = i32([0]).view(1, 1)
    y, r = tf.add_rms_norm(torch.empty(0, 64, device="cuda").half(), None, torch.ones(64, device="cuda").half())
    assert y.shape == (0, 64)
    q, k = tf.kv4_append(cache, table, i32([0, 0]), i32([0]), e, e, q=e, keys=True)
    assert q.shape == k.shape == (0, 2, 64)
    assert tf.kv4_read(cache, table, i32([0, 0]), i32([0]), 0)[0].shape == (0, 2, 64)
    assert tf.prompt_attention(e, e, e, i32([0, 0])).shape == (0, 2, 64)
    q = torch.randn(3, 2, 64, device="cuda").half()
    assert (tf.prompt_attention(q, e, e, i32([0, 3]), i32([0, 0])) == 0).all()
