"""8-bit products whose operands reach past 2^32 bytes: the same bits as calls on the
far parts alone."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_11357_amd import tilefuse
    tilefuse.load()
    return tilefuse


def ints(*shape):
    return torch.randint(-128, 128, shape, dtype=torch.int8, device="cuda")


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def test_many_rows(tf):
    """Codes of 4.3 GB, dense and by expert without rows."""
    M, K, N = 66000, 65536, 16
    q, s = ints(M, K), torch.rand(M, device="cuda") * 1e-6
    w, ws = ints(2, K, N), torch.rand(2, N, device="cuda")
    packed, one = tf.pack_w8a8(w, ws), tf.pack_w8a8(w[1].contiguous(), ws[1])
    far = tf.w8a8_gemm(q[-300:], s[-300:], one, K, N, dtype=torch.bfloat16)
    assert torch.equal(tf.w8a8_gemm(q, s, one, K, N, dtype=torch.bfloat16)[-300:], far)
    by = tf.w8a8_expert_gemm(q, s, packed, K, N, i32([0, M - 300, M]), dtype=torch.bfloat16)
    assert torch.equal(by[-300:], far)
    # few rows of each expert: the direct kernel
    assert torch.equal(tf.w8a8_expert_gemm(q[-8:], s[-8:], packed, K, N, i32([0, 0, 8]), dtype=torch.bfloat16), far[-8:])


def test_gathered_rows_up_to_the_limit(tf):
    """Rows at 4.29 GB of the codes; more than a gather's offsets hold is refused."""
    A, K, N = 65535, 65520, 24
    q, s = ints(A, K), torch.rand(A, device="cuda") * 1e-6
    packed = tf.pack_w8a8(ints(1, K, N), torch.rand(1, N, device="cuda"))
    last = torch.arange(A - 400, A, dtype=torch.int32, device="cuda").flip(0)
    for n in (5, 60, 400):
        got = tf.w8a8_expert_gemm(q, s, packed, K, N, i32([0, n]), last[:n].contiguous(), dtype=torch.bfloat16)
        mine = last[:n].long()
        assert torch.equal(got, tf.w8a8_gemm(q[mine], s[mine], packed, K, N, dtype=torch.bfloat16)), n
    big = torch.empty(65537, 65536, dtype=torch.int8, device="cuda")
    with pytest.raises(tf.TileFuseError) as err:
        tf.w8a8_expert_gemm(big, torch.empty(65537, device="cuda"), tf.pack_w8a8(ints(1, 65536, 8), torch.ones(1, 8, device="cuda")),
                            65536, 8, i32([0, 1]), i32([0]))
    assert err.value.status == tf.TF_ERR_SHAPE


@pytest.mark.parametrize("rows", [3, 200])
def test_weights_of_many_experts(tf, rows):
    """Packed weights of 4.7 GB: the last expert's."""
    E, K, N = 20, 14336, 16384
    q, s = ints(rows, K), torch.rand(rows, device="cuda") * 1e-6
    w, ws = ints(E, K, N), torch.rand(E, N, device="cuda")
    packed = tf.pack_w8a8(w, ws)
    last = tf.pack_w8a8(w[-1].contiguous(), ws[-1])
    assert torch.equal(packed[-last.numel():], last)
    got = tf.w8a8_expert_gemm(q, s, packed, K, N, i32([0] * E + [rows]), dtype=torch.bfloat16)
    assert torch.equal(got, tf.w8a8_gemm(q, s, last, K, N, dtype=torch.bfloat16))


def test_large_outputs(tf):
    """An output of 4.3 GB, its last rows."""
    M, K, N = 131200, 16, 16384
    q, s = ints(M, K), torch.rand(M, device="cuda") * 1e-3
    packed = tf.pack_w8a8(ints(K, N), torch.rand(N, device="cuda"))
    out = tf.w8a8_gemm(q, s, packed, K, N, dtype=torch.bfloat16)
    for part in (slice(0, 40), slice(65530, 65600), slice(M - 70, M)):
        assert torch.equal(out[part], tf.w8a8_gemm(q[part], s[part], packed, K, N, dtype=torch.bfloat16))
    sums = tf.combine_experts(out, torch.full((2, 1), 0.5, device="cuda"), i32([[M - 1], [0]]))
    assert torch.equal(sums, (out[[M - 1, 0]].float() * 0.5).bfloat16())
