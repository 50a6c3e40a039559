"""Forms of the attention calls' arguments, on the native and the general path."""
from __future__ import annotations

import pytest

from test_gpu_decoder_ops import filled, i32, tf  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "general"])
def path(request, tf, monkeypatch):
    if request.param == "general":
        monkeypatch.setattr(tf, "_ops", dict.fromkeys(("norm", "append", "read", "decode", "prompt"),
                                                      lambda *call: NotImplemented))


@pytest.mark.parametrize("lens", [[70, 33, 5], [40]], ids=str)
def test_decode_of_one_token_with_an_axis_of_its_own(tf, path, lens):
    """[batch, 1, heads, D] of a wider projection, whose token axis may have any
    stride."""
    B = len(lens)
    cache, table, *_ = filled(tf, "bf16", (8, 2, 128), lens, 32, 3)
    wide = torch.randn(B, 12, 128, device="cuda").bfloat16()
    q = wide[:, :8]
    want = tf.kv4_attention(q.contiguous(), cache, table, i32(lens))
    for form in (q.unsqueeze(1), wide[:, None][:, :, :8], q.as_strided((B, 1, 8, 128), (12 * 128, 8, 128, 1))):
        got = tf.kv4_attention(form, cache, table, i32(lens))
        assert got.shape == (B, 1, 8, 128) and torch.equal(got[:, 0], want)


def test_prompt_without_keys(tf, path):
    """Zeros in the rows that a sequence owns, the others as they were; the refusals of
    any other call."""
    q, none = torch.randn(7, 4, 64, device="cuda").half(), torch.empty(0, 2, 64, device="cuda").half()
    out = torch.full_like(q, 3.0)
    assert tf.prompt_attention(q, none, none, i32([0, 2, 5]), i32([0, 0, 0]), out=out) is out
    assert (out[:5] == 0).all() and (out[5:] == 3).all()
    with pytest.raises(tf.TileFuseError) as e:
        tf.prompt_attention(q, none, none, i32([0, 2, 5]), i32([0, 0, 0]), scale=-1.0)
    assert e.value.status == tf.TF_ERR_ARG


def test_decode_without_a_workspace_is_refused(tf, path):
    cache, table, *_ = filled(tf, "f16", (4, 2, 64), [40], 32, 1)
    with pytest.raises(ValueError, match="workspace"):
        tf.kv4_attention(torch.zeros(1, 4, 64, device="cuda").half(), cache, table, i32([40]), workspace=False)


def test_no_keys_of_any_stride(tf, path):
    """A tensor without elements is contiguous whatever its strides are."""
    q, none = torch.randn(3, 4, 64, device="cuda").half(), torch.empty_strided((0, 2, 64), (1, 1, 1), device="cuda").half()
    none = none.as_strided((0, 2, 64), (7, 3, 5))
    assert none.is_contiguous()
    assert (tf.prompt_attention(q, none, none, i32([0, 3]), i32([0, 0])) == 0).all()
    cache = tf.kv4_cache(1, 32, 2, 64)
    assert tf.kv4_append(cache, i32([0]).view(1, 1), i32([0, 0]), i32([0]), none, none, keys=True)[1].shape == (0, 2, 64)
