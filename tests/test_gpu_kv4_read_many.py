"""Reads of many short sequences."""
from __future__ import annotations

import pytest

from test_gpu_decoder_ops import i32, tf  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_read_of_one_token_of_many_sequences_and_heads(tf):
    """65536 sequences of one token, 260 heads: workgroups for a tile of each would be
    more than a launch has.  All without a page (NaN) but two."""
    H, D, B, at = 260, 64, 65536, (5, 65535)
    cache = tf.kv4_cache(2, 32, H, D, dtype=torch.bfloat16)
    kv = torch.randn(2, H, D, device="cuda").bfloat16()
    two, starts = i32([0, 1]).view(2, 1), i32([0, 31])
    tf.kv4_append(cache, two, i32([0, 1, 2]), starts, kv, 2 * kv)
    want = tf.kv4_read(cache, two, i32([0, 1, 2]), starts, 2)
    table, all_starts = torch.full((B, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    for i, b in enumerate(at):
        table[b], all_starts[b] = i, starts[i]
    cu = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    for got, w in zip(tf.kv4_read(cache, table, cu, all_starts, B), want):
        assert torch.equal(got[list(at)], w)
        missing = 0
        for part in got.split(8192):
            missing += int(torch.isnan(part).all(-1).sum())
        assert missing == (B - 2) * H


@pytest.mark.parametrize("tokens,batch", [(64, 64), (65, 1024), (3, 2000), (1, 5000), (130, 40)], ids=str)
def test_reads_around_the_choice_of_kernel(tf, tokens, batch):
    """The same bits as reads of a few sequences at a time."""
    H, D = 8, 128
    per = -(-(tokens + 31) // 32)
    cache = tf.kv4_cache(batch * per, 32, H, D, dtype=torch.float16)
    table = torch.randperm(batch * per, device="cuda").to(torch.int32).view(batch, per)
    starts = torch.arange(batch, device="cuda", dtype=torch.int32) * 7 % 32
    cu = torch.arange(batch + 1, device="cuda", dtype=torch.int32) * tokens
    kv = torch.randn(batch * tokens, H, D, device="cuda").half()
    tf.kv4_append(cache, table, cu, starts, kv, 3 * kv)
    got = tf.kv4_read(cache, table, cu, starts, batch * tokens)
    few = 3
    for b in range(0, batch, max(few, batch // 16)):
        n = min(few, batch - b)
        part = tf.kv4_read(cache, table[b:b + n], cu[:n + 1], starts[b:b + n], n * tokens)
        for g, p in zip(got, part):
            assert torch.equal(g[b * tokens:(b + n) * tokens], p)
