"""Sizes of a cache that pass their limits one by one and 64 bits together."""
from __future__ import annotations

import pytest

from paper_2606_11357_amd import tilefuse as tfb


@pytest.mark.parametrize("pages,page_size,kv_heads,head_dim", [
    (1041204194, 65536, 1024, 256),            # 2^64 bytes and 18 GB
    (2 ** 31 - 1, 65536, 1024, 256), (2 ** 31 - 1, 65536, 1024, 128), (2 ** 31 - 1, 65504, 600, 256)], ids=str)
def test_pool_beyond_64_bits(pages, page_size, kv_heads, head_dim):
    per_page = kv_heads * (page_size // 32) * (32 * head_dim + 256)
    assert pages * per_page > 2 ** 63
    assert tfb.load().tf_kv4_cache_bytes(pages, page_size, kv_heads, head_dim) == tfb.TF_ERR_SHAPE
    most = (2 ** 63 - 1) // per_page
    assert tfb.load().tf_kv4_cache_bytes(most, page_size, kv_heads, head_dim) == most * per_page
