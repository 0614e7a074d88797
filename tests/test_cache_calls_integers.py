"""Host integers of the calls on shared and bounded caches (no GPU is touched):
what does not fit the C ABI's 32 bits is refused, not taken by its low bits
(num_recent = 2^32 would keep no recent key, max_context_len = 2^32 + 500 cut
every context to 500)."""

import pytest
import torch

from paper_2607_13095_amd import hswa

FAR = ((1 << 31), (1 << 32) + 32, -(1 << 32) + 1, -(1 << 31) - 1)


def _cache(ns=2, pages=4, hkv=2, pg=16):
    return hswa.Cache(torch.zeros(hswa.k_pool_shape(pages, hkv, pg), dtype=torch.bfloat16),
                      torch.zeros(hswa.v_pool_shape(pages, hkv, pg), dtype=torch.bfloat16),
                      torch.zeros((ns, 2), dtype=torch.int32))


@pytest.mark.parametrize("n", FAR)
def test_sizes(n):
    sh = hswa.Shape(64, 8)
    for args in ((n, 1, 500), (2, n, 500), (2, 1, n)):
        with pytest.raises(ValueError, match="32 bits"):
            hswa.decode_scored_workspace_bytes(sh, *args)
    for args in ((n, 1, 500, 1, 100), (2, n, 500, 1, 100), (2, 1, n, 1, 100), (2, 1, 500, n, 100), (2, 1, 500, 1, n)):
        with pytest.raises(ValueError, match="32 bits"):
            hswa.decode_shared_workspace_bytes(sh, *args)


@pytest.mark.parametrize("n", FAR)
def test_calls(n):
    shape, cache, dst, layer = hswa.Shape(4, 2, 128, 16), _cache(), _cache(), hswa.Layer.full()
    q, i = torch.zeros((2, 4, 128), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    s, kept = torch.zeros((2, 2, 32)), torch.zeros((2, 2, 8), dtype=torch.int32)
    with pytest.raises(ValueError, match="max_context_len.*32 bits"):
        hswa.decode_shared(layer, shape, cache, q, i, n, i, i[:1], 16, q)
    with pytest.raises(ValueError, match="max_shared_len.*32 bits"):
        hswa.decode_shared(layer, shape, cache, q, i, 32, i, i[:1], n, q)
    with pytest.raises(ValueError, match="max_context_len.*32 bits"):
        hswa.decode_scored(layer, shape, cache, q, i, n, None, s, q)
    with pytest.raises(ValueError, match="max_context_len.*32 bits"):
        hswa.kv_evict(layer, shape, cache, dst, s, i, i, n, kept, i)
    with pytest.raises(ValueError, match="num_recent.*32 bits"):
        hswa.kv_evict(layer, shape, cache, dst, s, i, i, 32, kept, i, num_recent=n)
    with pytest.raises(ValueError, match="num_sinks.*32 bits"):
        hswa.kv_evict(layer, shape, cache, dst, s, i, i, 32, kept, i, num_sinks=n)


def test_rows_of_scores():
    """Rows of 2^31 positions and more (tensors without storage stand for them)."""
    shape, cache, dst, layer = hswa.Shape(2, 1, 128, 16), _cache(1, hkv=1), _cache(1, hkv=1), hswa.Layer.full()
    q, i = torch.zeros((1, 2, 128), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    far, kept = torch.empty((1, 1, (1 << 32) + 32), device="meta"), torch.zeros((1, 1, 8), dtype=torch.int32)
    with pytest.raises(ValueError, match="scores_out.*32 bits"):
        hswa.decode_scored(layer, shape, cache, q, i, 32, None, far, q)
    with pytest.raises(ValueError, match="scores.*32 bits"):
        hswa.kv_evict(layer, shape, cache, dst, far, i, i, 32, kept, i)
    with pytest.raises(ValueError, match="scores_out.*32 bits"):
        hswa.kv_evict(layer, shape, cache, dst, torch.zeros((1, 1, 32)), i, i, 32, kept, i, scores_out=far)
    with pytest.raises(ValueError, match="kept_out.*32 bits"):
        hswa.kv_evict(layer, shape, cache, dst, torch.zeros((1, 1, 32)), i, i, 32,
                      torch.empty((1, 1, 1 << 31), dtype=torch.int32, device="meta"), i)
