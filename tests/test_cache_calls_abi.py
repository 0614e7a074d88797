"""Refusals of the calls on shared and bounded caches, through the C ABI and
the binding, before any device work (no GPU is touched)."""

import ctypes

import pytest
import torch

from paper_2607_13095_amd import hswa

FAKE, FAKE2 = 0x1000, 0x2000  # non-null pointer values; validation must fail before any use
OK, INVALID, UNSUPPORTED, CAPACITY = 0, -1, -2, -3


def _shape(hq=64, hkv=8, d=128, pg=64, scale=0.088):
    return hswa._Shape(hq, hkv, d, pg, scale)


def _cache(stride=8, pages=10, table=FAKE):
    return hswa._Cache(FAKE, FAKE, pages, table, stride)


def _full():
    return hswa._Layer(hswa.HSWA_LAYER_FULL, 0)


def _evict(layer=None, shape=None, src=None, dst=None, scores=FAKE, stride=500, ctx=FAKE, budgets=FAKE, ns=2, maxc=500,
           recent=0, sinks=0, kept=FAKE, kstride=100, so=None, sostride=0, lens=FAKE):
    return hswa.load().hswa_kv_evict(layer or _full(), ctypes.byref(shape or _shape()),
                                     ctypes.byref(src or _cache()), ctypes.byref(dst or _cache(2, 10, FAKE2)), scores,
                                     stride, ctx, budgets, ns, maxc, recent, sinks, kept, kstride, so, sostride, lens, None)


@pytest.mark.parametrize("kw,code", [
    (dict(ns=0), OK),
    (dict(layer=hswa._Layer(hswa.HSWA_LAYER_SWA, 128)), UNSUPPORTED),
    (dict(layer=hswa._Layer(hswa.HSWA_LAYER_SWA_PAGED, 128)), UNSUPPORTED),
    (dict(layer=hswa._Layer(7, 128)), INVALID),
    (dict(shape=_shape(d=64)), UNSUPPORTED), (dict(shape=_shape(hq=63)), INVALID), (dict(shape=_shape(pg=48)), UNSUPPORTED),
    (dict(ns=-1), INVALID), (dict(maxc=0), INVALID), (dict(recent=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(kstride=0), INVALID), (dict(ns=1 << 20), UNSUPPORTED),
    (dict(stride=499), CAPACITY), (dict(src=_cache(7)), CAPACITY), (dict(dst=_cache(1, 10, FAKE2)), CAPACITY),
    (dict(so=FAKE2, sostride=99), CAPACITY),
    (dict(dst=_cache(8, 10, FAKE)), INVALID), (dict(so=FAKE, sostride=100), INVALID),
    (dict(src=_cache(pages=0)), INVALID),
    (dict(scores=None), INVALID), (dict(ctx=None), INVALID), (dict(budgets=None), INVALID), (dict(kept=None), INVALID),
    (dict(lens=None), INVALID),
])
def test_kv_evict_refusals(kw, code):
    assert _evict(**kw) == code


def _cpu_cache(ns=2, pages=4, hkv=2, pg=16):
    return hswa.Cache(torch.zeros(hswa.k_pool_shape(pages, hkv, pg), dtype=torch.bfloat16),
                      torch.zeros(hswa.v_pool_shape(pages, hkv, pg), dtype=torch.bfloat16),
                      torch.zeros((ns, 2), dtype=torch.int32))


def test_kv_evict_binding_refusals():
    shape, src, dst = hswa.Shape(4, 2, 128, 16), _cpu_cache(), _cpu_cache()
    i = torch.zeros(2, dtype=torch.int32)
    ok = dict(scores=torch.zeros((2, 2, 32)), kept_out=torch.zeros((2, 2, 8), dtype=torch.int32))

    def call(**kw):
        a = {**ok, **kw}
        hswa.kv_evict(hswa.Layer.full(), shape, src, dst, a["scores"], i, i, 32, a["kept_out"], i,
                      scores_out=a.get("scores_out"))

    with pytest.raises(ValueError):  # one row of scores per sequence and KV head
        call(scores=torch.zeros((2, 1, 32)))
    with pytest.raises(ValueError):
        call(kept_out=torch.zeros((2, 8), dtype=torch.int32))
    with pytest.raises(ValueError):
        call(scores_out=torch.zeros((1, 2, 8)))
    with pytest.raises(TypeError):
        call(kept_out=None)
    with pytest.raises(ValueError):  # not on the GPU
        call()
