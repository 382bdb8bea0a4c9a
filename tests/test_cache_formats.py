"""A cache's view says what its rows hold: calls that would read them as something else are refused, before anything is
called."""
import ctypes as C

import pytest

from paper_2606_26472_gb300 import build as B
from paper_2606_26472_gb300 import epikv as E
from paper_2606_26472_gb300.cache import KVCache

BAND = E.EPIKV_SCORE_BANDZ | E.EPIKV_SCORE_HSVAR


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()


def view(fmt):
    return KVCache(E.EPIKV_LAYOUT_CONTIGUOUS, 1, 2, 64, max_seqs=1, max_tokens=16, cache_format=fmt, device="cpu").view()


def context(**kw):
    c = C.c_void_p()               # no context: calls that come through are refused by the library
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def reaches_the_library(call):
    with pytest.raises(E.EpikvError) as err:
        call()
    assert err.value.status == E.EPIKV_EINVAL


SCORED = [lambda c, kv: E.epikv_score_update(c, 1, None, None, 1, None, kv, stream=0),
          lambda c, kv: E.epikv_step(c, 1, None, None, 1, None, None, None, kv, stream=0)]


@pytest.mark.parametrize("call", SCORED)
def test_scores_of_keys_and_values_need_bf16_rows(call):
    for kind in (E.EPIKV_SCORE_LAGKV, E.EPIKV_SCORE_KVKEY, E.EPIKV_SCORE_KVVAL, E.EPIKV_SCORE_LAGKEY):
        for kinds in (kind, kind | BAND):
            with pytest.raises(ValueError, match="bf16"):
                call(context(score_kinds=kinds), view(E.EPIKV_CACHE_E2M1))
            reaches_the_library(lambda: call(context(score_kinds=kinds), view(E.EPIKV_CACHE_BF16)))
    reaches_the_library(lambda: call(context(score_kinds=BAND), view(E.EPIKV_CACHE_E2M1)))
    reaches_the_library(lambda: call(context(score_kinds=kind), E.epikv_kv_view()))     # of which nothing is known


def test_lag_scores_without_a_workspace():
    with pytest.raises(ValueError, match="bf16"):
        E.epikv_lagkv_score_noalloc(view(E.EPIKV_CACHE_E2M1), 0, 16, 1, 2, 64, 4, 1e-6, 4, None, stream=0)
    reaches_the_library(lambda: E.epikv_lagkv_score_noalloc(view(E.EPIKV_CACHE_BF16), 0, 16, 1, 2, 64, 4, 1e-6, 4, None,
                                                            stream=0))


@pytest.mark.parametrize("mine,other", [(E.EPIKV_CACHE_BF16, E.EPIKV_CACHE_E2M1), (E.EPIKV_CACHE_E2M1, E.EPIKV_CACHE_BF16)])
def test_context_and_cache_agree(mine, other):
    c = context(heads=(2, 2, 64), cache_format=mine)
    calls = [lambda kv: E.epikv_append(c, 0, 1, None, None, 1, None, None, None, None, None, None, None, kv, stream=0),
             lambda kv: E.epikv_attention(c, 0, 1, None, None, 1, None, None, None, kv, stream=0),
             lambda kv: E.epikv_cache_read(c, 0, 1, None, None, None, None, kv, stream=0)]
    for call in calls:
        with pytest.raises(ValueError, match="cache_format"):
            call(view(other))
        reaches_the_library(lambda: call(view(mine)))
