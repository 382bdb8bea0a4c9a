"""The binding knows the tensors behind its rows: calls refuse those with fewer heads, channels or (where the host knows
their number) tokens than they take, before anything is called."""
import ctypes as C

import pytest
import torch

from paper_2606_26472_gb300 import build as B
from paper_2606_26472_gb300 import epikv as E

HQ, H, D = 8, 2, 128


@pytest.fixture(scope="module")
def ctx():
    B.build()
    c = C.c_void_p()               # no context: calls that come through are refused by the library
    c.heads = (HQ, H, D)
    return c


def rows(*shape):
    return E.rows(torch.zeros(*shape, dtype=torch.bfloat16))


def call(name, ctx, **kw):
    a = dict(q=rows(4, HQ, D), k=rows(4, H, D))
    a.update(o=a["q"], v=a["k"])
    a.update(kw)
    kv = E.epikv_kv_view()
    if name == "rope":
        E.epikv_rope(ctx, 4, HQ, a["q"], a["o"], None, None, stream=0)
    elif name == "append":
        E.epikv_append(ctx, 0, 1, None, None, 1, None, None, a["q"], a["o"], a["k"], a["v"], None, kv, stream=0)
    elif name == "attention":
        E.epikv_attention(ctx, 0, 1, None, None, 1, None, a["q"], a["o"], kv, stream=0)
    else:
        E.epikv_cache_read(ctx, 0, 4, None, None, a["k"], a["v"], kv, stream=0)


CALLS = [(n, r) for n, names in (("rope", "qo"), ("append", "qokv"), ("attention", "qo"), ("read", "kv")) for r in names]


@pytest.mark.parametrize("name,which", CALLS)
def test_smaller_tensors_are_refused(ctx, name, which):
    heads = H if which in "kv" else HQ
    for shape in ((4, heads, D // 2), (4, heads - 1, D)) + (((3, heads, D),) if name in ("rope", "read") else ()):
        with pytest.raises(ValueError, match=name):
            call(name, ctx, **{which: rows(*shape)})


@pytest.mark.parametrize("name,which", CALLS)
def test_tensors_that_hold_enough_reach_the_library(ctx, name, which):
    heads = H if which in "kv" else HQ
    wide = torch.zeros(9, 3 * heads, 2 * D, dtype=torch.bfloat16)
    for r in (rows(4, heads, D), E.rows(wide), E.rows(wide[:5, heads:2 * heads, D:]),
              E.epikv_rows(1 << 20, heads * D, D, E.EPIKV_TYPE_BF16)):      # memory of which no shape is known
        with pytest.raises(E.EpikvError) as err:
            call(name, ctx, **{which: r})
        assert err.value.status == E.EPIKV_EINVAL


def test_absent_rows_and_bare_handles(ctx):
    for c, kw in ((ctx, dict(q=None, o=None)), (C.c_void_p(), dict(q=rows(1, 1, 8)))):
        with pytest.raises(E.EpikvError) as err:
            call("append", c, **kw)
        assert err.value.status == E.EPIKV_EINVAL
