"""CPU checks of the chunk's attention, the weights and their way into eviction: configurations and host-side refusals."""
import pytest
import torch

from paper_2606_26472_gb300 import build as B
from paper_2606_26472_gb300 import epikv as E


@pytest.fixture(scope="module")
def lib():
    B.build()
    return E.load()


def cfg(**kw):
    return E.make_config(**{**dict(max_seqs=4, max_cache_tokens=1024, max_new_tokens=64), **kw})


def test_the_weight_kind_in_configurations(lib):
    W = E.EPIKV_SCORE_WEIGHT
    alone = E.epikv_workspace_bytes(cfg(score_kinds=W))
    assert alone > 0
    # the column of scores alone: as much more with another kind beside it
    for other in (E.EPIKV_SCORE_BANDZ, E.EPIKV_SCORE_LAGKV, 63):
        assert E.epikv_workspace_bytes(cfg(score_kinds=W | other)) == E.epikv_workspace_bytes(cfg(score_kinds=other)) + 4 * 4 * 1024
    # it needs nothing of the hidden states or windows
    assert E.epikv_workspace_bytes(cfg(score_kinds=W, hidden=0, n_band_a=0, z_window=0, lag=0)) == alone
    assert E.epikv_workspace_bytes(cfg(score_kinds=W, select_chunk=16)) > alone
    for bad in (dict(score_kinds=64), dict(score_kinds=64 | W), dict(score_kinds=256), dict(score_kinds=256 | W),
                dict(score_kinds=-1), dict(score_kinds=W, layer_budgets=1), dict(score_kinds=W | 1, layer_budgets=1)):
        assert E.epikv_workspace_bytes(cfg(**bad)) == 0, bad


def test_null_contexts(lib):
    assert lib.epikv_attention_chunk(None, 0, 1, None, None, 1, None, 1, 1, None, None, None, None, None) == E.EPIKV_EINVAL
    assert lib.epikv_attention_weights(None, 0, 1, None, None, 1, None, 1, 1, 0, None, None, 0, None, None,
                                       None) == E.EPIKV_EINVAL
    assert lib.epikv_weigh(None, 1, None, None, 1, 1.0, None) == E.EPIKV_EINVAL


def test_views_of_weights(lib):
    t = torch.zeros(3, 2, 40)
    w = E.weights_view(t)
    assert (w.ptr, w.stride_seq, w.stride_head, w.shape) == (t.data_ptr(), 80, 40, (3, 2, 40))
    w = E.weights_view(torch.zeros(2, 3, 40).transpose(0, 1)[:, :, 5:30])
    assert (w.stride_seq, w.stride_head, w.shape) == (40, 120, (3, 2, 25))
    for bad in (t[0], t.double(), t.transpose(1, 2), t.half()):
        with pytest.raises(ValueError):
            E.weights_view(bad)


class Handle:
    """What the binding knows of a context."""
    heads, cache_format, slots = (8, 2, 64), E.EPIKV_CACHE_BF16, (3, 40)


def test_rows_and_weights_that_are_too_small(lib):
    ok = E.rows(torch.zeros(5, 8, 64, dtype=torch.bfloat16))
    for bad in (E.rows(torch.zeros(5, 7, 64, dtype=torch.bfloat16)), E.rows(torch.zeros(5, 8, 32, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            E.epikv_attention_chunk(Handle, 0, 1, None, None, 1, None, bad, ok, None, stream=0)
        with pytest.raises(ValueError):
            E.epikv_attention_chunk(Handle, 0, 1, None, None, 1, None, ok, bad, None, stream=0)
        with pytest.raises(ValueError):
            E.epikv_attention_weights(Handle, 0, 1, None, None, 1, None, bad, None, E.weights_view(torch.zeros(3, 2, 40)), None,
                                      stream=0)
    for shape in ((2, 2, 40), (3, 1, 40), (3, 2, 39)):
        with pytest.raises(ValueError):
            E.epikv_attention_weights(Handle, 0, 1, None, None, 1, None, ok, None, E.weights_view(torch.zeros(shape)), None,
                                      stream=0)
        with pytest.raises(ValueError):
            E.epikv_weigh(Handle, 1, None, E.weights_view(torch.zeros(shape)), n_heads=2, stream=0)
    other = E.kv_view(16, 16, stride_layer=0, stride_token=128)
    other.cache_format = E.EPIKV_CACHE_E2M1
    for call in (lambda: E.epikv_attention_chunk(Handle, 0, 1, None, None, 1, None, ok, ok, other, stream=0),
                 lambda: E.epikv_attention_weights(Handle, 0, 1, None, None, 1, None, ok, None,
                                                   E.weights_view(torch.zeros(3, 2, 40)), other, stream=0)):
        with pytest.raises(ValueError):
            call()
