"""CPU checks of the cache operators' boundary: configurations, row shapes and host-side refusals."""
import ctypes as C

import pytest

from paper_2606_26472_gb300 import build as B
from paper_2606_26472_gb300 import epikv as E


@pytest.fixture(scope="module")
def lib():
    B.build()
    return E.load()


def cfg(**kw):
    base = dict(max_seqs=4, max_cache_tokens=1024, max_new_tokens=8)
    base.update(kw)
    return E.make_attn_config(**base)


def test_cache_rows(lib):
    assert E.epikv_cache_row(8, 128, E.EPIKV_CACHE_BF16) == (8, 128)
    for H in range(1, 33):
        for d in (64, 128, 256):
            used = H * (d // 2 + d // 16)
            if used > 4096:
                with pytest.raises(E.EpikvError):
                    E.epikv_cache_row(H, d, E.EPIKV_CACHE_E2M1)
                continue
            h, x = E.epikv_cache_row(H, d, E.EPIKV_CACHE_E2M1)
            assert h <= 32 and x in (8, 16, 32, 64, 128, 256) and h * x % 8 == 0
            assert used <= 2 * h * x <= used + 272          # little padding
            # a context of the eviction calls takes such rows
            assert E.epikv_workspace_bytes(E.make_config(max_seqs=2, max_cache_tokens=64, max_new_tokens=4,
                                                         num_kv_heads=h, head_dim=x)) > 0
    assert E.epikv_cache_row(8, 128, E.EPIKV_CACHE_E2M1) == (9, 32)
    for bad in ((0, 128, 0), (33, 64, 0), (8, 96, 0), (8, 128, 2), (16, 256, 0)):
        with pytest.raises(E.EpikvError):
            E.epikv_cache_row(*bad)


def test_configurations(lib):
    n = E.epikv_attn_workspace_bytes(cfg())
    assert n > 0 and n % 256 == 0
    assert E.epikv_attn_workspace_bytes(cfg(cache_format=E.EPIKV_CACHE_E2M1, kv_scale=4096)) > 0
    for bad in (dict(max_seqs=0), dict(max_seqs=5000), dict(max_cache_tokens=0), dict(max_new_tokens=0),
                dict(num_layers=0), dict(num_heads=12), dict(num_heads=0), dict(num_kv_heads=0), dict(head_dim=32),
                dict(cache_format=2), dict(softmax_scale=-1.0), dict(softmax_scale=float("inf")),
                dict(softmax_scale=float("nan")), dict(kv_scale=4096)):
        assert E.epikv_attn_workspace_bytes(cfg(**bad)) == 0, bad


def test_null_contexts_and_workspaces(lib):
    c, ctx = cfg(), C.c_void_p()
    need = E.epikv_attn_workspace_bytes(c)
    assert lib.epikv_attn_init(C.byref(ctx), C.byref(c), None, need, None) == E.EPIKV_EINVAL
    assert lib.epikv_attn_init(C.byref(ctx), C.byref(c), 0x1000 + 16, need, None) == E.EPIKV_EINVAL
    assert lib.epikv_attn_init(C.byref(ctx), C.byref(c), 0x1000, need - 1, None) == E.EPIKV_EINVAL
    assert lib.epikv_attn_init(None, C.byref(c), 0x1000, need, None) == E.EPIKV_EINVAL
    assert lib.epikv_rope(None, 1, 1, None, None, None, None, 0, None) == E.EPIKV_EINVAL
    assert lib.epikv_append(None, 0, 1, None, None, 1, None, 1, None, None, None, None, None, None, None,
                            None) == E.EPIKV_EINVAL
    assert lib.epikv_attention(None, 0, 1, None, None, 1, None, 1, 1, None, None, None, None, None) == E.EPIKV_EINVAL
    assert lib.epikv_cache_read(None, 0, 1, None, None, None, None, None, None) == E.EPIKV_EINVAL
    assert lib.epikv_rope_table(None, 1, None, None) == E.EPIKV_EINVAL
    assert lib.epikv_attn_get_error(None, None) == E.EPIKV_EINVAL
