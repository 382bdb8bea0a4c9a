"""The chunk's attention and the weights where no GPU is: their warps exchange registers, and a build whose compiler gives
them others than they count on refuses these calls alone.  What the host refuses is refused before anything is launched."""
import os
import subprocess
import sys

import pytest

from paper_2606_26472_gb300 import build as B

from .test_attn_registers import runtime  # noqa: F401  (a stand-in for the CUDA runtime that records launches)

_HEAD = r"""
import ctypes as C, itertools, sys
from paper_2606_26472_gb300 import epikv as E
count = C.c_int.in_dll(C.CDLL(sys.argv[1]), "launches")
P = 1 << 20                       # an address that nothing reads
def make(fmt, **kw):
    cfg = E.make_attn_config(**{**dict(max_seqs=2, max_cache_tokens=64, max_new_tokens=40, num_layers=2, num_heads=4,
                                       num_kv_heads=2, head_dim=128, cache_format=fmt), **kw})
    ctx = E.epikv_attn_init(cfg, P, E.epikv_attn_workspace_bytes(cfg), stream=0)
    heads, dim = E.epikv_cache_row(2, 128, fmt)
    units = heads * dim
    return ctx, E.kv_view(P, P, layout=E.EPIKV_LAYOUT_CONTIGUOUS, stride_layer=64 * units, stride_seq=64 * units,
                          stride_token=units)
lib = E.load()
q = E.epikv_rows(P, 4 * 128, 128, E.EPIKV_TYPE_BF16)
w = E.epikv_weights(P, 2 * 64, 64)
"""

_TAKEN = _HEAD + r"""
for fmt in (E.EPIKV_CACHE_BF16, E.EPIKV_CACHE_E2M1):
    ctx, view = make(fmt)
    for call in (lambda: E.epikv_attention(ctx, 0, 1, P, P, 1, P, q, q, view, stream=0),
                 lambda: E.epikv_attention_chunk(ctx, 0, 1, P, P, 40, P, q, q, view, stream=0),
                 lambda: E.epikv_attention_weights(ctx, 0, 1, P, P, 1, P, q, P, w, view, stream=0)):
        before = count.value
        try:
            call()
            print("taken" if count.value > before else "nothing", end=" ")
        except E.EpikvError as e:
            print("refused" if e.status == E.EPIKV_ECUDA and count.value == before else e.status, end=" ")
"""


def run(runtime, code, registers):  # noqa: F811
    r = subprocess.run([sys.executable, "-c", code, runtime], capture_output=True, text=True, cwd=B.ROOT,
                       env={**os.environ, "LD_PRELOAD": runtime, "TEST_REGISTERS": str(registers)})
    assert r.returncode == 0, r.stderr
    return r.stdout.split()


@pytest.mark.parametrize("registers,bf16,e2m1", [(168, "taken taken refused", "taken refused refused"),
                                                 (128, "refused refused taken", "refused taken taken"),
                                                 (120, "refused refused refused", "refused refused refused")])
def test_each_call_by_its_own_registers(runtime, registers, bf16, e2m1):  # noqa: F811
    assert run(runtime, _TAKEN, registers) == (bf16 + " " + e2m1).split()


_REFUSED = _HEAD + r"""
import copy
def with_(s, **kw):
    t = type(s)()
    C.memmove(C.byref(t), C.byref(s), C.sizeof(s))
    for k, v in kw.items():
        setattr(t, k, v)
    return t
for fmt in (E.EPIKV_CACHE_BF16, E.EPIKV_CACHE_E2M1):
    ctx, view = make(fmt)
    paged = with_(view, layout=E.EPIKV_LAYOUT_PAGED, block_table=P, block_size=16, max_blocks_per_seq=4, num_blocks=9,
                  stride_block=16 * view.stride_token)
    base = dict(ctx=ctx, layer=1, n=2, ids=P, cu=P, new=3, len=P, step=1, causal=1, q=q, out=q, lse=P, kv=view, last=0, add=0,
                w=w)
    def chunk(a):
        return lib.epikv_attention_chunk(a["ctx"], a["layer"], a["n"], a["ids"], a["cu"], a["new"], a["len"], a["step"],
                                         a["causal"], a["q"], a["out"], a["lse"], a["kv"], None)
    def weights(a):
        return lib.epikv_attention_weights(a["ctx"], a["layer"], a["n"], a["ids"], a["cu"], a["new"], a["len"], a["step"],
                                           a["causal"], a["last"], a["q"], a["lse"], a["add"], a["w"], a["kv"], None)
    both = [dict(ctx=None), dict(layer=-1), dict(layer=2), dict(n=-1), dict(n=3), dict(ids=None), dict(cu=None), dict(new=-1),
            dict(new=41), dict(len=None), dict(step=0), dict(causal=2), dict(causal=-1), dict(q=None), dict(lse=P + 2),
            dict(kv=None)]
    both += [dict(q=with_(q, **k)) for k in (dict(ptr=None), dict(ptr=P + 8), dict(stride_token=513), dict(stride_head=-128),
                                             dict(stride_token=-512), dict(type=E.EPIKV_TYPE_F16), dict(type=E.EPIKV_TYPE_F32))]
    both += [dict(kv=with_(view, **k)) for k in (dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2),
             dict(stride_token=view.stride_token - 8), dict(stride_token=view.stride_token + 1), dict(stride_layer=-8),
             dict(stride_layer=4), dict(stride_seq=-8), dict(stride_seq=12), dict(layout=2), dict(layout=-1))]
    both += [dict(kv=with_(paged, **k)) for k in (dict(block_table=None), dict(block_size=0), dict(max_blocks_per_seq=0),
             dict(num_blocks=0), dict(stride_block=-8), dict(stride_block=4), dict(stride_table_layer=-1))]
    only_chunk = [dict(out=None), dict(out=with_(q, ptr=P + 4)), dict(out=with_(q, type=E.EPIKV_TYPE_F32))]
    only_weights = [dict(last=-1), dict(add=2), dict(add=-1), dict(lse=None), dict(w=None)]
    only_weights += [dict(w=with_(w, **k)) for k in (dict(ptr=None), dict(ptr=P + 2), dict(stride_seq=-1), dict(stride_head=-1),
                     dict(stride_head=0), dict(stride_seq=0), dict(stride_head=63), dict(stride_seq=100),
                     dict(stride_seq=63, stride_head=126))]
    before = count.value
    for call, cases in ((chunk, both + only_chunk), (weights, both + only_weights)):
        for c in cases:
            if call(dict(base, **c)) != E.EPIKV_EINVAL or count.value != before:
                print(call.__name__, fmt, c)
    # no sequences or no queries: nothing to do, and nothing is asked of the rest
    print(chunk(dict(base, n=0, q=None, kv=None)), chunk(dict(base, new=0, q=None, ids=None)), weights(dict(base, n=0, w=None)),
          count.value - before, end=" ")
    # taken: pages, rows of weights with the sequences inside the heads, and gaps
    for kv in (view, paged):
        for ww in (w, E.epikv_weights(P, 64, 128), E.epikv_weights(P + 4, 1000, 65)):
            print(chunk(dict(base, kv=kv, lse=None)), weights(dict(base, kv=kv, w=ww, last=1 << 30)), end=" ")
    print()
"""


def test_refusals(runtime):  # noqa: F811
    """Registers that all of these calls would be refused by, had they come that far: EPIKV_ECUDA, not EPIKV_EINVAL."""
    assert run(runtime, _REFUSED, 120) == 2 * (["0"] * 4 + ["2"] * 12)
