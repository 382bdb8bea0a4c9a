"""The decode loop (examples/llama_decode.py) with the library's own append and attention: a bf16 and a 4-bit cache that
evictions shorten.  Every step's cache rows are followed: what eviction leaves is what was appended, row by row."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import epikv_oracle as O
from paper_2606_26472_gb300 import epikv as E
from synth import gen
from synth.device import as_u16

from .harness import assert_scores_close

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits", [16, 4])
def test_decode_with_eviction(gpu_lib, bits):
    import llama_decode as D
    shape = D.small_shape()
    prompt, steps, K, slack = 8, 200, 96, 16
    r = D.decode(shape, batch=4, prompt=prompt, steps=steps, budget=K, slack=slack, record=True, attention="library",
                 cache_bits=bits)
    assert E.epikv_get_error(r.ctx) == (E.EPIKV_OK, 0) and E.epikv_attn_get_error(r.attn.ctx) == (E.EPIKV_OK, 0)
    assert r.evictions >= 4 * 5 and r.tokens.shape == (4, steps)
    bt = r.cache.block_table.cpu().numpy()
    for b in range(4):
        ra = [gen.bf16_bits_to_f64(r.band_rows[(b, l)]) for l in shape.band_a]
        rb = [gen.bf16_bits_to_f64(r.band_rows[(b, l)]) for l in shape.band_b]
        pos, sc, n = E.epikv_read_slots(r.ctx, b, E.EPIKV_SCORE_BANDZ, 4096)
        pos = np.array(pos)
        assert n == r.n_cache[b] and pos[-1] == prompt + steps - 1 and list(pos[:prompt]) == list(range(prompt))
        assert_scores_close(sc, O.bandz_scores(ra, rb, 64)[pos], f"decode seq {b}")
        for w in range(2):
            rows = as_u16(r.cache.rows(w, b, np.arange(n), bt))
            np.testing.assert_array_equal(rows, r.kv_rows[b][w][pos])


def test_first_steps_agree_with_torch(gpu_lib):
    """Four steps of both attentions on the same tokens: bf16 rows differ by roundings of the rotation's angles alone, so
    the hidden states stay within a few units of bf16 of each other (2^-8 each layer's addition, eight layers)."""
    import llama_decode as D
    shape = D.small_shape()
    model = D.RandomLlama(shape, 3)
    toks = torch.randint(0, shape.vocab, (4, 3), generator=torch.Generator().manual_seed(1)).cuda()
    seqs = torch.arange(3, device="cuda")
    caches = [D.KVCache(E.EPIKV_LAYOUT_PAGED, shape.layers, shape.kv_heads, shape.head_dim, max_seqs=3, max_tokens=32)
              for _ in range(2)]
    attn = D.CacheAttention(shape, caches[1], 3, 32)
    for t in range(4):
        n = torch.full((3,), t, dtype=torch.int64, device="cuda")
        _, a = model.step(toks[t], n, caches[0], seqs, n, n + 1)
        attn.length.fill_(t)
        attn.position.fill_(t)
        _, b = model.step_library(toks[t], attn, caches[1])
        for x, y in zip(a, b):
            x, y = x.double(), y.double()
            assert float((x - y).norm() / x.norm()) < 8 * 2.0 ** -8


def test_refused_choices(gpu_lib):
    import llama_decode as D
    for kw in (dict(attention="other"), dict(cache_bits=8, attention="library"), dict(cache_bits=4)):
        with pytest.raises(ValueError):
            D.decode(D.small_shape(), steps=1, **kw)
