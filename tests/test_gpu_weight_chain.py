"""Eviction by attention weight as a decode loop runs it: rows appended, attention with its log-sums (a prompt through the chunk's
kernel, steps through the other), what the slots of every layer received, the scores, selection and compaction, again and again.
Each stage against its plain form over what the stage before left."""
import math

import numpy as np
import pytest
import torch

from paper_2606_26472_gb300 import epikv as E

from . import cache_ops as R
from .chunk_ops import check_attention, check_weights, queries
from .test_gpu_weights import plain_kept

pytestmark = pytest.mark.gpu
OK = (E.EPIKV_OK, 0)


class Chain:
    def __init__(self, bits, *, S=3, T=500, H=2, Hq=8, d=64, L=2, block=16, most=260):
        self.S, self.T, self.H, self.Hq, self.d, self.L = S, T, H, Hq, d, L
        self.c = R.Cache(seqs=S, T=T, H=H, d=d, bits=bits, block=block, layers=L, seed=31)
        self.actx = self.c.context(Hq, most)
        pool = self.c.c
        cfg = E.make_config(max_seqs=S, max_cache_tokens=T, max_new_tokens=most, num_layers=L, num_kv_heads=pool.H,
                            head_dim=pool.d, score_kinds=E.EPIKV_SCORE_WEIGHT)
        self.ws = torch.empty(E.epikv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        self.wctx = E.epikv_init(cfg, self.ws, self.ws.numel())
        self.prefill = (4, 0, 9)
        for s in range(S):
            E.epikv_seq_reset(self.wctx, s, self.prefill[s], E.EPIKV_SCORE_WEIGHT)
        self.held = [0] * S
        self.score = [np.zeros(0, np.float32) for _ in range(S)]
        self.weight = torch.full((S, H, T), -7.5, device="cuda")
        self.turn = 0

    def step(self, new, budget, chunk, decay, last=0):
        self.turn += 1
        S, H, Hq, d, held = self.S, self.H, self.Hq, self.d, list(self.held)
        view, most, total = self.c.c.view(), max(new), sum(new)
        seq_ids, cu, ln = R.batch(new, held)
        w = E.weights_view(self.weight)
        attention = E.epikv_attention_chunk if chunk else E.epikv_attention
        for l in range(self.L):
            k, v = (queries(total, H, d, 100 * self.turn + 10 * l + i) for i in (0, 1))
            q = queries(total, Hq, d, 100 * self.turn + 10 * l + 2)
            E.epikv_append(self.actx, l, S, seq_ids, cu, most, ln, None, None, None, E.rows(k), E.rows(v), None, view)
            out, lse = torch.empty_like(q), torch.empty(total, Hq, device="cuda")
            attention(self.actx, l, S, seq_ids, cu, most, ln, E.rows(q), E.rows(out), view, lse=lse)
            before = self.weight.clone()
            E.epikv_attention_weights(self.actx, l, S, seq_ids, cu, most, ln, E.rows(q), lse, w, view, add=l > 0, last=last)
            check_attention(self.c, q, out, lse, new, held, layer=l, what=f"turn {self.turn} layer {l}")
            check_weights(self.c, q, lse, new, held, self.weight, before, layer=l, add=l > 0, last=last,
                          what=f"turn {self.turn} layer {l}")
        E.epikv_score_update(self.wctx, S, seq_ids, cu, most, None, None)
        E.epikv_weigh(self.wctx, S, seq_ids, w, decay)
        wn = self.weight.cpu().numpy()
        n = [a + b for a, b in zip(held, new)]
        raw = [[[self.c.raw(i)[self.c.index(l, s, torch.arange(n[s]))].clone() for s in range(S)] for l in range(self.L)]
               for i in (0, 1)]
        kept = torch.full((S, self.T), -1, dtype=torch.int32, device="cuda")
        n_kept = torch.zeros(S, dtype=torch.int32, device="cuda")
        E.epikv_select(self.wctx, S, seq_ids, torch.tensor(budget, dtype=torch.int32, device="cuda"), None, kept, self.T, n_kept)
        E.epikv_compact(self.wctx, S, seq_ids, kept, self.T, view)
        kept, n_kept = kept.cpu().numpy(), n_kept.tolist()
        for s in range(S):
            old = np.concatenate([self.score[s], np.zeros(new[s], np.float32)])
            heads = wn[s, 0, :n[s]].copy()
            for h in range(1, H):
                heads = heads + wn[s, h, :n[s]]
            score = (np.float32(decay) * old).astype(np.float32) + heads
            want = plain_kept(score, budget[s], self.prefill[s])
            assert n_kept[s] == len(want)
            if len(want) < n[s]:
                np.testing.assert_array_equal(kept[s, :len(want)], want)
            self.score[s], self.held[s] = score[want], len(want)
            _, got, m = E.epikv_read_slots(self.wctx, s, E.EPIKV_SCORE_WEIGHT, self.T)
            assert m == len(want)
            np.testing.assert_array_equal(np.asarray(got, np.float32).view(np.int32), self.score[s].view(np.int32))
            for i in (0, 1):
                for l in range(self.L):
                    now = self.c.raw(i)[self.c.index(l, s, torch.arange(m))]
                    assert torch.equal(now, raw[i][l][s][torch.as_tensor(want, device="cuda")])
        assert E.epikv_attn_get_error(self.actx) == OK and E.epikv_get_error(self.wctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d,block", [(2, 8, 64, 16), (1, 4, 128, 0), (2, 2, 256, 16)])
def test_prompts_then_steps(gpu_lib, bits, H, Hq, d, block):
    """Prompts cut to a budget, single tokens whose log-sums come from the other attention, a turn of several tokens."""
    x = Chain(bits, H=H, Hq=Hq, d=d, block=block)
    x.step([200, 64, 251], [128, 128, 90], chunk=True, decay=1.0)
    for i in range(4):
        x.step([1, 1, 1], [128, 70, 90], chunk=i == 2, decay=0.9)
    x.step([37, 5, 80], [110, 60, 90], chunk=True, decay=0.5, last=16)
    x.step([1, 1, 1], [110, 60, 90], chunk=False, decay=0.9)
    assert math.isfinite(float(x.score[0].sum()))


def test_every_layer_adds_up_to_its_rows(gpu_lib):
    """What all slots of a sequence receive is one for every layer, token and query head, whatever was evicted before."""
    x = Chain(16, L=5)
    x.step([150, 1, 33], [64, 64, 64], chunk=True, decay=1.0)
    x.step([2, 3, 1], [500, 500, 500], chunk=False, decay=0.0)
    for s, n in enumerate((2, 3, 1)):
        assert abs(float(x.score[s].astype(np.float64).sum()) - 5 * n * x.Hq) < 1e-3


@pytest.mark.parametrize("bits", [16, 4])
def test_a_captured_step(gpu_lib, bits):
    """A whole decode step as one graph, its lengths those that the selection before left on the device: the bits of the same
    steps one by one."""
    ends = []
    for captured in (False, True):
        x = Chain(bits)
        x.step([100, 30, 171], [64, 64, 64], chunk=True, decay=1.0)
        S, view, w = x.S, x.c.c.view(), E.weights_view(x.weight)
        seq_ids, cu, ln = R.batch([1] * S, x.held)
        budget = torch.full((S,), 70, dtype=torch.int32, device="cuda")
        kept = torch.zeros(S, x.T, dtype=torch.int32, device="cuda")
        q, k, v = queries(S, x.Hq, x.d, 5), queries(S, x.H, x.d, 6), queries(S, x.H, x.d, 7)
        out, lse = torch.zeros_like(q), torch.zeros(S, x.Hq, device="cuda")
        s = torch.cuda.Stream()

        def step():
            for l in range(x.L):
                E.epikv_append(x.actx, l, S, seq_ids, cu, 1, ln, None, None, None, E.rows(k), E.rows(v), None, view, stream=s)
                E.epikv_attention(x.actx, l, S, seq_ids, cu, 1, ln, E.rows(q), E.rows(out), view, lse=lse, stream=s)
                E.epikv_attention_weights(x.actx, l, S, seq_ids, cu, 1, ln, E.rows(q), lse, w, view, add=l > 0, stream=s)
            E.epikv_score_update(x.wctx, S, seq_ids, cu, 1, None, None, stream=s)
            E.epikv_weigh(x.wctx, S, seq_ids, w, 0.75, stream=s)
            E.epikv_select(x.wctx, S, seq_ids, budget, None, kept, x.T, ln, stream=s)
            E.epikv_compact(x.wctx, S, seq_ids, kept, x.T, view, stream=s)
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        run = step
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                step()
            run = g.replay
        for i in range(12):
            q.copy_(queries(S, x.Hq, x.d, 40 + i))
            k.copy_(queries(S, x.H, x.d, 60 + i))
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
        assert E.epikv_attn_get_error(x.actx) == OK and E.epikv_get_error(x.wctx) == OK
        assert ln.tolist() == [70, 30 + 13, 70]
        slots = [E.epikv_read_slots(x.wctx, b, E.EPIKV_SCORE_WEIGHT, x.T) for b in range(S)]
        ends.append((out, lse, kept, [x.c.raw(i) for i in (0, 1)], x.weight, slots))
    a, b = ends
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    assert all(torch.equal(m, n) for m, n in zip(a[3], b[3])) and torch.equal(a[4], b[4])
    for m, n in zip(a[5], b[5]):
        assert list(m[0]) == list(n[0]) and list(m[1]) == list(n[1]) and m[2] == n[2]
