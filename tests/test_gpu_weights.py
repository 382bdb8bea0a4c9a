"""epikv_attention_weights against float64, and eviction by what epikv_weigh adds up against a plain selection."""
import math

import numpy as np
import pytest
import torch

from paper_2606_26472_gb300 import epikv as E
from paper_2606_26472_gb300.cache import KVCache

from . import cache_ops as R
from .chunk_ops import attend, check_attention, check_weights, lse64, queries, weigh
from .harness import oracle_kept

pytestmark = pytest.mark.gpu

SHAPES = [(8, 32, 128), (1, 1, 64), (1, 8, 128), (2, 14, 128), (3, 3, 64), (4, 32, 64), (5, 20, 128), (2, 4, 256),
          (4, 32, 256), (11, 11, 64), (1, 71, 64)]
OK = (E.EPIKV_OK, 0)


def fresh(c, extra=3):
    """Weights of every slot, and some behind the last, holding what no sum is."""
    return torch.full((c.S, c.H, c.T + extra), -7.5, device="cuda")


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", SHAPES)
def test_single_tokens(gpu_lib, bits, H, Hq, d):
    held = [0, 1, 14, 15, 16, 63, 64, 126, 127, 128, 129, 255, 300, 1023]
    for block in (16, 0, 7):
        c = R.Cache(seqs=14, T=1030, H=H, d=d, bits=bits, block=block, seed=H * d)
        ctx = c.context(Hq, 1)
        q = queries(14, Hq, d)
        seqs = list(range(13, -1, -1))
        lse = lse64(c, q, [1] * 14, held, seqs=seqs)
        w = fresh(c)
        before = w.clone()
        weigh(c, ctx, q, lse, [1] * 14, held, w, seqs=seqs)
        check_weights(c, q, lse, [1] * 14, held, w, before, seqs=seqs, what=f"block {block}")
        assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", SHAPES)
def test_ragged_chunks(gpu_lib, bits, H, Hq, d):
    new, held = [3, 0, 1, 17, 147, 8, 64], [0, 5, 200, 31, 77, 1500, 63]
    for block, last in ((16, 0), (0, 5), (48, 64)):
        c = R.Cache(seqs=7, T=1600, H=H, d=d, bits=bits, block=block, seed=H + d)
        ctx = c.context(Hq, 200)
        q = queries(sum(new), Hq, d)
        seqs = [3, 0, 6, 1, 2, 5, 4]
        lse = lse64(c, q, new, held, seqs=seqs)
        w = fresh(c)
        before = w.clone()
        weigh(c, ctx, q, lse, new, held, w, seqs=seqs, last=last)
        check_weights(c, q, lse, new, held, w, before, seqs=seqs, last=last, what=f"block {block}")
        before = w.clone()
        weigh(c, ctx, q, lse, new, held, w, seqs=seqs, last=last, add=True)
        check_weights(c, q, lse, new, held, w, before, seqs=seqs, last=last, add=True, what=f"block {block} added")
        assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", [(2, 8, 128), (1, 2, 64), (1, 1, 256), (2, 32, 128)])
def test_prompts(gpu_lib, bits, H, Hq, d):
    """Whole prompts and pieces, with the attention's own log-sums: a KV head's weights add up to its rows."""
    new, held = [700, 300, 1, 33], [0, 900, 9000, 4001]
    c = R.Cache(seqs=4, T=9100, H=H, d=d, bits=bits, seed=5)
    ctx = c.context(Hq, 700)
    q = queries(sum(new), Hq, d)
    _, lse = attend(c, ctx, q, new, held)
    w = fresh(c)
    before = w.clone()
    weigh(c, ctx, q, lse, new, held, w)
    check_weights(c, q, lse, new, held, w, before)
    for b, n in enumerate(new):
        total = w[b, :, :held[b] + n].double().sum(1) / (n * Hq // H)
        assert float((total - 1).abs().max()) < 1e-4
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d,block", [(8, 32, 128, 16), (16, 32, 64, 0), (4, 8, 256, 32), (3, 24, 128, 7)])
def test_decode_steps_of_long_caches(gpu_lib, bits, H, Hq, d, block):
    """One token of sequences with so many slots that each SM takes dozens of runs of them: every ring goes round often."""
    held = [5999 - 123 * b for b in range(24)]
    c = R.Cache(seqs=24, T=6000, H=H, d=d, bits=bits, block=block, seed=d)
    ctx = c.context(Hq, 1)
    q = queries(24, Hq, d)
    lse = lse64(c, q, [1] * 24, held)
    w = fresh(c)
    before = w.clone()
    weigh(c, ctx, q, lse, [1] * 24, held, w)
    check_weights(c, q, lse, [1] * 24, held, w, before)
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
def test_prefix_without_the_new_tokens(gpu_lib, bits):
    c = R.Cache(seqs=3, T=400, H=2, d=64, bits=bits, seed=2)
    ctx = c.context(6, 90)
    new, held = [5, 90, 3], [0, 399, 18]
    q = queries(98, 6, 64)
    lse = lse64(c, q, new, held, causal=False)
    w = fresh(c)
    before = w.clone()
    weigh(c, ctx, q, lse, new, held, w, causal=False)
    check_weights(c, q, lse, new, held, w, before, causal=False)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new,H,Hq", [(1, 2, 8), (40, 1, 4), (150, 2, 2)])
def test_what_is_not_seen(gpu_lib, bits, new, H, Hq):
    """NaN in slots from some place on: the slots before are as in the clean cache; rows whose lse is -inf give nothing."""
    held, T = 45, 256
    c = R.Cache(seqs=1, T=T, H=H, d=128, bits=bits, seed=3)
    ctx = c.context(Hq, 160)
    q = queries(new, Hq, 128)
    lse = lse64(c, q, [new], [held])
    lse[::3, 0] = -math.inf
    clean = fresh(c)
    before = clean.clone()
    weigh(c, ctx, q, lse, [new], [held], clean)
    check_weights(c, q, lse, [new], [held], clean, before)
    for first in sorted({held + new, held + new // 2 + 1, held}):
        raw = c.raw(0).clone()
        c.raw(0)[c.index(0, 0, torch.arange(first, T))] = 0x7F if bits == 4 else torch.tensor(
            [0xC0, 0x7F], dtype=torch.uint8, device="cuda").repeat(c.units)
        w = fresh(c)
        weigh(c, ctx, q, lse, [new], [held], w)
        assert torch.equal(w[:, :, :first], clean[:, :, :first]) and torch.equal(w[:, :, held + new:], before[:, :, held + new:])
        counted = (lse[max(0, first - held):] != -math.inf).view(-1, H, Hq // H).any(2).any(0)   # a head without rows: 0
        for h in range(H):
            bad = w[0, h, first:held + new]
            last = torch.nonzero((lse.view(new, H, -1)[:, h] != -math.inf).any(1)).max().item() + held + 1
            if bool(counted[h]):
                assert bool(bad[:max(0, last - first)].isnan().all())
        c.raw(0).copy_(raw)


def test_no_tokens(gpu_lib):
    """Entries without new tokens store zeros or leave what is there."""
    c = R.Cache(seqs=2, T=300, H=2, d=64, seed=2)
    ctx = c.context(4, 8)
    q, lse = queries(1, 4, 64), torch.zeros(1, 4, device="cuda")
    w = fresh(c)
    weigh(c, ctx, q, lse, [0, 0], [200, 0], w, add=True, max_new=8)
    assert bool((w == -7.5).all())
    for max_new in (8, 0):
        w = fresh(c)
        weigh(c, ctx, q, lse, [0, 0], [200, 0], w, max_new=max_new)
        assert not w[0, :, :200].any() and bool((w[0, :, 200:] == -7.5).all()) and bool((w[1] == -7.5).all())


@pytest.mark.parametrize("bits", [16, 4])
def test_strides_streams_and_graphs(gpu_lib, bits):
    """Weights [head][sequence][slot], queries out of wider rows, another stream, a replayed graph with other lengths."""
    c = R.Cache(seqs=3, T=700, H=2, d=128, bits=bits, seed=11)
    ctx = c.context(8, 64)
    wide = queries(100, 14, 128)
    q = wide[:, 3:11]
    new = [40, 10, 50]
    store = torch.full((2, 3, 800), -7.5, device="cuda")
    w = store.transpose(0, 1)
    seq_ids, cu, lens = R.batch(new, [0, 0, 0])
    lse = torch.zeros(100, 8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call = lambda: E.epikv_attention_weights(ctx, 0, 3, seq_ids, cu, 64, lens, E.rows(q), lse, E.weights_view(w), c.c.view())  # noqa: E731
    with torch.cuda.stream(s):
        g = None
        for held in ([300, 0, 11], [77, 600, 128], [1, 2, 3]):
            lens.copy_(torch.tensor(held, dtype=torch.int32))
            lse.copy_(lse64(c, q.contiguous(), new, held))
            store.fill_(-7.5)
            if g is None:
                call()
                check_weights(c, q.contiguous(), lse, new, held, w.contiguous(), torch.full((3, 2, 800), -7.5, device="cuda"))
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    call()
                store.fill_(-7.5)
            g.replay()
            check_weights(c, q.contiguous(), lse, new, held, w.contiguous(), torch.full((3, 2, 800), -7.5, device="cuda"))
    torch.cuda.current_stream().wait_stream(s)


def test_many_sequences(gpu_lib):
    """A whole batch of 4,096 short sequences."""
    S = 4096
    c = R.Cache(seqs=S, T=24, H=1, d=64, seed=15)
    ctx = c.context(2, 2)
    rng = np.random.default_rng(0)
    new, held = rng.integers(0, 3, S).tolist(), rng.integers(0, 20, S).tolist()
    q = queries(sum(new), 2, 64)
    _, lse = attend(c, ctx, q, new, held)
    w = fresh(c)
    weigh(c, ctx, q, lse, new, held, w)
    for b in range(0, S, 97):
        total = w[b, 0, :held[b] + new[b]].sum() / 2
        assert abs(float(total) - new[b]) < 1e-4 * max(1, new[b])
        assert bool((w[b, 0, held[b] + new[b]:] == -7.5).all())
    assert E.epikv_attn_get_error(ctx) == OK


def test_reported_and_skipped(gpu_lib):
    c = R.Cache(seqs=4, T=256, H=2, d=64, seed=14)
    ctx = c.context(4, 32)
    q = queries(64, 4, 64)
    lse = lse64(c, q, [32, 32], [100, 50], seqs=[0, 3])
    good = fresh(c)
    weigh(c, ctx, q, lse, [32, 32], [100, 50], good, seqs=[0, 3])
    for seqs, held, code in (([0, 9], [100, 50], E.EPIKV_DEV_BATCH), ([0, 3], [100, 225], E.EPIKV_DEV_CAPACITY)):
        w = fresh(c)
        weigh(c, ctx, q, lse, [32, 32], held, w, seqs=seqs)
        assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, code)
        assert torch.equal(w[0], good[0]) and bool((w[1:] == -7.5).all())
    table = c.c.block_table.clone()
    table[0, 2] = c.c.num_blocks
    seq_ids, cu, ln = R.batch([32], [100], [0])
    w = fresh(c)
    E.epikv_attention_weights(ctx, 0, 1, seq_ids, cu, 32, ln, E.rows(q), lse, E.weights_view(w), c.c.view(table))
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_SLOT)
    assert not w[0, :, 32:48].any()
    keep = [i for i in range(256) if not 32 <= i < 48]
    assert torch.equal(w[0][:, keep], good[0][:, keep])


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new,H,Hq,d", [(1, 2, 8, 64), (1, 3, 12, 128), (4, 2, 8, 256), (40, 2, 8, 128), (40, 1, 4, 64)])
def test_blocks_that_are_none(gpu_lib, bits, new, H, Hq, d):
    """Slots of blocks that the pool does not have receive nothing, all others what they did."""
    c = R.Cache(seqs=2, T=1600, H=H, d=d, bits=bits, seed=16)
    ctx = c.context(Hq, 40)
    held = [1500, 1201]
    q = queries(2 * new, Hq, d)
    lse = lse64(c, q, [new, new], held)
    good, w = fresh(c), fresh(c)
    weigh(c, ctx, q, lse, [new, new], held, good)
    table = c.c.block_table.clone()
    gone = torch.zeros(2, 1600 + 16, dtype=torch.bool, device="cuda")
    for s, blocks in ((0, (0, 16, 31, 40)), (1, (7, 60, 75))):
        for b, bad in zip(blocks, (c.c.num_blocks, -1, 1 << 30, -(1 << 31))):
            table[s, b] = bad
            gone[s, 16 * b:16 * b + 16] = True
    seq_ids, cu, ln = R.batch([new, new], held)
    E.epikv_attention_weights(ctx, 0, 2, seq_ids, cu, new, ln, E.rows(q), lse, E.weights_view(w), c.c.view(table))
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_SLOT)
    for s in range(2):
        top = held[s] + new
        here = gone[s, :top]
        assert not w[s, :, :top][:, here].any()
        assert torch.equal(w[s, :, :top][:, ~here], good[s, :, :top][:, ~here])
        assert bool((w[s, :, top:] == -7.5).all())


def test_two_contexts_at_once(gpu_lib):
    """Calls of two contexts on two streams, a captured one and an eager one: the bits of each alone."""
    calls = []
    for bits, new, seed in ((16, [1, 1, 1], 17), (4, [60, 3, 1], 18)):
        c = R.Cache(seqs=3, T=2600, H=4, d=128, bits=bits, seed=seed)
        ctx = c.context(16, 60)
        held = [2500, 17, 1300]
        q = queries(sum(new), 16, 128, seed)
        o, lse, w = torch.empty_like(q), torch.empty(sum(new), 16, device="cuda"), fresh(c)
        seq_ids, cu, ln = R.batch(new, held)
        s = torch.cuda.Stream()

        def call(c=c, ctx=ctx, q=q, o=o, lse=lse, w=w, seq_ids=seq_ids, cu=cu, ln=ln, s=s, most=max(new)):
            E.epikv_attention_chunk(ctx, 0, 3, seq_ids, cu, most, ln, E.rows(q), E.rows(o), c.c.view(), lse=lse, stream=s)
            E.epikv_attention_weights(ctx, 0, 3, seq_ids, cu, most, ln, E.rows(q), lse, E.weights_view(w), c.c.view(), stream=s)
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        calls.append((call, s, (o, lse, w), [x.clone() for x in (o, lse, w)], ctx))
    (eager, _, _, _, _), (other, s, _, _, _) = calls
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        other()
    for _, _, got, _, _ in calls:
        for x in got:
            x.zero_()
    calls[0][2][2].fill_(-7.5), calls[1][2][2].fill_(-7.5)
    torch.cuda.synchronize()
    for _ in range(20):
        eager()
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for _, _, got, want, ctx in calls:
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert E.epikv_attn_get_error(ctx) == OK


# ------------------------------------------------------------------ eviction by the weights
def plain_kept(score, K, prefill, cap=128):
    n = len(score)
    if n <= K:
        return np.arange(n)
    P = min(prefill, n)
    Rw = min(cap, K // 4, max(0, K - P))
    M = max(0, K - P - Rw)
    cand = np.arange(P, n - Rw)
    key = np.where(np.isnan(score[cand]), -np.inf, score[cand])
    top = cand[np.argsort(-key, kind="stable")[:M]]
    return np.sort(np.concatenate([np.arange(P), top, np.arange(n - Rw, n)]))


class Loop:
    """A cache of known rows that is updated, weighed, selected and compacted as a decode loop does."""

    def __init__(self, kinds, *, S=3, T=400, H=2, d=64, L=2, policies=None, prefill=(0, 5, 17)):
        self.S, self.H, self.T = S, H, T
        self.cache = KVCache(E.EPIKV_LAYOUT_PAGED, L, H, d, max_seqs=S, max_tokens=T)
        cfg = E.make_config(max_seqs=S, max_cache_tokens=T, max_new_tokens=T, num_layers=L, num_kv_heads=H, head_dim=d,
                            hidden=64, n_band_a=1, n_band_b=1, score_kinds=kinds)
        self.ws = torch.empty(E.epikv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        self.ctx = E.epikv_init(cfg, self.ws, self.ws.numel())
        self.kinds = kinds
        self.g = torch.Generator(device="cuda").manual_seed(3)
        for s in range(S):
            E.epikv_seq_reset(self.ctx, s, prefill[s], E.EPIKV_SCORE_WEIGHT if policies is None else policies[s])
        self.prefill = prefill
        self.score = [np.zeros(0, np.float32) for _ in range(S)]
        self.pos = [np.zeros(0, np.int64) for _ in range(S)]
        self.seen = [0] * S

    def update(self, seqs, new):
        seq_ids, cu, _ = R.batch(new, [0] * len(new), seqs)
        n = sum(new)
        hidden = [torch.randn(n, 64, generator=self.g, device="cuda").to(torch.bfloat16) for _ in range(2)]
        for s, m in zip(seqs, new):
            slots = np.arange(len(self.score[s]), len(self.score[s]) + m)
            for kind in (0, 1):
                for l in range(self.cache.L):
                    p = torch.arange(self.seen[s], self.seen[s] + m, device="cuda").float()[:, None, None]
                    self.cache.write_layer_rows(kind, s, l, slots, (p + 0.25 * kind).expand(m, self.H, self.cache.d).to(
                        torch.bfloat16))
            self.score[s] = np.concatenate([self.score[s], np.zeros(m, np.float32)])
            self.pos[s] = np.concatenate([self.pos[s], np.arange(self.seen[s], self.seen[s] + m)])
            self.seen[s] += m
        E.epikv_score_update(self.ctx, len(seqs), seq_ids, cu, max(new),
                             E.hidden_view(hidden, 64) if self.kinds & 5 else None, self.cache.view() if self.kinds & 58 else None)

    def weigh(self, seqs, decay, heads=None):
        w = torch.rand(self.S, self.H, self.T, generator=self.g, device="cuda").pow(8)
        E.epikv_weigh(self.ctx, len(seqs), R.batch([0] * len(seqs), [0] * len(seqs), seqs)[0], E.weights_view(w), decay,
                      n_heads=heads)
        wn = w.cpu().numpy()
        for s in seqs:
            n = len(self.score[s])
            total = wn[s, 0, :n].copy()
            for h in range(1, self.H if heads is None else heads):
                total = total + wn[s, h, :n]
            self.score[s] = (np.float32(decay) * self.score[s]).astype(np.float32) + total

    def check(self):
        for s in range(self.S):
            pos, score, n = E.epikv_read_slots(self.ctx, s, E.EPIKV_SCORE_WEIGHT, self.T)
            assert n == len(self.score[s])
            np.testing.assert_array_equal(np.asarray(pos), self.pos[s])
            np.testing.assert_array_equal(np.asarray(score, np.float32).view(np.int32), self.score[s].view(np.int32))

    def evict(self, seqs, budgets, by_weight=lambda s: True):
        seq_ids = R.batch([0] * len(seqs), [0] * len(seqs), seqs)[0]
        bud = torch.tensor(budgets, dtype=torch.int32, device="cuda")
        kept = torch.full((len(seqs), self.T), -1, dtype=torch.int32, device="cuda")
        n_kept = torch.zeros(len(seqs), dtype=torch.int32, device="cuda")
        E.epikv_select(self.ctx, len(seqs), seq_ids, bud, None, kept, self.T, n_kept)
        E.epikv_compact(self.ctx, len(seqs), seq_ids, kept, self.T, self.cache.view())
        kept, n_kept = kept.cpu().numpy(), n_kept.cpu().numpy()
        for i, (s, K) in enumerate(zip(seqs, budgets)):
            got = kept[i, :n_kept[i]] if len(self.score[s]) > K else np.arange(len(self.score[s]))
            if by_weight(s):
                np.testing.assert_array_equal(got, plain_kept(self.score[s], K, self.prefill[s]))
            self.score[s], self.pos[s] = self.score[s][got], self.pos[s][got]
            for kind in (0, 1):
                rows = self.cache.rows(kind, s, np.arange(len(got))).float()
                want = torch.tensor(self.pos[s], device="cuda").float()[:, None, None, None] + 0.25 * kind
                assert torch.equal(rows, want.to(torch.bfloat16).float().expand_as(rows))


@pytest.mark.parametrize("kinds", [E.EPIKV_SCORE_WEIGHT, E.EPIKV_SCORE_WEIGHT | E.EPIKV_SCORE_BANDZ,
                                   E.EPIKV_SCORE_WEIGHT | E.EPIKV_SCORE_LAGKV | E.EPIKV_SCORE_KVVAL,
                                   E.EPIKV_SCORE_WEIGHT | 63])
@pytest.mark.parametrize("step", [1, 37])
def test_evict_by_weight(gpu_lib, kinds, step):
    """Prompts, then steps of one or more tokens: scores, kept slots and rows over several evictions, bit for bit."""
    lp = Loop(kinds)
    lp.update([0, 1, 2], [150, 64, 201])
    lp.check()
    lp.weigh([0, 1, 2], 1.0)
    lp.check()
    lp.evict([0, 1, 2], [100, 100, 90])
    lp.check()
    for i in range(4):
        seqs = [0, 1, 2] if i % 2 else [2, 0]
        lp.update(seqs, [step] * len(seqs))
        lp.check()
        lp.weigh(seqs, 0.9, heads=None if i else 1)
        lp.weigh(seqs, 1.0)
        lp.check()
        lp.evict(seqs, [90] * len(seqs))
        lp.check()
    assert E.epikv_get_error(lp.ctx) == OK


def test_sequences_of_other_kinds_beside(gpu_lib):
    """One batch, one sequence by its weights, one by band z-scores: the weights move with the tokens of both."""
    lp = Loop(E.EPIKV_SCORE_WEIGHT | E.EPIKV_SCORE_BANDZ, policies=(E.EPIKV_SCORE_WEIGHT, E.EPIKV_SCORE_BANDZ,
                                                                     E.EPIKV_SCORE_WEIGHT))
    lp.update([0, 1, 2], [300, 280, 390])
    lp.weigh([0, 1, 2], 0.5)
    lp.evict([0, 1, 2], [128, 128, 255], by_weight=lambda s: s != 1)
    lp.check()
    assert E.epikv_get_error(lp.ctx) == OK


@pytest.mark.parametrize("T", [2000, 30000])
def test_large_evictions(gpu_lib, T):
    """Both selection kernels: caches of one CTA and of a cluster."""
    lp = Loop(E.EPIKV_SCORE_WEIGHT, S=2, T=T, H=1, d=64, L=1, prefill=(0, 40))
    lp.update([1, 0], [T, T - 77])
    lp.weigh([0, 1], 0.0)
    lp.evict([0, 1], [T // 3, T // 2])
    lp.check()


def test_reset_and_order(gpu_lib):
    """A reset sequence starts at 0 again; an update before the compaction is reported as with the other kinds."""
    lp = Loop(E.EPIKV_SCORE_WEIGHT)
    lp.update([0, 1, 2], [150, 150, 150])
    lp.weigh([0, 1, 2], 1.0)
    E.epikv_seq_reset(lp.ctx, 1, 5, E.EPIKV_SCORE_WEIGHT)
    lp.score[1], lp.pos[1], lp.seen[1] = np.zeros(0, np.float32), np.zeros(0, np.int64), 0
    lp.update([1], [40])
    lp.check()
    seq_ids, cu, _ = R.batch([1], [0], [0])
    kept = torch.zeros(1, 400, dtype=torch.int32, device="cuda")
    E.epikv_select(lp.ctx, 1, seq_ids, torch.tensor([50], dtype=torch.int32, device="cuda"), None, kept, 400, None)
    E.epikv_score_update(lp.ctx, 1, seq_ids, cu, 1, None, None)
    assert E.epikv_get_error(lp.ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_KEPT)
    bad = torch.tensor([7], dtype=torch.int32, device="cuda")
    E.epikv_weigh(lp.ctx, 1, bad, E.weights_view(torch.zeros(3, 2, 400, device="cuda")))
    assert E.epikv_get_error(lp.ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_BATCH)
    cu[1] = 399
    E.epikv_score_update(lp.ctx, 1, seq_ids, cu, 400, None, None)
    assert E.epikv_get_error(lp.ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_CAPACITY)


def test_step_with_weights(gpu_lib):
    """epikv_step of a context with the WEIGHT kind selects by the weights so far; new tokens' are 0."""
    lp = Loop(E.EPIKV_SCORE_WEIGHT, S=1, prefill=(0,))
    lp.update([0], [200])
    lp.weigh([0], 1.0)
    seq_ids, cu, _ = R.batch([10], [0], [0])
    n_out = torch.zeros(1, dtype=torch.int32, device="cuda")
    E.epikv_step(lp.ctx, 1, seq_ids, cu, 10, torch.tensor([64], dtype=torch.int32, device="cuda"), None, None, lp.cache.view(),
                 n_out)
    score = np.concatenate([lp.score[0], np.zeros(10, np.float32)])
    kept = plain_kept(score, 64, 0)
    pos, got, n = E.epikv_read_slots(lp.ctx, 0, E.EPIKV_SCORE_WEIGHT, 400)
    assert n == 64 and int(n_out) == 64
    np.testing.assert_array_equal(np.asarray(pos), kept)
    np.testing.assert_array_equal(np.asarray(got, np.float32), score[kept])


def test_refusals_of_weigh(gpu_lib):
    def context(kinds):
        cfg = E.make_config(max_seqs=3, max_cache_tokens=50, max_new_tokens=4, score_kinds=kinds)
        space = torch.empty(E.epikv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        return E.epikv_init(cfg, space, space.numel()), space
    (ctx, _a), (other, _b) = context(E.EPIKV_SCORE_WEIGHT), context(63)
    t = torch.zeros(3, 2, 50, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    w, p = E.weights_view(t), ids.data_ptr()
    nan, inf = float("nan"), float("inf")
    bad = [(other, 1, p, w, 2, 1.0), (None, 1, p, w, 2, 1.0), (ctx, -1, p, w, 2, 1.0), (ctx, 4, p, w, 2, 1.0), (ctx, 1, None, w, 2, 1.0),
           (ctx, 1, p, None, 2, 1.0), (ctx, 1, p, E.epikv_weights(None, 100, 50), 2, 1.0),
           (ctx, 1, p, E.epikv_weights(t.data_ptr() + 1, 100, 50), 2, 1.0), (ctx, 1, p, E.epikv_weights(t.data_ptr(), -100, 50), 2, 1.0),
           (ctx, 1, p, E.epikv_weights(t.data_ptr(), 100, -50), 2, 1.0), (ctx, 1, p, w, 0, 1.0), (ctx, 1, p, w, -1, 1.0),
           (ctx, 1, p, w, 1025, 1.0)] + [(ctx, 1, p, w, 2, d) for d in (-0.5, 1.5, nan, inf, -inf)]
    for a in bad:
        assert gpu_lib.epikv_weigh(*a, None) == E.EPIKV_EINVAL, a
    assert gpu_lib.epikv_weigh(ctx, 0, None, None, 0, 9.0, None) == E.EPIKV_OK      # no sequences
    assert gpu_lib.epikv_weigh(ctx, 1, p, w, 2, 0.0, None) == E.EPIKV_OK
    assert E.epikv_get_error(ctx) == OK
    for c in (ctx, other):
        E.epikv_destroy(c)


def test_weigh_of_sequences_that_are_none(gpu_lib):
    """Reported, and the others' scores are as without them."""
    cfg = E.make_config(max_seqs=2, max_cache_tokens=50, max_new_tokens=4, score_kinds=E.EPIKV_SCORE_WEIGHT)
    space = torch.empty(E.epikv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ctx = E.epikv_init(cfg, space, space.numel())
    ids = torch.tensor([7, 1], dtype=torch.int32, device="cuda")
    w = torch.rand(2, 1, 50, device="cuda")
    E.epikv_score_update(ctx, 1, ids[1:].clone(), torch.tensor([0, 3], dtype=torch.int32, device="cuda"), 3, None, None)
    E.epikv_weigh(ctx, 2, ids, E.weights_view(w))
    assert E.epikv_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_BATCH)
    assert E.epikv_read_slots(ctx, 1, E.EPIKV_SCORE_WEIGHT, 50)[1] == w[1, 0, :3].tolist()
    E.epikv_destroy(ctx)


def test_weigh_between_selection_and_compaction(gpu_lib):
    """The slots are others already: reported, the scores stay, and a sequence that was not cut takes its weights."""
    lp = Loop(E.EPIKV_SCORE_WEIGHT)
    lp.update([0, 1, 2], [150, 40, 300])
    lp.weigh([0, 1, 2], 1.0)
    seq_ids = R.batch([0] * 3, [0] * 3)[0]
    kept = torch.full((3, lp.T), -1, dtype=torch.int32, device="cuda")
    E.epikv_select(lp.ctx, 3, seq_ids, torch.full((3,), 100, dtype=torch.int32, device="cuda"), None, kept, lp.T, None)
    for s in (0, 2):
        got = plain_kept(lp.score[s], 100, lp.prefill[s])
        lp.score[s], lp.pos[s] = lp.score[s][got], lp.pos[s][got]
    lp.check()
    before = [x.copy() for x in lp.score]
    lp.weigh([0, 1, 2], 0.5)
    lp.score[0], lp.score[2] = before[0], before[2]
    assert E.epikv_get_error(lp.ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_KEPT)
    lp.check()
    E.epikv_compact(lp.ctx, 3, seq_ids, kept, lp.T, lp.cache.view())
    lp.weigh([0, 1, 2], 0.5)
    lp.check()
    assert E.epikv_get_error(lp.ctx) == OK


@pytest.mark.parametrize("new", [2, 60])
@pytest.mark.parametrize("bits,scale,keys", [(4, 0.0, 2.0 ** -60), (4, 0.0, 2.0 ** -100), (16, 3e38, 1.0), (4, 3e38, 1.0)])
def test_factors_that_leave_the_normal_numbers(gpu_lib, bits, scale, keys, new):
    """Query rows of zeros and of tiny numbers beside small or large scales."""
    ks = None if bits == 16 else torch.tensor([[[keys, 1.0]], [[1.0, 0.5]]], device="cuda")
    c = R.Cache(seqs=1, T=300, H=2, d=64, bits=bits, kv_scale=ks, seed=23)
    ctx = c.context(4, 60, softmax_scale=scale)
    q = queries(new, 4, 64)
    q[1::2] = (q[1::2].float() * 2.0 ** -120).to(torch.bfloat16)
    q[::4 if scale < 1 else 1] = 0
    lse = lse64(c, q, [new], [200], scale=scale or None)
    w = fresh(c)
    before = w.clone()
    weigh(c, ctx, q, lse, [new], [200], w)
    check_weights(c, q, lse, [new], [200], w, before, scale=scale or None)
    assert bool(w[:, :, :200 + new].isfinite().all())


@pytest.mark.parametrize("kinds", [E.EPIKV_SCORE_WEIGHT, E.EPIKV_SCORE_WEIGHT | E.EPIKV_SCORE_BANDZ | E.EPIKV_SCORE_HSVAR])
@pytest.mark.parametrize("T,C", [(700, 8), (700, 65536), (30000, 16)])
def test_chunks_of_positions_by_weight(gpu_lib, kinds, T, C):
    """Chunk-level selection ranks by the weights' column, whichever columns stand before it."""
    cfg = E.make_config(max_seqs=2, max_cache_tokens=T, max_new_tokens=T, hidden=64, n_band_a=1, n_band_b=1, score_kinds=kinds,
                        select_chunk=C)
    ws = torch.empty(E.epikv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ctx = E.epikv_init(cfg, ws, ws.numel())
    for s in range(2):
        E.epikv_seq_reset(ctx, s, 5 * s, E.EPIKV_SCORE_WEIGHT)
    g = torch.Generator(device="cuda").manual_seed(24)
    new = [T, T - 33]
    hidden = [torch.randn(sum(new), 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    seq_ids, cu, _ = R.batch(new, [0, 0])
    E.epikv_score_update(ctx, 2, seq_ids, cu, T, E.hidden_view(hidden, 64), None)
    w = torch.rand(2, 1, T, generator=g, device="cuda").pow(8)
    w[0, 0, 55] = float("nan")
    E.epikv_weigh(ctx, 2, seq_ids, E.weights_view(w))
    before = [E.epikv_read_slots(ctx, s, E.EPIKV_SCORE_WEIGHT, T) for s in range(2)]
    budgets = [T // 2, T // 5]
    kept = torch.full((2, T), -1, dtype=torch.int32, device="cuda")
    n_kept = torch.zeros(2, dtype=torch.int32, device="cuda")
    E.epikv_select(ctx, 2, seq_ids, torch.tensor(budgets, dtype=torch.int32, device="cuda"), None, kept, T, n_kept)
    for s in range(2):
        pos, score, n = before[s]
        assert n == new[s]
        np.testing.assert_array_equal(np.asarray(score, np.float32), w[s, 0, :n].cpu().numpy())
        want = oracle_kept(np.asarray(score), np.asarray(pos), budgets[s], 5 * s, 128, C)
        assert kept[s, :int(n_kept[s])].tolist() == list(want)
        after = E.epikv_read_slots(ctx, s, E.EPIKV_SCORE_WEIGHT, T)
        np.testing.assert_array_equal(np.asarray(after[1], np.float32), w[s, 0].cpu().numpy()[want])
    assert E.epikv_get_error(ctx) == OK


def test_more_work_than_is_counted(gpu_lib):
    """The entry that takes the sum to the limit and those behind it are reported and store nothing; those before it are done."""
    T, most = 1 << 24, 1 << 20
    c = R.Cache(seqs=3, T=64, H=1, d=64, seed=25)
    cfg = E.make_attn_config(max_seqs=3, max_cache_tokens=T, max_new_tokens=most, num_layers=1, num_heads=64, num_kv_heads=1,
                             head_dim=64)
    ws = torch.empty(E.epikv_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ctx = E.epikv_attn_init(cfg, ws, ws.numel())
    new, held = [3, most, 2], [50, T - most, 40]
    q = queries(3, 64, 64)
    seq_ids, cu, ln = R.batch(new, held)
    lse = lse64(c, q, [3], [50])
    w = torch.full((3, 1, 64), -7.5, device="cuda")
    before = w.clone()
    E.epikv_attention_weights(ctx, 0, 3, seq_ids, cu, most, ln, E.rows(q), lse, E.epikv_weights(w.data_ptr(), T, T), c.c.view())
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_CAPACITY)
    check_weights(c, q, lse, [3], [50], w, before)
    o, l = torch.full_like(q, float("nan")), torch.full((3, 64), float("nan"), device="cuda")
    E.epikv_attention_chunk(ctx, 0, 3, seq_ids, cu, most, ln, E.rows(q), E.rows(o), c.c.view(), lse=l)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_CAPACITY)
    check_attention(c, q, o, l, [3], [50])
    assert bool(o[3:].isnan().all()) and bool(l[3:].isnan().all())
