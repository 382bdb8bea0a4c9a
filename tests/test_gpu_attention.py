"""epikv_attention against float64: head layouts, lengths from none to thousands, ragged batches, pages that end inside
a tile, rows that see nothing, what stands in slots that a row does not see, and what is refused or reported."""
import math

import pytest
import torch

from paper_2606_26472_gb300 import epikv as E
from paper_2606_26472_gb300.cache import KVCache

from . import cache_ops as R

pytestmark = pytest.mark.gpu


def run(c, ctx, q, new, held, *, layer=0, seqs=None, causal=True, max_new=None, lse=True, out=None, stream=None):
    seq_ids, cu, ln = R.batch(new, held, seqs)
    n = q.shape[0]
    o = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    l = torch.full((n, q.shape[1]), float("nan"), device="cuda") if lse else None
    E.epikv_attention(ctx, layer, len(new), seq_ids, cu, max(new) if max_new is None else max_new, ln, E.rows(q),
                      E.rows(o), c.c.view(), lse=l, causal=causal, stream=stream)
    return o, l


def check(c, q, o, l, new, held, *, layer=0, seqs=None, causal=True, scale=None, what=""):
    scale = 1 / math.sqrt(c.d) if scale is None else scale
    t = 0
    for b, n in enumerate(new):
        s = b if seqs is None else seqs[b]
        top = held[b] + (n if causal else 0)
        k, v = c.read(0, layer, s, top), c.read(1, layer, s, top)
        limits = [held[b] + (i + 1 if causal else 0) for i in range(n)]
        ref = R.attention64(q[t:t + n], k, v, limits, scale)
        R.assert_attention_close(o[t:t + n], l[t:t + n] if l is not None else None, ref, f"{what} entry {b}")
        t += n


def queries(n, Hq, d, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, Hq, d, generator=g, device="cuda").to(torch.bfloat16)


SHAPES = [(8, 32, 128), (1, 1, 64), (1, 8, 128), (2, 14, 128), (3, 3, 64), (4, 32, 64), (5, 20, 128), (2, 4, 256),
          (4, 32, 256), (11, 11, 64), (16, 32, 64), (7, 7, 128), (1, 71, 64)]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", SHAPES)
def test_single_tokens(gpu_lib, bits, H, Hq, d):
    """One new token of each sequence: lengths around the edges of tiles and pages."""
    held = [0, 1, 14, 15, 16, 17, 30, 31, 32, 33, 63, 64, 127, 128, 300, 1023]
    for block in (16, 0, 7):
        c = R.Cache(seqs=16, T=1030, H=H, d=d, bits=bits, block=block, seed=H * d)
        ctx = c.context(Hq, 1)
        q = queries(16, Hq, d)
        seqs = list(range(15, -1, -1))
        o, l = run(c, ctx, q, [1] * 16, held, seqs=seqs)
        check(c, q, o, l, [1] * 16, held, seqs=seqs, what=f"block {block}")
        assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", SHAPES)
def test_several_tokens(gpu_lib, bits, H, Hq, d):
    """Ragged new tokens, none among them, over short and long caches: the causal edge at every place of a tile."""
    new, held = [3, 0, 1, 17, 47, 8], [0, 5, 200, 31, 77, 1500]
    for block in (16, 0, 48):
        c = R.Cache(seqs=6, T=1600, H=H, d=d, bits=bits, block=block, seed=H + d)
        ctx = c.context(Hq, 64)
        q = queries(sum(new), Hq, d)
        o, l = run(c, ctx, q, new, held)
        check(c, q, o, l, new, held, what=f"block {block}")
        assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("H,Hq,d", [(8, 32, 128), (11, 11, 64), (4, 16, 64), (2, 4, 128), (3, 6, 64), (1, 8, 128), (9, 9, 128),
                                     (5, 5, 64)])
def test_large_tiles(gpu_lib, H, Hq, d):
    """Caches that could hold enough for the largest tiles of 4-bit rows, short and longer entries."""
    held = [0, 15, 63, 64, 127, 128, 700, 5000]
    for block in (16, 0):
        c = R.Cache(seqs=8, T=20000, H=H, d=d, bits=4, block=block, seed=H + d)
        ctx = c.context(Hq, 1)
        q = queries(8, Hq, d)
        o, l = run(c, ctx, q, [1] * 8, held)
        check(c, q, o, l, [1] * 8, held, what=f"block {block}")
        assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("bits", [16, 4])
def test_prompt_and_long(gpu_lib, bits):
    c = R.Cache(seqs=2, T=20000, H=2, d=128, bits=bits, seed=5)
    ctx = c.context(8, 300)
    q = queries(301, 8, 128)
    o, l = run(c, ctx, q, [300, 1], [0, 19999])
    check(c, q, o, l, [300, 1], [0, 19999])


@pytest.mark.parametrize("bits", [16, 4])
def test_prefix_without_the_new_tokens(gpu_lib, bits):
    """causal=0: every query sees the held slots; none held: zeros and -inf; two parts join by their lse."""
    c = R.Cache(seqs=3, T=400, H=2, d=64, bits=bits, seed=2)
    ctx = c.context(6, 5)
    new, held = [5, 2, 3], [0, 399, 18]
    q = queries(10, 6, 64)
    o, l = run(c, ctx, q, new, held, causal=False)
    check(c, q, o, l, new, held, causal=False)
    assert not o[:5].any() and bool((l[:5] == -math.inf).all())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new", [1, 6, 40])
def test_unseen_slots_do_not_reach_a_row(gpu_lib, bits, new):
    """Slots behind a row's last one hold NaN: rows before them are untouched, rows that see them are NaN."""
    held, T = 45, 128
    c = R.Cache(seqs=1, T=T, H=2, d=128, bits=bits, seed=3)
    ctx = c.context(8, 64)
    q = queries(new, 8, 128)
    for first_bad in sorted({held + new, held + new // 2 + 1, held + 1}):
        if first_bad > held + new:
            continue
        saved = [c.raw(w).clone() for w in range(2)]
        idx = c.index(0, 0, torch.arange(first_bad, T))
        for w in range(2):
            c.raw(w)[idx] = 0x7F if bits == 4 else 0xFF
        o, l = run(c, ctx, q, [new], [held])
        good = first_bad - held
        k, v = c.read(0, 0, 0, held + new), c.read(1, 0, 0, held + new)
        ref = R.attention64(q[:good], k[:first_bad], v[:first_bad], [held + i + 1 for i in range(good)], 128 ** -0.5)
        R.assert_attention_close(o[:good], l[:good], ref, f"bad from {first_bad}")
        assert bool(o[good:].isnan().all())
        for w in range(2):
            c.raw(w).copy_(saved[w])


@pytest.mark.parametrize("bits", [16, 4])
def test_values_of_one_unseen_row(gpu_lib, bits):
    """An infinite value in the newest token's V alone, finite keys: earlier rows stay as they were."""
    c = R.Cache(seqs=1, T=64, H=1, d=64, bits=bits, seed=4)
    ctx = c.context(4, 8)
    q = queries(8, 4, 64)
    before, _ = run(c, ctx, q, [8], [30])
    c.raw(1)[c.index(0, 0, torch.arange(35, 36))] = 0x7F if bits == 4 else 0xFF
    after, _ = run(c, ctx, q, [8], [30])
    assert torch.equal(before[:5], after[:5]) and bool(after[5:].isnan().all())


def unbounded_reference(c, q, new, held, scale, what):
    """float64 outputs of the batch, infinities among the values included: the sums of products as they are."""
    outs, t = [], 0
    for b, n in enumerate(new):
        top = held[b] + n
        k, v = c.read(0, 0, b, top), c.read(1, 0, b, top)
        outs.append(R.attention64(q[t:t + n], k, v, [held[b] + i + 1 for i in range(n)], scale))
        t += n
    return outs


@pytest.mark.parametrize("block", [16, 7, 0])
@pytest.mark.parametrize("H,Hq,d", [(8, 32, 128), (9, 9, 128), (9, 18, 64), (1, 8, 128), (3, 6, 64), (6, 6, 256), (5, 5, 256)])
@pytest.mark.parametrize("new", [1, 5])
def test_infinite_values(gpu_lib, H, Hq, d, block, new):
    """Infinities of both signs in V's slots (seen by all rows, by some, by none; of one part of a long entry or the
    other): an output is the infinity that its row sees, NaN where it sees both signs, and as ever in other channels."""
    held = [3, 16, 40, 900, 2500]
    c = R.Cache(seqs=5, T=2600, H=H, d=d, bits=16, block=block, seed=H + d)
    pool = c.c.v.view(-1, H, d)
    inf = math.inf
    for b, n in enumerate(held):
        for slot, h, ch, x in ((0, 0, 0, inf), (n // 2, H - 1, 1, -inf), (n // 3, H - 1, d - 1, inf), (n, 0, 5, inf),
                               (n - 1, H // 2, 7, inf), (n // 2, H // 2, 7, -inf), (n + new - 1, H - 1, d - 2, -inf),
                               (n + new, 0, 9, inf), (n + new + 1, H - 1, 3, math.nan)):
            pool[c.index(0, b, torch.tensor([slot])), h, ch] = x
    ctx = c.context(Hq, 8)
    q = queries(5 * new, Hq, d)
    o, l = run(c, ctx, q, [new] * 5, held)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)
    seen = 0
    for b, ref in enumerate(unbounded_reference(c, q, [new] * 5, held, d ** -0.5, "")):
        want, lse, big, qk = ref
        part, lpart = o[b * new:(b + 1) * new], l[b * new:(b + 1) * new]
        odd = ~want.isfinite()
        seen += int(want.isinf().sum())
        assert torch.equal(part[odd].double().nan_to_num(nan=7.0), want[odd].nan_to_num(nan=7.0)), f"entry {b}"
        assert part[~odd].isfinite().all(), f"entry {b}"
        zero = torch.zeros_like(want)
        R.assert_attention_close(torch.where(odd, zero, part.double()), lpart,
                                 (torch.where(odd, zero, want), lse, torch.where(odd, zero, big), qk), f"entry {b}")
    assert seen >= 5 * new


@pytest.mark.parametrize("H,d", [(2, 64), (8, 128), (9, 128)])
def test_infinite_values_of_the_least_probable_slots(gpu_lib, H, d):
    """Probabilities far below 32 bits' least number are not 0: an infinity there is the output, whether the maximum
    moves away from it within a block's share of the slots, between its warps or between blocks."""
    T = 700
    c = R.Cache(seqs=1, T=T, H=H, d=d, bits=16, seed=6)
    ramp = torch.linspace(-20, 20, T, device="cuda")
    keys, vals = c.c.k.view(-1, H, d), c.c.v.view(-1, H, d)
    rows = c.index(0, 0, torch.arange(T))
    keys[rows] = 0
    keys[rows, :, 0] = ramp[:, None].to(torch.bfloat16)
    q = torch.zeros(1, H, d, device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 10.0
    for slot, ch, x in ((0, 3, math.inf), (5, 4, -math.inf), (T // 2, 5, math.inf), (1, 6, math.inf), (2, 6, -math.inf)):
        vals[rows[slot], :, ch] = x
    ctx = c.context(H, 1, softmax_scale=1.0)
    o, l = run(c, ctx, q, [1], [T - 1])
    want = R.attention64(q, c.read(0, 0, 0, T), c.read(1, 0, 0, T), [T], 1.0)[0]
    odd = ~want.isfinite()
    assert int(want.isinf().sum()) == 3 * H and int(want.isnan().sum()) == H
    assert torch.equal(o[odd].double().nan_to_num(nan=7.0), want[odd].nan_to_num(nan=7.0))
    assert o[~odd].isfinite().all()


def test_infinite_value_of_a_slot_of_no_weight(gpu_lib):
    """A score of minus infinity is a probability of exactly 0, which an infinite value makes NaN; the row's other
    channels and a row whose score is finite are as ever."""
    c = R.Cache(seqs=1, T=40, H=1, d=64, bits=16, seed=3)
    keys, vals = c.c.k.view(-1, 1, 64), c.c.v.view(-1, 1, 64)
    row = c.index(0, 0, torch.tensor([4]))
    keys[row] = 0
    keys[row, 0, 2] = -math.inf
    vals[row, 0, 10] = math.inf
    q = queries(1, 2, 64)
    q[0, :, 2] = 1.0
    ctx = c.context(2, 1)
    o, l = run(c, ctx, q, [1], [30])
    k, v = c.read(0, 0, 0, 31), c.read(1, 0, 0, 31)
    assert o[0, :, 10].isnan().all()
    k[4], v[4] = 0, 0
    p = torch.einsum("hd,td->ht", q[0].double(), k[:, 0]) * 64 ** -0.5
    p[:, 4] = -math.inf
    want = torch.softmax(p, -1) @ v[:, 0]
    rest = [ch for ch in range(64) if ch != 10]
    big = torch.softmax(p, -1) @ v[:, 0].abs()
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 1e-4) * big
    assert bool(((o[0].double() - want).abs() <= tol)[:, rest].all())


@pytest.mark.parametrize("bits", [16, 4])
def test_large_scores(gpu_lib, bits):
    """Scores in the hundreds of both signs, growing along the sequence: the running maximum moves at every tile."""
    c = R.Cache(seqs=1, T=700, H=2, d=64, bits=bits, seed=6)
    ramp = torch.linspace(-40, 40, 700, device="cuda")
    x = torch.ones(c.raw(0).shape[0], 2, 64, device="cuda")
    x[c.index(0, 0, torch.arange(700))] = ramp[:, None, None].expand(-1, 2, 64)
    c.put(c.c.k, x.to(torch.bfloat16), 0)
    ctx = c.context(4, 2)
    for sign in (1.0, -1.0):
        q = (queries(2, 4, 64).abs() + 0.5) * sign
        q = q.to(torch.bfloat16)
        o, l = run(c, ctx, q, [2], [690])
        check(c, q, o, l, [2], [690], what=f"sign {sign}")


@pytest.mark.parametrize("bits", [16, 4])
def test_query_magnitudes(gpu_lib, bits):
    c = R.Cache(seqs=1, T=100, H=2, d=128, bits=bits, seed=7)
    for mag in (0.0, 1e-30, 1e-3, 300.0, 1e5):
        ctx = c.context(8, 1, softmax_scale=0.0 if mag <= 1 else 0.05 / mag)
        q = (queries(1, 8, 128).float() * mag).to(torch.bfloat16)
        o, l = run(c, ctx, q, [1], [99])
        check(c, q, o, l, [1], [99], scale=None if mag <= 1 else float(torch.tensor(0.05 / mag)), what=f"|q| {mag}")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("down", [12, 19, 27])
def test_queries_of_unlike_channels(gpu_lib, d, down):
    """A row's largest channel meets keys of 0, channels 2^down smaller make the scores: each keeps its 8 bits."""
    s = torch.full((2, 1, 2), 2.0 ** (down - 13), device="cuda")
    c = R.Cache(seqs=1, T=300, H=2, d=d, bits=4, kv_scale=s, seed=16, spread=1.0)
    g = torch.Generator(device="cuda").manual_seed(17)
    k = torch.randn(c.raw(0).shape[0], 2, d, generator=g, device="cuda") * 500.0 * float(s[0, 0, 0])
    k[..., :16] = 0
    c.put(c.c.k, k.to(torch.bfloat16), 0)
    for first in (1.0, 1.7, 3e-20, 1e30):
        q = queries(2, 8, d).float() * 2.0 ** -down
        q[..., :16] = 0
        q[..., 3] = 1.0
        q = (q * first).to(torch.bfloat16)
        scale = float(torch.tensor(8.0 / d ** 0.5 / first, dtype=torch.float32))
        ctx = c.context(8, 2, softmax_scale=scale)
        o, l = run(c, ctx, q, [2], [290])
        check(c, q, o, l, [2], [290], scale=scale, what=f"first {first}")


def test_head_scales(gpu_lib):
    s = torch.rand(2, 2, 4, device="cuda") * 3 + 0.01
    c = R.Cache(seqs=2, T=200, H=4, d=64, bits=4, layers=2, kv_scale=s, seed=8)
    ctx = c.context(8, 3)
    q = queries(4, 8, 64)
    o, l = run(c, ctx, q, [3, 1], [150, 20], layer=1)
    check(c, q, o, l, [3, 1], [150, 20], layer=1)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("mag", [0.0, 1e-38, 1e-30, 1.0])
@pytest.mark.parametrize("held", [9, 40, 700])
def test_scores_of_next_to_nothing(gpu_lib, bits, mag, held):
    """Queries, head scales and softmax scales so small that their product is no 32-bit number: the scores are 0, and
    the row is the mean of the values that it sees, tiles that it sees in part among them."""
    H, d = 2, 64
    s = torch.full((2, 1, H), 1e-8, device="cuda") if bits == 4 else None
    c = R.Cache(seqs=1, T=704, H=H, d=d, bits=bits, kv_scale=s, seed=9, spread=1e-8 if bits == 4 else 1.0)
    for softmax_scale in (0.0, 1e-12, 1e-30):
        ctx = c.context(4, 3, softmax_scale=softmax_scale)
        q = (queries(3, 4, d).float() * mag).to(torch.bfloat16)
        o, l = run(c, ctx, q, [3], [held])
        scale = float(torch.tensor(softmax_scale, dtype=torch.float32)) if softmax_scale else None
        check(c, q, o, l, [3], [held], scale=scale, what=f"scale {softmax_scale}")


@pytest.mark.parametrize("bits", [16, 4])
def test_strided_rows_streams_and_graphs(gpu_lib, bits):
    """Queries inside a wider tensor, outputs head-major, another stream, a captured graph, the same bits each time."""
    c = R.Cache(seqs=4, T=600, H=8, d=128, bits=bits, seed=9)
    ctx = c.context(32, 2)
    new, held = [1, 2, 1, 2], [599, 100, 17, 333]
    wide = queries(6, 48, 128)
    q = wide[:, :32]
    a = torch.empty(32, 6, 128, dtype=torch.bfloat16, device="cuda")
    o, l = run(c, ctx, q, new, held, out=a.transpose(0, 1))
    check(c, q.contiguous(), o, l, new, held)
    first = a.clone()
    seq_ids, cu, ln = R.batch(new, held)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = torch.zeros_like(a)
    l2 = torch.zeros_like(l)
    torch.cuda.synchronize()
    kv, qr, orow = c.c.view(), E.rows(q), E.rows(b.transpose(0, 1))
    E.epikv_attention(ctx, 0, 4, seq_ids, cu, 2, ln, qr, orow, kv, lse=l2, stream=s)
    s.synchronize()
    assert torch.equal(b, first) and torch.equal(l2, l)
    b.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        E.epikv_attention(ctx, 0, 4, seq_ids, cu, 2, ln, qr, orow, kv)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(b, first)
    ln.copy_(torch.tensor([40, 300, 598, 5], dtype=torch.int32))     # the lengths are read on the device
    g.replay()
    torch.cuda.synchronize()
    check(c, q.contiguous(), b.transpose(0, 1), None, new, [40, 300, 598, 5])


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,block", [(8, 32, 16), (2, 8, 16), (8, 8, 7), (9, 9, 16), (3, 6, 48)])
@pytest.mark.parametrize("new", [1, 5])
def test_lengths_and_tables_of_a_layer(gpu_lib, bits, H, Hq, block, new):
    """As after per-layer budgets: lengths [entry][layer] read at one layer with their stride, every layer with blocks of
    its own; entries of no slots, of some, and of enough to be shared by many blocks of the grid and joined."""
    L, S, T, d = 3, 4, 3008, 64
    held = [[0, 5, 40], [2900, 17, 3000], [3000, 2999, 64], [31, 300, 1]]
    mb = -(-T // block)
    table = torch.randperm(L * S * mb, generator=torch.Generator().manual_seed(H)).view(L, S, mb).int()
    fmt = E.EPIKV_CACHE_E2M1 if bits == 4 else E.EPIKV_CACHE_BF16
    cache = KVCache(E.EPIKV_LAYOUT_PAGED, L, H, d, max_seqs=S, max_tokens=T, block_size=block, block_table=table.numpy(),
                    layer_tables=True, cache_format=fmt)
    units, g = cache.H * cache.d, torch.Generator(device="cuda").manual_seed(d)
    pools = []
    for pool in (cache.k, cache.v):
        x = torch.randn(L * S * mb * block, H, d, generator=g, device="cuda").to(torch.bfloat16)
        raw = pool.view(torch.uint8).view(-1, 2 * units)
        raw.copy_(R.pack(x, units) if bits == 4 else x.view(-1, units).view(torch.uint8))
        pools.append(raw)
    cfg = E.make_attn_config(max_seqs=S, max_cache_tokens=T, max_new_tokens=8, num_layers=L, num_heads=Hq, num_kv_heads=H,
                             head_dim=d, cache_format=fmt)
    ws = torch.empty(E.epikv_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ctx = E.epikv_attn_init(cfg, ws, ws.numel())
    seqs = [2, 0, 3, 1]
    seq_ids, cu, _ = R.batch([new] * S, [0] * S, seqs)
    lens = torch.tensor(held, dtype=torch.int32, device="cuda")
    q = queries(S * new, Hq, d)
    for layer in range(L):
        o, l = torch.full_like(q, float("nan")), torch.empty(S * new, Hq, device="cuda")
        E.epikv_attention(ctx, layer, S, seq_ids, cu, new, lens[:, layer:].data_ptr(), E.rows(q), E.rows(o), cache.view(),
                          lse=l, len_stride=L)
        for b in range(S):
            n = held[b][layer] + new
            slots = torch.arange(n)
            rows = (table[layer, seqs[b]].long()[slots // block] * block + slots % block).cuda()
            k, v = (p[rows] for p in pools)
            if bits == 4:
                k, v = R.values(k, H, d), R.values(v, H, d)
            else:
                k, v = (x.contiguous().view(torch.bfloat16).view(n, H, d).double() for x in (k, v))
            part = slice(b * new, (b + 1) * new)
            ref = R.attention64(q[part], k, v, [held[b][layer] + i + 1 for i in range(new)], d ** -0.5)
            R.assert_attention_close(o[part], l[part], ref, f"layer {layer} entry {b}")
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("n", [2, 7, 16, 40])
def test_probabilities_of_a_bf16_cache(gpu_lib, n):
    """Values of +1 and -1 whose sum nearly cancels: what is left shows the probabilities' own bits.  Two bf16 terms hold
    a probability to 2^-16 (each 2^-8 of what it takes); 32-bit sums of up to 40 products, their exponentials and the
    division add less than 2^-17.  One term alone would be outside the bound, which is checked on the reference."""
    H, d = 4, 64
    c = R.Cache(seqs=1, T=64, H=H, d=d, bits=16, seed=18, spread=0.05)
    sign = torch.where(torch.arange(c.c.v.numel() // (H * d)) % 2 == 0, 1.0, -1.0)
    vals = c.c.v.view(-1, H, d)
    vals[c.index(0, 0, torch.arange(64))] = sign[:64, None, None].to(torch.bfloat16).cuda().expand(64, H, d)
    ctx = c.context(16, 1)
    q = queries(1, 16, d)
    o, _ = run(c, ctx, q, [1], [n - 1])
    k, v = c.read(0, 0, 0, n), c.read(1, 0, 0, n)
    want, _, big, qk = R.attention64(q, k, v, [n], d ** -0.5)
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -15 + 2 * (d * 2.0 ** -24 * qk + 1e-6)[..., None]) * big
    assert bool(((o.double() - want).abs() <= tol).all())
    if n % 2:       # one value more of a sign: the output's own rounding hides the term
        return
    s = torch.einsum("hd,thd->ht", q[0].double(), k.repeat_interleave(4, 1)) * d ** -0.5
    p = torch.exp(s - s.amax(-1, keepdim=True))
    one = torch.einsum("ht,thd->hd", p.to(torch.bfloat16).double(), v.repeat_interleave(4, 1)) / p.sum(-1)[:, None]
    assert float(((one - want[0]).abs() > tol[0]).double().mean()) > 0.5


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,T,block", [(8, 300, 16), (2, 300, 16), (8, 20000, 16), (8, 300, 5), (12, 300, 16), (2, 300, 0)])
def test_rows_that_stand_apart(gpu_lib, bits, H, T, block):
    """A token's rows further apart than they are long, and K's and V's blocks in one allocation."""
    d, S, gap = 64, 8, 24
    c = R.Cache(seqs=S, T=T, H=H, d=d, bits=bits, block=block, seed=H)
    ctx = c.context(2 * H, 2)
    units, st = c.units, c.units + gap
    n = c.raw(0).shape[0]
    wide = torch.full((n, 2, st), float("nan"), dtype=torch.bfloat16, device="cuda")     # [row][K, V][units and a gap]
    for w in range(2):
        wide[:, w, :units].view(torch.int16).copy_(c.raw(w).view(torch.int16).view(n, units))
    k, v = wide.view(-1), wide.view(-1)[st:]
    if block:
        kv = E.kv_view(k, v, layout=E.EPIKV_LAYOUT_PAGED, stride_layer=0, stride_block=block * 2 * st, stride_token=2 * st,
                       block_table=c.c.block_table, max_blocks_per_seq=c.c.max_blocks, block_size=block,
                       num_blocks=c.c.num_blocks)
    else:
        kv = E.kv_view(k, v, layout=E.EPIKV_LAYOUT_CONTIGUOUS, stride_layer=0, stride_seq=T * 2 * st, stride_token=2 * st)
    held, new = [0, 1, 17, 40, 65, 128, 199, 298], [2] * S
    q = queries(2 * S, 2 * H, d)
    seq_ids, cu, ln = R.batch(new, held)
    o, l = torch.empty_like(q), torch.empty(2 * S, 2 * H, device="cuda")
    E.epikv_attention(ctx, 0, S, seq_ids, cu, 2, ln, E.rows(q), E.rows(o), kv, lse=l)
    check(c, q, o, l, new, held)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("S,stride", [(1, 1), (1, 0), (1, 100), (3, 100), (2, 144), (3, 1)])
def test_contiguous_sequences_closer_than_they_are_long(gpu_lib, bits, S, stride):
    """stride_seq of 0, one row or some: a single sequence whose stride says nothing, sequences that overlap.  Slot s of
    sequence b is row b * stride + s."""
    T, H, d = 304, 4, 64
    c = R.Cache(seqs=1, T=T + S * stride, H=H, d=d, bits=bits, block=0, seed=15)
    view = c.c.view()
    view.stride_seq = stride * c.units
    cfg = E.make_attn_config(max_seqs=S, max_cache_tokens=T, max_new_tokens=2, num_layers=1, num_heads=8, num_kv_heads=H,
                             head_dim=d, cache_format=c.fmt)
    ws = torch.empty(E.epikv_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ctx = E.epikv_attn_init(cfg, ws, ws.numel())
    q = queries(2 * S, 8, d)
    seq_ids, cu, ln = R.batch([2] * S, [T - 2 - 7 * b for b in range(S)])
    o, l = torch.empty_like(q), torch.empty(2 * S, 8, device="cuda")
    E.epikv_attention(ctx, 0, S, seq_ids, cu, 2, ln, E.rows(q), E.rows(o), view, lse=l)
    k, v = c.read(0, 0, 0, T + S * stride), c.read(1, 0, 0, T + S * stride)
    for b in range(S):
        n = T - 2 - 7 * b
        ref = R.attention64(q[2 * b:2 * b + 2], k[b * stride:b * stride + n + 2], v[b * stride:b * stride + n + 2],
                            [n + 1, n + 2], d ** -0.5)
        R.assert_attention_close(o[2 * b:2 * b + 2], l[2 * b:2 * b + 2], ref, f"sequence {b}")
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("block", [2 ** 24, 2 ** 26, 2 ** 27, 2 ** 31 - 16, 2 ** 31 - 1])
def test_one_block_holds_the_whole_sequence(gpu_lib, bits, block):
    """A block size far beyond the sequences: each has one block, at any size that the view's field takes."""
    T, S, H, d = 544, 3, 4, 128
    c = R.Cache(seqs=S, T=T, H=H, d=d, bits=bits, block=T, seed=12)
    view = c.c.view()
    view.block_size = block
    ctx = c.context(16, 3)
    new, held = [1, 3, 2], [0, 541, 64]
    q = queries(6, 16, d)
    seq_ids, cu, ln = R.batch(new, held)
    o, l = torch.empty_like(q), torch.empty(6, 16, device="cuda")
    E.epikv_attention(ctx, 0, S, seq_ids, cu, 3, ln, E.rows(q), E.rows(o), view, lse=l)
    check(c, q, o, l, new, held)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("bits", [16, 4])
def test_offsets_past_32_bits(gpu_lib, bits):
    """Two blocks 6 GB apart in one pool."""
    H, d, bs = 8, 128, 16
    h2, d2 = E.epikv_cache_row(H, d, E.EPIKV_CACHE_E2M1 if bits == 4 else E.EPIKV_CACHE_BF16)
    units = h2 * d2
    blocks = 3 * 2 ** 30 // (units * bs) + 2
    small = R.Cache(seqs=1, T=32, H=H, d=d, bits=bits, seed=10)
    pools = [torch.empty(blocks * bs * units, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for w in range(2):
        raw = pools[w].view(torch.uint8).view(-1, 2 * units)
        src = small.raw(w)[small.index(0, 0, torch.arange(32))]
        raw[(blocks - 1) * bs:] = src[:16]
        raw[:bs] = src[16:]
    bt = torch.tensor([[blocks - 1, 0]], dtype=torch.int32, device="cuda")
    kv = E.kv_view(pools[0], pools[1], layout=E.EPIKV_LAYOUT_PAGED, stride_layer=0, stride_block=bs * units,
                   stride_token=units, block_table=bt, max_blocks_per_seq=2, block_size=bs, num_blocks=blocks)
    ctx = small.context(32, 1)
    q = queries(1, 32, d)
    seq_ids, cu, ln = R.batch([1], [31])
    o = torch.empty_like(q)
    E.epikv_attention(ctx, 0, 1, seq_ids, cu, 1, ln, E.rows(q), E.rows(o), kv)
    check(small, q, o, None, [1], [31])
    x = torch.randn(1, H, d, device="cuda").to(torch.bfloat16)
    bt.copy_(bt.flip(1))
    E.epikv_append(ctx, 0, 1, seq_ids, cu, 1, ln, None, None, None, E.rows(x), E.rows(x), None, kv)
    want = R.pack(x, units)[0] if bits == 4 else x.view(1, -1).view(torch.uint8)[0]
    used = H * (d // 2 + d // 16) if bits == 4 else 2 * units
    assert torch.equal(pools[0].view(torch.uint8).view(-1, 2 * units)[blocks * bs - 1, :used], want[:used])
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


@pytest.mark.parametrize("bits", [16, 4])
def test_many_sequences(gpu_lib, bits):
    """More sequences than the grid has blocks, most of them short, none, or one long."""
    S = 700
    held = [(7 * i) % 60 for i in range(S)]
    held[333] = 5000
    new = [(i % 3) for i in range(S)]
    c = R.Cache(seqs=S, T=5003, H=1, d=64, bits=bits, seed=11)
    ctx = c.context(2, 2)
    q = queries(sum(new), 2, 64)
    o, l = run(c, ctx, q, new, held)
    check(c, q, o, l, new, held)


def long_batch(c, Hq, n_seq, max_new, **kw):
    """A context for more entries than the cache has sequences (attention only reads it)."""
    cfg = E.make_attn_config(max_seqs=n_seq, max_cache_tokens=c.T, max_new_tokens=max_new, num_layers=1, num_heads=Hq,
                             num_kv_heads=c.H, head_dim=c.d, cache_format=c.fmt, **kw)
    n = E.epikv_attn_workspace_bytes(cfg)
    c.ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    return E.epikv_attn_init(cfg, c.ws, n)


@pytest.mark.parametrize("new,heavy", [([33000], [0]), ([1] * 300 + [23300, 23300, 1], [300, 301])])
def test_long_prompts(gpu_lib, new, heavy):
    """Over 2^23 tiles in one prompt, and in two entries that one thread counts: every entry is taken."""
    T, H, Hq, d = 33008, 8, 32, 128
    c = R.Cache(seqs=2, T=T, H=H, d=d, bits=16, seed=13)
    ctx = long_batch(c, Hq, len(new), max(new))
    held = [0 if n > 1 else 50 + i for i, n in enumerate(new)]
    seqs = [i % 2 for i in range(len(new))]
    q = queries(sum(new), Hq, d)
    o, l = run(c, ctx, q, new, held, seqs=seqs)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)
    start = torch.tensor([0] + new).cumsum(0).tolist()
    for b in set(heavy) | {0, len(new) - 1}:
        for i in {0, new[b] // 3, max(new[b] - 3, 0)}:             # up to three tokens of each
            m = min(3, new[b] - i)
            t = start[b] + i
            top = held[b] + i + m
            k, v = c.read(0, 0, seqs[b], top), c.read(1, 0, seqs[b], top)
            ref = R.attention64(q[t:t + m], k, v, [held[b] + i + j + 1 for j in range(m)], d ** -0.5)
            R.assert_attention_close(o[t:t + m], l[t:t + m], ref, f"entry {b} from token {i}")


def test_more_work_than_is_counted(gpu_lib):
    """An entry of over 2^31 tiles is skipped with those behind it and reported; those before it are done."""
    T, H, Hq, d = 2 ** 22, 8, 32, 128
    c = R.Cache(seqs=1, T=64, H=H, d=d, bits=16, seed=14)
    small = c.c.view()
    table = torch.zeros(3, T // 16, dtype=torch.int32, device="cuda")    # many slots, one block
    table[:, :4] = c.c.block_table
    view = E.kv_view(c.c.k, c.c.v, layout=E.EPIKV_LAYOUT_PAGED, stride_layer=0, stride_block=small.stride_block,
                     stride_token=small.stride_token, block_table=table, max_blocks_per_seq=T // 16, block_size=16,
                     num_blocks=c.c.num_blocks)
    new, held = [2, 2 ** 16, 1], [40, T - 2 ** 16, 5]
    c.T = T
    ctx = long_batch(c, Hq, 3, max(new))
    n = sum(new)
    q = torch.zeros(n, Hq, d, dtype=torch.bfloat16, device="cuda")
    q[:2] = queries(2, Hq, d)
    out = torch.full_like(q, 7.0)
    seq_ids, cu, ln = R.batch(new, held)
    E.epikv_attention(ctx, 0, 3, seq_ids, cu, max(new), ln, E.rows(q), E.rows(out), view)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_CAPACITY)
    check(c, q[:2], out[:2], None, [2], [40])
    assert bool((out[2:] == 7.0).all())


def test_reported_and_skipped(gpu_lib):
    c = R.Cache(seqs=2, T=64, H=2, d=64, bits=4)
    ctx = c.context(2, 4)
    for kw, code in ((dict(new=[1, 1], held=[5, 64]), E.EPIKV_DEV_CAPACITY),
                     (dict(new=[1, 1], held=[5, -2]), E.EPIKV_DEV_CAPACITY),
                     (dict(new=[1, 1], held=[5, 5], seqs=[0, 9]), E.EPIKV_DEV_BATCH),
                     (dict(new=[1, 3], held=[5, 5], max_new=2), E.EPIKV_DEV_BATCH)):
        q = queries(sum(kw["new"]), 2, 64)
        o, l = run(c, ctx, q, **kw)
        assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, code)
        check(c, q[:1], o[:1], l[:1], [1], [5])
        assert bool(o[1:].isnan().all())
    c.c.block_table[1, 0] = -1
    q = queries(2, 2, 64)
    o, l = run(c, ctx, q, [1, 1], [5, 40])
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_SLOT)
    check(c, q[:1], o[:1], l[:1], [1], [5])


def test_refusals(gpu_lib):
    c = R.Cache(seqs=2, T=32, H=2, d=64, bits=16)
    ctx = c.context(4, 4)
    q = queries(3, 4, 64)
    seq_ids, cu, ln = R.batch([3], [0])
    ok = dict(layer=0, n=1, seq_ids=seq_ids, cu=cu, max_new=3, ln=ln, q=E.rows(q), o=E.rows(q.clone()),
              kv=c.c.view(), ls=1)

    def call(**kw):
        a = {**ok, **kw}
        E.epikv_attention(ctx, a["layer"], a["n"], a["seq_ids"], a["cu"], a["max_new"], a["ln"], a["q"], a["o"],
                          a["kv"], len_stride=a["ls"])

    call()
    call(n=0)
    call(max_new=0)
    for bad in (dict(layer=1), dict(n=3), dict(max_new=5), dict(seq_ids=None), dict(cu=None), dict(ln=None),
                dict(q=None), dict(o=None), dict(q=E.rows(q.float())), dict(o=E.rows(q.half())), dict(kv=None),
                dict(ls=0)):
        with pytest.raises(E.EpikvError) as err:
            call(**bad)
        assert err.value.status == E.EPIKV_EINVAL, bad
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)
