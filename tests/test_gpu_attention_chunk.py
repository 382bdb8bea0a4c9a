"""epikv_attention_chunk against float64: head layouts, chunks of one token to hundreds, ragged batches, pages that end
inside a tile, rows that see nothing, what stands in slots that a row does not see, strides, streams and graphs."""
import math

import pytest
import torch

from paper_2606_26472_gb300 import epikv as E

from . import cache_ops as R
from .chunk_ops import attend, check_attention, check_weights, queries

pytestmark = pytest.mark.gpu

SHAPES = [(8, 32, 128), (1, 1, 64), (1, 8, 128), (2, 14, 128), (3, 3, 64), (4, 32, 64), (5, 20, 128), (2, 4, 256),
          (4, 32, 256), (11, 11, 64), (1, 71, 64)]
OK = (E.EPIKV_OK, 0)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_tile(gpu_lib, bits, d):
    """One tile of rows and of slots."""
    c = R.Cache(seqs=1, T=256, H=1, d=d, bits=bits, seed=d)
    ctx = c.context(1, 128)
    q = queries(32, 1, d)
    o, l = attend(c, ctx, q, [32], [0])
    check_attention(c, q, o, l, [32], [0])
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", SHAPES)
def test_ragged_chunks(gpu_lib, bits, H, Hq, d):
    new, held = [3, 0, 1, 17, 147, 8, 64], [0, 5, 200, 31, 77, 1500, 63]
    for block in (16, 0, 7, 48):
        c = R.Cache(seqs=7, T=1600, H=H, d=d, bits=bits, block=block, seed=H + d)
        ctx = c.context(Hq, 200)
        q = queries(sum(new), Hq, d)
        seqs = [3, 0, 6, 1, 2, 5, 4]
        o, l = attend(c, ctx, q, new, held, seqs=seqs)
        check_attention(c, q, o, l, new, held, seqs=seqs, what=f"block {block}")
        assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", [(8, 32, 128), (1, 1, 64), (2, 4, 256)])
def test_single_tokens(gpu_lib, bits, H, Hq, d):
    held = [0, 1, 14, 15, 16, 63, 64, 65, 126, 127, 128, 129, 300, 1023]
    c = R.Cache(seqs=14, T=1030, H=H, d=d, bits=bits, seed=H * d)
    ctx = c.context(Hq, 1)
    q = queries(14, Hq, d)
    o, l = attend(c, ctx, q, [1] * 14, held)
    check_attention(c, q, o, l, [1] * 14, held)
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", [(2, 8, 128), (1, 2, 64), (1, 1, 256), (2, 32, 128)])
def test_prompts(gpu_lib, bits, H, Hq, d):
    """Whole prompts, pieces behind held slots, and one long cache."""
    new, held = [700, 300, 1, 33], [0, 900, 9000, 4001]
    c = R.Cache(seqs=4, T=9100, H=H, d=d, bits=bits, seed=5)
    ctx = c.context(Hq, 700)
    q = queries(sum(new), Hq, d)
    o, l = attend(c, ctx, q, new, held)
    check_attention(c, q, o, l, new, held)
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("bits", [16, 4])
def test_prefix_without_the_new_tokens(gpu_lib, bits):
    """causal=0: every query sees the held slots; none held: zeros and -inf."""
    c = R.Cache(seqs=3, T=400, H=2, d=64, bits=bits, seed=2)
    ctx = c.context(6, 90)
    new, held = [5, 90, 3], [0, 399, 18]
    q = queries(98, 6, 64)
    o, l = attend(c, ctx, q, new, held, causal=False)
    check_attention(c, q, o, l, new, held, causal=False)
    assert not o[:5].any() and bool((l[:5] == -math.inf).all())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("H,Hq,d", [(2, 8, 128), (1, 1, 64), (1, 4, 256)])
@pytest.mark.parametrize("new", [1, 40, 150])
def test_unseen_slots_do_not_reach_a_row(gpu_lib, bits, H, Hq, d, new):
    """From some slot on the cache holds NaN: rows that do not see it are as in the clean cache bit for bit, rows that see it
    are NaN."""
    held, T = 45, 256
    c = R.Cache(seqs=1, T=T, H=H, d=d, bits=bits, seed=3)
    ctx = c.context(Hq, 160)
    q = queries(new, Hq, d)
    clean, lclean = attend(c, ctx, q, [new], [held])
    for first in sorted({held + new, held + new // 2 + 1, held + 1}):
        raw = [c.raw(w).clone() for w in (0, 1)]
        rows = c.index(0, 0, torch.arange(first, T))
        for w in (0, 1):
            c.raw(w)[rows] = 0x7F if bits == 4 else torch.tensor([0xC0, 0x7F], dtype=torch.uint8,
                                                                 device="cuda").repeat(c.units)
        o, l = attend(c, ctx, q, [new], [held])
        n = min(new, max(0, first - held))
        assert torch.equal(o[:n], clean[:n]) and torch.equal(l[:n], lclean[:n])
        assert bool(o[n:].isnan().all())
        for w in (0, 1):
            c.raw(w).copy_(raw[w])


@pytest.mark.parametrize("H,Hq,d", [(1, 4, 128), (2, 2, 64), (1, 3, 256)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinite_values(gpu_lib, H, Hq, d, sign):
    """An infinite value is the output of the rows that see it, in its channel alone."""
    held, new = 100, 70
    c = R.Cache(seqs=1, T=200, H=H, d=d, seed=4)
    ctx = c.context(Hq, 70)
    q = queries(new, Hq, d)
    clean, _ = attend(c, ctx, q, [new], [held])
    for slot in (3, 100, 131, 169):
        row, ch = int(c.index(0, 0, [slot])[0]), slot % d
        pool = c.c.v.view(-1, H, d)
        keep = pool[row, H - 1, ch].clone()
        pool[row, H - 1, ch] = sign * math.inf
        o, _ = attend(c, ctx, q, [new], [held])
        pool[row, H - 1, ch] = keep
        sees = torch.arange(new, device="cuda") + held >= slot
        mine = torch.zeros(new, Hq, d, dtype=torch.bool, device="cuda")
        mine[sees, Hq - Hq // H:, ch] = True
        assert bool((o[mine] == sign * math.inf).all())
        assert torch.equal(o[~mine], clean[~mine])


def test_scores_of_minus_infinity(gpu_lib):
    """Keys of -inf beside queries above 0: rows whose every score is -inf give zeros and -inf."""
    c = R.Cache(seqs=1, T=300, H=1, d=64, seed=6)
    ctx = c.context(2, 64)
    q = queries(64, 2, 64)
    q[:, :, 5] = q[:, :, 5].abs() + 0.5
    q[:, 1, 5] = -q[:, 1, 5]                        # the other head's scores are +inf
    pool = c.c.k.view(-1, 64)
    pool[c.index(0, 0, torch.arange(0, 210)), 5] = -math.inf
    o, l = attend(c, ctx, q, [64], [180])
    assert not o[:30, 0].any() and bool((l[:30, 0] == -math.inf).all())
    assert bool(o[30:, 0].isfinite().all()) and bool(l[30:, 0].isfinite().all())
    assert bool(o[:, 1].isnan().all())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("mag", [2.0 ** -60, 1e-3, 30.0, 2.0 ** 20])
def test_query_magnitudes(gpu_lib, bits, mag):
    """Maxima that grow along the slots and queries far from 1; scores up to the millions stay exact enough."""
    c = R.Cache(seqs=1, T=800, H=2, d=128, bits=bits, seed=7)
    ctx = c.context(4, 80, softmax_scale=0.09 / mag if mag > 1 else 0.0)
    q = (queries(80, 4, 128).float() * mag).to(torch.bfloat16)
    o, l = attend(c, ctx, q, [80], [700])
    check_attention(c, q, o, l, [80], [700], scale=0.09 / mag if mag > 1 else None)


@pytest.mark.parametrize("bits", [16, 4])
def test_growing_maxima(gpu_lib, bits):
    """Each tile's scores are far above the last one's, so that sums are rescaled in every tile."""
    c = R.Cache(seqs=1, T=1024, H=1, d=64, bits=bits, seed=8)
    x = torch.randn(1024, 1, 64, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda") * 0.1
    x += torch.arange(1024, device="cuda")[:, None, None] / 64.0
    flat = torch.zeros_like(c.raw(0)).view(torch.bfloat16)
    order = c.index(0, 0, torch.arange(1024))
    if bits == 16:
        flat[order] = x.to(torch.bfloat16).view(1024, 64)
        c.raw(0).copy_(flat.view(torch.uint8))
    else:
        c.raw(0)[order] = R.pack(x.to(torch.bfloat16), c.units)
    ctx = c.context(1, 130)
    q = queries(130, 1, 64).abs()
    o, l = attend(c, ctx, q, [130], [890])
    check_attention(c, q, o, l, [130], [890])


def test_head_scales(gpu_lib):
    ks = torch.tensor([[[0.01, 3.0], [1.0, 0.5]], [[20.0, 0.125], [1e-3, 1.0]]], device="cuda")
    c = R.Cache(seqs=2, T=300, H=2, d=64, bits=4, layers=2, kv_scale=ks, seed=10)
    ctx = c.context(4, 60)
    q = queries(90, 4, 64)
    for layer in (0, 1):
        o, l = attend(c, ctx, q, [30, 60], [200, 100], layer=layer)
        check_attention(c, q, o, l, [30, 60], [200, 100], layer=layer)


@pytest.mark.parametrize("bits", [16, 4])
def test_strided_rows_streams_and_graphs(gpu_lib, bits):
    """Rows out of wider ones, a length array with a stride, another stream, and a graph replayed with other lengths."""
    c = R.Cache(seqs=3, T=700, H=2, d=128, bits=bits, seed=11)
    ctx = c.context(8, 64)
    wide = queries(100, 14, 128)
    q, buf = wide[:, 3:11], torch.zeros(100, 11, 128, dtype=torch.bfloat16, device="cuda")
    out = buf[:, 2:10]
    lse = torch.zeros(100, 8, device="cuda")
    lens = torch.zeros(3, 5, dtype=torch.int32, device="cuda")
    seq_ids, cu, _ = R.batch([40, 10, 50], [0, 0, 0])
    cases = ([300, 0, 11], [77, 600, 128])
    s = torch.cuda.Stream()
    call = lambda: E.epikv_attention_chunk(ctx, 0, 3, seq_ids, cu, 64, lens[:, 2:], E.rows(q), E.rows(out), c.c.view(),  # noqa: E731
                                           lse=lse, len_stride=5)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lens[:, 2] = torch.tensor(cases[0], dtype=torch.int32, device="cuda")
        call()
        check_attention(c, q.contiguous(), out, lse, [40, 10, 50], cases[0])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        for held in cases:
            lens[:, 2] = torch.tensor(held, dtype=torch.int32, device="cuda")
            out.zero_()
            g.replay()
            check_attention(c, q.contiguous(), out, lse, [40, 10, 50], held)
    torch.cuda.current_stream().wait_stream(s)
    assert not buf[:, :2].any() and not buf[:, 10:].any()


@pytest.mark.parametrize("bits", [16, 4])
def test_repeated_calls_agree(gpu_lib, bits):
    """The same call gives the same bits, whatever else was computed between."""
    c = R.Cache(seqs=4, T=3000, H=2, d=128, bits=bits, seed=12)
    ctx = c.context(8, 200)
    new, held = [200, 1, 64, 130], [2000, 2999, 0, 777]
    q = queries(sum(new), 8, 128)
    first = attend(c, ctx, q, new, held)
    for _ in range(3):
        attend(c, ctx, q[:64], [64], [100])
        again = attend(c, ctx, q, new, held)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("bits", [16, 4])
def test_many_sequences(gpu_lib, bits):
    """More of them than a warp has lanes, most with little or nothing to do."""
    S = 200
    c = R.Cache(seqs=S, T=330, H=2, d=64, bits=bits, seed=19)
    ctx = c.context(6, 90)
    new = [(0, 1, 3, 90, 0, 7, 2)[b % 7] for b in range(S)]
    held = [(b * 37) % 240 if b % 5 else 0 for b in range(S)]
    seqs = [(b * 73 + 11) % S for b in range(S)]
    q = queries(sum(new), 6, 64)
    o, l = attend(c, ctx, q, new, held, seqs=seqs)
    check_attention(c, q, o, l, new, held, seqs=seqs)
    assert E.epikv_attn_get_error(ctx) == OK


def test_offsets_past_32_bits(gpu_lib):
    """A contiguous cache of more than 2^32 bytes, its last sequence's slots far behind that."""
    S, T, H, d = 5, 262144, 8, 128
    c = R.Cache(seqs=1, T=16, H=H, d=d, block=0)
    k = torch.zeros(S * T, H, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator(device="cuda").manual_seed(13)
    held, new = 1000, 40
    lo = (S - 1) * T
    for x in (k, v):
        x[lo:lo + held + new] = torch.randn(held + new, H, d, generator=g, device="cuda").to(torch.bfloat16)
    cfg = E.make_attn_config(max_seqs=S, max_cache_tokens=T, max_new_tokens=new, num_layers=1, num_heads=16, num_kv_heads=H,
                             head_dim=d)
    ws = torch.empty(E.epikv_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ctx = E.epikv_attn_init(cfg, ws, ws.numel())
    kv = E.kv_view(k, v, stride_layer=0, stride_seq=T * H * d, stride_token=H * d)
    q = queries(new, 16, d)
    o, l = torch.empty_like(q), torch.empty(new, 16, device="cuda")
    seq_ids, cu, ln = R.batch([new], [held], [S - 1])
    E.epikv_attention_chunk(ctx, 0, 1, seq_ids, cu, new, ln, E.rows(q), E.rows(o), kv, lse=l)
    ref = R.attention64(q, k[lo:lo + held + new].double(), v[lo:lo + held + new].double(), [held + i + 1 for i in range(new)],
                        d ** -0.5)
    assert float((o.double() - ref[0]).abs().max()) <= float(((2.0 ** -8) * 2.1 * ref[2]).max())
    assert E.epikv_attn_get_error(ctx) == OK


def test_reported_and_skipped(gpu_lib):
    """Entries that cannot be taken are reported and leave their rows; the others are right (where a row's slots are split
    goes by the whole batch's work, so not the same bits as without them)."""
    c = R.Cache(seqs=4, T=256, H=2, d=64, seed=14)
    ctx = c.context(4, 32)
    q = queries(64, 4, 64)
    for seqs, held, code in (([0, 9], [100, 50], E.EPIKV_DEV_BATCH), ([0, -1], [100, 50], E.EPIKV_DEV_BATCH),
                             ([0, 3], [100, 225], E.EPIKV_DEV_CAPACITY), ([0, 3], [100, -1], E.EPIKV_DEV_CAPACITY)):
        o, l = attend(c, ctx, q, [32, 32], held, seqs=seqs)
        assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, code)
        check_attention(c, q[:32], o[:32], l[:32], [32], [100])
        assert bool(o[32:].isnan().all()) and bool(l[32:].isnan().all())
    # a block that the pool does not have: its slots are rows of zeros
    table = c.c.block_table.clone()
    table[0, 2] = c.c.num_blocks
    seq_ids, cu, ln = R.batch([32], [100], [0])
    o, l = torch.empty_like(q[:32]), torch.empty(32, 4, device="cuda")
    E.epikv_attention_chunk(ctx, 0, 1, seq_ids, cu, 32, ln, E.rows(q[:32]), E.rows(o), c.c.view(table), lse=l)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_SLOT)
    k, v = c.read(0, 0, 0, 132), c.read(1, 0, 0, 132)
    k[32:48], v[32:48] = 0, 0
    ref = R.attention64(q[:32], k, v, [101 + i for i in range(32)], 0.125)
    assert float((l.double() - ref[1]).abs().max()) < 1e-4
    assert float((o.double() - ref[0]).abs().max()) <= float(((2.0 ** -8) * 2.1 * ref[2]).max())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_infinities_in_many_short_segments(gpu_lib, bits, d):
    """Each CTA takes a dozen items of one tile, each with a value that is infinite (over 4-bit rows: 16 that are NaN) in a slot
    that its first rows do not see."""
    S, held, new = 900, 20, 16
    c = R.Cache(seqs=S, T=48, H=2, d=d, bits=bits, seed=20)
    ctx = c.context(2, new)
    q = queries(S * new, 2, d)
    clean, lse = attend(c, ctx, q, [new] * S, [held] * S)
    at = [held + 1 + b % (new - 1) for b in range(S)]
    for b in range(S):
        row = int(c.index(0, b, [at[b]])[0])
        if bits == 16:
            c.c.v.view(-1, 2, d)[row, 1, b % d] = math.inf
        else:
            c.raw(1)[row, d + d // 16] = 0x7F             # the second head's first scale
    o, l = attend(c, ctx, q, [new] * S, [held] * S)
    sees = (torch.arange(new, device="cuda") + held >= torch.tensor(at, device="cuda")[:, None])          # [S, new]
    bad = torch.zeros(S, new, 2, d, dtype=torch.bool, device="cuda")
    if bits == 16:
        ch = torch.nn.functional.one_hot(torch.arange(S, device="cuda") % d, d).bool()
        bad[:, :, 1] = sees[..., None] & ch[:, None]
    else:
        bad[:, :, 1, :16] = sees[..., None]
    bad = bad.view(S * new, 2, d)
    assert bool((o[bad] == math.inf).all() if bits == 16 else o[bad].isnan().all())
    assert torch.equal(o[~bad], clean[~bad]) and torch.equal(l, lse)
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("H,Hq,d", [(2, 2, 64), (1, 1, 128), (2, 4, 64), (1, 2, 256)])
def test_infinities_in_every_tile_that_not_all_rows_see(gpu_lib, H, Hq, d):
    """Items whose rows end in three tiles in a row: the copying warps look through each, and find some in one warp's rows."""
    S, held, new = 120, 100, 300
    c = R.Cache(seqs=S, T=400, H=H, d=d, seed=21)
    ctx = c.context(Hq, new)
    q = queries(S * new, Hq, d)
    clean, lse = attend(c, ctx, q, [new] * S, [held] * S)
    at = torch.arange(S, device="cuda") % 7 + held + torch.tensor([[20], [140], [290]], device="cuda")      # [3, S]
    pool, bad = c.c.v.view(-1, H, d), torch.zeros(S, new, Hq, d, dtype=torch.bool, device="cuda")
    for i in range(3):
        for b in range(S):
            pool[int(c.index(0, b, [int(at[i, b])])[0]), H - 1, (5 * b + i) % d] = -math.inf
        sees = torch.arange(new, device="cuda") + held >= at[i][:, None]
        ch = torch.nn.functional.one_hot((5 * torch.arange(S, device="cuda") + i) % d, d).bool()
        bad[:, :, Hq - Hq // H:] |= (sees[..., None] & ch[:, None])[:, :, None]
    o, l = attend(c, ctx, q, [new] * S, [held] * S)
    assert E.epikv_attn_get_error(ctx) == OK
    bad = bad.view(S * new, Hq, d)
    # (beside the infinity a row may also have probabilities of exactly 0 in slots that all rows of an item see: NaN there)
    assert bool((~o[bad].isfinite()).all()) and torch.equal(o[~bad], clean[~bad]) and torch.equal(l, lse)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new,H,Hq,d", [(1, 2, 8, 64), (90, 2, 2, 128), (40, 1, 8, 256), (200, 3, 3, 64)])
def test_blocks_that_are_none(gpu_lib, bits, new, H, Hq, d):
    """Slots of blocks that the pool does not have are rows of zeros, all others what they are: tiles with such blocks between
    tiles without, in several sequences."""
    S, T, held = 12, 1700, 1400
    c = R.Cache(seqs=S, T=T, H=H, d=d, bits=bits, seed=22)
    ctx = c.context(Hq, new)
    q = queries(S * new, Hq, d)
    table = c.c.block_table.clone()
    gone = torch.zeros(S, T + 16, dtype=torch.bool, device="cuda")
    for s in range(S):
        for i, t in enumerate(range(s % 3, 12, 2)):          # every second tile of 128 slots
            b = 8 * t + (3 * i + s) % 8
            if 16 * b < held:
                table[s, b] = (c.c.num_blocks, -1, 1 << 30, -(1 << 31))[i % 4]
                gone[s, 16 * b:16 * b + 16] = True
    seq_ids, cu, ln = R.batch([new] * S, [held] * S)
    o, l = torch.empty_like(q), torch.empty(S * new, Hq, device="cuda")
    E.epikv_attention_chunk(ctx, 0, S, seq_ids, cu, new, ln, E.rows(q), E.rows(o), c.c.view(table), lse=l)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_SLOT)
    whole = c.read

    def with_zeros(w, layer, s, top):
        x = whole(w, layer, s, top).clone()
        x[gone[s, :top]] = 0
        return x
    c.read = with_zeros
    check_attention(c, q, o, l, [new] * S, [held] * S)


@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("bits,scale,keys", [(4, 0.0, 2.0 ** -60), (4, 1e-30, 1.0), (4, 0.0, 2.0 ** -100), (16, 3e38, 1.0), (4, 3e38, 1.0),
                                             (16, 1e-45, 1.0)])
def test_factors_that_leave_the_normal_numbers(gpu_lib, bits, scale, keys, d):
    """Query rows of zeros (a padded batch's) and of tiny numbers beside small or large scales: a score of 0 stays one, and what a
    row does not see stays unseen."""
    ks = None if bits == 16 else torch.tensor([[[keys, 1.0]], [[1.0, 0.5]]], device="cuda")
    c = R.Cache(seqs=1, T=300, H=2, d=d, bits=bits, kv_scale=ks, seed=23)
    ctx = c.context(4, 60, softmax_scale=scale)
    q = queries(60, 4, d)
    q[1::2] = (q[1::2].float() * 2.0 ** -120).to(torch.bfloat16)
    q[::4 if scale < 1 else 1] = 0
    o, l = attend(c, ctx, q, [60], [200])
    check_attention(c, q, o, l, [60], [200], scale=scale or None)
    assert bool(o.isfinite().all())


@pytest.mark.parametrize("bits", [16, 4])
def test_a_long_prompt(gpu_lib, bits):
    """70,001 tokens at once, some of its rows against 64 bits."""
    n, d = 70001, 64
    c = R.Cache(seqs=1, T=n, H=1, d=d, bits=bits, seed=26)
    ctx = c.context(1, n)
    q = queries(n, 1, d)
    o, l = attend(c, ctx, q, [n], [0])
    k, v = c.read(0, 0, 0, n), c.read(1, 0, 0, n)
    for i in (0, 1, 127, 128, 129, 255, 256, 4096, 33333, 65535, 65536, n - 130, n - 1):
        ref, lse, big, qk = R.attention64(q[i:i + 1], k[:i + 1], v[:i + 1], [i + 1], d ** -0.5)
        ds = d * 2.0 ** -24 * qk + 1e-6
        p = (2.0 ** -8 if bits == 16 else 2.0 ** -11) + 2.0 ** -21 + i * 2.0 ** -24
        tiny = 0.0 if bits == 16 else (i + 1) * 2.0 ** -32 * float(v[:i + 1].abs().max())
        assert bool(((o[i].double() - ref[0]).abs() <= 2.0 ** -8 * ref[0].abs() + (p + 2 * ds[0, :, None]) * big[0] + tiny).all()), i
        assert bool(((l[i].double() - lse[0]).abs() <= ds[0] + 2.0 ** -22 * (1 + lse[0].abs()) + (i + 1) * 2.0 ** -24).all()), i
    assert E.epikv_attn_get_error(ctx) == OK


def test_rows_behind_the_last_sequence(gpu_lib):
    """A batch padded with entries of no tokens and rows behind them: those stay as they were."""
    c = R.Cache(seqs=4, T=200, H=2, d=128, seed=27)
    ctx = c.context(8, 40)
    q = queries(64, 8, 128)
    o, l = torch.full_like(q, 3.0), torch.full((64, 8), 3.0, device="cuda")
    seq_ids, cu, ln = R.batch([40, 0, 7, 0], [30, 100, 0, 0])
    E.epikv_attention_chunk(ctx, 0, 4, seq_ids, cu, 40, ln, E.rows(q), E.rows(o), c.c.view(), lse=l)
    check_attention(c, q[:47], o[:47], l[:47], [40, 0, 7, 0], [30, 100, 0, 0])
    assert bool((o[47:] == 3.0).all()) and bool((l[47:] == 3.0).all())
    again = torch.full_like(q, 3.0)                      # without the log-sums
    E.epikv_attention_chunk(ctx, 0, 4, seq_ids, cu, 40, ln, E.rows(q), E.rows(again), c.c.view())
    assert torch.equal(again, o)
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("H,Hq", [(1, 1024), (2, 600)])
def test_many_query_heads(gpu_lib, H, Hq):
    """More query heads of a KV head than an item has rows."""
    c = R.Cache(seqs=2, T=300, H=H, d=64, seed=28)
    ctx = c.context(Hq, 5)
    q = queries(7, Hq, 64)
    o, l = attend(c, ctx, q, [5, 2], [250, 3])
    check_attention(c, q, o, l, [5, 2], [250, 3])
    assert E.epikv_attn_get_error(ctx) == OK


@pytest.mark.parametrize("layout", ["layer tables", "contiguous", "contiguous, closer than long"])
@pytest.mark.parametrize("H,Hq,d,new,held", [(2, 8, 64, [50, 1, 0], [200, 131, 77]), (1, 2, 128, [140, 3, 9], [0, 160, 255]),
                                             (2, 2, 256, [1, 1, 1], [16, 299, 100])])
def test_rows_within_wider_rows(gpu_lib, layout, H, Hq, d, new, held):
    """K and V of a token side by side in one pool, by blocks of each layer's own table, or contiguous with a gap behind each
    sequence or with its end within the next one: the chunk's attention, and the weights that its log-sums give."""
    S, T, L, bs = 3, 304, 2, 16
    g = torch.Generator(device="cuda").manual_seed(29)
    row = 2 * H * d + 64                                       # and 64 values more
    at = torch.empty(L, S, T, dtype=torch.long, device="cuda")  # of a slot's row
    if layout == "layer tables":
        mb = T // bs
        table = torch.randperm(L * S * mb, generator=g, device="cuda").int().view(L, S, mb)
        at[:] = (table.long()[..., None] * bs + torch.arange(bs, device="cuda")).view(L, S, T)
        rows = L * S * mb * bs
        kw = dict(layout=E.EPIKV_LAYOUT_PAGED, block_table=table, max_blocks_per_seq=mb, block_size=bs, num_blocks=L * S * mb,
                  stride_layer=0, stride_block=bs * row, stride_table_layer=S * mb)
    else:
        apart = T + 5 if layout == "contiguous" else T - 4      # (no sequence here holds its last 4 slots)
        at[:] = (torch.arange(L, device="cuda")[:, None, None] * (S * apart + 7) + torch.arange(S, device="cuda")[:, None] * apart
                 + torch.arange(T, device="cuda"))
        rows = int(at.max()) + 1
        kw = dict(layout=E.EPIKV_LAYOUT_CONTIGUOUS, stride_layer=(S * apart + 7) * row, stride_seq=apart * row)
    pool = torch.randn(rows, row, generator=g, device="cuda").to(torch.bfloat16)
    kv = E.kv_view(pool, pool[:, H * d:], stride_token=row, **kw)
    cfg = E.make_attn_config(max_seqs=S, max_cache_tokens=T, max_new_tokens=200, num_layers=L, num_heads=Hq, num_kv_heads=H,
                             head_dim=d)
    ws = torch.empty(E.epikv_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ctx = E.epikv_attn_init(cfg, ws, ws.numel())

    class Rows:
        def __init__(self):
            self.d, self.H, self.bits = d, H, 16

        def read(self, w, layer, s, n):
            return pool[at[layer, s, :n]][:, w * H * d:(w + 1) * H * d].view(n, H, d).double()
    q = queries(sum(new), Hq, d)
    seq_ids, cu, ln = R.batch(new, held)
    for layer in range(L):
        o, l = torch.empty_like(q), torch.empty(sum(new), Hq, device="cuda")
        E.epikv_attention_chunk(ctx, layer, S, seq_ids, cu, 200, ln, E.rows(q), E.rows(o), kv, lse=l)
        check_attention(Rows(), q, o, l, new, held, layer=layer, what=f"layer {layer}")
        w = torch.full((S, H, T), -7.5, device="cuda")
        before = w.clone()
        E.epikv_attention_weights(ctx, layer, S, seq_ids, cu, 200, ln, E.rows(q), l, E.weights_view(w), kv)
        check_weights(Rows(), q, l, new, held, w, before, layer=layer, what=f"layer {layer}")
        E.epikv_attention_weights(ctx, layer, S, seq_ids, cu, 200, ln, E.rows(q), l, E.weights_view(w), kv, last=1)
        check_weights(Rows(), q, l, new, held, w, w.clone(), layer=layer, last=1, what=f"layer {layer}, one token")
    assert E.epikv_attn_get_error(ctx) == OK
