"""epikv_append and epikv_cache_read: the stored rows bit for bit (bf16 and 4 bits), nothing else written, rotation by
position at slots that are not positions, and what is refused or reported."""
import pytest
import torch

from paper_2606_26472_gb300 import epikv as E

from . import cache_ops as R

pytestmark = pytest.mark.gpu

HALF, INTER = E.EPIKV_ROPE_HALF, E.EPIKV_ROPE_INTERLEAVED


def make(n, Hq, H, d, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, Hq + 2 * H, d, generator=g, device="cuda").to(torch.bfloat16)


def append(c, ctx, qkv, Hq, new, held, pos, view, layer=0, seqs=None, q=True, max_new=None):
    H = c.H
    seq_ids, cu, ln = R.batch(new, held, seqs)
    q_out = torch.full((qkv.shape[0], Hq, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    p = torch.tensor(pos, dtype=torch.int32, device="cuda") if pos is not None else None
    E.epikv_append(ctx, layer, len(new), seq_ids, cu, max(new) if max_new is None else max_new, ln, p,
                   E.rows(qkv[:, :Hq]) if q else None, E.rows(q_out) if q else None, E.rows(qkv[:, Hq:Hq + H]),
                   E.rows(qkv[:, Hq + H:]), view, c.c.view())
    return q_out


def expected(c, qkv, Hq, new, held, pos, cs, dim, layout, layer=0, seqs=None):
    """(rotated queries, the pools' bytes after the call)."""
    H, seqs = c.H, list(range(len(new))) if seqs is None else seqs
    at = torch.cat([torch.arange(n) + p for n, p in zip(new, pos or [0] * len(new))]).cuda() if sum(new) else None
    turned = qkv[:, :Hq + H]
    if dim:
        turned = R.rotate32(turned, cs[at], dim, layout)
    pools = [c.raw(0).clone(), c.raw(1).clone()]
    used = 2 * c.units if c.bits == 16 else H * (c.d // 2 + c.d // 16)
    t = 0
    for b, n in enumerate(new):
        idx = c.index(layer, seqs[b], torch.arange(held[b], held[b] + n))
        for w, x in enumerate((turned[t:t + n, Hq:], qkv[t:t + n, Hq + H:])):
            x = x.contiguous()
            g = None if c.kv_scale is None else c.kv_scale[w, layer]
            rows = x.view(n, H * c.d).view(torch.uint8) if c.bits == 16 else R.pack(x, c.units, g)
            pools[w][idx, :used] = rows[:, :used]
        t += n
    return turned[:, :Hq], pools


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("block", [0, 16, 7])
@pytest.mark.parametrize("H,Hq,d,dim,layout", [(8, 32, 128, 128, HALF), (1, 1, 64, 64, INTER), (2, 14, 128, 96, INTER),
                                               (3, 3, 256, 256, HALF), (5, 5, 64, 48, HALF), (4, 8, 128, 34, HALF),
                                               (1, 8, 256, 18, INTER), (2, 2, 64, 0, HALF), (11, 11, 128, 112, HALF)])
def test_rows_bit_for_bit(gpu_lib, bits, block, H, Hq, d, dim, layout):
    new, held, pos = [1, 0, 37, 16, 5], [0, 9, 15, 48, 130], [0, 3, 900, 48, 1995]
    c = R.Cache(seqs=6, T=137, H=H, d=d, bits=bits, block=block, layers=2, seed=H + d)
    ctx = c.context(Hq, 64)
    cs = R.table64(2000, dim).float().cuda() if dim else None
    view = E.rope_view(cs, layout) if dim else None
    qkv = make(sum(new), Hq, H, d, seed=dim)
    seqs = [4, 0, 2, 5, 1]
    want_q, want = expected(c, qkv, Hq, new, held, pos, cs, dim, layout, layer=1, seqs=seqs)
    q_out = append(c, ctx, qkv, Hq, new, held, pos, view, layer=1, seqs=seqs)
    assert torch.equal(q_out, want_q)
    for w in range(2):
        assert torch.equal(c.raw(w), want[w]), f"pool {w}"
    # reading back gives the values that the rows stand for
    rows_seq = torch.tensor([s for s, n in zip(seqs, new) for _ in range(n)], dtype=torch.int32, device="cuda")
    rows_slot = torch.tensor([h + i for h, n in zip(held, new) for i in range(n)], dtype=torch.int32, device="cuda")
    n = sum(new)
    kv = [torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    E.epikv_cache_read(ctx, 1, n, rows_seq, rows_slot, E.rows(kv[0]), E.rows(kv[1]), c.c.view())
    for w in range(2):
        t = 0
        for s, h, m in zip(seqs, held, new):
            ref = c.read(w, 1, s, h + m)[h:]
            assert torch.equal(kv[w][t:t + m].double(), ref.to(torch.bfloat16).double())
            t += m
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


def test_quantisation_edges(gpu_lib):
    """Ties, zeros of both signs, tiny, huge, infinite and NaN groups."""
    d = 64
    x = torch.zeros(8, 1, d)
    x[0, 0, :16] = torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -5, .2, -.2, 0, -0.0])
    x[1] = torch.randn(d) * 1e-4                        # scales among E4M3's subnormals, or zero
    x[2] = torch.randn(d) * 1e5                         # saturates
    x[3, 0, :16] = torch.randn(16)
    x[3, 0, 3] = float("inf")
    x[4, 0, 16:32] = torch.randn(16)
    x[4, 0, 20] = float("nan")
    x[5] = torch.randn(d) * 3e38
    x[6] = torch.randn(d) * 1e-38
    x = x.to(torch.bfloat16).cuda()
    for block in (0, 16):
        c = R.Cache(seqs=1, T=8, H=1, d=d, bits=4, block=block)
        ctx = c.context(1, 8)
        qkv = torch.cat([x, x, x.flip(0)], 1).contiguous()
        _, want = expected(c, qkv, 1, [8], [0], None, None, 0, HALF)
        append(c, ctx, qkv, 1, [8], [0], None, None, q=False)
        for w in range(2):
            assert torch.equal(c.raw(w), want[w])
        assert c.read(0, 0, 0, 8)[4, 0, 16:32].isnan().all() and c.read(0, 0, 0, 8)[4, 0, :16].isfinite().all()


def test_every_bf16_against_every_scale(gpu_lib):
    """Every positive bf16 value of a binade range beside every maximum's scale: all quotients near a boundary."""
    mant = torch.arange(128).float() / 128 + 1                       # all significands
    tops = (mant[None, :] * 2.0 ** torch.arange(-8, 9)[:, None]).flatten()
    vals = (mant[None, :] * 2.0 ** torch.arange(-5, 1)[:, None]).flatten()
    x = torch.zeros(tops.numel(), 64)
    gen = torch.Generator().manual_seed(5)
    for g in range(4):
        x[:, 16 * g] = tops
        pick = torch.randint(0, vals.numel(), (tops.numel(), 15), generator=gen)
        sign = torch.randint(0, 2, pick.shape, generator=gen).float() * 2 - 1
        x[:, 16 * g + 1:16 * g + 16] = vals[pick] * sign * 2.0 ** torch.floor(torch.log2(tops))[:, None]
    x = x.to(torch.bfloat16).cuda().view(-1, 1, 64)
    n = x.shape[0]
    c = R.Cache(seqs=1, T=n, H=1, d=64, bits=4, block=0)
    ctx = c.context(1, n)
    qkv = torch.cat([x, x, -x.flip(0)], 1).contiguous()
    _, want = expected(c, qkv, 1, [n], [0], None, None, 0, HALF)
    append(c, ctx, qkv, 1, [n], [0], None, None, q=False)
    for w in range(2):
        assert torch.equal(c.raw(w), want[w])


def test_every_significand_at_every_scale(gpu_lib):
    """For each of E4M3's positive scales, subnormal ones too, every bf16 value from an eighth of it to its group's
    maximum, of both signs in turn: 15 of them beside the maximum in each group of 16."""
    groups = []
    every = torch.arange(1, 0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    positive = torch.arange(0x0001, 0x7F80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    scales = (positive / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn).float()     # what a maximum gives
    for s in every.tolist():
        tops = positive[scales == s]
        assert tops.numel(), s
        for top in {tops[0].item(), tops[-1].item(), tops[tops.numel() // 2].item()} if s < 448 else {2688.0, 3000.0, 1e5}:
            top = torch.tensor(top).to(torch.bfloat16).item()
            x = positive[(positive >= s / 8) & (positive <= top)]
            x = torch.cat([x, x.new_zeros(-x.numel() % 15)]).view(-1, 15)
            x = x * (1.0 - 2.0 * (torch.arange(x.numel()) % 2)).view(-1, 15)
            groups.append(torch.cat([x.new_full((x.shape[0], 1), top), x], 1))
    x = torch.cat(groups)
    x = torch.cat([x, x.new_zeros(-x.shape[0] % 4, 16)]).view(-1, 1, 64).to(torch.bfloat16).cuda()
    n = x.shape[0]
    c = R.Cache(seqs=1, T=n, H=1, d=64, bits=4, block=0)
    ctx = c.context(1, n)
    qkv = torch.cat([x, x, -x.flip(0)], 1).contiguous()
    _, want = expected(c, qkv, 1, [n], [0], None, None, 0, HALF)
    append(c, ctx, qkv, 1, [n], [0], None, None, q=False)
    for w in range(2):
        assert torch.equal(c.raw(w), want[w])
    got = c.raw(0)[c.index(0, 0, torch.arange(n))][:, 32:36].flatten()
    assert set(range(1, 0x7F)) <= set(got.tolist())


def test_head_scales(gpu_lib):
    s = torch.rand(2, 3, 2, device="cuda") * 30 + 0.01
    c = R.Cache(seqs=2, T=40, H=2, d=64, bits=4, layers=3, kv_scale=s, spread=20.0)
    ctx = c.context(4, 8)
    qkv = make(9, 4, 2, 64) * 20
    _, want = expected(c, qkv, 4, [4, 5], [3, 30], None, None, 0, HALF, layer=2)
    append(c, ctx, qkv, 4, [4, 5], [3, 30], None, None, layer=2)
    for w in range(2):
        assert torch.equal(c.raw(w), want[w])


def test_layer_lengths_read_with_a_stride(gpu_lib):
    c = R.Cache(seqs=2, T=64, H=2, d=64, bits=16, layers=3)
    ctx = c.context(2, 4)
    qkv = make(4, 2, 2, 64)
    _, want = expected(c, qkv, 2, [2, 2], [10, 40], None, None, 0, HALF, layer=1)
    seq_ids, cu, _ = R.batch([2, 2], [0, 0])
    lens = torch.tensor([[1, 10, 2], [3, 40, 4]], dtype=torch.int32, device="cuda")
    E.epikv_append(ctx, 1, 2, seq_ids, cu, 2, lens[:, 1:].data_ptr(), None, None, None, E.rows(qkv[:, 2:4]),
                   E.rows(qkv[:, 4:]), None, c.c.view(), len_stride=3)
    for w in range(2):
        assert torch.equal(c.raw(w), want[w])


def test_queries_in_place_on_another_stream(gpu_lib):
    c = R.Cache(seqs=1, T=64, H=2, d=128, bits=4)
    ctx = c.context(8, 16)
    cs = R.table64(100, 128).float().cuda()
    qkv = make(16, 8, 2, 128)
    want_q, want = expected(c, qkv, 8, [16], [20], [70], cs, 128, HALF)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    seq_ids, cu, ln = R.batch([16], [20])
    p = torch.tensor([70], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    q = E.rows(qkv[:, :8])
    E.epikv_append(ctx, 0, 1, seq_ids, cu, 16, ln, p, q, q, E.rows(qkv[:, 8:10]), E.rows(qkv[:, 10:]),
                   E.rope_view(cs), c.c.view(), stream=s)
    s.synchronize()
    assert torch.equal(qkv[:, :8], want_q)
    for w in range(2):
        assert torch.equal(c.raw(w), want[w])


def test_reported_and_skipped(gpu_lib):
    """What the device finds wrong is reported and written nowhere; the rest of the batch is done."""
    cs = R.table64(50, 64).float().cuda()
    cases = [(dict(new=[2, 2], held=[0, 63]), E.EPIKV_DEV_CAPACITY, [0]),
             (dict(new=[2, 2], held=[0, -1]), E.EPIKV_DEV_CAPACITY, [0]),
             (dict(new=[2, 2], held=[0, 0], seqs=[0, 2]), E.EPIKV_DEV_BATCH, [0]),
             (dict(new=[2, 3], held=[0, 0], max_new=2), E.EPIKV_DEV_BATCH, [0]),
             (dict(new=[2, 2], held=[0, 0], pos=[0, 49]), E.EPIKV_DEV_POSITION, None),
             (dict(new=[2, 2], held=[0, 0], pos=[0, -1]), E.EPIKV_DEV_POSITION, None)]
    for kw, code, good in cases:
        c = R.Cache(seqs=2, T=64, H=2, d=64, bits=4)
        ctx = c.context(2, 4)
        kw.setdefault("pos", [0, 0])
        qkv = make(sum(kw["new"]), 2, 2, 64)
        before = [c.raw(0).clone(), c.raw(1).clone()]
        append(c, ctx, qkv, 2, kw["new"], kw["held"], kw["pos"], E.rope_view(cs), seqs=kw.get("seqs"),
               max_new=kw.get("max_new"))
        assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, code), kw
        if good is not None:
            _, want = expected(c, qkv[:2], 2, [2], [0], [0], cs, 64, HALF)
            for w in range(2):
                assert not torch.equal(c.raw(w), before[w])
                idx = c.index(0, 0, torch.arange(2))
                assert torch.equal(c.raw(w)[idx], want[w][idx])
                before[w][idx] = want[w][idx]
                assert torch.equal(c.raw(w), before[w]), kw
    c = R.Cache(seqs=1, T=32, H=2, d=64, bits=16)
    ctx = c.context(2, 4)
    c.c.block_table[0, 1] = 99
    before = [c.raw(0).clone(), c.raw(1).clone()]
    append(c, ctx, make(2, 2, 2, 64), 2, [2], [16], None, None)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_SLOT)
    for w in range(2):
        assert torch.equal(c.raw(w), before[w])
    out = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    t = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    E.epikv_cache_read(ctx, 0, 3, t(0, 0, 1), t(3, 16, 0), E.rows(out), None, c.c.view())
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_SLOT)
    assert out[0].any() and not out[1:].any()


def test_refusals(gpu_lib):
    c = R.Cache(seqs=2, T=32, H=2, d=64, bits=16)
    ctx = c.context(4, 4)
    qkv = make(3, 4, 2, 64)
    seq_ids, cu, ln = R.batch([3], [0])
    cs = R.table64(50, 64).float().cuda()
    ok = dict(layer=0, n=1, seq_ids=seq_ids, cu=cu, max_new=3, ln=ln, pos=ln, q=E.rows(qkv[:, :4]),
              qo=E.rows(qkv[:, :4].clone()), k=E.rows(qkv[:, 4:6]), v=E.rows(qkv[:, 6:]), rope=E.rope_view(cs),
              kv=c.c.view(), ls=1)

    def call(**kw):
        a = {**ok, **kw}
        E.epikv_append(ctx, a["layer"], a["n"], a["seq_ids"], a["cu"], a["max_new"], a["ln"], a["pos"], a["q"],
                       a["qo"], a["k"], a["v"], a["rope"], a["kv"], len_stride=a["ls"])

    call()
    call(n=0)
    narrow = c.c.view()
    narrow.stride_token = 64
    skew = c.c.view()
    skew.stride_block += 4
    nobt = c.c.view()
    nobt.block_table = None
    f32 = E.rows(qkv[:, 4:6].float())
    for bad in (dict(layer=1), dict(layer=-1), dict(n=3), dict(n=-1), dict(max_new=5), dict(max_new=-1),
                dict(seq_ids=None), dict(cu=None), dict(ln=None), dict(pos=None), dict(q=None), dict(qo=None),
                dict(k=None), dict(v=None), dict(k=f32), dict(kv=None), dict(kv=narrow), dict(kv=skew),
                dict(kv=nobt), dict(ls=0)):
        with pytest.raises(E.EpikvError) as err:
            call(**bad)
        assert err.value.status == E.EPIKV_EINVAL, bad
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)
