"""Rotary positions against float64: layouts, part of a head, types, strides, in place, the inverse as gradient,
and the table's scalings."""
import math

import pytest
import torch

from paper_2606_26472_gb300 import epikv as E

from . import cache_ops as R

pytestmark = pytest.mark.gpu

HALF, INTER = E.EPIKV_ROPE_HALF, E.EPIKV_ROPE_INTERLEAVED
# rounding to nearest with 8, 11 and 24 significant bits
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def context(d):
    cfg = E.make_attn_config(max_seqs=1, max_cache_tokens=1, max_new_tokens=1, num_layers=1, num_heads=1,
                             num_kv_heads=1, head_dim=d)
    ws = torch.empty(E.epikv_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    return E.epikv_attn_init(cfg, ws, ws.numel()), ws


def close(y, ref, x, dtype, what):
    """Three 32-bit roundings of terms no larger than the pair's magnitudes, one rounding of the result."""
    err = (y.double() - ref).abs()
    tol = UNIT[dtype] * ref.abs() * 1.01 + 4 * 2.0 ** -24 * x.double().abs().amax(-1, keepdim=True) + 2.0 ** -25 * (
        dtype == torch.float16)
    assert bool((err <= tol).all()), (what, float((err / tol).max()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layout", [HALF, INTER])
@pytest.mark.parametrize("d,dim,heads,n", [(64, 64, 1, 1), (64, 48, 3, 7), (64, 18, 40, 5), (128, 128, 40, 33),
                                           (128, 112, 5, 130), (128, 32, 17, 3), (128, 34, 9, 2), (256, 256, 8, 9),
                                           (256, 66, 3, 4), (256, 2, 2, 3)])
def test_rotation(gpu_lib, dtype, layout, d, dim, heads, n):
    g = torch.Generator(device="cuda").manual_seed(d + dim + n)
    ctx, _ws = context(d)
    cs = R.table64(5000, dim).float().cuda()
    wide = torch.randn(n, heads + 2, d, generator=g, device="cuda").to(dtype)
    x = wide[:, 1:heads + 1] if (d * wide.element_size()) % 16 == 0 else wide[:, :heads]
    keep = wide.clone()
    pos = torch.randint(0, 5000, (n,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 4999
    view = E.rope_view(cs, layout)
    for inverse in (False, True):
        out = torch.full((n, heads, d), float("nan"), dtype=dtype, device="cuda")
        E.epikv_rope(ctx, n, heads, E.rows(x), E.rows(out), pos, view, inverse=inverse)
        close(out, R.rotate64(x, cs[pos.long()], dim, layout, inverse), x, dtype, (inverse,))
        assert torch.equal(out[..., dim:], x[..., dim:])
    assert torch.equal(wide, keep)
    E.epikv_rope(ctx, n, heads, E.rows(x), E.rows(x), pos, view)          # in place, among other heads
    again = torch.empty_like(out)
    E.epikv_rope(ctx, n, heads, E.rows(keep[:, 1:heads + 1] if x.storage_offset() else keep[:, :heads]),
                 E.rows(again), pos, view)
    assert torch.equal(x, again)
    off = 1 if x.storage_offset() else 0
    assert torch.equal(wide[:, :off], keep[:, :off]) and torch.equal(wide[:, heads + off:], keep[:, heads + off:])
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)


def test_head_major_rows(gpu_lib):
    ctx, _ws = context(128)
    x = torch.randn(6, 50, 128, device="cuda").to(torch.bfloat16).transpose(0, 1)     # [tokens, heads, d] of [heads, tokens, d]
    out = torch.empty(50, 6, 128, dtype=torch.bfloat16, device="cuda")
    cs = R.table64(64, 128).float().cuda()
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    E.epikv_rope(ctx, 50, 6, E.rows(x), E.rows(out), pos, E.rope_view(cs))
    close(out, R.rotate64(x, cs[pos.long()], 128, HALF), x, torch.bfloat16, "head major")


@pytest.mark.parametrize("layout", [HALF, INTER])
def test_inverse_is_the_gradient(gpu_lib, layout):
    """L(x) = sum g * rope(x) is linear: its gradient is the inverse rotation of g, and equals differences of L."""
    ctx, _ws = context(64)
    cs = R.table64(100, 48).float().cuda()
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, g = (torch.randn(4, 2, 64, generator=gen, device="cuda") for _ in range(2))
    pos = torch.tensor([0, 1, 50, 99], dtype=torch.int32, device="cuda")
    view = E.rope_view(cs, layout)
    dx, y0, y1 = (torch.empty_like(x) for _ in range(3))
    E.epikv_rope(ctx, 4, 2, E.rows(g), E.rows(dx), pos, view, inverse=True)
    a = x.double().requires_grad_()
    (R.rotate64(a, cs[pos.long()], 48, layout) * g.double()).sum().backward()
    assert float((dx.double() - a.grad).abs().max()) < 4 * 2.0 ** -24 * float(g.abs().max()) * 2
    E.epikv_rope(ctx, 4, 2, E.rows(x), E.rows(y0), pos, view)
    for k in range(0, 4 * 2 * 64, 37):
        e = torch.zeros(4 * 2 * 64, device="cuda")
        e[k] = 1.0
        E.epikv_rope(ctx, 4, 2, E.rows(x + e.view_as(x)), E.rows(y1), pos, view)
        diff = float(((y1.double() - y0.double()) * g.double()).sum())
        assert abs(diff - float(dx.view(-1)[k])) < 64 * 2.0 ** -24 * 8 * float(g.abs().max())


def test_position_outside_the_table(gpu_lib):
    ctx, _ws = context(64)
    cs = R.table64(10, 64).float().cuda()
    x = torch.randn(4, 3, 64, device="cuda").to(torch.bfloat16)
    out = torch.zeros_like(x)
    pos = torch.tensor([3, 10, -1, 9], dtype=torch.int32, device="cuda")
    E.epikv_rope(ctx, 4, 3, E.rows(x), E.rows(out), pos, E.rope_view(cs))
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_EDEVICE, E.EPIKV_DEV_POSITION)
    assert E.epikv_attn_get_error(ctx) == (E.EPIKV_OK, 0)
    assert not out[1:3].any() and out[0].any() and out[3].any()


@pytest.mark.parametrize("kw", [dict(), dict(scaling=E.EPIKV_ROPE_LINEAR, factor=4.0),
                                dict(scaling=E.EPIKV_ROPE_NTK, factor=8.0, theta=500000.0),
                                dict(scaling=E.EPIKV_ROPE_BYPARTS, factor=8.0, low=1.0, high=4.0, original=8192),
                                dict(scaling=E.EPIKV_ROPE_BYPARTS, factor=16.0, low=1.0, high=32.0, original=4096,
                                     magnitude=0.1 * math.log(16.0) + 1)])
def test_table(gpu_lib, kw):
    dim, n = 96, 70001
    t = E.epikv_rope_table(E.make_rope_config(dim, **kw), n)
    theta, factor = kw.get("theta", 10000.0), kw.get("factor", 1.0)
    kind = kw.get("scaling", E.EPIKV_ROPE_PLAIN)
    if kind == E.EPIKV_ROPE_NTK:
        theta *= factor ** (dim / (dim - 2))
    f = theta ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    if kind == E.EPIKV_ROPE_LINEAR:
        f = f / factor
    if kind == E.EPIKV_ROPE_BYPARTS:
        g = ((kw["original"] * f / (2 * math.pi) - kw["low"]) / (kw["high"] - kw["low"])).clamp(0, 1)
        f = f * ((1 - g) / factor + g)
    a = torch.arange(n, dtype=torch.float64)[:, None] * f
    m = float(torch.tensor(kw.get("magnitude", 1.0), dtype=torch.float32))
    ref = torch.stack([a.cos(), a.sin()], -1) * m
    # an angle of up to 7e4 is off by a few units of 2^-52 of it; the value is rounded once
    assert float((t.cpu().double() - ref).abs().max()) < 2.0 ** -24 * m + 1e-9


def test_refusals(gpu_lib):
    ctx, _ws = context(64)
    cs = R.table64(10, 64).float().cuda()
    x = torch.randn(4, 3, 64, device="cuda").to(torch.bfloat16)
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    ok = dict(n=4, h=3, x=E.rows(x), y=E.rows(x.clone()), pos=pos, rope=E.rope_view(cs))

    def call(**kw):
        a = {**ok, **kw}
        E.epikv_rope(ctx, a["n"], a["h"], a["x"], a["y"], a["pos"], a["rope"])

    call()
    call(n=0)
    long = E.rope_view(R.table64(10, 128).float().cuda())
    odd = E.epikv_rows(x.data_ptr(), 3 * 64, 60, E.EPIKV_TYPE_BF16)
    off = E.epikv_rows(x.data_ptr() + 2, 3 * 64, 64, E.EPIKV_TYPE_BF16)
    no_layout = E.rope_view(cs, 2)
    for bad in (dict(n=-1), dict(x=None), dict(y=None), dict(pos=None), dict(rope=None), dict(rope=long), dict(x=odd),
                dict(x=off), dict(y=E.rows(x.float())), dict(rope=no_layout)):
        with pytest.raises(E.EpikvError) as err:
            call(**bad)
        assert err.value.status == E.EPIKV_EINVAL, bad
    for bad in (dict(dim=3), dict(dim=0), dict(theta=1.0), dict(scaling=4), dict(scaling=1, factor=0.5),
                dict(scaling=3, low=4.0, high=4.0), dict(scaling=3, original=0), dict(dim=2, scaling=2),
                dict(magnitude=float("nan"))):
        with pytest.raises(E.EpikvError):
            E.epikv_rope_table(E.make_rope_config(**{"dim": 64, **bad}), 4)
    with pytest.raises(ValueError):
        E.rows(x.transpose(1, 2))
    with pytest.raises(ValueError):
        E.rope_view(cs.double())
