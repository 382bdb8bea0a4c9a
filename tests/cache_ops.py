"""Plain forms of the cache operators, in 64 bits or exactly, and a cache to run them on."""
import numpy as np
import torch

from paper_2606_26472_gb300 import epikv as E
from paper_2606_26472_gb300.cache import KVCache

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


# ------------------------------------------------------------------ 4-bit rows
def quantize(x, g=None):
    """Codes (0..15) and scale bytes of bf16 [n, H, d]; g: a positive float32 scale per head or None.  The definition
    in include/epikv.h with its 32-bit divisions, each rounded once."""
    n, H, d = x.shape
    y = x.float()
    if g is not None:
        y = y / g.float()[None, :, None]
    y = y.view(n, H, d // 16, 16)
    top = (y.abs().amax(-1) / 6.0).clamp(max=448.0)
    scale = top.to(torch.float8_e4m3fn)
    s = scale.float()[..., None]
    z = torch.where(s > 0, y / s, torch.zeros_like(y)).double()
    edges = ((E2M1[1:] + E2M1[:-1]) / 2).to(x.device)
    code = torch.zeros(z.shape, dtype=torch.int64, device=x.device)
    for i, e in enumerate(edges.tolist()):       # a tie goes to the even code
        code += ((z.abs() > e) | ((z.abs() == e) & (i % 2 == 1))).long()
    code += 8 * torch.signbit(z).long()
    nan = y.isnan().any(-1)
    byte = torch.where(nan, torch.full_like(scale.view(torch.uint8), 0x7F), scale.view(torch.uint8))
    code = torch.where(nan[..., None], torch.zeros_like(code), code)
    return code.view(n, H, d), byte


def pack(x, units, g=None):
    """bf16 [n, H, d] as 4-bit rows, uint8 [n, 2 * units] (padding zero)."""
    n, H, d = x.shape
    code, byte = quantize(x, g)
    out = torch.zeros(n, 2 * units, dtype=torch.uint8, device=x.device)
    c = code.view(n, H, d // 2, 2)
    out[:, :H * d // 2] = (c[..., 0] + 16 * c[..., 1]).to(torch.uint8).reshape(n, H * d // 2)
    out[:, H * d // 2:H * (d // 2 + d // 16)] = byte.reshape(n, H * d // 16)
    return out


def values(packed, H, d, g=None):
    """The float64 values [n, H, d] that 4-bit rows stand for."""
    n = packed.shape[0]
    c = packed[:, :H * d // 2].long()
    code = torch.stack([c & 15, c >> 4], -1).view(n, H, d // 16, 16)
    lut = torch.cat([E2M1, -E2M1]).to(packed.device)
    s = packed[:, H * d // 2:H * (d // 2 + d // 16)].contiguous().view(torch.float8_e4m3fn).double()
    v = (lut[code] * s.view(n, H, d // 16, 1)).view(n, H, d)
    return v if g is None else v * g.double()[None, :, None]


# ------------------------------------------------------------------ rotation
def table64(n_pos, dim, theta=10000.0):
    f = theta ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1)


def rotate64(x, cs, dim, layout, inverse=False):
    """float64 [n, heads, d] rotated by cs [n, dim / 2, 2]."""
    y = x.double().clone()
    i = torch.arange(dim // 2, device=x.device)
    lo, hi = (i, i + dim // 2) if layout == E.EPIKV_ROPE_HALF else (2 * i, 2 * i + 1)
    c, s = cs[:, None, :, 0].double(), cs[:, None, :, 1].double() * (-1 if inverse else 1)
    y[..., lo] = x[..., lo].double() * c - x[..., hi].double() * s
    y[..., hi] = x[..., hi].double() * c + x[..., lo].double() * s
    return y


def rotate32(x, cs, dim, layout):
    """The same, each product and sum rounded to 32 bits, the result to bf16."""
    y = x.float().clone()
    i = torch.arange(dim // 2, device=x.device)
    lo, hi = (i, i + dim // 2) if layout == E.EPIKV_ROPE_HALF else (2 * i, 2 * i + 1)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    y[..., lo] = x[..., lo].float() * c - x[..., hi].float() * s
    y[..., hi] = x[..., hi].float() * c + x[..., lo].float() * s
    return y.to(torch.bfloat16)


# ------------------------------------------------------------------ a cache
class Cache:
    """One or more layers of K and V, their values known: kv[w][layer, seq, slot] is bf16 [H, d]."""

    def __init__(self, *, seqs, T, H, d, bits=16, block=16, layers=1, seed=0, kv_scale=None, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        fmt = E.EPIKV_CACHE_E2M1 if bits == 4 else E.EPIKV_CACHE_BF16
        self.S, self.T, self.H, self.d, self.bits, self.L, self.fmt = seqs, T, H, d, bits, layers, fmt
        kw = {}
        if block:
            mb = (T + block - 1) // block
            perm = np.random.default_rng(seed).permutation(seqs * mb).astype(np.int32).reshape(seqs, mb)
            kw = dict(block_size=block, block_table=perm)
        layout = E.EPIKV_LAYOUT_PAGED if block else E.EPIKV_LAYOUT_CONTIGUOUS
        self.c = KVCache(layout, layers, H, d, max_seqs=seqs, max_tokens=T, cache_format=fmt, **kw)
        self.kv_scale = kv_scale
        channel = torch.exp(0.5 * torch.randn(H, d, generator=g, device="cuda"))
        for w, pool in enumerate((self.c.k, self.c.v)):
            n = pool.numel() // (self.c.H * self.c.d)
            x = torch.randn(n, H, d, generator=g, device="cuda") * spread * (0.7 * channel if w == 0 else 1.0)
            self.put(pool, x.to(torch.bfloat16), w)

    @property
    def units(self):
        return self.c.H * self.c.d

    def raw(self, w):
        """uint8 [rows, bytes] of the whole pool."""
        pool = self.c.v if w else self.c.k
        return pool.view(torch.uint8).view(-1, 2 * self.units)

    def put(self, pool, x, w):
        if self.bits == 16:
            pool.view(-1, self.H, self.d).copy_(x)
            return
        if self.kv_scale is None:
            pool.view(torch.uint8).view(-1, 2 * self.units).copy_(pack(x, self.units))
            return
        per = x.shape[0] // self.L
        for l in range(self.L):
            pool.view(torch.uint8).view(-1, 2 * self.units)[l * per:(l + 1) * per].copy_(
                pack(x[l * per:(l + 1) * per], self.units, self.kv_scale[w, l]))

    def index(self, layer, seq, slots):
        """Rows of raw() that hold the slots."""
        slots = torch.as_tensor(slots, device="cuda").long()
        if self.c.layout == E.EPIKV_LAYOUT_CONTIGUOUS:
            return (layer * self.S + seq) * self.T + slots
        bs = self.c.block_size
        return layer * self.c.num_blocks * bs + self.c.block_table[seq].long()[slots // bs] * bs + slots % bs

    def read(self, w, layer, seq, n):
        """float64 [n, H, d] of slots 0..n-1."""
        r = self.raw(w)[self.index(layer, seq, torch.arange(n))]
        if self.bits == 16:
            return r.contiguous().view(torch.bfloat16).view(n, self.H, self.d).double()
        return values(r, self.H, self.d, None if self.kv_scale is None else self.kv_scale[w, layer])

    def context(self, Hq, max_new, **kw):
        cfg = E.make_attn_config(max_seqs=self.S, max_cache_tokens=self.T, max_new_tokens=max_new,
                                 num_layers=self.L, num_heads=Hq, num_kv_heads=self.H, head_dim=self.d,
                                 cache_format=self.fmt, kv_scale=self.kv_scale, **kw)
        n = E.epikv_attn_workspace_bytes(cfg)
        assert n > 0
        self.ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        return E.epikv_attn_init(cfg, self.ws, n)


def batch(new, held, seqs=None):
    """Device arrays (seq_ids, cu_new, len) of a batch."""
    seqs = list(range(len(new))) if seqs is None else seqs
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return t(seqs), t(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), t(held)


def attention64(q, k, v, limits, scale):
    """float64 attention of rows q [m, Hq, d] over k, v [T, H, d]; row i sees slots below limits[i].  Returns (out,
    lse, sum_j p_j |v_j|, the largest sum_c |q_c k_jc| * scale of a row's slots): the last two scale the tolerances."""
    m, Hq, d = q.shape
    rep = Hq // k.shape[1]
    k, v = (x.repeat_interleave(rep, 1) for x in (k, v))
    seen = torch.arange(k.shape[0], device=q.device)[None, :] < torch.as_tensor(limits, device=q.device)[:, None]
    kz = torch.where(seen.any(0)[:, None, None], k, torch.zeros_like(k))
    s = torch.einsum("mhd,thd->mht", q.double(), kz) * scale
    s = s.masked_fill(~seen[:, None, :], -torch.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(seen[:, None, :], torch.exp(s - lse[..., None]), torch.zeros_like(s))
    some = seen.any(1)
    p = torch.where(some[:, None, None], p, torch.zeros_like(p))
    out = torch.zeros(m, Hq, d, dtype=torch.float64, device=q.device)
    big = torch.zeros_like(out)
    for i in range(m):                           # only what the row sees enters its sums
        n = int(limits[i])
        if n > 0:
            out[i] = torch.einsum("ht,thd->hd", p[i, :, :n], v[:n])
            big[i] = torch.einsum("ht,thd->hd", p[i, :, :n], v[:n].abs())
    qk = torch.einsum("mhd,thd->mht", q.double().abs(), kz.abs()) * abs(scale)
    qk = torch.where(seen[:, None, :], qk, torch.zeros_like(qk)).amax(-1) if k.shape[0] else torch.zeros_like(lse)
    return out, torch.where(some[:, None], lse, torch.full_like(lse, -torch.inf)), big, qk


def assert_attention_close(out, lse, ref, what=""):
    """Bounds: a score is a 32-bit sum of d products (d 2^-24 of the sum of magnitudes) and so an absolute error of a
    log-probability; a probability is rounded to 11 bits or more before its product (2^-11 of sum p|v| with the
    running sums); the output is rounded once to bf16 (8 significant bits: 2^-8)."""
    o, l, big, qk = ref
    d = o.shape[-1]
    ds = d * 2.0 ** -24 * qk + 1e-6
    err = (out.double() - o).abs()
    tol = 2.0 ** -8 * o.abs() + (2.0 ** -11 + 2 * ds[..., None]) * big + 1e-30
    bad = ~(err <= tol) & ~(out.double().isnan() & o.isnan())
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outputs off, first at {bad.nonzero()[0].tolist()}, " \
                          f"worst {float((err / tol).nan_to_num(0).max()):.3g} of the bound"
    if lse is not None:
        fin = l.isfinite()
        assert torch.equal(lse[~fin].double().nan_to_num(7.0), l[~fin].nan_to_num(7.0)), f"{what}: lse of empty rows"
        e = (lse.double() - l)[fin].abs()
        t = (ds + 2.0 ** -22 * (1 + l.abs()))[fin]
        assert bool((e <= t).all()), f"{what}: lse off by {float((e / t).max()):.3g} of the bound"
