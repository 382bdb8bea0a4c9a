"""Plain forms in 64 bits and error bounds of the chunk's attention and of what slots receive of it."""
import math

import torch

from paper_2606_26472_gb300 import epikv as E

from . import cache_ops as R


def queries(n, Hq, d, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, Hq, d, generator=g, device="cuda").to(torch.bfloat16)


def attend(c, ctx, q, new, held, *, layer=0, seqs=None, causal=True, max_new=None, lse=True, out=None, stream=None):
    seq_ids, cu, ln = R.batch(new, held, seqs)
    o = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    l = torch.full(q.shape[:2], float("nan"), device="cuda") if lse else None
    E.epikv_attention_chunk(ctx, layer, len(new), seq_ids, cu, max(new) if max_new is None else max_new, ln, E.rows(q),
                            E.rows(o), c.c.view(), lse=l, causal=causal, stream=stream)
    return o, l


def check_attention(c, q, o, l, new, held, *, layer=0, seqs=None, causal=True, scale=None, what=""):
    """A probability is rounded once, by half a step of its type (bf16 2^-8, half 2^-11, or 2^-32 of the row's largest where
    a half has no more bits); the other parts as in cache_ops.assert_attention_close, with the 32-bit sum over the slots."""
    scale = 1 / math.sqrt(c.d) if scale is None else scale
    t = 0
    for b, n in enumerate(new):
        s = b if seqs is None else seqs[b]
        top = held[b] + (n if causal else 0)
        k, v = c.read(0, layer, s, top), c.read(1, layer, s, top)
        limits = [held[b] + (i + 1 if causal else 0) for i in range(n)]
        ref, lse, big, qk = R.attention64(q[t:t + n], k, v, limits, scale)
        ds = c.d * 2.0 ** -24 * qk + 1e-6
        p = 2.0 ** -8 if c.bits == 16 else 2.0 ** -11
        tiny = 0.0 if c.bits == 16 or top == 0 else top * 2.0 ** -32 * float(v.abs().max())
        tol = 2.0 ** -8 * ref.abs() + (p + 2.0 ** -21 + top * 2.0 ** -24 + 2 * ds[..., None]) * big + tiny + 1e-30
        err = (o[t:t + n].double() - ref).abs()
        bad = ~(err <= tol) & ~(o[t:t + n].isnan() & ref.isnan())
        assert not bad.any(), (f"{what} entry {b}: {int(bad.sum())} of {bad.numel()} outputs off, first at "
                               f"{bad.nonzero()[0].tolist()}, worst {float((err / tol).nan_to_num(9e9).max()):.3g} of the bound")
        if l is not None:
            got, fin = l[t:t + n].double(), lse.isfinite()
            assert torch.equal(got[~fin].nan_to_num(7.0), lse[~fin].nan_to_num(7.0)), f"{what} entry {b}: lse of empty rows"
            e = (got - lse)[fin].abs()
            bound = (ds + 2.0 ** -22 * (1 + lse.abs()) + top * 2.0 ** -24)[fin]
            assert bool((e <= bound).all()), f"{what} entry {b}: lse off by {float((e / bound).max()):.3g} of the bound"
        t += n


def weigh(c, ctx, q, lse, new, held, w, *, layer=0, seqs=None, causal=True, last=0, add=False, max_new=None, stream=None):
    seq_ids, cu, ln = R.batch(new, held, seqs)
    E.epikv_attention_weights(ctx, layer, len(new), seq_ids, cu, max(new) if max_new is None else max_new, ln, E.rows(q), lse,
                              E.weights_view(w), c.c.view(), causal=causal, last=last, add=add, stream=stream)


def lse64(c, q, new, held, *, layer=0, seqs=None, causal=True, scale=None):
    """The rows' log-sums as the 32-bit numbers that an attention call would give."""
    scale = 1 / math.sqrt(c.d) if scale is None else scale
    out, t = [], 0
    for b, n in enumerate(new):
        s = b if seqs is None else seqs[b]
        top = held[b] + (n if causal else 0)
        k = c.read(0, layer, s, top)
        limits = [held[b] + (i + 1 if causal else 0) for i in range(n)]
        out.append(R.attention64(q[t:t + n], k, k, limits, scale)[1].float())
        t += n
    return torch.cat(out) if out else torch.zeros(q.shape[:2], device="cuda")


def check_weights(c, q, lse, new, held, w, before, *, layer=0, seqs=None, causal=True, last=0, add=False, scale=None,
                  what=""):
    """w against the sums of exp(score - lse).  Scores are 32-bit sums of d products; the exponent is formed in 32 bits
    from numbers up to |score| + |lse| (2^-22 of them), the exponential is good to 2^-22, the sum over the rows to 2^-24
    a term; below 2^-126 an exponential is 0.  Everything that is not an entry's slot is as before."""
    scale = 1 / math.sqrt(c.d) if scale is None else scale
    rep = q.shape[1] // c.H
    left = before.clone()
    t = 0
    for b, n in enumerate(new):
        s = b if seqs is None else seqs[b]
        top = held[b] + (n if causal else 0)
        if top == 0:
            t += n
            continue
        k = c.read(0, layer, s, top)
        first = max(0, n - last) if last else 0
        qq, ll = q[t + first:t + n].double(), lse[t + first:t + n].double()
        m = n - first
        t += n
        left[s, :, :top] = w[s, :, :top]
        want = torch.zeros(c.H, top, dtype=torch.float64, device="cuda")
        rel = torch.zeros(c.H, top, dtype=torch.float64, device="cuda")
        if m:
            seen = torch.arange(top, device="cuda") < torch.tensor([held[b] + (first + i + 1 if causal else 0) for i in range(m)],
                                                                   device="cuda")[:, None]
            for h in range(c.H):
                sc = torch.einsum("mrd,td->mrt", qq[:, h * rep:(h + 1) * rep], k[:, h]) * scale
                l_ = ll[:, h * rep:(h + 1) * rep, None]
                p = torch.where(seen[:, None] & (l_ != -math.inf), torch.exp(sc - l_), torch.zeros_like(sc))
                mag = torch.einsum("mrd,td->mrt", qq[:, h * rep:(h + 1) * rep].abs(), k[:, h].abs()) * abs(scale)
                r = c.d * 2.0 ** -24 * mag + 2.0 ** -22 * (2 + sc.abs() + l_.abs()) + m * rep * 2.0 ** -24
                want[h] = p.sum((0, 1))
                rel[h] = torch.where(p > 0, p * r, torch.zeros_like(p)).sum((0, 1))
        old = before[s, :, :top].double() if add else torch.zeros_like(want)
        got = w[s, :, :top].double()
        err = (got - (old + want)).abs()
        tol = rel * 1.01 + 2.0 ** -24 * (old + want).abs() + m * rep * 2.0 ** -126
        bad = ~(err <= tol) & ~(got.isnan() & want.isnan()) & ~(got == old + want)
        assert not bad.any(), (f"{what} entry {b}: {int(bad.sum())} of {bad.numel()} weights off, first at "
                               f"{bad.nonzero()[0].tolist()}, worst {float((err / tol).nan_to_num(9e9).max()):.3g} of the bound")
    assert torch.equal(left.view(torch.int32), w.view(torch.int32)), f"{what}: written outside the entries' slots"
