"""The operators of prompts and of eviction by attention weight, as cases that can be timed.

Three kinds of call, by ``case["op"]``:

  chunk     a chunk of new tokens of each sequence attends over the slots of one layer's cache (bf16 or 4 bits), many
            query rows at a time
  weights   what each slot of one layer's cache received of the new tokens' attention: for every KV head the sum, over
            the new tokens and the query heads that read it, of exp(score - lse)
  evict     caches cut by what their slots received: the tokens are registered, the KV heads' weights of one or more
            steps are added up to the slots' scores (older ones decayed), and the kept slots are chosen

A 4-bit row of a token holds, for each head, d/2 bytes of codes (channel 2i in the low half of byte i), then for each
head d/16 bytes of scales: the value of a channel is its E2M1 code times the E4M3 scale of its 16 channels.  Rows are
counted in units of 2 bytes.
"""
import math

import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
RECENCY = 128          # the library's default


def listed():
    m = dict(heads=32, kv_heads=8, dim=128)
    return [
        # a few tokens of each of eight sequences, as drafts are checked or short turns are taken in
        dict(m, name="chunk_short8", op="chunk", bits=16, seqs=8, new=16, new_lo=16, held=4096, held_lo=4096, block=16),
        # a whole prompt into an empty cache
        dict(m, name="chunk_prompt_4k", op="chunk", bits=16, seqs=1, new=4096, new_lo=4096, held=0, held_lo=0, block=16),
        # the largest: the last piece of a long prompt that is taken in by pieces
        dict(m, name="chunk_long_2k", op="chunk", bits=16, seqs=1, new=2048, new_lo=2048, held=14336, held_lo=14336, block=16),
        # turns of unequal lengths, sizes that nothing divides, contiguous cache
        dict(name="chunk_ragged_odd", op="chunk", bits=16, heads=24, kv_heads=4, dim=64, seqs=6, new=211, new_lo=13, held=3001,
             held_lo=999, block=0),
        # pieces of prompts over 4-bit caches
        dict(m, name="chunk4_batch8", op="chunk", bits=4, seqs=8, new=256, new_lo=256, held=4096, held_lo=2048, block=16),
        # the smallest: a decode step of four short sequences
        dict(m, name="weights_decode4", op="weights", bits=16, seqs=4, new=1, new_lo=1, held=143, held_lo=128, block=16,
             last=0),
        # a decode step of a ragged serving batch
        dict(m, name="weights_decode64", op="weights", bits=16, seqs=64, new=1, new_lo=1, held=8192, held_lo=2048, block=16,
             last=0),
        # the same over 4-bit caches at their budget
        dict(m, name="weights4_decode32", op="weights", bits=4, seqs=32, new=1, new_lo=1, held=8319, held_lo=8192, block=16,
             last=0),
        # a whole prompt
        dict(m, name="weights_prompt_4k", op="weights", bits=16, seqs=1, new=4096, new_lo=4096, held=0, held_lo=0, block=16,
             last=0),
        # what the last 64 tokens of prompts' pieces look at, contiguous cache
        dict(name="weights_last64_odd", op="weights", bits=16, heads=24, kv_heads=4, dim=64, seqs=3, new=1003, new_lo=701,
             held=4099, held_lo=2999, block=0, last=64),
        # one 2,048-token sequence cut to 512
        dict(name="evict1_2k", op="evict", kv_heads=8, seqs=1, tokens=2048, tokens_lo=2048, budget=512, prefill=0, steps=1),
        # long sequences of unequal lengths cut to 4,096, the weights of a prompt and of what came behind it
        dict(name="evict6_32k", op="evict", kv_heads=8, seqs=6, tokens=32768, tokens_lo=12345, budget=4096, prefill=100,
             steps=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges; none costs more than the largest listed one."""
    op = rng.choice(["chunk", "chunk", "chunk", "weights", "weights", "weights", "evict"])
    if op == "evict":
        tokens = _log_int(rng, 300, 32768)
        return dict(op=op, kv_heads=rng.choice([1, 2, 4, 8]), seqs=rng.randint(1, 6), tokens=tokens,
                    tokens_lo=rng.randint(tokens // 3, tokens), budget=_log_int(rng, 64, max(65, tokens // 2)),
                    prefill=rng.choice([0, 0, 17, 100]), steps=rng.choice([1, 1, 2, 3]))
    dim = rng.choice([64, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8, 8] if dim < 256 else [1, 2, 4])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 7, 8])
    case = dict(op=op, bits=rng.choice([16, 16, 4]), heads=heads, kv_heads=kv_heads, dim=dim,
                block=rng.choice([0, 16, 16, 32, 64, 7]))
    if op == "weights" and rng.random() < 0.5:
        seqs, new = _log_int(rng, 1, 64), 1
        most = min(65536, 64 * 5120 * 1024 // (seqs * kv_heads * dim))
    else:
        seqs = _log_int(rng, 1, 16)
        new = _log_int(rng, 2, max(2, min(2048, 4096 // seqs)))
        # scores are within those of the long piece, caches within 512 MB of values
        most = min(16384, 2048 * 15360 * 32 * 128 // (seqs * heads * new * dim), 64 * 4096 * 1024 // (seqs * kv_heads * dim))
    held = _log_int(rng, 1, max(16, most)) if rng.random() < 0.85 else 0
    case.update(seqs=seqs, new=new, new_lo=rng.randint(max(1, new // 3), new), held=held,
                held_lo=rng.randint(held // 3, held))
    if op == "weights":
        case["last"] = rng.choice([0, 0, 16, 64])
    return case


# ---------------------------------------------------------------- sizes

def _spread(lo, hi, n):
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _row_units(case):
    """(units of one token's row of K or V, bytes of it that are in use).  The library moves rows as H' x d' bf16
    units with d' a power of two up to 256 and H' at most 32: a 4-bit row is padded until it is such a product."""
    H, d = case["kv_heads"], case["dim"]
    if case["bits"] == 16:
        return H * d, 2 * H * d
    used = H * (d // 2 + d // 16)
    units = -(-used // 16) * 8
    while units // min(256, units & -units) > 32:
        units += 8
    return units, used


def work(case):
    if case["op"] == "evict":
        n, h = sum(_spread(case["tokens_lo"], case["tokens"], case["seqs"])), case["kv_heads"]
        kept = case["seqs"] * min(case["budget"], case["tokens"])
        return {"bytes": n * (case["steps"] * (4 * h + 8) + 8) + 4 * kept, "flops": n * case["steps"] * (h + 1)}
    hq, h, d = case["heads"], case["kv_heads"], case["dim"]
    new = _spread(case["new_lo"], case["new"], case["seqs"])
    held = _spread(case["held_lo"], case["held"], case["seqs"])
    used = _row_units(case)[1]
    if case["op"] == "chunk":
        seen = sum(x * k + x * (x + 1) // 2 for x, k in zip(new, held))
        return {"bytes": 2 * used * sum(x + k for x, k in zip(new, held)) + sum(new) * hq * (4 * d + 4),
                "flops": 4 * d * hq * seen}
    seen = rows = 0
    for x, k in zip(new, held):
        y = min(x, case["last"] or x)
        seen += y * (k + x) - y * (y - 1) // 2
        rows += y
    slots = sum(x + k for x, k in zip(new, held))
    return {"bytes": used * slots + rows * hq * (2 * d + 4) + slots * h * 4, "flops": 2 * d * hq * seen}


# ---------------------------------------------------------------- inputs

def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _pack(rows, units):
    """bf16 rows [n, H, d] as 4-bit rows [n, units] of 2-byte units."""
    n, h, d = rows.shape
    y = rows.float().view(n, h, d // 16, 16)
    scale = (y.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = scale.float()[..., None]
    z = torch.where(s > 0, y / s, torch.zeros_like(y))
    a = z.abs()
    # to the nearest of E2M1's values, ties to the even code
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int()
            + (a >= 3.5).int() + (a > 5.0).int())
    code = (code + 8 * torch.signbit(z).int()).view(n, h, d // 2, 2)
    out = torch.zeros(n, units * 2, dtype=torch.uint8, device=rows.device)
    out[:, :h * d // 2] = (code[..., 0] + 16 * code[..., 1]).to(torch.uint8).view(n, h * d // 2)
    out[:, h * d // 2:h * (d // 2 + d // 16)] = scale.view(torch.uint8).view(n, h * d // 16)
    return out


def _values(rows, h, d, dtype=torch.float32):
    """4-bit rows [..., bytes] as the values they stand for, [..., h, d]."""
    lut = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=rows.device, dtype=dtype)
    c = rows[..., :h * d // 2].int()
    v = torch.stack([lut[c & 15], lut[c >> 4]], -1).view(*rows.shape[:-1], h, d // 16, 16)
    s = rows[..., h * d // 2:h * (d // 2 + d // 16)].contiguous().view(torch.float8_e4m3fn).to(dtype)
    return (v * s.view(*rows.shape[:-1], h, d // 16, 1)).view(*rows.shape[:-1], h, d)


def _prepare_evict(case, g, gc, st):
    S, h, dev = case["seqs"], case["kv_heads"], "cuda"
    n = torch.tensor(_spread(case["tokens_lo"], case["tokens"], S))[torch.randperm(S, generator=gc)]
    st["n"] = n.tolist()
    st["cu"] = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(dev, torch.int32)
    st["seq_ids"] = torch.randperm(S, generator=gc).to(dev, torch.int32)
    st["budget"] = torch.full((S,), case["budget"], dtype=torch.int32, device=dev)
    # a few slots receive most of the weight
    shape = (case["steps"], S, h, case["tokens"])
    st["weights"] = 0.05 * torch.exp(2.0 * torch.randn(*shape, generator=g, device=dev))
    st["stride"] = max(case["budget"], case["prefill"])
    st["kept"] = torch.full((S, st["stride"]), -1, dtype=torch.int32, device=dev)
    st["n_kept"] = torch.zeros(S, dtype=torch.int32, device=dev)
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    gc = torch.Generator().manual_seed(seed)
    dev = torch.device("cuda")
    st = {"case": case}
    if case["op"] == "evict":
        return _prepare_evict(case, g, gc, st)
    S, hq, h, d, bs = case["seqs"], case["heads"], case["kv_heads"], case["dim"], case["block"]
    new = torch.tensor(_spread(case["new_lo"], case["new"], S))[torch.randperm(S, generator=gc)]
    held = torch.tensor(_spread(case["held_lo"], case["held"], S))[torch.randperm(S, generator=gc)]
    n = int(new.sum())
    room = case["held"] + case["new"]
    units, _ = _row_units(case)
    st.update(room=room, units=units, n=n, new=new.tolist(), held=held.tolist())
    st["len"] = held.to(dev, torch.int32)
    st["cu"] = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).to(dev, torch.int32)
    st["seq_list"] = torch.randperm(S, generator=gc).tolist()
    st["seq_ids"] = torch.tensor(st["seq_list"], dtype=torch.int32, device=dev)
    if bs:
        blocks = -(-room // bs)
        st["blocks"] = blocks
        st["block_table"] = torch.randperm(S * blocks, generator=gc).view(S, blocks).to(dev, torch.int32)
        pool_rows = S * blocks * bs
    else:
        pool_rows = S * room
    st["q"] = _normal(g, n, hq, d)
    # keys: a few channels are much larger than the others, the same ones for every token
    channel = 0.7 * torch.exp(0.5 * torch.randn(h, d, generator=g, device=dev))
    k, v = [], []
    for at in range(0, pool_rows, 65536):
        m = min(65536, pool_rows - at)
        kk = (torch.randn(m, h, d, generator=g, device=dev) * channel).to(torch.bfloat16)
        k.append(_pack(kk, units) if case["bits"] == 4 else kk.view(m, units))
        vv = _normal(g, m, h, d)
        v.append(_pack(vv, units) if case["bits"] == 4 else vv.view(m, units))
    # every row is 2-byte units, whatever it holds
    st["k_pool"], st["v_pool"] = (torch.cat(x).view(torch.bfloat16) for x in (k, v))
    if case["op"] == "chunk":
        st["out"] = torch.empty(n, hq, d, dtype=torch.bfloat16, device=dev)
        st["lse"] = torch.empty(n, hq, device=dev)
    else:
        # the attention's log-sums, and a row of weights for each sequence and KV head
        st["lse"] = _attend(st, lse_only=True)
        st["weights"] = torch.zeros(S, h, room, device=dev)
    return st


# ---------------------------------------------------------------- the plain forms

def _pool_rows(st, seq, slots):
    """Rows of the pool that hold the given slots of sequence `seq`."""
    bs = st["case"]["block"]
    if not bs:
        return seq * st["room"] + slots
    return st["block_table"][seq][slots // bs].long() * bs + slots % bs


def _cache(st, pool, seq, n, dtype=torch.float32):
    """Slots 0 .. n - 1 of a sequence as values [h, n, d]."""
    c = st["case"]
    rows = st[pool].view(-1, st["units"])[_pool_rows(st, seq, torch.arange(n, device="cuda"))]
    if c["bits"] == 16:
        x = rows.view(n, c["kv_heads"], c["dim"]).to(dtype)
    else:
        x = _values(rows.view(torch.uint8), c["kv_heads"], c["dim"], dtype)
    return x.transpose(0, 1)


def _scores(st, b, first=0):
    """Scores [h, tokens * rep, slots] of the tokens from `first` on of entry b, in 32 bits; minus infinity where a token
    does not see a slot."""
    c = st["case"]
    h, d = c["kv_heads"], c["dim"]
    rep, n, held = c["heads"] // h, st["new"][b], st["held"][b]
    at = sum(st["new"][:b])
    q = st["q"][at + first:at + n].float().view(n - first, h, rep, d).permute(1, 0, 2, 3).reshape(h, -1, d)
    s = torch.matmul(q, _cache(st, "k_pool", st["seq_list"][b], held + n).transpose(1, 2)) * (1.0 / math.sqrt(d))
    token = torch.arange(first, n, device="cuda").repeat_interleave(rep)
    return s.masked_fill_(torch.arange(held + n, device="cuda") > held + token[:, None], -math.inf)


def _tokens_first(x, h, rep):
    """[h, tokens * rep, ...] as [tokens, h * rep, ...]."""
    return x.view(h, -1, rep, *x.shape[2:]).transpose(0, 1).reshape(-1, h * rep, *x.shape[2:])


def _attend(st, lse_only=False):
    c = st["case"]
    h, rep = c["kv_heads"], c["heads"] // c["kv_heads"]
    outs, lses = [], []
    for b in range(c["seqs"]):
        s = _scores(st, b)
        top = s.amax(-1, keepdim=True)
        p = s.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        lses.append(_tokens_first((top + torch.log(total))[..., 0], h, rep))
        if not lse_only:
            o = torch.matmul(p, _cache(st, "v_pool", st["seq_list"][b], st["held"][b] + st["new"][b])) / total
            outs.append(_tokens_first(o, h, rep))
    lse = torch.cat(lses)
    return lse if lse_only else {"out": torch.cat(outs).to(torch.bfloat16), "lse": lse}


def _plain_weights(st):
    c = st["case"]
    h, rep = c["kv_heads"], c["heads"] // c["kv_heads"]
    at = 0
    for b in range(c["seqs"]):
        n = st["new"][b]
        first = max(0, n - c["last"]) if c["last"] else 0
        s = _scores(st, b, first)
        lse = st["lse"][at + first:at + n].view(n - first, h, rep).transpose(0, 1).reshape(h, -1, 1)
        st["weights"][st["seq_list"][b], :, :s.shape[-1]] = s.sub_(lse).exp_().sum(1)
        at += n
    return st["weights"]


DECAY = 0.75


def _plain_evict(st):
    c = st["case"]
    K = c["budget"]
    for b, seq in enumerate(st["seq_ids"].tolist()):
        n = st["n"][b]
        score = torch.zeros(n, device="cuda")
        for w in st["weights"][:, seq, :, :n]:
            total = w[0]
            for row in w[1:]:
                total = total + row
            score = score * DECAY + total
        if n <= K:
            st["n_kept"][b] = n
            continue
        p = min(c["prefill"], n)
        recent = min(RECENCY, K // 4, max(0, K - p))
        ranked = torch.sort(score[p:n - recent], descending=True, stable=True).indices[:max(0, K - p - recent)] + p
        slot = torch.arange(n, device="cuda")
        keep = (slot < p) | (slot >= n - recent)
        keep[ranked] = True
        kept = slot[keep]
        st["kept"][b, :len(kept)] = kept.int()
        st["n_kept"][b] = len(kept)
    return {"kept": st["kept"], "n_kept": st["n_kept"]}


# ---------------------------------------------------------------- the framework's calls

def _handle(st):
    """The context, the views and the rows' descriptions that a program makes once and keeps."""
    from paper_2606_26472_gb300 import epikv as E
    c = st["case"]
    st["E"] = E
    if c["op"] == "evict":
        cfg = E.make_config(max_seqs=c["seqs"], max_cache_tokens=c["tokens"], max_new_tokens=c["tokens"], num_layers=1,
                            num_kv_heads=c["kv_heads"], head_dim=128, score_kinds=E.EPIKV_SCORE_WEIGHT, recency_cap=RECENCY)
        st["ws"] = torch.empty(E.epikv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        st["ctx"] = E.epikv_init(cfg, st["ws"], st["ws"].numel())
        st["views"] = [E.weights_view(w) for w in st["weights"]]
        return st["ctx"]
    cfg = E.make_attn_config(max_seqs=c["seqs"], max_cache_tokens=st["room"], max_new_tokens=c["new"], num_layers=1,
                             num_heads=c["heads"], num_kv_heads=c["kv_heads"], head_dim=c["dim"],
                             cache_format=E.EPIKV_CACHE_E2M1 if c["bits"] == 4 else E.EPIKV_CACHE_BF16)
    units, bs = st["units"], c["block"]
    if bs:
        st["kv"] = E.kv_view(st["k_pool"], st["v_pool"], layout=E.EPIKV_LAYOUT_PAGED, stride_layer=0, stride_block=bs * units,
                             stride_token=units, block_table=st["block_table"], max_blocks_per_seq=st["blocks"],
                             block_size=bs, num_blocks=c["seqs"] * st["blocks"])
    else:
        st["kv"] = E.kv_view(st["k_pool"], st["v_pool"], layout=E.EPIKV_LAYOUT_CONTIGUOUS, stride_layer=0,
                             stride_seq=st["room"] * units, stride_token=units)
    st["q_rows"] = E.rows(st["q"])
    if c["op"] == "chunk":
        st["out_rows"] = E.rows(st["out"])
    else:
        st["view"] = E.weights_view(st["weights"])
    st["ws"] = torch.empty(E.epikv_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    st["ctx"] = E.epikv_attn_init(cfg, st["ws"], st["ws"].numel())
    return st["ctx"]


def _own(st):
    c = st["case"]
    ctx = st.get("ctx") or _handle(st)
    E = st["E"]
    if c["op"] == "chunk":
        E.epikv_attention_chunk(ctx, 0, c["seqs"], st["seq_ids"], st["cu"], c["new"], st["len"], st["q_rows"], st["out_rows"],
                                st["kv"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if c["op"] == "weights":
        E.epikv_attention_weights(ctx, 0, c["seqs"], st["seq_ids"], st["cu"], c["new"], st["len"], st["q_rows"], st["lse"],
                                  st["view"], st["kv"], last=c["last"])
        return st["weights"]
    for seq in range(c["seqs"]):
        E.epikv_seq_reset(ctx, seq, c["prefill"], E.EPIKV_SCORE_WEIGHT)
    E.epikv_score_update(ctx, c["seqs"], st["seq_ids"], st["cu"], c["tokens"], None, None)
    for view in st["views"]:
        E.epikv_weigh(ctx, c["seqs"], st["seq_ids"], view, DECAY)
    E.epikv_select(ctx, c["seqs"], st["seq_ids"], st["budget"], None, st["kept"], st["stride"], st["n_kept"])
    return {"kept": st["kept"], "n_kept": st["n_kept"]}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _attend(state) if op == "chunk" else _plain_weights(state) if op == "weights" else _plain_evict(state)


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """Attention head by head over each sequence's own slots; whole numbers have no such value."""
    if case["op"] == "evict":
        return None
    st = prepare(case, seed)
    hq, h, d = case["heads"], case["kv_heads"], case["dim"]
    out = torch.empty(st["n"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["n"], hq, dtype=torch.float64, device="cuda")
    weights = torch.zeros(case["seqs"], h, st["room"], dtype=torch.float64, device="cuda")
    at = 0
    for b, seq in enumerate(st["seq_list"]):
        m, held = st["new"][b], st["held"][b]
        k = _cache(st, "k_pool", seq, held + m, torch.float64)
        v = _cache(st, "v_pool", seq, held + m, torch.float64)
        later = torch.ones(m, held + m, device="cuda").triu(held + 1).bool()
        for j in range(hq):
            g = j * h // hq
            s = st["q"][at:at + m, j].double() @ k[g].T * d ** -0.5
            s.masked_fill_(later, -math.inf)
            if case["op"] == "chunk":
                lse[at:at + m, j] = torch.logsumexp(s, 1)
                out[at:at + m, j] = torch.softmax(s, 1) @ v[g]
                continue
            w = torch.exp(s - st["lse"][at:at + m, j, None].double())
            weights[seq, g, :held + m] += w[m - case["last"] if 0 < case["last"] < m else 0:].sum(0)
        at += m
    return {"out": out, "lse": lse} if case["op"] == "chunk" else weights
