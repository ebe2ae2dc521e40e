"""The attention side of a compressed block, as cases to be timed: between the
query/key/value projections and the output projection.

Four operators work on a paged cache whose keys and values are held in 4 bits:
the norm of each query and key head with its rotation (`norm`), appending new
keys and values to the cache with the keys' rotation on the way (`append`),
reading them back as BF16 (`read`), and attention over the cache (`attn`), for
single tokens, a few drafted tokens and prompts.

Where `own` is false, run() computes the plain form in torch (32 bits, rounded
once); where it is true, it calls the library.  Both read the same state: the
pages in the library's layout, the page table and lengths on the device.

A page holds `page` tokens (a multiple of 32) of every key/value head.  Per
head: the key codes, D/2 bytes a token (two codes a byte, even channel low);
the value codes, for each 32 tokens D rows of 16 bytes (two tokens a byte,
even token low); the key scales, one byte for 32 channels of a token; the
value scales, one byte a token; padded to 128 bytes.  Codes are E2M1, a scale
byte b stands for 2^(b - 127), and 255 for NaN.
"""
import math
import random

import torch

own = False

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
MAX_LEN = 32768


def _case(name, op, heads, dim, **more):
    """heads: query heads / key-value heads.  seqs: sequences; ctx: the most
    tokens of one in the cache, new ones included; new: the most new tokens of
    one; ragged: lengths (and new tokens) differ; page: tokens a page; window:
    positions a query sees (0: all); dtype of the inputs of norm and append;
    fused: q, k and v are columns of one buffer; rot: rotated dimensions;
    pairs: rotation of neighbours instead of halves; norm: with weights."""
    c = {"name": name, "op": op, "heads": heads, "dim": dim, "seqs": 1, "ctx": 0, "new": 1,
         "ragged": False, "page": 64, "window": 0, "dtype": "f32", "fused": False, "rot": 0,
         "pairs": False, "norm": False}
    c.update(more)
    return c


def listed():
    return [
        # one generated token's 64 query and 8 key heads, in fp32 as the fused
        # decode-GEMV leaves them: the smallest call, all latency
        _case("norm one token", "norm", "64/8", 128, new=1, rot=128, norm=True),
        # an odd prompt of a model without the norm: rotation alone of q and k
        # as columns of a joint projection's output, half of the channels, in
        # neighbouring pairs
        _case("rotate odd prompt", "norm", "32/32", 128, new=777, dtype="bf16", fused=True, rot=64,
              pairs=True),
        # four prompts of 2048 tokens
        _case("norm prompts", "norm", "64/8", 128, new=8192, dtype="bf16", rot=128, norm=True),
        # a generation step of eight sequences: one token each, and its values
        # read back
        _case("append step", "append", "64/8", 128, seqs=8, ctx=4096, ragged=True, rot=128),
        # prompts of up to 2048 tokens behind cached ones, 32 heads, and their
        # values read back
        _case("append prompts", "append", "32/32", 128, seqs=4, ctx=2500, new=2048, ragged=True,
              dtype="bf16", fused=True, rot=128, page=128),
        # one sequence handed to other code
        _case("read one", "read", "64/8", 128, ctx=1001, new=1001, page=32),
        # the whole cache of eight sequences
        _case("read batch", "read", "64/8", 128, seqs=8, ctx=4096, new=4096),
        # one token over the 512-token context, 32 heads of their own
        _case("decode one", "attn", "32/32", 128, ctx=512),
        # a generation step of eight sequences at 4096 tokens
        _case("decode batch", "attn", "64/8", 128, seqs=8, ctx=4096),
        # long sequences of unlike length, one of them empty
        _case("decode long ragged", "attn", "64/8", 128, seqs=16, ctx=32768, ragged=True, page=128),
        # drafted tokens to be verified, small heads, a sliding window
        _case("verify window", "attn", "16/4", 64, seqs=5, ctx=1500, new=4, ragged=True, page=32,
              window=512),
        # the second half of a 4096-token prompt
        _case("prompt", "attn", "64/8", 128, ctx=4096, new=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "append", "read", "attn", "attn", "attn"])
    heads = rng.choice(["64/8", "32/32", "32/8", "16/4", "16/16", "40/8", "28/4", "8/1"])
    hq, hk = (int(v) for v in heads.split("/"))
    dim = rng.choice([128, 128, 64])
    page = rng.choice([32, 64, 128, 256])
    rot = rng.choice([dim, dim, dim // 2, 0])
    dtype, fused = rng.choice(["f32", "bf16"]), rng.random() < 0.4
    pairs, ragged = rng.random() < 0.3, rng.random() < 0.5
    if op == "norm":
        most = 8192 * 72 * 128 // ((hq + hk) * dim)
        dim = rng.choice([dim, 80, 96, 256])
        rot = rng.choice([dim, dim, dim // 32 * 16, 0])
        return _case_d(op, heads, dim, new=_log(rng, 1, min(8192, most // 2)), dtype=dtype,
                       fused=fused, rot=rot, pairs=pairs, norm=rot == 0 or rng.random() < 0.7)
    if op in ("append", "read"):
        seqs = _log(rng, 1, 64)
        top = min(4096, max(1, 32768 * 8 * 128 // (seqs * hk * dim)))
        new = _log(rng, 1, top)
        return _case_d(op, heads, dim, seqs=seqs, ctx=min(8192, new + _log(rng, 1, 4096)) if
                       op == "append" else new, new=new, ragged=ragged, dtype=dtype, fused=fused,
                       rot=rot if op == "append" else 0, pairs=pairs, page=page)
    kind = rng.choice(["one", "one", "few", "prompt"])
    if kind == "prompt":
        seqs = rng.choice([1, 1, 2, 4])
        new = _log(rng, 9, 2048)
        area = 64 * 2048 * 4096 * 128 // (hq * dim * new * seqs)
        ctx = min(max(new, _log(rng, new, 8192)), max(new, area))
        if area < new:
            seqs, new, ctx = 1, min(new, 1024), min(ctx, 2048)
    else:
        new = 1 if kind == "one" else rng.randint(2, 8)
        seqs = _log(rng, 1, 64)
        top = 16 * 32768 * 8 * 128 // (2 * seqs * hk * dim)
        ctx = max(new, _log(rng, 1, min(MAX_LEN, top)))
    window = 0 if rng.random() < 0.7 else _log(rng, 16, 4096)
    return _case_d("attn", heads, dim, seqs=seqs, ctx=ctx, new=new, ragged=ragged, page=page,
                   window=window)


def _case_d(op, heads, dim, **more):
    c = _case("", op, heads, dim, **more)
    del c["name"]
    return c


def _heads(case):
    return tuple(int(v) for v in case["heads"].split("/"))


def _lengths(case):
    """(cached tokens, new tokens) of each sequence, from the case alone.
    Ragged: the first is the longest, every seventh from the fourth is empty,
    the others anything in between."""
    n, ctx, new = case["seqs"], case["ctx"], case["new"]
    if not case["ragged"]:
        return [ctx] * n, [new] * n
    r = random.Random("%d %d %d" % (n, ctx, new))
    lens, news = [], []
    for i in range(n):
        w = new if i == 0 else 0 if i % 7 == 3 else r.randint(1, new)
        t = ctx if i == 0 else 0 if i % 7 == 3 else r.randint(w, ctx)
        if case["op"] == "read":
            t = w
        lens.append(t)
        news.append(w)
    return lens, news


def _sizes(case):
    """Bytes of a page: key codes, value codes, key scales and value scales of
    a head, their padded sum, and the page."""
    _, hk = _heads(case)
    d, p = case["dim"], case["page"]
    parts = (p * d // 2, p * d // 2, p * d // 32, p)
    head = -(-sum(parts) // 128) * 128
    return parts, head, head * hk


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) % (1 << 62))
    return g


# ------------------------------------------------------------------ plain form
def _codes(x, group):
    """E2M1 codes of x (32 bits, the last axis in groups) and their scale
    bytes: the scale brings the group's largest magnitude to between 3.5 and 7,
    a value goes to the nearest code, ties to the even one."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // group, group)
    top = g.abs().amax(dim=-1)
    b = (((top.view(torch.int32) + 0x200000) >> 23) - 2).clamp(24, 252)
    b = torch.where(torch.isfinite(g).all(dim=-1), b, 255)
    y = (g / ((b << 23).view(torch.float32))[..., None]).abs()
    c = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) +
         (y >= 3.5) + (y > 5.0))
    c = c + 8 * torch.signbit(g)
    return c.to(torch.uint8).reshape(x.shape), b.to(torch.uint8)


def _values(codes, scale, group):
    """The values of codes (uint8 0..15, the last axis in groups) and scale bytes."""
    table = torch.tensor(E2M1 + [-v for v in E2M1], device=codes.device)
    v = table[codes.int()]
    s = (scale.int() << 23).view(torch.float32)
    s = torch.where(scale == 255, torch.nan, s)
    return (v.reshape(*scale.shape, group) * s[..., None]).reshape(v.shape)


def _page_parts(pages, case):
    """Views of pages [P, bytes]: key codes [P, H, page, D/2], value codes
    [P, H, page/32, D, 16], key scale bytes [P, H, page/32, 2, 4, D/32, 4]
    (token t of 32 at [t/16, t%4, :, t%16/4]), value scales [P, H, page]."""
    (kc, vc, ks, vs), head, _ = _sizes(case)
    hk, d, p = _heads(case)[1], case["dim"], case["page"]
    h = pages.view(pages.shape[0], hk, head)
    n = pages.shape[0]
    return (h[..., :kc].unflatten(-1, (p, d // 2)),
            h[..., kc:kc + vc].unflatten(-1, (p // 32, d, 16)),
            h[..., kc + vc:kc + vc + ks].unflatten(-1, (p // 32, 2, 4, d // 32, 4)),
            h[..., kc + vc + ks:kc + vc + ks + vs].view(n, hk, p))


def _pack(k, v, case):
    """Pages of keys and values [P, H, page, D] (32 bits)."""
    n, hk, p, d = k.shape
    pages = torch.zeros(n, _sizes(case)[2], dtype=torch.uint8, device=k.device)
    pk, pv, sk, sv = _page_parts(pages, case)
    c, s = _codes(k, 32)
    pk.copy_(c[..., 0::2] | c[..., 1::2] << 4)
    sk.copy_(s.view(n, hk, p // 32, 2, 4, 4, d // 32).permute(0, 1, 2, 3, 5, 6, 4))
    c, s = _codes(v, d)
    c = c.view(n, hk, p // 32, 32, d).transpose(-1, -2)
    pv.copy_(c[..., 0::2] | c[..., 1::2] << 4)
    sv.copy_(s[..., 0])
    return pages


def _unpack(pages, case):
    """Keys and values [P, H, page, D] of pages, in 32 bits."""
    pk, pv, sk, sv = _page_parts(pages, case)
    n, hk, p, _ = pk.shape
    d = case["dim"]
    c = torch.stack((pk & 15, pk >> 4), dim=-1).view(n, hk, p, d)
    s = sk.permute(0, 1, 2, 3, 6, 4, 5).reshape(n, hk, p, d // 32)
    k = _values(c, s, 32)
    c = torch.stack((pv & 15, pv >> 4), dim=-1).view(n, hk, p // 32, d, 32)
    c = c.transpose(-1, -2).reshape(n, hk, p, d)
    return k, _values(c, sv[..., None], d)


def _rotate(x, cos, sin, rot, pairs):
    """x [T, H, D] (32 bits) with its first `rot` channels rotated by the
    rows cos and sin [T, rot/2]."""
    if not rot:
        return x
    c, s = cos[:, None], sin[:, None]
    if pairs:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    return torch.cat((y, x[..., rot:]), dim=-1)


def _rows(st):
    """For each new token: its sequence and its place there."""
    start = st["seq_start"].long()
    t = torch.arange(st["tokens"], device=start.device)
    seq = torch.searchsorted(start[1:].contiguous(), t, right=True)
    place = st["kv_len"].long()[seq] - start[seq + 1] + t
    return seq, place


def _plain_norm(st):
    case, out = st["case"], []
    c, s = (st[n][st["positions"].long()] for n in ("cos", "sin")) if case["rot"] else (None, None)
    for x, w in ((st["q"], st["qw"]), (st["k"], st["kw"])):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + st["eps"]) * w.float()
        out.append(_rotate(x, c, s, case["rot"], case["pairs"]).to(torch.bfloat16))
    return out


def _plain_append(st):
    case = st["case"]
    d, p = case["dim"], case["page"]
    seq, place = _rows(st)
    k, v = st["k"].float(), st["v"].float()
    if case["rot"]:
        k = _rotate(k, st["cos"][place], st["sin"][place], case["rot"], case["pairs"])
    page, slot = st["table"][seq, place // p].long(), place % p
    pk, pv, sk, sv = _page_parts(st["pages"], case)
    c, s = _codes(k, 32)
    pk[page, :, slot] = c[..., 0::2] | c[..., 1::2] << 4
    sk[page, :, slot // 32, slot % 32 // 16, slot % 4, :, slot % 16 // 4] = s
    c, s = _codes(v, d)
    sv[page, :, slot] = s[..., 0]
    even = slot % 2 == 0
    at = (page[even], slice(None), slot[even] // 32, slice(None), slot[even] % 32 // 2)
    pv[at] = (pv[at] & 240) | c[even]
    at = (page[~even], slice(None), slot[~even] // 32, slice(None), slot[~even] % 32 // 2)
    pv[at] = (pv[at] & 15) | c[~even] << 4


def _plain_read(st):
    case = st["case"]
    d, p = case["dim"], case["page"]
    seq, place = _rows(st)
    page, slot = st["table"][seq, place // p].long(), place % p
    pk, pv, sk, sv = _page_parts(st["pages"], case)
    c = pk[page, :, slot]
    k = _values(torch.stack((c & 15, c >> 4), dim=-1).flatten(-2),
                sk[page, :, slot // 32, slot % 32 // 16, slot % 4, :, slot % 16 // 4], 32)
    c = pv[page, :, slot // 32, :, slot % 32 // 2]
    c = (c >> (4 * (slot % 2)).to(torch.uint8)[:, None, None]) & 15
    v = _values(c, sv[page, :, slot][..., None], d)
    return [k.to(torch.bfloat16), v.to(torch.bfloat16)]


def _plain_attn(st):
    """Scores, a softmax whose statistics are in 32 bits, and the sum of the
    values, over all sequences at once, padded to the longest."""
    case = st["case"]
    hq, hk = _heads(case)
    d, n = case["dim"], case["seqs"]
    used = -(-st["max_len"] // case["page"])
    k, v = _unpack(st["pages"][st["table"][:, :used].reshape(-1).long()], case)
    k = k.view(n, used, hk, -1, d).transpose(1, 2).reshape(n, hk, -1, d)
    v = v.view(n, used, hk, -1, d).transpose(1, 2).reshape(n, hk, -1, d)
    tokens = k.shape[2]
    seq, place = _rows(st)
    row = torch.arange(st["tokens"], device=seq.device) - st["seq_start"].long()[seq]
    q = torch.zeros(n, st["max_new"], hq, d, device=k.device)
    q[seq, row] = st["q"].float()
    q = q.view(n, -1, hk, hq // hk, d).permute(0, 2, 1, 3, 4).reshape(n, hk, -1, d)
    s = torch.matmul(q, k.transpose(-1, -2)) * st["scale"]
    s = s.view(n, hk, st["max_new"], hq // hk, tokens)
    at = torch.full((n, st["max_new"]), -1, device=k.device)
    at[seq, row] = place
    t = torch.arange(tokens, device=k.device)
    seen = t <= at[..., None]
    if case["window"]:
        seen &= t > at[..., None] - case["window"]
    s = torch.where(seen[:, None, :, None], s, -torch.inf)
    m = s.amax(dim=-1, keepdim=True)
    s = torch.exp(s - torch.where(torch.isfinite(m), m, 0.0))
    total = s.sum(dim=-1, keepdim=True)
    # slots behind a sequence's end hold anything
    v = torch.where((t < st["kv_len"][:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(s.view(n, hk, -1, tokens), v).view(n, hk, st["max_new"], hq // hk, d)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(n, st["max_new"], hq, d)
    return o[seq, row].to(torch.bfloat16)


# --------------------------------------------------------------------- inputs
def _new_rows(case, g, tokens):
    """q, k and v [T, heads, D] as the projections leave them."""
    hq, hk = _heads(case)
    d = case["dim"]
    kind = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    x = torch.randn(tokens, hq + 2 * hk, d, device="cuda", generator=g)
    # a few channels of every key head are large, tokens differ in size
    x[:, hq:hq + hk] *= torch.exp(0.6 * torch.randn(1, hk, d, device="cuda", generator=g))
    x *= torch.exp(0.3 * torch.randn(tokens, 1, 1, device="cuda", generator=g))
    x = x.to(kind)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    return (q, k, v) if case["fused"] else (q.contiguous(), k.contiguous(), v.contiguous())


def _tables(case, rows):
    """cos and sin of the positions below `rows`, [rows, rot/2]."""
    f = 500000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda").double() / case["rot"])
    a = torch.arange(rows, device="cuda").double()[:, None] * f
    return a.cos().float(), a.sin().float()


def _cache(case, g, pages):
    """Pages of earlier tokens: keys with large channels, values of unlike size."""
    hk, d, p = _heads(case)[1], case["dim"], case["page"]
    out = torch.empty(pages, _sizes(case)[2], dtype=torch.uint8, device="cuda")
    channel = torch.exp(0.6 * torch.randn(1, hk, 1, d, device="cuda", generator=g))
    step = max(1, (1 << 25) // (hk * p * d))
    for i in range(0, pages, step):
        n = min(step, pages - i)
        k = torch.randn(n, hk, p, d, device="cuda", generator=g) * channel
        v = torch.randn(n, hk, p, d, device="cuda", generator=g)
        v *= torch.exp(0.4 * torch.randn(n, hk, p, 1, device="cuda", generator=g))
        out[i:i + n] = _pack(k, v, case)
    return out


def prepare(case, seed):
    g = _generator(seed)
    hq, hk = _heads(case)
    d, op = case["dim"], case["op"]
    st = {"case": dict(case), "eps": 1e-5, "scale": 1.0 / math.sqrt(d)}
    if op == "norm":
        tokens = case["new"]
        q, k, _ = _new_rows(case, g, tokens)
        st.update(tokens=tokens, q=q, k=k, qw=None, kw=None)
        if case["norm"]:
            w = 1 + 0.2 * torch.randn(2, d, device="cuda", generator=g)
            st["qw"], st["kw"] = w.to(torch.bfloat16)
        if case["rot"]:
            st["cos"], st["sin"] = _tables(case, max(4096, tokens))
        st["positions"] = torch.randint(0, max(4096, tokens), (tokens,), dtype=torch.int32,
                                        device="cuda", generator=g)
        st["out"] = [torch.empty(tokens, h, d, dtype=torch.bfloat16, device="cuda")
                     for h in (hq, hk)]
    else:
        lens, news = _lengths(case)
        starts = [sum(news[:i]) for i in range(len(news) + 1)]
        p = case["page"]
        width = max(1, -(-max(lens) // p))
        used = sum(-(-t // p) for t in lens)
        spare = torch.randperm(used + 1, device="cuda", generator=g).int()
        table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, t in enumerate(lens):
            table[i, :-(-t // p)] = spare[at:at + -(-t // p)]
            at += -(-t // p)
        st.update(table=table, tokens=starts[-1], max_new=max(news), max_len=max(lens),
                  seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                  kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))
        st["pages"] = _cache(case, g, used + 1)
        q, k, v = _new_rows(case, g, starts[-1])
        if op == "attn":
            st["q"] = (1.5 * q).to(torch.bfloat16)
            st["out"] = torch.empty(starts[-1], hq, d, dtype=torch.bfloat16, device="cuda")
        else:
            st["out"] = [torch.empty(starts[-1], hk, d, dtype=torch.bfloat16, device="cuda")
                         for _ in range(2)]
        if op == "append":
            st.update(k=k, v=v)
            if case["rot"]:
                st["cos"], st["sin"] = _tables(case, max(4096, max(lens)))
    if own:  # the handles that a serving program keeps beside its tensors
        import paper_2601_22787_amd as eq
        st["eq"] = eq
        st["rope"] = eq.Rope(st["cos"], st["sin"], pairs=case["pairs"]) if case["rot"] else None
        if op != "norm":
            st["cache"] = eq.KvCache(st["pages"], page_tokens=case["page"], kv_heads=hk, head_dim=d)
            st["batch"] = eq.KvBatch(st["seq_start"], st["kv_len"], st["table"],
                                     n_tokens=st["tokens"], max_new=st["max_new"],
                                     max_len=st["max_len"])
        if op == "attn":
            st["ws"] = eq.attn_workspace(st["cache"], st["batch"], hq)
    return st


def run(st):
    op = st["case"]["op"]
    if not own:
        if op == "norm":
            return _plain_norm(st)
        if op == "attn":
            return _plain_attn(st)
        if op == "append":
            _plain_append(st)
        return _plain_read(st)
    eq, out = st["eq"], st["out"]
    if op == "norm":
        eq.eq_qk_norm_rope(st["q"], st["k"], out[0], out[1], q_weight=st["qw"], k_weight=st["kw"],
                           eps=st["eps"], rope=st["rope"], positions=st["positions"])
    elif op == "attn":
        eq.eq_attn_kv4(st["cache"], st["batch"], st["q"], st["scale"], out, st["ws"],
                       window=st["case"]["window"])
    else:
        if op == "append":
            eq.eq_kv_append(st["cache"], st["batch"], st["k"], st["v"], rope=st["rope"])
        eq.eq_kv_read(st["cache"], st["batch"], out[0], out[1])
    return out


def _seen(case):
    """Query-key pairs, and cached tokens that any query sees, summed over the
    sequences."""
    pairs = cached = 0
    for t, w in zip(*_lengths(case)):
        win = case["window"] or t
        pairs += sum(min(win, i) for i in range(t - w + 1, t + 1))
        cached += min(t, win + w - 1) if w else 0
    return pairs, cached


def work(case):
    """Bytes: inputs, tables' rows and outputs once, cached tokens at 4 bits a
    value and their scales.  FLOPs: attention's two products."""
    hq, hk = _heads(case)
    d, op = case["dim"], case["op"]
    item = 4 if case["dtype"] == "f32" else 2
    packed = hk * (d + d // 32 + 1)  # a token's codes and scales
    if op == "norm":
        n = case["new"]
        return {"bytes": n * (hq + hk) * d * (item + 2) + n * (4 * case["rot"] + 4), "flops": 0}
    tokens = sum(_lengths(case)[1])
    if op == "attn":
        pairs, cached = _seen(case)
        return {"bytes": cached * packed + tokens * hq * d * 4, "flops": 4 * pairs * hq * d}
    bytes_ = tokens * (packed + 2 * hk * d * 2)
    if op == "append":
        bytes_ += tokens * (packed + 2 * hk * d * item + 4 * case["rot"])
    return {"bytes": bytes_, "flops": 0}


# ------------------------------------------------------------- 64-bit results
def _stored64(x, group):
    """What the cache keeps of x (64 bits, the last axis in groups)."""
    shape = x.shape
    g = x.reshape(-1, group)
    top = g.abs().amax(dim=1, keepdim=True)
    mant, expo = torch.frexp(top)  # top = mant 2^expo, mant in [1/2, 1)
    e = (expo - 3 + (mant >= 0.875)).clamp(24 - 127, 252 - 127)
    y = torch.ldexp(g, -e)
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y)[1].clamp(1, 3) - 2)
    y = (torch.round(y / step) * step).clamp(-6, 6)
    return torch.ldexp(y, e).reshape(shape)


def _turn64(x, at, case):
    """x [H, T, D] (64 bits) rotated at the positions `at`, from the 32-bit
    table that the call reads."""
    r = case["rot"]
    if not r:
        return x
    cos, sin = _tables(case, int(at.max()) + 1)
    z = torch.complex(cos[at].double(), sin[at].double())
    y = x.clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if case["pairs"] else (slice(0, r // 2), slice(r // 2, r))
    w = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * z
    y[..., a], y[..., b] = w.real, w.imag
    return y


def _head64(st, page, h):
    """Keys and values [T, D] in 64 bits of head h in a list of pages."""
    case = st["case"]
    d, p = case["dim"], case["page"]
    (a, b, c, _), head, _ = _sizes(case)
    raw = st["pages"][page][:, h * head:(h + 1) * head].long()

    def value(code, byte):
        m, e = code & 1, (code >> 1) & 3
        mag = torch.where(e == 0, m * 0.5, (1 + m * 0.5) * torch.pow(2.0, (e - 1).double()))
        return torch.where(code >= 8, -mag, mag) * torch.pow(2.0, (byte - 127).double())

    t = torch.arange(p, device="cuda")
    ch = torch.arange(d, device="cuda")
    key = raw[:, (t[:, None] * (d // 2) + ch // 2)] >> 4 * (ch % 2) & 15
    val = raw[:, a + (t[:, None] // 32 * d + ch) * 16 + t[:, None] % 32 // 2]
    val = val >> 4 * (t[:, None] % 2) & 15
    ks = raw[:, a + b + t[:, None] // 16 * (d // 2) + (t[:, None] % 4 * (d // 32) + ch // 32) * 4 +
             t[:, None] % 16 // 4]
    vs = raw[:, a + b + c + t]
    return value(key, ks).view(-1, d), value(val, vs[..., None]).view(-1, d)


def exact(case, seed):
    st = prepare(case, seed)
    hq, hk = _heads(case)
    d, op = case["dim"], case["op"]
    if op == "norm":
        at, out = st["positions"].long(), []
        for x, w in ((st["q"], st["qw"]), (st["k"], st["kw"])):
            y = x.double().transpose(0, 1)
            if w is not None:
                size = torch.sqrt((y ** 2).sum(dim=-1, keepdim=True) / d + st["eps"])
                y = y / size * w.double()
            out.append(_turn64(y, at, case).transpose(0, 1).contiguous())
        return out
    lens, news = _lengths(case)
    if op == "append":
        k, v = st["k"].double().transpose(0, 1), st["v"].double().transpose(0, 1)
        at = torch.cat([torch.arange(t - w, t, device="cuda") for t, w in zip(lens, news)])
        return [_stored64(_turn64(k, at, case), 32).transpose(0, 1).contiguous(),
                _stored64(v, d).transpose(0, 1).contiguous()]
    if op == "read":
        out = torch.empty(2, st["tokens"], hk, d, dtype=torch.float64, device="cuda")
    else:
        out = torch.zeros(st["tokens"], hq, d, dtype=torch.float64, device="cuda")
    row, group = 0, hq // hk
    for i, (t, w) in enumerate(zip(lens, news)):
        if not w:
            continue
        page = st["table"][i, :-(-t // case["page"])].long()
        for h in range(hk):
            k, v = (x[:t] for x in _head64(st, page, h))
            if op == "read":
                out[0, row:row + w, h], out[1, row:row + w, h] = k[t - w:], v[t - w:]
                continue
            last = torch.arange(t - w, t, device="cuda")[:, None]
            j = torch.arange(t, device="cuda")
            hidden = (j > last) | (j <= last - (case["window"] or t))
            for c in range(h * group, (h + 1) * group):
                s = st["q"][row:row + w, c].double() @ k.t() * st["scale"]
                s = torch.softmax(s.masked_fill_(hidden, -torch.inf), dim=1)
                out[row:row + w, c] = s @ v
        row += w
    return [out[0], out[1]] if op == "read" else out
