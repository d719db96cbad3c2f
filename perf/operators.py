"""Attention over a 4-bit cache of keys and values, as cases to time: what lies between the maps that make q, k
and v of a decode step and the map that takes the attention's output.

Four kinds of case:

  plan    block tables and slot maps from the requests' lengths, on the GPU (``KVCache.plan``)
  append  keys and values of new tokens into the cache, and back as later steps see them
          (``KVCache.append``, ``KVCache.read``)
  attend  attention of new tokens over the cache (``KVCache.attend``): one token per sequence, a few (a
          draft that is checked), or a chunk of a prompt
  step    the three in turn, as one layer of a decode step makes them

The cache, for every token and head and 64 channels at a time (the last ones of a head may be fewer):

  s = f16((max - min) / 15)   mid = f16(min + 8 s)   code = clamp(rint((x - mid) / s) + 8, 0, 15), 8 where s = 0
  value = s (code - 8) + mid

with single fp32 operations.  A page holds, per head, tiles of 16 tokens: K then V, of either per 64 channels 512 bytes
of codes and 64 of (s, mid) pairs.  Token t, channel c of K: lane 4 (t % 8) + c / 16, its bytes 8 (t / 8) + c % 16 / 2;
of V: lane 4 (c / 8) + t % 8 / 2, its bytes 8 (t / 8) + 4 (c % 8 / 4) + 2 (t % 2) + c % 4 / 2; 16 bytes a lane, the
even channel in the lower half of its byte.  The pair of token t is the (2 (t % 8) + t / 8)-th.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    def plan(name, seqs, old, new, page):
        return dict(name=name, kind="plan", seqs=seqs, old=old, new=new, page=page)

    def append(name, tokens, heads, dim, page, dtype, strided):
        return dict(name=name, kind="append", tokens=tokens, heads=heads, dim=dim, page=page, dtype=dtype, strided=strided)

    def attend(name, seqs, heads, shared, dim, length, new, page, dtype, ragged, kind="attend"):
        return dict(name=name, kind=kind, seqs=seqs, heads=heads, shared=shared, dim=dim, length=length, new=new,
                    page=page, dtype=dtype, ragged=ragged)

    return [
        # one request goes on by a token
        plan("plan one token", 1, 700, 1, 64),
        # a server's start: prompts of 512 requests
        plan("plan prompts", 512, 0, 8000, 32),
        # GPT-2's heads, batch 1
        append("append one token", 1, 12, 64, 16, "float32", True),
        # GPT-J's heads, the largest call of the gated layer, k and v as columns of its y
        append("append 64 tokens", 64, 16, 256, 64, "float32", True),
        # prompts at OPT's heads
        append("append a prompt", 16001, 32, 128, 64, "bfloat16", False),
        # the first tokens of one request
        attend("attend first tokens", 1, 12, 1, 64, 33, 1, 16, "float32", False),
        # one request with a long cache: the tokens have to be split over the GPU
        attend("attend one long", 1, 16, 1, 256, 32771, 1, 64, "float32", False),
        # a full batch, requests of all lengths
        attend("attend batch", 64, 32, 1, 128, 4096, 1, 64, "float32", True),
        # shared heads (four q heads per kv head), many requests, small pages
        attend("attend shared heads", 128, 8, 4, 128, 8192, 1, 16, "bfloat16", True),
        # drafts of five tokens, heads of a width that is no multiple of 64
        attend("attend drafts", 16, 32, 1, 80, 2000, 5, 32, "float16", True),
        # chunks of prompts
        attend("attend chunks", 4, 12, 1, 64, 1500, 256, 64, "float32", True),
        # one layer of a decode step at OPT's heads
        attend("step 64 tokens", 64, 32, 1, 128, 2048, 1, 64, "float32", True, kind="step"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "step"])
    page = rng.choice([16, 32, 48, 64, 128])
    if kind == "plan":
        return dict(kind=kind, seqs=log(1, 512), old=log(1, 8000) - 1, new=log(1, 8000), page=page)
    dim, dtype = rng.choice([40, 64, 80, 96, 128, 128, 192, 256]), rng.choice(list(DTYPES))
    if kind == "append":
        heads = rng.choice([1, 4, 8, 12, 16, 32])
        tokens = min(log(1, 16001), 16001 * 32 * 128 // (heads * dim) // 2 if dtype == "float32" else 16001 * 16 * 128 // (heads * dim))
        return dict(kind=kind, tokens=max(1, tokens), heads=heads, dim=dim, page=page, dtype=dtype, strided=rng.random() < 0.5)
    heads, shared = rng.choice([1, 2, 4, 8, 12, 16, 32]), rng.choice([1, 1, 1, 2, 4, 5, 8])
    shared = min(shared, 64 // heads)
    seqs, length = log(1, 128), log(1, 32771)
    new = 1 if kind == "step" else rng.choice([1, 1, 1, 1, rng.randint(2, 8), log(9, 256)])
    while seqs * length * heads * dim > 64 * 4096 * 32 * 128:
        seqs, length = (max(1, seqs // 2), length) if seqs > 1 and rng.random() < 0.5 else (seqs, max(1, length // 2))
    while seqs * min(new, length) * heads * shared * length * dim > 4 * 256 * 12 * 1500 * 64 and new > 1:
        new //= 2
    return dict(kind=kind, seqs=seqs, heads=heads, shared=shared, dim=dim, length=length, new=min(new, length), page=page, dtype=dtype,
                ragged=rng.random() < 0.7)


def spread(n, largest, ragged, least=0):
    """n lengths of up to `largest`, all of it or in between."""
    if not ragged or n == 1:
        return [largest] * n
    return [least + int((largest - least) * math.modf((i + 1) * 0.6180339887498949)[0]) + (largest > least) for i in range(n)]


def requests(case):
    """(tokens in the cache before the step, new tokens) of each request; of an attention that is ragged every 13th has none."""
    if case["kind"] == "plan":
        return spread(case["seqs"], case["old"], True), spread(case["seqs"], case["new"], True, 1)
    if case["kind"] == "step":
        return [n - 1 for n in spread(case["seqs"], case["length"], case["ragged"], 1)], [1] * case["seqs"]
    news = [0 if case["ragged"] and i % 13 == 12 else case["new"] for i in range(case["seqs"])]
    lens = spread(case["seqs"], case["length"], case["ragged"], case["new"])
    return [n - m if m else 0 for n, m in zip(lens, news)], news


def work(case):
    kind = case["kind"]
    if kind == "plan":
        old, new = requests(case)
        took = sum(-(-(a + b) // case["page"]) - -(-a // case["page"]) for a, b in zip(old, new))
        return {"bytes": 8 * sum(new) + 8 * took + 20 * case["seqs"], "flops": 0}
    size = 4 if case["dtype"] == "float32" else 2
    row = case["heads"] * (case["dim"] + -(-case["dim"] // 64) * 8)   # of the cache: a token's k and v
    if kind == "append":
        n = case["tokens"]
        # rows in, their codes out, codes in and the values out
        return {"bytes": n * (2 * case["heads"] * case["dim"] * (size + 4) + 2 * row), "flops": n * 2 * case["heads"] * case["dim"] * 6}
    old, new = requests(case)
    seen = sum(a + b for a, b in zip(old, new) if b)
    pairs = sum(b * a + b * (b + 1) // 2 for a, b in zip(old, new))
    q = case["heads"] * case["shared"]
    got = {"bytes": seen * row + sum(new) * 2 * q * case["dim"] * size, "flops": pairs * q * case["dim"] * 4}
    if kind == "step":
        got["bytes"] += sum(new) * (2 * case["heads"] * case["dim"] * size + 8) + 20 * case["seqs"]
    return got


# ---- the cache's form ----------------------------------------------------------------------------------------------

def quantise(x):
    """x [..., D] -> codes [..., D] and (s, mid) [..., groups, 2]."""
    D = x.shape[-1]
    G = -(-D // 64)
    x = x.float()
    # (the last group's missing channels repeat its first one, which changes neither bound)
    xg = torch.cat([x, x[..., (G - 1) * 64:(G - 1) * 64 + 1].expand(*x.shape[:-1], G * 64 - D)], -1).unflatten(-1, (G, 64))
    lo, hi = xg.amin(-1), xg.amax(-1)
    s = ((hi - lo) / 15).clamp(max=65504.0).half()
    mid = (lo + 8 * s.float()).clamp(-65504.0, 65504.0).half()
    bad = ~torch.isfinite(xg).all(-1)
    s, mid = s.masked_fill(bad, math.nan), mid.masked_fill(bad, math.nan)
    at = torch.round((xg - mid.float()[..., None]) / s.float()[..., None]) + 8
    codes = torch.where((s == 0)[..., None], 8.0, at.clamp(0, 15)).nan_to_num(0).to(torch.uint8)
    return codes.flatten(-2)[..., :D], torch.stack([s, mid], -1)


def padded(codes):
    return torch.nn.functional.pad(codes, (0, -codes.shape[-1] % 64))


def k_bytes(codes):
    """[..., D] -> bytes [..., groups, 4 lanes, 8]"""
    c = padded(codes).unflatten(-1, (-1, 4, 8, 2))
    return c[..., 0] | c[..., 1] << 4


def v_bytes(codes):
    """[..., D] -> bytes [..., groups, 8 octets, 2, 2]"""
    c = padded(codes).unflatten(-1, (-1, 8, 2, 2, 2))
    return c[..., 0] | c[..., 1] << 4


def places(pool):
    """pool [pages, heads, tiles, 2, groups, 576] -> codes of K [.., 8 tokens, 4, 2 halves, 8] and of V
    [.., 8 octets, 4 pairs, 2 halves, 2, 2 of a pair, 2], (s, mid) of either [.., 8 tokens, 2 halves, 2]."""
    codes, pairs = pool[..., :512], pool[..., 512:].view(torch.float16).unflatten(-1, (8, 2, 2))
    return (codes[:, :, :, 0].unflatten(-1, (8, 4, 2, 8)), codes[:, :, :, 1].unflatten(-1, (8, 4, 2, 2, 2, 2)),
            pairs[:, :, :, 0], pairs[:, :, :, 1])


def write(pool, page, inside, k, v):
    """k, v [n, heads, D] at token `inside` of pages `page`."""
    kc, kp = quantise(k)
    vc, vp = quantise(v)
    K, V, Ks, Vs = places(pool)
    tile, t = inside // 16, inside % 16
    K[page, :, tile, :, t % 8, :, t // 8] = k_bytes(kc)
    V[page, :, tile, :, :, t % 8 // 2, t // 8, :, t % 2] = v_bytes(vc)
    Ks[page, :, tile, :, t % 8, t // 8] = kp
    Vs[page, :, tile, :, t % 8, t // 8] = vp


def numbers(bytes_, pairs, D):
    """bytes [..., groups, 32] and (s, mid) [..., groups, 2] -> values [..., D]."""
    codes = torch.stack([bytes_ & 15, bytes_ >> 4], -1).flatten(-2).float() - 8
    return (codes * pairs[..., :1].float() + pairs[..., 1:].float()).flatten(-2)[..., :D]


def whole_pages(pool, D):
    """pool [pages, heads, tiles, 2, groups, 576] -> k, v [pages, heads, tokens, D]"""
    K, V, Ks, Vs = places(pool)
    k = K.permute(0, 1, 2, 6, 4, 3, 5, 7).flatten(-2).flatten(2, 4)                # pages heads (tiles halves 8) groups 32
    v = V.permute(0, 1, 2, 6, 5, 8, 3, 4, 7, 9).flatten(-3).flatten(2, 5)
    ks = Ks.permute(0, 1, 2, 5, 4, 3, 6).flatten(2, 4)
    vs = Vs.permute(0, 1, 2, 5, 4, 3, 6).flatten(2, 4)
    return numbers(k, ks, D), numbers(v, vs, D)


# ---- inputs --------------------------------------------------------------------------------------------------------

def generator(case, seed, device="cuda"):
    g = torch.Generator(device)
    g.manual_seed(seed * 1000003 + sum(ord(c) * (i + 1) for i, c in enumerate(repr(sorted(case.items())))) % 999983)
    return g


def heads_scale(heads, dim, g):
    """Channels of a head differ in size; a few stand out, as a model's keys have it."""
    size = 0.5 + torch.rand(heads, dim, device="cuda", generator=g)
    return torch.where(torch.rand(heads, dim, device="cuda", generator=g) < 0.03, 4 * size, size)


def prepare(case, seed):
    g = generator(case, seed)
    kind, page = case["kind"], case["page"]
    s = {"case": case}

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    if kind == "append":
        n, heads, dim = case["tokens"], case["heads"], case["dim"]
        n_pages = -(-n // page) * 5 // 4 + 2
        seqs, most, tokens = 1, n, n
    else:
        old, new = requests(case)
        seqs, tokens = len(old), sum(new)
        heads, dim = case.get("heads", 1), case.get("dim", 64)
        most = max(a + b for a, b in zip(old, new))
        # attend's requests have their new tokens in the cache, plan's and step's get pages for them
        held = [a + b for a, b in zip(old, new)] if kind == "attend" else old
        used = [-(-a // page) for a in held]
        n_pages = sum(-(-(a + b) // page) for a, b in zip(old, new)) + 7
    order = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    G, tiles, max_pages = -(-dim // 64), page // 16, -(-most // page)
    s.update(n_pages=n_pages, seqs=seqs, most=most, tokens=tokens, heads=heads, dim=dim)
    s["pool"] = torch.empty(n_pages, heads, tiles, 2, G, 576, dtype=torch.uint8, device="cuda") if kind != "plan" else \
        torch.zeros(n_pages, heads, tiles, 2, G, 576, dtype=torch.uint8, device="cuda")

    if kind == "append":
        # tokens of two requests' pages in turn, one of them not at a page's start; every 50th is a row of padding
        at = (torch.arange(n, device="cuda") + 5) % (-(-n // page) * page)
        s["slots"] = (order[at // page] * page + at % page).to(torch.int32)
        s["slots"][49::50] = -1
        s["pool"].zero_()
    else:
        table = torch.full((seqs, max_pages), -1, dtype=torch.int32)
        listed_order, at = order.cpu(), 0
        for i, n in enumerate(used):
            table[i, :n] = listed_order[at:at + n]
            at += n
        s["table"] = table.cuda()
        s["free"] = torch.cat([order[at:], order.new_full((at,), -1)])
        s["n_free"] = ints([n_pages - at])
        s["lens"], s["n_new"] = ints(held), ints(new)
        s["q_start"] = ints([0] + list(np.cumsum(new)))

    if kind != "plan":
        ks, vs = heads_scale(heads, dim, g), heads_scale(heads, dim, g).clamp(max=1.5)
        dtype = DTYPES[case["dtype"]]
        if kind != "append":
            some = max(1, (1 << 26) // (heads * page * dim))
            K, V, Ks, Vs = places(s["pool"])
            for p in range(0, n_pages, some):
                m = min(some, n_pages - p)
                for codes_at, pairs_at, size, of_v in ((K, Ks, ks, False), (V, Vs, vs, True)):
                    x = torch.randn(m, heads, tiles, 2, 8, dim, device="cuda", generator=g) * size[:, None, None, None]
                    c, pairs = quantise(x)
                    if of_v:   # [m heads tiles halves 8 groups 8 2 2] -> [m heads tiles groups 8 4 halves 2 2 2]
                        b = v_bytes(c).unflatten(4, (4, 2))
                        codes_at[p:p + m] = b.permute(0, 1, 2, 6, 7, 4, 3, 8, 5, 9)
                    else:      # [m heads tiles halves 8 groups 4 8] -> [m heads tiles groups 8 4 halves 8]
                        codes_at[p:p + m] = k_bytes(c).permute(0, 1, 2, 5, 4, 6, 3, 7)
                    pairs_at[p:p + m] = pairs.permute(0, 1, 2, 5, 4, 3, 6)
        # q, k and v of the new tokens, as columns of one buffer as the map before leaves them, or each for itself
        rows, q_heads = tokens + (3 if kind == "attend" and case["ragged"] else 0), heads * case.get("shared", 1)
        if case.get("strided", case["dtype"] == "float32"):
            y = torch.randn(rows, (q_heads + 2 * heads) * dim, device="cuda", generator=g)
            y = y.to(dtype).split([q_heads * dim, heads * dim, heads * dim], -1)
            q, k, v = (part.unflatten(-1, (-1, dim)) for part in y)
        else:
            q, k, v = (torch.randn(rows, h, dim, device="cuda", generator=g).to(dtype) for h in (q_heads, heads, heads))
        k.mul_(ks), v.mul_(vs)
        s.update(q=q.mul_(1.5), k=k, v=v)
        s["out"] = torch.full((rows, q_heads, dim), 0.03125, dtype=dtype, device="cuda")
    if own:
        s["cache"] = c = handle(case, s)
        if kind != "append":
            c.table.copy_(s["table"]), c.lens.copy_(s["lens"])
            c.free.copy_(s["free"]), c.n_free.copy_(s["n_free"])
            c.q_start.copy_(s["q_start"]), c.kv_len.copy_(s["lens"])
    return s


def handle(case, s):
    import paper_2605_03109_b200 as gsi
    return gsi.KVCache(s["heads"], s["dim"], s["n_pages"], max_seqs=s["seqs"], max_len=s["most"], page_tokens=case["page"],
                       max_tokens=s["tokens"], pages=s["pool"])


# ---- one pass ------------------------------------------------------------------------------------------------------

def plain_plan(s):
    page, seqs = s["case"]["page"], s["seqs"]
    old, new, n_free = s["lens"].long(), s["n_new"].long(), s["n_free"].long()
    held, after = -(-old // page), -(-(old + new) // page)
    need = after - held
    upto = need.cumsum(0)
    q_end = new.cumsum(0)
    ok = (need == 0) | (upto <= n_free)
    table = s["table"].clone()
    j = torch.arange(table.shape[1], device="cuda")
    of = (upto - need)[:, None] + j - held[:, None]           # which page of the step it is
    mine = ok[:, None] & (j >= held[:, None]) & (j < after[:, None])
    table = torch.where(mine, s["free"][(n_free - 1 - of).clamp(0, len(s["free"]) - 1)], table)
    i = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(q_end, i, right=True).clamp(max=seqs - 1)
    pos = old[seq] + i - (q_end - new)[seq]
    fine = (i < q_end[-1]) & ok[seq]
    slots = torch.where(fine, table[seq, (pos // page).clamp(max=table.shape[1] - 1)] * page + pos % page, -1)
    took = torch.where(ok, need, 0).sum()
    return {"table": table, "q_start": torch.cat([q_end.new_zeros(1), q_end]).int(), "kv_len": torch.where(ok, old + new, 0).int(),
            "slots": slots.int(), "positions": torch.where(fine, pos, -1).int(),
            "counts": torch.stack([q_end[-1], took, n_free[0] - took, (~ok).sum()]).int()}


def plain_attend(s, table, q_start, kv_len, rows_of=None):
    case, q = s["case"], s["q"]
    page, dim, shared = case["page"], s["dim"], case["shared"]
    k, v = whole_pages(s["pool"][table.clamp(min=0).flatten().long()], dim)
    k, v = (x.unflatten(0, table.shape).transpose(1, 2).flatten(2, 3) for x in (k, v))     # seqs heads tokens dim
    starts, most = q_start[:-1].long(), case["new"]
    news = q_start[1:].long() - starts
    i = torch.arange(most, device="cuda")
    live = i < news[:, None]
    row = (starts[:, None] + i).clamp(max=len(q) - 1)
    x = q[row].float().unflatten(2, (-1, shared))                                          # seqs new heads shared dim
    x = x.permute(0, 2, 3, 1, 4).flatten(2, 3) / math.sqrt(dim)
    scores = x @ k.transpose(2, 3)                                                         # seqs heads (shared new) tokens
    sees = torch.arange(k.shape[2], device="cuda") <= (kv_len.long() - news)[:, None, None] + i[:, None]
    sees = sees.repeat(1, shared, 1)[:, None]
    top = scores.masked_fill(~sees, -math.inf).amax(-1, keepdim=True)
    p = torch.where(sees, torch.exp(scores - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = p.sum(-1, keepdim=True)
    o = (p @ torch.where((torch.arange(k.shape[2], device="cuda") < kv_len[:, None])[:, None, :, None], v, 0.0)) / torch.where(total > 0, total, 1.0)
    o = o.unflatten(2, (shared, most)).permute(0, 3, 1, 2, 4).flatten(2, 3)                 # seqs new q_heads dim
    out = s["out"].clone()
    out[row[live]] = o[live].to(out.dtype)
    return out


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        c = s["cache"]
        if kind == "plan":
            c.plan(s["n_new"], commit=False)
            return {"table": c.table, "q_start": c.q_start, "kv_len": c.kv_len, "slots": c.slots, "positions": c.positions,
                    "counts": c.counts}
        if kind == "append":
            c.append(s["k"], s["v"], slots=s["slots"])
            k, v = c.read(s["slots"])
            return {"k": k, "v": v}
        if kind == "attend":
            return {"out": c.attend(s["q"], out=s["out"])}
        c.plan(s["n_new"], commit=False)
        c.append(s["k"], s["v"])
        return {"out": c.attend(s["q"], out=s["out"]), "slots": c.slots, "kv_len": c.kv_len}
    if kind == "plan":
        return plain_plan(s)
    if kind == "attend":
        return {"out": plain_attend(s, s["table"], s["q_start"], s["lens"])}
    page, pool = case["page"], s["pool"]
    if kind == "append":
        live = s["slots"] >= 0
        at = s["slots"][live].long()
        write(pool, at // page, at % page, s["k"][live], s["v"][live])
        K, V, Ks, Vs = places(pool)
        tile, t = at % page // 16, at % 16
        got = []
        for b, pairs in ((K[at // page, :, tile, :, t % 8, :, t // 8].flatten(-2), Ks),
                         (V[at // page, :, tile, :, :, t % 8 // 2, t // 8, :, t % 2].flatten(-3), Vs)):
            values = torch.zeros(len(live), s["heads"], s["dim"], device="cuda")
            values[live] = numbers(b, pairs[at // page, :, tile, :, t % 8, t // 8], s["dim"])
            got.append(values)
        return {"k": got[0], "v": got[1]}
    p = plain_plan(s)
    at = p["slots"].long()
    write(pool, at // page, at % page, s["k"], s["v"])
    return {"out": plain_attend(s, p["table"], p["q_start"], p["kv_len"]), "slots": p["slots"], "kv_len": p["kv_len"]}


# ---- from the definition, in 64 bits -------------------------------------------------------------------------------

def rounded(x):
    """x [n, heads, dim] as the cache holds it: the roundings of the definition, then 64 bits."""
    got = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[-1], 64):
        part = x[..., c:c + 64].float()
        lo, hi = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
        s = ((hi - lo) / 15).half().float()
        mid = (lo + s * 8).half().float()
        steps = torch.round((part - mid) / torch.where(s == 0, 1.0, s)).clamp(-8, 7)
        got[..., c:c + 64] = mid.double() + torch.where(s == 0, 0.0, steps).double() * s.double()
    return got


def cached(s, pages, n):
    """k, v [n, heads, dim] of a request's first n tokens, byte by byte."""
    page, dim, pool = s["case"]["page"], s["dim"], s["pool"]
    p = torch.arange(n, device="cuda")
    where = pages.long()[p // page][:, None]
    tile, t = (p % page // 16)[:, None], (p % 16)[:, None]
    c = torch.arange(dim, device="cuda")[None]
    group, c = c // 64, c % 64
    pair = 512 + 4 * (2 * (t % 8) + t // 8)
    got = []
    for kv, byte in ((0, 16 * (4 * (t % 8) + c // 16) + 8 * (t // 8) + c % 16 // 2),
                     (1, 16 * (4 * (c // 8) + t % 8 // 2) + 8 * (t // 8) + 4 * (c % 8 // 4) + 2 * (t % 2) + c % 4 // 2)):
        def at(i):
            return pool[where, :, tile, kv, group, i.expand(n, dim)].permute(0, 2, 1).int()     # tokens heads dim
        code = at(byte) >> 4 * (c % 2) & 15
        step, mid = ((at(pair + i) | at(pair + i + 1) << 8).to(torch.int16).view(torch.float16).double() for i in (0, 2))
        got.append(step * (code - 8).double() + mid)
    return got


def exact(case, seed):
    s = prepare(case, seed)
    kind, page = case["kind"], case["page"]
    if kind == "append":
        live = (s["slots"] >= 0)[:, None, None]
        return {"k": torch.where(live, rounded(s["k"]), 0.0), "v": torch.where(live, rounded(s["v"]), 0.0)}
    table, lens, news = s["table"].cpu().numpy().copy(), s["lens"].cpu().numpy(), s["n_new"].cpu().numpy()
    slots, positions = np.full(s["tokens"], -1, np.int32), np.full(s["tokens"], -1, np.int32)
    free, left, took, refused = s["free"].cpu().numpy(), int(s["n_free"]), 0, 0
    kv_len, starts, asked, row = lens.copy(), [0], 0, 0
    if kind != "attend":
        for i in range(s["seqs"]):
            have, want = -(-int(lens[i]) // page), -(-int(lens[i] + news[i]) // page)
            asked += want - have
            fine = want == have or asked <= left
            if fine:
                for j in range(have, want):
                    table[i, j] = free[left - 1 - took]
                    took += 1
                pos = np.arange(lens[i], lens[i] + news[i])
                slots[row:row + news[i]] = table[i, pos // page] * page + pos % page
                positions[row:row + news[i]] = pos
                kv_len[i] = lens[i] + news[i]
            else:
                refused += 1
                kv_len[i] = 0
            row += int(news[i])
            starts.append(row)
    if kind == "plan":
        return {"table": table, "q_start": np.array(starts, np.int32), "kv_len": kv_len, "slots": slots, "positions": positions,
                "counts": np.array([row, took, left - took, refused], np.int32)}
    out = s["out"].double()
    new_k, new_v = (rounded(s["k"]), rounded(s["v"])) if kind == "step" else (None, None)
    at, shared = 0, case["shared"]
    for i in range(s["seqs"]):
        n, m = int(kv_len[i]), int(news[i])
        if m == 0:
            continue
        old = n - m if kind == "step" else n
        k, v = cached(s, torch.from_numpy(table[i]).cuda(), old) if old else (s["q"].new_zeros(0, s["heads"], s["dim"], dtype=torch.float64),) * 2
        if kind == "step":
            k, v = torch.cat([k, new_k[at:at + m]]), torch.cat([v, new_v[at:at + m]])
        for h in range(s["heads"]):
            q = s["q"][at:at + m, h * shared:(h + 1) * shared].double()                        # m shared dim
            w = torch.einsum("msd,nd->msn", q, k[:, h]) * s["dim"] ** -0.5
            behind = torch.arange(n, device="cuda")[None] > (n - m + torch.arange(m, device="cuda"))[:, None]
            w = torch.softmax(w.masked_fill(behind[:, None], -math.inf), -1)
            out[at:at + m, h * shared:(h + 1) * shared] = torch.einsum("msn,nd->msd", w, v[:, h])
        at += m
    if kind == "step":
        return {"out": out, "slots": slots, "kv_len": kv_len}
    return {"out": out}
