"""A cache of keys and values in 4 bits, restated in numpy: the numbers of one row, the places of a page, a plan, and
attention in 64 bits with a bound on what a kernel may be off by."""
import numpy as np

F = np.float32


def quantise(x):
    """x [..., D] -> codes [..., D], s and mid [..., groups] (float16): single fp32 operations, as the header has them."""
    x = np.asarray(x, F)
    D = x.shape[-1]
    G = -(-D // 64)
    codes = np.zeros(x.shape, np.uint8)
    s, mid = (np.zeros(x.shape[:-1] + (G,), np.float16) for _ in range(2))
    with np.errstate(all="ignore"):
        for g in range(G):
            part = x[..., 64 * g:64 * g + 64]
            lo, hi = part.min(-1), part.max(-1)
            step = np.minimum((hi - lo) * F(1 / 15), F(65504)).astype(np.float16)
            centre = np.clip(lo + F(8) * step.astype(F), F(-65504), F(65504)).astype(np.float16)
            at = np.rint((part - centre.astype(F)[..., None]) / step.astype(F)[..., None]) + F(8)
            c = np.where(step[..., None] == 0, F(8), np.clip(at, 0, 15))
            bad = ~np.isfinite(part).all(-1)
            s[..., g] = np.where(bad, np.float16(np.nan), step)
            mid[..., g] = np.where(bad, np.float16(np.nan), centre)
            codes[..., 64 * g:64 * g + 64] = np.where(np.isnan(c), 0, c)
    return codes, s, mid


def values(codes, s, mid):
    """One fp32 rounding: the product is exact."""
    D = codes.shape[-1]
    s, mid = (np.repeat(v.astype(np.float64), 64, -1)[..., :D] for v in (s, mid))
    return (s * (codes.astype(np.float64) - 8) + mid).astype(F)


def k_byte(t, c):
    return ((t % 8) * 4 + c // 16) * 16 + t // 8 * 8 + c % 16 // 2


def v_byte(t, c):
    return (c // 8 * 4 + t % 8 // 2) * 16 + t // 8 * 8 + c % 8 // 4 * 4 + t % 2 * 2 + c % 4 // 2


def pair_byte(t):
    return 512 + (2 * (t % 8) + t // 8) * 4


def block(desc, slot, head, group, is_v):
    """First byte of the block of 16 tokens and 64 channels that holds the token in `slot`."""
    n_heads, dim, page_tokens = desc
    G, tiles = -(-dim // 64), page_tokens // 16
    page, tile = slot // page_tokens, slot % page_tokens // 16
    return (((page * n_heads + head) * tiles + tile) * 2 + is_v) * G * 576 + group * 576


def decode(pool, desc, slots, heads=None):
    """(codes, s, mid) of K and of V, [n][heads][...], of the tokens in `slots`; pool: bytes; heads: all, or some of them."""
    n_heads, dim, _ = desc
    G = -(-dim // 64)
    slots = np.asarray(slots, np.int64).reshape(-1, 1, 1)
    h = np.arange(n_heads) if heads is None else np.asarray(heads)
    h, c, g, t = h.reshape(1, -1, 1), np.arange(dim), np.arange(G), slots % 16
    got = []
    for is_v in (0, 1):
        at = block(desc, slots, h, 0, is_v)
        codes = pool[at + c // 64 * 576 + (v_byte if is_v else k_byte)(t, c % 64)] >> (4 * (c % 2)).astype(np.uint8) & 15
        pairs = np.ascontiguousarray(pool[(at + 576 * g + pair_byte(t))[..., None] + np.arange(4)]).view(np.float16)
        got.append((codes, pairs[..., 0], pairs[..., 1]))
    return got


def plan(lens, n_new, n_free, free, table, page_tokens, n_pages, max_tokens):
    """What a plan leaves: dict of arrays, and lens and n_free after it."""
    lens, table = lens.copy(), table.copy()
    S, room = len(n_new), table.shape[1] * page_tokens
    q_start, kv_len = np.zeros(S + 1, np.int64), np.zeros(S, np.int64)
    slots, positions = np.full(max_tokens, -1, np.int64), np.full(max_tokens, -1, np.int64)
    asked = took = refused = 0
    for i in range(S):
        n, add = int(lens[i]), int(n_new[i])
        row = q_start[i]
        q_start[i + 1] = row + max(add, 0)
        ok = add >= 0 and n + add <= room and q_start[i + 1] <= max_tokens
        if ok:
            have, want = -(-n // page_tokens), -(-(n + add) // page_tokens)
            asked += want - have
            ok = want == have or asked <= n_free
        if not ok:
            refused += 1
            continue
        for j in range(have, want):
            table[i, j] = free[n_free - 1 - took]
            took += 1
        for j in range(add):
            positions[row + j] = n + j
            slots[row + j] = table[i, (n + j) // page_tokens] * page_tokens + (n + j) % page_tokens
        kv_len[i] = lens[i] = n + add
    return dict(table=table, q_start=q_start, kv_len=kv_len, slots=slots, positions=positions,
                counts=np.array([q_start[-1], took, n_free - took, refused])), lens, n_free - took


def attend(q, k, v, scale, sixteen):
    """One row and head in 64 bits: q [D], k and v each (codes, s, mid) of the n tokens that it sees.

    Returns the output [D] and what a kernel may be off by, apart from the output's own rounding.  With u the half step
    of the operands (2^-23 for two f16 terms, 2^-12 for one):
      scores: an fp32 q is off by 2^-24 of its largest channel, and the sums of codes and q are exact; a 16-bit q is exact, and
      the tensor cores truncate, at most one step of 2^-23 of
      the sum of the terms' sizes per instruction and fp32 addition, 4 and 2 for each 64 channels, 24 at most, and three
      roundings of the scaling; the sizes are those of q x (code s) and of the offset mid - 8 s;
      probabilities: e^x is off by 2^-22 and by the rounding of its argument, 3 x 2^-24 |score|; the rounding to the
      operand, u, and 2^-24 for the product with s;
      the output: up to 32 (128) instructions between sums in fp32, and 40 steps of 2^-23 of the sum of the terms' sizes in all.  That is
      less than the worst that can come of long shares, where each lane adds hundreds of terms in fp32: attend_of_long_shares."""
    u = 2.0 ** -12 if sixteen else 2.0 ** -23
    kv, ks, vs = [], [], []
    for codes, s, mid in (k, v):
        D = codes.shape[-1]
        s, mid = (np.repeat(x.astype(np.float64), 64, -1)[..., :D] for x in (s, mid))
        kv.append(s * (codes.astype(np.float64) - 8) + mid)
        ks.append(15 * s + np.abs(mid - 8 * s))
        vs.append(8 * s + np.abs(mid))
    q = q.astype(np.float64)
    score = kv[0] @ q * scale
    size = ks[0] @ np.abs(q) * abs(scale)
    off = size * 27 * 2.0 ** -23
    if not sixteen:
        off = off + ks[0].sum(1) * np.abs(q).max() * abs(scale) * 2.0 ** -24
    p = np.exp(score - score.max())
    total = p.sum()
    p = p / total
    rel = 2 * off.max() + 2 * (2.0 ** -22 + 3 * 2.0 ** -24 * np.abs(score).max() * 2) + u + 2.0 ** -23 + 40 * 2.0 ** -23
    return p @ kv[1], (p[:, None] * vs[1]).sum(0) * rel


def attend_of_long_shares(q, k, v, scale, sixteen, sets, parts):
    """attend() where warps have up to `sets` sets of tiles each, and a row's sums come of `parts` of them.  Beside the 32 truncated
    additions between sums in fp32 (128 of 16-bit rows), a lane adds two tokens a set to the sum of the probabilities and two to the mid part, and a flushed
    sum every 32 sets; then come its 32 lanes (5 additions) and the parts: 2^-24 of the sum of the terms' sizes each, and e^x between the
    flushed sums, the parts and the rest, 2^-22."""
    want, off = attend(q, k, v, scale, sixteen)
    (kc, kscale, kmid), (_, s, mid) = k, v
    D = kc.shape[-1]
    wide = lambda x: np.repeat(x.astype(np.float64), 64, -1)[..., :D]  # noqa: E731
    score = (wide(kscale) * (kc.astype(np.float64) - 8) + wide(kmid)) @ q.astype(np.float64) * scale
    p = np.exp(score - score.max())
    sizes = (p / p.sum()) @ (8 * wide(s) + np.abs(wide(mid)))
    return want, off + sizes * ((4 * sets + sets // 32 + 2 * 5 + 2 * parts) * 2.0 ** -24 + 2 * 2.0 ** -22 + (96 * 2.0 ** -23 if sixteen else 0))
