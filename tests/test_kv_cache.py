"""Keys and values in 4 bits, and attention over them: the pages' layout, refusals, tables and slot maps, new rows, and
attention against 64 bits (``_kv.py`` derives how far a kernel may be off)."""
import ctypes as C

import numpy as np
import pytest
import torch

import _kv as R

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def gsi():
    import paper_2605_03109_b200 as g
    return g


def desc(n_heads=2, head_dim=64, page_tokens=32, n_pages=8, max_seqs=4, max_pages=4, max_tokens=16):
    from paper_2605_03109_b200.binding import GsiKvDesc
    return GsiKvDesc(n_heads, head_dim, page_tokens, n_pages, max_seqs, max_pages, max_tokens)


# ---- without a GPU -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n_heads,dim,page_tokens", [(1, 64, 16), (3, 80, 48), (2, 256, 32), (2, 40, 16)])
def test_every_element_has_a_place_of_its_own(n_heads, dim, page_tokens):
    g, n_pages = gsi(), 3
    d = desc(n_heads, dim, page_tokens, n_pages)
    page = g.lib.gsi_kv_page_bytes(C.byref(d))
    assert page == n_heads * page_tokens // 16 * 2 * -(-dim // 64) * 576
    code, pair = C.c_size_t(), C.c_size_t()
    seen, pairs = set(), {}
    for slot in range(n_pages * page_tokens):
        for h in range(n_heads):
            for is_v in (0, 1):
                for c in range(dim):
                    assert g.lib.gsi_kv_locate(C.byref(d), slot, h, c, is_v, C.byref(code), C.byref(pair)) == 0
                    at = R.block((n_heads, dim, page_tokens), slot, h, c // 64, is_v)
                    assert code.value == at + (R.v_byte if is_v else R.k_byte)(slot % 16, c % 64)
                    assert pair.value == at + R.pair_byte(slot % 16)
                    assert at // page == slot // page_tokens and pair.value + 4 <= n_pages * page
                    seen.add((code.value, c % 2))
                    pairs.setdefault(pair.value, set()).add((slot, h, is_v, c // 64))
    assert len(seen) == n_pages * page_tokens * n_heads * 2 * dim
    assert all(len(v) == 1 for v in pairs.values())
    used = {b for b, _ in seen}
    assert not any(p + i in used for p in pairs for i in range(4))


def test_places_behind_32_bits():
    g = gsi()
    d = desc(64, 256, 4096, 400000, 4, 4, 16)
    code, pair = C.c_size_t(), C.c_size_t()
    slot = 399999 * 4096 + 4095
    assert g.lib.gsi_kv_locate(C.byref(d), slot, 63, 255, 1, C.byref(code), C.byref(pair)) == 0
    at = R.block((64, 256, 4096), slot, 63, 3, 1)
    assert at > 1 << 40 and (code.value, pair.value) == (at + R.v_byte(15, 63), at + R.pair_byte(15))


def test_what_is_refused_on_the_host():
    g = gsi()
    lib, INVALID, UNSUPPORTED, WORKSPACE = g.lib, 1, 2, 6
    assert lib.gsi_kv_workspace_bytes(C.byref(desc())) > 0
    assert lib.gsi_kv_page_bytes(None) == lib.gsi_kv_workspace_bytes(None) == 0
    h = C.c_void_p()
    for bad, why in ((dict(n_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=257), UNSUPPORTED),
                     (dict(page_tokens=24), UNSUPPORTED), (dict(page_tokens=4112), UNSUPPORTED), (dict(n_pages=0), INVALID),
                     (dict(n_pages=1 << 27), UNSUPPORTED), (dict(max_pages=1 << 27), UNSUPPORTED),
                     (dict(max_seqs=g.GSI_KV_MAX_SEQS + 1), UNSUPPORTED), (dict(max_tokens=0), INVALID)):
        d = desc(**bad)
        assert lib.gsi_kv_page_bytes(C.byref(d)) == lib.gsi_kv_workspace_bytes(C.byref(d)) == 0, bad
        assert lib.gsi_kv_create(C.byref(d), 4096, 1 << 40, None, C.byref(h)) == why, bad
    d = desc()
    assert lib.gsi_kv_create(C.byref(d), 4096 + 16, 1 << 40, None, C.byref(h)) == INVALID
    assert lib.gsi_kv_create(C.byref(d), 4096, 16, None, C.byref(h)) == WORKSPACE
    assert lib.gsi_kv_create(C.byref(d), 4096, 1 << 40, None, None) == INVALID
    assert h.value is None
    code, pair = C.c_size_t(), C.c_size_t()
    for slot, head, channel, is_v in ((-1, 0, 0, 0), (256, 0, 0, 0), (0, 2, 0, 0), (0, -1, 0, 0), (0, 0, 64, 0), (0, 0, 0, 2)):
        assert lib.gsi_kv_locate(C.byref(d), slot, head, channel, is_v, C.byref(code), C.byref(pair)) == INVALID
    # without a handle nothing is looked at
    assert lib.gsi_kv_plan(None, 4, 1, 1, 4, 4, 4, 4, 4, 4, 4, 4, 4, None) == INVALID
    assert lib.gsi_kv_release(None, 4, 1, 4, 4, 4, 4, None) == INVALID
    assert lib.gsi_kv_append(None, 16, 16, 1, 1, 1, 1, 1, 16, 1, 16, None) == INVALID
    assert lib.gsi_kv_read(None, 16, 16, 1, 1, 16, 16, None) == INVALID
    assert lib.gsi_kv_attend(None, 16, 1, 1, 1, 1, 1, 1.0, 16, 16, 16, 1, 16, 16, 1, 1, None) == INVALID
    assert lib.gsi_kv_get_status(None, None) == INVALID
    assert lib.gsi_kv_destroy(None) == INVALID


def test_a_cache_without_a_device_is_refused():
    g = gsi()
    with pytest.raises(g.GsiError):
        g.KVCache(2, 300, 8, 4, 64)
    with pytest.raises(g.GsiError):
        g.KVCache(2, 64, 8, 4, 64, page_tokens=20)
    with pytest.raises(AssertionError):
        g.KVCache(2, 64, 8, 4, 64, pages=torch.zeros(8 * 9216, dtype=torch.uint8))


def test_what_the_calls_refuse_before_the_library_sees_it():
    """Tensors of another shape, type or device than the cache's; here the cache's device is the host, so every call that
    passes the checks would fail, and every one below has to stop before."""
    from paper_2605_03109_b200 import binding
    calls = binding._calls
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    state = calls.kv_state(0, 2, 64, 2, torch.zeros(2 * 8 * 9216, dtype=torch.uint8), i(4, 4), i(4), i(8), i(1), i(5), i(4), i(16), i(16), i(4))
    rows = lambda n, heads=2, dim=64, dtype=torch.float32: torch.zeros(n, heads, dim, dtype=dtype)  # noqa: E731
    plain = (AssertionError, TypeError)
    for n_new in (torch.zeros(4), i(2, 2), i(8)[::2], torch.zeros(4, dtype=torch.int64), [1]):
        with pytest.raises(plain):
            calls.kv_plan(state, n_new, True, None)
    for done in (torch.zeros(4), i(4), [True]):
        with pytest.raises(plain):
            calls.kv_release(state, done, None)
    ok = rows(3)
    for k, v, layer, slots in ((rows(3, 3), ok, 0, None), (ok, rows(3, 2, 32), 0, None), (rows(3, dim=128)[..., ::2], ok, 0, None),
                               (ok, rows(2), 0, None), (ok, rows(3, dtype=torch.float16), 0, None), (ok, ok, 2, None), (ok, ok, -1, None),
                               (ok.double(), ok.double(), 0, None), (ok, ok, 0, i(2)), (ok, ok, 0, i(4)), (ok, ok, 0, torch.zeros(3)),
                               (rows(17), rows(17), 0, None), (ok[0], ok[0], 0, None), (None, ok, 0, None)):
        with pytest.raises(plain):
            calls.kv_append(state, k, v, layer, slots, None)
    for q, layer, out in ((rows(3, 3), 0, None), (rows(3, 4, 32), 0, None), (rows(3, 4).double(), 0, None), (rows(3, 4), 2, None),
                          (rows(3, 4), 0, rows(3, 2)), (rows(3, 4), 0, rows(2, 4)), (rows(3, 4), 0, rows(3, 4, dtype=torch.float16)),
                          (rows(3, 0), 0, None), (rows(3, 4), 0, 5)):
        with pytest.raises(plain):
            calls.kv_attend(state, q, layer, 1.0, out, None)
    with pytest.raises(plain):
        calls.kv_read(state, torch.zeros(3), 0, torch.zeros(0), None)
    with pytest.raises(plain):
        calls.kv_read(state, i(3), 2, torch.zeros(0), None)
    with pytest.raises(plain):
        calls.kv_read(state, i(3), 0, torch.zeros(0, dtype=torch.float64), None)
    with pytest.raises(ValueError):
        calls.kv_plan(None, i(4), True, None)


def test_the_restated_numbers():
    """The definition's own properties, on the CPU: half a step, plus the roundings of s and mid."""
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((200, 80)) * np.exp(rng.uniform(-4, 4, (200, 1)))).astype(np.float32)
    codes, s, mid = R.quantise(x)
    got = R.values(codes, s, mid)
    S, M = (np.repeat(v.astype(np.float64), 64, -1)[:, :80] for v in (s, mid))
    assert (np.abs(got - x.astype(np.float64)) <= S * (0.5 + 8 * 2.0 ** -11 + 2.0 ** -20) + np.abs(M) * 2.0 ** -11).all()
    assert codes.max() == 15 and codes.min() == 0
    flat = R.quantise(np.full((1, 64), 0.3, np.float32))
    assert (flat[0] == 8).all() and R.values(*flat)[0, 0] == np.float32(np.float16(0.3))


def test_how_far_a_value_may_be_off():
    """The bound that the header states: ranges from f16's subnormal steps, and below, to the largest that do not saturate,
    centres from 0 to far outside the range; and where it ends."""
    rng = np.random.default_rng(81)
    n, D = 20000, 64
    size = np.exp(rng.uniform(np.log(1e-10), np.log(3e6), (n, 1)))
    centre = rng.choice([0.0, 1.0, -1.0], (n, 1)) * np.exp(rng.uniform(np.log(1e-9), np.log(7e4), (n, 1)))
    shape = rng.choice(4, (n, 1))
    x = np.where(shape == 0, rng.standard_normal((n, D)) / 4, np.where(shape == 1, rng.uniform(-1, 1, (n, D)),
                 np.where(shape == 2, rng.choice([-1.0, 1.0], (n, D)), np.linspace(-1, 1, D))))
    x = (x * size + centre).astype(np.float32)
    codes, s, mid = R.quantise(x)
    got, s, mid = R.values(codes, s, mid).astype(np.float64), s.astype(np.float64), mid.astype(np.float64)
    off = np.abs(got - x.astype(np.float64)).max(1, keepdims=True)
    ds, dm = np.maximum(2.0 ** -11 * s, 2.0 ** -25), np.maximum(2.0 ** -11 * np.abs(mid), 2.0 ** -25)
    bound = np.maximum(s / 2, 15 * ds) + dm + 2.0 ** -22 * np.abs(x).max(1, keepdims=True)
    free = (s < 65504) & (np.abs(mid) < 65504)
    assert (off <= bound)[free].all()
    assert (free & (s == 0)).sum() > 500 and (free & (s > 0) & (s < 2.0 ** -14)).sum() > 500 and (~free).sum() > 100
    assert (off > s / 2 + 2.0 ** -11 * np.abs(mid) + 2.0 ** -11 * 8 * s)[free].any()      # (half a step and the normal roundings are not all)
    assert ((x.max(1) - x.min(1) > 15 * 65472) | (np.abs(x.min(1) + 8 * s[:, 0]) > 65472))[~free[:, 0]].all()
    assert (off > bound)[~free].any()


# ---- on the GPU ----------------------------------------------------------------------------------------------------

gpu = pytest.mark.gpu


def state_of(c):
    return {n: getattr(c, n).cpu().numpy() for n in ("table", "q_start", "kv_len", "slots", "positions", "counts", "lens", "n_free", "free")}


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype).cuda()


def read_back(c, slots, layer=0):
    pool = c.pages.view(-1).cpu().numpy()
    per = len(pool) // c.n_layers
    return R.decode(pool[layer * per:(layer + 1) * per], (c.n_heads, c.head_dim, c.page_tokens), slots)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,heads,dim,page", [(1, 12, 64, 16), (3, 2, 40, 16), (37, 3, 80, 48), (65, 2, 256, 64), (8, 1, 1, 16), (33, 2, 129, 32), (16, 2, 96, 16)])
def test_rows_are_held_as_the_definition_has_them(dtype, n, heads, dim, page):
    g, rng = gsi(), np.random.default_rng(dim + n)
    c = g.KVCache(heads, dim, 5, 2, 64, page_tokens=page, max_tokens=n, n_layers=2)
    c.pages.fill_(0xA5)
    before = c.pages.clone()
    slots = rng.permutation(5 * page)[:n].astype(np.int32)
    if n > 20:
        slots[:16] = np.arange(16) + 16          # whole tiles too
        slots[16:] = rng.permutation(np.setdiff1d(np.arange(5 * page), np.arange(16, 32)))[:n - 16]
        slots[5], slots[20] = -1, -7             # ... with rows that go nowhere
    buffer = rows(rng, (n, 2 * heads * dim + 3), dtype) * torch.exp(rows(rng, (n, 1), torch.float32)).to(dtype)
    k, v = buffer[:, 3:3 + heads * dim].unflatten(1, (heads, dim)), buffer[:, 3 + heads * dim:].unflatten(1, (heads, dim))
    k[0, 0, 0] = 0.0
    k[-1, 0] = 0.25                              # a group without extent
    v[0, -1, dim // 2] = 3000.0
    c.append(k, v, layer=1, slots=ints(slots))
    live = slots >= 0
    want = [R.quantise(x.float().cpu().numpy()) for x in (k, v)]
    for (codes, s, mid), (wc, ws, wm) in zip(read_back(c, slots[live], 1), want):
        assert np.array_equal(codes, wc[live]) and np.array_equal(s, ws[live]) and np.array_equal(mid, wm[live])
    # ... every other byte is as it was (tokens share bytes with no other: half a byte is another channel's)
    assert torch.equal(c.pages[0], before[0])
    others = np.setdiff1d(np.arange(5 * page), slots[live])
    for now, then in zip(read_back(c, others, 1), R.decode(before.view(-1).cpu().numpy(), (heads, dim, page), others)):
        for a, b in zip(now, then):
            assert np.array_equal(a.view(np.uint8 if a.dtype == np.uint8 else np.uint16), b.view(np.uint8 if b.dtype == np.uint8 else np.uint16))
    # ... and read as these numbers
    for out in DTYPES:
        for got, w in zip(c.read(ints(slots), layer=1, dtype=out), want):
            x = torch.from_numpy(np.where(live[:, None, None], R.values(*w), np.float32(0))).to(out)
            assert got.dtype == out and torch.equal(got.cpu(), x)
    assert c.status() == 0


@gpu
def test_rows_that_are_not_ordinary_numbers():
    g = gsi()
    c = g.KVCache(1, 128, 1, 1, 16, page_tokens=16)
    x = torch.zeros(9, 1, 128)
    x[0] = torch.linspace(-1e6, 1e6, 128)
    x[1, 0, 5] = float("nan")
    x[2, 0, 64], x[2, 0, 3] = float("inf"), 1.0
    x[3] = torch.linspace(3e38, -3e38, 128)          # a range that passes fp32
    x[4] = torch.linspace(0, 1e-6, 128)              # steps below f16's normal ones
    x[5] = torch.linspace(-1e-40, 1e-40, 128)
    x[6] = -0.0
    x[7] = 1000 + torch.linspace(0, 1e-3, 128)
    x[8, 0, 100] = -float("inf")
    c.append(x.cuda(), -x.cuda(), slots=ints(list(range(9))))
    for got, raw, sign in zip(c.read(ints(list(range(9)))), read_back(c, range(9)), (1, -1)):
        codes, s, mid = R.quantise(sign * x.numpy())
        assert np.array_equal(raw[1], s, equal_nan=True) and np.array_equal(raw[2], mid, equal_nan=True)
        fine = ~np.isnan(np.repeat(s, 64, -1))
        assert np.array_equal(raw[0][fine], codes[fine])
        assert np.array_equal(got.cpu().numpy(), R.values(codes, s, mid), equal_nan=True)


@gpu
def test_a_slot_behind_the_pool_is_reported_and_passed_over():
    g = gsi()
    c = g.KVCache(1, 64, 2, 1, 16, page_tokens=16)
    c.pages.fill_(0)
    k = torch.randn(3, 1, 64, device="cuda")
    c.append(k, k, slots=ints([-1, 5, -2 ** 31]))
    assert c.status() == 0
    c.append(k, k, slots=ints([32, 6, 2 ** 31 - 1]))
    assert c.status() == 1
    got, _ = c.read(ints([5, 32, 6]))
    assert torch.equal(got[1], torch.zeros_like(got[1])) and got[0].any() and got[2].any()


@gpu
@pytest.mark.parametrize("seed", range(6))
def test_plans_and_releases_are_the_ones_of_the_definition(seed):
    g, rng = gsi(), np.random.default_rng(seed)
    page, n_seqs = int(rng.choice([16, 48, 64])), int(rng.choice([1, 3, 33, 600]))
    n_pages, max_tokens = int(rng.integers(1, 4 * n_seqs + 2)), int(rng.integers(1, 40 * n_seqs + 2))
    c = g.KVCache(1, 64, n_pages, n_seqs, 5 * page - 3, page_tokens=page, max_tokens=max_tokens)
    c.free.copy_(torch.from_numpy(rng.permutation(n_pages).astype(np.int32)))
    s = state_of(c)
    lens, n_free, free, table = s["lens"].astype(np.int64), n_pages, s["free"].copy(), s["table"].astype(np.int64)
    for step in range(8):
        n_new = rng.choice([0, 1, 1, 1, int(rng.integers(0, 3 * page))], n_seqs) if step else rng.integers(0, 2 * page, n_seqs)
        if step == 3:
            n_new[rng.integers(n_seqs)] = -5
            n_new[rng.integers(n_seqs)] = 2 ** 31 - 1
        n = n_seqs if step != 4 else max(1, n_seqs // 2)
        commit = step != 5
        want, lens_after, free_after = R.plan(lens, n_new[:n], n_free, free, table, page, n_pages, max_tokens)
        c.plan(ints(n_new[:n].tolist()), commit=commit)
        got = state_of(c)
        want["q_start"], want["counts"] = np.minimum(want["q_start"], 2 ** 31 - 1), np.minimum(want["counts"], 2 ** 31 - 1)
        for name in ("q_start", "kv_len"):
            assert np.array_equal(got[name][:len(want[name])], want[name]), (step, name)
        for name in ("table", "slots", "positions", "counts"):
            assert np.array_equal(got[name], want[name]), (step, name)
        table = want["table"]
        if commit:
            lens, n_free = lens_after, free_after
        assert np.array_equal(got["lens"], lens) and got["n_free"][0] == n_free, step
        live = want["slots"][want["slots"] >= 0]
        assert len(np.unique(live)) == len(live)
        # some end
        done = rng.random(n_seqs) < 0.3
        back = [int(table[i, j]) for i in range(n_seqs) if done[i] for j in range(-(-int(lens[i]) // page))]
        for i in np.nonzero(done)[0]:
            table[i, :-(-int(lens[i]) // page)] = -1
            lens[i] = 0
        free[n_free:n_free + len(back)] = back[::-1]
        n_free += len(back)
        c.release(torch.from_numpy(done).cuda() if step % 2 else torch.from_numpy(done.astype(np.uint8) * 7).cuda())
        got = state_of(c)
        assert np.array_equal(got["table"], table) and np.array_equal(got["lens"], lens) and got["n_free"][0] == n_free
        assert np.array_equal(got["free"][:n_free], free[:n_free])
    assert c.status() == 0


@gpu
def test_a_plan_for_empty_requests_and_their_release_leave_the_pool_as_it_was():
    g = gsi()
    c = g.KVCache(1, 64, 4000, 2048, 160, page_tokens=16, max_tokens=30000)
    free = c.free.clone()
    n_new = torch.arange(2048, dtype=torch.int32, device="cuda") % 23
    for _ in range(3):
        c.plan(n_new)
        assert c.counts.cpu().tolist()[3] == 0
        c.release(torch.ones(2048, dtype=torch.bool, device="cuda"))
        assert torch.equal(c.free, free) and c.n_free.item() == 4000 and not c.lens.any() and (c.table == -1).all()


def slots_of(c, kv_len, table):
    got = [table[i, np.arange(n) // c.page_tokens] * c.page_tokens + np.arange(n) % c.page_tokens for i, n in enumerate(kv_len)]
    return np.concatenate(got).astype(np.int32)


def fill(c, rng, kv_len, table):
    """Random tokens of the lengths `kv_len`; everything else of the pool is what makes a kernel that reads it wrong."""
    c.pages.fill_(0xFF)      # (all codes 15, all pairs NaN)
    slots = slots_of(c, kv_len, table)
    if len(slots):
        g = torch.Generator("cuda").manual_seed(int(rng.integers(1 << 30)))
        k, v = (torch.randn(len(slots), c.n_heads, c.head_dim, device="cuda", generator=g) * s for s in (1.5, 1.0))
        k[:, :, 0] *= 5
        c.append(k, v + 0.1, slots=torch.from_numpy(slots).cuda())
    return slots


def fill_and_read(c, rng, kv_len, table):
    return read_back(c, fill(c, rng, kv_len, table))


def check(c, q, out, before, kv, kv_len, news, scale):
    """Every row of out against 64 bits, or as it was."""
    sixteen = out.dtype != torch.float32
    half = torch.finfo(out.dtype).eps / 2
    shared = q.shape[1] // c.n_heads
    qn, got = q.float().cpu().numpy(), out.double().cpu().numpy()
    row = first = 0
    for n, m in zip(kv_len, news):
        part = [[x[first:first + n] for x in t] for t in kv]
        for i in range(m):
            sees = n - m + i + 1
            for h in range(q.shape[1]):
                have = [[x[:max(sees, 0), h // shared] for x in t] for t in part]
                if sees <= 0:
                    assert not got[row, h].any()
                    continue
                want, off = R.attend(qn[row, h], *have, scale, sixteen)
                tol = off + half * np.abs(want) + (6e-8 if out.dtype == torch.float16 else 0)   # (f16's smallest step)
                assert (np.abs(got[row, h] - want) <= tol).all(), (row, h, sees, float((np.abs(got[row, h] - want) / tol).max()))
            row += 1
        first += n
    assert torch.equal(out[row:], before[row:])


def a_cache(heads, dim, page, kv_len, news, rng, extra=2):
    pages = [-(-n // page) for n in kv_len]
    n_pages = sum(pages) + extra
    c = gsi().KVCache(heads, dim, n_pages, len(kv_len), max(max(kv_len), 1) + page, page_tokens=page, max_tokens=max(sum(news), 1))
    order = rng.permutation(n_pages)
    table = np.full(c.table.shape, -1, np.int64)
    at = 0
    for i, p in enumerate(pages):
        table[i, :p] = order[at:at + p]
        at += p
    c.table.copy_(torch.from_numpy(table))
    c.kv_len.copy_(ints(kv_len))
    c.q_start.copy_(ints([0] + np.cumsum(news).tolist()))
    return c, table


LENGTHS = [
    ("one", [1], [1]),
    ("around a tile", [15, 16, 17, 0, 1, 32, 33], [1, 1, 1, 0, 1, 1, 1]),
    ("several rows", [5, 40, 2, 130, 16], [5, 3, 2, 7, 16]),
    ("rows that see nothing", [0, 2, 20, 0], [2, 5, 1, 0]),
    ("many warps", [700, 129, 300], [1, 2, 1]),
]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name,kv_len,news", LENGTHS, ids=[x[0] for x in LENGTHS])
@pytest.mark.parametrize("heads,shared,dim,page", [(2, 1, 64, 16), (1, 4, 128, 32), (2, 3, 80, 48), (1, 1, 256, 64), (1, 9, 40, 16), (1, 2, 192, 16)])
def test_attention_is_the_one_in_64_bits(dtype, name, kv_len, news, heads, shared, dim, page):
    rng = np.random.default_rng(len(name) + dim)
    c, table = a_cache(heads, dim, page, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    n = sum(news)
    q = rows(rng, (n + 2, heads * shared, dim), dtype, 1.3)
    out = torch.full_like(q, 9.0)
    before = out.clone()
    assert c.attend(q, out=out) is out
    check(c, q, out, before, kv, kv_len, news, dim ** -0.5)
    again = c.attend(q)
    assert torch.equal(again[:n], out[:n])
    assert c.status() == 0


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_any_stride(dtype):
    rng = np.random.default_rng(3)
    kv_len, news = [37, 5], [3, 1]
    c, table = a_cache(2, 64, 16, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    wide = rows(rng, (4, 3 + 5 * 64), dtype)
    q = wide[:, 3:3 + 4 * 64].unflatten(1, (4, 64))                     # rows that begin nowhere in particular
    turned = rows(rng, (4, 4, 64), dtype).transpose(0, 1)               # heads outside, tokens inside
    out = torch.full((4, 4, 70), 9.0, dtype=dtype, device="cuda")
    for x in (q, turned, q[:, :1].expand(4, 4, 64)):
        got = out[:, :, 5:69]
        c.attend(x, scale=0.3, out=got)
        check(c, x, got, got, kv, kv_len, news, 0.3)
        assert (out[:, :, :5] == 9).all() and (out[:, :, 69:] == 9).all()


@gpu
@pytest.mark.parametrize("size", [1e-30, 1e-6, 1.0, 1e6, 1e30])
def test_q_of_any_size(size):
    rng = np.random.default_rng(4)
    c, table = a_cache(1, 128, 16, [45], [1], rng)
    kv = fill_and_read(c, rng, [45], table)
    q = rows(rng, (1, 2, 128), torch.float32)
    q = (q.double() * size).float()
    q[:, 1, ::3] = 0.0
    out = c.attend(q, scale=0.1 / size)
    check(c, q, out, out, kv, [45], [1], float(np.float32(0.1 / size)))


@gpu
def test_values_of_any_size_side_by_side():
    """Steps of V that differ by 2^40 between tokens, heads and groups of one cache."""
    rng = np.random.default_rng(6)
    c, table = a_cache(2, 128, 16, [200], [1], rng)
    n = 200
    k = torch.from_numpy(rng.standard_normal((n, 2, 128)).astype(np.float32)).cuda()
    v = torch.from_numpy((rng.standard_normal((n, 2, 128)) * 2.0 ** rng.integers(-20, 15, (n, 2, 1))).astype(np.float32)).cuda()
    v[:, 1, :64] = 0.0
    v[50:150, 0, 64:] = 7.5
    c.pages.fill_(0xFF)
    slots = [int(table[0, p // 16] * 16 + p % 16) for p in range(n)]
    c.append(k, v, slots=ints(slots))
    for dtype in (torch.float32, torch.bfloat16):
        q = rows(rng, (1, 2, 128), dtype, 0.7)
        out = c.attend(q)
        check(c, q, out, out, read_back(c, slots), [n], [1], 128 ** -0.5)


@gpu
def test_what_is_not_a_number_stays_where_it_is_seen():
    rng = np.random.default_rng(7)
    kv_len, news = [60, 40], [20, 1]
    for dtype in (torch.float32, torch.float16):
        c, table = a_cache(2, 128, 16, kv_len, news, rng)
        kv = fill_and_read(c, rng, kv_len, table)
        q = rows(rng, (21, 2, 128), dtype)
        clean = c.attend(q)
        check(c, q, clean, clean, kv, kv_len, news, 128 ** -0.5)
        # token 50 of the first request (rows 10.. see it): a NaN in v's second group of head 0, infinity in k of head 1
        slot = ints([int(table[0, 3] * 16 + 2)])
        k, v = (torch.randn(1, 2, 128, device="cuda") for _ in range(2))
        v[0, 0, 70], k[0, 1, 3] = float("nan"), float("inf")
        c.append(k, v, slots=slot)
        out = c.attend(q)
        assert torch.equal(out[:10], clean[:10]) and torch.equal(out[20:], clean[20:])
        assert out[10:20, 0, :64].isfinite().all() and out[10:20, 0, 64:].isnan().all() and out[10:20, 1].isnan().all()
        # ... and of q
        q[3, 1, 5] = float("nan")
        out = c.attend(q)
        assert out[3, 1].isnan().all() and torch.equal(out[3, 0], clean[3, 0])
        assert torch.equal(out[:3], clean[:3]) and torch.equal(out[4:10], clean[4:10])
        assert c.status() == 0


@gpu
def test_pages_and_lengths_outside_are_reported():
    rng = np.random.default_rng(8)
    kv_len, news = [40, 40, 40], [1, 2, 1]
    for bad in (-1, 1 << 30, 99):
        c, table = a_cache(1, 64, 16, kv_len, news, rng)
        kv = fill_and_read(c, rng, kv_len, table)
        q = rows(rng, (4, 1, 64), torch.float32)
        clean = c.attend(q)
        assert c.status() == 0
        c.table[1, 1] = bad
        out = c.attend(q)
        assert out[1:3].isnan().all() and torch.equal(out[0], clean[0]) and torch.equal(out[3], clean[3])
        assert c.status() == 1
    c, table = a_cache(1, 64, 16, kv_len, news, rng)
    fill(c, rng, kv_len, table)
    clean = c.attend(q)
    c.kv_len[2] = 16 * c.table.shape[1] + 1
    out = c.attend(q)
    assert out[3].isnan().all() and torch.equal(out[:3], clean[:3]) and c.status() == 1
    c.kv_len[2] = -7
    out = c.attend(q)
    assert not out[3].any() and torch.equal(out[:3], clean[:3])


@gpu
def test_requests_over_the_whole_grid():
    """More requests than CTAs, requests that take many CTAs, and both at once: against 64 bits, twice the same."""
    rng = np.random.default_rng(9)
    for heads, dim, kv_len in ((1, 64, [int(x) for x in rng.integers(0, 40, 900)]), (1, 128, [6000]), (2, 64, [2000] + [3] * 100 + [0] * 30 + [1500])):
        news = [1] * len(kv_len)
        c, table = a_cache(heads, dim, 64, kv_len, news, rng)
        kv = fill_and_read(c, rng, kv_len, table)
        for dtype in (torch.float32, torch.bfloat16):
            q = rows(rng, (len(news), heads, dim), dtype)
            out = c.attend(q)
            check(c, q, out, out, kv, kv_len, news, dim ** -0.5)
            for _ in range(3):
                assert torch.equal(c.attend(q), out)


def check_some(c, q, out, kv_len, news, slots, scale, which):
    """check() of the rows of some (request, head of the cache)."""
    pool = c.pages.view(-1).cpu().numpy()
    first, row = np.concatenate([[0], np.cumsum(kv_len)]), np.concatenate([[0], np.cumsum(news)])
    shared, sixteen, half = q.shape[1] // c.n_heads, out.dtype != torch.float32, torch.finfo(out.dtype).eps / 2
    qn, got = q.float().cpu().numpy(), out.double().cpu().numpy()
    for i, h in which:
        k, v = R.decode(pool, (c.n_heads, c.head_dim, c.page_tokens), slots[first[i]:first[i + 1]], [h])
        for m in sorted({0, news[i] // 2, news[i] - 1}):
            sees = kv_len[i] - news[i] + m + 1
            for x in sorted({h * shared, h * shared + shared - 1}):
                want, off = R.attend(qn[row[i] + m, x], *[[y[:sees, 0] for y in z] for z in (k, v)], scale, sixteen)
                tol = off + half * np.abs(want)
                assert (np.abs(got[row[i] + m, x] - want) <= tol).all(), (i, h, m, x)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("shared,new", [(1, 1), (2, 1), (1, 3), (5, 1), (2, 9)])
def test_one_long_request_over_the_whole_grid(dtype, dim, shared, new):
    """Sums of hundreds of warps meet: of one row and of many."""
    rng = np.random.default_rng(dim + shared)
    kv_len, news = [20011], [new]
    c, table = a_cache(1, dim, 48, kv_len, news, rng)
    slots = fill(c, rng, kv_len, table)
    q = rows(rng, (new, shared, dim), dtype)
    out = c.attend(q)
    check_some(c, q, out, kv_len, news, slots, dim ** -0.5, [(0, 0)])
    assert torch.equal(c.attend(q), out) and c.status() == 0


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("seqs,heads,length,new", [(8, 64, 10007, 1), (8, 32, 5009, 4), (4, 16, 20011, 2)])
def test_long_shares(dtype, seqs, heads, length, new):
    """Every warp has more tokens than the tensor cores sum at a time."""
    rng = np.random.default_rng(seqs)
    kv_len, news = [length - 13 * i for i in range(seqs)], [new] * seqs
    c, table = a_cache(heads, 64, 64, kv_len, news, rng)
    slots = fill(c, rng, kv_len, table)
    q = rows(rng, (sum(news), heads, 64), dtype)
    out = c.attend(q)
    which = [(0, 0), (seqs - 1, heads - 1)] + [(int(rng.integers(seqs)), int(rng.integers(heads))) for _ in range(6)]
    check_some(c, q, out, kv_len, news, slots, 0.125, which)
    assert torch.equal(c.attend(q), out)


@gpu
@pytest.mark.parametrize("dim", [1, 3, 8, 65, 129, 193, 255])
def test_heads_of_any_width(dim):
    rng = np.random.default_rng(dim)
    kv_len, news = [70, 3, 18], [1, 1, 2]
    c, table = a_cache(2, dim, 16, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    for dtype in DTYPES:
        q = rows(rng, (4, 4, dim), dtype)
        out = torch.full((4, 4, dim + 1), 9.0, dtype=dtype, device="cuda")
        c.attend(q, out=out[:, :, :dim])
        check(c, q, out[:, :, :dim], out[:, :, :dim], kv, kv_len, news, dim ** -0.5)
        assert (out[:, :, dim] == 9).all()


@gpu
def test_many_q_heads_and_scales_of_any_sign():
    rng = np.random.default_rng(12)
    kv_len, news = [33, 100], [1, 3]
    c, table = a_cache(1, 64, 16, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    for dtype in (torch.float32, torch.bfloat16):
        q = rows(rng, (4, 71, 64), dtype)
        for scale in (0.125, -0.2, 0.0):
            out = c.attend(q, scale=scale)
            check(c, q, out, out, kv, kv_len, news, scale)


@gpu
def test_scores_that_rise_and_fall():
    """Running maxima that move with every token, by little and by much, and one token that takes it all."""
    rng = np.random.default_rng(13)
    n = 900
    c, table = a_cache(1, 64, 16, [n], [1], rng)
    v = torch.randn(n, 1, 64, device="cuda")
    for name in ("up", "down", "saw", "peak"):
        x = torch.linspace(-30, 30, n)
        x = {"up": x, "down": -x, "saw": x * torch.where(torch.arange(n) % 7 < 3, 1.0, -1.0), "peak": torch.where(torch.arange(n) == 457, 200.0, 0.01 * x)}[name]
        k = torch.randn(n, 1, 64, device="cuda") * 0.01
        k[:, 0, 5] = x.cuda()
        slots = slots_of(c, [n], table)
        c.append(k, v, slots=torch.from_numpy(slots).cuda())
        for dtype in (torch.float32, torch.bfloat16):
            q = rows(rng, (1, 3, 64), dtype, 0.1)
            q[0, :, 5] = torch.tensor([1.0, -3.0, 0.2])
            out = c.attend(q, scale=1.0)
            check(c, q, out, out, read_back(c, slots), [n], [1], 1.0)


@gpu
def test_a_pool_behind_32_bits():
    g = gsi()
    page_bytes = 8 * 64 // 16 * 2 * 2 * 576
    n_pages = 5 * 2 ** 30 // page_bytes
    k, v, q = (torch.randn(80, 8, 128, device="cuda") for _ in range(3))
    big = g.KVCache(8, 128, n_pages, 2, 100, page_tokens=64, max_tokens=80)
    assert big.pages.numel() > 1 << 32 and big.page_bytes == page_bytes
    big.free.copy_(torch.arange(n_pages, dtype=torch.int32, device="cuda"))        # the last page goes first
    big.plan(ints([50, 30]))
    assert big.table[:, 0].cpu().tolist() == [n_pages - 1, n_pages - 2]
    big.append(k, v)
    out = big.attend(q)
    live = big.slots.cpu().numpy()
    small = g.KVCache(8, 128, 4, 2, 100, page_tokens=64, max_tokens=80)
    small.plan(ints([50, 30]))
    small.append(k, v)
    assert torch.equal(small.attend(q), out)
    for a, b in zip(small.read(small.slots), big.read(big.slots)):
        assert torch.equal(a, b) and a.any()
    assert live.min() > (n_pages - 3) * 64 and big.status() == 0


@gpu
def test_a_captured_step_moves_on_by_itself():
    """Plan, append and attention of two layers in one graph: replays are the eager steps."""
    g = gsi()

    def one():
        c = g.KVCache(2, 64, 40, 3, 128, page_tokens=16, n_layers=2, max_tokens=3)
        return c, torch.zeros(3, 4, 64, device="cuda"), [torch.zeros(3, 2, 64, device="cuda") for _ in range(4)], ints([1, 1, 1])

    def step(c, q, kv, n_new, out):
        c.plan(n_new)
        for layer in range(2):
            c.append(kv[2 * layer], kv[2 * layer + 1], layer)
            out[layer].copy_(c.attend(q, layer))

    torch.manual_seed(1)
    inputs = [[torch.randn(3, 4, 64, device="cuda")] + [torch.randn(3, 2, 64, device="cuda") for _ in range(4)] for _ in range(40)]
    eager, want = one(), []
    outs = [torch.zeros(3, 4, 64, device="cuda") for _ in range(2)]
    for x in inputs:
        step(eager[0], x[0], x[1:], eager[3], outs)
        want.append([o.clone() for o in outs])
    c, q, kv, n_new = one()
    got = [torch.zeros(3, 4, 64, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(c, q, kv, n_new, got)
    torch.cuda.current_stream().wait_stream(side)
    for i, x in enumerate(inputs):
        q.copy_(x[0])
        for to, of in zip(kv, x[1:]):
            to.copy_(of)
        graph.replay()
        for a, b in zip(got, want[i]):
            assert torch.equal(a, b), i
    n_new[1] = 0                         # a request pauses
    graph.replay()
    assert c.lens.cpu().tolist() == [41, 40, 41] and c.counts.cpu().tolist()[0] == 2 and c.status() == 0


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_captured_attention_goes_by_the_lengths_of_its_replay(dtype):
    """Captured with short requests, replayed with long ones, and the other way round."""
    rng = np.random.default_rng(21)
    long, short, news = [5000, 1, 700, 0], [3, 40, 0, 17], [2, 1, 1, 1]
    for first, then in ((short, long), (long, short)):
        c, table = a_cache(2, 128, 16, [max(a, b) for a, b in zip(long, short)], news, rng)
        kv = fill_and_read(c, rng, [max(a, b) for a, b in zip(long, short)], table)
        at = np.concatenate([[0], np.cumsum([max(a, b) for a, b in zip(long, short)])])
        q = rows(rng, (6, 4, 128), dtype)
        out = torch.zeros_like(q)
        c.kv_len.copy_(ints(first))
        c.attend(q, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.attend(q, out=out)
        for lens in (then, first, then):
            c.kv_len.copy_(ints(lens))
            out.fill_(9.0)
            before = out.clone()
            graph.replay()
            of = [[np.concatenate([x[at[i]:at[i] + n] for i, n in enumerate(lens)]) for x in z] for z in kv]
            check(c, q, out, before, of, lens, news, 128 ** -0.5)
            assert torch.equal(c.attend(q)[:5], out[:5])
        assert c.status() == 0


@gpu
@pytest.mark.parametrize("n_seqs,page,heads", [(2048, 16, 1), (3, 4096, 2), (17, 112, 3)])
def test_the_ends_of_the_sizes(n_seqs, page, heads):
    """As many requests as there can be, the largest pages, pages whose tiles are no power of two; planned, not laid out here."""
    g, rng = gsi(), np.random.default_rng(n_seqs)
    n_new = rng.integers(0, 2 * page if n_seqs < 100 else 20, n_seqs)
    c = g.KVCache(heads, 64, int(sum(-(-n // page) for n in n_new)) + n_seqs, n_seqs, 3 * page, page_tokens=page, max_tokens=int(n_new.sum()),
                  pages=torch.full((int(sum(-(-n // page) for n in n_new)) + n_seqs, heads * page * 72), 0xFF, dtype=torch.uint8, device="cuda"))
    c.plan(ints(n_new.tolist()))
    n = int(n_new.sum())
    k, v = (torch.randn(n, heads, 64, device="cuda") for _ in range(2))
    c.append(k, v)
    c.plan(ints([1] * n_seqs), commit=False)
    more = [torch.randn(n_seqs, heads, 64, device="cuda") for _ in range(3)]
    c.append(more[1], more[2])
    out = c.attend(more[0])
    lens = (n_new + 1).tolist()
    table = c.table.cpu().numpy().astype(np.int64)
    check(c, more[0], out, out, read_back(c, slots_of(c, lens, table)), lens, [1] * n_seqs, 0.125)
    assert c.status() == 0


@gpu
def test_streams_of_their_own():
    """Two caches on two streams at once, each with its own workspace, against one after the other."""
    rng = np.random.default_rng(11)
    made = []
    for i in range(2):
        kv_len, news = [900, 17, 300 + i], [1, 1, 2]
        c, table = a_cache(2, 128, 32, kv_len, news, rng)
        fill(c, rng, kv_len, table)
        q = rows(rng, (4, 4, 128), torch.float32)
        made.append((c, q, c.attend(q)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    outs = [[], []]
    for _ in range(20):
        for i, (c, q, _) in enumerate(made):
            outs[i].append(torch.zeros_like(q))
    torch.cuda.synchronize()
    for r in range(20):
        for i, (c, q, _) in enumerate(made):
            c.attend(q, out=outs[i][r], stream=streams[i])
    torch.cuda.synchronize()
    for i, (_, _, want) in enumerate(made):
        assert all(torch.equal(o, want) for o in outs[i])


@gpu
def test_between_the_maps_of_a_block():
    """What it is for: q, k, v as columns of one group's y, attention, the next group's x; over steps, against 64 bits."""
    import synthetic as S
    g = gsi()
    d, heads, dim, n, k = 512, 4, 128, 3, 64
    P = S.store_basis(S.gen_basis(d, k, 91)).cuda()
    qkv = g.Layer([S.gen_weight(d, d, 92 + j).cuda() for j in range(3)], P, 0.0, max_tokens=n)
    out = g.Layer([S.gen_weight(d, d, 95).cuda()], P, 0.0, max_tokens=n)
    c = g.KVCache(heads, dim, 12, n, 64, page_tokens=16, max_tokens=n)
    n_new = ints([1] * n)
    torch.manual_seed(2)
    x = torch.randn(n, d, device="cuda") * 2
    for step in range(20):
        y, _, _ = qkv.forward(x)
        q, key, value = (part.unflatten(1, (heads, dim)) for part in y.split(d, 1))
        c.plan(n_new)
        c.append(key, value)
        a = c.attend(q)
        x, _, _ = out.forward(a.view(n, d))
        x = x / x.norm(dim=1, keepdim=True) * 40
        lens = c.lens.cpu().tolist()
        assert lens == [step + 1] * n
        table = c.table.cpu().numpy()
        slots = [int(table[i, p // 16] * 16 + p % 16) for i in range(n) for p in range(step + 1)]
        check(c, q, a, a, read_back(c, slots), lens, [1] * n, dim ** -0.5)
    codes, s, mid = R.quantise(key.float().cpu().numpy())
    got, _ = c.read(c.slots)
    assert np.array_equal(got.cpu().numpy(), R.values(codes, s, mid))
    assert c.status() == qkv.status() == out.status() == 0


@gpu
def test_a_closed_cache_and_its_calls():
    g = gsi()
    c = g.KVCache(1, 64, 2, 2, 16, page_tokens=16)
    with pytest.raises(g.GsiError):
        c.plan(ints([1, 1, 1]))              # more requests than the cache has room for
    with pytest.raises(AssertionError):
        c.attend(torch.zeros(1, 1, 64))      # on the host
    with pytest.raises(g.GsiError):
        c.attend(torch.zeros(1, 1, 64, device="cuda"), scale=float("inf"))
    assert c.attend(torch.zeros(0, 1, 64, device="cuda")).shape == (0, 1, 64)
    c.append(*(torch.zeros(0, 1, 64, device="cuda"),) * 2)
    assert c.read(ints([]))[0].shape == (0, 1, 64)
    c.close()
    with pytest.raises(g.GsiError):
        c.plan(ints([1]))


def attend_of(c, q, n_seqs):
    """The library's call with a number of requests of its own."""
    from paper_2605_03109_b200 import binding
    g, out = gsi(), torch.full_like(q, 9.0)
    status = g.lib.gsi_kv_attend(c.handle, q.data_ptr(), {torch.float32: g.GSI_F32, torch.bfloat16: g.GSI_BF16}[q.dtype], q.stride(0), q.stride(1),
                                 q.shape[0], q.shape[1], c.head_dim ** -0.5, c.q_start.data_ptr(), c.kv_len.data_ptr(), c.table.data_ptr(), n_seqs,
                                 c.pages.data_ptr(), out.data_ptr(), out.stride(0), out.stride(1), binding._stream_ptr(None))
    assert status == 0
    return out


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_few_requests_and_many_are_shared_out_alike(dtype):
    """Up to 32 requests a warp shares out by itself, more the block: empty ones behind them change nothing, call after call."""
    rng = np.random.default_rng(31)
    kv_len, news = [900, 17, 300, 1] + [0] * 36, [1, 1, 1, 1] + [0] * 36
    c, table = a_cache(2, 128, 16, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    q = rows(rng, (6, 2, 128), dtype)
    want = attend_of(c, q, 40)
    check(c, q, want, torch.full_like(q, 9.0), kv, kv_len, news, 128 ** -0.5)
    for _ in range(20):
        for n in (4, 32, 33):
            assert torch.equal(attend_of(c, q, n), want)


def put(c, k, v, kv_len, table):
    slots = slots_of(c, kv_len, table)
    c.pages.fill_(0xFF)
    c.append(k, v, slots=torch.from_numpy(slots).cuda())
    return read_back(c, slots)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** -20])
@pytest.mark.parametrize("dim,shared", [(128, 1), (128, 5), (256, 2)])
def test_blocks_of_one_head_whose_values_differ_in_size(dtype, size, dim, shared):
    """The block beside does not take bits away: each is within the bound of its own size."""
    rng = np.random.default_rng(41)
    kv_len, news = [150, 33], [1, 2]
    c, table = a_cache(1, dim, 16, kv_len, news, rng)
    k, v = (torch.from_numpy(rng.standard_normal((183, 1, dim)).astype(np.float32)).cuda() for _ in range(2))
    v[..., 64:] *= size                              # (2^-20: steps that are subnormal in f16; 2^20: past its range)
    kv = put(c, k, (v / 64 if size == 2.0 ** 20 else v), kv_len, table)
    q = rows(rng, (3, shared, dim), dtype)
    out = c.attend(q)
    if dtype == torch.float16:                       # (values that fp16 does not hold are compared as they are held)
        out = out.clamp(-65504, 65504)
    check(c, q, out, out, kv, kv_len, news, dim ** -0.5)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("small,large", [(1.0, 3e4), (1e-3, 1e4), (1e-5, 1e2)])
def test_a_token_that_is_not_seen_yet_takes_no_bits_away(dtype, small, large):
    """Rows of a chunk beside a later token whose values are larger by far: the numbers of a call without that token's size."""
    rng = np.random.default_rng(42)
    kv_len, news = [70], [9]
    c, table = a_cache(1, 128, 16, kv_len, news, rng)
    k, v = (torch.from_numpy(rng.standard_normal((70, 1, 128)).astype(np.float32)).cuda() for _ in range(2))
    v *= small
    put(c, k, v, kv_len, table)
    q = rows(rng, (9, 2, 128), dtype)
    plain = c.attend(q)
    v[69] *= large / small
    kv = put(c, k, v, kv_len, table)
    out = c.attend(q)
    check(c, q, out, out, kv, kv_len, news, 128 ** -0.5)
    assert torch.equal(out[:8], plain[:8])


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at", [0, 40, 99, 199])
def test_a_large_value_with_a_small_probability(dtype, at):
    """A token of a score far below the others' and of values far above them, seen first, in between and last."""
    rng = np.random.default_rng(43 + at)
    c, table = a_cache(1, 64, 16, [200], [1], rng)
    k, v = (torch.from_numpy(rng.standard_normal((200, 1, 64)).astype(np.float32)).cuda() * w for w in (0.3, 3e-5))
    k[:, 0, 5] = 0.0
    k[at], v[at] = -40.0, v[at] * 3e8
    kv = put(c, k, v, [200], table)
    q = torch.zeros(1, 3, 64, dtype=dtype, device="cuda")
    q[0, :, 5] = torch.tensor([1.0, 0.75, -0.125])   # e^-40, e^-30, and one that sees it as the largest of all
    out = c.attend(q, scale=1.0)
    check(c, q, out, out, kv, [200], [1], 1.0)


@gpu
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("shared,new", [(1, 1), (2, 1), (4, 1), (5, 5)])
def test_probabilities_of_fp16_rows_have_22_bits(dim, shared, new):
    """11 bits would show beside the outputs' own 11: within the bound of fp32 rows.  (Scores are small, so that their share of
    the bound is; few tokens, so that roundings do not cancel.)"""
    dtype = torch.float16
    rng = np.random.default_rng(dim + shared)
    kv_len, news, scale = [new, new + 1, 11, 40], [new] * 4, 1e-3
    c, table = a_cache(1, dim, 16, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    q = rows(rng, (4 * new, shared, dim), dtype)
    qn, got, half = q.float().cpu().numpy(), c.attend(q, scale=scale).double().cpu().numpy(), torch.finfo(dtype).eps / 2
    first = 0
    for i, n in enumerate(kv_len):
        for m in range(new):
            for h in range(shared):
                have = [[x[first:first + n - new + m + 1, 0] for x in t] for t in kv]
                want, off = R.attend(qn[i * new + m, h], *have, scale, False)
                tol = off + half * np.abs(want) + 3e-8   # (half of f16's smallest step)
                assert (np.abs(got[i * new + m, h] - want) <= tol).all(), (i, m, h)
        first += n


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,heads,seqs,new,length", [(64, 128, 3, 1, 160007), (128, 16, 3, 1, 160007), (64, 32, 2, 4, 120011), (256, 16, 4, 1, 100003), (64, 16, 2, 16, 60001)])
def test_hundreds_of_sets_of_tiles_a_warp(dtype, dim, heads, seqs, new, length):
    """Long requests (their tables name the same pages again and again): sums are handed over many times, of every type of row."""
    rng = np.random.default_rng(dim + new)
    g, page, n_pages = gsi(), 64, 37
    c = g.KVCache(heads, dim, n_pages, seqs, length, page_tokens=page, max_tokens=seqs * new)
    fill(c, rng, [n_pages * page], np.arange(n_pages)[None])
    lens, news = [length - 1000 * i for i in range(seqs)], [new] * seqs
    table = rng.integers(0, n_pages, tuple(c.table.shape))
    c.table.copy_(torch.from_numpy(table))
    c.kv_len.copy_(ints(lens))
    c.q_start.copy_(ints([new * i for i in range(seqs + 1)]))
    q = rows(rng, (seqs * new, heads, dim), dtype)
    out = c.attend(q)
    assert torch.equal(c.attend(q), out) and c.status() == 0
    qn, got, half = q.float().cpu().numpy(), out.double().cpu().numpy(), torch.finfo(dtype).eps / 2
    pool = c.pages.view(-1).cpu().numpy()
    tiles = sum(-(-n // 16) for n in lens) * heads * -(-new // 4)       # (of a set or less each; at least four rows a unit but for single ones)
    sets, parts = -(-tiles // (148 * 12)) + 8, -(-2400 // (seqs * heads)) + 2
    for i, h in ((0, 0), (seqs - 1, heads - 1), (seqs // 2, heads // 3)):
        k, v = R.decode(pool, (heads, dim, page), slots_of(c, [lens[i]], table[i:i + 1]), [h])
        for m in sorted({0, new - 1}):
            sees = lens[i] - new + m + 1
            want, off = R.attend_of_long_shares(qn[i * new + m, h], *[[y[:sees, 0] for y in z] for z in (k, v)], dim ** -0.5, dtype != torch.float32, sets, parts)
            tol = off + half * np.abs(want) + (3e-8 if dtype == torch.float16 else 0)
            assert (np.abs(got[i * new + m, h] - want) <= tol).all(), (i, h, m, float((np.abs(got[i * new + m, h] - want) / tol).max()))


def planned(c, lens):
    """Tokens in an empty cache for requests of `lens`."""
    c.plan(ints(lens))
    k, v = (torch.randn(sum(lens), c.n_heads, c.head_dim, device="cuda") for _ in range(2))
    c.append(k, v)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_an_attention_goes_by_the_plan_that_ran_last(dtype):
    """Plans of eight requests and of four, captured and not, before an attention that was captured behind the other."""
    g, rng = gsi(), np.random.default_rng(51)
    lens = [40, 3, 100, 17, 5, 64, 1, 30]
    for captured, last in (([1] * 8, [3, 1, 1, 1]), ([3, 1, 1, 1], [1] * 8), ([2, 0, 1], [1] * 8)):
        c = g.KVCache(2, 64, 64, 8, 200, page_tokens=16, max_tokens=300)
        planned(c, lens)
        q = rows(rng, (10, 4, 64), dtype)
        out = torch.full_like(q, 9.0)
        first, then = ints(captured), ints(last)

        def expect():
            """From the tensors alone."""
            starts, kv_len, table = c.q_start.cpu().tolist(), c.kv_len.cpu().tolist(), c.table.cpu().numpy().astype(np.int64)
            news = [b - a for a, b in zip(starts, starts[1:])]
            return read_back(c, slots_of(c, kv_len, table)), kv_len, news

        c.plan(first)
        c.append(*(torch.randn(sum(captured), 2, 64, device="cuda") for _ in range(2)))
        c.attend(q, out=out)
        torch.cuda.synchronize()
        plan_graph, attend_graph = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(plan_graph):
            c.plan(first, commit=False)
        with torch.cuda.graph(attend_graph):
            c.attend(q, out=out)
        for replay in (False, True):         # eager, and replayed attention behind an eager plan of another number
            c.plan(then, commit=False)
            assert c.q_start.cpu().tolist()[len(last):] == [sum(last)] * (9 - len(last)) and not c.kv_len[len(last):].any()
            new = torch.randn(sum(last), 2, 64, device="cuda")
            c.append(new, new)
            out.fill_(9.0)
            attend_graph.replay() if replay else c.attend(q, out=out)
            check(c, q, out, torch.full_like(q, 9.0), *expect(), 0.125)
            # ... and an eager one behind the replayed plan
            plan_graph.replay()
            assert c.counts.cpu().tolist()[0] == sum(captured)
            new = torch.randn(sum(captured), 2, 64, device="cuda")
            c.append(new, new)
            out.fill_(9.0)
            attend_graph.replay() if replay else c.attend(q, out=out)
            check(c, q, out, torch.full_like(q, 9.0), *expect(), 0.125)
        assert c.status() == 0


@gpu
def test_a_plan_of_the_library_writes_what_it_is_asked_for():
    """Without GSI_KV_ALL_SEQS: nothing behind its own requests; flags that there are not are refused."""
    from paper_2605_03109_b200 import binding
    g = gsi()
    c = g.KVCache(1, 64, 16, 6, 64, page_tokens=16, max_tokens=8)
    n_new = ints([2, 1, 3])

    def plan(commit):
        return g.lib.gsi_kv_plan(c.handle, n_new.data_ptr(), 3, commit, c.lens.data_ptr(), c.n_free.data_ptr(), c.free.data_ptr(), c.table.data_ptr(),
                                 c.q_start.data_ptr(), c.kv_len.data_ptr(), c.slots.data_ptr(), c.positions.data_ptr(), c.counts.data_ptr(),
                                 binding._stream_ptr(None))

    for commit, behind in ((0, False), (1, False), (2, True), (3, True)):
        c.q_start.fill_(77)
        c.kv_len.fill_(77)
        before = c.lens.clone()
        assert plan(commit) == 0
        assert c.q_start.cpu().tolist() == [0, 2, 3, 6] + [6 if behind else 77] * 3
        assert c.kv_len.cpu().tolist()[:3] == (before[:3] + n_new).cpu().tolist() and c.kv_len.cpu().tolist()[3:] == [0 if behind else 77] * 3
        assert torch.equal(c.lens - before, torch.cat([n_new, ints([0] * 3)]) * (commit & 1))
    assert plan(4) == plan(-1) == 1


@gpu
def test_outputs_are_of_the_memory_of_the_stream_that_writes_them():
    """Memory that the current stream has given back may still be in use there; an output's own goes back when both streams are done with it."""
    rng = np.random.default_rng(61)
    kv_len, news = [900, 17], [40, 8]
    c, table = a_cache(2, 128, 16, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    q = rows(rng, (48, 4, 128), torch.float32)
    want = c.attend(q)
    check(c, q, want, want, kv, kv_len, news, 128 ** -0.5)
    slots = torch.from_numpy(slots_of(c, kv_len, table)[:48]).cuda()
    values = c.read(slots)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for call, given in ((lambda s: [c.attend(q, stream=s)], want), (lambda s: c.read(slots, stream=s), values[0])):
        for stream in (side, side.cuda_stream):
            old = [torch.full_like(given, 3.0) for _ in range(8)]
            places = {x.data_ptr() for x in old}
            torch.cuda._sleep(20_000_000)                 # (some 10 ms)
            sums = [x.sum() for x in old]
            del old
            got = call(stream)
            assert not places & {x.data_ptr() for x in got}
            side.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, [want] if len(got) == 1 else values))
            assert all(x.item() == 3.0 * given.numel() for x in sums)
            # used by the current stream, given back, asked for again
            places = {x.data_ptr() for x in got}
            torch.cuda._sleep(20_000_000)
            sums = [x.double().sum() for x in got]
            del got
            again = call(stream)
            assert not places & {x.data_ptr() for x in again}
            torch.cuda.synchronize()
            assert [x.item() for x in sums] == [x.double().sum().item() for x in again]
    assert c.status() == 0


@gpu
def test_a_cache_made_on_another_stream_is_ready_there():
    g, side = gsi(), torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        torch.cuda._sleep(100_000_000)                    # the current stream is busy (some 50 ms)
        c = g.KVCache(2, 64, 8, 2, 64, page_tokens=16, max_tokens=40, stream=stream)
        with torch.cuda.stream(side):
            n_new = ints([33, 7])
            q, k, v = (torch.randn(40, 2, 64, device="cuda") for _ in range(3))
            c.plan(n_new)
            c.append(k, v)
            out = c.attend(q)
        side.synchronize()
        lens = [33, 7]
        check(c, q, out, out, read_back(c, slots_of(c, lens, c.table.cpu().numpy().astype(np.int64))), lens, lens, 0.125)
        assert c.counts.cpu().tolist() == [40, 4, 4, 0] and c.status() == 0


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_without_a_request_are_zeros_in_a_new_tensor(dtype):
    """Padded batches, requests that pause: no memory that was never written reaches the next map."""
    rng = np.random.default_rng(71)
    kv_len, news = [30, 0, 7], [2, 0, 1]
    c, table = a_cache(2, 64, 16, kv_len, news, rng)
    kv = fill_and_read(c, rng, kv_len, table)
    q = rows(rng, (8, 4, 64), dtype)
    side = torch.cuda.Stream()
    for stream in (None, side):
        with torch.cuda.stream(stream):
            for _ in range(3):
                old = [torch.full_like(q, float("nan")) for _ in range(4)]
                del old
                out = c.attend(q, stream=stream)
        torch.cuda.synchronize()
        check(c, q, out, torch.zeros_like(out), kv, kv_len, news, 0.125)
        assert not out[3:].any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.attend(q)
    for _ in range(2):
        out.fill_(float("nan"))
        graph.replay()
        check(c, q, out, torch.zeros_like(out), kv, kv_len, news, 0.125)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,shared,dim,page,kv_len,news", [
    (2, 1, 64, 64, [300], [300]),                                # a whole prompt
    (1, 4, 128, 16, [257, 130, 33], [257, 1, 33]),               # prompts beside a request that goes on
    (2, 2, 80, 48, [700, 256, 20], [256, 255, 20]),              # chunks, odd ones
    (1, 1, 256, 64, [1000, 64], [128, 64]),
    (1, 3, 192, 32, [129, 400], [129, 61]),
])
def test_chunks_and_whole_prompts(dtype, heads, shared, dim, page, kv_len, news):
    """Many new rows of a request: each against the tokens up to its own, through plan and append as well."""
    rng = np.random.default_rng(dim + len(kv_len))
    g, seqs = gsi(), len(kv_len)
    c = g.KVCache(heads, dim, sum(-(-n // page) for n in kv_len) + 3, seqs, max(kv_len), page_tokens=page, max_tokens=sum(kv_len))
    c.pages.fill_(0xFF)
    make = lambda n: (rows(rng, (n, heads, dim), torch.float32, 1.5), rows(rng, (n, heads, dim), torch.float32) + 0.1)  # noqa: E731
    old = [n - m for n, m in zip(kv_len, news)]
    if any(old):
        c.plan(ints(old))
        c.append(*make(sum(old)))
    c.plan(ints(news))
    c.append(*make(sum(news)))
    q = rows(rng, (sum(news) + 1, heads * shared, dim), dtype, 1.3)
    out = torch.full_like(q, 9.0)
    c.attend(q, out=out)
    assert (out[-1] == 9).all() and c.status() == 0 and c.kv_len.cpu().tolist() == kv_len
    kv = read_back(c, slots_of(c, kv_len, c.table.cpu().numpy().astype(np.int64)))
    qn, got, half = q.float().cpu().numpy(), out.double().cpu().numpy(), torch.finfo(dtype).eps / 2
    first, row = np.concatenate([[0], np.cumsum(kv_len)]), np.concatenate([[0], np.cumsum(news)])
    for i in range(seqs):
        some = set(range(0, news[i], 13)) | {1, 7, 8, 15, 16, 17, 31, 32, 63, 64, news[i] - 2, news[i] - 1}
        for m in sorted(x for x in some if 0 <= x < news[i]):
            sees = old[i] + m + 1
            for h in sorted({m % (heads * shared), heads * shared - 1}):
                have = [[x[first[i]:first[i] + sees, h // shared] for x in t] for t in kv]
                want, off = R.attend(qn[row[i] + m, h], *have, dim ** -0.5, dtype != torch.float32)
                tol = off + half * np.abs(want) + (3e-8 if dtype == torch.float16 else 0)
                assert (np.abs(got[row[i] + m, h] - want) <= tol).all(), (i, m, h, float((np.abs(got[row[i] + m, h] - want) / tol).max()))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_bad_page_of_a_prompt_is_that_of_the_rows_that_see_it(dtype):
    rng = np.random.default_rng(91)
    c, table = a_cache(2, 64, 16, [100, 40], [100, 1], rng)
    fill(c, rng, [100, 40], table)
    q = rows(rng, (101, 2, 64), dtype)
    clean = c.attend(q)
    assert c.status() == 0 and clean.isfinite().all()
    c.table[0, 3] = -1                      # tokens 48 .. 63
    out = c.attend(q)
    assert torch.equal(out[:48], clean[:48]) and out[48:100].isnan().all() and torch.equal(out[100], clean[100])
    assert c.status() == 1
