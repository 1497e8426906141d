"""ls_cache_write, ls_cache_read and ls_paged_attend: stored bits, the way back, attention over pages in 64 bits, and what is left out."""
import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(p):
    return binding.PagedCache(**{n: x.cuda() for n, x in p.items()})


def _host(cache):
    return {n: getattr(cache, n).cpu() for n in ("k", "v", "k_exp", "v_exp") if getattr(cache, n) is not None}


def _places(lens, pos, table, page):
    """Of each row in order: sequence, index in it, page, place in the page."""
    return [(s, i, int(table[s, (pos[s] + i) // page]), (pos[s] + i) % page) for s, n in enumerate(lens) for i in range(n)]


def _written(p, kind, rows, places, name):
    """The pages after `rows` [N,Hkv,d] went to their places."""
    at = torch.tensor([x[2] for x in places]), torch.tensor([x[3] for x in places])
    if kind == "bf16":
        p[name][at[0], :, at[1]] = rows.to(torch.bfloat16)
    else:
        E = pu.exponents(rows)
        p[name + "_exp"][at[0], :, at[1]] = E
        p[name][at[0], :, at[1]] = pu.codes(rows, E)


def _same(a, b):
    return all(torch.equal(a[n].view(torch.uint8) if n in ("k", "v") else a[n], b[n].view(torch.uint8) if n in ("k", "v") else b[n]) for n in b)


MOVES = [
    # lens, pos, Hkv, d, page
    ([1], [0], 1, 64, 16),
    ([1, 1, 1], [15, 16, 0], 3, 128, 16),            # a token each, at a page's last place and at its first
    ([37, 0, 5], [3, 7, 250], 2, 128, 32),
    ([300, 129], [0, 100], 8, 64, 64),
    ([500], [77], 5, 128, 128),
    ([40, 41], [255, 256], 4, 128, 256),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("lens,pos,Hkv,d,page", MOVES)
def test_write_and_read(lens, pos, Hkv, d, page, packed, kind, dtype):
    print("cache move", lens, pos, Hkv, d, page, packed, kind, dtype, flush=True)
    rng = np.random.default_rng(sum(lens) + page)
    ends = [a + n for a, n in zip(pos, lens)]
    pages = sum(-(-e // page) for e in ends) + 2
    p = pu.pool(rng, pages, Hkv, page, d, kind)
    table = pu.table_for(rng, ends, page, pages)
    B, most = len(lens), max(lens)
    rows = [pu.rnd(rng, sum(lens), Hkv, d, scale=s, dtype=dtype) for s in (1.0, 30.0)]
    cache, places = _cache(p), _places(lens, pos, table, page)
    if packed:
        shape = binding.make_shape(B, Hkv, Hkv, d, 1, sum(lens), 1, dtype)
        dev, kw = [x.cuda() for x in rows], dict(starts=_i32(np.concatenate([[0], np.cumsum(lens)])))
    else:
        shape = binding.make_shape(B, Hkv, Hkv, d, 1, most, 1, dtype)
        dev, kw = [torch.full((B, Hkv, most, d), float("nan"), dtype=dtype, device="cuda") for _ in rows], dict(count=_i32(lens))
        for x, y in zip(rows, dev):
            for r, (s, i, _, _) in enumerate(places):
                y[s, :, i] = x[r].cuda()
    ctx = binding.Context(workspace=0)
    ctx.ls_cache_write(shape, cache, dev[0], dev[1], table.cuda(), _i32(pos), **kw)
    assert ctx.ls_poll_status() == 0
    want = {n: x.clone() for n, x in p.items()}
    for name, x in zip(("k", "v"), rows):
        _written(want, kind, x, places, name)
    assert _same(_host(cache), want)
    back = [torch.full_like(x, 7.0) for x in dev]
    ctx.ls_cache_read(shape, cache, table.cuda(), back[0], back[1], _i32(pos), **kw)
    assert ctx.ls_poll_status() == 0
    for name, got in zip(("k", "v"), back):
        ref = torch.full_like(got.cpu(), 7.0)
        for r, (s, i, pg, pl) in enumerate(places):
            x = pu.stored(want, name)[pg, :, pl].to(dtype)
            if packed:
                ref[r] = x
            else:
                ref[s, :, i] = x
        assert torch.equal(got.cpu(), ref)


def test_rounding_of_every_kind_of_value():
    """Halfway cases, the smallest and largest numbers, zeros of both signs, infinities and NaN."""
    d = 64
    base = torch.cat([torch.tensor([0.0, -0.0, 1.0625, 1.1875, -1.0625, 448.0, -448.0, 464.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 1.5 * 2.0 ** -9]),
                      torch.linspace(-3, 3, d - 12)])
    rows = torch.stack([base * f for f in (1.0, 2.0 ** -20, 2.0 ** 100, 2.0 ** -118, 2.0 ** -126, 1e-45, 0.0, 0.77)]).clone()
    odd = rows[:4].clone()
    odd[0, 3], odd[1, 5], odd[2, 7], odd[3, :] = float("inf"), -float("inf"), float("nan"), float("nan")
    rows = torch.cat([rows, odd])[:, None]                    # [12,1,d]
    E = pu.exponents(rows)
    assert int(E.min()) == 10 and int(E.max()) > 200
    p = dict(k=torch.zeros(1, 1, 16, d, dtype=torch.uint8), v=torch.zeros(1, 1, 16, d, dtype=torch.uint8),
             k_exp=torch.zeros(1, 1, 16, dtype=torch.uint8), v_exp=torch.zeros(1, 1, 16, dtype=torch.uint8))
    cache = _cache(p)
    shape = binding.make_shape(1, 1, 1, d, 1, 12, 1, "f32")
    ctx = binding.Context(workspace=0)
    print("cache rounding", flush=True)
    ctx.ls_cache_write(shape, cache, rows.cuda(), rows.cuda(), _i32([[0]]), starts=_i32([0, 12]))
    torch.cuda.synchronize()
    got = _host(cache)
    assert torch.equal(got["k_exp"][0, 0, :12], E[:, 0]) and torch.equal(got["k"], got["v"])
    want, have = pu.codes(rows, E)[:, 0], got["k"][0, 0, :12]
    nan = (want & 0x7F) == 0x7F
    assert torch.equal((have & 0x7F) == 0x7F, nan) and torch.equal(have[~nan], want[~nan])
    finite = torch.isfinite(rows[:, 0])
    back = pu.values(have, E[:, 0])
    err = (back[finite].double() - rows[:, 0][finite].double()).abs()
    scale = torch.ldexp(torch.ones(1, dtype=torch.float64), E.int() - 127)[:, :1].expand(-1, d)[finite]
    assert (err <= torch.maximum(rows[:, 0][finite].double().abs() * 2.0 ** -4, scale * 2.0 ** -10)).all()


def test_strided_rows():
    """Rows as slices of one projection, and head by head with gaps; read into rows of other strides."""
    rng = np.random.default_rng(1)
    T, Hkv, d, page = 70, 2, 128, 16
    x = pu.rnd(rng, T, 3 * Hkv * d).cuda()
    k, v = x[:, Hkv * d:2 * Hkv * d].unflatten(1, (Hkv, d)), x[:, 2 * Hkv * d:].unflatten(1, (Hkv, d))
    p = pu.pool(rng, 8, Hkv, page, d, "bf16")
    cache, table = _cache(p), pu.table_for(rng, [T], page, 8)
    shape = binding.make_shape(1, Hkv, Hkv, d, 1, T, 1, "bf16")
    ctx = binding.Context(workspace=0)
    print("cache strides", flush=True)
    ctx.ls_cache_write(shape, cache, k, v, table.cuda(), starts=_i32([0, T]))
    whole = torch.full((2, Hkv + 1, T + 3, d), 9.0, dtype=torch.bfloat16, device="cuda")
    kr, vr = (whole[i, 1:, 2:-1].transpose(0, 1) for i in (0, 1))
    ctx.ls_cache_read(shape, cache, table.cuda(), kr, vr, starts=_i32([0, T]))
    torch.cuda.synchronize()
    assert torch.equal(kr, k) and torch.equal(vr, v)
    whole[:, 1:, 2:-1] = 9.0
    assert (whole == 9.0).all()


def test_positions_that_are_nowhere():
    """A page number outside the pool, a place beyond the table, a negative position: those rows are left out, the others are not, and the status word says so."""
    rng = np.random.default_rng(2)
    Hkv, d, page = 2, 64, 16
    p = pu.pool(rng, 3, Hkv, page, d, "bf16")
    table = torch.tensor([[0, 3, 1], [2, -1, -5]], dtype=torch.int32)
    rows = pu.rnd(rng, 2, Hkv, 60, d)
    shape = binding.make_shape(2, Hkv, Hkv, d, 1, 60, 1, "bf16")
    cache, ctx = _cache(p), binding.Context(workspace=0)
    pos = [-4, 5]
    print("cache nowhere", flush=True)
    ctx.ls_cache_write(shape, cache, rows.cuda(), rows.cuda(), table.cuda(), _i32(pos))
    assert ctx.ls_poll_status() == binding.LS_STAT_PAGE_RANGE
    want = {n: x.clone() for n, x in p.items()}
    back = torch.full((2, Hkv, 60, d), 3.0, dtype=torch.bfloat16)
    for s in range(2):
        for i in range(60):
            q = pos[s] + i
            pg = int(table[s, q // page]) if 0 <= q < 48 else -1
            if 0 <= pg < 3:
                want["k"][pg, :, q % page] = want["v"][pg, :, q % page] = rows[s, :, i]
                back[s, :, i] = rows[s, :, i]
    assert _same(_host(cache), want)
    got = [torch.full((2, Hkv, 60, d), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx.ls_cache_read(shape, cache, table.cuda(), got[0], got[1], _i32(pos))
    assert ctx.ls_poll_status() == binding.LS_STAT_PAGE_RANGE
    assert torch.equal(got[0].cpu(), back) and torch.equal(got[1].cpu(), back)


def test_starts_and_counts_out_of_range():
    rng = np.random.default_rng(3)
    p = pu.pool(rng, 4, 1, 16, 64, "bf16")
    rows = pu.rnd(rng, 30, 1, 64)
    shape = binding.make_shape(3, 1, 1, 64, 1, 30, 1, "bf16")
    cache, ctx = _cache(p), binding.Context(workspace=0)
    table = _i32([[0], [1], [2]])
    print("cache starts", flush=True)
    ctx.ls_cache_write(shape, cache, rows.cuda(), rows.cuda(), table, starts=_i32([0, 10, 5, 9]))
    assert ctx.ls_poll_status() == binding.LS_STAT_STARTS
    want = {n: x.clone() for n, x in p.items()}
    want["k"][0, 0, :10] = want["v"][0, 0, :10] = rows[:10, 0]
    assert _same(_host(cache), want)
    padded = pu.rnd(rng, 3, 1, 4, 64)
    ctx.ls_cache_write(binding.make_shape(3, 1, 1, 64, 1, 4, 1, "bf16"), cache, padded.cuda(), padded.cuda(), table, count=_i32([-7, 2, 99]))
    assert ctx.ls_poll_status() == 0
    want["k"][1, 0, :2] = want["v"][1, 0, :2] = padded[1, 0, :2]
    want["k"][2, 0, :4] = want["v"][2, 0, :4] = padded[2, 0]
    assert _same(_host(cache), want)


def test_many_sequences():
    """More sequences than a workgroup has threads, most of them without rows."""
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.choice([0, 0, 1, 3], 700)]
    B, T = len(lens), sum(lens)
    p = pu.pool(rng, B, 1, 16, 64, "e4m3")
    table = torch.from_numpy(rng.permutation(B).astype(np.int32))[:, None].contiguous()
    pos = [int(x) for x in rng.integers(0, 13, B)]
    rows = pu.rnd(rng, T, 1, 64)
    shape = binding.make_shape(B, 1, 1, 64, 1, T, 1, "bf16")
    cache, ctx = _cache(p), binding.Context(workspace=0)
    print("cache 700 sequences", flush=True)
    ctx.ls_cache_write(shape, cache, rows.cuda(), rows.cuda(), table.cuda(), _i32(pos), starts=_i32(np.concatenate([[0], np.cumsum(lens)])))
    want = {n: x.clone() for n, x in p.items()}
    for name in ("k", "v"):
        _written(want, "e4m3", rows, _places(lens, pos, table, 16), name)
    torch.cuda.synchronize()
    assert _same(_host(cache), want)


# ---- ls_paged_attend

def _attend(p, q, table, lens, n=None, lse=True, poison=0x7FC00000, times=1, scale=0.0):
    B, Hq, d = q.shape
    cache = _cache(p)
    shape = binding.make_shape(B, Hq, cache.k.shape[1], d, n or max(1, max(lens)), 1, 1, "bf16", scale)
    ctx = binding.Context(workspace=binding.paged_workspace_bytes(shape))
    ctx.debug_fill_workspace(poison)
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    ls = torch.full((B, Hq), float("nan"), device="cuda") if lse else None
    for _ in range(times):
        ctx.ls_paged_attend(shape, cache, q.cuda(), table.cuda(), _i32(lens), out, ls)
    torch.cuda.synchronize()
    return out.cpu(), None if ls is None else ls.cpu(), ctx.ls_poll_status()


def _check(p, q, table, lens, out, lse, scale=None):
    B, Hq, d = q.shape
    K, V = pu.stored(p, "k"), pu.stored(p, "v")
    Hkv, page = K.shape[1], K.shape[2]
    G = Hq // Hkv
    for b, n in enumerate(lens):
        at = [(int(table[b, i // page]), i % page) for i in range(n)]
        keep = [i for i, (pg, _) in enumerate(at) if 0 <= pg < K.shape[0]]
        pg, pl = torch.tensor([at[i][0] for i in keep], dtype=torch.long), torch.tensor([at[i][1] for i in keep], dtype=torch.long)
        for j in range(Hkv):
            ref = pu.attention(q[b, j * G:(j + 1) * G], K[pg, j, pl], V[pg, j, pl], np.full(G, len(keep)), scale or d ** -0.5)
            pu.check(out[b, j * G:(j + 1) * G], None if lse is None else lse[b, j * G:(j + 1) * G], ref, torch.bfloat16)


TOKENS = [
    # lens, Hq, Hkv, d, page
    ([1], 4, 1, 64, 16),
    ([15, 16, 17, 31, 32, 33], 8, 2, 128, 16),       # either side of pages and tiles
    ([0, 100, 0, 1], 8, 8, 128, 32),                 # empty ones among others
    ([519, 2000], 32, 8, 128, 16),                   # one workgroup a head, and parts
    ([5003], 32, 1, 64, 64),                         # 32 query heads, many parts of few heads
    ([5003], 17, 1, 128, 256),
    ([3000, 7, 1200], 12, 3, 128, 128),
    ([40000], 4, 1, 64, 32),                         # a wave's page list is renewed
]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,Hq,Hkv,d,page", TOKENS)
def test_attend_matches(lens, Hq, Hkv, d, page, kind):
    print("paged", lens, Hq, Hkv, d, page, kind, flush=True)
    rng = np.random.default_rng(len(lens) + Hq)
    pages = sum(-(-n // page) for n in lens) + 2
    p = pu.pool(rng, pages, Hkv, page, d, kind)
    q = pu.rnd(rng, len(lens), Hq, d, scale=1.5)
    table = pu.table_for(rng, lens, page, pages)
    out, lse, status = _attend(p, q, table, lens, times=3)
    assert status == 0
    _check(p, q, table, lens, out, lse)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_more_than_64_sequences(kind):
    rng = np.random.default_rng(8)
    lens = [int(x) for x in rng.integers(0, 90, 130)] + [3000]
    p = pu.pool(rng, sum(-(-n // 16) for n in lens), 2, 16, 64, kind)
    q, table = pu.rnd(rng, len(lens), 4, 64), pu.table_for(rng, lens, 16, p["k"].shape[0])
    print("paged 131 sequences", kind, flush=True)
    out, lse, status = _attend(p, q, table, lens)
    assert status == 0
    _check(p, q, table, lens, out, lse)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_what_lies_behind_the_length_does_not_matter(kind):
    """NaN values, codes and exponents behind the last position of a page, and table entries that are no pages."""
    rng = np.random.default_rng(9)
    lens = [5, 50, 100]
    p = pu.pool(rng, 12, 2, 32, 128, kind)
    table = pu.table_for(rng, lens, 32, 12, width=7)
    clean = {n: x.clone() for n, x in p.items()}
    for b, n in enumerate(lens):
        pg, pl = int(table[b, (n - 1) // 32]), (n - 1) % 32 + 1
        for name in ("k", "v"):
            if kind == "bf16":
                p[name][pg, :, pl:] = float("nan")
            else:
                p[name][pg, :, pl:], p[name + "_exp"][pg, :, pl:] = 0x7F, 255
    q = pu.rnd(rng, 3, 8, 128)
    print("paged poison", kind, flush=True)
    out, lse, status = _attend(p, q, table, lens, n=7 * 32)
    assert status == 0
    _check(clean, q, table, lens, out, lse)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pages_that_are_nowhere(kind):
    """Keys of pages outside the pool are not seen; a sequence that has none but those is empty; lengths beyond the table are clamped."""
    rng = np.random.default_rng(10)
    p = pu.pool(rng, 6, 2, 16, 64, kind)
    table = torch.tensor([[0, 6, 1, -1], [-1, -2, 99, 7], [2, 3, 4, 5], [6, 6, 6, 2]], dtype=torch.int32)
    q = pu.rnd(rng, 4, 4, 64)
    print("paged nowhere", kind, flush=True)
    out, lse, status = _attend(p, q, table, [50, 64, 64, 60], n=64)
    assert status == binding.LS_STAT_PAGE_RANGE
    _check(p, q, table, [50, 64, 64, 60], out, lse)
    out, lse, status = _attend(p, q[:1], table[2:3], [1000], n=5000)
    assert status == binding.LS_STAT_PAGE_RANGE
    _check(p, q[:1], table[2:3], [64], out, lse)
    out, lse, status = _attend(p, q[:1], table[2:3], [-3], n=64)
    assert status == 0 and (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,Hq,Hkv,d,first,last", [
    ([70, 70], 8, 2, 128, 40, 41),                   # one workgroup a head
    ([70, 70], 8, 2, 64, 0, 70),                     # no other key
    ([5003], 32, 1, 64, 100, 101),                   # parts, put together by a launch of their own
    ([5003], 32, 1, 64, 0, 3000),                    # parts that have no other key
    ([2000, 2000], 4, 2, 128, 1999, 2000),           # parts, put together by the last of them
    ([2000, 2000], 4, 2, 128, 0, 1500)])
def test_no_number_that_is_seen_stays_none(lens, Hq, Hkv, d, first, last, kind):
    """NaN keys first .. last - 1 in head 0 of sequence 0: so are its heads' results; all others have the same bits as with numbers there."""
    print("paged NaN", lens, Hq, Hkv, d, first, last, kind, flush=True)
    rng = np.random.default_rng(17)
    pages = sum(-(-n // 16) for n in lens)
    p = pu.pool(rng, pages, Hkv, 16, d, kind)
    q, table = pu.rnd(rng, len(lens), Hq, d), pu.table_for(rng, lens, 16, pages)
    out, lse, _ = _attend(p, q, table, lens)
    at = torch.arange(first, last)
    p["k"][table[0, at // 16].long(), 0, at % 16] = float("nan") if kind == "bf16" else 0x7F
    got, got_lse, status = _attend(p, q, table, lens, times=2)
    assert status == 0
    hit = torch.zeros(out.shape[:2], dtype=torch.bool)
    hit[0, :Hq // Hkv] = True
    assert torch.isnan(got[hit]).all() and torch.isnan(got_lse[hit]).all()
    assert torch.equal(got[~hit], out[~hit]) and torch.equal(got_lse[~hit], lse[~hit])


def test_shared_pages_no_lse_and_scale():
    """Two sequences with the same first pages, and no normaliser asked for."""
    rng = np.random.default_rng(11)
    p = pu.pool(rng, 6, 2, 16, 128, "e4m3")
    table = torch.tensor([[0, 1, 2], [0, 1, 5]], dtype=torch.int32)
    q = pu.rnd(rng, 2, 4, 128)
    print("paged shared", flush=True)
    out, _, status = _attend(p, q, table, [40, 48], lse=False, scale=0.05)
    assert status == 0
    _check(p, q, table, [40, 48], out, None, scale=float(np.float32(0.05)))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_large_logits(kind):
    rng = np.random.default_rng(12)
    lens = [700]
    p = pu.pool(rng, 44, 2, 16, 128, kind, scale=4.0)
    q, table = pu.rnd(rng, 1, 8, 128, scale=6.0), pu.table_for(rng, lens, 16, 44)
    print("paged large", kind, flush=True)
    out, lse, _ = _attend(p, q, table, lens)
    _check(p, q, table, lens, out, lse)


def test_powers_far_from_one():
    """Rows of V that differ by 2^60 and rows of K of the smallest power."""
    rng = np.random.default_rng(13)
    p = pu.pool(rng, 3, 1, 16, 64, "e4m3")
    p["k_exp"][0], p["v_exp"][0, 0, ::2], p["v_exp"][1] = 10, 187, 60
    q, table = pu.rnd(rng, 1, 2, 64), torch.tensor([[0, 1, 2]], dtype=torch.int32)
    print("paged powers", flush=True)
    out, lse, _ = _attend(p, q, table, [40])
    _check(p, q, table, [40], out, lse)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_more_than_the_chip_holds(kind):
    """Calls on more than 256 MB, whose pages are read past the caches: attention over 73001 keys of 16 heads (the sequences' pages repeat), and rows of nine heads read back."""
    rng = np.random.default_rng(18)
    lens, H, d, page = [70000, 3001], 16, 128, 256
    p = pu.pool(rng, 40, H, page, d, kind)
    q = pu.rnd(rng, 2, H, d, scale=1.5)
    table = torch.from_numpy(rng.integers(0, 40, (2, 274)).astype(np.int32))
    assert sum(lens) * H * 2 * d * (2 if kind == "bf16" else 1) > 256 << 20
    print("paged past the chip", kind, flush=True)
    out, lse, status = _attend(p, q, table, lens, times=2)
    assert status == 0
    K, V = pu.stored(p, "k"), pu.stored(p, "v")
    for b, n in enumerate(lens):
        at = torch.arange(n)
        pg, pl = table[b, at // page].long(), at % page
        for h in (0, 9, 15):
            pu.check(out[b, h:h + 1], lse[b, h:h + 1], pu.attention(q[b, h:h + 1], K[pg, h, pl], V[pg, h, pl], np.full(1, n), d ** -0.5), torch.bfloat16)

    lens, H, n = [36000, 35977], 9, 36000
    p = {name: x[:, :H].contiguous() for name, x in p.items()}
    assert 2 * n * H * 2 * d * (4 if kind == "bf16" else 3) > 256 << 20
    rows = [torch.full((2, H, n, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx = binding.Context(workspace=0)
    print("read past the chip", kind, flush=True)
    ctx.ls_cache_read(binding.make_shape(2, H, H, d, n, n, 1, "bf16"), _cache(p), table.cuda(), *rows, pos=_i32([5, 100]), count=_i32(lens))
    torch.cuda.synchronize()
    assert ctx.ls_poll_status() == 0
    for name, got in zip(("k", "v"), rows):
        held = pu.stored(p, name).to(torch.bfloat16).cuda()
        for b, m in enumerate(lens):
            at = torch.arange(m) + [5, 100][b]
            pg, pl = table[b, at // page].long().cuda(), (at % page).cuda()
            for h in range(H):
                assert torch.equal(got[b, h, :m], held[pg, h, pl])
            assert torch.isnan(got[b, :, m:]).all()


def test_the_last_pages_of_a_large_pool():
    """Pages whose rows lie beyond 2^31 elements and 2^32 bytes of the pool."""
    pages, Hkv, page, d = 70000, 2, 128, 128
    k = torch.zeros(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31 and pages * Hkv * page * d * 2 > 2 ** 32
    cache = binding.PagedCache(k, v)
    rng = np.random.default_rng(14)
    rows = [pu.rnd(rng, 200, Hkv, d) for _ in range(2)]
    table = _i32([[pages - 1, pages - 2]])
    ctx = binding.Context(workspace=1 << 22)
    shape = binding.make_shape(1, 4, Hkv, d, 200, 200, 1, "bf16")
    print("paged large pool", flush=True)
    ctx.ls_cache_write(shape, cache, rows[0].cuda(), rows[1].cuda(), table, starts=_i32([0, 200]))
    q, out, lse = pu.rnd(rng, 1, 4, d), torch.empty(1, 4, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 4, device="cuda")
    ctx.ls_paged_attend(shape, cache, q.cuda(), table, _i32([200]), out, lse)
    torch.cuda.synchronize()
    for j in range(Hkv):
        ref = pu.attention(q[0, 2 * j:2 * j + 2], rows[0][:, j], rows[1][:, j], np.full(2, 200), d ** -0.5)
        pu.check(out[0, 2 * j:2 * j + 2].cpu(), lse[0, 2 * j:2 * j + 2].cpu(), ref, torch.bfloat16)


def test_counters_that_are_off_and_the_other_decode_call():
    """The counters are ls_decode_attend's: calls of both in turn are sound, and calls that found them off spoil two calls at most."""
    rng = np.random.default_rng(15)
    lens = [4000]
    p = pu.pool(rng, 250, 2, 16, 128, "bf16")
    q, table = pu.rnd(rng, 1, 8, 128), pu.table_for(rng, lens, 16, 250)
    cache = _cache(p)
    shape = binding.make_shape(1, 8, 2, 128, 4000, 1, 1, "bf16")
    ctx = binding.Context(workspace=max(binding.paged_workspace_bytes(shape), binding.decode_workspace_bytes(shape, 4000, 0)))
    flat = [x[table[0, :250].long()].transpose(0, 1).reshape(1, 2, -1, 128)[:, :, :4000].contiguous().cuda() for x in (p["k"], p["v"])]
    dq, dt, dl = q.cuda(), table.cuda(), _i32(lens)
    outs = [torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    print("paged counters", flush=True)
    for turn in range(6):
        if turn == 3:
            ctx.debug_set_counters(1)
        for i in range(3):
            for x in outs:
                x.fill_(float("nan"))
            ctx.ls_paged_attend(shape, cache, dq, dt, dl, outs[0])
            ctx.ls_decode_attend(shape, dq, flat[0], flat[1], None, None, None, outs[1])
        torch.cuda.synchronize()
        for x in outs:
            _check(p, q, table, lens, x.cpu(), None)


def test_captured_calls_replay():
    """A token's rows into the cache and the attention over them, in a graph: every replay as the same calls without."""
    rng = np.random.default_rng(16)
    lens = [1500, 90]
    for kind in ("bf16", "e4m3"):
        p = pu.pool(rng, 110, 2, 16, 128, kind)
        table = pu.table_for(rng, [n + 16 for n in lens], 16, 110).cuda()
        cache, plain = _cache(p), _cache(p)
        shape = binding.make_shape(2, 8, 2, 128, 1600, 1, 1, "bf16")
        ctx = binding.Context(workspace=binding.paged_workspace_bytes(shape))
        other = binding.Context(workspace=binding.paged_workspace_bytes(shape))
        q, k, v = pu.rnd(rng, 2, 8, 128).cuda(), pu.rnd(rng, 2, 2, 1, 128).cuda(), pu.rnd(rng, 2, 2, 1, 128).cuda()
        pos, ln = _i32(lens), _i32([n + 1 for n in lens])
        out, ref = torch.empty_like(q), torch.empty_like(q)

        def call(c, pages, o):
            c.ls_cache_write(shape, pages, k, v, table, pos)
            c.ls_paged_attend(shape, pages, q, table, ln, o)

        print("paged graph", kind, flush=True)
        call(other, plain, ref)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(ctx, cache, out)
        for i in range(6):
            q.copy_(torch.roll(q, 1, 2)); k.copy_(torch.roll(k, 3, 3)); pos.add_(i > 0); ln.add_(i > 0)
            g.replay()
            torch.cuda.synchronize()
            call(other, plain, ref)
            torch.cuda.synchronize()
            assert torch.equal(out, ref) and _same(_host(cache), _host(plain)), i


def test_what_the_binding_refuses():
    rng = np.random.default_rng(17)
    p = pu.pool(rng, 4, 2, 16, 64, "e4m3")
    cache, ctx = _cache(p), binding.Context(workspace=1 << 20)
    d = {n: x.cuda() for n, x in p.items()}
    for bad in (dict(k=d["k"], v=d["v"]), dict(k=d["k"].float(), v=d["v"].float()), dict(d, k_exp=d["k_exp"][:2]), dict(d, v=d["v"][:3]),
                dict(d, k=d["k"].transpose(0, 1)), dict(d, k=p["k"]), dict(k=d["k"].to(torch.bfloat16), v=d["v"].to(torch.bfloat16), k_exp=d["k_exp"], v_exp=d["v_exp"])):
        with pytest.raises(ValueError):
            binding.PagedCache(**bad)
    rows, table, pos = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device="cuda"), _i32([[0, 1], [2, 3]]), _i32([0, 0])
    shape = binding.make_shape(2, 4, 2, 64, 32, 3, 1, "bf16")
    for change in (dict(k=rows.float()), dict(k=rows[:1]), dict(table=table[:1]), dict(table=table.long()), dict(pos=pos[:1]), dict(count=_i32([1])),
                   dict(starts=_i32([0, 1, 2])), dict(k=rows.transpose(2, 3)), dict(table=None)):
        a = dict(k=rows, v=rows, table=table, pos=pos)
        a.update(change)
        with pytest.raises((ValueError, binding.LoopServeError)):
            ctx.ls_cache_write(shape, cache, **a)
        with pytest.raises((ValueError, binding.LoopServeError)):
            ctx.ls_cache_read(shape, cache, **a)
    with pytest.raises(binding.LoopServeError):            # rows of an output that overlap
        ctx.ls_cache_read(shape, cache, table, rows[:, :, :1].expand(2, 2, 3, 64), rows, pos)
    with pytest.raises(binding.LoopServeError):            # another number of heads than the cache has
        ctx.ls_cache_write(binding.make_shape(2, 4, 4, 64, 32, 3, 1, "bf16"), cache, torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16, device="cuda"),
                           torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16, device="cuda"), table, pos)
    q, out, ln = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"), _i32([3, 4])
    for change in (dict(q=q.float()), dict(q=q[:, :2]), dict(out=out.transpose(0, 1)), dict(lens=ln.long()), dict(lens=ln[:1]), dict(table=table.cpu()), dict(lens=None),
                   dict(lse=torch.zeros(2, 2, device="cuda"))):
        a = dict(q=q, table=table, lens=ln, out=out)
        a.update(change)
        with pytest.raises((ValueError, binding.LoopServeError)):
            ctx.ls_paged_attend(shape, cache, **a)
    big = binding.make_shape(2, 4, 2, 64, 100000, 1, 1, "bf16")
    with pytest.raises(binding.LoopServeError):            # workspace too small
        binding.Context(workspace=256).ls_paged_attend(big, cache, q, table, ln, out)
