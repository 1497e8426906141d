"""Pages of 4-bit floats: stored bits, the way back, attention over them in 64 bits, and what is left out."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests import paged4_util as p4
from tests import paged_util as pu
from tests.test_gpu_cache import MOVES, TOKENS, _attend, _cache, _host, _i32, _places

pytestmark = pytest.mark.gpu


def _same(a, b):
    return all(torch.equal(a[n], b[n]) for n in b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("lens,pos,Hkv,d,page", MOVES)
def test_write_and_read(lens, pos, Hkv, d, page, packed, dtype):
    print("cache4 move", lens, pos, Hkv, d, page, packed, dtype, flush=True)
    rng = np.random.default_rng(sum(lens) + page)
    ends = [a + n for a, n in zip(pos, lens)]
    pages = sum(-(-e // page) for e in ends) + 2
    p = p4.pool(rng, pages, Hkv, page, d)
    table = pu.table_for(rng, ends, page, pages)
    B, most = len(lens), max(lens)
    rows = [pu.rnd(rng, sum(lens), Hkv, d, scale=s, dtype=dtype) for s in (1.0, 30.0)]
    cache, places = _cache(p), _places(lens, pos, table, page)
    if packed:
        shape = binding.make_shape(B, Hkv, Hkv, d, 1, sum(lens), 1, dtype)
        dev, kw = [x.cuda() for x in rows], dict(starts=_i32(np.concatenate([[0], np.cumsum(lens)])))
    else:
        shape = binding.make_shape(B, Hkv, Hkv, d, 1, most, 1, dtype)
        dev, kw = [torch.full((B, Hkv, most, d), float("nan"), dtype=dtype) for _ in rows], dict(count=_i32(lens))
        for x, y in zip(rows, dev):
            for r, (s, i, _, _) in enumerate(places):
                y[s, :, i] = x[r]
        dev = [y.cuda() for y in dev]
    ctx = binding.Context(workspace=0)
    ctx.ls_cache_write(shape, cache, dev[0], dev[1], table.cuda(), _i32(pos), **kw)
    assert ctx.ls_poll_status() == 0
    want = {n: x.clone() for n, x in p.items()}
    for name, x in zip(("k", "v"), rows):
        p4.write(want, name, x, places)
    assert _same(_host(cache), want)
    back = [torch.full_like(x, 7.0) for x in dev]
    ctx.ls_cache_read(shape, cache, table.cuda(), back[0], back[1], _i32(pos), **kw)
    assert ctx.ls_poll_status() == 0
    for name, got in zip(("k", "v"), back):
        ref = torch.full_like(got.cpu(), 7.0)
        stored = p4.stored(want, name)
        for r, (s, i, pg, pl) in enumerate(places):
            x = stored[pg, :, pl].to(dtype)
            if packed:
                ref[r] = x
            else:
                ref[s, :, i] = x
        assert torch.equal(got.cpu(), ref)


def test_rounding_of_every_kind_of_value():
    """Every tie and its neighbours, the border of the powers of two, the smallest and largest numbers, zeros of both signs, infinities and NaN."""
    d = 128
    ties = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 6.5])
    near = torch.cat([ties, torch.nextafter(ties, torch.full_like(ties, 9.0)), torch.nextafter(ties, torch.full_like(ties, -9.0)), -ties])       # 64
    tops = torch.tensor([7.0, 7.000001, 6.999999, 3.5])                  # at most 7; beyond; just below; half
    groups = torch.stack([torch.cat([near[32 * i:32 * i + 31], t[None]]) for t in tops for i in (0, 1)])        # [8,32]
    base = groups.flatten().view(2, d)
    rows = torch.cat([base * f for f in (1.0, 2.0 ** -20, 2.0 ** 100, 2.0 ** -122, 2.0 ** -126, 2.0 ** -140, 2.0 ** 125, 0.0, 0.77)])
    odd = base.repeat(2, 1)
    odd[0, 3], odd[1, 40], odd[2, 70], odd[3, :] = float("inf"), -float("inf"), float("nan"), float("nan")
    rows = torch.cat([rows, odd])[:, None]                    # [22,1,d]
    rows[12, 0, :32] = 3.4e38
    E = p4.exponents(rows)
    assert int(E.min()) == 2 and int(E[E < 255].max()) == 253 and int((E == 255).sum()) == 7
    n = rows.shape[0]
    cache = _cache(p4.empty(2, 1, 16, d, fill=0xA5))
    shape = binding.make_shape(1, 1, 1, d, 1, n, 1, "f32")
    ctx = binding.Context(workspace=0)
    print("cache4 rounding", flush=True)
    ctx.ls_cache_write(shape, cache, rows.cuda(), rows.cuda(), _i32([[0, 1]]), starts=_i32([0, n]))
    torch.cuda.synchronize()
    got = _host(cache)
    codes, exps = got["k"].view(32, -1)[:n], got["k_exp"].view(32, -1)[:n]
    assert torch.equal(exps, E[:, 0]) and _same(got, dict(k=got["v"], k_exp=got["v_exp"]))
    assert torch.equal(codes, p4.codes(rows, E)[:, 0])
    assert (got["k"].view(32, -1)[n:] == 0xA5).all() and (got["k_exp"].view(32, -1)[n:] == 0xA5).all()
    fine = (exps < 255).repeat_interleave(32, 1)
    err = (p4.values(codes, exps) - rows[:, 0].double()).abs()[fine]
    unit = torch.exp2(exps.double() - 127).repeat_interleave(32, 1)[fine]
    x = rows[:, 0].double().abs()[fine] / unit
    # half a step: 1/4 up to 2, 1/2 up to 4, 1 beyond, up to 7 (and above 1.75 * 2^127, where the largest power is not enough, nothing is)
    assert (err <= unit * torch.where(x <= 2, 0.25, torch.where(x <= 4, 0.5, 1.0))).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_every_byte_and_exponent_is_read(d, dtype):
    """All codes in either half of a byte under every exponent byte: code * 2^(E - 127) rounded to the rows' type, 255: no number."""
    byte = torch.arange(256).to(torch.uint8)
    rows = 256 * 256 * 2 // d                                 # every byte under every exponent
    E = torch.arange(256).to(torch.uint8).repeat_interleave(256 // 16)      # a group has 16 bytes
    p = dict(k=byte.repeat(256).view(-1, 1, 16, d // 2), k_exp=E.view(-1, 1, 16, d // 32))
    p.update(v=p["k"].flip(3).contiguous(), v_exp=p["k_exp"].flip(3).contiguous())
    want = {n: p4.stored(p, n).reshape(rows, d).to(dtype) for n in ("k", "v")}
    back = [torch.zeros(rows, 1, d, dtype=dtype, device="cuda") for _ in range(2)]
    print("cache4 bytes", d, dtype, flush=True)
    binding.Context(workspace=0).ls_cache_read(binding.make_shape(1, 1, 1, d, 1, rows, 1, dtype), _cache(p),
                                               torch.arange(rows // 16, dtype=torch.int32, device="cuda")[None], *back, starts=_i32([0, rows]))
    torch.cuda.synchronize()
    for n, x in zip(("k", "v"), back):
        x = x[:, 0].cpu()
        same = (x == want[n]) | (torch.isnan(x) & torch.isnan(want[n]))
        assert same.all(), torch.nonzero(~same)[:5].tolist()
        assert torch.equal(torch.signbit(x)[~torch.isnan(x)], torch.signbit(want[n])[~torch.isnan(x)])


def _check(p, q, table, lens, out, lse, scale=None):
    B, Hq, d = q.shape
    K, V = p4.stored(p, "k"), p4.stored(p, "v")
    Hkv, page = K.shape[1], K.shape[2]
    G = Hq // Hkv
    for b, n in enumerate(lens):
        i = torch.arange(n)
        pg, pl = table[b].long()[i // page], i % page
        keep = (pg >= 0) & (pg < K.shape[0])
        pg, pl = pg[keep], pl[keep]
        for j in range(Hkv):
            ref = pu.attention(q[b, j * G:(j + 1) * G], K[pg, j, pl], V[pg, j, pl], np.full(G, len(pg)), scale or d ** -0.5)
            pu.check(out[b, j * G:(j + 1) * G], None if lse is None else lse[b, j * G:(j + 1) * G], ref, torch.bfloat16)


@pytest.mark.parametrize("lens,Hq,Hkv,d,page", TOKENS + [
    ([300, 7], 12, 2, 64, 256), ([700, 20, 1], 40, 2, 64, 16), ([1900], 64, 2, 128, 32)])
def test_attend_matches(lens, Hq, Hkv, d, page):
    print("paged4", lens, Hq, Hkv, d, page, flush=True)
    rng = np.random.default_rng(len(lens) + Hq)
    pages = sum(-(-n // page) for n in lens) + 2
    p = p4.pool(rng, pages, Hkv, page, d)
    q = pu.rnd(rng, len(lens), Hq, d, scale=1.5)
    table = pu.table_for(rng, lens, page, pages)
    out, lse, status = _attend(p, q, table, lens, times=3)
    assert status == 0
    _check(p, q, table, lens, out, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_each_place_of_a_tile(d):
    """One key a sequence that all weight lies on, in each place of 70 positions: its row of V, value by value (groups of 32 have powers of their own)."""
    rng = np.random.default_rng(3)
    n = 70
    p = p4.pool(rng, n * 5, 1, 16, d)
    p["v_exp"] = torch.from_numpy(rng.integers(90, 160, p["v_exp"].shape).astype(np.uint8))
    table = torch.arange(n * 5, dtype=torch.int32).view(n, 5)
    k = torch.zeros(n, 80, d)
    k[torch.arange(n), torch.arange(n), 5] = 4.0
    p["k_exp"] = p4.exponents(k).view(n * 5, 1, 16, -1)
    p["k"] = p4.codes(k, p4.exponents(k)).view(n * 5, 1, 16, -1)
    q = torch.zeros(n, 3, d).bfloat16()
    q[:, :, 5] = 512.0
    print("paged4 places", d, flush=True)
    out, lse, status = _attend(p, q, table, [n] * n, scale=1.0)
    want = p4.stored(p, "v").view(n, 80, d)[torch.arange(n), torch.arange(n)].to(torch.bfloat16)
    assert status == 0 and torch.equal(out, want[:, None].expand(n, 3, d)) and ((lse - 2048.0).abs() <= 2048 * 2.0 ** -22).all()


def test_more_than_64_sequences():
    rng = np.random.default_rng(8)
    lens = [int(x) for x in rng.integers(0, 90, 130)] + [3000]
    p = p4.pool(rng, sum(-(-n // 16) for n in lens), 2, 16, 64)
    q, table = pu.rnd(rng, len(lens), 4, 64), pu.table_for(rng, lens, 16, p["k"].shape[0])
    print("paged4 131 sequences", flush=True)
    out, lse, status = _attend(p, q, table, lens)
    assert status == 0
    _check(p, q, table, lens, out, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_what_lies_behind_the_length_does_not_matter(d):
    """Exponents of no number behind the last position of a page, and table entries that are no pages."""
    rng = np.random.default_rng(9)
    lens = [5, 50, 100]
    p = p4.pool(rng, 12, 2, 32, d)
    table = pu.table_for(rng, lens, 32, 12, width=7)
    clean = {n: x.clone() for n, x in p.items()}
    for b, n in enumerate(lens):
        pg, pl = int(table[b, (n - 1) // 32]), (n - 1) % 32 + 1
        for name in ("k", "v"):
            p[name][pg, :, pl:], p[name + "_exp"][pg, :, pl:] = 0x77, 255
    q = pu.rnd(rng, 3, 8, d)
    print("paged4 poison", d, flush=True)
    out, lse, status = _attend(p, q, table, lens, n=7 * 32)
    assert status == 0
    _check(clean, q, table, lens, out, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_pages_that_are_nowhere(d):
    rng = np.random.default_rng(10)
    p = p4.pool(rng, 6, 2, 16, d)
    p["v_exp"][0, :, :] = 255                                # (the page that is read in the place of none; of a sequence of its own below)
    clean = {n: x.clone() for n, x in p.items()}
    table = torch.tensor([[6, 1, -1, 3], [-1, -2, 99, 7], [2, 3, 4, 5], [6, 6, 6, 2]], dtype=torch.int32)
    q = pu.rnd(rng, 4, 4, d)
    print("paged4 nowhere", d, flush=True)
    out, lse, status = _attend(p, q, table, [50, 64, 64, 60], n=64)
    assert status == binding.LS_STAT_PAGE_RANGE
    _check(clean, q, table, [50, 64, 64, 60], out, lse)
    out, lse, status = _attend(p, q[:1], table[2:3], [1000], n=5000)
    assert status == binding.LS_STAT_PAGE_RANGE
    _check(clean, q[:1], table[2:3], [64], out, lse)
    out, lse, status = _attend(p, q[:1], table[2:3], [-3], n=64)
    assert status == 0 and (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("d", [64, 128])
def test_every_exponent_byte_is_attended_to(d):
    """One key a sequence, whose output is its row of V; no number where the byte is 255, in its 32 values alone."""
    groups = d // 32
    codes = torch.arange(256).to(torch.uint8)
    p = p4.empty(256, 1, 16, d)
    p["v"][:] = codes.repeat(2)[:d // 2]
    p["v_exp"][:, 0, 0, :] = (torch.arange(256)[:, None] + 64 * torch.arange(groups)).to(torch.uint8)
    p["v_exp"][:, 0, 1:, :] = 255
    p["k_exp"][:] = 127
    print("paged4 bytes of V", d, flush=True)
    out, _, status = _attend(p, torch.ones(256, 1, d).bfloat16(), torch.arange(256, dtype=torch.int32)[:, None], [1] * 256)
    want = p4.stored(p, "v")[:, 0, 0].to(torch.bfloat16)
    assert status == 0 and (torch.isnan(want).sum(1) > 0).sum() == groups
    same = (out[:, 0] == want) | (torch.isnan(out[:, 0]) & torch.isnan(want))
    assert same.all(), torch.nonzero(~same)[:5].tolist()


def test_every_exponent_byte_of_keys():
    """Logits of single keys: a query that is a power of two in one column brings the stored value near one; the normaliser of one key is its logit."""
    d = 128
    bits = torch.arange(256)
    p = p4.empty(256, 1, 16, d)
    p["k"][:] = torch.arange(64).to(torch.uint8) * 3 + 1
    p["k_exp"][:] = bits.to(torch.uint8)[:, None, None, None]
    p["v"][:], p["v_exp"][:] = 0x22, 127
    value = p4.stored(p, "k")[:, 0, 0]
    back = torch.exp2((127 - bits).clamp_min(-126).double())
    for col in (0, 1, 31, 32, 63, 64, 77, 127):
        q = torch.zeros(256, 1, d, dtype=torch.bfloat16)
        q[:, 0, col] = back.to(torch.bfloat16)
        print("paged4 bytes of K", col, flush=True)
        out, lse, _ = _attend(p, q, bits.int()[:, None], [1] * 256, scale=1.0)
        x, got = value.to(torch.bfloat16).double()[:, col] * back, lse[:, 0].double()
        nan = ~torch.isfinite(value.to(torch.bfloat16)).all(1)         # (of whichever column: 0 times infinity, which 2^128 is, or times no number)
        assert nan.sum() == 3 and torch.equal(torch.isnan(got), nan)
        assert ((got - x).abs() <= 2.0 ** -22 * x.abs())[~nan].all(), col
        assert (out[~nan] == 1.0).all() and torch.isnan(out[nan]).all()


@pytest.mark.parametrize("n,at", [(2, 1), (40, 35), (40, 3), (64, 50), (3000, 1234)])
def test_a_group_that_is_none(n, at):
    """Of a row of V that is seen: the 32 columns of the group become no number, the others do not."""
    rng = np.random.default_rng(44)
    p = p4.pool(rng, -(-n // 16), 2, 16, 128)
    p["v_exp"][at // 16, 1, at % 16, 2] = 255
    q, table = pu.rnd(rng, 1, 4, 128), torch.arange(-(-n // 16), dtype=torch.int32)[None]
    print("paged4 none", n, at, flush=True)
    out, lse, status = _attend(p, q, table, [n])
    assert status == 0 and torch.isfinite(lse).all()
    none = torch.isnan(out[0])
    assert none[2:, 64:96].all() and not none[2:, :64].any() and not none[2:, 96:].any() and not none[:2].any()


def test_shared_pages_no_lse_and_scale():
    rng = np.random.default_rng(11)
    p = p4.pool(rng, 4, 2, 64, 128)
    table = torch.tensor([[0, 1, 2], [0, 1, 3], [1, 1, 1]], dtype=torch.int32)
    q = pu.rnd(rng, 3, 6, 128)
    print("paged4 shared", flush=True)
    out, lse, _ = _attend(p, q, table, [150, 190, 192], lse=False, scale=0.11)
    _check(p, q, table, [150, 190, 192], out, None, scale=float(np.float32(0.11)))


def test_the_last_pages_of_a_large_pool():
    """Rows and exponents beyond 2^32 bytes and 2^31 elements of the pools."""
    d, Hkv, page = 128, 8, 256
    pages = (1 << 32) // (Hkv * page * d // 2) + 3           # bytes of codes beyond 2^32
    cache = binding.PagedCache(*(torch.zeros(pages, Hkv, page, w, dtype=torch.uint8, device="cuda") for w in (64, 64, 4, 4)))
    rng = np.random.default_rng(12)
    T = 700
    rows = [pu.rnd(rng, T, Hkv, d) for _ in range(2)]
    table = _i32([[pages - 1, 0, pages - 2]])
    ctx = binding.Context(workspace=1 << 22)
    print("cache4 large pool", pages, flush=True)
    ctx.ls_cache_write(binding.make_shape(1, Hkv, Hkv, d, 1, T, 1, "bf16"), cache, *(x.cuda() for x in rows), table, starts=_i32([0, T]))
    back = [torch.empty(T, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx.ls_cache_read(binding.make_shape(1, Hkv, Hkv, d, 1, T, 1, "bf16"), cache, table, *back, starts=_i32([0, T]))
    want = [p4.values(p4.codes(x, p4.exponents(x)), p4.exponents(x)) for x in rows]
    for x, y in zip(back, want):
        assert torch.equal(x.cpu().double(), y)
    q = pu.rnd(rng, 1, 16, d)
    out, lse = torch.empty(1, 16, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 16, device="cuda")
    ctx.ls_paged_attend(binding.make_shape(1, 16, Hkv, d, T, 1, 1, "bf16"), cache, q.cuda(), table, _i32([T]), out, lse)
    assert ctx.ls_poll_status() == 0
    for j in range(Hkv):
        ref = pu.attention(q[0, 2 * j:2 * j + 2], want[0][:, j], want[1][:, j], [T, T], d ** -0.5)
        pu.check(out[0, 2 * j:2 * j + 2].cpu(), lse[0, 2 * j:2 * j + 2].cpu(), ref, torch.bfloat16)


@pytest.mark.parametrize("seed", range(30))
def test_token_shapes(seed):
    rng = np.random.default_rng(6000 + seed)
    log = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))
    Hkv, G, d, page = int(rng.choice([1, 2, 3, 8, 20])), int(rng.choice([1, 2, 5, 16, 17, 32])), int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 128, 256]))
    B = int(rng.choice([1, 2, 7, 40, 64, 65, 90]))
    lens = [log(1, max(60, 60000 // (B * Hkv))) - int(rng.random() < 0.1) for _ in range(B)]
    pages = max(1, sum(-(-n // page) for n in lens))
    print("paged4 shape", seed, Hkv, G, d, page, B, lens[:6], flush=True)
    p = p4.pool(rng, pages, Hkv, page, d)
    q, table = pu.rnd(rng, B, Hkv * G, d, scale=1.5), pu.table_for(rng, lens, page, pages)
    out, lse, status = _attend(p, q, table, lens, n=int(max(1, max(lens)) * rng.choice([1, 1, 3])), times=2)
    assert status == 0
    _check(p, q, table, lens, out, lse)


def test_what_the_binding_refuses():
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    k, e = u8(3, 2, 16, 64), u8(3, 2, 16, 4)
    assert binding.PagedCache(k, k, e, e).struct.d == 128 and binding.PagedCache(k, k, e, e).struct.type == binding.LS_CACHE_E2M1
    four = k.view(torch.float4_e2m1fn_x2)
    assert binding.PagedCache(four, four, e, e).struct.d == 128
    for bad in (lambda: binding.PagedCache(k, k, e), lambda: binding.PagedCache(k, k, u8(3, 2, 16, 2), u8(3, 2, 16, 2)),
                lambda: binding.PagedCache(four, four, u8(3, 2, 16), u8(3, 2, 16)), lambda: binding.PagedCache(k, k, e, e.cpu()),
                lambda: binding.PagedCache(k.view(torch.float8_e4m3fn), k.view(torch.float8_e4m3fn), e, e), lambda: binding.PagedCache(k, k, e, u8(3, 2, 16)),
                lambda: binding.PagedCache(four, four)):
        with pytest.raises(ValueError):
            bad()
    cache, ctx = binding.PagedCache(k, k.clone(), e, e.clone()), binding.Context(workspace=0)
    rows = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.LoopServeError, match="differ"):          # d of the shape is 64, and of the pages 128
        ctx.ls_cache_write(binding.make_shape(1, 2, 2, 64, 1, 2, 1, "bf16"), cache, rows, rows, _i32([[0]]), starts=_i32([0, 2]))


@pytest.mark.parametrize("B,Hkv,Hq,n", [(16, 8, 8, 1632), (16, 8, 8, 1633), (127, 1, 2, 513), (127, 1, 2, 512), (40, 4, 4, 2048), (40, 4, 8, 2049), (70, 2, 2, 1792), (70, 2, 2, 1793)])
def test_heads_that_stay_whole(B, Hkv, Hq, n):
    """Sequences at either side of the length from which their heads are cut, which goes by how many heads there are."""
    rng = np.random.default_rng(B + n)
    lens = [int(x) for x in rng.integers(0, 40, B)]
    lens[3], lens[B - 1] = n, n - 1
    pages = sum(-(-x // 64) for x in lens)
    p = p4.pool(rng, pages, Hkv, 64, 64)
    q, table = pu.rnd(rng, B, Hq, 64, scale=1.5), pu.table_for(rng, lens, 64, pages)
    print("paged4 whole", B, Hkv, Hq, n, flush=True)
    out, lse, status = _attend(p, q, table, lens, times=3)
    assert status == 0
    _check(p, q, table, lens, out, lse)


@pytest.mark.parametrize("B,Hkv,Hq,d,n", [(16, 8, 8, 64, 1152), (16, 8, 8, 64, 1153), (66, 1, 2, 64, 1153), (64, 1, 2, 128, 512), (64, 1, 2, 128, 513), (40, 4, 8, 64, 2304), (40, 4, 4, 128, 2305),
                                         (70, 2, 2, 64, 2304), (70, 2, 40, 64, 2305)])
def test_heads_that_are_cut_from_a_length_on(B, Hkv, Hq, d, n):
    """Sequences at either side of the lengths from which heads are cut into parts, where the others are short."""
    rng = np.random.default_rng(B + n)
    lens = [int(x) for x in rng.integers(0, 40, B)]
    lens[3], lens[B - 1], lens[B // 2] = n, n - 1, 0
    pages = sum(-(-x // 64) for x in lens)
    p = p4.pool(rng, pages, Hkv, 64, d)
    q, table = pu.rnd(rng, B, Hq, d, scale=1.5), pu.table_for(rng, lens, 64, pages)
    print("paged4 cut", B, Hkv, Hq, d, n, flush=True)
    out, lse, status = _attend(p, q, table, lens, times=3)
    assert status == 0
    _check(p, q, table, lens, out, lse)


@pytest.mark.parametrize("lens,Hq,Hkv,d", [([28129], 32, 1, 128), ([9001], 32, 1, 64), ([0, 20000, 1, 700], 32, 1, 128), ([12000, 0, 511, 513, 14001], 40, 2, 64), ([1] * 30 + [16384] + [0] * 10, 24, 1, 128)])
def test_parts_that_a_launch_more_puts_together(lens, Hq, Hkv, d):
    """Many parts of many query heads, beside sequences of one part and of none, over unlike calls on the same workspace."""
    rng = np.random.default_rng(sum(lens) + d)
    pages = sum(-(-x // 64) for x in lens)
    p = p4.pool(rng, pages, Hkv, 64, d)
    q, table = pu.rnd(rng, len(lens), Hq, d, scale=1.5), pu.table_for(rng, lens, 64, pages)
    print("paged4 joined", lens[:5], Hq, Hkv, d, flush=True)
    out, lse, status = _attend(p, q, table, lens, times=3)
    assert status == 0
    _check(p, q, table, lens, out, lse)


def test_workspace_by_the_type_of_the_pages():
    """Where each head's parts are is kept for 4-bit pages alone: the others take a workspace that has the parts' results and no more, and nothing is written beyond it."""
    B, Hq, Hkv, d, n, page = 16, 32, 8, 64, 3000, 64
    rng = np.random.default_rng(11)
    lens, q = [n] + [int(x) for x in rng.integers(0, n, B - 1)], pu.rnd(rng, B, Hq, d)
    shape = binding.make_shape(B, Hq, Hkv, d, n, 1, 1, "bf16")
    cuts, most = (C.c_int32 * B)(), C.c_int32()
    units = binding.load_library().ls_debug_paged_cuts(C.byref(shape), (C.c_int32 * B)(*lens), cuts, C.byref(most))
    parts = -(-units * (Hq // Hkv) * (d + 4) * 4 // 256) * 256
    assert most.value > 1 and parts + 8 * B * Hkv <= binding.paged_workspace_bytes(shape)
    pages = sum(-(-x // page) for x in lens)
    table = pu.table_for(rng, lens, page, pages)
    for kind in ("bf16", "e4m3", "e2m1"):
        p = p4.pool(rng, pages, Hkv, page, d) if kind == "e2m1" else pu.pool(rng, pages, Hkv, page, d, kind)
        cache, got = _cache(p), []
        for bytes_ in (binding.paged_workspace_bytes(shape), parts, parts - 256):
            print("paged workspace", kind, bytes_, flush=True)
            ctx, out = binding.Context(workspace=bytes_), torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
            call = lambda: ctx.ls_paged_attend(shape, cache, q.cuda(), table.cuda(), _i32(lens), out)
            if bytes_ < (parts + 8 * B * Hkv if kind == "e2m1" else parts):
                with pytest.raises(binding.LoopServeError):
                    call()
                continue
            call()
            got.append(out.cpu())
        assert all(torch.equal(x, got[0]) for x in got) and not got[0].isnan().any() and len(got) == (1 if kind == "e2m1" else 2)
