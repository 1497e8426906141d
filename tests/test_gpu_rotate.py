"""ls_norm_rotate: norms and rotations against 64 bits, and pages as ls_cache_write makes them of the rotated rows."""
import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests import paged4_util as p4
from tests import paged_util as pu
from tests.test_gpu_cache import _cache, _host, _i32

pytestmark = pytest.mark.gpu


def _freq(dims, base=10000.0):
    return torch.pow(torch.tensor(base, dtype=torch.float64), -torch.arange(0, dims, 2, dtype=torch.float64) / dims).float()


def _expect(x, w, eps, freq, positions, neighbours):
    """Rows [..,R,H,d] in 64 bits, and what fp32 may add: the result, and the bound of its error before it is rounded to the rows' type.

    The sum of d squares, 16 in a lane and 3 steps over lanes, is off by 19 2^-24 of itself, its root and the reciprocal of that by half of it and 2^-23, the sum with eps and the two
    products by 2^-24 each: 15 2^-24 at most.  Sine and cosine are off by their last rounding, those of the polynomials and of the reduced angle: 4 2^-24.  The two products of a turned
    value add 2 2^-24: 21, for which 32 stand.  What the angle is off by in 64 bits: 2^-52 |t|."""
    x = x.double()
    y = x if w is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + float(np.float32(eps))) * w.double()
    r = 0 if freq is None else 2 * freq.shape[0]
    out, size = y.clone(), y.abs()
    if r:
        t = positions.double()[..., None] * freq.double()
        c, s = torch.cos(t)[..., None, :], torch.sin(t)[..., None, :]
        i = torch.arange(r // 2)
        u, v = (2 * i, 2 * i + 1) if neighbours else (i, i + r // 2)
        a, b = y[..., u], y[..., v]
        out[..., u], out[..., v] = a * c - b * s, b * c + a * s
        both = (a.abs() + b.abs()) * (1.0 + 2.0 ** -52 * t.abs()[..., None, :] * 2.0 ** 19)
        size = size.clone()
        size[..., u] = size[..., v] = both
    return out, size * 2.0 ** -19


def _check(got, want, dtype):
    out, err = want
    half = pu.HALF[dtype]
    tiny = 2.0 ** -134 if dtype == torch.bfloat16 else 2.0 ** -150          # half a step of the subnormal ones
    tol = half * out.abs() + err * (1 + half) + tiny
    off = (got.double().cpu() - out).abs()
    assert (off <= tol).all(), (float((off / tol).max()), [int(x) for x in np.unravel_index(int((off / tol).argmax()), off.shape)])


CASES = [
    # rows, Hq, Hkv, d, dims, neighbours, norms, base
    (1, 1, 1, 64, 64, False, "qk", 1e4),
    (1, 32, 8, 128, 128, False, "qk", 5e5),
    (5, 4, 1, 64, 32, True, "k", 1e4),
    (37, 12, 3, 128, 96, False, "q", 1e4),
    (37, 12, 3, 128, 96, True, "qk", 1e4),
    (130, 8, 8, 64, 16, False, "qk", 1e4),
    (130, 8, 2, 64, 48, True, "", 1e4),
    (33, 5, 5, 128, 0, False, "qk", 1e4),
    (3, 64, 1, 128, 112, False, "qk", 1e4),
    (3000, 16, 4, 128, 128, True, "qk", 1e6),
    (5003, 6, 2, 64, 64, False, "qk", 1e4),
    (700, 33, 11, 64, 32, False, "q", 1e4),
    (3, 256, 2, 128, 128, False, "qk", 1e4),               # more heads than a workgroup takes
    (201, 500, 4, 64, 64, True, "qk", 1e4),
    (20000, 1, 1, 64, 64, False, "k", 1e4),                # few of many rows
    (2500, 40, 8, 128, 64, True, "qk", 1e4),
]


def _rotation(rng, d, dims, neighbours, norms, base, eps=1e-6):
    freq = _freq(dims, base) if dims else None
    w = {n: torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)) if n in norms else None for n in "qk"}
    dev = lambda t: None if t is None else t.cuda()
    return freq, w, binding.Rotation(dev(freq), neighbours, dev(w["q"]), dev(w["k"]), eps)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("form", ["packed", "padded", "fused, in place"])
@pytest.mark.parametrize("rows,Hq,Hkv,d,dims,neighbours,norms,base", CASES)
def test_rows(rows, Hq, Hkv, d, dims, neighbours, norms, base, form, dtype):
    print("rotate", rows, Hq, Hkv, d, dims, neighbours, norms, form, dtype, flush=True)
    rng = np.random.default_rng(rows + d + dims)
    freq, w, rotation = _rotation(rng, d, dims, neighbours, norms, base)
    B = 3 if form == "padded" else 1
    positions = torch.from_numpy(rng.integers(0, 200000, (B, rows)).astype(np.int32))
    q, k = (pu.rnd(rng, B, rows, H, d, scale=2.0, dtype=dtype) for H in (Hq, Hkv))
    ctx = binding.Context(workspace=0)
    shape = binding.make_shape(B, Hq, Hkv, d, 1, rows, 1, dtype)
    if form == "padded":
        dq, dk = (x.transpose(1, 2).contiguous().cuda() for x in (q, k))
        oq, ok = (torch.full_like(x, float("nan")) for x in (dq, dk))
        ctx.ls_norm_rotate(shape, rotation, dq, dk, oq, ok, positions.cuda())
        oq, ok = (x.transpose(1, 2) for x in (oq, ok))
    elif form == "packed":
        dq, dk = q[0].cuda(), k[0].cuda()
        oq, ok = (torch.full_like(x, float("nan")) for x in (dq, dk))
        many = binding.make_shape(7, Hq, Hkv, d, 1, rows, 1, dtype)          # packed rows are counted as they are, however many sequences the shape has
        ctx.ls_norm_rotate(many, rotation, dq, dk, oq, ok, positions[0].cuda())
        oq, ok = oq[None], ok[None]
    else:
        x = torch.full((rows, Hq + 2 * Hkv, d), 9.0, dtype=dtype, device="cuda")
        oq, ok = x[:, :Hq], x[:, Hq:Hq + Hkv]
        oq[:], ok[:] = q[0].cuda(), k[0].cuda()
        ctx.ls_norm_rotate(shape, rotation, oq, ok, oq, ok, positions[0].cuda())
        assert (x[:, Hq + Hkv:] == 9.0).all()
        oq, ok = oq[None], ok[None]
    assert ctx.ls_poll_status() == 0
    for got, x, n in ((oq, q, "q"), (ok, k, "k")):
        _check(got, _expect(x, w[n], 1e-6, freq, positions, neighbours), dtype)


def _pool(kind, pages, Hkv, page, d):
    if kind == "e2m1":
        return p4.empty(pages, Hkv, page, d, fill=0x5A)
    p = {n: torch.full((pages, Hkv, page, d), 3.0).bfloat16() if kind == "bf16" else torch.full((pages, Hkv, page, d), 0x5A, dtype=torch.uint8) for n in "kv"}
    if kind == "e4m3":
        p.update({n + "_exp": torch.full((pages, Hkv, page), 0x5A, dtype=torch.uint8) for n in "kv"})
    return p


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("lens,pos,Hq,Hkv,d,dims,neighbours,page", [
    ([1, 1, 1, 1], [15, 16, 0, 33], 8, 2, 128, 128, False, 16),
    ([37, 1, 5], [3, 7, 250], 12, 3, 64, 64, False, 32),
    ([300, 129], [0, 100], 4, 4, 128, 32, False, 64),
    ([70], [77], 5, 5, 128, 96, True, 128),
    ([900, 41], [255, 256], 4, 1, 64, 48, True, 256),
    ([10], [0], 2, 1, 64, 0, False, 16),
])
def test_pages_are_those_of_rows_written(lens, pos, Hq, Hkv, d, dims, neighbours, page, kind, dtype):
    """Keys and values into pages by slots, with and without rows of keys, against rotated rows that ls_cache_write puts there by the table: the same bits."""
    print("rotate into pages", lens, pos, Hq, Hkv, d, dims, neighbours, page, kind, dtype, flush=True)
    rng = np.random.default_rng(sum(lens) + page)
    _, _, rotation = _rotation(rng, d, dims, neighbours, "qk", 1e4)
    T, ends = sum(lens), [a + n for a, n in zip(pos, lens)]
    pages = sum(-(-e // page) for e in ends) + 2
    table = pu.table_for(rng, ends, page, pages)
    at = [(s, pos[s] + i) for s, n in enumerate(lens) for i in range(n)]
    positions = _i32([p for _, p in at])
    slots = torch.tensor([int(table[s, p // page]) * page + p % page for s, p in at], device="cuda")
    q, k, v = (pu.rnd(rng, T, H, d, scale=2.0, dtype=dtype).cuda() for H in (Hq, Hkv, Hkv))
    ctx = binding.Context(workspace=0)
    shape = binding.make_shape(len(lens), Hq, Hkv, d, 1, T, 1, dtype)
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    ctx.ls_norm_rotate(shape, rotation, q, k, oq, ok, positions)
    want = _cache(_pool(kind, pages, Hkv, page, d))
    ctx.ls_cache_write(shape, want, ok, v, table.cuda(), _i32(pos), starts=_i32(np.concatenate([[0], np.cumsum(lens)])))
    want = _host(want)
    for rows in (True, False):
        cache = _cache(_pool(kind, pages, Hkv, page, d))
        gq, gk = torch.full_like(q, float("nan")), torch.full_like(k, float("nan")) if rows else None
        ctx.ls_norm_rotate(shape, rotation, q, k, gq, gk, positions, cache, v, slots)
        assert ctx.ls_poll_status() == 0 and torch.equal(gq, oq) and (not rows or torch.equal(gk, ok))
        got = _host(cache)
        assert all(torch.equal(got[n].view(torch.uint8), want[n].view(torch.uint8)) for n in want)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_slots_that_are_nowhere(kind):
    """Negative ones without a word, ones beyond the pool with one; their rows are rotated all the same.  Padded sequences, and strided v."""
    rng = np.random.default_rng(5)
    Hq, Hkv, d, page, n = 4, 2, 64, 16, 9
    _, _, rotation = _rotation(rng, d, d, False, "k", 1e4)
    q, k, v = (pu.rnd(rng, 2, n, H, d).cuda().transpose(1, 2) for H in (Hq, Hkv, Hkv))
    slots = torch.tensor([[0, -1, 5, 47, -2 ** 63, 16, 31, 32, 1], [2, 3, -1, -1, -1, -1, -1, -1, 46]], device="cuda")
    shape, ctx = binding.make_shape(2, Hq, Hkv, d, 1, n, 1, "bf16"), binding.Context(workspace=0)
    oq, ok = torch.empty(2, Hq, n, d, dtype=torch.bfloat16, device="cuda"), torch.empty(2, Hkv, n, d, dtype=torch.bfloat16, device="cuda")
    print("rotate nowhere", kind, flush=True)
    ctx.ls_norm_rotate(shape, rotation, q, k, oq, ok)                    # (positions: the rows' numbers)
    cache = _cache(_pool(kind, 3, Hkv, page, d))
    got = torch.empty_like(oq)
    ctx.ls_norm_rotate(shape, rotation, q, k, got, None, None, cache, v, slots)
    assert ctx.ls_poll_status() == 0 and torch.equal(got, oq)
    want = _cache(_pool(kind, 3, Hkv, page, d))
    for b in range(2):
        for i in range(n):
            s = int(slots[b, i])
            if s >= 0:
                ctx.ls_cache_write(binding.make_shape(1, Hkv, Hkv, d, 1, 1, 1, "bf16"), want, ok[b:b + 1, :, i:i + 1].contiguous(), v[b:b + 1, :, i:i + 1].contiguous(),
                                   _i32([[s // page]]), _i32([s % page]))
    first = _host(want)
    assert all(torch.equal(_host(cache)[x].view(torch.uint8), first[x].view(torch.uint8)) for x in first)
    for bad in (48, 2 ** 40, 2 ** 63 - 1):
        slots[0, 1] = bad
        ctx.ls_norm_rotate(shape, rotation, q, k, got, None, None, cache, v, slots)
        assert ctx.ls_poll_status() == binding.LS_STAT_PAGE_RANGE and torch.equal(got, oq)
        assert all(torch.equal(_host(cache)[x].view(torch.uint8), first[x].view(torch.uint8)) for x in first)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6, 1.0])
def test_rows_whose_squares_leave_fp32(eps, dtype):
    """From 2^-140 to 2^125: and zeros, which stay zeros (no number without eps, as the formula has it), infinities and NaN."""
    rng = np.random.default_rng(6)
    d, scales = 128, [-140, -130, -100, -70, -64, -60, -31, -20, 0, 40, 50, 60, 64, 100, 122, 125]
    x = torch.stack([pu.rnd(rng, 2, d, dtype=torch.float32).clamp(-3, 3) * 2.0 ** s for s in scales]).to(dtype)
    x[3, 1, 1:] = 0                                          # one value alone
    w = torch.full((d,), 0.75)
    rotation = binding.Rotation(None, False, w.cuda(), w.cuda(), eps)
    n = x.shape[0]
    ctx, shape = binding.Context(workspace=0), binding.make_shape(1, 2, 2, d, 1, n, 1, dtype)
    oq, ok = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda")
    print("rotate ranges", eps, dtype, flush=True)
    ctx.ls_norm_rotate(shape, rotation, x.cuda(), x.cuda(), oq, ok)
    torch.cuda.synchronize()
    oq, ok = oq.cpu(), ok.cpu()
    want, err = _expect(x, w, eps, None, None, False)
    none = (x == 0).all(-1) & (eps == 0)                     # (2^-140 is nothing in bf16: 0 / 0)
    assert torch.equal(torch.isnan(want), none[..., None].expand(want.shape)) and torch.isnan(oq[none]).all() and torch.isnan(ok[none]).all()
    assert torch.equal(oq[~none], ok[~none])
    _check(oq[~none], (want[~none], err[~none]), dtype)
    x = torch.zeros(4, 2, d, dtype=dtype)
    x[1, 0, 5], x[2, 1, 7], x[3, 0, 9] = float("inf"), float("nan"), -float("inf")
    x[1, 0, 6] = x[3, 1, :] = 1.0
    shape = binding.make_shape(1, 2, 2, d, 1, 4, 1, dtype)
    oq, ok = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda")
    ctx.ls_norm_rotate(shape, rotation, x.cuda(), x.cuda(), oq, ok)
    oq = oq.cpu()
    y = x.double()
    want = y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(np.float32(eps))) * 0.75
    assert torch.equal(torch.isnan(oq), torch.isnan(want)) and ((oq.double() - want).abs() <= pu.HALF[dtype] * want.abs() + 2.0 ** -19 * want.abs())[~torch.isnan(want)].all()


def test_neighbouring_rows_do_not_matter():
    """A row between ones of infinities and NaN has the bits that it has alone."""
    rng = np.random.default_rng(7)
    for d, Hq, Hkv in ((64, 6, 2), (128, 3, 3)):
        _, _, rotation = _rotation(rng, d, d // 2, True, "qk", 1e4)
        q, k = (pu.rnd(rng, 33, H, d).cuda() for H in (Hq, Hkv))
        shape, ctx = binding.make_shape(1, Hq, Hkv, d, 1, 33, 1, "bf16"), binding.Context(workspace=0)
        a, b, c, e = (torch.empty_like(x) for x in (q, k, q, k))
        print("rotate neighbours", d, flush=True)
        ctx.ls_norm_rotate(shape, rotation, q, k, a, b)
        odd = torch.arange(33, device="cuda") % 2 == 1
        q[odd, ::2], k[odd], q[~odd, 1] = float("nan"), float("inf"), float("inf")
        ctx.ls_norm_rotate(shape, rotation, q, k, c, e)
        torch.cuda.synchronize()
        keep = [h for h in range(Hq) if h != 1]
        assert torch.equal(c[~odd][:, keep], a[~odd][:, keep]) and torch.equal(e[~odd], b[~odd])
        if Hq > 3:
            assert torch.equal(c[odd][:, 3::2], a[odd][:, 3::2])


@pytest.mark.parametrize("neighbours", [False, True])
def test_far_and_negative_positions(neighbours):
    """Angles up to 2^31 and of either sign, at every quarter turn: what is off is what fp32 holds of sine and cosine."""
    rng = np.random.default_rng(8)
    d = 128
    freq = _freq(d, 1e4)
    freq[:3] = torch.tensor([1.0, 0.5, np.pi / 2])
    at = np.concatenate([[0, 1, -1, 2, 3, 4, 2147483647, -2147483648, 1 << 24, (1 << 24) + 1, 16777259, 262143], rng.integers(-2 ** 31, 2 ** 31, 200), np.arange(5, 60)])
    positions = torch.from_numpy(at.astype(np.int32))
    n = len(at)
    q, k = pu.rnd(rng, n, 1, d, dtype=torch.float32), torch.ones(n, 1, d)
    rotation = binding.Rotation(freq.cuda(), neighbours)
    ctx, shape = binding.Context(workspace=0), binding.make_shape(1, 1, 1, d, 1, n, 1, "f32")
    oq, ok = torch.empty_like(q, device="cuda"), torch.empty_like(k, device="cuda")
    print("rotate far", neighbours, flush=True)
    ctx.ls_norm_rotate(shape, rotation, q.cuda(), k.cuda(), oq, ok, positions.cuda())
    torch.cuda.synchronize()
    for got, x in ((oq, q), (ok, k)):
        _check(got, _expect(x, None, 0, freq, positions, neighbours), torch.float32)


def test_more_rows_than_a_launch_has_workgroups_for():
    """Rows of a query and a key head, 64 to a workgroup, that take a second launch (queries in, keys and values share one place in memory): the first and the last ones are right."""
    n, d = (1 << 29) + 1003, 64
    rng = np.random.default_rng(9)
    freq, w, rotation = _rotation(rng, d, d, False, "qk", 1e4)
    q, k, v = (pu.rnd(rng, 1, 1, d) for _ in range(3))
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    slots[-3:] = torch.arange(3, device="cuda")
    cache = binding.PagedCache(*(torch.zeros(1, 1, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    out = torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda")
    ctx, shape = binding.Context(workspace=0), binding.make_shape(1, 1, 1, d, 1, n, 1, "bf16")
    print("rotate many rows", flush=True)
    ctx.ls_norm_rotate(shape, rotation, *(x.cuda().expand(n, 1, d) for x in (q, k)), out, None, None, cache, v.cuda().expand(n, 1, d), slots)
    assert ctx.ls_poll_status() == 0
    at = torch.tensor([0, 1, 2, 1 << 28, (1 << 28) + 1, n // 2, n - 3, n - 2, n - 1])
    _check(out[at.cuda()], _expect(q.expand(9, 1, d), w["q"], 1e-6, freq, at, False), torch.bfloat16)
    _check(cache.k[0, 0, :3, None].cpu(), _expect(k.expand(3, 1, d), w["k"], 1e-6, freq, at[-3:], False), torch.bfloat16)
    assert torch.equal(cache.v[0, 0, :3].cpu(), v[0].expand(3, d)) and (cache.k[0, 0, 3:] == 0).all() and (cache.v[0, 0, 3:] == 0).all()


def test_captured_call_on_another_stream():
    """Recorded once and replayed with new inputs in between, on a stream of its own, beside eager calls."""
    rng = np.random.default_rng(10)
    Hq, Hkv, d = 8, 2, 128
    _, _, rotation = _rotation(rng, d, d, False, "qk", 1e4)
    q, k, v = (pu.rnd(rng, 4, H, d).cuda() for H in (Hq, Hkv, Hkv))
    positions, slots = _i32([3, 4, 5, 6]), torch.tensor([0, 17, 33, -1], device="cuda")
    shape, ctx = binding.make_shape(1, Hq, Hkv, d, 1, 4, 1, "bf16"), binding.Context(workspace=0)
    cache, other = (_cache(_pool("e2m1", 3, Hkv, 16, d)) for _ in range(2))
    a, b = torch.empty_like(q), torch.empty_like(q)
    call = lambda out, c: ctx.ls_norm_rotate(shape, rotation, q, k, out, None, positions, c, v, slots)
    print("rotate captured", flush=True)
    call(a, cache)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        call(a, cache)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(pu.rnd(rng, *x.shape))
        positions.add_(1000)
        slots.copy_(torch.tensor([i, 20 - i, -1, 40 + i]))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        call(b, other)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        if i == 0:
            for n in ("k", "v", "k_exp", "v_exp"):           # (what the eager call and the recording itself left)
                getattr(other, n).copy_(getattr(cache, n))
        else:
            x, y = _host(cache), _host(other)
            assert all(torch.equal(x[n], y[n]) for n in x)


def test_what_the_binding_refuses():
    f32 = lambda *s: torch.zeros(*s, device="cuda")
    for bad in (lambda: binding.Rotation(f32(4, 16)), lambda: binding.Rotation(f32(32).double()), lambda: binding.Rotation(f32(32).cpu()),
                lambda: binding.Rotation(f32(64)[::2]), lambda: binding.Rotation(f32(32), q_weight=f32(64).bfloat16())):
        with pytest.raises(ValueError):
            bad()
    ctx, shape = binding.Context(workspace=0), binding.make_shape(1, 4, 2, 64, 1, 3, 1, "bf16")
    row = lambda H, n=3: torch.zeros(n, H, 64, dtype=torch.bfloat16, device="cuda")
    cache = binding.PagedCache(*(torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    good = binding.Rotation(f32(32), q_weight=f32(64))
    call = lambda rot=good, q=row(4), k=row(2), oq=row(4), ok=row(2), **kw: ctx.ls_norm_rotate(shape, rot, q, k, oq, ok, **kw)
    call()
    call(cache=cache, v=row(2), slots=slots)
    for kw in (dict(q=row(3)), dict(q=row(4).float()), dict(k=row(2, 4)), dict(q=row(4).cpu()), dict(oq=None), dict(positions=slots), dict(positions=slots.int()[:2]), dict(cache=cache),
               dict(cache=cache, v=row(2)), dict(v=row(2), slots=slots), dict(cache=cache, v=row(2), slots=slots.int()), dict(rot=binding.Rotation(f32(32), q_weight=f32(128))),
               dict(q=row(4)[None].transpose(1, 2), k=row(2))):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(ok=None), dict(rot=binding.Rotation(f32(4))), dict(rot=binding.Rotation(f32(40))), dict(rot=binding.Rotation(f32(32), eps=-1.0)), dict(rot=binding.Rotation(f32(32), eps=float("nan"))),
               dict(rot=binding.Rotation(f32(33)[1:])), dict(oq=row(1).expand(3, 4, 64)),
               dict(cache=binding.PagedCache(*(torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))), v=row(2), slots=slots)):
        with pytest.raises(binding.LoopServeError):
            call(**kw)
