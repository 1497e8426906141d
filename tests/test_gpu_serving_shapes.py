"""Seeded random shapes through the calls on pages and packed sequences, and forms of them that the lists of cases leave out."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests import paged_util as pu
from tests.test_gpu_cache import _attend, _cache, _host, _i32, _places, _same, _written
from tests.test_gpu_cache import _check as _check_token
from tests.test_gpu_packed import _check, _inputs, _run

pytestmark = pytest.mark.gpu


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("seed", range(30))
def test_packed_shapes(seed):
    rng = np.random.default_rng(1000 + seed)
    Hkv, G, d = int(rng.choice([1, 2, 3, 4, 5, 8, 16])), int(rng.choice([1, 2, 3, 4, 7, 8, 33])), int(rng.choice([64, 128]))
    dtype = torch.float32 if seed % 3 == 0 else torch.bfloat16
    B = int(rng.choice([1, 2, 5, 17, 64, 65, 100]))
    most = max(40, 12000 // (B * (1 + Hkv * G // 16)))
    keys = [_log(rng, 1, most) - int(rng.random() < 0.1) for _ in range(B)]
    rows = [int(r) for r in (keys if rng.random() < 0.4 else [min(_log(rng, 1, 60), k + int(rng.integers(0, 3))) for k in keys])]
    if sum(rows) == 0 or sum(keys) == 0:
        keys[0] = rows[0] = 1
    print("packed shape", seed, Hkv, G, d, dtype, B, keys[:6], rows[:6], flush=True)
    q, k, v = _inputs(seed, Hkv * G, Hkv, d, keys, rows, dtype)
    out, lse = _run(q, k, v, keys, rows)
    _check(q, k, v, keys, rows, out, lse, heads=sorted({0, int(rng.integers(Hkv * G)), Hkv * G - 1}))


@pytest.mark.parametrize("seed", range(30))
def test_token_shapes(seed):
    rng = np.random.default_rng(2000 + seed)
    Hkv, G, d, page = int(rng.choice([1, 2, 3, 8, 20])), int(rng.choice([1, 2, 5, 16, 17, 32])), int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 128, 256]))
    kind = "e4m3" if seed % 2 else "bf16"
    B = int(rng.choice([1, 2, 7, 40, 64, 65, 90]))
    lens = [_log(rng, 1, max(60, 60000 // (B * Hkv))) - int(rng.random() < 0.1) for _ in range(B)]
    pages = max(1, sum(-(-n // page) for n in lens))
    print("paged shape", seed, Hkv, G, d, page, kind, B, lens[:6], flush=True)
    p = pu.pool(rng, pages, Hkv, page, d, kind)
    q, table = pu.rnd(rng, B, Hkv * G, d, scale=1.5), pu.table_for(rng, lens, page, pages)
    out, lse, status = _attend(p, q, table, lens, n=int(max(1, max(lens)) * rng.choice([1, 1, 3])), times=2)
    assert status == 0
    _check_token(p, q, table, lens, out, lse)


@pytest.mark.parametrize("seed", range(20))
def test_moved_shapes(seed):
    rng = np.random.default_rng(3000 + seed)
    Hkv, d, page = int(rng.choice([1, 2, 3, 7, 8, 32])), int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 128, 256]))
    kind, dtype, packed = ["bf16", "e4m3"][seed % 2], [torch.bfloat16, torch.float32][seed // 2 % 2], seed % 3 > 0
    lens = [_log(rng, 1, 400) - int(rng.random() < 0.2) for _ in range(int(rng.choice([1, 2, 9, 300 // Hkv])))]
    lens[0] = max(lens[0], 1)
    pos = [int(x) for x in rng.integers(0, 3 * page, len(lens))]
    ends = [a + n for a, n in zip(pos, lens)]
    pages = sum(-(-e // page) for e in ends)
    print("cache shape", seed, Hkv, d, page, kind, dtype, packed, lens[:6], flush=True)
    p, table, B, most = pu.pool(rng, pages, Hkv, page, d, kind), pu.table_for(rng, ends, page, pages), len(lens), max(lens)
    rows = [pu.rnd(rng, sum(lens), Hkv, d, scale=s, dtype=dtype) for s in (1.0, 30.0)]
    places, cache = _places(lens, pos, table, page), _cache(p)
    if packed:
        dev, kw = [x.cuda() for x in rows], dict(starts=_i32(np.concatenate([[0], np.cumsum(lens)])))
    else:
        dev, kw = [torch.full((B, Hkv, most, d), float("nan"), dtype=dtype) for _ in rows], dict(count=_i32(lens))
        s, i = (torch.tensor([x[j] for x in places]) for j in (0, 1))
        for x, y in zip(rows, dev):
            y[s, :, i] = x
        dev = [x.cuda() for x in dev]
    shape = binding.make_shape(B, Hkv, Hkv, d, 1, sum(lens) if packed else most, 1, dtype)
    ctx = binding.Context(workspace=0)
    ctx.ls_cache_write(shape, cache, *dev, table.cuda(), _i32(pos), **kw)
    assert ctx.ls_poll_status() == 0
    want = {n: x.clone() for n, x in p.items()}
    for name, x in zip(("k", "v"), rows):
        _written(want, kind, x, places, name)
    assert _same(_host(cache), want)
    back = [torch.full_like(x, 7.0) for x in dev]
    ctx.ls_cache_read(shape, cache, table.cuda(), *back, _i32(pos), **kw)
    assert ctx.ls_poll_status() == 0
    s, i, pg, pl = (torch.tensor([x[j] for x in places]) for j in range(4))
    for name, got in zip(("k", "v"), back):
        ref = torch.full_like(got.cpu(), 7.0)
        x = pu.stored(want, name)[pg, :, pl].to(dtype)
        if packed:
            ref[:] = x
        else:
            ref[s, :, i] = x
        assert torch.equal(got.cpu(), ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("G,Hkv,d,keys,rows", [
    (33, 1, 64, [70, 3], [70, 3]), (64, 2, 128, [50, 0, 31], [50, 2, 31]), (128, 1, 128, [40, 33], [40, 1]),
    (200, 1, 64, [37, 64], [37, 5]),                       # one query spans blocks
    (130, 1, 128, [3000], [2]), (64, 2, 64, [2500, 40], [5, 40])])           # cut items
def test_many_query_heads_of_a_kv_head(G, Hkv, d, keys, rows, dtype):
    print("packed many heads", G, Hkv, d, keys, rows, dtype, flush=True)
    q, k, v = _inputs(41, G * Hkv, Hkv, d, keys, rows, dtype)
    out, lse = _run(q, k, v, keys, rows)
    _check(q, k, v, keys, rows, out, lse, heads=sorted({0, 1, G // 2, G - 1, G * Hkv - 1}))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv,d,n,m", [(3, 4, 2, 64, 4000, 20), (2, 8, 2, 128, 5003, 33), (1, 6, 3, 128, 3000, 1)])
def test_cut_items_of_a_padded_batch(B, Hq, Hkv, d, n, m, dtype):
    rng = np.random.default_rng(42)
    q, k, v = pu.rnd(rng, B, Hq, m, d, dtype=dtype), pu.rnd(rng, B, Hkv, n, d, dtype=dtype), pu.rnd(rng, B, Hkv, n, d, dtype=dtype)
    shape = binding.make_shape(B, Hq, Hkv, d, n, m, 1, dtype)
    units = (C.c_int64 * 2)()
    assert binding.load_library().ls_debug_packed_units(C.byref(shape), 0, units) == 0 and units[0] > 0
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(B, Hq, m, device="cuda")
    print("packed padded, cut", B, Hq, Hkv, d, n, m, dtype, flush=True)
    ctx = binding.Context(workspace=binding.packed_workspace_bytes(shape))
    ctx.debug_fill_workspace(0x7FC00000)
    ctx.ls_packed_prefill(shape, q.cuda(), k.cuda(), v.cuda(), None, None, out, lse)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(Hq):
            g = h // (Hq // Hkv)
            pu.check(out[b, h].cpu(), lse[b, h].cpu(), pu.attention(q[b, h], k[b, g], v[b, g], np.arange(n - m, n), d ** -0.5), dtype)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_few_rows_of_a_wide_padded_batch(kind):
    """Rows enough in the tensors that their pages are read past the caches, of which the counts leave a few."""
    rng = np.random.default_rng(43)
    B, H, d, n, page = 2, 8, 128, 40000, 64
    p, lens = pu.pool(rng, 20, H, page, d, kind), [130, 7]
    assert B * n * H * 2 * d * (4 if kind == "bf16" else 3) > 256 << 20
    table = pu.table_for(rng, [500, 7], page, 20)
    rows = [torch.full((B, H, n, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx = binding.Context(workspace=0)
    print("read few of a wide batch", kind, flush=True)
    ctx.ls_cache_read(binding.make_shape(B, H, H, d, n, n, 1, "bf16"), _cache(p), table.cuda(), *rows, pos=_i32([370, 0]), count=_i32(lens))
    assert ctx.ls_poll_status() == 0
    for name, got in zip(("k", "v"), rows):
        held = pu.stored(p, name).to(torch.bfloat16)
        for b, (m, first) in enumerate(zip(lens, (370, 0))):
            at = torch.arange(m) + first
            assert torch.equal(got[b, :, :m].cpu().transpose(0, 1), held[table[b, at // page].long(), :, at % page])
            assert (got[b, :, m:] == 7.0).all()
