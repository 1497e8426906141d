"""Calls on pages and packed sequences at the ends of what they allow: many sequences, many rows, infinities across parts, every exponent byte."""
import sys

import numpy as np
import pytest
import torch

import paper_2507_13681_amd as package
from paper_2507_13681_amd import binding
from tests import paged_util as pu
from tests.test_gpu_cache import _attend, _i32
from tests.test_gpu_packed import _check, _inputs, _run, _starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv", [(2, 1), (4, 2), (6, 3), (8, 8), (16, 16)])
@pytest.mark.parametrize("at", [0, 63, 64, 100, 129])
@pytest.mark.parametrize("which", ["both", "q", "k"])
def test_starts_that_are_none_behind_many_sequences(Hq, Hkv, at, which):
    """130 sequences, of which one's starts descend: it and all behind it are passed by, and the status word says so, wherever it stands."""
    rng = np.random.default_rng(at + Hq)
    lens = [int(x) for x in rng.choice([0, 1, 5, 33, 40], 130)]
    lens[at] = max(lens[at], 1)
    T = sum(lens)
    q, k, v = _inputs(at, Hq, Hkv, 64, lens, lens, torch.bfloat16)
    good = _starts(lens)
    bad = good.clone()
    bad[at + 1:] = bad[at] - 1                             # (of sequence 0: leaves the rows)
    qs, ks = (bad if which != "k" else good).cuda(), (bad if which != "q" else good).cuda()
    shape = binding.make_shape(130, Hq, Hkv, 64, T, T, 1, "bf16")
    ctx = binding.Context(workspace=binding.packed_workspace_bytes(shape))
    out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((Hq, T), 5.0, device="cuda")
    print("packed bad starts", Hq, Hkv, at, which, flush=True)
    ctx.ls_packed_prefill(shape, q.cuda(), k.cuda(), v.cuda(), qs, ks, out, lse)
    status = ctx.ls_poll_status()
    end = int(good[at])
    assert (out[end:] == 5.0).all() and (lse[:, end:] == 5.0).all()
    _check(q[:end], k[:end], v[:end], lens[:at], lens[:at], out[:end].cpu(), lse[:, :end].cpu())
    assert status == binding.LS_STAT_STARTS


def _odd_columns(n, d):
    """(key, column, value): infinities all over the keys, a column each; a NaN; both infinities in one column."""
    at = [(int(i * (n - 1) / (d - 5)), i, float("inf") if i % 2 else -float("inf")) for i in range(d - 4)]
    return at + [(n // 3, d - 4, float("nan")), (n // 5, d - 3, float("inf")), (n - 1 - n // 5, d - 3, -float("inf"))]


def _same_with_odd(out, got, want):
    """got: what `out` becomes where `want` is not finite; the same bits elsewhere."""
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[fine], out[fine]) and torch.equal(got[torch.isinf(want)].double(), want[torch.isinf(want)].double())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,keys,rows", [(128, 4000, 20), (64, 4000, 20), (128, 2777, 40), (64, 300, 300)])
def test_infinite_values_of_cut_items(d, keys, rows, dtype):
    """Single infinities in V reach the rows that see them in whichever part of an item they are, as in a whole one."""
    q, k, v = _inputs(31, 4, 2, d, [keys], [rows], dtype, scale=0.5)
    print("packed odd parts", d, keys, rows, dtype, flush=True)
    v2 = v.clone()
    for r, c, x in _odd_columns(keys, d):
        v2[r, 0, c] = x
    for room in (None, 0):                                 # in parts, and whole
        out, lse = _run(q, k, v, [keys], [rows], room=room)
        got, got_lse = _run(q, k, v2, [keys], [rows], room=room)
        want = out.double().clone()
        for r, c, x in _odd_columns(keys, d):
            want[max(0, r - (keys - rows)):, :2, c] += x
        _same_with_odd(out, got, want)
        assert torch.equal(lse, got_lse)


@pytest.mark.parametrize("lens,Hq,Hkv,d", [
    ([70, 70], 8, 2, 128),                           # one workgroup a head
    ([2000, 2000], 4, 2, 128),                       # parts, put together by the last of them
    ([1900], 4, 2, 64),
    ([5003], 32, 1, 64),                             # parts, put together by a launch of their own
    ([5003], 32, 1, 128), ([20000], 17, 1, 128)])
def test_infinite_values_of_pages(lens, Hq, Hkv, d):
    """Single infinities in V, however many parts there are and whoever puts them together."""
    print("paged odd values", lens, Hq, Hkv, d, flush=True)
    rng = np.random.default_rng(19)
    pages = sum(-(-n // 16) for n in lens)
    p = pu.pool(rng, pages, Hkv, 16, d, "bf16")
    q, table = pu.rnd(rng, len(lens), Hq, d, scale=0.5), pu.table_for(rng, lens, 16, pages)
    out, lse, _ = _attend(p, q, table, lens)
    want = out.double().clone()
    for r, c, x in _odd_columns(lens[0], d):
        p["v"][table[0, r // 16].long(), 0, r % 16, c] = x
        want[0, :Hq // Hkv, c] += x
    got, got_lse, status = _attend(p, q, table, lens, times=2)
    assert status == 0
    _same_with_odd(out, got, want)
    assert torch.equal(lse, got_lse)


@pytest.mark.parametrize("d,n", [(64, (1 << 29) + 5), (128, (1 << 28) + 5)])
def test_more_rows_than_a_launch_has_threads_for(d, n):
    """Rows whose places take more than 2^32 threads to find (the rows share one place in memory): the last five are written, packed and padded."""
    rows = pu.rnd(np.random.default_rng(1), 1, 1, d).cuda()
    pool = torch.zeros(1, 1, 16, d, dtype=torch.bfloat16, device="cuda")
    ctx, table = binding.Context(workspace=0), _i32([[0]])
    print("cache many rows", d, n, flush=True)
    cache = binding.PagedCache(pool.clone(), pool.clone())
    ctx.ls_cache_write(binding.make_shape(1, 1, 1, d, 1, n, 1, "bf16"), cache, rows.expand(n, 1, d), rows.expand(n, 1, d), table, starts=_i32([n - 5, n]))
    assert ctx.ls_poll_status() == 0
    for x in (cache.k, cache.v):
        assert torch.equal(x[0, 0, :5], rows[0].expand(5, d)) and (x[0, 0, 5:] == 0).all()
    cache = binding.PagedCache(pool.clone(), pool.clone())
    padded = rows[None].expand(2, 1, n // 2, d)
    ctx.ls_cache_write(binding.make_shape(2, 1, 1, d, 1, n // 2, 1, "bf16"), cache, padded, padded, _i32([[-1], [0]]), count=_i32([0, 3]))
    assert ctx.ls_poll_status() == 0
    for x in (cache.k, cache.v):
        assert torch.equal(x[0, 0, :3], rows[0].expand(3, d)) and (x[0, 0, 3:] == 0).all()


def _every_byte(part):
    """64 codes, a row of them for each exponent byte, and the values that they stand for."""
    codes = (torch.arange(64) + 64 * part).to(torch.uint8)
    value = codes.view(pu.E4M3).double()[None] * torch.exp2(torch.arange(256).double() - 127)[:, None]
    value[255] = float("nan")
    return codes, value


def _equal(got, want):
    return ((got == want) | (torch.isnan(got) & torch.isnan(want))).all(-1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("part", [0, 1, 2, 3])
def test_every_exponent_byte_is_read(part, dtype):
    """code * 2^(E - 127), rounded to the rows' type; 255: no number."""
    codes, value = _every_byte(part)
    k = codes.expand(16, 1, 16, 64).contiguous().cuda()
    E = torch.arange(256).to(torch.uint8).view(16, 1, 16).cuda()
    rows = [torch.zeros(256, 1, 64, dtype=dtype, device="cuda") for _ in range(2)]
    print("cache bytes", part, dtype, flush=True)
    binding.Context(workspace=0).ls_cache_read(binding.make_shape(1, 1, 1, 64, 1, 256, 1, dtype), binding.PagedCache(k, k.clone(), E, E.clone()),
                                               torch.arange(16, dtype=torch.int32, device="cuda")[None], *rows, starts=_i32([0, 256]))
    torch.cuda.synchronize()
    for x in rows:
        same = _equal(x[:, 0].cpu(), value.to(dtype))
        assert same.all(), torch.nonzero(~same)[:, 0].tolist()


@pytest.mark.parametrize("part", [0, 1, 2, 3])
def test_every_exponent_byte_is_attended_to(part):
    """One key a sequence, whose output is its row of V; with an equal row at the byte 0 or 255 behind the length, which does not matter."""
    codes, value = _every_byte(part)
    v = codes.expand(256, 1, 16, 64).contiguous()
    E = torch.arange(256).to(torch.uint8)[:, None, None].expand(256, 1, 16).contiguous()
    E[:, :, 1] = 255
    p = dict(k=torch.full((256, 1, 16, 64), 0x38, dtype=torch.uint8), v=v, k_exp=torch.full((256, 1, 16), 127, dtype=torch.uint8), v_exp=E)
    print("paged bytes of V", part, flush=True)
    out, _, status = _attend(p, torch.ones(256, 1, 64).bfloat16(), torch.arange(256, dtype=torch.int32)[:, None], [1] * 256)
    assert status == 0
    same = _equal(out[:, 0], value.to(torch.bfloat16))
    assert same.all(), torch.nonzero(~same)[:, 0].tolist()


def test_every_exponent_byte_of_keys():
    """Logits of single keys: a query that is a power of two in one column brings the stored value, as bf16 has it, near one; the normaliser of one key is its logit."""
    codes, value = _every_byte(0)
    bits = torch.arange(256)
    E = bits.to(torch.uint8)[:, None, None].expand(256, 1, 16).contiguous()
    p = dict(k=codes.expand(256, 1, 16, 64).contiguous(), v=torch.full((256, 1, 16, 64), 0x38, dtype=torch.uint8), k_exp=E, v_exp=torch.full((256, 1, 16), 127, dtype=torch.uint8))
    back = torch.exp2((127 - bits).clamp_min(-126).double())
    for col in (1, 3, 8, 9, 40, 63):
        q = torch.zeros(256, 1, 64, dtype=torch.bfloat16)
        q[:, 0, col] = back.to(torch.bfloat16)
        print("paged bytes of K", col, flush=True)
        out, lse, _ = _attend(p, q, bits.int()[:, None], [1] * 256, scale=1.0)
        x, got = value.to(torch.bfloat16).double()[:, col] * back, lse[:, 0].double()
        nan = torch.isnan(x)
        # the factor log2(e), the product with it, the factor ln(2) and the product with that: 2^-24 each
        assert torch.equal(torch.isnan(got), nan) and ((got - x).abs() <= 2.0 ** -22 * x.abs())[~nan].all(), col
        assert (out[~nan] == 1.0).all() and torch.isnan(out[nan]).all()


@pytest.mark.parametrize("n,at", [(2, 1), (40, 35), (40, 3), (64, 50)])
@pytest.mark.parametrize("how", ["byte", "code", "bf16"])
def test_a_value_that_is_none_and_weighs_nothing(how, n, at):
    """A key that is seen with a weight of 0 in fp32, and whose row of V is no number, in whole and partial tiles: 0 times NaN."""
    rng = np.random.default_rng(44)
    kind = "bf16" if how == "bf16" else "e4m3"
    p = pu.pool(rng, 4, 1, 16, 64, kind)
    k = torch.zeros(4, 1, 16, 64)
    k[..., 0] = 1.0
    k[at // 16, 0, at % 16, 0] = -8.0
    if kind == "bf16":
        p["k"], p["v"][at // 16, 0, at % 16] = k.bfloat16(), float("nan")
    else:
        p["k_exp"] = pu.exponents(k)
        p["k"] = pu.codes(k, p["k_exp"])
        p["v_exp" if how == "byte" else "v"][at // 16, 0, at % 16] = 255 if how == "byte" else 0x7F
    q = torch.zeros(1, 2, 64).bfloat16()
    q[..., 0] = 100.0
    print("paged weightless", how, n, at, flush=True)
    out, lse, status = _attend(p, q, torch.arange(4, dtype=torch.int32)[None], [n], scale=1.0)
    assert status == 0 and torch.isnan(out).all() and torch.isfinite(lse).all()


def test_a_context_without_the_module_of_pages(monkeypatch):
    """It is loaded by the first call on pages or packed sequences, and no other call needs it."""
    monkeypatch.delitem(sys.modules, "paper_2507_13681_amd._lspages", raising=False)
    monkeypatch.delattr(package, "_lspages", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2507_13681_amd._lspages", None)
    rng = np.random.default_rng(45)
    q, k = pu.rnd(rng, 1, 2, 1, 64).cuda(), pu.rnd(rng, 1, 1, 5, 64).cuda()
    shape = binding.make_shape(1, 2, 1, 64, 5, 1, 1, "bf16")
    print("context without pages", flush=True)
    ctx = binding.Context(workspace=1 << 20)
    out = torch.full_like(q[:, :, 0], float("nan"))
    ctx.ls_decode_attend(shape, q[:, :, 0].contiguous(), k, k, None, None, None, out)
    assert ctx.ls_poll_status() == 0 and torch.isfinite(out).all()
    with pytest.raises(binding.LoopServeError, match="_lspages"):
        ctx.ls_packed_prefill(shape, q, k, k, None, None, torch.empty_like(q))
    monkeypatch.undo()
    whole = torch.full_like(q, float("nan"))
    ctx.ls_packed_prefill(shape, q, k, k, None, None, whole)
    torch.cuda.synchronize()
    assert torch.isfinite(whole).all()


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_as_large_as_the_header_allows(sign, dtype):
    """Up to 2^30 in magnitude, 2^24 apart: each row is the value of the largest key that it sees, by its weight as the type has it, and its normaliser that key's logit."""
    n, d = 64, 64
    rng = np.random.default_rng(46)
    order = torch.from_numpy(rng.permutation(n))
    q, k, v = torch.zeros(n, 2, d), torch.zeros(n, 1, d), pu.rnd(rng, n, 1, d, dtype=dtype)
    q[..., 0], k[:, 0, 0] = 2.0 ** 15, (order + 1).float() * 2.0 ** 9 * sign
    q, k = q.to(dtype), k.to(dtype)
    print("packed largest logits", sign, dtype, flush=True)
    out, lse = _run(q, k, v, [n], [n], scale=1.0)
    step = pu.HALF[dtype]
    x = (k[:, 0, 0].double() * 2.0 ** 15)
    for i in range(n):
        best = int(x[:i + 1].argmax())
        want = v[best, 0].double()
        # the weight and the result are rounded once each in bf16; in fp32 the division and the product
        assert ((out[i].double() - want).abs() <= 2.02 * step * want.abs()).all()
        assert ((lse[:, i].double() - x[best]).abs() <= 2.0 ** -22 * x[best].abs()).all()
    if dtype == torch.float32:
        return
    p = dict(k=k.view(4, 1, 16, d).contiguous(), v=v.view(4, 1, 16, d).contiguous())
    out, lse, _ = _attend(p, q[:1], torch.arange(4, dtype=torch.int32)[None], [n], scale=1.0)
    best = int(x.argmax())
    assert ((out[0].double() - v[best, 0].double()).abs() <= 2.02 * step * v[best, 0].double().abs()).all()
    assert ((lse[0].double() - x[best]).abs() <= 2.0 ** -22 * x[best].abs()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (4, 4, 128), (8, 2, 128)])
def test_a_row_does_not_depend_on_its_neighbours_logits(Hq, Hkv, d, dtype):
    """One row whose logits rise from step to step, so that its reference moves all the time: all others have the same bits as without that."""
    n, at = 300, 159
    q, k, v = _inputs(47, Hq, Hkv, d, [n], [n], dtype, scale=0.6)
    q[..., 1], k[..., 1] = 0.0, (torch.arange(n) // 32).to(dtype)[:, None]
    print("packed neighbour", Hq, Hkv, d, dtype, flush=True)
    out, lse = _run(q, k, v, [n], [n], room=0)
    q[at, :, 1] = 8.0 * d ** 0.5
    got, got_lse = _run(q, k, v, [n], [n], room=0)
    others = torch.arange(n) != at
    assert torch.equal(got_lse[:, others], lse[:, others]) and torch.equal(got[others], out[others])
    assert not torch.equal(got[at], out[at])


N_MOST = 2147483000                                        # the most rows that a call takes


def test_the_longest_sequence_of_a_prompt():
    """A row on as many keys as there can be (all in one place): equal weights, whose number the normaliser counts."""
    v = torch.exp2(torch.randint(-3, 4, (1, 1, 64)).float()).bfloat16().cuda()
    q, k = torch.zeros(2, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    shape = binding.make_shape(1, 1, 1, 64, N_MOST, 2, 1, "bf16")
    out, lse = torch.empty_like(q), torch.empty(1, 2, device="cuda")
    ctx = binding.Context(workspace=binding.packed_workspace_bytes(shape))
    print("packed longest", flush=True)
    ctx.ls_packed_prefill(shape, q, k.expand(N_MOST, 1, 64), v.expand(N_MOST, 1, 64), _i32([0, 2]), _i32([0, N_MOST]), out, lse)
    torch.cuda.synchronize()
    assert torch.equal(out, v.expand(2, 1, 64))            # (sums of powers of two: exact)
    assert (lse.double() - np.log(N_MOST)).abs().max() <= 2.0 ** -20 * np.log(N_MOST)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_the_longest_sequence_of_pages(kind):
    """A token on as many keys as there can be, all on one page, behind another sequence of 33."""
    p = pu.pool(np.random.default_rng(48), 1, 1, 256, 64, kind)
    row = torch.exp2(torch.randint(-3, 4, (64,)).float())
    if kind == "bf16":
        p["v"][:] = row.bfloat16()
    else:
        p["v"][:], p["v_exp"][:] = row.to(pu.E4M3).view(torch.uint8), 127
    table = torch.zeros(2, -(-N_MOST // 256), dtype=torch.int32)
    print("paged longest", kind, flush=True)
    out, lse, status = _attend(p, torch.zeros(2, 2, 64).bfloat16(), table, [33, N_MOST])
    assert status == 0 and torch.equal(out, row.bfloat16().expand(2, 2, 64))
    n = torch.tensor([33.0, N_MOST]).double().log()[:, None]
    assert ((lse.double() - n).abs() <= 2.0 ** -20 * n).all()


def test_as_many_sequences_as_there_can_be():
    """65535 of them, a row or none each: what a single key gives is its row of V."""
    B, d = 65535, 64
    rng = np.random.default_rng(49)
    lens = [int(x) for x in rng.choice([0, 1], B)]
    T = sum(lens)
    q, k, v = (pu.rnd(rng, T, 1, d).cuda() for _ in range(3))
    starts = _starts(lens).cuda()
    shape = binding.make_shape(B, 1, 1, d, T, T, 1, "bf16")
    ctx = binding.Context(workspace=max(binding.packed_workspace_bytes(shape), binding.paged_workspace_bytes(binding.make_shape(B, 1, 1, d, 1, 1, 1, "bf16"))))
    out = torch.full_like(q, float("nan"))
    print("many sequences: packed", flush=True)
    ctx.ls_packed_prefill(shape, q, k, v, starts, starts, out)
    assert ctx.ls_poll_status() == 0 and torch.equal(out, v)
    pool = torch.zeros(B, 1, 16, d, dtype=torch.bfloat16, device="cuda")
    cache = binding.PagedCache(pool, pool.clone())
    table, pos = torch.from_numpy(rng.permutation(B).astype(np.int32))[:, None].cuda().contiguous(), _i32([0] * B)
    print("many sequences: pages", flush=True)
    ctx.ls_cache_write(binding.make_shape(B, 1, 1, d, 1, T, 1, "bf16"), cache, k, v, table, pos, starts)
    seq = torch.tensor(lens).nonzero()[:, 0].cuda()
    assert ctx.ls_poll_status() == 0 and torch.equal(cache.v[table[seq, 0].long(), 0, 0], v[:, 0]) and torch.equal(cache.k[table[seq, 0].long(), 0, 0], k[:, 0])
    token = torch.full((B, 1, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    print("many sequences: tokens", flush=True)
    ctx.ls_paged_attend(binding.make_shape(B, 1, 1, d, 1, 1, 1, "bf16"), cache, torch.ones_like(token), table, _i32(lens), token)
    want = torch.zeros_like(token)
    want[seq] = v
    assert ctx.ls_poll_status() == 0 and torch.equal(token, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,seen", [(70, 50), (70, 69), (70, None), (3000, 5), (3000, None)])
def test_logits_of_minus_infinity(n, seen, dtype):
    """They weigh nothing: one finite key gives its row of V, and rows without any are as rows without a key; whole items and parts."""
    q, k, v = _inputs(50, 4, 1, 64, [n], [3], dtype)
    q, k[..., 0] = q.abs(), -float("inf")
    if seen is not None:
        k[seen, 0, 0] = 1.0
    print("packed minus infinity", n, seen, dtype, flush=True)
    out, lse = _run(q, k, v, [n], [3])
    sees = torch.arange(n - 3, n) >= (n if seen is None else seen)
    want = torch.where(sees[:, None, None], v[seen or 0], torch.zeros(())).expand(3, 4, 64)
    assert ((out.double() - want.double()).abs() <= pu.HALF[dtype] * 2.02 * want.double().abs()).all()
    assert torch.equal(torch.isneginf(lse), ~sees.expand(4, 3)) and not torch.isnan(lse).any()
    if dtype == torch.bfloat16:
        pages = -(-n // 16)
        p = {name: torch.zeros(pages, 1, 16, 64, dtype=dtype) for name in "kv"}
        p["k"].view(-1, 64)[:n], p["v"].view(-1, 64)[:n] = k[:, 0], v[:, 0]
        token, tl, status = _attend(p, q[2:], torch.arange(pages, dtype=torch.int32)[None], [n])
        assert status == 0 and ((token[0].double() - want[2].double()).abs() <= pu.HALF[dtype] * 2.02 * want[2].double().abs()).all()
        assert torch.isneginf(tl).all() == (seen is None) and not torch.isnan(tl).any()
