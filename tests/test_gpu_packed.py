"""ls_packed_prefill against attention in 64 bits: lengths, heads, types, strides, rows without keys, cut items, refusals."""
import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


def _starts(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32)


def _inputs(seed, Hq, Hkv, d, keys, rows, dtype, scale=1.3):
    rng = np.random.default_rng(seed)
    return (pu.rnd(rng, sum(rows), Hq, d, scale=scale, dtype=dtype), pu.rnd(rng, sum(keys), Hkv, d, dtype=dtype), pu.rnd(rng, sum(keys), Hkv, d, dtype=dtype))


def _context(shape, room=None):
    return binding.Context(workspace=binding.packed_workspace_bytes(shape) if room is None else room)


def _run(q, k, v, keys, rows, lse=True, room=None, scale=0.0):
    Hq, Hkv, d = q.shape[1], k.shape[1], q.shape[2]
    shape = binding.make_shape(len(keys), Hq, Hkv, d, k.shape[0], q.shape[0], 1, q.dtype, scale)
    ctx = _context(shape, room)
    ctx.debug_fill_workspace(0x7FC00000) if ctx.workspace else None
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    ls = torch.full((Hq, q.shape[0]), float("nan"), device="cuda") if lse else None
    ctx.ls_packed_prefill(shape, q.cuda(), k.cuda(), v.cuda(), _starts(rows).cuda(), _starts(keys).cuda(), out, ls)
    torch.cuda.synchronize()
    assert ctx.ls_poll_status() == 0
    return out.cpu(), None if ls is None else ls.cpu()


def _check(q, k, v, keys, rows, out, lse, scale=None, heads=None):
    Hq, Hkv, d = q.shape[1], k.shape[1], q.shape[2]
    sk, sq = _starts(keys), _starts(rows)
    for s, (nk, nq) in enumerate(zip(keys, rows)):
        for h in heads or range(Hq):
            a, b = int(sq[s]), int(sk[s])
            ref = pu.attention(q[a:a + nq, h], k[b:b + nk, h // (Hq // Hkv)], v[b:b + nk, h // (Hq // Hkv)],
                               np.arange(nk - nq, nk), scale or d ** -0.5)
            pu.check(out[a:a + nq, h], None if lse is None else lse[h, a:a + nq], ref, q.dtype)


CASES = [
    # heads, d, keys, rows
    (4, 2, 128, [1], None),
    (4, 2, 128, [31, 32, 33, 1, 64], None),          # steps of 32 keys, and either side
    (8, 2, 128, [257, 0, 5, 128], None),             # an empty sequence among others
    (4, 4, 64, [300, 77], None),                     # a query head each
    (32, 1, 64, [70, 3], None),                      # 32 query heads of one KV head
    (12, 3, 128, [100, 45], None),                   # heads that share XCDs unevenly; four and ...
    (10, 2, 128, [90, 130], None),                   # ... five rows a query: blocks end inside one
    (3, 1, 64, [201], None),
    (16, 16, 128, [65], None),
    (24, 24, 64, [40, 40], None),
    (8, 2, 128, [700, 1200, 90], [61, 1, 90]),       # later turns
    (4, 1, 128, [3000], [2]),                        # few rows, many keys: cut into parts
    (4, 1, 64, [5003], [40]),
    (8, 8, 128, [1111, 900], [33, 129]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,d,keys,rows", CASES)
def test_matches_attention(Hq, Hkv, d, keys, rows, dtype):
    rows = rows or keys
    print("packed", Hq, Hkv, d, keys, rows, dtype, flush=True)
    q, k, v = _inputs(len(keys) + Hq, Hq, Hkv, d, keys, rows, dtype)
    out, lse = _run(q, k, v, keys, rows)
    _check(q, k, v, keys, rows, out, lse)


def test_more_sequences_than_are_sorted():
    """65 sequences and more go by sequence, and are not cut."""
    rng = np.random.default_rng(4)
    keys = [int(x) for x in rng.integers(0, 60, 150)]
    q, k, v = _inputs(9, 4, 2, 64, keys, keys, torch.bfloat16)
    print("packed 150 sequences", flush=True)
    out, lse = _run(q, k, v, keys, keys)
    _check(q, k, v, keys, keys, out, lse)


def test_items_beyond_what_is_resident():
    """More items than workgroups are resident: none is cut, the longest go first."""
    keys = [1500, 700, 3, 2000]
    q, k, v = _inputs(3, 32, 8, 64, keys, keys, torch.bfloat16)
    print("packed many items", flush=True)
    out, lse = _run(q, k, v, keys, keys)
    _check(q, k, v, keys, keys, out, lse, heads=[0, 13, 31])


@pytest.mark.parametrize("Hkv,keys", [(4, [100] * 50 + [2500]), (4, [2500] + [100] * 50), (8, [100] * 50 + [1000, 1, 0, 800, 1250])])
def test_one_long_sequence_among_short_ones(Hkv, keys):
    """More items than workgroups are resident; one so long that the sequences are put in order, and none."""
    q, k, v = _inputs(4, 4 * Hkv, Hkv, 128, keys, keys, torch.bfloat16)
    print("packed one long", Hkv, len(keys), flush=True)
    out, lse = _run(q, k, v, keys, keys)
    _check(q, k, v, keys, keys, out, lse, heads=[0, 7, 15])


@pytest.mark.parametrize("room", [0, 40 * (128 * 128 + 256) * 4])
def test_less_workspace(room):
    """Without room for parts items are whole, with some there are fewer parts."""
    keys, rows = [3000, 500], [7, 50]
    q, k, v = _inputs(5, 4, 2, 128, keys, rows, torch.bfloat16)
    print("packed room", room, flush=True)
    out, lse = _run(q, k, v, keys, rows, room=room)
    _check(q, k, v, keys, rows, out, lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_before_the_first_key(dtype):
    """More queries than keys: the first ones see none, and a sequence without keys leaves zeros."""
    keys, rows = [5, 0, 40], [150, 4, 41]
    q, k, v = _inputs(6, 4, 2, 64, keys, rows, dtype)
    print("packed empty rows", dtype, flush=True)
    out, lse = _run(q, k, v, keys, rows)
    _check(q, k, v, keys, rows, out, lse)
    assert (out[:145] == 0).all() and torch.isneginf(lse[:, :145]).all() and (out[150:154] == 0).all()


def test_scale_and_no_lse():
    keys = [90]
    q, k, v = _inputs(7, 4, 2, 128, keys, keys, torch.bfloat16)
    print("packed scale", flush=True)
    out, _ = _run(q, k, v, keys, keys, lse=False, scale=0.03)
    _check(q, k, v, keys, keys, out, None, scale=float(np.float32(0.03)))


@pytest.mark.parametrize("kind", ["fused", "head_major", "spread"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(kind, dtype):
    """q, k, v as slices of one projection, head by head, and with gaps; out head by head."""
    keys, (Hq, Hkv, d) = [200, 33], (6, 2, 128)
    q, k, v = _inputs(8, Hq, Hkv, d, keys, keys, dtype)
    T = sum(keys)
    if kind == "fused":
        x = torch.cat([q.reshape(T, -1), k.reshape(T, -1), v.reshape(T, -1)], 1).cuda()
        dq, dk, dv = (y.unflatten(1, (-1, d)) for y in x.split([Hq * d, Hkv * d, Hkv * d], 1))
    elif kind == "head_major":
        dq, dk, dv = (y.transpose(0, 1).contiguous().cuda().transpose(0, 1) for y in (q, k, v))
    else:
        def spread(y):
            z = torch.full((T * 3, y.shape[1] + 1, d + 16), float("nan"), dtype=dtype, device="cuda")
            z[::3, :-1, :d] = y.cuda()
            return z[::3, :-1, :d]
        dq, dk, dv = spread(q), spread(k), spread(v)
    shape = binding.make_shape(len(keys), Hq, Hkv, d, T, T, 1, dtype)
    whole = torch.full((Hq + 2, T + 5, d), 3.0, dtype=dtype, device="cuda")
    out = whole[1:-1, 2:-3].transpose(0, 1)
    print("packed strides", kind, dtype, flush=True)
    _context(shape).ls_packed_prefill(shape, dq, dk, dv, _starts(keys).cuda(), _starts(keys).cuda(), out)
    torch.cuda.synchronize()
    _check(q, k, v, keys, keys, out.cpu().contiguous(), None)
    whole[1:-1, 2:-3] = 3.0
    assert (whole == 3.0).all()                        # nothing beside the rows


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_padded_batch(dtype):
    """[B,H,n,d] without starts, as the other calls have it: equal lengths, and the last rows of each."""
    rng = np.random.default_rng(2)
    B, Hq, Hkv, d, n, m = 3, 4, 2, 64, 333, 50
    q, k, v = pu.rnd(rng, B, Hq, m, d, dtype=dtype), pu.rnd(rng, B, Hkv, n, d, dtype=dtype), pu.rnd(rng, B, Hkv, n, d, dtype=dtype)
    shape = binding.make_shape(B, Hq, Hkv, d, n, m, 1, dtype)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(B, Hq, m, device="cuda")
    print("packed padded", dtype, flush=True)
    _context(shape).ls_packed_prefill(shape, q.cuda(), k.cuda(), v.cuda(), None, None, out, lse)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(Hq):
            pu.check(out[b, h].cpu(), lse[b, h].cpu(), pu.attention(q[b, h], k[b, h // 2], v[b, h // 2], np.arange(n - m, n), d ** -0.5), dtype)


def test_rows_behind_the_last_sequence_stay():
    keys, T = [40, 25], 80
    q, k, v = _inputs(1, 4, 2, 64, [T], [T], torch.bfloat16)
    shape = binding.make_shape(2, 4, 2, 64, T, T, 1, "bf16")
    out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((4, T), 5.0, device="cuda")
    starts = torch.tensor([3, 43, 68], dtype=torch.int32, device="cuda")
    k[:3], k[68:], v[:3], v[68:] = (float("nan"),) * 4     # and rows of no sequence are not read
    print("packed rows behind", flush=True)
    _context(shape).ls_packed_prefill(shape, q.cuda(), k.cuda(), v.cuda(), starts, starts, out, lse)
    torch.cuda.synchronize()
    _check(q[3:68], k[3:68], v[3:68], keys, keys, out[3:68].cpu(), lse[:, 3:68].cpu())
    for x in (out[:3], out[68:], lse[:, :3], lse[:, 68:]):
        assert (x == 5.0).all()


@pytest.mark.parametrize("bad", [[0, 10, 5, 40], [0, 10, 41, 40], [-1, 10, 20, 40], [0, 10, 20, 41]])
def test_starts_that_are_none(bad):
    """From the first sequence whose starts descend or leave the rows on, nothing is computed, and the status word says so."""
    T = 40
    q, k, v = _inputs(1, 4, 2, 64, [T], [T], torch.bfloat16)
    shape = binding.make_shape(3, 4, 2, 64, T, T, 1, "bf16")
    starts = torch.tensor(bad, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 5.0, device="cuda")
    ctx = _context(shape)
    print("packed bad starts", bad, flush=True)
    ctx.ls_packed_prefill(shape, q.cuda(), k.cuda(), v.cuda(), starts, starts, out)
    assert ctx.ls_poll_status() == binding.LS_STAT_STARTS
    good = next(i for i in range(3) if not 0 <= bad[i] <= bad[i + 1] <= T)
    end = bad[good] if good else 0
    if good:
        lens = [bad[i + 1] - bad[i] for i in range(good)]
        _check(q[:end], k[:end], v[:end], lens, lens, out[:end].cpu(), None)
    assert (out[end:] == 5.0).all()


@pytest.mark.parametrize("step", [4.0, 40.0])
def test_logits_that_rise(step):
    """Every step of 32 keys has larger logits than the ones before: the reference moves all the time."""
    n, d = 600, 64
    rng = np.random.default_rng(0)
    q = torch.zeros(n, 2, d); q[..., 0] = 8.0
    k = pu.rnd(rng, n, 1, d, scale=0.1, dtype=torch.float32); k[:, 0, 0] = torch.arange(n) // 32 * step
    q, k, v = q.bfloat16(), k.bfloat16(), pu.rnd(rng, n, 1, d)
    print("packed rising", step, flush=True)
    out, lse = _run(q, k, v, [n], [n])
    _check(q, k, v, [n], [n], out, lse)


def test_a_captured_call_replays():
    """Into a graph and back, with eager work between, cut items and whole ones."""
    for keys, rows in (([900, 40], [30, 40]), ([300, 77], [300, 77])):
        q, k, v = _inputs(2, 4, 2, 128, keys, rows, torch.bfloat16)
        shape = binding.make_shape(2, 4, 2, 128, sum(keys), sum(rows), 1, "bf16")
        ctx = _context(shape)
        dq, dk, dv, out = q.cuda(), k.cuda(), v.cuda(), torch.empty_like(q, device="cuda")
        lse = torch.empty(4, sum(rows), device="cuda")
        qs, ks = _starts(rows).cuda(), _starts(keys).cuda()
        call = lambda: ctx.ls_packed_prefill(shape, dq, dk, dv, qs, ks, out, lse)
        print("packed graph", keys, flush=True)
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            call()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        for i in range(4):
            dq.copy_(torch.roll(q, i, 0))
            g.replay()
            torch.cuda.synchronize()
            got, got_lse = out.clone(), lse.clone()
            call()
            torch.cuda.synchronize()
            assert torch.equal(got, out) and torch.equal(got_lse, lse)


def test_what_the_binding_refuses():
    q, k, v = _inputs(1, 4, 2, 64, [40], [40], torch.bfloat16)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    st = _starts([40]).cuda()
    shape = binding.make_shape(1, 4, 2, 64, 40, 40, 1, "bf16")
    ctx, out = _context(shape), torch.empty_like(q)
    bad = [
        dict(q=q.float()), dict(q=q.cpu()), dict(k=k[:-1]), dict(v=v.transpose(1, 2)), dict(q_starts=st.long()), dict(q_starts=st[:1]),
        dict(out=out[None]), dict(lse=torch.empty(4, 39, device="cuda")), dict(lse=torch.empty(40, 4, device="cuda").T), dict(k_starts=st[::2]),
    ]
    for change in bad:
        a = dict(q=q, k=k, v=v, q_starts=st, k_starts=st, out=out, lse=None)
        a.update(change)
        with pytest.raises((ValueError, binding.LoopServeError)):
            ctx.ls_packed_prefill(shape, **a)
    with pytest.raises(binding.LoopServeError):            # rows of an output that overlap
        ctx.ls_packed_prefill(shape, q, k, v, st, st, out[:1].expand(40, 4, 64))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("Hq,Hkv,d,n,at,dtype", [
    (4, 4, 128, 200, 101, torch.bfloat16), (8, 2, 128, 300, 150, torch.bfloat16), (4, 2, 64, 130, 64, torch.bfloat16), (32, 1, 64, 70, 33, torch.bfloat16),
    (4, 2, 128, 100, 37, torch.float32), (4, 1, 64, 90, 31, torch.float32)])
def test_what_a_row_does_not_see_does_not_reach_it(Hq, Hkv, d, n, at, dtype, bad):
    """Keys and values from a position on are no numbers: the rows before it have the same bits as with numbers there."""
    q, k, v = _inputs(21, Hq, Hkv, d, [n], [n], dtype)
    print("packed future", Hq, Hkv, d, n, at, dtype, bad, flush=True)
    out, lse = _run(q, k, v, [n], [n])
    k2, v2 = k.clone(), v.clone()
    k2[at:], v2[at:] = bad, bad
    got, got_lse = _run(q, k2, v2, [n], [n])
    assert torch.equal(got[:at], out[:at]) and torch.equal(got_lse[:, :at], lse[:, :at])
    assert not torch.isfinite(got[at:]).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,keys,rows,at", [(4, 2, 200, 200, 60), (4, 2, 200, 200, 0), (2, 1, 4000, 20, 0), (2, 1, 4000, 20, 3970), (2, 1, 4000, 4000, 1000)])
def test_no_number_that_is_seen_stays_none(Hq, Hkv, keys, rows, at, dtype):
    """A NaN key of head 0: the output and the normaliser of its heads' rows that see it are none either, whole items and parts; what else there is keeps its bits."""
    q, k, v = _inputs(23, Hq, Hkv, 128, [keys], [rows], dtype)
    print("packed NaN", Hq, Hkv, keys, rows, at, dtype, flush=True)
    out, lse = _run(q, k, v, [keys], [rows])
    k[at, 0] = float("nan")
    got, got_lse = _run(q, k, v, [keys], [rows])
    hit = torch.zeros(rows, Hq, dtype=torch.bool)
    hit[max(0, at - (keys - rows)):, :Hq // Hkv] = True
    assert torch.isnan(got[hit]).all() and torch.isnan(got_lse.T[hit]).all()
    assert torch.equal(got[~hit], out[~hit]) and torch.equal(got_lse.T[~hit], lse.T[~hit])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_that_are_not_finite_reach_those_who_see_them(dtype):
    """Single infinities and NaN in V: in their column of the output, from their position on, what the sum gives; in other columns and before, the same bits."""
    n, d = 140, 64
    q, k, v = _inputs(22, 4, 2, d, [n], [n], dtype, scale=0.5)
    print("packed odd values", dtype, flush=True)
    out, _ = _run(q, k, v, [n], [n])
    v2 = v.clone()
    places = {(50, 0, 3): float("inf"), (90, 0, 3): -float("inf"), (131, 1, 40): float("nan"), (139, 1, 63): -float("inf"), (0, 0, 10): float("inf")}
    for (r, h, c), x in places.items():
        v2[r, h, c] = x
    got, _ = _run(q, k, v2, [n], [n])
    want = out.double().clone()
    for (r, h, c), x in places.items():
        want[r:, 2 * h:2 * h + 2, c] += x
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[fine], out[fine]) and torch.equal(got[torch.isinf(want)].double(), want[torch.isinf(want)])


def test_the_same_bits_every_time():
    """Cut items and whole ones: parts are put together in one order."""
    for keys, rows in (([5003, 900], [20, 30]), ([300, 77, 800], [300, 77, 800])):
        q, k, v = _inputs(23, 8, 2, 128, keys, rows, torch.bfloat16)
        print("packed bits", keys, flush=True)
        first = _run(q, k, v, keys, rows)
        for _ in range(3):
            again = _run(q, k, v, keys, rows)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_rows_far_apart():
    """Rows whose elements lie beyond 2^31 of the tensor."""
    n, Hq, Hkv, d, step = 1200, 2, 1, 64, 1 << 21
    q, k, v = _inputs(24, Hq, Hkv, d, [n], [n], torch.bfloat16)
    whole = torch.zeros(n * step, dtype=torch.bfloat16, device="cuda")
    rows = whole.view(n, step)
    dk, dv, dq, out = (rows[:, a:a + w * d].unflatten(1, (w, d)) for a, w in ((0, Hkv), (1024, Hkv), (2048, Hq), (4096, Hq)))
    dk.copy_(k), dv.copy_(v), dq.copy_(q)
    shape = binding.make_shape(1, Hq, Hkv, d, n, n, 1, "bf16")
    print("packed far apart", flush=True)
    _context(shape).ls_packed_prefill(shape, dq, dk, dv, _starts([n]).cuda(), _starts([n]).cuda(), out)
    torch.cuda.synchronize()
    assert (n - 1) * step > 2 ** 31
    _check(q, k, v, [n], [n], out.cpu().contiguous(), None)
