"""What the calls on pages and packed sequences decide on the host, and what the kernels share with it: refusals, pages, counts of work (no GPU)."""
import ctypes as C
import os
import random

import pytest

from paper_2507_13681_amd import binding, build

HERE = 1 << 20                                             # an address, 16-byte aligned, that nothing follows


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.LIB):
        build.build_library()
    return binding.load_library()


def _rows(seq=0, row=512, head=128, data=HERE):
    return binding.LsRows(data, seq, row, head)


def _shape(**kw):
    a = dict(B=2, Hq=8, Hkv=4, d=128, n=100, n_hat=100, w=1, dtype="bf16")
    a.update(kw)
    return binding.make_shape(**a)


def _cache(**kw):
    a = dict(Hkv=4, d=128, page=32, type=1, pages=10, k=HERE, v=HERE, k_exp=HERE, v_exp=HERE)
    a.update(kw)
    return binding.LsCache(*[a[f[0]] for f in binding.LsCache._fields_])


def test_layouts_match_the_header():
    assert C.sizeof(binding.LsCache) == 56 and binding.LsCache.pages.offset == 16 and binding.LsCache.v_exp.offset == 48
    assert C.sizeof(binding.LsRows) == 32


EINVAL, ESHAPE = -1, -2
PACKED = [
    (dict(), 0), (dict(starts=False), 0),
    (dict(shape=dict(d=96)), ESHAPE), (dict(shape=dict(Hq=6)), ESHAPE), (dict(shape=dict(B=0)), ESHAPE), (dict(shape=dict(n=0)), ESHAPE),
    (dict(shape=dict(n_hat=0)), ESHAPE), (dict(shape=dict(n_hat=2 ** 31)), ESHAPE), (dict(shape=dict(n_hat=2 ** 30 + 9)), ESHAPE),
    (dict(shape=dict(n_hat=2 ** 62, Hq=16)), ESHAPE),       # times the query heads of a KV head it is 2^64
    (dict(shape=dict(B=9000)), ESHAPE), (dict(q=_rows(data=None)), EINVAL), (dict(q=None), EINVAL), (dict(k=_rows(data=HERE + 8)), EINVAL),
    (dict(v=_rows(row=516)), EINVAL), (dict(v=_rows(head=-128)), ESHAPE), (dict(k=_rows(row=2 ** 26)), ESHAPE), (dict(q=_rows(row=2 ** 58)), ESHAPE),
    (dict(out=_rows(row=512, head=128)), ESHAPE),           # eight heads in the room of four
    (dict(out=_rows(row=0)), ESHAPE), (dict(k=_rows(row=0, head=0)), 0), (dict(q_starts=None), EINVAL), (dict(k_starts=HERE + 2), EINVAL),
    (dict(lse=HERE + 1), EINVAL), (dict(starts=False, out=_rows(seq=8, row=1024)), ESHAPE), (dict(starts=False, out=_rows(seq=102400, row=1024)), 0),
]


@pytest.mark.parametrize("change,want", PACKED)
def test_packed_refusals(lib, change, want):
    a = dict(q=_rows(row=1024, seq=102400), k=_rows(seq=51200), v=_rows(seq=51200), out=_rows(row=1024, seq=102400), q_starts=HERE, k_starts=HERE, lse=None)
    a.update({n: x for n, x in change.items() if n in a})
    if change.get("starts") is False:
        a.update(q_starts=None, k_starts=None)
    s = _shape(**change.get("shape", {}))
    ref = lambda r: None if r is None else C.byref(r)
    assert lib.ls_debug_check_packed(C.byref(s), ref(a["q"]), ref(a["k"]), ref(a["v"]), a["q_starts"], a["k_starts"], ref(a["out"]), a["lse"]) == want


MOVE = [
    (dict(), 0, 0), (dict(starts=None), 0, 0), (dict(starts=None, count=HERE), 0, 0), (dict(count=HERE), EINVAL, EINVAL),
    (dict(cache=None), EINVAL, EINVAL), (dict(cache=dict(page=24)), ESHAPE, ESHAPE), (dict(cache=dict(page=8)), ESHAPE, ESHAPE), (dict(cache=dict(page=512)), ESHAPE, ESHAPE),
    (dict(cache=dict(d=64)), ESHAPE, ESHAPE), (dict(cache=dict(Hkv=2)), ESHAPE, ESHAPE), (dict(cache=dict(type=2)), EINVAL, EINVAL), (dict(cache=dict(pages=0)), ESHAPE, ESHAPE),
    (dict(cache=dict(k_exp=None)), EINVAL, EINVAL), (dict(cache=dict(type=0, k_exp=None, v_exp=None)), 0, 0), (dict(cache=dict(v=HERE + 4)), EINVAL, EINVAL),
    (dict(table=None), EINVAL, EINVAL), (dict(max_pages=0), ESHAPE, ESHAPE), (dict(pos=HERE + 1), EINVAL, EINVAL),
    (dict(k=_rows(row=0)), 0, ESHAPE), (dict(v=_rows(row=256)), 0, ESHAPE),                     # rows that overlap: read, but not written
    (dict(shape=dict(n_hat=0)), ESHAPE, ESHAPE), (dict(shape=dict(B=30000, Hq=1)), ESHAPE, ESHAPE), (dict(shape=dict(Hq=0)), 0, 0),
    (dict(shape=dict(n_hat=2147483000, n=1), starts=None), ESHAPE, ESHAPE),
]


@pytest.mark.parametrize("change,write,read", MOVE)
def test_move_refusals(lib, change, write, read):
    a = dict(cache={}, k=_rows(seq=51200), v=_rows(seq=51200), starts=HERE, count=None, table=HERE, max_pages=4, pos=None)
    a.update({n: x for n, x in change.items() if n in a})
    s = _shape(**change.get("shape", {}))
    cache = None if a["cache"] is None else C.byref(_cache(**a["cache"]))
    for w, want in ((1, write), (0, read)):
        assert lib.ls_debug_check_move(C.byref(s), cache, C.byref(a["k"]), C.byref(a["v"]), a["starts"], a["count"], a["table"], a["max_pages"], a["pos"], w) == want


PAGED = [
    (dict(), 0), (dict(shape=dict(dtype="f32")), ESHAPE), (dict(shape=dict(Hq=132)), ESHAPE), (dict(shape=dict(Hq=128)), 0), (dict(shape=dict(n=0)), ESHAPE),
    (dict(shape=dict(n=2 ** 31)), ESHAPE), (dict(q=None), EINVAL), (dict(q=HERE + 2), EINVAL), (dict(out=None), EINVAL), (dict(len=None), EINVAL), (dict(table=None), EINVAL),
    (dict(table=HERE + 2), EINVAL), (dict(max_pages=-1), ESHAPE), (dict(lse=HERE + 2), EINVAL), (dict(cache=dict(v_exp=HERE + 4)), EINVAL), (dict(cache=dict(page=48)), ESHAPE),
]


@pytest.mark.parametrize("change,want", PAGED)
def test_paged_refusals(lib, change, want):
    a = dict(cache={}, q=HERE, table=HERE, max_pages=4, len=HERE, out=HERE, lse=None)
    a.update({n: x for n, x in change.items() if n in a})
    s = _shape(**change.get("shape", {}))
    assert lib.ls_debug_check_paged(C.byref(s), C.byref(_cache(**a["cache"])), a["q"], a["table"], a["max_pages"], a["len"], a["out"], a["lse"]) == want
    if change.get("shape"):
        assert (lib.ls_paged_workspace_bytes(C.byref(s)) == 0) == (want != 0)


def test_pages(lib):
    t = (C.c_int32 * 8)(0, 5, 9, -1, 10, 2147483647, -2147483648, 3)
    at = lambda b, pos: lib.ls_debug_page_of(t, 4, 10, 32, b, pos)
    assert [at(0, p) for p in (0, 31, 32, 63, 64, 96, 127, 128, -1, 2 ** 40)] == [0, 0, 5, 5, 9, -1, -1, -1, -1, -1]
    assert [at(1, p) for p in (0, 32, 64, 96)] == [-1, -1, -1, 3]


def test_counts_of_packed_work(lib):
    """Blocks, steps and counts against the definition, row by row."""
    rng = random.Random(1)
    out = (C.c_int64 * 4)()
    for _ in range(400):
        G = rng.choice([1, 2, 3, 4, 5, 8, 12, 16, 31, 32, 64, 200])
        queries, keys = rng.randint(1, 700), rng.choice([0, rng.randint(0, 900), rng.randint(0, 5000)])
        rows = queries * G
        last = [keys - queries + r // G for r in range(rows)]
        blocks = -(-rows // 128)
        steps = [max(0, (max(last[128 * j:128 * (j + 1)]) + 32) // 32) for j in range(blocks)]
        for j in (0, blocks - 1, rng.randrange(blocks)):
            x = rng.choice([-1, 0, steps[j], steps[j] - 1, rng.randint(0, 200)])
            lib.ls_debug_packed_counts(keys, queries, G, j, x, out)
            assert out[0] == blocks and out[1] == steps[j], (keys, queries, G, j)
            assert out[2] == sum(s > x for s in steps), (keys, queries, G, x, steps)
            assert out[3] >= sum(steps)
        assert steps == sorted(steps)                      # what counting them from the end relies on


def test_parts_of_packed_items_fit_into_their_units(lib):
    """However the rows are shared out among sequences, a KV head's items and parts are no more than its share of the workgroups."""
    rng = random.Random(2)
    out, units = (C.c_int64 * 4)(), (C.c_int64 * 2)()
    cut = 0
    for _ in range(300):
        Hkv, G, d = rng.choice([1, 2, 3, 4, 8, 16, 24]), rng.choice([1, 4, 5, 8]), rng.choice([64, 128])
        B = rng.choice([1, 2, 5, 40, 64])
        rows = [rng.choice([0, 1, rng.randint(0, 300)]) for _ in range(B)]
        keys = [r + rng.choice([0, rng.randint(0, 9000), -rng.randint(0, r)]) for r in rows]
        s = binding.make_shape(B, Hkv * G, Hkv, d, max(1, sum(keys)), max(1, sum(rows)), 1, rng.choice(["bf16", "f32"]))
        assert lib.ls_debug_packed_units(C.byref(s), 1, units) == 0
        n, items = units[0], 0
        work = 0
        steps = []
        for k, r in zip(keys, rows):
            lib.ls_debug_packed_counts(k, r, G, 0, 0, out)
            items += out[0]
            work += out[3]
            for j in range(out[0]):
                lib.ls_debug_packed_counts(k, r, G, j, 0, out)
                steps.append(out[1])
        assert items * Hkv <= units[1]
        if n == 0:
            continue
        assert n > units[1] and n % 8 == 0
        length = lib.ls_debug_packed_length(C.byref(s), work, items, max(steps, default=0))
        cut += length < 1 << 28
        parts = sum(max(1, -(-x // length)) for x in steps)
        assert parts <= n // Hkv, (parts, n, Hkv)
        assert n * (128 * d + 256) * 4 <= lib.ls_packed_workspace_bytes(C.byref(s))
    assert cut > 50


def test_cuts_of_paged_work(lib):
    """However long the sequences are, parts and workgroups are no more than the call has room for."""
    rng = random.Random(3)
    for _ in range(400):
        Hkv, B = rng.choice([1, 2, 3, 8, 24, 300]), rng.choice([1, 2, 7, 64, 130])
        most = rng.choice([1, 512, 513, 4096, 4128, rng.randint(1, 200000)])
        lens = [rng.choice([0, 1, most, rng.randint(0, most)]) for _ in range(B)]
        s = binding.make_shape(B, Hkv, Hkv, 64, most, 1, 1, "bf16")
        a, cuts, room = (C.c_int32 * B)(*lens), (C.c_int32 * B)(), C.c_int32()
        units = lib.ls_debug_paged_cuts(C.byref(s), a, cuts, C.byref(room))
        assert all(1 <= c <= room.value for c in cuts), (list(cuts), room.value)
        assert sum(cuts) * Hkv <= units
        assert lib.ls_paged_workspace_bytes(C.byref(s)) >= (units * 68 * 4 if room.value > 1 else 0)
