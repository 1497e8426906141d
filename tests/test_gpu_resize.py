"""ls_cache_resize against its definition, sequence by sequence on the host: rings, tables, starts, positions, slots, and what is refused a sequence."""
import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests.test_gpu_cache import _i32

pytestmark = pytest.mark.gpu
OUT, RANGE, STARTS = binding.LS_STAT_PAGES_OUT, binding.LS_STAT_PAGE_RANGE, binding.LS_STAT_STARTS


def expect(free, state, add, lens, table, page, n_rows, padded=False):
    """(dict of all outputs, status) from numpy arrays; padded: n_rows of each sequence."""
    free, table, new = free.copy(), table.copy(), lens.astype(np.int64).copy()
    pages, room = len(free), min(table.shape[1] * page, 2 ** 31 - 1)
    head, count, status = int(state[0]), int(state[1]), 0
    if not (0 <= head < pages and 0 <= count <= pages):
        head = count = 0
        status |= RANGE
    was = free.copy()
    room_for = len(lens) * n_rows if padded else n_rows
    starts, positions, slots = [0], np.zeros(room_for, np.int32), np.full(room_for, -1, np.int64)
    asked = taken = given = 0
    full = False
    for b in range(len(lens)):
        old, by = int(lens[b]), int(add[b])
        now, ok = max(0, old + by), 0 <= old <= room
        have, want = -(-old // page), -(-now // page)
        rows = max(by, 0)
        full = rows > n_rows if padded else full or starts[-1] + rows > n_rows
        if not ok:
            status |= RANGE
        if rows and full:
            status |= STARTS
            rows = 0
        first = b * n_rows if padded else starts[-1]
        starts.append(starts[-1] + rows)
        if ok and by < 0:
            for j in range(want, have):
                if given < pages - count:
                    free[(head + count + given) % pages] = table[b, j]
                else:
                    status |= RANGE
                given += 1
            new[b] = now
        elif rows and ok:
            if now > room:
                status |= RANGE
                continue
            asked += want - have
            if want > have and asked > count:
                status |= OUT
                continue
            for j in range(have, want):
                table[b, j] = was[(head + taken) % pages]
                taken += 1
            new[b] = now
            p = np.arange(old, now)
            at = table[b, p // page].astype(np.int64)
            good = (at >= 0) & (at < pages)
            if not good.all():
                status |= RANGE
            positions[first:first + rows] = p
            slots[first:first + rows] = np.where(good, at * page + p % page, -1)
    given = min(given, pages - count)
    state = np.array([(head + taken) % pages, count - taken + given], np.int32)
    shape = (len(lens), n_rows) if padded else (n_rows,)
    return dict(free=free, state=state, lens=new.astype(np.int32), table=table, starts=np.array(starts, np.int32), positions=positions.reshape(shape), slots=slots.reshape(shape)), status


class Server:
    """The state on the GPU and on the host, and a call on both."""

    def __init__(self, B, pages, page, max_pages, in_place=True):
        pool = torch.zeros(pages, 1, page, 64, dtype=torch.bfloat16, device="cuda")
        self.cache, self.page, self.in_place = binding.PagedCache(pool, pool), page, in_place
        self.dev = binding.alloc_pages(self.cache, B, max_pages)
        self.host = {n: x.cpu().numpy() for n, x in self.dev.items()}
        self.ctx = binding.Context(workspace=0)

    def set(self, **kw):
        for n, x in kw.items():
            self.host[n] = np.array(x, np.int32).reshape(self.host[n].shape)
            self.dev[n].copy_(torch.from_numpy(self.host[n]))

    def step(self, add, n_rows=None, without=(), padded=False):
        """without starts: padded"""
        B, padded = len(add), padded or "starts" in without
        without = tuple(without) + (("starts",) if padded else ())
        n_rows = n_rows or max(1, int(np.maximum(add, 0).max() if padded else np.maximum(add, 0).astype(np.int64).sum()))
        d, h = self.dev, self.host
        want, status = expect(h["free"], h["state"], np.array(add), h["lens"], h["table"], self.page, n_rows, padded)
        shape = binding.make_shape(B, 1, 1, 64, 1, n_rows, 1, "bf16")
        size = (B, n_rows) if padded else (n_rows,)
        rows = dict(starts=_i32([77] * (B + 1)), positions=torch.full(size, 77, dtype=torch.int32, device="cuda"), slots=torch.full(size, 77, dtype=torch.int64, device="cuda"))
        new = {} if self.in_place else dict(new_state=_i32([77, 77]), new_lens=_i32([77] * B))
        self.ctx.ls_cache_resize(shape, self.cache, d["free"], d["state"], _i32([int(x) for x in add]), d["lens"], d["table"], **new,
                                 **{n: None if n in without else x for n, x in rows.items()})
        assert self.ctx.ls_poll_status() == status, (status,)
        if new:
            assert torch.equal(d["state"].cpu(), torch.from_numpy(h["state"])) and torch.equal(d["lens"].cpu(), torch.from_numpy(h["lens"]))
            d["state"], d["lens"] = new["new_state"], new["new_lens"]
        for n, x in {**d, **rows}.items():
            if n in without:
                assert (x == 77).all(), n
            else:
                assert np.array_equal(x.cpu().numpy(), want[n]), (n, x.cpu().numpy(), want[n])
        self.host = {n: want[n] for n in h}
        return want, status


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,page,pages,max_pages", [(1, 16, 40, 30), (3, 32, 50, 20), (24, 16, 300, 64), (65, 64, 400, 40), (1024, 16, 6000, 40), (1025, 16, 5000, 40), (2500, 32, 9000, 30)])
def test_a_server(B, page, pages, max_pages, in_place):
    """Sequences that begin, go on token by token, are cut and end, on a ring that goes round several times and is empty now and then."""
    print("resize server", B, page, pages, max_pages, in_place, flush=True)
    rng = np.random.default_rng(B + page)
    s = Server(B, pages, page, max_pages, in_place)
    seen = 0
    for i in range(40 if B < 100 else 14):
        lens = s.host["lens"]
        kind = rng.choice(5, B, p=[0.15, 0.5, 0.15, 0.1, 0.1])
        new = rng.integers(1, max(2, 2 * pages * page // B), B)
        add = np.where(kind == 0, new, np.where(kind == 1, 1, np.where(kind == 2, -lens, np.where(kind == 3, -rng.integers(1, 3 * page, B), 0))))
        if i % 4 == 3:                                         # each sequence has rows of its own
            _, status = s.step(add, n_rows=max(1, int(np.maximum(add, 0).max()) + int(rng.choice([0, 1, 7, -3]))), without=("positions",) if i == 7 else ("slots",) if i == 11 else (), padded=True)
            seen |= status
            continue
        _, status = s.step(add, n_rows=max(1, int(np.maximum(add, 0).sum()) + int(rng.choice([0, 1, 100, -3]))), without=("positions",) if i == 5 else ("slots",) if i == 6 else ())
        seen |= status
    held = s.host["table"][np.arange(max_pages)[None] < -(-s.host["lens"] // page)[:, None]]
    head, count = s.host["state"]
    ring = s.host["free"][(head + np.arange(count)) % pages]
    assert sorted(np.concatenate([held, ring])) == list(range(pages))            # no page is lost, and none is there twice
    assert seen & OUT or B < 24                             # (few sequences are as long as they can be before the ring is empty)


def test_many_rows():
    """Prompts as a large server has them, which many workgroups share out, in place and not."""
    rng = np.random.default_rng(2)
    for in_place in (True, False):
        s = Server(700, 70000, 16, 2048, in_place)
        s.step(np.where(np.arange(700) % 9 == 0, rng.integers(1, 12000, 700), 0))
        add = np.where(np.arange(700) % 9 == 0, 1, np.where(np.arange(700) % 7 == 0, rng.integers(1, 9000, 700), 0))
        add[::63] = -s.host["lens"][::63]
        print("resize many rows", in_place, int(add[add > 0].sum()), flush=True)
        s.step(add, n_rows=int(np.maximum(add, 0).sum()) + 5000)
        s.step(-s.host["lens"], n_rows=9000)
        assert (s.host["lens"] == 0).all() and s.host["state"][1] == 70000


def test_what_a_sequence_is_refused():
    s = Server(6, 12, 16, 4)
    print("resize refusals", flush=True)
    _, status = s.step([64, 65, 10, 0, 16, 64])                   # the second would be longer than 4 pages
    assert status == RANGE and list(s.host["lens"]) == [64, 0, 10, 0, 16, 64]
    s = Server(6, 12, 16, 4)
    _, status = s.step([64, 65, 10, 0, 16, 64], n_rows=200)       # 219 rows: the last one's have no room
    assert status == RANGE | STARTS and list(s.host["lens"]) == [64, 0, 10, 0, 16, 0]
    _, status = s.step([0, 64, 0, 33, 0, 1], n_rows=98)           # six pages are left: four, then three are asked for, then one
    assert status == OUT and list(s.host["lens"]) == [64, 64, 10, 0, 16, 0]
    _, status = s.step([-64, 0, 1, 0, -1, 16], n_rows=20)         # what is given back is there for the next call; one place of a page is not
    assert status == 0 and list(s.host["lens"]) == [0, 64, 11, 0, 15, 16]
    _, status = s.step([1, 0, 0, 50, 1, 0])
    assert status == 0 and s.host["state"][1] == 0
    _, status = s.step([15, 0, 5, 1, 0, 0])                       # nothing is left, and nothing is needed
    assert status == 0
    _, status = s.step([1, 0, 1, 1, 1, 1], n_rows=50)             # the first and the last two need pages
    assert status == OUT and list(s.host["lens"]) == [16, 64, 16, 52, 16, 16]


def test_lengths_and_rings_that_are_none():
    for lens, state, add in (([-5, 3, 65, 64], [0, 8], [4, 4, 4, -4]), ([0, 0, 0, 0], [-1, 4], [4, 0, 0, 1]), ([0, 20, 0, 0], [8, 4], [4, -20, 0, 1]), ([0, 0, 9, 0], [2, 9], [4, 1, -3, 1]),
                             ([16, 16, 0, 0], [3, 8], [-16, -16, 4, 0]), ([64, 64, 64, 0], [7, 5], [-64, -64, -64, 20]), ([2147483647, -2147483648, 0, 1], [0, 8], [2147483647, -2147483648, 1, -1])):
        s = Server(4, 8, 16, 4)
        s.set(lens=lens, state=state, table=np.arange(16) % 11 - 1, free=[3, 1, 7, 5, 0, 2, 6, 4])
        print("resize none", lens, state, add, flush=True)
        s.step(add, n_rows=30)


def test_pages_of_the_table_that_are_none():
    """A length's pages that are no pages: the rows there have no slot, the status word says so, and the others are as they are."""
    s = Server(2, 8, 16, 4)
    s.set(lens=[5, 20], table=[[9, -1, -1, -1], [3, -2, -1, -1]])
    print("resize bad pages", flush=True)
    _, status = s.step([20, 5])
    assert status == RANGE


@pytest.mark.parametrize("in_place", [True, False])
def test_sums_beyond_32_bits(in_place):
    """Thousands of sequences that ask for 2^31 - 1 rows each: one of the first ones has room."""
    B = 3000
    s = Server(B, 16, 256, 3, in_place)
    add = np.full(B, 2147483647, np.int64)
    add[0], add[1], add[5] = 700, -1, 0
    print("resize large sums", in_place, flush=True)
    _, status = s.step(add, n_rows=9001)
    assert status == STARTS and s.host["lens"][0] == 700
    add = np.full(B, -2147483648, np.int64)
    add[7] = 300
    _, status = s.step(add, n_rows=9001)
    assert status == 0 and s.host["lens"][0] == 0 and s.host["lens"][7] == 300
    add = np.full(B, 2147483647, np.int64)
    add[11], add[13] = 40, 400
    _, status = s.step(add, n_rows=400, padded=True)
    assert status == STARTS and s.host["lens"][11] == 40 and s.host["lens"][13] == 400


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,each,max_pages", [(1024, 2300000, 8), (1024, 4000000, 15625), (1024, 4194303, 16384), (2500, 4000000, 15625), (2500, 4194303, 8)])
def test_sums_between_31_and_32_bits(B, each, max_pages, in_place):
    """Sequences whose rows are few for 64 of them (less than 2^28) and more than 2^31 for a thousand; a table in which they would fit, or not.  The last one asks for a row."""
    s = Server(B, 64, 256, max_pages, in_place)
    add = np.full(B, each, np.int64)
    add[:4], add[B - 1] = (700, 0, 1, 257), 1
    print("resize sums of 32 bits", B, each, max_pages, in_place, flush=True)
    _, status = s.step(add, n_rows=9001)
    assert status == STARTS and list(s.host["lens"]) == [700, 0, 1, 257] + [0] * (B - 4)
    _, status = s.step(add, n_rows=9001, padded=True)
    assert status == STARTS and list(s.host["lens"]) == [1400, 0, 2, 514] + [0] * (B - 5) + [1]


@pytest.mark.parametrize("in_place", [True, False])
def test_two_billion_rows(in_place):
    """Starts of as many rows as a call can have, without positions and slots: 500 sequences have room, and three find pages."""
    B, each, page, max_pages, pages = 1024, 4000000, 256, 15625, 3 * 15625 + 100
    s = Server(B, pages, page, max_pages, in_place)
    d, starts = s.dev, _i32([77] * (B + 1))
    table = d["table"].clone()
    new = {} if in_place else dict(new_state=_i32([77, 77]), new_lens=_i32([77] * B))
    print("resize two billion rows", in_place, flush=True)
    s.ctx.ls_cache_resize(binding.make_shape(B, 1, 1, 64, 1, 2000000000, 1, "bf16"), s.cache, d["free"], d["state"], _i32([each] * B), d["lens"], d["table"], starts=starts, **new)
    assert s.ctx.ls_poll_status() == OUT | STARTS
    table[:3] = torch.arange(3 * max_pages, dtype=torch.int32, device="cuda").view(3, max_pages)
    assert torch.equal(starts.cpu().long(), torch.arange(B + 1).clamp(max=500) * each)
    assert new.get("new_lens", d["lens"]).tolist() == [each] * 3 + [0] * (B - 3) and new.get("new_state", d["state"]).tolist() == [3 * max_pages, 100]
    assert torch.equal(d["table"], table) and torch.equal(d["free"], torch.arange(pages, dtype=torch.int32, device="cuda"))


def test_pages_given_back_beyond_31_bits():
    """A thousand sequences that end, of more pages than 2^31 in all: the ring takes those that it has room for, the first ones in order."""
    B, max_pages, page, pages = 1024, 2200000, 16, 50
    s = Server(1, pages, page, 4)
    print("resize pages given back beyond 31 bits", flush=True)
    table = torch.full((B, max_pages), 7, dtype=torch.int32, device="cuda")      # 9 GB; entries behind the room of the ring are not looked at
    table[0, :100] = torch.arange(100, 200, dtype=torch.int32, device="cuda")
    free, state, lens, starts = _i32(list(range(pages))), _i32([45, 20]), _i32([page * max_pages] * B), _i32([77] * (B + 1))
    s.ctx.ls_cache_resize(binding.make_shape(B, 1, 1, 64, 1, 10, 1, "bf16"), s.cache, free, state, _i32([-2147483648] * B), lens, table, starts=starts)
    assert s.ctx.ls_poll_status() == RANGE
    assert lens.tolist() == [0] * B and state.tolist() == [45, 50] and starts.tolist() == [0] * (B + 1)
    assert free.tolist() == list(range(15)) + list(range(100, 130)) + list(range(45, 50))


def test_as_many_sequences_as_there_can_be():
    B = 65535
    s = Server(B, B, 16, 1)
    rng = np.random.default_rng(3)
    add = rng.integers(0, 17, B)
    print("resize 65535", flush=True)
    s.step(add)
    s.step(np.where(rng.random(B) < 0.5, -s.host["lens"], 16 - s.host["lens"]))
    s.step(np.where(s.host["lens"] == 16, rng.integers(-16, 1, B), rng.integers(-2, 17, B)), padded=True)


def test_a_captured_decode_loop():
    """A step that updates lengths and ring in place, recorded once: each replay is the next step; eager calls on other contexts in between."""
    B = 40
    s, other = Server(B, 200, 16, 10), Server(B, 200, 16, 10)
    rng = np.random.default_rng(4)
    for x in (s, other):
        x.step([int(v) for v in np.random.default_rng(5).integers(1, 40, B)])
    add, shape = _i32([1] * B), binding.make_shape(B, 1, 1, 64, 1, B, 1, "bf16")
    rows = dict(starts=_i32([0] * (B + 1)), positions=_i32([0] * B), slots=torch.zeros(B, dtype=torch.int64, device="cuda"))
    graph = torch.cuda.CUDAGraph()
    print("resize captured", flush=True)
    with torch.cuda.graph(graph):
        s.ctx.ls_cache_resize(shape, s.cache, s.dev["free"], s.dev["state"], add, s.dev["lens"], s.dev["table"], **rows)
    for i in range(30):
        by = [1] * B
        if i % 3 == 2:
            by = [int(x) for x in rng.choice([1, 0, -5], B)]
        add.copy_(torch.tensor(by, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, status = other.step(by, n_rows=B)
        for n, x in {**s.dev, **rows}.items():
            assert np.array_equal(x.cpu().numpy(), want[n]), (i, n)
        assert s.ctx.ls_poll_status() == status


def test_what_the_binding_refuses():
    s = Server(3, 8, 16, 4)
    d = s.dev
    shape = binding.make_shape(3, 1, 1, 64, 1, 5, 1, "bf16")
    add, i64 = _i32([1, 0, 0]), torch.zeros(5, dtype=torch.int64, device="cuda")
    call = lambda free=d["free"], state=d["state"], add=add, lens=d["lens"], table=d["table"], **kw: s.ctx.ls_cache_resize(shape, s.cache, free, state, add, lens, table, **kw)
    call(slots=i64, positions=_i32([0] * 5), starts=_i32([0] * 4))
    call(slots=i64[None].expand(3, 5).contiguous(), positions=_i32([[0] * 5] * 3))
    for kw in (dict(free=d["free"][:7]), dict(state=_i32([0, 8, 0])), dict(add=add.long()), dict(add=add.cpu()), dict(lens=_i32([0] * 4)), dict(table=d["table"][:2]), dict(table=d["table"].t()),
               dict(slots=i64.int()), dict(slots=i64[:4]), dict(slots=i64), dict(positions=i64), dict(starts=_i32([0] * 4), slots=i64[None].expand(3, 5).contiguous()), dict(starts=_i32([0] * 3)), dict(new_lens=_i32([0] * 2))):
        with pytest.raises(ValueError):
            call(**kw)
    both = _i32([0] * 4)
    for kw in (dict(add=None), dict(table=None), dict(lens=both[:3], new_lens=both[1:]), dict(state=both[:2], new_state=both[1:3])):
        with pytest.raises(binding.LoopServeError):
            call(**kw)
