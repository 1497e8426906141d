"""A server's steps as they would be made: tables resized, queries and keys normed and rotated into pages, attention, on pages of every type; prompts, a recorded decode loop, cut and
ended dialogues, and the calls that take whole contexts."""
import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests import paged4_util as p4
from tests import paged_util as pu
from tests.test_gpu_cache import _host, _i32
from tests.test_gpu_rotate import _check as _check_rotated
from tests.test_gpu_rotate import _expect, _rotation

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE, PAGES, MOST = 8, 2, 128, 16, 120, 40


def _stored(kind, rows):
    """Rows [n,Hkv,D] as pages of this type hold them, in 64 bits."""
    if kind == "bf16":
        return rows.double()
    if kind == "e4m3":
        return pu.values(pu.codes(rows, pu.exponents(rows)), pu.exponents(rows)).double()
    return p4.values(p4.codes(rows, p4.exponents(rows)), p4.exponents(rows))


class Server:
    def __init__(self, B, kind, seed):
        self.B, self.kind, self.rng = B, kind, np.random.default_rng(seed)
        u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
        if kind == "bf16":
            pool = [torch.zeros(PAGES, HKV, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        elif kind == "e4m3":
            pool = [u8(PAGES, HKV, PAGE, D), u8(PAGES, HKV, PAGE, D), u8(PAGES, HKV, PAGE), u8(PAGES, HKV, PAGE)]
        else:
            pool = [u8(PAGES, HKV, PAGE, D // 2), u8(PAGES, HKV, PAGE, D // 2), u8(PAGES, HKV, PAGE, D // 32), u8(PAGES, HKV, PAGE, D // 32)]
        self.cache = binding.PagedCache(*pool)
        self.at = binding.alloc_pages(self.cache, B, MOST)
        self.freq, self.w, self.rotation = _rotation(self.rng, D, D, False, "qk", 1e4)
        self.ctx = binding.Context(workspace=8 << 20)
        self.k = [torch.zeros(0, HKV, D, dtype=torch.bfloat16) for _ in range(B)]           # rotated, as rows; and v
        self.v = [x.clone() for x in self.k]

    def rows(self, T):
        x = pu.rnd(self.rng, T, HQ + 2 * HKV, D).cuda()
        return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]

    def resize(self, add, T):
        out = dict(starts=_i32([0] * (self.B + 1)), positions=_i32([0] * T), slots=torch.zeros(T, dtype=torch.int64, device="cuda"))
        self.ctx.ls_cache_resize(binding.make_shape(self.B, HQ, HKV, D, 1, T, 1, "bf16"), self.cache, self.at["free"], self.at["state"], add, self.at["lens"], self.at["table"], **out)
        return out

    def keep(self, add, k, v, starts):
        """What the dialogues are now, on the host."""
        k, v, starts = k.cpu(), v.cpu(), starts.tolist()
        for b, n in enumerate(add):
            if n < 0:
                self.k[b], self.v[b] = self.k[b][:max(0, len(self.k[b]) + n)], self.v[b][:max(0, len(self.v[b]) + n)]
            else:
                self.k[b], self.v[b] = (torch.cat([old, new[starts[b]:starts[b] + n]]) for old, new in ((self.k[b], k), (self.v[b], v)))
        assert self.at["lens"].tolist() == [len(x) for x in self.k]

    def check_tokens(self, q, out, lse):
        for b in range(self.B):
            K, V = _stored(self.kind, self.k[b]), _stored(self.kind, self.v[b])
            for j in range(HKV):
                g = slice(j * HQ // HKV, (j + 1) * HQ // HKV)
                ref = pu.attention(q[b, g].cpu(), K[:, j], V[:, j], np.full(HQ // HKV, len(K)), D ** -0.5)
                pu.check(out[b, g].cpu(), lse[b, g].cpu(), ref, torch.bfloat16)


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_steps_of_a_server(kind, padded):
    """padded: in the decode steps each dialogue has a row of its own, whether it goes on or not."""
    print("serving step", kind, padded, flush=True)
    B = 4
    s = Server(B, kind, 21)
    # ---- two prompts, in a step padded to a fixed number of rows
    add, T = [130, 0, 47, 0], 200
    at = s.resize(_i32(add), T)
    q, k, v = s.rows(T)
    shape = binding.make_shape(B, HQ, HKV, D, T, T, 1, "bf16")
    rq, rk = (torch.full((T, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (HQ, HKV))
    s.ctx.ls_norm_rotate(shape, s.rotation, q, k, rq, rk, at["positions"], s.cache, v, at["slots"])
    assert s.ctx.ls_poll_status() == 0
    for got, x, n in ((rq, q, "q"), (rk, k, "k")):
        _check_rotated(got, _expect(x.cpu(), s.w[n], 1e-6, s.freq, at["positions"].cpu(), False), torch.bfloat16)
    s.keep(add, rk, v, at["starts"])
    out, lse = torch.full_like(rq, 7.0), torch.full((HQ, T), 7.0, device="cuda")
    s.ctx.ls_packed_prefill(shape, rq, rk, v, at["starts"], at["starts"], out, lse)
    assert s.ctx.ls_poll_status() == 0 and (out[177:] == 7.0).all()
    for first, n in ((0, 130), (130, 47)):
        for h in range(HQ):
            rows = slice(first, first + n)
            ref = pu.attention(rq[rows, h].cpu(), rk[rows, h // 4].cpu(), v[rows, h // 4].cpu(), np.arange(n), D ** -0.5)
            pu.check(out[rows, h].cpu(), lse[h, rows].cpu(), ref, torch.bfloat16)
    # ---- a decode step, recorded: a row for each dialogue that goes on, none for the others
    by, at = _i32([0] * B), dict(starts=_i32([0] * (B + 1)), positions=_i32([0] * B), slots=torch.zeros(B, dtype=torch.int64, device="cuda"))
    if padded:
        at = dict(starts=None, positions=at["positions"][:, None], slots=at["slots"][:, None])
    rows_of = _i32([0, 1, 2, 3]) if padded else at["starts"]
    seen = (lambda x: x[:, :, None]) if padded else (lambda x: x)
    qkv = torch.zeros(B, HQ + 2 * HKV, D, dtype=torch.bfloat16, device="cuda")
    rq, rk = torch.zeros(B, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, HKV, D, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros_like(rq), torch.zeros(B, HQ, device="cuda")
    one = binding.make_shape(B, HQ, HKV, D, MOST * PAGE, 1 if padded else B, 1, "bf16")

    def step():
        s.ctx.ls_cache_resize(one, s.cache, s.at["free"], s.at["state"], by, s.at["lens"], s.at["table"], **at)
        q, k, v = seen(qkv[:, :HQ]), seen(qkv[:, HQ:HQ + HKV]), seen(qkv[:, HQ + HKV:])
        s.ctx.ls_norm_rotate(one, s.rotation, q, k, seen(rq), seen(rk), at["positions"], s.cache, v, at["slots"])
        s.ctx.ls_paged_attend(one, s.cache, rq, s.at["table"], s.at["lens"], out, lse)

    step()                                                 # (nobody grows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(24):
        add = [1, int(not padded or i % 3 != 1), 1, int(i >= 10)]
        by.copy_(torch.tensor(add, dtype=torch.int32))
        qkv.copy_(pu.rnd(s.rng, *qkv.shape))
        torch.cuda.synchronize()
        graph.replay()
        assert s.ctx.ls_poll_status() == 0
        s.keep(add, rk, qkv[:, HQ + HKV:], rows_of)
        if i in (0, 9, 10, 23):                            # (before the fourth has a row the queries' rows are the dialogues')
            s.check_tokens(rq, out, lse)
    # ---- one is cut, one ends, and another prompt finds room in what they gave back
    add = [-100, 60, -71, 0]
    at2 = s.resize(_i32(add), 64)
    q, k, v = s.rows(64)
    rq2, rk2 = torch.empty(64, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(64, HKV, D, dtype=torch.bfloat16, device="cuda")
    s.ctx.ls_norm_rotate(binding.make_shape(B, HQ, HKV, D, 1, 64, 1, "bf16"), s.rotation, q, k, rq2, rk2, at2["positions"], s.cache, v, at2["slots"])
    assert s.ctx.ls_poll_status() == 0
    s.keep(add, rk2, v, at2["starts"])
    assert [len(x) for x in s.k] == [54, 76 if padded else 84, 0, 14]
    for i in range(3):
        by.copy_(torch.tensor([1, 1, 0, 1], dtype=torch.int32))
        qkv.copy_(pu.rnd(s.rng, *qkv.shape))
        torch.cuda.synchronize()
        graph.replay()
        assert s.ctx.ls_poll_status() == 0
        s.keep([1, 1, 0, 1], rk, qkv[:, HQ + HKV:], rows_of)
    s.check_tokens(rq, out, lse)                           # (packed rows of a step in which one is idle are not the dialogues': a query is a query)
    # ---- a context back in order, as the scoring and the retention take it
    n = len(s.k[1])
    back = [torch.zeros(1, HKV, n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    s.ctx.ls_cache_read(binding.make_shape(1, HQ, HKV, D, n, n, 1, "bf16"), s.cache, s.at["table"][1:2], *back)
    for x, rows in zip(back, (s.k[1], s.v[1])):
        assert torch.equal(x[0].transpose(0, 1).cpu().double(), _stored(kind, rows))
    keep = [torch.empty(1, HKV, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    idx, cnt = torch.empty(1, HKV, 16, dtype=torch.int32, device="cuda"), torch.empty(1, HKV, dtype=torch.int32, device="cuda")
    s.ctx.ls_kv_compress(binding.make_shape(1, HQ, HKV, D, n, 1, 16, "bf16"), 16, pu.rnd(s.rng, 1, HQ, 16, D).cuda(), *back, idx, cnt, *keep)
    assert s.ctx.ls_poll_status() == 0
    for j in range(HKV):
        assert torch.equal(keep[1][0, j], back[1][0, j][idx[0, j].long()])
    # ---- no page is lost, and none is there twice
    lens, table = s.at["lens"].tolist(), s.at["table"].cpu()
    held = [int(x) for b in range(B) for x in table[b, :-(-lens[b] // PAGE)]]
    head, count = s.at["state"].tolist()
    ring = s.at["free"].cpu()[(head + torch.arange(count)) % PAGES].tolist()
    assert sorted(held + ring) == list(range(PAGES))
    assert _host(s.cache)["k"].shape[0] == PAGES


def test_calls_on_streams_of_their_own():
    """The three calls of a step on a stream that is not the default one, which waits for nothing else; the same bits as on the default stream."""
    print("serving step stream", flush=True)
    got = []
    for own in (False, True):
        s = Server(2, "e2m1", 5)
        stream = torch.cuda.Stream() if own else torch.cuda.current_stream()
        q, k, v = s.rows(70)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            at = s.resize(_i32([33, 37]), 70)
            rq, rk = torch.empty(70, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(70, HKV, D, dtype=torch.bfloat16, device="cuda")
            s.ctx.ls_norm_rotate(binding.make_shape(2, HQ, HKV, D, 1, 70, 1, "bf16"), s.rotation, q, k, rq, rk, at["positions"], s.cache, v, at["slots"])
            out, lse = torch.empty(2, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(2, HQ, device="cuda")
            s.ctx.ls_paged_attend(binding.make_shape(2, HQ, HKV, D, 100, 1, 1, "bf16"), s.cache, rq[[32, 69]].contiguous(), s.at["table"], s.at["lens"], out, lse)
        stream.synchronize()
        got.append([rq, rk, out, lse, s.at["table"], s.at["lens"], at["slots"], s.cache.k, s.cache.k_exp, s.cache.v])
    assert all(torch.equal(a, b) for a, b in zip(*got))
