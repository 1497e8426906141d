"""The calls on pages and packed sequences one after the other, as a serving program makes them: prompts of different lengths, tokens, a second turn, retention."""
import numpy as np
import pytest
import torch

from paper_2507_13681_amd import binding
from tests import paged_util as pu

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE = 8, 2, 128, 16


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(lens):
    return _i32(np.concatenate([[0], np.cumsum(lens)]))


class Dialogues:
    """Their keys and values as a program would compute them (on the host, bf16), and their pages on the GPU."""

    def __init__(self, seed, lens, room, kind):
        self.rng = np.random.default_rng(seed)
        self.B, self.kind = len(lens), kind
        need = -(-room // PAGE)
        self.table = torch.from_numpy(self.rng.permutation(self.B * need).astype(np.int32).reshape(self.B, need)).cuda()
        dt = torch.bfloat16 if kind == "bf16" else torch.uint8
        pool = {n: torch.zeros(self.B * need, HKV, PAGE, D, dtype=dt, device="cuda") for n in ("k", "v")}
        if kind == "e4m3":
            pool.update({n + "_exp": torch.zeros(self.B * need, HKV, PAGE, dtype=torch.uint8, device="cuda") for n in ("k", "v")})
        self.cache = binding.PagedCache(**pool)
        self.k = [torch.zeros(0, HKV, D, dtype=torch.bfloat16) for _ in lens]
        self.v = [x.clone() for x in self.k]
        # one context for all calls of the dialogues, as big as the largest wants
        full = binding.make_shape(self.B, HQ, HKV, D, room, room, 16, "bf16")
        self.ctx = binding.Context(workspace=max(binding.workspace_bytes(full, 64), binding.packed_workspace_bytes(full), binding.paged_workspace_bytes(full),
                                                 binding.packed_workspace_bytes(binding.make_shape(self.B, HQ, HKV, D, self.B * room, 64, 1, "bf16")),
                                                 binding.decode_workspace_bytes(full, 64, 0)))

    def stored(self, b, name):
        """What the cache should stand for."""
        x = getattr(self, name)[b].float()
        return x if self.kind == "bf16" else pu.values(pu.codes(x, pu.exponents(x)), pu.exponents(x))

    def lens(self):
        return [x.shape[0] for x in self.k]

    def add(self, rows):
        """New rows of each: into the pages, behind what is there; returns them packed, with the queries."""
        pos = _i32(self.lens())
        new = [[pu.rnd(self.rng, m, HKV, D, scale=s) for m in rows] for s in (1.3, 1.0)]
        q = [pu.rnd(self.rng, m, HQ, D, scale=1.5) for m in rows]
        for b in range(self.B):
            self.k[b], self.v[b] = torch.cat([self.k[b], new[0][b]]), torch.cat([self.v[b], new[1][b]])
        k, v = (torch.cat(x).cuda() for x in new)
        shape = binding.make_shape(self.B, HQ, HKV, D, 1, sum(rows), 1, "bf16")
        self.ctx.ls_cache_write(shape, self.cache, k, v, self.table, pos, _starts(rows))
        return q, k, v

    def read(self):
        """All of it back, [B,Hkv,longest,d], with zeros behind each."""
        n = max(self.lens())
        k, v = (torch.zeros(self.B, HKV, n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.ctx.ls_cache_read(binding.make_shape(self.B, HQ, HKV, D, n, n, 1, "bf16"), self.cache, self.table, k, v, count=_i32(self.lens()))
        return k, v


def _check_rows(q, out, lse, K, V, rows, first):
    """Rows of one dialogue, the last of K's positions."""
    n = K.shape[0]
    for h in range(HQ):
        j = h // (HQ // HKV)
        ref = pu.attention(q[:, h], K[:, j], V[:, j], np.arange(n - rows, n), D ** -0.5)
        pu.check(out[first:first + rows, h].cpu(), lse[h, first:first + rows].cpu(), ref, torch.bfloat16)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_dialogue_batch(kind):
    prompts = [300, 37, 129]
    s = Dialogues(3, prompts, 480, kind)
    print("flow", kind, flush=True)
    # the first turns, attended over as they come from the projection
    q, k, v = s.add(prompts)
    T = sum(prompts)
    dq, out, lse = torch.cat(q).cuda(), torch.empty(T, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(HQ, T, device="cuda")
    s.ctx.ls_packed_prefill(binding.make_shape(3, HQ, HKV, D, T, T, 1, "bf16"), dq, k, v, _starts(prompts), _starts(prompts), out, lse)
    for b, first in enumerate(np.concatenate([[0], np.cumsum(prompts)])[:3]):
        _check_rows(q[b], out, lse, s.k[b], s.v[b], prompts[b], int(first))
    # twenty tokens, each into the pages and then over them
    for _ in range(20):
        q, _, _ = s.add([1, 1, 1])
        dq = torch.cat(q).cuda()
        out, lse = torch.empty_like(dq), torch.empty(3, HQ, device="cuda")
        s.ctx.ls_paged_attend(binding.make_shape(3, HQ, HKV, D, 480, 1, 1, "bf16"), s.cache, dq, s.table, _i32(s.lens()), out, lse)
    for b, n in enumerate(s.lens()):
        _check_rows(q[b], out[b:b + 1], lse[b][:, None], s.stored(b, "k"), s.stored(b, "v"), 1, 0)
    # a second turn over what the cache holds: read back, packed by hand, the new rows last
    rows = [45, 80, 1]
    q, _, _ = s.add(rows)
    k, v = s.read()
    for b, n in enumerate(s.lens()):
        for name, x in (("k", k), ("v", v)):
            assert torch.equal(x[b, :, :n].transpose(0, 1).float().cpu(), s.stored(b, name)) and (x[b, :, n:] == 0).all()
    dk, dv = (torch.cat([x[b, :, :n].transpose(0, 1) for b, n in enumerate(s.lens())]) for x in (k, v))
    T = sum(rows)
    dq, out, lse = torch.cat(q).cuda(), torch.empty(T, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(HQ, T, device="cuda")
    s.ctx.ls_packed_prefill(binding.make_shape(3, HQ, HKV, D, sum(s.lens()), T, 1, "bf16"), dq, dk, dv, _starts(rows), _starts(s.lens()), out, lse)
    for b, first in enumerate(np.concatenate([[0], np.cumsum(rows)])[:3]):
        _check_rows(q[b], out, lse, s.stored(b, "k"), s.stored(b, "v"), rows[b], int(first))
    # the first dialogue's turn by lines instead: with all of them it is the same attention
    n, m = s.lens()[0], rows[0]
    shape = binding.make_shape(1, HQ, HKV, D, n, m, 32, "bf16")
    k0, v0 = k[:1, :, :n].contiguous(), v[:1, :, :n].contiguous()
    q0 = dq[:m].transpose(0, 1)[None].contiguous()
    sel = binding.alloc_select(shape)
    score = binding.alloc_score(shape)
    s.ctx.ls_score(shape, q0[:, :, -32:].contiguous(), k0, score["vert"], score["slash"], score["vmax"], score["smax"], score["total"])
    s.ctx.ls_select(shape, 1.0, score["vert"], score["slash"], score["vmax"], score["smax"], score["total"], sel["v_idx"], sel["v_cnt"], sel["s_idx"], sel["s_cnt"])
    sel["s_idx"][:], sel["s_cnt"][:], sel["v_cnt"][:] = torch.arange(n, dtype=torch.int32, device="cuda"), n, 0
    out0 = torch.empty_like(q0)
    s.ctx.ls_sparse_prefill(shape, q0, k0, v0, sel["v_idx"], sel["v_cnt"], sel["s_idx"], sel["s_cnt"], out0)
    err = (out0[0].transpose(0, 1).float() - out[:m].float()).abs()
    assert err.max() <= 2e-2 and err.mean() <= 5e-3
    # retention: the last 16 queries rank each dialogue's cache, 64 rows of each KV head stay, in fresh pages
    assert s.ctx.ls_poll_status() == 0
    budget, last = 64, max(s.lens())
    keep = torch.empty(3, HKV, budget, D, dtype=torch.bfloat16, device="cuda"), torch.empty(3, HKV, budget, D, dtype=torch.bfloat16, device="cuda")
    for b, n in enumerate(s.lens()):
        shape = binding.make_shape(1, HQ, HKV, D, n, 1, 16, "bf16")
        idx, cnt = torch.empty(1, HKV, budget, dtype=torch.int32, device="cuda"), torch.empty(1, HKV, dtype=torch.int32, device="cuda")
        q_obs = pu.rnd(s.rng, 1, HQ, 16, D).cuda()
        s.ctx.ls_kv_compress(shape, budget, q_obs, k[b:b + 1, :, :n].contiguous(), v[b:b + 1, :, :n].contiguous(), idx, cnt, keep[0][b:b + 1], keep[1][b:b + 1])
    pages = 3 * budget // PAGE
    dt = s.cache.k.dtype
    pool = {x: torch.zeros(pages, HKV, PAGE, D, dtype=dt, device="cuda") for x in ("k", "v")}
    if kind == "e4m3":
        pool.update({x + "_exp": torch.zeros(pages, HKV, PAGE, dtype=torch.uint8, device="cuda") for x in ("k", "v")})
    small, table = binding.PagedCache(**pool), _i32(s.rng.permutation(pages).reshape(3, -1).tolist())
    s.ctx.ls_cache_write(binding.make_shape(3, HQ, HKV, D, last, budget, 1, "bf16"), small, keep[0], keep[1], table)
    q = pu.rnd(s.rng, 3, HQ, D).cuda()
    shape = binding.make_shape(3, HQ, HKV, D, budget, 1, 1, "bf16")
    a, b = torch.empty_like(q), torch.empty_like(q)
    s.ctx.ls_paged_attend(shape, small, q, table, _i32([budget] * 3), a)
    # (values that came out of an 8-bit cache go back into one unchanged)
    s.ctx.ls_decode_attend(shape, q, keep[0], keep[1], None, None, None, b)
    assert s.ctx.ls_poll_status() == 0
    for i in range(3):
        for h in range(HQ):
            K, V = keep[0][i, h // 4].cpu(), keep[1][i, h // 4].cpu()
            for x in (a, b):
                pu.check(x[i, h:h + 1].cpu(), None, pu.attention(q[i, h:h + 1].cpu(), K, V, [budget], D ** -0.5), torch.bfloat16)
