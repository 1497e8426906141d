"""The paged cache and dense attention around it: what is timed, the plain form of each operator, and its values in 64 bits.

Four kinds of case, the steps of a serving program whose dialogues keep their keys and values in pages:

  prompt  ls_packed_prefill: causal attention of prompts (or of the new rows of later turns) of different lengths, packed
          one behind the other.
  write   ls_cache_write: rows of K and V into the pages of their sequences, as bf16 or in 8 bits (e4m3, a power of two
          for each row).
  read    ls_cache_read: the way back, rows in order for the calls that take whole contexts.
  token   ls_paged_attend: one new token of each sequence over its pages.

`own` False: elementary torch operations in 32 bits, rounded once at the end.  `own` True: the library's calls.
"""
import math

import torch

own = False


def _prompt(name, keys, rows="", **kw):
    c = dict(name=name, kind="prompt", keys=keys, rows=rows or keys, Hq=32, Hkv=8, d=128, dtype="bf16", fused=False)
    c.update(kw)
    return c


def _cache(kind, name, lens, at, **kw):
    """lens: rows of each sequence; at: where in their sequences they begin."""
    c = dict(name=name, kind=kind, lens=lens, at=at, Hkv=8, d=128, page=64, cache="e4m3", dtype="bf16", packed=True)
    c.update(kw)
    return c


def _token(name, lens, **kw):
    c = dict(name=name, kind="token", lens=lens, Hq=32, Hkv=8, d=128, page=64, cache="bf16")
    c.update(kw)
    return c


def listed():
    return [
        # the opening turn of a 32k dialogue, whole, before anything is known of its lines: the longest prompt
        _prompt("prompt_32k", "32768"),
        # what a server has waiting: prompts of many lengths, q, k and v as they leave one projection
        _prompt("prompts_ragged", "5003,61,1777,1,8192,300,128,2500,17,777,4096,1045", fused=True),
        # follow-up questions deep in four dialogues: few new rows, long histories
        _prompt("follow_ups", "12347,8192,3001,20000", "61,200,17,1"),
        # short prompts of a small fp32 model
        _prompt("prompts_fp32", "1024,37,300", Hq=4, Hkv=1, d=64, dtype="f32"),
        # that opening turn's keys and values, quantised as they go into the cache
        _cache("write", "write_32k", "32768", "0"),
        # one token's rows of each sequence of a small batch, at the end of what it has: the smallest call there is
        _cache("write", "write_token", "1,1,1,1", "2064,16384,511,5462", packed=False, page=16),
        # the cache of four dialogues back in order, as the retention call takes it
        _cache("read", "read_16k_b4", "16384,16384,16384,16384", "0,0,0,0", packed=False),
        # a stretch of some ragged bf16 caches in pages of 16, into fp32 rows
        _cache("read", "read_ragged", "777,1,2500,131", "16,5,1000,0", page=16, cache="bf16", dtype="f32", Hkv=4, d=64),
        # one token over a short bf16 cache of one dialogue
        _token("token_b1", "519", page=16),
        # one token of four dialogues of 70B-class heads over 8-bit caches
        _token("token_16k_b4", "16384,16384,16384,16384", Hq=64, cache="e4m3"),
        # the longest context there is, bf16
        _token("token_131k", "131072", page=128),
        # a batch of sequences of very different ages, one of them empty
        _token("tokens_ragged", "9000,17,33,2048,1,12347,600,0,4100,250,31000,75,1500,333,5003,64,20000,901,3500,129,8191,40,700,2600",
               cache="e4m3", page=32),
    ]


HEADS = [(32, 8), (64, 8), (16, 4), (8, 2), (8, 8), (4, 1), (32, 1), (12, 3)]
MOST_CELLS = 32 * 32768 * 32769 // 2           # (query head, query, key) triples of the longest prompt listed
MOST_ROWS = 8 * 128 * 65536                    # heads x values x rows of K (and of V) of the largest cache call


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(xs):
    return ",".join(str(x) for x in xs)


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "write", "read", "token", "token"])
    hq, hkv = rng.choice(HEADS)
    d = rng.choice([64, 128, 128])
    if kind == "prompt":
        f32 = rng.random() < 0.2
        keys = [_log(rng, 1, 4096 if f32 else 32768) for _ in range(rng.choice([1, 1, 2, 5, 16]))]
        later = rng.random() < 0.3
        rows = [min(k, _log(rng, 1, 600)) if later else k for k in keys]
        most = MOST_CELLS // 32 if f32 else MOST_CELLS
        while sum(hq * r * (2 * k - r + 1) // 2 for r, k in zip(rows, keys)) > most:
            keys = [max(1, k * 3 // 4) for k in keys]
            rows = [min(r, k) for r, k in zip(rows, keys)]
        return dict(kind=kind, keys=_text(keys), rows=_text(rows), Hq=hq, Hkv=hkv, d=d, dtype="f32" if f32 else "bf16",
                    fused=not later and rng.random() < 0.5)
    page = rng.choice([16, 32, 64, 128])
    cache = rng.choice(["bf16", "e4m3", "e4m3"])
    if kind == "token":
        lens = [_log(rng, 1, 131072) - (rng.random() < 0.05) for _ in range(rng.choice([1, 1, 2, 4, 13, 32, 64]))]
        while 2 * hkv * d * sum(lens) > MOST_ROWS * 4:
            lens = [x * 3 // 4 for x in lens]
        return dict(kind=kind, lens=_text(lens), Hq=hq, Hkv=hkv, d=d, page=page, cache=cache)
    tokens = kind == "write" and rng.random() < 0.3        # a token of each sequence, or more
    lens = [1 if tokens else _log(rng, 1, 32768) for _ in range(rng.choice([1, 2, 4, 13, 32]))]
    while hkv * d * max(len(lens) * max(lens), 1) > MOST_ROWS:
        lens = [max(1, x * 3 // 4) for x in lens]
    at = [0 if rng.random() < 0.4 else _log(rng, 1, 8192) for _ in lens]
    return dict(kind=kind, lens=_text(lens), at=_text(at), Hkv=hkv, d=d, page=page, cache=cache,
                dtype="f32" if rng.random() < 0.2 else "bf16", packed=not tokens and rng.random() < 0.5)


# ---- inputs ------------------------------------------------------------------------------------------

def _ints(text):
    return [int(x) for x in text.split(",")]


def _starts(lens):
    out = [0]
    for x in lens:
        out.append(out[-1] + x)
    return out


def _i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _prompt_inputs(c, g):
    """q [Tq,Hq,d], k, v [Tk,Hkv,d]: noise, a direction that every query leans to and the first keys have, and slow waves along
    the positions that near keys and queries share."""
    Hq, Hkv, d, dt = c["Hq"], c["Hkv"], c["d"], _type(c["dtype"])
    keys, rows = _ints(c["keys"]), _ints(c["rows"])
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    Tq, Tk = sum(rows), sum(keys)
    if c["fused"]:
        x = torch.empty(Tk, (Hq + 2 * Hkv) * d, dtype=dt, device="cuda")
        q = x[:, :Hq * d].unflatten(1, (Hq, d))
        k = x[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
        v = x[:, (Hq + Hkv) * d:].unflatten(1, (Hkv, d))
    else:
        q, k, v = (torch.empty(t, h, d, dtype=dt, device="cuda") for t, h in ((Tq, Hq), (Tk, Hkv), (Tk, Hkv)))
    at_k = torch.cat([torch.arange(n, device="cuda") for n in keys]).float()
    at_q = torch.cat([torch.arange(n - r, n, device="cuda") for n, r in zip(keys, rows)]).float()
    w = rnd(8) / 48
    waves = lambda p: torch.cat([torch.cos(p[:, None] * w), torch.sin(p[:, None] * w)], 1)
    lean, near = (4.0 * math.sqrt(d)) ** 0.5, (3.0 * math.sqrt(d) / 8) ** 0.5
    for j in range(Hkv):
        E = torch.linalg.qr(rnd(d, 17))[0].T.contiguous()
        k[:, j] = (rnd(Tk, d) + near * (waves(at_k) @ E[:16]) + lean * (at_k < 4).float()[:, None] * E[16]).to(dt)
        for h in range(j * (Hq // Hkv), (j + 1) * (Hq // Hkv)):
            q[:, h] = (0.8 * rnd(Tq, d) + near * (waves(at_q) @ E[:16]) + lean * E[16]).to(dt)
        v[:, j] = rnd(Tk, d).to(dt)
    return q, k, v


def _exponents(x):
    """Of rows of fp32 values: 127 + e for the least power of two 2^e, of 2^-117 and above, by which they fit into e4m3 (448)."""
    m, e = torch.frexp(x.abs().amax(-1))
    E = e + 118 + (m > 0.875)
    return torch.where(m == 0, 10, E.clamp_min(10)).to(torch.uint8)


def _power(E):
    """2^(E - 127) from its bits (torch.ldexp multiplies by what pow gives, which need not be one)."""
    return (E.int() << 23).view(torch.float32)[..., None]


def _codes(x, E):
    return (x * _power(254 - E.int())).to(torch.float8_e4m3fn)


def _values(codes, E):
    return codes.view(torch.float8_e4m3fn).float() * _power(E)


def _pool(c, pages, fill):
    """K and V pages [pages,Hkv,page,d] (8-bit codes as bytes), and for those the exponents [pages,Hkv,page]."""
    out = {}
    for name in ("k", "v"):
        x = fill(pages, c["Hkv"], c["page"], c["d"])
        if c["cache"] == "bf16":
            out[name] = x.to(torch.bfloat16)
        else:
            out[name + "_exp"] = _exponents(x)
            out[name] = _codes(x, out[name + "_exp"]).view(torch.uint8)
    return out


def _table(lens, page, spare, g):
    """Pages of each sequence, drawn from the whole pool; entries past its end are no page."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, device="cuda", generator=g).int()
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    for s, (a, b) in enumerate(zip(_starts(need), _starts(need)[1:])):
        table[s, :b - a] = order[a:b]
    return table, pages


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    s = dict(case=c)
    if c["kind"] == "prompt":
        s["q"], s["k"], s["v"] = _prompt_inputs(c, g)
        s["keys"], s["rows"] = _ints(c["keys"]), _ints(c["rows"])
        s["k_starts"], s["q_starts"] = _i32(_starts(s["keys"])), _i32(_starts(s["rows"]))
        if own:
            from paper_2507_13681_amd import binding
            s["shape"] = binding.make_shape(len(s["keys"]), c["Hq"], c["Hkv"], c["d"], sum(s["keys"]), sum(s["rows"]), 1, c["dtype"])
            s["ctx"] = binding.Context(workspace=binding.packed_workspace_bytes(s["shape"]))
            s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
            s["lse"] = torch.empty(c["Hq"], sum(s["rows"]), device="cuda")
        return s
    lens = s["lens"] = _ints(c["lens"])
    B = len(lens)
    if c["kind"] == "token":
        s["table"], pages = _table(lens, c["page"], 3, g)
        s["pool"] = _pool(c, pages, rnd)
        s["q"] = (1.5 * rnd(B, c["Hq"], c["d"])).to(torch.bfloat16)
        s["len"] = _i32(lens)
        if own:
            from paper_2507_13681_amd import binding
            s["shape"] = binding.make_shape(B, c["Hq"], c["Hkv"], c["d"], max(1, max(lens)), 1, 1, "bf16")
            s["ctx"] = binding.Context(workspace=binding.paged_workspace_bytes(s["shape"]))
            s["cache"] = binding.PagedCache(**s["pool"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(B, c["Hq"], device="cuda")
        return s
    at = s["at"] = _ints(c["at"])
    s["table"], pages = _table([a + n for a, n in zip(at, lens)], c["page"], 3, g)
    s["pos"] = _i32(at)
    dt = _type(c["dtype"])
    shape = (sum(lens), c["Hkv"], c["d"]) if c["packed"] else (B, c["Hkv"], max(lens), c["d"])
    s["starts"] = _i32(_starts(lens)) if c["packed"] else None
    s["count"] = None if c["packed"] else _i32(lens)
    if c["kind"] == "write":
        s["pool"] = _pool(c, pages, lambda *z: torch.zeros(*z, device="cuda"))
        big = 1 + 9 * (torch.rand(c["Hkv"], 1, c["d"], device="cuda", generator=g) < 0.04).float()      # a few channels of K are large
        big = big.transpose(0, 1) if c["packed"] else big
        s["k_rows"], s["v_rows"] = (rnd(*shape) * big).to(dt), rnd(*shape).to(dt)
    else:
        s["pool"] = _pool(c, pages, rnd)
        s["k_rows"], s["v_rows"] = torch.zeros(shape, dtype=dt, device="cuda"), torch.zeros(shape, dtype=dt, device="cuda")
    if own:
        from paper_2507_13681_amd import binding
        s["shape"] = binding.make_shape(B, c["Hkv"], c["Hkv"], c["d"], max(1, max(lens)), shape[0] if c["packed"] else shape[2], 1, c["dtype"])
        s["ctx"] = binding.Context(workspace=0)
        s["cache"] = binding.PagedCache(**s["pool"])
    return s


# ---- the plain forms ---------------------------------------------------------------------------------

AT_ONCE = 1 << 28                              # logits that are held at a time


def _plain_prompt(s):
    c = s["case"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    G = Hq // Hkv
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    lse = torch.empty(Hq, s["q"].shape[0], device="cuda")
    for k0, nk, q0, nq in zip(_starts(s["keys"]), s["keys"], _starts(s["rows"]), s["rows"]):
        for j in range(Hkv):
            K, V = s["k"][k0:k0 + nk, j].float(), s["v"][k0:k0 + nk, j].float()
            Kt = K.T.contiguous()
            step = max(1, AT_ONCE // (G * nk))
            for r0 in range(0, nq, step):
                r1 = min(nq, r0 + step)
                hi = nk - nq + r1              # keys that the last of these rows sees
                Q = s["q"][q0 + r0:q0 + r1, j * G:(j + 1) * G].float().transpose(0, 1).reshape(-1, d)
                x = (Q @ Kt[:, :hi]) / math.sqrt(d)
                hidden = torch.arange(hi, device="cuda")[None] > torch.arange(nk - nq + r0, hi, device="cuda")[:, None]
                x.view(G, r1 - r0, hi).masked_fill_(hidden[None], -math.inf)
                m = x.amax(1, keepdim=True)
                p = torch.exp(x - m)
                l = p.sum(1, keepdim=True)
                o = (p @ V[:hi]) / l
                out[q0 + r0:q0 + r1, j * G:(j + 1) * G] = o.view(G, r1 - r0, d).transpose(0, 1).to(out.dtype)
                lse[j * G:(j + 1) * G, q0 + r0:q0 + r1] = (m + torch.log(l)).view(G, r1 - r0)
    return dict(out=out, lse=lse)


def _places(s):
    """Of every row that a write or read moves: its page, its place in the page, and where it is in the rows."""
    c, page = s["case"], s["case"]["page"]
    seq = torch.cat([torch.full((n,), i, device="cuda") for i, n in enumerate(s["lens"])])
    i = torch.cat([torch.arange(n, device="cuda") for n in s["lens"]])
    p = s["pos"].long()[seq] + i
    return s["table"].long()[seq, p // page], p % page, (torch.arange(len(i), device="cuda") if c["packed"] else seq, i)


def _moved(x, c, at):
    """The rows [N,Hkv,d] at those places."""
    return x[at[0]] if c["packed"] else x[at[0], :, at[1]]


def _plain_write(s):
    c, pool = s["case"], s["pool"]
    page, place, at = _places(s)
    for name in ("k", "v"):
        x = _moved(s[name + "_rows"], c, at).float()
        if c["cache"] == "bf16":
            pool[name][page, :, place] = x.to(torch.bfloat16)
        else:
            E = _exponents(x)
            pool[name][page, :, place] = _codes(x, E).view(torch.uint8)
            pool[name + "_exp"][page, :, place] = E


def _rows_of(pool, name, c, page, place):
    x = pool[name][page, :, place]
    return x.float() if c["cache"] == "bf16" else _values(x, pool[name + "_exp"][page, :, place])


def _plain_read(s):
    c, pool = s["case"], s["pool"]
    page, place, at = _places(s)
    for name in ("k", "v"):
        x = _rows_of(pool, name, c, page, place).to(_type(c["dtype"]))
        if c["packed"]:
            s[name + "_rows"][:] = x
        else:
            s[name + "_rows"][at[0], :, at[1]] = x


def _plain_token(s):
    c = s["case"]
    B, Hq, Hkv, d = len(s["lens"]), c["Hq"], c["Hkv"], c["d"]
    out = torch.zeros_like(s["q"])
    lse = torch.full((B, Hq), -math.inf, device="cuda")
    for b, n in enumerate(s["lens"]):
        if n == 0:
            continue
        pages = s["table"][b, :-(-n // c["page"])].long()
        K, V = ((s["pool"][t][pages].float() if c["cache"] == "bf16" else _values(s["pool"][t][pages], s["pool"][t + "_exp"][pages]))
                .transpose(0, 1).reshape(Hkv, -1, d)[:, :n] for t in ("k", "v"))
        x = torch.matmul(s["q"][b].float().view(Hkv, Hq // Hkv, d), K.transpose(1, 2).contiguous()) / math.sqrt(d)
        m = x.amax(2, keepdim=True)
        p = torch.exp(x - m)
        l = p.sum(2, keepdim=True)
        out[b] = (torch.matmul(p, V.contiguous()) / l).view(Hq, d).to(out.dtype)
        lse[b] = (m + torch.log(l)).view(Hq)
    return dict(out=out, lse=lse)


def run(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "prompt":
        if not own:
            return _plain_prompt(s)
        s["ctx"].ls_packed_prefill(s["shape"], s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], s["out"], s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if kind == "token":
        if not own:
            return _plain_token(s)
        s["ctx"].ls_paged_attend(s["shape"], s["cache"], s["q"], s["table"], s["len"], s["out"], s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if kind == "write":
        if own:
            s["ctx"].ls_cache_write(s["shape"], s["cache"], s["k_rows"], s["v_rows"], s["table"], s["pos"], s["starts"], s["count"])
        else:
            _plain_write(s)
        return {n: x.view(torch.float8_e4m3fn) if n in ("k", "v") and c["cache"] == "e4m3" else x for n, x in s["pool"].items()}
    if own:
        s["ctx"].ls_cache_read(s["shape"], s["cache"], s["table"], s["k_rows"], s["v_rows"], s["pos"], s["starts"], s["count"])
    else:
        _plain_read(s)
    return dict(k=s["k_rows"], v=s["v_rows"])


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _attention64(Q, K, V, last):
    """Q [R,d], K, V [n,d]; row r sees the keys 0 .. last[r]."""
    x = torch.matmul(Q.double(), K.double().T.contiguous()) / math.sqrt(Q.shape[1])
    x = torch.where(torch.arange(K.shape[0], device="cuda")[None] <= last[:, None], x, -math.inf)
    lse = torch.logsumexp(x, 1)
    return torch.matmul(torch.exp(x - lse[:, None]), V.double()), lse


# every value that e4m3 has, in ascending order from 0: 2^-9 times 0 .. 7, then eight to each power of two, up to 448
_E4M3 = [k * 2.0 ** -9 for k in range(8)] + [(8 + k) * 2.0 ** (e - 10) for e in range(1, 16) for k in range(8)][:-1]


def _powers64():
    """2^-117 .. 2^120"""
    return torch.tensor([2.0 ** e for e in range(-117, 121)], dtype=torch.float64, device="cuda")


def _nearest_e4m3(y):
    v = torch.tensor(_E4M3, dtype=torch.float64, device="cuda")
    a = y.abs().clamp(max=448.0)
    hi = torch.searchsorted(v, a).clamp(max=len(_E4M3) - 1)
    lo = (hi - 1).clamp(min=0)
    down, up = a - v[lo], v[hi] - a
    at = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return v[at] * torch.sign(y)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "prompt":
        Hq, G = c["Hq"], c["Hq"] // c["Hkv"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(Hq, s["q"].shape[0], dtype=torch.float64, device="cuda")
        k0 = q0 = 0
        for nk, nq in zip(s["keys"], s["rows"]):
            step = max(1, (AT_ONCE // 4) // nk)
            for r in range(0, nq, step):
                e = min(nq, r + step)
                last = torch.arange(nk - nq + r, nk - nq + e, device="cuda")
                hi = nk - nq + e
                for h in range(Hq):
                    out[q0 + r:q0 + e, h], lse[h, q0 + r:q0 + e] = _attention64(
                        s["q"][q0 + r:q0 + e, h], s["k"][k0:k0 + hi, h // G], s["v"][k0:k0 + hi, h // G], last)
            k0, q0 = k0 + nk, q0 + nq
        return dict(out=out, lse=lse)
    if c["kind"] == "token":
        B, Hq, G = len(s["lens"]), c["Hq"], c["Hq"] // c["Hkv"]
        out = torch.zeros(B, Hq, c["d"], dtype=torch.float64, device="cuda")
        lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(s["lens"]):
            if n == 0:
                continue
            p = torch.arange(n, device="cuda")
            page, place = s["table"][b].long()[p // c["page"]], p % c["page"]
            for j in range(c["Hkv"]):
                K, V = (_stored64(s["pool"], t, c, page, j, place) for t in ("k", "v"))
                out[b, j * G:(j + 1) * G], lse[b, j * G:(j + 1) * G] = _attention64(
                    s["q"][b, j * G:(j + 1) * G], K, V, torch.full((G,), n, device="cuda"))
        return dict(out=out, lse=lse)
    packed, first = c["packed"], 0
    out = {n: x.view(torch.float8_e4m3fn).double() if n in ("k", "v") and c["cache"] == "e4m3" else x.double() if n in ("k", "v") else x.clone()
           for n, x in s["pool"].items()} if c["kind"] == "write" else {n: s[n + "_rows"].double() for n in ("k", "v")}
    for b, n in enumerate(s["lens"]):
        p = s["at"][b] + torch.arange(n, device="cuda")
        page, place = s["table"][b].long()[p // c["page"]], p % c["page"]
        for j in range(c["Hkv"]):
            for t in ("k", "v"):
                rows = (slice(first, first + n), j) if packed else (b, j, slice(0, n))
                if c["kind"] == "read":
                    out[t][rows] = _stored64(s["pool"], t, c, page, j, place)
                    continue
                x = s[t + "_rows"][rows].double()
                if c["cache"] == "bf16":
                    out[t][page, j, place] = x
                    continue
                big = x.abs().amax(1).clamp(min=448 * 2.0 ** -117)
                e = torch.searchsorted(_powers64() * 448.0, big)      # the least power of two that is enough
                out[t][page, j, place] = _nearest_e4m3(x / _powers64()[e][:, None])
                out[t + "_exp"][page, j, place] = (e + 10).to(torch.uint8)
        first += n
    return out


def _stored64(pool, t, c, page, j, place):
    x = pool[t][page, j, place]
    if c["cache"] == "bf16":
        return x.double()
    return x.view(torch.float8_e4m3fn).double() * _powers64()[pool[t + "_exp"][page, j, place].long() - 10][:, None]


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    c = case
    d, Hkv = c["d"], c["Hkv"]
    if c["kind"] == "prompt":
        keys, rows, e = _ints(c["keys"]), _ints(c["rows"]), 2 if c["dtype"] == "bf16" else 4
        cells = c["Hq"] * sum(r * (2 * k - r + 1) // 2 for r, k in zip(rows, keys))
        return dict(bytes=e * d * 2 * (c["Hq"] * sum(rows) + Hkv * sum(keys)) + 4 * c["Hq"] * sum(rows), flops=4.0 * d * cells)
    n = sum(_ints(c["lens"]))
    stored = 2 * d if c["cache"] == "bf16" else d + 1                 # bytes of a row in the cache
    if c["kind"] == "token":
        B = len(_ints(c["lens"]))
        return dict(bytes=2 * Hkv * stored * n + (4 * d + 4) * B * c["Hq"] + 4 * n // c["page"], flops=4.0 * d * c["Hq"] * n)
    return dict(bytes=2 * Hkv * n * (stored + d * (2 if c["dtype"] == "bf16" else 4)) + 4 * n // c["page"], flops=0)
