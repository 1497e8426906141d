"""A serving step around the paged cache: what is timed, the plain form of each operator, and its values in 64 bits.

Four kinds of case, in the order in which a step of a serving program makes the calls:

  resize  ls_cache_resize: pages taken and given back, block tables, packed starts, positions and slots of the step's rows,
          from how much each sequence grows or shrinks.
  rotate  ls_norm_rotate: norms of queries and keys head by head and the rotation by their positions in one pass, into rows
          and, by their slots, into pages.
  turn    ls_cache_write, then ls_cache_read, on pages of 4-bit floats (e2m1, a power of two for each 32 values): a turn's
          rows go in, and the whole context comes back in order for the calls that take whole contexts.
  token   ls_paged_attend over such pages: one new token of each sequence.

`own` False: elementary torch operations in 32 bits (angles in 64), rounded once at the end.  `own` True: the library's calls.
"""
import math

import torch

own = False


def _resize(name, lens, add, **kw):
    """lens: positions that each sequence has; add: by how many it grows (or, negative, shrinks)."""
    c = dict(name=name, kind="resize", lens=lens, add=add, page=64, max_pages=2048, spare=4096, padding=0)
    c.update(kw)
    return c


def _rotate(name, rows, at, **kw):
    """rows: of each sequence; at: the position of its first one."""
    c = dict(name=name, kind="rotate", rows=rows, at=at, Hq=32, Hkv=8, d=128, dims=128, dtype="bf16", neighbours=False,
             norms="qk", fused=True, to="rows", page=64)
    c.update(kw)
    return c


def _turn(name, at, rows, **kw):
    """at: positions that each sequence has in its pages; rows: those of its new turn."""
    c = dict(name=name, kind="turn", at=at, rows=rows, Hkv=8, d=128, page=64, dtype="bf16", packed=True)
    c.update(kw)
    return c


def _token(name, lens, **kw):
    c = dict(name=name, kind="token", lens=lens, Hq=32, Hkv=8, d=128, page=64)
    c.update(kw)
    return c


def _text(xs):
    return ",".join(str(x) for x in xs)


def listed():
    many = [(137 * i * i + 911 * i) % 4001 for i in range(512)]
    return [
        # a decode step of a batch of sequences of very different ages: one token each, two have just ended, one is idle
        _resize("resize_step", "9000,17,33,2048,1,12347,600,0,4100,250,31000,75,1500,333,5003,64,20000,901,3500,129,8191,40,700,2600",
                "1,1,1,1,1,-12347,1,1,1,1,1,1,1,1,1,1,-20000,1,0,1,1,1,1,1", page=16),
        # prompts of many lengths are let in beside running sequences, in a step padded to a fixed number of rows
        _resize("resize_prompts", "0,0,0,0,0,0,0,0,0,0,0,0,31000,4096,777,20000", "5003,61,1777,1,8192,300,128,2500,17,777,4096,1045,1,1,-777,1",
                padding=100),
        # a large server's step: every eighth of 512 sequences begins with a prompt of up to 32k, every 31st one ends
        _resize("resize_512", _text(0 if i % 8 == 0 else 1 + x for i, x in enumerate(many)),
                _text(1 + 8 * many[i] if i % 8 == 0 else -1 - many[i] if i % 31 == 0 else 1 for i in range(512)), page=16, spare=70000),
        # one token of four dialogues, K and V straight into the pages: the call that each layer of a decode step makes
        _rotate("rotate_token", "1,1,1,1", "2064,16384,511,5462", to="pages", page=16),
        # the opening turn of a 32k dialogue, q, k and v as they leave one projection
        _rotate("rotate_32k", "32768", "0"),
        # what a server has waiting: prompts of many lengths, K both as rows for the attention and into the pages
        _rotate("rotate_prompts", "5003,61,1777,1,8192,300,128,2500,17,777,4096,1045", "0,0,0,0,0,0,0,0,0,0,0,0", to="both"),
        # a small fp32 model, half of each head rotated, neighbours as pairs, only keys normed; the last one's turn is a late one
        _rotate("rotate_fp32", "1024,37,300", "0,500,260000", Hq=4, Hkv=1, d=64, dims=32, dtype="f32", neighbours=True, norms="k", fused=False),
        # the newest third of a 32k dialogue into 4-bit pages, and the whole context back
        _turn("turn_32k", "21845", "10923"),
        # short follow-ups of some ragged caches, padded, fp32 rows
        _turn("turn_ragged", "777,1,2500,131", "5,61,1,12", page=16, Hkv=4, d=64, dtype="f32", packed=False),
        # one token over a short cache of one dialogue
        _token("token_b1", "519", page=16),
        # one token of four dialogues of 70B-class heads
        _token("token_16k_b4", "16384,16384,16384,16384", Hq=64),
        # the longest context there is
        _token("token_131k", "131072", page=128),
    ]


HEADS = [(32, 8), (64, 8), (16, 4), (8, 2), (8, 8), (4, 1), (32, 1), (12, 3)]
MOST_ROWS = 32768 * 40 * 128                   # rows x heads x values of the largest rotation listed
MOST_CACHE = 8 * 128 * 32768                   # heads x values x positions of the largest context that comes back
MOST_SEEN = 8 * 128 * 131072                   # heads x values x positions that tokens attend over
MOST_NEW = 1 << 20                             # rows that sequences grow by


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["resize", "rotate", "rotate", "turn", "token", "token"])
    hq, hkv = rng.choice(HEADS)
    d = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    if kind == "resize":
        B = _log(rng, 1, 700)
        lens, add = [], []
        for _ in range(B):
            what = rng.choice(["new", "run", "run", "run", "run", "end", "cut", "idle"])
            n = 0 if what == "new" else _log(rng, 1, 20000)
            lens.append(n)
            add.append(_log(rng, 1, 8192) if what == "new" else 1 if what == "run" else -n if what == "end" else -min(n, rng.randint(1, 40)) if what == "cut" else 0)
        while sum(max(x, 0) for x in add) > MOST_NEW:
            add = [x // 2 if x > 1 else x for x in add]
        # sometimes fewer pages are left than are asked for
        asked = sum(-(-(n + x) // page) + (-n // page) for n, x in zip(lens, add) if x > 0)
        spare = max(1, asked // 2) if rng.random() < 0.2 else asked + rng.randint(1, 300)
        return dict(kind=kind, lens=_text(lens), add=_text(add), page=page, max_pages=-(-40000 // page), spare=spare, padding=rng.choice([0, 0, 1, 33, 500]))
    if kind == "rotate":
        token = rng.random() < 0.3
        rows = [1 if token else _log(rng, 1, 32768) for _ in range(rng.choice([1, 1, 2, 5, 16, 40]))]
        while sum(rows) * (hq + hkv) * d > MOST_ROWS // 2:
            rows = [max(1, x * 3 // 4) for x in rows]
        at = [0 if rng.random() < 0.4 else _log(rng, 1, 262144) for _ in rows]
        to = rng.choice(["rows", "pages", "both"])
        while to != "rows" and sum(a + r for a, r in zip(at, rows)) * hkv * d > MOST_SEEN:
            at = [a // 2 for a in at]
        f32 = rng.random() < 0.2 and to == "rows"
        return dict(kind=kind, rows=_text(rows), at=_text(at), Hq=hq, Hkv=hkv, d=d, dims=rng.choice([d, d, d // 2, d // 4, 48]), dtype="f32" if f32 else "bf16",
                    neighbours=rng.random() < 0.3, norms=rng.choice(["qk", "qk", "k", ""]), fused=rng.random() < 0.5, to=to, page=page)
    if kind == "token":
        lens = [_log(rng, 1, 131072) - (rng.random() < 0.05) for _ in range(rng.choice([1, 1, 2, 4, 13, 32, 64]))]
        while hkv * d * len(lens) * max(lens) > MOST_SEEN:
            lens = [x * 3 // 4 for x in lens]
        return dict(kind=kind, lens=_text(lens), Hq=hq, Hkv=hkv, d=d, page=page)
    rows = [_log(rng, 1, 16384) for _ in range(rng.choice([1, 2, 4, 13]))]
    at = [0 if rng.random() < 0.3 else _log(rng, 1, 16384) for _ in rows]
    while hkv * d * len(rows) * max(a + r for a, r in zip(at, rows)) > MOST_CACHE:
        rows, at = [max(1, x * 3 // 4) for x in rows], [x * 3 // 4 for x in at]
    return dict(kind=kind, at=_text(at), rows=_text(rows), Hkv=hkv, d=d, page=page, dtype="f32" if rng.random() < 0.2 else "bf16", packed=rng.random() < 0.6)


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


def _table(lens, page, spare, g, width=0):
    """Pages of each sequence, drawn from the whole pool; entries past its end are no page.  And the pages that are left."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + spare, device="cuda", generator=g).int()
    n = torch.tensor(need, device="cuda")
    j = torch.arange(max(width, 1, max(need)), device="cuda")[None]
    at = (n.cumsum(0) - n)[:, None] + j
    table = torch.where(j < n[:, None], order[at.clamp(max=max(0, sum(need) - 1))] if sum(need) else 0, -1).int()
    return table, order[sum(need):].contiguous()


# The values of e2m1's codes, and the magnitudes that a code begins behind (ties go to the even one)
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
_TIES = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]


def _power(E):
    """2^(E - 127) from its bits"""
    return (E.int() << 23).view(torch.float32)


def _codes4(x, bounds):
    """Rows of fp32 values [..,d] as e2m1: bytes of two codes [..,d/2], and an exponent byte for each 32 values: the least power of two 2^(E-127), of
    2^-125 and above, by which their largest is 7 or less."""
    g = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1))
    E = torch.where(m == 0, 2, (e + 124 + (m > 0.875)).clamp_min(2))
    y = g * _power(254 - E)[..., None]
    code = (torch.bucketize(y.abs(), bounds, out_int32=True) + 8 * torch.signbit(y)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, E.to(torch.uint8)


def _bounds():
    """bucketize() counts the bounds below a value: those whose tie goes up are one step lower."""
    t = torch.tensor(_TIES, device="cuda")
    return torch.where(torch.arange(7, device="cuda") % 2 == 1, torch.nextafter(t, torch.zeros_like(t)), t)


def _pairs():
    """[256,2]: what the two codes of a byte stand for."""
    v = torch.tensor(_E2M1 + [-x for x in _E2M1], device="cuda")
    b = torch.arange(256, device="cuda")
    return torch.stack([v[b & 15], v[b >> 4]], 1)


def _values4(codes, E, pairs):
    return (pairs[codes.int()].flatten(-2).unflatten(-1, (-1, 32)) * _power(E)[..., None]).flatten(-2)


def _pool4(c, pages, rnd):
    bounds = _bounds()
    out = {}
    for name in ("k", "v"):
        out[name], out[name + "_exp"] = _codes4(rnd(pages, c["Hkv"], c["page"], c["d"]), bounds)
    return out


def _places(at, rows):
    """Of rows in order: whose each is, its number there, its position."""
    n = torch.tensor(rows, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), n)
    i = torch.arange(sum(rows), device="cuda") - (n.cumsum(0) - n)[seq]
    return seq, i, torch.tensor(at, device="cuda")[seq] + i


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    s = dict(case=c)
    if own:
        from paper_2507_13681_amd import binding
    if c["kind"] == "resize":
        lens, add = _ints(c["lens"]), _ints(c["add"])
        B, rows = len(lens), max(1, sum(max(x, 0) for x in add) + c["padding"])
        s["table"], left = _table(lens, c["page"], c["spare"], g, c["max_pages"])
        pages = s["pages"] = sum(-(-n // c["page"]) for n in lens) + c["spare"]
        head = int(torch.randint(pages, (1,), device="cuda", generator=g))
        s["free"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")          # a ring: it begins anywhere
        s["free"][(head + torch.arange(len(left), device="cuda")) % pages] = left
        s["state"], s["lens"], s["add"] = _i32([head, len(left)]), _i32(lens), _i32(add)
        s["new_state"], s["new_lens"], s["starts"] = torch.empty_like(s["state"]), torch.empty_like(s["lens"]), _i32([0] * (B + 1))
        s["positions"], s["slots"] = _i32([0] * rows), torch.zeros(rows, dtype=torch.int64, device="cuda")
        if own:
            s["shape"] = binding.make_shape(B, 1, 1, 64, 1, rows, 1, "bf16")
            s["ctx"] = binding.Context(workspace=0)
            pool = torch.empty(2, pages, 1, c["page"], 64, dtype=torch.bfloat16, device="cuda")       # of one layer
            s["cache"] = binding.PagedCache(pool[0], pool[1])
        return s
    if c["kind"] == "rotate":
        Hq, Hkv, d, dt = c["Hq"], c["Hkv"], c["d"], _type(c["dtype"])
        rows, at = _ints(c["rows"]), _ints(c["at"])
        T, H = sum(rows), Hq + 2 * Hkv
        x = torch.empty(T, H, d, dtype=dt, device="cuda")
        for h in range(H):                                 # heads of different sizes, and a few channels that are large
            x[:, h] = (rnd(T, d) * (0.5 + 0.3 * (h % 5)) * (1 + 7 * (torch.rand(d, device="cuda", generator=g) < 0.04))).to(dt)
        s["q"], s["k"], s["v"] = (x[:, a:b] if c["fused"] else x[:, a:b].clone() for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, H)))
        seq, i, p = _places(at, rows)
        s["positions"] = p.int()
        s["freq"] = torch.pow(torch.tensor(500000.0, dtype=torch.float64), -torch.arange(0, c["dims"], 2, dtype=torch.float64) / c["dims"]).float().cuda()
        s["q_weight"] = 1 + 0.2 * rnd(d) if "q" in c["norms"] else None
        s["k_weight"] = 1 + 0.2 * rnd(d) if "k" in c["norms"] else None
        s["eps"] = 1e-6
        s["q_out"] = torch.empty(T, Hq, d, dtype=dt, device="cuda")
        s["k_out"] = torch.empty(T, Hkv, d, dtype=dt, device="cuda") if c["to"] != "pages" else None
        s["pool"] = s["slots"] = None
        if c["to"] != "rows":
            table, left = _table([a + r for a, r in zip(at, rows)], c["page"], 3, g)
            pages = int(table.max()) + 4
            s["slots"] = table.long()[seq, p // c["page"]] * c["page"] + p % c["page"]
            s["pool"] = {n: torch.zeros(pages, Hkv, c["page"], d, dtype=torch.bfloat16, device="cuda") for n in ("k", "v")}
        if own:
            s["shape"] = binding.make_shape(1, Hq, Hkv, d, T, T, 1, c["dtype"])
            s["ctx"] = binding.Context(workspace=0)
            s["rotation"] = binding.Rotation(s["freq"], neighbours=c["neighbours"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"])
            s["cache"] = binding.PagedCache(**s["pool"]) if s["pool"] else None
        return s
    if c["kind"] == "token":
        lens = _ints(c["lens"])
        B = len(lens)
        s["table"], left = _table(lens, c["page"], 3, g)
        s["pool"] = _pool4(c, max(int(s["table"].max()), 0) + 4, rnd)
        s["q"] = (1.5 * rnd(B, c["Hq"], c["d"])).to(torch.bfloat16)
        s["len"], s["pairs"], s["most"] = _i32(lens), _pairs(), max(1, max(lens))
        if own:
            s["shape"] = binding.make_shape(B, c["Hq"], c["Hkv"], c["d"], max(1, max(lens)), 1, 1, "bf16")
            s["ctx"] = binding.Context(workspace=binding.paged_workspace_bytes(s["shape"]))
            s["cache"] = binding.PagedCache(**s["pool"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(B, c["Hq"], device="cuda")
        return s
    at, rows = _ints(c["at"]), _ints(c["rows"])
    B, ends, dt = len(at), [a + r for a, r in zip(at, rows)], _type(c["dtype"])
    s["table"], left = _table(ends, c["page"], 3, g)
    s["pool"] = _pool4(c, int(s["table"].max()) + 4, rnd)
    s["bounds"], s["pairs"] = _bounds(), _pairs()
    s["new"], s["whole"] = _places(at, rows), _places([0] * B, ends)        # places of the rows that go in, and of those that come back
    form = lambda n: (sum(n), c["Hkv"], c["d"]) if c["packed"] else (B, c["Hkv"], max(n), c["d"])
    big = 1 + 9 * (torch.rand(c["Hkv"], 1, c["d"], device="cuda", generator=g) < 0.04).float()      # a few channels of K are large
    s["k_rows"], s["v_rows"] = (rnd(*form(rows)) * (big.transpose(0, 1) if c["packed"] else big)).to(dt), rnd(*form(rows)).to(dt)
    s["k_back"], s["v_back"] = torch.zeros(form(ends), dtype=dt, device="cuda"), torch.zeros(form(ends), dtype=dt, device="cuda")
    s["pos"] = _i32(at)
    s["starts"], s["count"] = (_i32(_starts(rows)), None) if c["packed"] else (None, _i32(rows))
    s["all_starts"], s["all_count"] = (_i32(_starts(ends)), None) if c["packed"] else (None, _i32(ends))
    if own:
        s["shape"], s["all_shape"] = (binding.make_shape(B, c["Hkv"], c["Hkv"], c["d"], 1, sum(n) if c["packed"] else max(n), 1, c["dtype"]) for n in (rows, ends))
        s["ctx"] = binding.Context(workspace=0)
        s["cache"] = binding.PagedCache(**s["pool"])
    return s


# ---- the plain forms ---------------------------------------------------------------------------------

def _plain_resize(s):
    """What needs no pages, or asks for no more than are left behind those before it, gets them."""
    c = s["case"]
    page, pages, room = c["page"], s["pages"], c["max_pages"] * c["page"]
    old, add = s["lens"].long(), s["add"].long()
    n_rows = len(s["slots"])
    head, count = s["state"].long()
    new = (old + add).clamp_min(0)
    rows = add.clamp_min(0)
    rows = torch.where(rows.cumsum(0) <= n_rows, rows, 0)
    starts = torch.cat([torch.zeros_like(rows[:1]), rows.cumsum(0)])
    have, want = (old + page - 1) // page, (new + page - 1) // page
    grows = (rows > 0) & (new <= room)
    need = torch.where(grows, want - have, 0)
    behind = need.cumsum(0)
    grows &= (need == 0) | (behind <= count)
    taken = torch.where(grows & (need > 0), behind, 0).amax()
    shrinks = add < 0
    give = torch.where(shrinks, have - want, 0)
    j = torch.arange(c["max_pages"], device="cuda")[None]
    to = head + count + (give.cumsum(0) - give)[:, None] + j - want[:, None]
    free = torch.cat([s["free"], s["free"][:1]])           # (one place more, for what is not given back)
    free[torch.where(shrinks[:, None] & (j >= want[:, None]) & (j < have[:, None]), to % pages, pages)] = s["table"]
    here = (head + (behind - need)[:, None] + j - have[:, None]) % pages
    s["table"] = torch.where(grows[:, None] & (j >= have[:, None]) & (j < want[:, None]), s["free"][here], s["table"])
    s["free"] = free[:pages]
    r = torch.arange(n_rows, device="cuda")
    b = torch.searchsorted(starts[1:], r, right=True)
    on = b < len(old)
    b = b.clamp(max=len(old) - 1)
    on &= grows[b]
    p = torch.where(on, old[b] + r - starts[b], 0)
    slots = torch.where(on, s["table"].long()[b, p // page] * page + p % page, -1)
    state = torch.stack([(head + taken) % pages, count - taken + give.sum()])
    return dict(free=s["free"], state=state.int(), lens=torch.where(grows | shrinks, new, old).int(), table=s["table"], starts=starts.int(),
                positions=p.int(), slots=slots)


def _plain_rotate(s):
    c = s["case"]
    r = c["dims"]
    angle = s["positions"].double()[:, None] * s["freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def one(x, w):
        x = x.float()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w
        a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["neighbours"] else (x[..., :r // 2], x[..., r // 2:r])
        y = [a * cos - b * sin, b * cos + a * sin]
        y = torch.stack(y, -1).flatten(-2) if c["neighbours"] else torch.cat(y, -1)
        return torch.cat([y, x[..., r:]], -1).to(_type(c["dtype"]))

    q, k = one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])
    if c["to"] != "rows":
        page, place = s["slots"] // c["page"], s["slots"] % c["page"]
        s["pool"]["k"][page, :, place] = k
        s["pool"]["v"][page, :, place] = s["v"]
    return dict(q=q, k=k if c["to"] != "pages" else None, pool=s["pool"])


def _page_places(s, places):
    seq, i, p = places
    return s["table"].long()[seq, p // s["case"]["page"]], p % s["case"]["page"]


def _plain_turn(s):
    c = s["case"]
    page, place = _page_places(s, s["new"])
    page_all, place_all = _page_places(s, s["whole"])
    back = {}
    for name in ("k", "v"):
        x = s[name + "_rows"] if c["packed"] else s[name + "_rows"][s["new"][0], :, s["new"][1]]
        codes, exps = s["pool"][name], s["pool"][name + "_exp"]
        codes[page, :, place], exps[page, :, place] = _codes4(x.float(), s["bounds"])
        y = _values4(codes[page_all, :, place_all], exps[page_all, :, place_all], s["pairs"]).to(_type(c["dtype"]))
        if c["packed"]:
            back[name] = y
        else:
            back[name] = s[name + "_back"]
            back[name][s["whole"][0], :, s["whole"][1]] = y
    return back


def _plain_token(s):
    c = s["case"]
    Hkv, d = c["Hkv"], c["d"]
    B = len(s["len"])
    pages = s["table"].long().clamp_min(0)
    K, V = (_values4(s["pool"][t][pages], s["pool"][t + "_exp"][pages], s["pairs"]).transpose(1, 2).reshape(B, Hkv, -1, d)[:, :, :s["most"]] for t in ("k", "v"))
    x = torch.matmul(s["q"].float().view(B, Hkv, -1, d), K.transpose(2, 3).contiguous()) / math.sqrt(d)
    x = torch.where(torch.arange(s["most"], device="cuda") < s["len"][:, None, None, None], x, -math.inf)
    some = (s["len"] > 0)[:, None, None, None]
    m = torch.where(some, x.amax(3, keepdim=True), 0)
    p = torch.exp(x - m)
    l = p.sum(3, keepdim=True)
    out = torch.where(some, torch.matmul(p, V.contiguous()) / l, 0)
    return dict(out=out.view(B, c["Hq"], d).to(torch.bfloat16), lse=(m + torch.log(l)).view(B, c["Hq"]))


def run(s):
    kind = s["case"]["kind"]
    if not own:
        if kind == "resize":
            return _plain_resize(s)
        if kind == "rotate":
            return _plain_rotate(s)
        if kind == "turn":
            return _plain_turn(s)
        return _plain_token(s)
    ctx = s["ctx"]
    if kind == "resize":
        ctx.ls_cache_resize(s["shape"], s["cache"], s["free"], s["state"], s["add"], s["lens"], s["table"], new_state=s["new_state"], new_lens=s["new_lens"],
                            starts=s["starts"], positions=s["positions"], slots=s["slots"])
        return dict(free=s["free"], state=s["new_state"], lens=s["new_lens"], table=s["table"], starts=s["starts"], positions=s["positions"], slots=s["slots"])
    if kind == "rotate":
        ctx.ls_norm_rotate(s["shape"], s["rotation"], s["q"], s["k"], s["q_out"], s["k_out"], positions=s["positions"],
                           cache=s["cache"], v=s["v"] if s["cache"] else None, slots=s["slots"])
        return dict(q=s["q_out"], k=s["k_out"], pool=s["pool"])
    if kind == "turn":
        ctx.ls_cache_write(s["shape"], s["cache"], s["k_rows"], s["v_rows"], s["table"], s["pos"], s["starts"], s["count"])
        ctx.ls_cache_read(s["all_shape"], s["cache"], s["table"], s["k_back"], s["v_back"], starts=s["all_starts"], count=s["all_count"])
        return dict(k=s["k_back"], v=s["v_back"])
    ctx.ls_paged_attend(s["shape"], s["cache"], s["q"], s["table"], s["len"], s["out"], s["lse"])
    return dict(out=s["out"], lse=s["lse"])


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _exact_resize(s):
    """Sequence by sequence, on the host."""
    c = s["case"]
    page, pages, room = c["page"], s["pages"], c["max_pages"] * c["page"]
    free, table, lens, add = s["free"].tolist(), s["table"].cpu(), s["lens"].tolist(), s["add"].tolist()
    head, count = s["state"].tolist()
    n_rows = len(s["slots"])
    starts, positions, slots = [0], torch.zeros(n_rows, dtype=torch.int32), torch.full((n_rows,), -1)
    got, asked, taken, given, room_left = free[:], 0, 0, 0, True
    for b, (old, by) in enumerate(zip(lens, add)):
        new, have = max(0, old + by), -(-old // page)
        want = -(-new // page)
        rows = max(by, 0)
        room_left = room_left and starts[-1] + rows <= n_rows
        rows = rows if room_left else 0
        starts.append(starts[-1] + rows)
        if by < 0:
            for j in range(want, have):
                got[(head + count + given) % pages] = int(table[b, j])
                given += 1
            lens[b] = new
        elif rows and new <= room:
            asked += want - have
            if want > have and asked > count:
                continue
            if want > have:
                taken = asked
                first = head + asked - (want - have)
                table[b, have:want] = torch.tensor([free[(first + j) % pages] for j in range(want - have)], dtype=torch.int32)
            p = torch.arange(old, new)
            positions[starts[b]:starts[b + 1]] = p.int()
            slots[starts[b]:starts[b + 1]] = table[b].long()[p // page] * page + p % page
            lens[b] = new
    state = [(head + taken) % pages, count - taken + given]
    return dict(free=_i32(got), state=_i32(state), lens=_i32(lens), table=table.cuda(), starts=_i32(starts), positions=positions.cuda(), slots=slots.cuda())


def _exact_rotate(s):
    c = s["case"]
    r = c["dims"]
    first = torch.arange(r // 2, device="cuda") * (2 if c["neighbours"] else 1)
    second = first + (1 if c["neighbours"] else r // 2)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["freq"].double())
    out = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for h in range(x.shape[1]):
            z = x[:, h].double()
            if w is not None:
                z = z * torch.rsqrt(torch.linalg.vector_norm(z, dim=1, keepdim=True) ** 2 / c["d"] + s["eps"]) * w.double()
            y[:, h] = z
            t = torch.complex(z[:, first], z[:, second]) * turn
            y[:, h, first], y[:, h, second] = t.real, t.imag
        out.append(y)
    pool = None
    if s["pool"] is not None:
        pool = {n: x.double() for n, x in s["pool"].items()}
        flat = {n: x.transpose(1, 2).reshape(-1, c["Hkv"], c["d"]) for n, x in pool.items()}
        flat["k"][s["slots"]], flat["v"][s["slots"]] = out[1], s["v"].double()
        pool = {n: x.view(-1, c["page"], c["Hkv"], c["d"]).transpose(1, 2) for n, x in flat.items()}
    return dict(q=out[0], k=out[1] if c["to"] != "pages" else None, pool=pool)


def _stored64(s, name, page, place, head):
    """[n,d] of one KV head"""
    v = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=torch.float64, device="cuda")
    two = s["pool"][name][page, head, place].long()
    x = torch.stack([v[two % 16], v[two // 16]], 2).reshape(len(two), -1)
    E = s["pool"][name + "_exp"][page, head, place].double()
    return x * torch.exp2(E - 127).repeat_interleave(32, 1)


def _nearest64(x):
    """Rows [n,d] as 4 bits hold them: of all powers of two 2^-125 .. 2^126 the least that is enough for each 32 values, and the nearest code."""
    g = x.unflatten(-1, (-1, 32))
    powers = torch.exp2(torch.arange(-125, 127, dtype=torch.float64, device="cuda"))
    p = powers[torch.searchsorted(7 * powers, g.abs().amax(-1).clamp_min(7 * 2.0 ** -125))][..., None]
    a = (g / p).abs()
    v = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
    hi = torch.searchsorted(v, a.clamp(max=6.0)).clamp(max=7)
    lo = (hi - 1).clamp_min(0)
    down, up = a - v[lo], v[hi] - a
    return (v[torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)] * torch.sign(g) * p).flatten(-2)


def _exact_turn(s):
    c = s["case"]
    out = {n: s[n + "_back"].double() for n in ("k", "v")}
    new = whole = 0
    for b, (at, rows) in enumerate(zip(_ints(c["at"]), _ints(c["rows"]))):
        p = torch.arange(at, device="cuda")
        page, place = s["table"][b].long()[p // c["page"]], p % c["page"]
        for n in ("k", "v"):
            for h in range(c["Hkv"]):
                x = s[n + "_rows"][new:new + rows, h] if c["packed"] else s[n + "_rows"][b, h, :rows]
                y = torch.cat([_stored64(s, n, page, place, h), _nearest64(x.double())])
                if c["packed"]:
                    out[n][whole:whole + at + rows, h] = y
                else:
                    out[n][b, h, :at + rows] = y
        new, whole = new + rows, whole + at + rows
    return out


def _exact_token(s):
    c = s["case"]
    G, d = c["Hq"] // c["Hkv"], c["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_ints(c["lens"])):
        if n == 0:
            continue
        p = torch.arange(n, device="cuda")
        page, place = s["table"][b].long()[p // c["page"]], p % c["page"]
        for j in range(c["Hkv"]):
            x = torch.matmul(s["q"][b, j * G:(j + 1) * G].double(), _stored64(s, "k", page, place, j).T.contiguous()) / math.sqrt(d)
            lse[b, j * G:(j + 1) * G] = torch.logsumexp(x, 1)
            out[b, j * G:(j + 1) * G] = torch.matmul(torch.softmax(x, 1), _stored64(s, "v", page, place, j))
    return dict(out=out, lse=lse)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "resize":
        return _exact_resize(s)
    if case["kind"] == "rotate":
        return _exact_rotate(s)
    if case["kind"] == "turn":
        return _exact_turn(s)
    return _exact_token(s)


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "resize":
        lens, add, page = _ints(c["lens"]), _ints(c["add"]), c["page"]
        pages = sum(abs(-(-(n + x) // page) + (-n // page)) for n, x in zip(lens, add))
        return dict(bytes=20 * len(lens) + 8 * pages + 12 * (sum(max(x, 0) for x in add) + c["padding"]), flops=0)
    d, Hkv, e = c["d"], c["Hkv"], 2 if c.get("dtype") != "f32" else 4
    if c["kind"] == "rotate":
        T = sum(_ints(c["rows"]))
        moved = 2 * c["Hq"] + Hkv + Hkv * {"rows": 1, "pages": 3, "both": 4}[c["to"]]            # rows of heads that are read or written
        return dict(bytes=T * (moved * d * e + 4 + (8 if c["to"] != "rows" else 0)), flops=T * (c["Hq"] + Hkv) * 6.0 * d)
    stored = d // 2 + d // 32                                                                    # bytes of a row in the cache
    if c["kind"] == "token":
        lens = _ints(c["lens"])
        return dict(bytes=2 * Hkv * stored * sum(lens) + (4 * d + 4) * len(lens) * c["Hq"] + 4 * sum(lens) // c["page"], flops=4.0 * d * c["Hq"] * sum(lens))
    rows, whole = sum(_ints(c["rows"])), sum(_ints(c["at"])) + sum(_ints(c["rows"]))
    return dict(bytes=2 * Hkv * ((rows + whole) * (stored + d * e)), flops=0)
