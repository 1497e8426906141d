"""Pages of 4-bit floats (e2m1, a power of two for each 32 values) in plain form, in 64 bits."""
import torch

from tests import paged_util as pu

CODES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
BOTH = torch.cat([CODES, -CODES])


def exponents(x):
    """[..,d] -> [..,d/32]: the least byte E from 2 to 253 with max |x| <= 7 * 2^(E - 127); 255 where a value is infinite or none."""
    g = x.double().unflatten(-1, (-1, 32))
    top = torch.where(torch.isfinite(g), g.abs(), 0.0).amax(-1)
    E = 2 + torch.searchsorted(7 * torch.exp2(torch.arange(2, 254).double() - 127), top)
    return torch.where(torch.isfinite(g).all(-1), E, 255).to(torch.uint8)


def codes(x, E):
    """[..,d] -> [..,d/2] bytes: x * 2^(127 - E) to the nearest code, ties to the one with an even number; zeros where E is 255."""
    g = x.double().unflatten(-1, (-1, 32)) * torch.exp2(127 - E.double())[..., None]
    dist = (g.abs().clamp(max=6.0)[..., None] - CODES).abs()
    near = dist <= dist.amin(-1, keepdim=True)
    n = torch.arange(8)
    best = torch.where(near, n + 8 * (n % 2), 99).amin(-1) % 8          # of two that are as near, the even one
    best = torch.where(E[..., None] == 255, 0, best + 8 * torch.signbit(g)).flatten(-2).to(torch.uint8)
    return best[..., 0::2] | best[..., 1::2] << 4


def values(c, E):
    """fp64 [..,d]"""
    x = torch.stack([BOTH[(c & 15).long()], BOTH[(c >> 4).long()]], -1).flatten(-2)
    p = torch.where(E == 255, torch.nan, torch.exp2(E.double() - 127))
    return (x.unflatten(-1, (-1, 32)) * p[..., None]).flatten(-2)


def pool(rng, pages, Hkv, page, d, scale=1.0):
    """Random pages on the CPU: dict(k, v, k_exp, v_exp)."""
    out = {}
    for name in ("k", "v"):
        x = pu.rnd(rng, pages, Hkv, page, d, scale=scale, dtype=torch.float32)
        out[name + "_exp"] = exponents(x)
        out[name] = codes(x, out[name + "_exp"])
    return out


def empty(pages, Hkv, page, d, fill=0):
    u8 = dict(dtype=torch.uint8)
    return dict(k=torch.full((pages, Hkv, page, d // 2), fill, **u8), v=torch.full((pages, Hkv, page, d // 2), fill, **u8),
                k_exp=torch.full((pages, Hkv, page, d // 32), fill, **u8), v_exp=torch.full((pages, Hkv, page, d // 32), fill, **u8))


def stored(p, name):
    """What the pages hold, fp64 [pages,Hkv,page,d]."""
    return values(p[name], p[name + "_exp"])


def write(p, name, rows, places):
    """rows [N,Hkv,d] to places (sequence, index, page, place in the page)."""
    pg, pl = torch.tensor([x[2] for x in places]), torch.tensor([x[3] for x in places])
    E = exponents(rows)
    p[name + "_exp"][pg, :, pl] = E
    p[name][pg, :, pl] = codes(rows, E)
