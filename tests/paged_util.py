"""Plain forms in 64 bits of the calls on pages and packed sequences, and how far results may be from them."""
import numpy as np
import torch

E4M3 = torch.float8_e4m3fn
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # largest relative error of one rounding


def rnd(rng, *shape, scale=1.0, dtype=torch.bfloat16):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype)


def attention(q, k, v, last, scale):
    """Row r of q [R,d] over the keys 0 .. last[r] of k, v [n,d], in 64 bits: out, lse, and the bounds of what a kernel may be off by.

    A kernel's logit is a sum of d products in fp32, off by at most (d + 2) 2^-24 sum |q k| scale, and the exponent that it becomes by 2^-22 of itself for its factor and sum and of 1 for the
    exponential; so far its probabilities are off, relatively, and once more by `half` where they are rounded to the storage type.  Sums over n keys in fp32 add
    n 2^-24 at most.  The output is a mean of v with these weights, divided by their sum, and rounded once."""
    q, k, v = (x.double().numpy() for x in (q, k, v))
    R, n = q.shape[0], k.shape[0]
    x = q @ k.T * scale
    x = np.where(np.arange(n)[None] <= np.asarray(last)[:, None], x, -np.inf)
    seen = np.isfinite(x).any(1) if n else np.zeros(R, bool)
    out, lse = np.zeros((R, v.shape[1])), np.full(R, -np.inf)
    err, lerr = np.zeros(R), np.zeros(R)
    mean_abs = np.zeros_like(out)
    if seen.any():
        y = x[seen]
        m = y.max(1, keepdims=True)
        p = np.exp(y - m)
        l = p.sum(1, keepdims=True)
        out[seen] = p @ v / l
        mean_abs[seen] = p @ np.abs(v) / l
        lse[seen] = (m + np.log(l))[:, 0]
        most = np.where(np.isfinite(y), np.abs(q[seen]) @ np.abs(k).T * scale, 0.0).max(1)
        size = np.where(np.isfinite(y), np.abs(y), 0.0).max(1)
        one = (q.shape[1] + 2) * 2.0 ** -24 * most + 2.0 ** -22 * (1.0 + 2.0 * size)
        err[seen] = 2.0 * one + 2.0 * n * 2.0 ** -24 + 2.0 ** -21
        lerr[seen] = one + n * 2.0 ** -24 + 2.0 ** -21 * (1.0 + np.abs(lse[seen]))
    return out, lse, mean_abs, err, lerr


def check(got, got_lse, ref, dtype):
    """got [R,d], got_lse [R] or None against what attention() gave."""
    out, lse, mean_abs, err, lerr = ref
    half = HALF[dtype]
    got = got.double().cpu().numpy()
    tol = half * np.abs(out) + (err[:, None] + (half if dtype == torch.bfloat16 else 0.0)) * mean_abs * 1.01 + 1e-30
    off = np.abs(got - out)
    assert np.isfinite(got).all()
    assert (off <= tol).all(), (float((off / tol).max()), np.unravel_index(int((off / tol).argmax()), off.shape))
    empty = np.isneginf(lse)
    assert (got[empty] == 0).all()
    if got_lse is not None:
        got_lse = got_lse.double().cpu().numpy()
        assert np.isneginf(got_lse[empty]).all()
        assert (np.abs(got_lse[~empty] - lse[~empty]) <= lerr[~empty]).all(), float((np.abs(got_lse[~empty] - lse[~empty]) - lerr[~empty]).max())


def exponents(x):
    """127 + e of the least power of two 2^e >= 2^-117 by which each row's largest finite value is at most 448, from its bits."""
    x = x.float()
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    u = top.view(torch.int32)
    e = (u >> 23) - 8 + ((u & 0x7FFFFF) > 0x600000).int()
    return e.clamp_min(10).to(torch.uint8)


def power(E):
    return (E.int() << 23).view(torch.float32)[..., None]


def codes(x, E):
    """e4m3 of x 2^(127 - E), as bytes."""
    return (x.float() * power(254 - E.int())).to(E4M3).view(torch.uint8)


def values(c, E):
    return c.view(E4M3).float() * power(E)


def pool(rng, pages, Hkv, page, d, kind, scale=1.0):
    """Random pages on the CPU: dict(k, v[, k_exp, v_exp])."""
    out = {}
    for name in ("k", "v"):
        x = rnd(rng, pages, Hkv, page, d, scale=scale, dtype=torch.float32)
        if kind == "bf16":
            out[name] = x.to(torch.bfloat16)
        else:
            out[name + "_exp"] = exponents(x)
            out[name] = codes(x, out[name + "_exp"])
    return out


def stored(p, name):
    """What the pages hold, fp32 [pages,Hkv,page,d]."""
    return p[name].float() if name + "_exp" not in p else values(p[name], p[name + "_exp"])


def table_for(rng, lens, page, pages, width=None):
    """Distinct pages of each sequence; entries past its end are no page."""
    need = [-(-n // page) for n in lens]
    assert sum(need) <= pages
    order = rng.permutation(pages)
    width = width or max(1, max(need))
    t, at = np.full((len(lens), width), -1, np.int32), 0
    for s, m in enumerate(need):
        t[s, :m] = order[at:at + m]
        at += m
    return torch.from_numpy(t)
