"""ls_norm_rotate: what the host refuses (no GPU)."""
import ctypes as C

import pytest

from paper_2507_13681_amd import binding
from tests.test_serving_host import EINVAL, ESHAPE, HERE, _cache, _rows, _shape, lib  # noqa: F401


def test_layout_matches_the_header():
    assert C.sizeof(binding.LsRotation) == 40 and binding.LsRotation.dims.offset == 24 and binding.LsRotation.eps.offset == 32


NAN, INF = float("nan"), float("inf")
ROTATE = [
    (dict(), 0), (dict(cache=None, v=None, slots=None), 0), (dict(k_out=None), 0), (dict(positions=None), 0), (dict(rot=dict(dims=0, freq=None)), 0),
    (dict(rot=dict(q_weight=None, k_weight=None)), 0), (dict(rot=dict(eps=0.0, pairs=1)), 0),
    (dict(k_out=None, cache=None, v=None, slots=None), EINVAL), (dict(v=None), EINVAL), (dict(slots=None), EINVAL), (dict(cache=None), EINVAL), (dict(rot=None), EINVAL),
    (dict(rot=dict(freq=None)), EINVAL), (dict(rot=dict(freq=HERE + 4)), EINVAL), (dict(rot=dict(k_weight=HERE + 8)), EINVAL), (dict(rot=dict(pairs=2)), EINVAL),
    (dict(rot=dict(dims=8)), ESHAPE), (dict(rot=dict(dims=144)), ESHAPE), (dict(rot=dict(dims=-16)), ESHAPE), (dict(rot=dict(eps=-1e-9)), EINVAL), (dict(rot=dict(eps=NAN)), EINVAL),
    (dict(rot=dict(eps=INF)), EINVAL), (dict(positions=HERE + 2), EINVAL), (dict(slots=HERE + 4), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(q_out=None), EINVAL),
    (dict(q_out=_rows(row=512, head=128, seq=102400)), ESHAPE), (dict(k_out=_rows(row=0, seq=51200)), ESHAPE), (dict(k=_rows(row=0, head=0, data=HERE + (1 << 24))), 0), (dict(v=_rows(data=HERE + 8)), EINVAL),
    (dict(shape=dict(d=96)), ESHAPE), (dict(shape=dict(Hq=6)), ESHAPE), (dict(shape=dict(n_hat=0)), ESHAPE), (dict(shape=dict(n_hat=2 ** 31)), ESHAPE), (dict(shape=dict(n_hat=2 ** 62)), ESHAPE),
    (dict(shape=dict(n_hat=2147483000)), ESHAPE), (dict(shape=dict(B=0)), ESHAPE), (dict(shape=dict(B=9000)), ESHAPE), (dict(cache=dict(page=24)), ESHAPE), (dict(cache=dict(Hkv=2)), ESHAPE),
    (dict(cache=dict(type=2)), EINVAL), (dict(cache=dict(type=4)), 0), (dict(cache=dict(type=0, k_exp=None, v_exp=None)), 0), (dict(cache=dict(type=4, v_exp=None)), EINVAL), (dict(cache=dict(pages=0)), ESHAPE),
]

AT = HERE + (1 << 24)
ROTATE += [     # in place, with the strides of the rows that are read and with others; of a row or a head the stride is nobody's
    (dict(q=_rows(row=1024, seq=102400, data=AT), q_out=_rows(row=1024, seq=102400, data=AT)), 0), (dict(q=_rows(row=2048, seq=204800, data=AT), q_out=_rows(row=1024, seq=102400, data=AT)), EINVAL),
    (dict(q=_rows(row=1024, seq=204800, data=AT), q_out=_rows(row=1024, seq=102400, data=AT)), EINVAL), (dict(k=_rows(seq=51200, data=AT), k_out=_rows(seq=51200, data=AT)), 0),
    (dict(k=_rows(row=0, head=0, data=AT), k_out=_rows(seq=51200, data=AT)), EINVAL), (dict(k=_rows(row=2048, seq=51200, data=AT), k_out=_rows(seq=51200, data=AT), shape=dict(n_hat=1)), 0),
]


@pytest.mark.parametrize("change,want", ROTATE)
def test_refusals(lib, change, want):  # noqa: F811
    a = dict(rot={}, q=_rows(row=1024, seq=102400), k=_rows(seq=51200), positions=HERE, q_out=_rows(row=1024, seq=102400), k_out=_rows(seq=51200), cache={}, v=_rows(seq=51200), slots=HERE)
    a.update({n: x for n, x in change.items() if n in a})
    s = _shape(**change.get("shape", {}))
    rot = None
    if a["rot"] is not None:
        r = dict(freq=HERE, q_weight=HERE, k_weight=HERE, dims=128, pairs=0, eps=1e-6)
        r.update(a["rot"])
        rot = C.byref(binding.LsRotation(*[r[f[0]] for f in binding.LsRotation._fields_]))
    ref = lambda x: None if x is None else C.byref(x)
    cache = None if a["cache"] is None else C.byref(_cache(**a["cache"]))
    assert lib.ls_debug_check_rotate(C.byref(s), rot, ref(a["q"]), ref(a["k"]), a["positions"], ref(a["q_out"]), ref(a["k_out"]), cache, ref(a["v"]), a["slots"]) == want
