"""ls_cache_resize: what the host refuses (no GPU)."""
import ctypes as C

import pytest

from paper_2507_13681_amd import binding
from tests.test_serving_host import EINVAL, ESHAPE, HERE, _cache, _shape, lib  # noqa: F401

RESIZE = [
    (dict(), 0), (dict(new_state=HERE, new_len=HERE + 4096), 0), (dict(starts=None, positions=None, slots=None), 0),
    (dict(free=None), EINVAL), (dict(state=None), EINVAL), (dict(new_state=None), EINVAL), (dict(add=None), EINVAL), (dict(len=None), EINVAL), (dict(new_len=None), EINVAL),
    (dict(table=None), EINVAL), (dict(cache=None), EINVAL), (dict(free=HERE + 2), EINVAL), (dict(slots=HERE + 4), EINVAL), (dict(starts=HERE + 1), EINVAL), (dict(positions=HERE + 3), EINVAL),
    (dict(new_state=HERE + 4), EINVAL), (dict(new_state=HERE - 4), EINVAL), (dict(new_state=HERE + 8), 0), (dict(new_len=HERE + 4100), EINVAL), (dict(new_len=HERE + 4104), 0),
    (dict(max_pages=0), ESHAPE), (dict(max_pages=-3), ESHAPE), (dict(cache=dict(page=12)), ESHAPE), (dict(cache=dict(pages=2 ** 31)), ESHAPE), (dict(cache=dict(pages=2 ** 31 - 1)), 0),
    (dict(cache=dict(type=4)), 0), (dict(cache=dict(type=7)), EINVAL), (dict(cache=dict(Hkv=3)), ESHAPE),
    (dict(shape=dict(n_hat=0)), ESHAPE), (dict(shape=dict(n_hat=2 ** 31)), ESHAPE), (dict(shape=dict(B=0)), ESHAPE), (dict(shape=dict(B=17000)), ESHAPE), (dict(shape=dict(Hq=0)), 0),
    (dict(shape=dict(n_hat=2147483000)), 0), (dict(starts=None, shape=dict(n_hat=2147483000)), ESHAPE), (dict(starts=None, shape=dict(n_hat=1073741500)), 0),
]

RESIZE += [(dict(add=HERE + 4096), EINVAL), (dict(add=HERE + 4100), EINVAL), (dict(add=HERE + 4092), EINVAL), (dict(add=HERE + 4104), 0), (dict(add=HERE + 4096, new_len=HERE + 8192), 0)]

# the cache and the shape are checked as the other calls on pages check theirs, although its page and its number of pages are all that is used
RESIZE += [(dict(cache=dict(k=None)), EINVAL), (dict(cache=dict(v=HERE + 8)), EINVAL), (dict(cache=dict(k_exp=None)), EINVAL), (dict(cache=dict(k_exp=None, v_exp=None, type=0)), 0),
           (dict(cache=dict(Hkv=8), shape=dict(Hkv=8, B=8191), add=16 * HERE), 0), (dict(cache=dict(Hkv=8), shape=dict(Hkv=8, B=8192), add=16 * HERE), ESHAPE), (dict(cache=dict(Hkv=1), shape=dict(Hkv=1, B=65535), add=16 * HERE), 0),
           (dict(shape=dict(dtype="f32")), 0), (dict(cache=dict(d=64)), ESHAPE)]


@pytest.mark.parametrize("change,want", RESIZE)
def test_refusals(lib, change, want):  # noqa: F811
    a = dict(cache={}, free=HERE, state=HERE, new_state=HERE, add=HERE, len=HERE + 4096, new_len=HERE + 4096, table=HERE, max_pages=4, starts=HERE, positions=HERE, slots=HERE)
    a.update({n: x for n, x in change.items() if n in a})
    s = _shape(**change.get("shape", {}))
    cache = None if a["cache"] is None else C.byref(_cache(**a["cache"]))
    assert lib.ls_debug_check_resize(C.byref(s), cache, *(a[n] for n in ("free", "state", "new_state", "add", "len", "new_len", "table", "max_pages", "starts", "positions", "slots"))) == want


def test_the_status_bit():
    assert binding.LS_STAT_PAGES_OUT == 256
