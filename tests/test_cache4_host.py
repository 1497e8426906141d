"""Pages of 4-bit floats: what the host refuses, and what the compiler made of their kernels (no GPU)."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2507_13681_amd import binding, build
from tests.test_serving_host import EINVAL, ESHAPE, HERE, _cache, _rows, _shape, lib  # noqa: F401

CACHES = [
    (dict(type=4), 0), (dict(type=4, d=64), ESHAPE), (dict(type=3), EINVAL), (dict(type=5), EINVAL), (dict(type=-1), EINVAL), (dict(type=4, k_exp=None), EINVAL),
    (dict(type=4, v_exp=None), EINVAL), (dict(type=4, k_exp=HERE + 8), EINVAL), (dict(type=4, k=HERE + 8), EINVAL), (dict(type=4, page=8), ESHAPE), (dict(type=4, pages=0), ESHAPE),
]


@pytest.mark.parametrize("cache,want", CACHES)
def test_refusals(lib, cache, want):  # noqa: F811
    s, c, r = _shape(), _cache(**cache), _rows(seq=51200)
    for write in (0, 1):
        assert lib.ls_debug_check_move(C.byref(s), C.byref(c), C.byref(r), C.byref(r), HERE, None, HERE, 4, None, write) == want
    assert lib.ls_debug_check_paged(C.byref(s), C.byref(c), HERE, HERE, 4, HERE, HERE, None) == want


def test_built_kernels(tmp_path):
    """Four instances without scratch memory, of which a compute unit can hold two workgroups of 16 query heads or fewer; rows come through registers, not by transfers."""
    out = tmp_path / "source.s"
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "ls_paged4.hip"), "-o", str(out)],
                   check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    text = out.read_text()
    assert "_load_lds_" not in text
    told = {re.search(r"^\s*\.name:\s+(\S+)", k, flags=re.M)[1]: k for k in text.split("  - .agpr_count:")[1:]}
    assert len(told) == 4 and all("paged_kernel" in n for n in told)
    field = lambda k, name: int(re.search(rf"^\s*\.{name}:\s+(\d+)", k, flags=re.M)[1])
    for name, k in told.items():
        assert field(k, "private_segment_fixed_size") == 0, name
        assert field(k, "vgpr_count") <= (128 if "ELi1ELi4E" in name else 256), name
