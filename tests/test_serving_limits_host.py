"""Host-side facts that the ends of the calls on pages and packed sequences rest on (no GPU)."""
import ctypes as C
import os
import random

import pytest

from paper_2507_13681_amd import binding, build


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.LIB):
        build.build_library()
    return binding.load_library()


def test_packed_calls_have_workgroups_without_an_item(lib):
    """However the rows are shared out among sequences, a KV head has fewer items than the call reckons with: who finds none sees all starts."""
    rng = random.Random(4)
    out, units = (C.c_int64 * 4)(), (C.c_int64 * 2)()
    for _ in range(300):
        Hkv, G, B = rng.choice([1, 2, 3, 8, 16]), rng.choice([1, 2, 4, 5, 128, 200]), rng.choice([1, 2, 65, 130, 300])
        B = min(B, 65535 // (Hkv * G))
        rows = [rng.choice([0, 1, 2, 127, 128, 129, rng.randint(0, 400)]) for _ in range(B)]
        spare = rng.choice([0, 0, 1, 300])                 # rows behind the last sequence
        s = binding.make_shape(B, Hkv * G, Hkv, 64, 1, max(1, sum(rows) + spare), 1, "bf16")
        assert lib.ls_debug_packed_units(C.byref(s), 1, units) == 0
        items = 0
        for r in rows:
            lib.ls_debug_packed_counts(r, r, G, 0, 0, out)
            items += out[0]
        assert units[1] % Hkv == 0 and items < units[1] // Hkv
