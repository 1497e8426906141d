"""Host-side facts that the ends of the calls on pages and packed sequences rest on (no GPU)."""
import ctypes as C
import os
import random
import subprocess
import sys
import textwrap

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


HERE = 1 << 20                                             # an address, 16-byte aligned, that nothing follows


@pytest.mark.parametrize("B,H,rows,starts,want", [
    (1, 128, 1 << 24, True, -2), (1, 128, (1 << 24) - 256, True, 0),          # blocks of 128 rows of all heads, and one for each sequence and head
    (128, 1, 1 << 24, False, -2), (128, 1, (1 << 24) - 128, False, 0), (4, 1, (1 << 29) - 512, False, 0), (4, 1, 1 << 29, False, -2)])
def test_more_blocks_than_a_launch_has_threads_for(lib, B, H, rows, starts, want):
    """A call whose grid would have 2^32 threads is refused: HIP would run what is left of them."""
    s = binding.make_shape(B, H, H, 64, 100, rows, 1, "bf16")
    many = binding.LsRows(HERE, 0 if starts else rows * H * 64, H * 64, 64)
    keys = binding.LsRows(HERE, 0 if starts else 100 * H * 64, H * 64, 64)
    at = HERE if starts else None
    assert lib.ls_debug_check_packed(C.byref(s), C.byref(many), C.byref(keys), C.byref(keys), at, at, C.byref(many), None) == want


def _python(code):
    return subprocess.run([sys.executable, "-c", textwrap.dedent(code)], cwd=os.path.dirname(build._DIR), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def test_the_calls_that_were_there_do_without_the_module_of_pages(lib):
    r = _python("""
        import sys
        from paper_2507_13681_amd import binding
        binding.load_library(), binding._load_native()
        assert "paper_2507_13681_amd._lspages" not in sys.modules
        sys.modules["paper_2507_13681_amd._lspages"] = None          # none that could be loaded
        binding._load_native()
        try:
            binding._load_pages()
        except binding.LoopServeError as e:
            assert "_lspages" in str(e)
        else:
            raise AssertionError
    """)
    assert r.returncode == 0, r.stdout


def test_another_pytorch_is_refused(lib):
    """The module reads tensors by what the headers said of them."""
    r = _python("""
        import torch
        from paper_2507_13681_amd import binding
        was = str(torch.__version__)
        torch.__version__ = "0.1"
        try:
            binding._load_pages()
        except binding.LoopServeError as e:
            assert was in str(e) and "0.1" in str(e), e
        else:
            raise AssertionError
        torch.__version__ = was
        assert binding._load_pages().packed_prefill
    """)
    assert r.returncode == 0, r.stdout
