"""What the compiler made of the kernels of pages and packed sequences: waits ahead of barriers, registers, no scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2507_13681_amd import build
from tests.test_transfer_waits import _transfers_at_barriers

# source: kernels with transfers (by the beginning of their names) and their instances
TRANSFERS = {"ls_paged.hip": [("paged_kernelI", 8)], "ls_packed.hip": [("packed_kernelI", 4)], "ls_cache.hip": []}
# bf16 instances of which a CU is to have so many waves on each of its SIMDs at once: 512 registers are shared by them
WAVES = {"ls_packed.hip": {"packed_kernelINS_6bf16_tELi128E": 3, "packed_kernelINS_6bf16_tELi64E": 4}}


@pytest.mark.parametrize("source", TRANSFERS)
def test_built_kernels(tmp_path, source):
    out = tmp_path / "source.s"
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)],
                   check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    text = out.read_text()
    code, current = {}, []
    for line in text.splitlines():
        start = re.match(r"(_ZN2ls\w+):", line)
        if start:
            code[start[1]] = current = []
        elif line.startswith(".Lfunc_end"):
            current = []
        else:
            current.append(line)
    seen = set()
    for name, instances in TRANSFERS[source]:
        found = {k: v for k, v in code.items() if re.match(rf"_ZN2ls\d+{name}", k)}
        assert len(found) == instances, (name, list(found))
        for k, lines in found.items():
            assert any("_load_lds_" in x for x in lines) and any("s_barrier" in x for x in lines), k
            assert not _transfers_at_barriers(lines), k
        seen |= set(found)
    assert not [k for k, lines in code.items() if k not in seen and any("_load_lds_" in x for x in lines)]
    told = {re.search(r"^\s*\.name:\s+(\S+)", k, flags=re.M)[1]: k for k in text.split("  - .agpr_count:")[1:]}
    field = lambda k, name: int(re.search(rf"^\s*\.{name}:\s+(\d+)", k, flags=re.M)[1])
    assert told
    for name, k in told.items():
        assert field(k, "private_segment_fixed_size") == 0, name
    for part, waves in WAVES.get(source, {}).items():
        instances = [field(k, "vgpr_count") for n, k in told.items() if part in n]
        assert instances and max(instances) <= 512 // waves // 8 * 8, (part, instances)
