"""The gated layer's kernels and those of the rows in 8 bits keep what they keep in registers: none has scratch memory, whose loads would wait behind the requests and stores
that these kernels leave under way.  Read from this library's own build."""
import os
import subprocess

import pytest

from tests.test_handover import OBJDUMP, code_objects

pytestmark = pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")


@pytest.mark.parametrize("name,variants", [("7k_gatedI", 19), ("11k_gated_anyI", 10), ("11k_gated_fewI", 2), ("8k_store8I", 2), ("7k_load8I", 2), ("12k_norm8_gradI", 28), ("15k_norm8_dx_longI", 2), ("20k_norm8_dparams_longI", 2)])
def test_no_variant_has_scratch_memory(tmp_path, name, variants):
    found = {}
    for path in code_objects(tmp_path):
        for line in subprocess.run([OBJDUMP, "-t", path], check=True, capture_output=True, text=True).stdout.splitlines():
            if line.endswith(".private_seg_size") and name in line:
                found[line.split()[-1]] = int(line.split()[0], 16)
    assert len(found) == variants, sorted(found)
    assert not {symbol: size for symbol, size in found.items() if size}
