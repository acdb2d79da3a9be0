"""What the kernels of the training operators keep, they keep in registers: none has scratch memory, whose loads would wait behind the requests and
stores that these kernels leave under way.  Read from this library's own build.
"""
import os
import subprocess

import pytest

from tests.test_handover import OBJDUMP, code_objects

pytestmark = pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")


@pytest.mark.parametrize("name,variants", [("9k_productI", 16), ("13k_product_anyI", 4), ("6k_joinI", 2), ("7k_embedI", 2), ("16k_embed_grad_fewI", 8), ("12k_sort_count", 1),
                                           ("12k_sort_place", 1), ("14k_embed_chunksI", 2), ("12k_embed_gradI", 8), ("14k_clip_squares", 1), ("12k_clip_scale", 1),
                                           ("6k_normI", 15), ("11k_norm_gradI", 15), ("11k_norm_join", 1), ("11k_norm_longI", 2), ("14k_norm_dx_longI", 2), ("19k_norm_dparams_longI", 2)])
def test_no_variant_has_scratch_memory(tmp_path, name, variants):
    found = {}
    for path in code_objects(tmp_path):
        for line in subprocess.run([OBJDUMP, "-t", path], check=True, capture_output=True, text=True).stdout.splitlines():
            if line.endswith(".private_seg_size") and name in line:
                found[line.split()[-1]] = int(line.split()[0], 16)
    assert len(found) == variants, sorted(found)
    assert not {symbol: size for symbol, size in found.items() if size}
