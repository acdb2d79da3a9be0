"""Kernels whose workgroups hand data to each other inside a launch: the write-back of the L2 has to be done before the flag is raised
that tells other workgroups of the data.

A workgroup behind another L2 that sees the flag while the write-back is under way reads what memory held before.  Seldom enough for a test of
results to miss it; in the machine code of this library's own build it can be seen.
"""
import os
import re

import pytest

from tests.test_handover import LABEL, OBJDUMP, kernels

pytestmark = pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")


def unfinished(code):
    """(write-backs of the L2, those of them behind which something else than the wait for them comes first)."""
    total, bad = 0, 0
    for at, line in enumerate(code):
        if not line.startswith("buffer_wbl2"):
            continue
        total += 1
        for after in code[at + 1:]:
            if re.match(r"s_waitcnt .*vmcnt\(0\)", after):
                break
            if re.match(LABEL + "|s_cbranch|s_branch|s_endpgm|s_barrier|global_|buffer_|flat_|scratch_", after):
                bad += 1
                break
    return total, bad


def test_the_reader_tells_both_forms_apart():
    assert unfinished(["buffer_wbl2 sc1", "s_waitcnt vmcnt(0)", "global_atomic_add v0, v1, s[0:1]"]) == (1, 0)
    assert unfinished(["s_waitcnt vmcnt(0)", "buffer_wbl2 sc1", "global_atomic_add v0, v1, s[0:1]", "s_waitcnt vmcnt(0)"]) == (1, 1)
    assert unfinished(["buffer_wbl2 sc1", LABEL, "s_waitcnt vmcnt(0)"]) == (1, 1)


@pytest.mark.parametrize("name,variants", [("k_topk_group", 3), ("k_module_persist", 1)])
def test_the_write_back_is_done_before_the_flag_of_a_handover(tmp_path, name, variants):
    found = kernels(tmp_path, name)
    assert len(found) == variants
    for symbol, code in found.items():
        assert unfinished(code) == (1, 0), symbol


def test_no_other_kernel_writes_an_l2_back(tmp_path):
    """A kernel that begins to hand data over joins the list above."""
    found = kernels(tmp_path, "k_")
    assert len(found) > 50
    for symbol, code in found.items():
        if "k_topk_group" not in symbol and "k_module_persist" not in symbol:
            assert unfinished(code) == (0, 0), symbol
