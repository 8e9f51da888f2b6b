"""Properties of the paged kernels that only their generated code shows (compiled on the CPU, see test_generated_code.py)."""
import os
import re

import pytest

from paper_2509_21354_amd import build as kvev_build
from tests.test_generated_code import assembly, kernels, waits_before_ticket

pytestmark = pytest.mark.skipif(not os.path.exists(kvev_build.HIPCC), reason="needs hipcc")


def waited(lines):
    """The lines with a barrier put behind every wait for all vector memory operations."""
    return [x for s in lines for x in ([s, "s_barrier"] if s.startswith("s_waitcnt") and "vmcnt(0)" in s else [s])]


def test_partials_are_in_memory_before_the_ticket(tmp_path):
    """The workgroup that draws a unit's last ticket reads partials which others wrote: every storing wave waits for its stores
    before the barrier behind which the ticket is drawn."""
    found = {}
    for n, lines in kernels(assembly("page_attention.hip", tmp_path)).items():
        if "page_attention_kernel" in n:
            one_wave = re.search(r"I[ft]Li\d+ELi1E", n)                         # has no barrier: the wait stands for it
            found[n] = waits_before_ticket(waited(lines) if one_wave else lines)
    assert len(found) == 32 and all(ok is True for ok in found.values()), [n for n, ok in found.items() if ok is not True]


@pytest.mark.parametrize("name,kernel,most", [("page_attention.hip", "page_attention_kernelIt", 168), ("page_frame.hip", "page_frame_kernel", 256)])
def test_registers_are_not_spilt(name, kernel, most, tmp_path):
    """Three waves of page_attention_kernel on a SIMD (two with 32 queries), two of page_frame_kernel: spills within a chunk cost most of what the kernels
    gain (four waves of the first: 629 us against 367)."""
    asm = assembly(name, tmp_path)
    rows = [(n, int(v), int(s)) for n, v, s in re.findall(r"\.name:\s+(_Z\S+)(?:(?!\.name:)[\s\S])*?\.vgpr_count:\s+(\d+)\s+\.vgpr_spill_count:\s+(\d+)", asm)]
    rows = [r for r in rows if kernel in r[0]]
    assert len(rows) == (20 if kernel.startswith("page_att") else 3)
    most_of = {n: 256 if n.endswith("ELi2EEEvNS_12PageAttnArgsE") else most for n, _, _ in rows}
    assert all(v <= most_of[n] and s == 0 for n, v, s in rows if "Li8E" not in n or kernel.startswith("page_f")), rows
