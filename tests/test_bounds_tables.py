"""The bounds-check build looks addresses up in a table that is one per source file, and lets everything pass where a file's own is empty: each file
of the state space language model's operators that launches a kernel fills its table."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1810_00952_b200", "csrc")
FILES = ("causal_conv.cu", "selective_scan.cu", "selective_scan_grad.cu", "linear_logprob.cu", "linear_logprob_tc.cu", "sequence.cu")


@pytest.mark.parametrize("name", FILES)
def test_files_that_launch_kernels_fill_their_table(name):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert "launch_pdl" in text
    assert re.search(r"\bBoundsReg \w+;|\bregister_buffers\(", text), name


def test_epilogues_of_the_head_check_their_accesses():
    """Each of their accesses to global memory that is not a TMA tile store stands under a check."""
    with open(os.path.join(CSRC, "linear_logprob_tc.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for member in ("part", "at", "lse", "dlogp"):
        for use in re.finditer(r"[^\n]*\bp\.%s\s*(?:\[|\+)[^\n]*" % member, text):
            assert "relay_in_bounds(" in use.group(0), use.group(0).strip()
