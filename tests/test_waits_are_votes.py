"""A device-side wait that gives up takes the whole warp with it: in the product kernels every bounded wait is a vote of
the warp, since the code after it (shuffles, tensor-memory loads) needs all lanes."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_10537_b200", "csrc")


@pytest.mark.parametrize("name", ["mx_gemm.cu", "mx_gemm_grouped.cu"])
def test_every_wait_is_a_vote(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    waits = [s for s in re.split(r"[;{}]", text) if re.search(r"\bmbar_wait(_warp)?\(", s)]
    assert len(waits) >= 5
    lone = [" ".join(s.split()) for s in waits if re.search(r"\bmbar_wait\(", s) and "__all_sync(0xffffffffu," not in s]
    assert not lone, lone
