"""What the attention kernel's source has to keep to beside its results (no GPU needed)."""
import os
import re

from paper_2609_15030_gb300 import build


def test_register_shares_are_moved_by_whole_warpgroups():
    """setmaxnreg is an instruction of a warpgroup: its four warps have to execute the same one.  The last
    warpgroup's warps have different roles, so it stands in front of the branches on these."""
    with open(os.path.join(build.CSRC, "attn_tc.cuh")) as f:
        src = f.read()
    calls = re.findall(r"\b(fewer|more)_registers<", src)
    assert sorted(calls) == ["fewer", "more"]
    shares = re.search(r"\n    if \(warp >= C::kSoftmax\) \{\s+fewer_registers<C::kLessRegs>\(\);\n.*"
                       r"\n    \} else \{\n(?: +//[^\n]*\n)*        more_registers<C::kMoreRegs>\(\);", src, re.S)
    assert shares is not None
    # the roles lie inside the first branch
    assert "if (warp == C::kSoftmax + 3) {" in shares.group() and "warp < C::kSoftmax + NG" in shares.group()
