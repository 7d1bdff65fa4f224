"""Every role of the 8-bit float product waits for the kernels before it before its first bounded wait: the time limit of those waits is for
this kernel's own progress, and no kernel of the library lasts long enough to show the difference on a device."""
import os
import re

import paper_2111_09389_b200 as package

SOURCE = os.path.join(os.path.dirname(package.__file__), "csrc", "matmul_e4m3.cu")


def test_each_role_waits_for_the_kernels_before_it_first():
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    body = text[text.index("const uint32_t tmem_base ="):text.index("struct MmPlan")]
    before = text[text.index("__global__"):text.index("const uint32_t tmem_base =")]
    assert "mbar_wait(" not in before
    roles = re.split(r"\bif \(warp (?:== \d|>= \d)\) \{", body)[1:5]
    assert len(roles) == 4
    for n, role in enumerate(roles):
        waits = role.index("mbar_wait(")
        # warp 2 has waited in front of its first loads
        earlier = "pdl_wait()" in role[:waits] or (n == 2 and re.search(r"if \(warp == 2\) \{[^}]*pdl_wait\(\)", before))
        assert earlier, f"role {n} may start its time limit while other kernels run"
