"""What the order of a kernel's text decides, checked without a GPU."""
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2512_09427_b200", "csrc")
HOLDERS = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and "tcgen05.alloc" in open(os.path.join(CSRC, f)).read())


def test_some_kernels_hold_tensor_memory():
    assert {"decode_umma.cu", "prefix_umma.cu"} <= set(HOLDERS)


@pytest.mark.parametrize("name", HOLDERS)
def test_dependents_are_let_go_behind_the_allocation(name):
    """A dependent block that takes tensor memory holds it until the kernel ahead has ended.  So no block of that kernel may
    still have to allocate when the dependents are let go: they begin once every block has said so."""
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    alloc, go = code.index("tcgen05.alloc"), [m.start() for m in re.finditer(r"griddepcontrol\.launch_dependents", code)]
    assert go and alloc < min(go)
