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


def test_a_prefix_call_is_refused_before_its_first_launch():
    """Everything that can refuse the call (the tensor map of the widened prefix among it) stands before the kernel that
    the call launches first; behind it only a launch can fail."""
    with open(os.path.join(CSRC, "api.cu")) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    body = code[code.index("int32_t odma_decode_attention_prefix("):]
    body = body[:body.index("\n}\n")]
    launched = body[body.index("launch_"):]
    assert "ODMA_ERR_INVALID" not in launched and "make_tensor_map" not in launched
    assert "make_tensor_map" in body
