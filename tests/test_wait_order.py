"""Bounded waits of the adapters' kernels start only when what they wait for no longer depends on the kernel in front, which may take
longer than such a wait does (about a second) before it gives up with AB_ERR_TIMEOUT.  Read from the source: a kernel in front that takes
as long is nothing to run in a test."""
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_01067_b200", "csrc", "ab_adapter_tc.cu")


def body(name):
    s = open(SRC).read()
    a = re.search(r"\n%s\(const __grid_constant__" % name, s).start()
    at = s.index("{\n", a)
    depth, i = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(s[i], 0)
        if depth == 0:
            return s[at:i]
        i += 1


def roles(text):
    """What the loader, the MMA warp and the others do."""
    a, b = text.index("  if (warp == 0) {"), text.index("  } else if (warp == 1) {")
    c = text.index("\n  } else {", b)
    return text[a:b], text[b:c], text[c:text.index("\n  }\n", c + 5)]


def test_every_role_of_the_wide_kernel_waits_for_the_kernel_in_front():
    loader, mma, rest = roles(body("wide_kernel"))
    for what in (loader, mma):          # the adapters' slabs are loaded from T, which the kernel in front writes
        assert "for_runs(" in what and 0 < what.find("dep_wait()") < what.index("for_runs(")
    assert 0 < rest.find("dep_wait()") < rest.index("mbar_wait")


def test_the_gradients_wait_before_anything_else():
    text = body("adapter_grad_tc_kernel")
    assert 0 < text.find("dep_wait()") < text.index("mbar_wait")


def test_the_kernel_for_few_rows_waits_before_its_accumulator_is_wanted():
    rest = roles(body("few_kernel"))[2]
    assert 0 < rest.find("dep_wait()") < rest.index("mbar_wait")
