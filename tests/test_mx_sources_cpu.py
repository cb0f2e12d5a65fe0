"""How the kernels on rows of microscaled matrices read, from their source.

They start while the kernel before them may still be running, and what they read may
be what it writes.  Nothing in the language keeps a load that says that its memory is
constant (the read-only path, __ldg and its kin, or a const pointer without aliases,
which the compiler may turn into one) behind the wait for that kernel.
"""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_15803_gb300", "csrc")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def test_no_row_is_read_as_if_it_never_changed():
    text = source("wq4_mx.cu")
    assert "grid_dependency_wait" in text
    assert re.findall(r"__ld\w+\(|ld\.global\S*\.nc|__restrict__", text) == []
