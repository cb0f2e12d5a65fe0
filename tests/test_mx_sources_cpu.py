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


def statement_end(text, i):
    """Behind the statement that begins at i: a block, a for / if / while and what it governs, or up to a semicolon."""
    while text[i].isspace():
        i += 1
    if text[i] == "{":
        depth = 0
        for j in range(i, len(text)):
            depth += (text[j] == "{") - (text[j] == "}")
            if depth == 0:
                return j + 1
    m = re.match(r"(for|if|while)\s*\(", text[i:])
    if not m:
        return text.index(";", i) + 1
    depth = 0
    for j in range(i + m.end() - 1, len(text)):
        depth += (text[j] == "(") - (text[j] == ")")
        if depth == 0:
            return statement_end(text, j + 1)


def test_both_of_a_pair_wait_for_the_last_arrivals_on_their_barriers():
    """The commits of the pair's MMAs arrive on barriers of both CTAs.  One that has seen them on its own barriers
    knows nothing of the other's: each waits for the last on every slot and for the one after all MMAs, or an
    arrival could come when its shared memory is another kernel's."""
    text = source("wq4_mx_gemm.cu")
    text = text[text.index("mx_gemm_pair_kernel"):text.index("launch_pair")]
    assert "tc::commit_pair(&empty[" in text and "tc::commit_pair(drain" in text
    while "if (rank == 0)" in text:                    # what is left is executed in both
        i = text.index("if (rank == 0)")
        text = text[:i] + text[statement_end(text, i):]
    assert "mbar_wait(drain, 0" in text
    assert re.search(r"mbar_wait\(&empty\[i % S\], \(i / S\) & 1", text)
