"""Kernels that come up while the launch before them on the stream still runs (they wait for it on the device) must not tell the compiler that what
they read is constant for as long as they run: a `const __restrict__` parameter allows exactly that, and loads through the non-coherent path or in front
of the wait.  Checked on the source: what the compiler makes of it is not looked at."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_24270_b200", "csrc")


def functions(text):
    """(head, body) of every function whose head may name parameters, by counting braces."""
    for m in re.finditer(r"^(?:template[^\n]*\n)?(?:static )?__(?:global|device)__[^;{]*\{", text, re.M):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        yield m.group(0), text[m.end():i]


def without_comments(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


WAITS = re.compile(r"dep_wait\(\)|griddepcontrol\.wait")


def kernels_and_what_they_call(text):
    found = list(functions(text))
    waiting = [(head, body) for head, body in found if "__global__" in head and WAITS.search(body)]
    called = {w for _, body in waiting for w in re.findall(r"\b(\w+)\b", body)}
    for _ in range(4):                                  # and what those call
        for head, body in found:
            if "__device__" in head and called & set(re.findall(r"(\w+)\s*\(", head)):
                called |= set(re.findall(r"\b(\w+)\b", body))
    return [h for h, _ in waiting], [h for h, _ in found if "__device__" in h and called & set(re.findall(r"(\w+)\s*\(", h))]


@pytest.mark.parametrize("name", sorted(os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "*.cu"))))
def test_no_promise_of_constant_inputs(name):
    for heads in kernels_and_what_they_call(without_comments(os.path.join(CSRC, name))):
        for head in heads:
            assert "__restrict__" not in head, head


def test_the_check_sees_the_kernels():
    kernels, helpers = kernels_and_what_they_call(without_comments(os.path.join(CSRC, "kv4.cu")))
    assert len(kernels) == 10 and any("k_kv4_fork_copy" in h for h in kernels)
    assert any("copy_pages" in h for h in helpers) and any("copy16" in h for h in helpers)
    assert any("k_attn_combine" in h for h in kernels_and_what_they_call(without_comments(os.path.join(CSRC, "attention.cu")))[0])
