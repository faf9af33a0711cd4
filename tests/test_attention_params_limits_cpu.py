"""Host side, without a GPU, of what the calls for the global norm, rows, relative position bias and query/key norms
promise at their limits: which calls they refuse, and the rules that their kernels' sources keep."""
import os
import re

import pytest

from paper_2108_01624_b200 import binding as b
from paper_2108_01624_b200 import build as builder

ARG, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -6
OK, NO_DEVICE = 0, -4               # a call that was accepted: launched, or no device to launch on


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return b.lib()


def closing(text, at, pair):
    """Index behind the bracket that closes the one at text[at]."""
    depth = 0
    for i in range(at, len(text)):
        depth += (text[i] == pair[0]) - (text[i] == pair[1])
        if depth == 0:
            return i + 1
    raise AssertionError("unbalanced")


def kernels():
    """(file, name, parameters, body) of every kernel of the library, comments left out."""
    for f in sorted(os.listdir(builder.CSRC)):
        if not f.endswith((".cu", ".cuh")):
            continue
        text = re.sub(r"//[^\n]*", "", open(os.path.join(builder.CSRC, f)).read())
        for m in re.finditer(r"__global__\s+void\s+", text):
            at = m.end()
            if text.startswith("__launch_bounds__", at):
                at = closing(text, text.index("(", at), "()")
            name = re.compile(r"\s*(\w+)\s*\(").match(text, at)
            end = closing(text, name.end() - 1, "()")
            body = text.index("{", end)
            yield f, name.group(1), text[name.end():end - 1], text[body:closing(text, body, "{}")]


def test_kernels_that_start_early_promise_nothing_about_their_pointers():
    """A kernel launched with launch_chained starts while its predecessor still writes, so none of its pointers may be
    __restrict__ (for a const one that says the data do not change during the kernel; a load could then move before the wait),
    none of its loads non-coherent, and it waits before anything else."""
    found = list(kernels())
    chained = {name for f in os.listdir(builder.CSRC) if f.endswith(".cu")
               for call in re.findall(r"launch_chained\(([^,]*(?:<[^>]*>[^,]*)*),", open(os.path.join(builder.CSRC, f)).read())
               for name in re.findall(r"\bk_\w+", call)}
    waiting = {name for _, name, _, body in found if "wait_for_predecessor()" in body}
    assert len(found) > 20 and len(waiting) >= 9 and chained == waiting
    for f, name, params, body in found:
        if name in waiting:
            assert "__restrict__" not in params, (f, name)
            assert "__ldg" not in body and ".nc." not in body and "__restrict__" not in body, (f, name)
            before = body[1:body.index("wait_for_predecessor()")]
            assert all(re.match(r"(constexpr|(extern\s+)?__shared__)\b", s.strip()) for s in before.split(";") if s.strip()), (f, name)
