"""The vocabulary head's losses at the ends of their ranges, without a GPU: index arithmetic of the kernels at the largest sizes
that the calls take (which are not run), by their source and the limits of the calls."""
import ctypes as C
import os
import re

import pytest

from paper_2108_01624_b200 import binding as b
from paper_2108_01624_b200 import build as builder

MOST_TOKENS, MOST_WORDS = 1 << 26, 1 << 26           # of a head; its calls refuse more
LIMIT = {"int": 2 ** 31 - 1, "unsigned": 2 ** 32 - 1, "long long": 2 ** 63 - 1}


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(builder.CSRC, name)).read())


def test_strides_over_a_grid_fit_their_counters():
    """for (type i = first of the block; i < end; i += blocks * step): a counter passes its end by one stride at most, which
    must not leave its type.  The largest grids have a block for every 8 tokens."""
    blocks = (MOST_TOKENS + 7) // 8
    loops = [m for f in ("dp_vocab.cu", "dp_vocab_cross.cu", "dp_distill.cu")
             for m in re.finditer(r"for \((long long|int|unsigned) (\w+) = [^;]*; [^;]*; \2 \+= (?:\(long long\))?gridDim\.x \* (\w+)\)", source(f))]
    assert len(loops) >= 2
    for m in loops:
        step = int(m[3]) if m[3].isdigit() else 1
        assert MOST_WORDS + MOST_TOKENS + blocks * step <= LIMIT[m[1]], m[0]


def test_the_cross_terms_tasks_fit_their_counter():
    """Up to 2^31 - 1 tasks of an example (more are refused), in steps of up to 64 blocks: the last step ends behind them."""
    text = source("dp_vocab_cross.cu")
    loops = re.findall(r"for \(([\w ]+) task = blockIdx\.x; task < a\.all; task \+= a\.chunks\)", text)
    assert len(loops) == 2 and "all > 0x7fffffffll" in text
    assert all(2 ** 31 - 1 + 64 <= LIMIT[t] for t in loops)


@pytest.mark.parametrize("N, ld, at, ld_out", [
    (6, 500, 2, 500), (6, 500, 998, 500), (6, 500, 500 * 10 + 998, 500), (6, 512, 1024 - 998, 512), (6, 512, -2, 512),   # a row ahead or behind
    (6, 1100, 1202, 1100), (6, 1100, 1200, 550), (1, 0, 998, 0), (1, 7000, -998, 9000), (6, 500, 0, 1000), (6, 1000, 2 * 500 * 5, 500)])
def test_distillation_refuses_rows_that_overlap_others(N, ld, at, ld_out):
    """Rows of 500 bf16 words; dlogits `at` bytes behind logits.  In place, or beside them, is allowed; in part over them is not."""
    builder.build()
    P = 1 << 20
    p = b.dp_distill(1, 0, N, 500, 8, 2.0, P, ld, P, P, P)
    assert b.lib().dp_distill_loss(C.byref(p), P, P + at, ld_out, None) == -1


def test_shared_arrays_that_are_copied_to_by_16_bytes_say_so():
    """cp.async writes 16 aligned bytes; bulk copies into swizzled tiles start where the kernel has aligned to 1024 bytes itself."""
    for f in ("dp_vocab.cu", "dp_vocab_cross.cu", "dp_distill.cu"):
        for align, name, after in re.findall(r"extern __shared__ (.*?)uint8_t (\w+)\[\];(.{600})", source(f), re.S):
            assert "__align__(16)" in align or f"({name}) + 1023) & ~uintptr_t(1023)" in after, (f, name)


@pytest.mark.parametrize("at, ld", [(0, 64), (0, 80), (64, 64), (-2, 64), (30 * 128, 64), (126, 128)])
def test_the_states_gradient_may_not_lie_over_them(at, ld):
    """The clipped sum reads the states again.  31 rows of 64 bf16 numbers, dX `at` bytes behind X."""
    builder.build()
    P = 1 << 20
    h = b.dp_vocab_head(1, 31, 1, 64, 1000, P, 64, P, 64, None, P, None)
    assert b.lib().dp_vocab_loss_backward(C.byref(h), P, P + at, ld, P, 0, P, 1 << 40, None) == -1
