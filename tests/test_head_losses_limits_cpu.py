"""The vocabulary head's losses at the ends of their ranges, without a GPU: index arithmetic of the kernels at the largest sizes
that the calls take (which are not run), by their source and the limits of the calls."""
import os
import re

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
