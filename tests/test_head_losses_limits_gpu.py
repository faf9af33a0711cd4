"""The vocabulary head's losses at the ends of their ranges and between streams, on the GPU."""
import math

import pytest
import torch

import paper_2108_01624_b200 as dp
from paper_2108_01624_b200.synth import HEAD, LayerSpec

from .test_head_losses_gpu import BF16, DEV, F32, Case, workspace

pytestmark = pytest.mark.gpu


def test_microbatches_of_changing_size_on_a_stream_of_the_callers():
    """Buffers that a larger or smaller microbatch replaces are not handed out while the stream that used them is behind."""
    sizes = [5, 9, 4, 12]
    cases = [Case(B, 6, 64, 700, F32, dead=0.0, seed=B) for B in sizes]
    heads = [c.head() for c in cases]

    def run(step, stream):
        kept = []
        for c, head in zip(cases, heads):
            step.head_backward(0, head, c.lse, None, stream=stream)
            step.accumulate_microbatch([], stream=stream)
            # what the current stream allocates and writes meanwhile
            kept += [torch.full((n,), 7.0, device=DEV) for n in sizes for _ in range(4)]
        return kept
    spec = [LayerSpec(HEAD, 700, 64, True, "mlm")]
    hyper = dict(C=0.7, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0)
    want, got = dp.DPStep(spec, DEV, **hyper), dp.DPStep(spec, DEV, **hyper)
    run(want, None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)                          # some 30 ms: everything below is enqueued behind it
    kept = run(got, side)
    torch.cuda.synchronize()
    assert torch.equal(want.acc, got.acc) and bool(want.acc.any())
    assert all(bool((t == 7.0).all()) for t in kept)
