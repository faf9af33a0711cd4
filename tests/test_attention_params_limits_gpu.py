"""GPU: what the calls for rows and query/key norms promise at their limits, against 64 bits.  HALF is a single rounding's
part of a value."""
import pytest
import torch

from paper_2108_01624_b200 import binding as b

from .test_attention_params_gpu import DEV, F32, HALF, gen, randn, within

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)


# ---- rows ---------------------------------------------------------------------------------------------------------
# An example whose squared norm came out too small would be clipped too little, so the error must not grow with the width:
# the sum is formed in 64 bits and rounded once per launch (of up to 128 tensors), once more where it is added to.
@pytest.mark.parametrize("B,width", [(3, 1), (2, 1 << 20), (3, (1 << 24) + 5), (1, 1 << 28)])
def test_squared_norms_of_wide_rows_do_not_lose_with_the_width(B, width):
    if torch.cuda.mem_get_info()[0] < 16 * B * width + (1 << 30):
        pytest.skip("needs more free device memory")
    x = torch.empty(B, width, device=DEV)
    for i in range(B):
        x[i] = (0.1, 0.7, 1.0 / 3.0)[i]                                # equal values: every rounding of a run falls the same way
    sq = torch.full((B,), float("nan"), device=DEV)
    rows = b.RowList([(x, None)])
    b.dp_rows_sqnorms(rows, sq)
    ref = width * x[:, 0].double().square()
    within(sq, ref, ref * HALF[F32] * 1.0001)
    b.dp_rows_sqnorms(rows, sq, True)
    within(sq, 2 * ref, 2 * ref * 2 * HALF[F32] * 1.0001)


@pytest.mark.parametrize("widths", [[100003, 64, 7], [512] * 300])
def test_squared_norms_of_many_rows_are_rounded_once_per_launch(widths):
    g = gen(1)
    xs = [randn(g, 5, w) for w in widths]
    sq = torch.empty(5, device=DEV)
    b.dp_rows_sqnorms(b.RowList([(x, None) for x in xs]), sq)
    ref = sum(x.double().square().sum(1) for x in xs)
    within(sq, ref, ref * -(-len(widths) // 128) * HALF[F32] * 1.0001)
