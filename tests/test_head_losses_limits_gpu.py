"""The vocabulary head's losses at the ends of their ranges and between streams, on the GPU."""
import math

import pytest
import torch

import paper_2108_01624_b200 as dp
from paper_2108_01624_b200.synth import HEAD, LayerSpec

from .test_head_losses_gpu import BF16, DEV, F32, Case, check_distill, distill_case, workspace

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


def norm_errors(B, T, d, V, dtype, bias=True, seed=0):
    """Signed errors of the squared norms relative to the definition from the same lse, one per example."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(B, T, d, generator=g, device=DEV).to(dtype)
    w = (torch.randn(V, d, generator=g, device=DEV) * (2.0 / math.sqrt(d))).to(dtype)
    y = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
    b = torch.randn(V, generator=g, device=DEV) if bias else None
    head = dp.VocabHead(x, w, y, bias=b)
    ws, loss, lse, sq = workspace(head), torch.empty(B, T, device=DEV), torch.empty(B, T, device=DEV), torch.empty(B, device=DEV)
    dp.dp_vocab_loss(head, loss, lse, workspace=ws)
    dp.dp_vocab_loss_backward(head, lse, None, sq, workspace=ws)
    ref = torch.empty(B, dtype=torch.float64, device=DEV)
    for i in range(B):
        xd = x[i].double()
        G = (xd @ w.double().t() + (b.double() if bias else 0.0) - lse[i].double()[:, None]).exp()
        G[torch.arange(T, device=DEV), y[i].long()] -= 1.0
        ref[i] = (G.t() @ xd).pow(2).sum() + (G.sum(0).pow(2).sum() if bias else 0.0)
    return (sq.double() - ref) / ref


# What the tensor cores drop makes norms too small, so an example could add more than C: less than 2^-23 of what has been summed
# at each step of 16, and no sum is longer than 32 steps: 2 * 32 * 2^-23 of the squares, which are products of two such sums.
# Exponentials take 2 * 2^-20; G in two bf16 numbers 2 * 2^-17 for a token alone, to either side, less in the mean over examples
# and tokens (4 sigma of 100 single tokens: 2^-18).  Together 2^-16 of a squared norm in the mean, whatever the sizes.
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B, T, d, V", [(100, 1, 1024, 40), (100, 1, 65536, 40), (64, 20, 8192, 300), (64, 32, 768, 3000)])
def test_norms_of_short_examples_are_right_in_the_mean(B, T, d, V, dtype):
    r = norm_errors(B, T, d, V, dtype)
    assert abs(float(r.mean())) <= 2.0 ** -16, (float(r.mean()), float(r.min()), float(r.max()))


# Longer examples: rows of planes beyond 128 go through the layers' norm kernels, whose sums are of the same length here: Grams of
# both operands (their widths in parts), or the gradient itself (its rows in parts).
@pytest.mark.parametrize("B, T, d, V, dtype", [(32, 70, 768, 3000, BF16), (32, 33, 768, 3000, F32), (8, 512, 8192, 300, BF16), (3, 70, 65536, 40, F32),
                                               (8, 512, 96, 3000, BF16), (4, 5000, 64, 500, BF16), (4, 5000, 64, 500, F32), (2, 100000, 16, 40, BF16)])
def test_norms_of_long_examples_are_right_in_the_mean(B, T, d, V, dtype):
    r = norm_errors(B, T, d, V, dtype)
    assert abs(float(r.mean())) <= 2.0 ** -16, (float(r.mean()), float(r.min()), float(r.max()))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [300, 5003, 130001])
@pytest.mark.parametrize("tau", [1e-30, 1e-20, 1e-12, 1e-8, 1e-4, 1e6, 1e15])
def test_distillation_over_the_range_of_temperatures(tau, V, dtype):
    """Rows of every form: a warp's, shared memory's, those beyond.  Exponents of up to 10^31, losses from 10^-29 to 10^31."""
    z, ids, t, w = distill_case(2, 3, V, 6, dtype)
    check_distill(z, ids, t, tau, w, torch.full_like(z, float("nan")))


@pytest.mark.parametrize("V", [300, 6000, 130001])
def test_distilled_rows_beside_the_logits(V):
    """Logits and their gradient as columns of one buffer, and in every other row of one: no element in common."""
    z, ids, t, w = distill_case(2, 3, V, 7, BF16)
    wide = torch.full((2, 3, 2 * V), 5.0, dtype=BF16, device=DEV)
    wide[..., V:] = z
    check_distill(wide[..., V:], ids, t, 2.0, w, wide[..., :V])
    rows = torch.full((2, 6, V), 5.0, dtype=BF16, device=DEV)
    rows[:, ::2] = z
    check_distill(rows[:, ::2], ids, t, 2.0, w, rows[:, 1::2])
    assert torch.equal(rows[:, ::2].nan_to_num(), z.nan_to_num()) and torch.equal(wide[..., V:].nan_to_num(), z.nan_to_num())
    with pytest.raises(dp.binding.DpError):
        dp.dp_distill_loss(wide[..., V:], ids, t, 2.0, torch.empty(2, 3, device=DEV), wide[..., 1:V + 1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_gradient_from_the_losss_own_lse(dtype):
    """Chained through an fp32 lse, every exponential moves by what that is off, G at the label of a token that the model is sure of by
    as much in absolute terms: against the definition from the logits alone."""
    c = Case(4, 16, 256, 500, dtype, sure=6.0, dead=0.1, bias=False, weights=False)
    head = c.head()
    ws, loss, lse = workspace(head), torch.empty(4, 16, device=DEV), torch.empty(4, 16, device=DEV)
    dx, sq = torch.empty_like(c.x), torch.empty(4, device=DEV)
    acc_w = torch.zeros(500, 256, device=DEV)
    dp.dp_vocab_loss(head, loss, lse, workspace=ws)
    dp.dp_vocab_loss_backward(head, lse, dx, sq, workspace=ws)
    dp.dp_vocab_loss_clipped_accumulate(head, lse, torch.ones(4, device=DEV), acc_w, workspace=ws)
    p = (c.z - c.lse64[..., None]).exp()
    y = torch.zeros_like(p).scatter_(-1, c.labels.clamp(min=0).long()[..., None], 1.0)
    # 1 - p at the label as the sum of the others
    others = torch.where(y > 0, 0.0, p).sum(-1, keepdim=True)
    G = c.w[..., None] * torch.where(y > 0, -others, p)
    assert 0 < float(others[c.live].min()) < 1e-7
    moved = (c.dz.amax(-1) + 2.0 ** -20 + 2.0 ** -23 * c.lse64.abs()).expm1()[..., None]          # of the lse, as its own test bounds it
    dG = c.w[..., None] * p * (moved + torch.where(y > 0, 2.0 ** -20, c.dz.expm1() + 2.0 ** -20))
    w, x = c.weight.double(), c.xd.flatten(0, 1)
    r = 2 * 2.0 ** -16 if dtype == F32 else 2.0 ** -8
    ref = G @ w
    tol = dG @ w.abs() + (r + 2.0 ** -15) * ((G.abs() + dG) @ w.abs()) + (2.0 ** -24 if dtype == F32 else 2.0 ** -8) * ref.abs()
    assert bool(((dx.double() - ref).abs() <= 1.02 * tol + 1e-37).all())
    G, dG = G.flatten(0, 1), dG.flatten(0, 1)
    ref = G.t() @ x
    tol = dG.t() @ x.abs() + ((2 if dtype == F32 else 1) * 2.0 ** -16 + 2.0 ** -15) * ((G.abs() + dG).t() @ x.abs()) + 2.0 ** -23 * ref.abs()
    assert bool(((acc_w.double() - ref).abs() <= 1.02 * tol).all())


# Three blocks of G, two of which fill a piece of at most 1 GiB, the last piece one: dX, norms and sums over unequal pieces.  Short
# examples, and long ones by either kernel with their bias apart (bf16) or as a column (fp32); widths that are no multiple of 4 and 8.
@pytest.mark.parametrize("B, T, d, dtype, bias", [(2800, 9, 18, F32, True), (252, 100, 24, F32, True), (2500, 20, 20, BF16, False), (500, 100, 18, BF16, True),
                                                  (715, 70, 264, BF16, True)])
def test_unequal_pieces_of_the_vocabulary(B, T, d, dtype, bias):
    c = Case(B, T, d, 6000, dtype, bias=bias, dead=0.2)
    head = c.head()
    rows = (4 if dtype == F32 else 2) * B * T
    assert 2 <= (1 << 30) // (rows * 2048 * 2) < 3 and dp.dp_vocab_workspace_bytes(head) < 2 << 30
    c.check_backward(sq0=torch.rand(B, device=DEV))
    c.check_backward(out=torch.zeros(B, T, d + 3, dtype=dtype, device=DEV)[..., :d])
    c.check_sum()
    assert dp.dp_poll_status() == 0
