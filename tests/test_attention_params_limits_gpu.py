"""GPU: what the calls for rows and query/key norms promise at their limits, against 64 bits.  HALF is a single rounding's
part of a value."""
import math
from decimal import Decimal, localcontext

import pytest
import torch

from paper_2108_01624_b200 import binding as b

from .test_attention_params_gpu import BF16, DEV, F32, HALF, QK_REL, gen, randn, within

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


# ---- angles -------------------------------------------------------------------------------------------------------
TWO_PI = Decimal("6.28318530717958647692528676655900576839433879875021164194988918")


def exact_angles(pos, freq):
    """(cosine, sine) [positions, frequencies] of pos * freq, reduced by whole turns in 60 digits."""
    with localcontext() as ctx:
        ctx.prec = 60
        ang = [[float((Decimal(p) * Decimal(f)) % TWO_PI) for f in freq] for p in pos]
    ang = torch.tensor(ang, dtype=torch.float64, device=DEV)
    return ang.cos(), ang.sin()


# The angle: a whole number of 2^-32 turns (rounded down), plus the fraction of a turn's own rounding times up to 2^31
# positions, together below 1.6 * 2^-32.
TURN = 1.6 * 2 * math.pi * 2.0 ** -32
# fp32, relative to the value itself, so zeros stay sharp: the remainder from the nearest quarter turn in 24 bits moves a sine by
# at most 2^-24 of itself and a cosine by less; the function 2 ulp (4 * 2^-24), the norm's reciprocal root 2 ulp, and the two
# products that carry them.
FP32_REL = (1 + 4 + 4 + 2) * 2.0 ** -24 * 1.001
# bf16, of the pair's length: the angle in 24 bits (2^-26 of a turn, 9.4e-8), times pi in fp32 (1.2e-7, and 8.8e-8 of the constant),
# and the hardware's sine (2^-21.41) and cosine (2^-21.19): 3.0e-7 + hypot(3.6e-7, 4.2e-7) < 2^-20.
BF16_ABS = 2.0 ** -20


def hard_positions(freq):
    """Positions all over 32 bits, and those that lie near quarter turns of the first two frequencies."""
    g = torch.Generator().manual_seed(5)
    far = torch.randint(-(1 << 31), 1 << 31, (1500,), generator=g).tolist()
    near = torch.randint(-100000, 100000, (1500,), generator=g).tolist()
    quarter = [int(round(k * math.pi / 2 / freq[i])) for i in (0, 1) for k in range(-300, 300)]
    return far + near + quarter + [0, 1, -1, 355, -355, 710, 103993, 104348, 245850922, (1 << 31) - 1, -(1 << 31)]


# width, turned part, neighbouring pairs: single elements; vectors in fp32; vectors in both types
@pytest.mark.parametrize("dim,rot,inter", [(8, 2, False), (8, 8, False), (8, 8, True), (32, 32, False)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_angles_of_any_position(dtype, dim, rot, inter):
    freq = [1.0, 0.8315] if rot > 2 else [1.0]
    pos = hard_positions([1.0, 0.8315])
    cos, sin = exact_angles(pos, freq)
    inv_freq = torch.zeros(rot // 2, dtype=torch.float64)
    inv_freq[:len(freq)] = torch.tensor(freq, dtype=torch.float64)
    P, n = len(pos), len(freq)
    places = [(2 * j, 2 * j + 1) if inter else (j, j + rot // 2) for j in range(n)]
    positions = torch.tensor(pos, dtype=torch.int32, device=DEV).view(P, 1)
    # heads whose mean square is exactly 1 and whose turned pairs are (a, 0): the output is (a cos, a sin)
    a = 1.0 if rot == 2 else 2.0 if dim == 8 else 4.0
    head = torch.zeros(dim)
    for p, _ in places:
        head[p] = a
    if rot == 2:
        head[2:6] = torch.tensor([1.0, 1.0, 1.0, 2.0])
    assert float(head.square().mean()) == 1.0
    x = head.to(DEV, dtype).expand(P, 1, 1, dim).contiguous()
    out = torch.empty_like(x)
    b.dp_qknorm_rope(x, None, out, None, None, None, 0.0, inv_freq, positions, None, inter)
    # backward: with a head of ones the gain's rows are the gradient turned back, (cos, -sin) of a pair (1, 0)
    ones, dy, dx = torch.ones_like(x), torch.zeros_like(x), torch.empty_like(x)
    for p, _ in places:
        dy[..., p] = 1.0
    rows = torch.empty(P, dim, device=DEV)
    b.dp_qknorm_rope_backward(ones, None, dy, None, dx, None, None, None, rows, None, 0.0, inv_freq, positions, None, inter,
                              workspace=torch.empty(b.dp_qknorm_workspace_bytes(x, None), dtype=torch.uint8, device=DEV))
    out, rows = out.view(P, dim).double() / a, rows.double()
    absolute = TURN if dtype == F32 else TURN + BF16_ABS
    for j, (p, q) in enumerate(places):
        for got, ref, rounded in ((out[:, p], cos[:, j], True), (out[:, q], sin[:, j], True),
                                  (rows[:, p], cos[:, j], False), (rows[:, q], -sin[:, j], False)):
            rel = FP32_REL + (HALF[dtype] * 1.01 if rounded and dtype != F32 else 0.0)
            within(got, ref, ref.abs() * rel + absolute * (1 + rel), f"pair {j}")


# ---- layouts of outputs -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_outputs_in_any_nested_layout_and_none_that_overlaps(dtype):
    g = gen(2)
    H, Tq, Tk = 3, 40, 56
    table = randn(g, 32, H)
    want = torch.empty(H, Tq, Tk, dtype=dtype, device=DEV)
    b.dp_relpos_bias(table, want)
    for room, cut in ((torch.empty(Tq, H, Tk, dtype=dtype, device=DEV), lambda r: r.transpose(0, 1)),
                      (torch.empty(H, Tq + 3, Tk + 5, dtype=dtype, device=DEV), lambda r: r[:, 2:Tq + 2, 1:Tk + 1]),
                      (torch.empty(Tq, 2, H, Tk, dtype=dtype, device=DEV), lambda r: r[:, 1].transpose(0, 1))):
        room.fill_(9.0)
        out = cut(room)
        b.dp_relpos_bias(table, out)
        assert torch.equal(out, want)
        out.fill_(9.0)
        assert bool((room == 9).all())                                 # nothing beside it was written
    for bad in (torch.empty(1, Tq, Tk, dtype=dtype, device=DEV).expand(H, Tq, Tk),
                torch.empty(2 * Tq * Tk, dtype=dtype, device=DEV).as_strided((H, Tq, Tk), (Tq * Tk // 2, Tk, 1))):
        with pytest.raises(b.DpError):
            b.dp_relpos_bias(table, bad)
    B, T, n, D = 2, 9, 3, 64
    x, dy = randn(g, B, T, n, D, dtype=dtype), randn(g, B, T, n, D, dtype=dtype)
    freq, work = b.rope_frequencies(D), torch.empty(b.dp_qknorm_workspace_bytes(x, None), dtype=torch.uint8, device=DEV)
    want, dwant = torch.empty_like(x), torch.empty_like(x)

    def backward(dx, dout=dy):
        b.dp_qknorm_rope_backward(x, None, dout, None, dx, None, None, None, None, None, 1e-6, freq, workspace=work)
    b.dp_qknorm_rope(x, None, want, None, None, None, 1e-6, freq)
    backward(dwant)
    # another form of the kernel may serve a layout: both are within QK_REL of a pair's length (at most sqrt(D) = 8, a normed
    # head's) and a rounding of the definition, the backward pass within 2 QK_REL of r (|u| + |hat| mean |u hat|) <= r |u| (1 + 8)
    size = 8 * QK_REL
    r = x.double().square().mean(-1, keepdim=True).rsqrt()
    dsize = 2 * QK_REL * r * 2 ** 0.5 * float(dy.double().abs().max()) * 9
    for room, cut in ((torch.empty(B, n, T, D, dtype=dtype, device=DEV), lambda r: r.transpose(1, 2)),
                      (torch.empty(B, T, n, 3, D, dtype=dtype, device=DEV), lambda r: r[:, :, :, 1]),
                      (torch.empty(n, T, B, D + 1, dtype=dtype, device=DEV), lambda r: r.permute(2, 1, 0, 3)[..., 1:])):
        out = cut(room.fill_(9.0))
        b.dp_qknorm_rope(x, None, out, None, None, None, 1e-6, freq)
        within(out, want, 2.02 * (want.double().abs() * HALF[dtype] + size))
        backward(out)
        within(out, dwant, 2.02 * (dwant.double().abs() * HALF[dtype] + dsize))
        out.fill_(9.0)
        assert bool((room == 9).all())
    for dim in (0, 1, 2):
        bad = torch.empty_like(x).narrow(dim, 0, 1).expand_as(x)
        with pytest.raises(b.DpError):
            b.dp_qknorm_rope(x, None, bad, None, None, None, 1e-6, freq)
        with pytest.raises(b.DpError):
            backward(bad)
        backward(dwant, dy.narrow(dim, 0, 1).expand_as(dy))            # an input may be broadcast
