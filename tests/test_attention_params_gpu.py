"""GPU parity, in 64 bits, of the global norm and clip, the clipped AdamW step, per-example rows, the relative position
bias with its per-example gradient, and the rotated query/key norms with their backward pass.

Tolerances.  A single rounding of an output is eps / 2 of its value (HALF below).  A sum of n fp32 terms formed by a
tree of depth d after runs of length m is off by at most (m + d) eps/2 of the sum of the terms' magnitudes; the tests use
that bound with the kernels' run lengths rounded up, on the sum of magnitudes computed beside the sum itself.
"""
import math

import pytest
import torch

from paper_2108_01624_b200 import binding as b

from .test_attention_params_cpu import whole_number_starts

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def within(got, ref, bound, what=""):
    """|got - ref| <= bound, element by element; bound may be a tensor."""
    err = (got.double() - ref.double()).abs()
    bound = torch.as_tensor(bound, dtype=torch.float64, device=err.device)
    assert bool((err <= bound).all()), f"{what}: off by {float((err - bound).max()):.3e} more than allowed"


# ---- global norm and clip -----------------------------------------------------------------------------------------
def norm_workspace():
    return torch.empty(b.dp_global_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)


def sqnorm_of(tensors, accumulate_into=False, start=None):
    out = torch.full((1,), float("nan"), dtype=torch.float64, device=DEV) if start is None else start
    return b.dp_global_sqnorm(tensors, out, accumulate_into, norm_workspace())


# 32 squares in a fp32 run, then fp64: relative to a sum of squares (all terms positive)
SQ_REL = 34 * 2.0 ** -24


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", [[1], [7], [4096], [1, 0, 3, 17, 100003], [4160], [1 << 20, 5, 1 << 14, 8193], [3] * 130,
                                   [11] * 1500, [70000] * 40])
def test_global_norm_and_clip(dtype, sizes):
    g = gen(1)
    ts = [randn(g, n, dtype=dtype) * 0.5 for n in sizes]
    ref = sum(float(t.double().square().sum()) for t in ts)
    sq = sqnorm_of(ts)
    assert float(sq) == pytest.approx(ref, rel=SQ_REL)
    assert float(sqnorm_of(ts)) == float(sq)                          # bit for bit
    sqnorm_of(ts, True, sq)
    assert float(sq) == pytest.approx(2 * ref, rel=SQ_REL)
    for max_norm in (0.25 * math.sqrt(ref), 4 * math.sqrt(ref)):
        sq = sqnorm_of(ts)
        f = min(1.0, max_norm / math.sqrt(ref))
        outs = [torch.full_like(t, float("nan")) for t in ts]
        told = torch.empty(2, device=DEV)
        b.dp_clip_by_global_norm(ts, outs, sq, max_norm, told)
        # the factor carries the sum's error halved by the root, and one rounding; the product one more
        for t, o in zip(ts, outs):
            ref_o = t.double() * f
            within(o, ref_o, ref_o.abs() * (SQ_REL + 2 * HALF[F32] + HALF[dtype]))
        assert float(told[0]) == pytest.approx(math.sqrt(ref), rel=SQ_REL + HALF[F32])
        assert float(told[1]) == pytest.approx(f, rel=SQ_REL + HALF[F32])
        same = [t.clone() for t in ts]
        b.dp_clip_by_global_norm(same, None, sq, max_norm)             # in place
        assert all(torch.equal(s, o) for s, o in zip(same, outs))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift_in,shift_out", [(0, 1), (1, 0), (3, 3), (5, 2)])
def test_global_clip_of_unaligned_views(dtype, shift_in, shift_out):
    g = gen(2)
    n = 30011
    big, room = randn(g, n + 16, dtype=dtype), torch.full((n + 16,), 7.0, dtype=dtype, device=DEV)
    x, o = big[shift_in:shift_in + n], room[shift_out:shift_out + n]
    ref = float(x.double().square().sum())
    sq = sqnorm_of([x])
    assert float(sq) == pytest.approx(ref, rel=SQ_REL)
    b.dp_clip_by_global_norm([x], [o], sq, 1.0)
    want = x.double() / math.sqrt(ref)
    within(o, want, want.abs() * (SQ_REL + 2 * HALF[F32] + HALF[dtype]))
    assert bool((room[:shift_out] == 7).all()) and bool((room[shift_out + n:] == 7).all())


def test_global_norm_beyond_the_range_of_fp32_squares():
    for scale in (1e25, 1e-25, 3e38, 1e-38):
        t = torch.full((1000,), scale, device=DEV)
        t[::2] = 0.0
        x = float(t[1].double())
        assert float(sqnorm_of([t])) == pytest.approx(500 * x * x, rel=1e-12)
        out = torch.empty_like(t)
        sq = sqnorm_of([t])
        b.dp_clip_by_global_norm([t], [out], sq, 2e-38)
        f = min(1.0, 2e-38 / (math.sqrt(500) * x))
        if f > 1e-37:                                                  # the factor itself is an fp32 number
            within(out, t.double() * f, (t.double() * f).abs() * 4 * HALF[F32] + 2.0 ** -149)


def test_global_norm_special_values():
    zero = [torch.zeros(5000, device=DEV), torch.zeros(0, device=DEV)]
    sq, told = sqnorm_of(zero), torch.empty(2, device=DEV)
    out = [torch.full((5000,), 3.0, device=DEV), torch.empty(0, device=DEV)]
    b.dp_clip_by_global_norm(zero, out, sq, 1.0, told)
    assert float(sq) == 0.0 and told.tolist() == [0.0, 1.0] and float(out[0].abs().max()) == 0.0
    empty = torch.full((1,), float("nan"), dtype=torch.float64, device=DEV)
    assert float(b.dp_global_sqnorm([], empty, False, norm_workspace())) == 0.0
    for bad, factor in ((float("inf"), 0.0), (float("nan"), float("nan"))):
        t = torch.ones(100, device=DEV)
        t[37] = bad
        sq, out = sqnorm_of([t]), torch.empty_like(t)
        b.dp_clip_by_global_norm([t], [out], sq, 1.0, told)
        assert str(float(told[1])) == str(factor)
        assert str(float(out[0])) == str(factor) and math.isnan(float(out[37]))


@pytest.mark.parametrize("n,shift", [(1, 0), (4, 0), (4160, 0), (100003, 0), (5000, 1)])
@pytest.mark.parametrize("zero_g", [False, True])
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
def test_clipped_adamw_step(n, shift, zero_g, max_norm):
    g0 = gen(3)
    flat = [randn(g0, n + shift)[shift:] for _ in range(4)]
    th, m, v, g = flat[0] * 0.02, flat[1] * 1e-3, flat[2].square() * 1e-4 + 1e-8, flat[3].contiguous()
    th, m, v = th.contiguous(), m.contiguous(), v.contiguous()
    hp = dict(lr=1e-2, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.1, t=7)
    sq = sqnorm_of([g])
    f = min(1.0, max_norm / math.sqrt(float(g.double().square().sum())))
    gd = g.double() * f
    rm = 0.9 * m.double() + 0.1 * gd
    rv = 0.999 * v.double() + 0.001 * gd ** 2
    up = (rm / (1 - 0.9 ** 7)) / ((rv / (1 - 0.999 ** 7)).sqrt() + 1e-11)
    rt = th.double() - 1e-2 * (up + 0.1 * th.double())
    keep = g.clone()
    # the plain call on the clipped gradient, for comparison
    t2, m2, v2 = th.clone(), m.clone(), v.clone()
    scaled = torch.empty_like(g)
    b.dp_clip_by_global_norm([g], [scaled], sq, max_norm)
    b.dp_adamw_step(t2, m2, v2, scaled, *(hp[k] for k in ("lr", "beta1", "beta2", "xi", "weight_decay", "t")))
    b.dp_clip_adamw_step(th, m, v, g, zero_g, sq, max_norm, *(hp[k] for k in ("lr", "beta1", "beta2", "xi", "weight_decay", "t")))
    mag_m = 0.9 * m2.double().abs() + gd.abs()
    within(m, rm, (rm.abs() + mag_m) * 8 * HALF[F32], "m")             # two products, a sum, the factor
    within(v, rv, rv * (2 * SQ_REL + 8 * HALF[F32]), "v")
    # quotient and root are hardware approximations, each within 2^-22; m's own error moves the quotient by its share
    share = (mag_m * 8 * HALF[F32]) / (1 - 0.9 ** 7) / ((rv / (1 - 0.999 ** 7)).sqrt() + 1e-11)
    within(th, rt, 1e-2 * (up.abs() * 2.0 ** -20 + share) + 4 * HALF[F32] * (rt.abs() + 1e-2 * up.abs()) + 2.0 ** -40, "theta")
    # the plain call on the written-out clipped gradient meets the same bounds (its last bits may differ: the compiler
    # chooses per kernel which product of a sum of two it keeps unrounded)
    within(m2, rm, (rm.abs() + mag_m) * 8 * HALF[F32], "m")
    within(v2, rv, rv * (2 * SQ_REL + 8 * HALF[F32]), "v")
    within(t2, rt, 1e-2 * (up.abs() * 2.0 ** -20 + share) + 4 * HALF[F32] * (rt.abs() + 1e-2 * up.abs()) + 2.0 ** -40, "theta")
    assert torch.equal(g, torch.zeros_like(g) if zero_g else keep)


# ---- rows ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,widths", [(1, [1]), (5, [33]), (256, [512, 64, 64, 3]), (3, [100003]), (37, [64] * 150), (1000, [31])])
def test_rows_norms_and_clipped_sum(B, widths):
    g = gen(4)
    pairs = [(randn(g, B, w) * 10.0 ** randn(g, B, 1).clamp(-1, 1), randn(g, w)) for w in widths]
    start = [a.double().clone() for _, a in pairs]
    rows = b.RowList(pairs)
    sq = torch.full((B,), float("nan"), device=DEV)
    b.dp_rows_sqnorms(rows, sq)
    ref = sum(x.double().square().sum(1) for x, _ in pairs)
    runs = sum(-(-w // 256) for w in widths) + 16 + -(-len(widths) // 128)
    within(sq, ref, ref * runs * HALF[F32] * 1.01)
    once = sq.clone()
    b.dp_rows_sqnorms(rows, sq, True)
    within(sq, 2 * once.double(), 2 * ref * 2 * HALF[F32] * 1.01 * (1 + -(-len(widths) // 128)))
    clip = torch.rand(B, generator=g, device=DEV)
    b.dp_rows_clipped_accumulate(rows, clip)
    for (x, a), s in zip(pairs, start):
        terms = x.double() * clip.double()[:, None]
        mag = terms.abs().sum(0) + s.abs()
        within(a, s + terms.sum(0), mag * (-(-B // 16) + 18) * HALF[F32])


# ---- relative position bias ---------------------------------------------------------------------------------------
def bucket_map(nb, distance, both, Tq, Tk, offset):
    half = nb // 2 if both else nb
    starts = torch.tensor(whole_number_starts(nb, distance, both))
    rel = torch.arange(Tk)[None, :] - (torch.arange(Tq) + offset)[:, None]
    n = rel.abs() if both else (-rel).clamp(min=0)
    bucket = torch.searchsorted(starts, n, right=True) - 1
    return (bucket + half * (rel > 0) if both else bucket).to(DEV), rel.to(DEV)


BIAS_CASES = [
    # heads, Tq, Tk, buckets, distance, both sides, offset
    (16, 128, 128, 32, 128, True, 0), (3, 1, 1, 32, 128, True, 0), (2, 1, 513, 32, 128, False, 512),
    (5, 17, 129, 16, 20, True, -7), (4, 257, 255, 8, 64, False, 0), (1, 300, 520, 64, 1000, True, 100),
    (2, 130, 1024, 4, 3, True, 5000), (2, 40, 64, 256, 129, True, 0), (1, 1100, 24, 2, 2, False, 0),
    (7, 64, 2056, 32, 9, True, 13)]


@pytest.mark.parametrize("table_dtype", [F32, BF16])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("case", BIAS_CASES)
def test_relpos_bias_is_the_table_rounded_once(case, out_dtype, table_dtype):
    H, Tq, Tk, nb, distance, both, offset = case
    table = randn(gen(5), nb, H, dtype=table_dtype)
    bucket, _ = bucket_map(nb, distance, both, Tq, Tk, offset)
    want = table.float().to(out_dtype)[bucket].permute(2, 0, 1)
    out = torch.full((H, Tq, Tk), float("nan"), dtype=out_dtype, device=DEV)
    b.dp_relpos_bias(table, out, distance, both, offset)
    assert torch.equal(out, want)
    # rows with a gap behind them, which stays as it was
    room = torch.full((H, Tq, Tk + 8), 9.0, dtype=out_dtype, device=DEV)
    b.dp_relpos_bias(table, room[:, :, :Tk], distance, both, offset)
    assert torch.equal(room[:, :, :Tk], want) and bool((room[:, :, Tk:] == 9).all())


def relpos_rows(G, nb, distance, both, offset, causal, q_len, k_len):
    """(sums, sums of magnitudes) [B, nb, H] in 64 bits."""
    B, H, Tq, Tk = G.shape
    bucket, rel = bucket_map(nb, distance, both, Tq, Tk, offset)
    keep = torch.ones(B, 1, Tq, Tk, dtype=torch.bool, device=DEV)
    if causal:
        keep &= rel <= 0
    if q_len is not None:
        keep &= torch.arange(Tq, device=DEV)[None, None, :, None] < q_len[:, None, None, None]
    if k_len is not None:
        keep &= torch.arange(Tk, device=DEV)[None, None, None, :] < k_len[:, None, None, None]
    x = torch.where(keep, G.double(), 0.0).reshape(B, H, -1)
    out = []
    for y in (x, x.abs()):
        r = torch.zeros(B, H, nb, dtype=torch.float64, device=DEV)
        r.index_add_(2, bucket.reshape(-1), y)
        out.append(r.transpose(1, 2))
    return out


GRAD_CASES = [
    # B, heads, Tq, Tk, buckets, distance, both sides, offset
    (4, 16, 128, 128, 32, 128, True, 0), (2, 3, 1, 1, 32, 128, True, 0), (3, 2, 1, 513, 32, 128, False, 512),
    (2, 5, 17, 129, 16, 20, True, -7), (1, 4, 257, 254, 8, 64, False, 0), (2, 1, 300, 520, 64, 1000, True, 100),
    (1, 2, 130, 1024, 4, 3, True, 5000), (2, 2, 40, 64, 256, 129, True, 0), (1, 1, 1100, 24, 2, 2, False, 0),
    (2, 2, 520, 776, 32, 128, True, 256), (300, 9, 8, 8, 32, 128, True, 0), (3, 1, 33, 300, 32, 128, True, -300),
    (1, 1, 2000, 40, 32, 128, False, -1000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("case", GRAD_CASES)
def test_relpos_bias_grad_per_example(case, ragged, causal, dtype):
    B, H, Tq, Tk, nb, distance, both, offset = case
    g = gen(6)
    G = randn(g, B, H, Tq, Tk, dtype=dtype)
    q_len = k_len = None
    if ragged:
        q_len = torch.randint(-1, Tq + 3, (B,), generator=g, device=DEV, dtype=torch.int32)      # 0 and too long among them
        k_len = torch.randint(0, Tk + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        q_len[0], k_len[0] = (0, Tk) if B > 1 else (Tq, Tk)
    ref, mag = relpos_rows(G, nb, distance, both, offset, causal, q_len, k_len)
    if causal or ragged:                                               # what does not count may hold anything
        _, rel = bucket_map(nb, distance, both, Tq, Tk, offset)
        away = torch.zeros(B, 1, Tq, Tk, dtype=torch.bool, device=DEV)
        if causal:
            away |= rel > 0
        if ragged:
            away |= torch.arange(Tq, device=DEV)[None, None, :, None] >= q_len[:, None, None, None]
            away |= torch.arange(Tk, device=DEV)[None, None, None, :] >= k_len[:, None, None, None]
        bad = torch.tensor([float("nan"), float("inf"), torch.finfo(dtype).min], device=DEV).to(dtype)
        fill = bad[torch.randint(0, 3, (B, 1, Tq, Tk), generator=g, device=DEV)].expand_as(G)
        G = torch.where(away, fill, G)
    work = torch.empty(b.dp_relpos_workspace_bytes(G, nb), dtype=torch.uint8, device=DEV)
    rows = torch.full((B, nb, H), float("nan"), device=DEV)
    args = (distance, both, offset, causal, q_len, k_len)
    b.dp_relpos_bias_grad(G, rows, *args, workspace=work)
    # along a diagonal, then over a bucket's diagonals shared by the lanes, then over units: no term meets more adds
    # than the two sides and the units of its head together
    adds = min(Tq, 512) + (Tq + Tk) // 4 + 5 + (-(-Tq // 32)) * (-(-Tk // 32)) + 1
    within(rows, ref, mag * adds * HALF[F32])
    again = torch.empty_like(rows)
    b.dp_relpos_bias_grad(G, again, *args, workspace=work)
    assert torch.equal(rows, again)
    b.dp_relpos_bias_grad(G, again, *args, accumulate_into=True, workspace=work)      # a further layer
    within(again, 2 * rows.double(), 2 * rows.double().abs() * HALF[F32] * 1.01)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_relpos_bias_grad_of_strided_and_broadcast_scores(dtype):
    g = gen(7)
    B, H, Tq, Tk, nb = 3, 2, 40, 48, 32
    wide = randn(g, B, Tq, H, Tk + 5, dtype=dtype)
    for G in (wide[..., :Tk].transpose(1, 2),                          # rows apart, heads behind queries, odd strides
              wide[..., 3:3 + Tk].transpose(1, 2),                     # not 16-byte aligned
              randn(g, 1, H, Tq, Tk, dtype=dtype).expand(B, H, Tq, Tk),
              randn(g, B, 1, Tq, Tk, dtype=dtype).expand(B, H, Tq, Tk)):
        ref, mag = relpos_rows(G, nb, 128, True, 0, False, None, None)
        rows = torch.empty(B, nb, H, device=DEV)
        work = torch.empty(b.dp_relpos_workspace_bytes(G, nb), dtype=torch.uint8, device=DEV)
        b.dp_relpos_bias_grad(G, rows, 128, True, workspace=work)
        within(rows, ref, mag * 120 * HALF[F32])


def test_relpos_gradient_against_differences_of_the_bias():
    """<G, bias> is linear in the table: its change along any direction is <rows summed over examples, direction>."""
    g = gen(8)
    B, H, Tq, Tk, nb = 2, 4, 50, 70, 32
    G = randn(g, B, H, Tq, Tk)
    rows = torch.empty(B, nb, H, device=DEV)
    work = torch.empty(b.dp_relpos_workspace_bytes(G, nb), dtype=torch.uint8, device=DEV)
    b.dp_relpos_bias_grad(G, rows, 60, True, 3, workspace=work)
    for seed in range(3):
        table, step = randn(gen(20 + seed), nb, H), randn(gen(30 + seed), nb, H)
        lo, hi = torch.empty(H, Tq, Tk, device=DEV), torch.empty(H, Tq, Tk, device=DEV)
        b.dp_relpos_bias(table - step, lo, 60, True, 3)
        b.dp_relpos_bias(table + step, hi, 60, True, 3)
        diff = (G.double() * (hi.double() - lo.double())).sum((1, 2, 3)) / 2
        want = (rows.double() * step.double()).sum((1, 2))
        # the tables' sums are rounded to fp32 (|table| + |step| <= 12), the rows by their adds
        slack = G.double().abs().sum((1, 2, 3)) * 12 * 2 * HALF[F32] + rows.double().abs().sum((1, 2)) * 200 * HALF[F32] * 12
        within(diff, want, slack)


# ---- query/key norms with rotation --------------------------------------------------------------------------------
def pair_places(rot, interleaved):
    p = torch.arange(rot, device=DEV)
    return (p.view(-1, 2) if interleaved else p.view(2, -1).t()) if rot else p.view(0, 2)


def rotate64(x, pos, inv_freq, interleaved, sign=1.0):
    places = pair_places(2 * inv_freq.numel(), interleaved)
    ang = sign * pos.double()[..., None, None] * inv_freq.to(DEV)
    a, c = x[..., places[:, 0]], x[..., places[:, 1]]
    y = x.clone()
    y[..., places[:, 0]] = a * ang.cos() - c * ang.sin()
    y[..., places[:, 1]] = c * ang.cos() + a * ang.sin()
    return y


QK_CASES = [
    # B, T, query heads, key heads, dim, rot, interleaved, first position, layout
    (2, 5, 4, 2, 64, 64, False, 0, "fused"), (3, 1, 32, 8, 128, 128, False, 100000, "fused"),
    (2, 9, 3, 1, 80, 32, True, 7, "heads first"), (1, 33, 2, 2, 128, 64, False, 0, "plain"),
    (2, 3, 1, 1, 6, 4, False, 5, "plain"), (1, 4, 2, 1, 2, 2, True, 1, "plain"), (2, 7, 3, 3, 50, 24, True, 0, "fused"),
    (1, 3, 2, 1, 512, 512, False, 1 << 30, "plain"), (1, 2, 5, 2, 510, 100, False, 0, "plain"),
    (2, 6, 9, 0, 256, 256, True, -20, "plain"), (2, 6, 0, 3, 96, 0, False, 0, "plain"), (1, 600, 1, 1, 16, 16, False, 0, "plain"),
    (1, 40, 20, 4, 192, 96, False, 3, "shifted"), (4, 130, 12, 12, 64, 64, True, 0, "fused")]


def qk_inputs(case, dtype, seed):
    B, T, hq, hk, D, rot, inter, first, layout = case
    g = gen(seed)

    def heads(n):
        if n == 0:
            return None
        if layout == "heads first":
            return randn(g, B, n, T, D, dtype=dtype).transpose(1, 2)
        if layout == "shifted":                                        # heads that start off the 16-byte grid
            return randn(g, B, T, n, D + 1, dtype=dtype)[..., 1:]
        return randn(g, B, T, n, D, dtype=dtype)

    if layout == "fused":
        x = randn(g, B, T, (hq + 2 * hk) * D, dtype=dtype)
        q, k = x[..., :hq * D].unflatten(-1, (hq, D)), x[..., hq * D:(hq + hk) * D].unflatten(-1, (hk, D))
    else:
        q, k = heads(hq), heads(hk)
    pos = (torch.arange(T, dtype=torch.int32, device=DEV) + first).expand(B, T).contiguous()
    pos[B - 1] += 3 if first < (1 << 30) else 0
    return q, k, 1 + 0.3 * randn(g, D), 1 + 0.3 * randn(g, D), pos, b.rope_frequencies(rot) if rot else None


NONE = torch.zeros(0, dtype=torch.float64)
# angle: 2^-32 of a turn, then rounded to fp32 (2 pi 2^-25), sine and cosine within 2 ulp; norm: a fp32 sum of dim
# squares in runs of 16 with a tree of 5, a reciprocal root within 2 ulp; three products and a sum.  Relative to the
# pair's length, which bounds either element.
QK_REL = (2 * math.pi + 4 + 21 / 2 + 4 + 6) * 2.0 ** -24 * 1.5


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", QK_CASES)
def test_qknorm_rope(case, dtype):
    B, T, hq, hk, D, rot, inter, first, layout = case
    eps = 1e-6
    q, k, gq, gk, pos, freq = qk_inputs(case, dtype, 9)
    outs = [None if x is None else torch.full(x.shape, float("nan"), dtype=dtype, device=DEV) for x in (q, k)]
    b.dp_qknorm_rope(q, k, outs[0], outs[1], gq, gk, eps, freq, pos, None, inter)
    for x, gain, out in ((q, gq, outs[0]), (k, gk, outs[1])):
        if x is None:
            continue
        xd = x.double()
        y = xd * (xd.square().mean(-1, keepdim=True) + eps).rsqrt() * gain.double()
        ref = rotate64(y, pos, NONE if freq is None else freq, inter)
        length = rotate64(y, pos * 0, NONE if freq is None else freq, inter).abs()
        places = pair_places(rot, inter)
        both = torch.linalg.vector_norm(torch.stack([y[..., places[:, 0]], y[..., places[:, 1]]]), dim=0)
        length[..., places[:, 0]], length[..., places[:, 1]] = both, both
        within(out, ref, length * QK_REL + ref.abs() * HALF[dtype] * 1.001 + (length * QK_REL * HALF[dtype]))
        # in place, where the layout has its own memory
        y2 = x.clone() if layout != "fused" else None
        if y2 is not None and dtype == BF16 and y2.stride() == x.stride():
            args = (y2, None, y2, None, gain, None) if x is q else (None, y2, None, y2, None, gain)
            b.dp_qknorm_rope(*args, eps, freq, pos, None, inter)
            assert torch.equal(y2, out)


def test_qknorm_without_gain_positions_or_rotation():
    x = randn(gen(10), 2, 6, 3, 64)
    out, out2 = torch.empty_like(x), torch.empty_like(x)
    freq = b.rope_frequencies(64)
    b.dp_qknorm_rope(x, None, out, None, None, None, 1e-5, freq)
    pos = torch.arange(6, dtype=torch.int32, device=DEV).expand(2, 6).contiguous()
    b.dp_qknorm_rope(x, None, out2, None, torch.ones(64, device=DEV), None, 1e-5, freq, pos)
    assert torch.equal(out, out2)
    b.dp_qknorm_rope(x, None, out, None, None, None, 1e-5, None)
    ref = x.double() * (x.double().square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    within(out, ref, ref.abs() * QK_REL)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", QK_CASES)
def test_qknorm_rope_backward(case, dtype):
    B, T, hq, hk, D, rot, inter, first, layout = case
    eps = 1e-6
    q, k, gq, gk, pos, freq = qk_inputs(case, dtype, 11)
    g = gen(12)
    dys = [None if x is None else randn(g, *x.shape, dtype=dtype) for x in (q, k)]
    dxs = [None if x is None else torch.full(x.shape, float("nan"), dtype=dtype, device=DEV) for x in (q, k)]
    rows = [None if x is None else torch.full((B, D), float("nan"), device=DEV) for x in (q, k)]
    work = torch.empty(b.dp_qknorm_workspace_bytes(q, k), dtype=torch.uint8, device=DEV)

    def call(accumulate=False):
        b.dp_qknorm_rope_backward(q, k, dys[0], dys[1], dxs[0], dxs[1], gq, gk, rows[0], rows[1], eps, freq, pos, None,
                                  inter, accumulate, work)
    call()
    once = [None if r is None else r.clone() for r in rows]
    call()
    for x, gain, dy, dx, row, first_row in ((q, gq, dys[0], dxs[0], rows[0], once[0]), (k, gk, dys[1], dxs[1], rows[1], once[1])):
        if x is None:
            continue
        assert torch.equal(row, first_row)
        xd, fr = x.double(), NONE if freq is None else freq
        r = (xd.square().mean(-1, keepdim=True) + eps).rsqrt()
        hat, u = xd * r, rotate64(dy.double(), pos, fr, inter, -1.0)
        w = u * gain.double()
        mean = (w * hat).mean(-1, keepdim=True)
        ref = r * (w - hat * mean)
        # u carries the pair's error; the mean a sum of dim products of such
        places = pair_places(rot, inter)
        length = u.abs()
        both = torch.linalg.vector_norm(torch.stack([u[..., places[:, 0]], u[..., places[:, 1]]]), dim=0)
        length[..., places[:, 0]], length[..., places[:, 1]] = both, both
        wl = length * gain.double().abs()
        mag = r * (wl + hat.abs() * (wl * hat.abs()).mean(-1, keepdim=True))
        within(dx, ref, mag * 2 * QK_REL + ref.abs() * HALF[dtype] * 1.001 + mag * 2 * QK_REL * HALF[dtype], "dx")
        terms = (length * hat.abs()).sum((1, 2))
        heads = x.shape[2]
        adds = T * heads + 16                                          # at most every term in one run
        within(row, (u * hat).sum((1, 2)), terms * (QK_REL * 2 + min(adds, 600) * HALF[F32]), "gain rows")
    call(True)
    for row, first_row in zip(rows, once):
        if row is not None:
            within(row, 2 * first_row.double(), 2 * first_row.double().abs() * 1.01 * HALF[F32])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_qknorm_skips_tokens_behind_an_example(dtype):
    g = gen(13)
    B, T, H, D = 5, 70, 3, 64
    lengths = torch.tensor([0, 1, T, T + 9, 37], dtype=torch.int32, device=DEV)
    x, dy = randn(g, B, T, H, D, dtype=dtype), randn(g, B, T, H, D, dtype=dtype)
    away = torch.arange(T, device=DEV)[None, :] >= lengths[:, None]
    x[away], dy[away] = float("nan"), float("inf")
    gain, freq = 1 + 0.1 * randn(g, D), b.rope_frequencies(D)
    out, dx, rows = (torch.full(s, 5.0, dtype=d, device=DEV) for s, d in ((x.shape, dtype), (x.shape, dtype), ((B, D), F32)))
    work = torch.empty(b.dp_qknorm_workspace_bytes(x, None), dtype=torch.uint8, device=DEV)
    b.dp_qknorm_rope(x, None, out, None, gain, None, 1e-6, freq, None, lengths)
    b.dp_qknorm_rope_backward(x, None, dy, None, dx, None, gain, None, rows, None, 1e-6, freq, None, lengths, workspace=work)
    assert bool((out[away] == 5).all()) and bool((dx[away] == 5).all())
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(rows).all()) and bool((rows[0] == 0).all())
    for i in (1, 2, 4):
        n = int(lengths[i])
        o1, d1, r1 = torch.empty(1, n, H, D, dtype=dtype, device=DEV), torch.empty(1, n, H, D, dtype=dtype, device=DEV), torch.empty(1, D, device=DEV)
        xi, dyi = x[i:i + 1, :n].contiguous(), dy[i:i + 1, :n].contiguous()
        b.dp_qknorm_rope(xi, None, o1, None, gain, None, 1e-6, freq)
        b.dp_qknorm_rope_backward(xi, None, dyi, None, d1, None, gain, None, r1, None, 1e-6, freq,
                                  workspace=torch.empty(b.dp_qknorm_workspace_bytes(xi, None), dtype=torch.uint8, device=DEV))
        assert torch.equal(out[i, :n], o1[0]) and torch.equal(dx[i, :n], d1[0])
        within(rows[i], r1[0], (x[i, :n].double().abs().max() * 60 * dy[i, :n].double().abs().sum((0, 1))) * HALF[F32])


def test_qknorm_of_a_zero_head_without_eps_is_contained():
    """0 * rsqrt(0) is not a number; it must not reach other heads' outputs."""
    x = randn(gen(14), 1, 3, 5, 64)
    x[0, 1, 2] = 0.0
    out = torch.empty_like(x)
    b.dp_qknorm_rope(x, None, out, None, None, None, 0.0, b.rope_frequencies(64))
    bad = torch.isnan(out)
    assert bool(bad[0, 1, 2].all()) and int(bad.sum()) == 64


def test_qknorm_backward_against_differences():
    g = gen(15)
    B, T, H, D = 2, 4, 2, 16
    x, dy, gain = randn(g, B, T, H, D), randn(g, B, T, H, D), 1 + 0.2 * randn(g, D)
    freq = b.rope_frequencies(8)
    dx, rows = torch.empty_like(x), torch.empty(B, D, device=DEV)
    work = torch.empty(b.dp_qknorm_workspace_bytes(x, None), dtype=torch.uint8, device=DEV)
    b.dp_qknorm_rope_backward(x, None, dy, None, dx, None, gain, None, rows, None, 1e-3, freq, workspace=work)

    def f(x_, gain_):
        y = torch.empty_like(x_)
        b.dp_qknorm_rope(x_, None, y, None, gain_, None, 1e-3, freq)
        return (y.double() * dy.double()).sum((1, 2, 3))
    h = 2.0 ** -6
    # central differences: error h^2 / 6 times a third derivative (below 60 |dy| |v|^3 at these sizes) + fp32 / h
    noise = dy.double().abs().sum((1, 2, 3)) * 3 * QK_REL / h
    for seed in range(3):
        v = randn(gen(40 + seed), B, T, H, D) / math.sqrt(T * H * D)
        diff = (f(x + h * v, gain) - f(x - h * v, gain)) / (2 * h)
        within(diff, (dx.double() * v.double()).sum((1, 2, 3)), noise + 10 * h * h, "dx")
        u = randn(gen(50 + seed), D) / math.sqrt(D)
        diff = (f(x, gain + h * u) - f(x, gain - h * u)) / (2 * h)
        within(diff, (rows.double() * u.double()).sum(1), noise, "gain")


# ---- streams, captured graphs --------------------------------------------------------------------------------------
def test_calls_run_on_the_stream_they_are_given_and_replay_in_a_graph():
    g = gen(16)
    B, H, T, nb, D = 3, 2, 96, 32, 64
    G, x, dy = randn(g, B, H, T, T, dtype=BF16), randn(g, B, T, H, D, dtype=BF16), randn(g, B, T, H, D, dtype=BF16)
    grads = [randn(g, 5000), randn(g, 37)]
    outs = [torch.empty_like(t) for t in grads]
    gain, freq = torch.ones(D, device=DEV), b.rope_frequencies(D)
    rows, gr = torch.empty(B, nb, H, device=DEV), torch.empty(B, D, device=DEV)
    out, dx = torch.empty_like(x), torch.empty_like(x)
    acc, acc2 = torch.zeros(nb, H, device=DEV), torch.zeros(D, device=DEV)
    sq, clip, total = torch.empty(B, device=DEV), torch.empty(B, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
    works = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in
             (b.dp_relpos_workspace_bytes(G, nb), b.dp_qknorm_workspace_bytes(x, None), b.dp_global_norm_workspace_bytes())]
    theta, m, v = (torch.ones(5000, device=DEV) for _ in range(3))
    bias = torch.empty(H, T, T, dtype=BF16, device=DEV)

    def chain(stream=None):
        b.dp_relpos_bias(acc, bias, stream=stream)
        b.dp_qknorm_rope(x, None, out, None, gain, None, 1e-6, freq, stream=stream)
        b.dp_relpos_bias_grad(G, rows, workspace=works[0], stream=stream)
        b.dp_qknorm_rope_backward(x, None, dy, None, dx, None, gain, None, gr, None, 1e-6, freq, workspace=works[1], stream=stream)
        rl = b.RowList([(rows, acc), (gr, acc2)])
        b.dp_rows_sqnorms(rl, sq, stream=stream)
        b.dp_clip_factors(sq, 1.0, clip, stream=stream)
        b.dp_rows_clipped_accumulate(rl, clip, stream=stream)
        b.dp_global_sqnorm(grads, total, False, works[2], stream=stream)
        b.dp_clip_by_global_norm(grads, outs, total, 1.0, stream=stream)
        b.dp_clip_adamw_step(theta, m, v, grads[0], False, total, 1.0, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, stream=stream)

    def state():
        return [t.clone() for t in (bias, out, rows, dx, gr, sq, clip, acc, acc2, total, *outs, theta, m, v)]

    def reset():
        acc.zero_(), acc2.zero_(), theta.fill_(1), m.fill_(1), v.fill_(1)
    chain()
    want = state()
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    chain(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, state()))
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for new in (1, 2):
        for t, s in ((G, 0), (x, 1), (dy, 2)):
            t.copy_(randn(gen(60 + 10 * new + s), *t.shape, dtype=BF16))
        reset()
        graph.replay()
        torch.cuda.synchronize()
        got = state()
        reset()
        chain()
        assert all(torch.equal(p, q) for p, q in zip(got, state()))


def test_offsets_beyond_32_bits():
    """Scores and heads whose last elements lie more than 2^31 elements behind the first (views with large strides over one
    allocation of 9 GB)."""
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB of free device memory")
    big = torch.empty((1 << 32) + (1 << 20), dtype=BF16, device=DEV)
    far = 1 << 31
    G = big.as_strided((3, 1, 8, 64), (far, 64, 64, 1))
    g = gen(17)
    G.copy_(randn(g, 3, 1, 8, 64, dtype=BF16))
    ref, mag = relpos_rows(G, 32, 128, True, 0, False, None, None)
    rows = torch.empty(3, 32, 1, device=DEV)
    b.dp_relpos_bias_grad(G, rows, workspace=torch.empty(b.dp_relpos_workspace_bytes(G, 32), dtype=torch.uint8, device=DEV))
    within(rows, ref, mag * 100 * HALF[F32])
    x = big.as_strided((3, 2, 2, 64), (far, 128, 64, 1))
    x.copy_(randn(g, 3, 2, 2, 64, dtype=BF16))
    small, out = x.contiguous(), torch.empty(3, 2, 2, 64, dtype=BF16, device=DEV)
    freq = b.rope_frequencies(64)
    b.dp_qknorm_rope(small, None, out, None, None, None, 1e-6, freq)
    b.dp_qknorm_rope(x, None, x, None, None, None, 1e-6, freq)
    assert torch.equal(x, out)
    del G, x
    room = big.as_strided((3, 8, 64), (far, 64, 1))
    table = randn(g, 32, 3)
    b.dp_relpos_bias(table, room)
    near = torch.empty(3, 8, 64, dtype=BF16, device=DEV)
    b.dp_relpos_bias(table, near)
    assert torch.equal(room, near)
