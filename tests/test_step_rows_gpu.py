"""Whole macro-steps on the GPU with the attention block's own trainables: a relative position table shared by two
layers and the gains of the query and key norms, their per-example gradients formed by the library from the scores'
and the rotated heads' gradients, beside an ordinary linear layer; and the global-norm clip before the update."""
import math

import numpy as np
import pytest
import torch

from paper_2108_01624_b200 import DPStep, RowList, synth

from .helpers import LINEAR, LayerSpec, O, assert_update_close, b, random_layers, rel_l2, to_np, to_oracle_layers
from .test_attention_params_gpu import NONE, gen, relpos_rows, randn, rotate64

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

DEV = "cuda:0"
B, T, H, HK, D, NB = 6, 64, 4, 2, 32, 16
SPECS = [LayerSpec(LINEAR, 128, 64, True, "fc")] + synth.attention_param_specs(H, D, NB)


def per_example(mb, dtype):
    """The library's per-example gradients of one microbatch, and the same in 64 bits."""
    g = gen(500 + mb)
    scale = 10.0 ** (torch.rand(B, 1, 1, 1, generator=g, device=DEV) * 2 - 1) * 0.02
    k_len = torch.randint(1, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    rows = torch.empty(B, NB, H, device=DEV)
    ref = torch.zeros(B, NB, H, dtype=torch.float64, device=DEV)
    for layer in range(2):                                             # both layers' scores use the one table
        G = (randn(g, B, H, T, T) * scale).to(dtype)
        work = torch.empty(b.dp_relpos_workspace_bytes(G, NB), dtype=torch.uint8, device=DEV)
        b.dp_relpos_bias_grad(G, rows, 40, True, k_len=k_len, accumulate_into=layer > 0, workspace=work)
        ref += relpos_rows(G, NB, 40, True, 0, False, None, k_len)[0]
    qkv = randn(g, B, T, (H + 2 * HK) * D, dtype=dtype)
    q, k = qkv[..., :H * D].unflatten(-1, (H, D)), qkv[..., H * D:(H + HK) * D].unflatten(-1, (HK, D))
    dq, dk = (randn(g, *x.shape) * scale for x in (q, k))
    dq, dk = dq.to(dtype), dk.to(dtype)
    gain, freq = 1 + 0.1 * randn(g, D), b.rope_frequencies(D)
    gq, gk = torch.empty(B, D, device=DEV), torch.empty(B, D, device=DEV)
    work = torch.empty(b.dp_qknorm_workspace_bytes(q, k), dtype=torch.uint8, device=DEV)
    b.dp_qknorm_rope_backward(q, k, dq, dk, torch.empty_like(dq), torch.empty_like(dk), gain, gain, gq, gk, 1e-6, freq,
                              workspace=work)
    pos = torch.arange(T, device=DEV).expand(B, T)
    refs = []
    for x, dy in ((q, dq), (k, dk)):
        xd = x.double()
        hat = xd * (xd.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        refs.append((rotate64(dy.double(), pos, freq, False, -1.0) * hat).sum((1, 2)))
    return [gq.view(B, 1, D), gk.view(B, 1, D), rows], [r.cpu().numpy().reshape(B, -1) for r in (*refs, ref)]


@pytest.mark.parametrize("max_grad_norm", [None, 1e-3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_macro_steps_with_attention_parameters(dtype, max_grad_norm):
    hp = dict(C=0.05, sigma=0.8, lr=1e-2, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.5)
    step = DPStep(SPECS, DEV, seed=9, max_grad_norm=max_grad_norm, **hp)
    th = synth.initial_weights(step.n_flat, 1, DEV)
    step.theta.copy_(th)
    r_th, r_m, r_v = to_np(th), np.zeros(step.n_flat), np.zeros(step.n_flat)
    for t in (1, 2):
        flat, clipped = np.zeros(step.n_flat), []
        for mb in range(2):
            data = random_layers(SPECS[:1], B, T, dtype, DEV, seed=70 + 10 * t + mb, g_scale=0.005)
            grads, refs = per_example(10 * t + mb, dtype)
            data = data + [synth.LayerData(sp, G=gr) for sp, gr in zip(SPECS[1:], grads)]
            sq, clip = step.accumulate_microbatch(step.layer_list(data), rows=step.row_list(data))
            ol = to_oracle_layers(data[:1])
            n_ref = O.per_example_sqnorms(ol) + sum((r ** 2).sum(1) for r in refs)
            c_ref = O.clip_factors(n_ref, hp["C"])
            np.testing.assert_allclose(to_np(sq), n_ref, rtol=2e-3)
            np.testing.assert_allclose(to_np(clip), c_ref, rtol=1e-3)
            clipped += list(c_ref)
            acc = O.clipped_accumulate(ol, c_ref, O.zero_accumulators(ol))
            for k, a in enumerate(acc[0]):
                flat[step.offsets[0][k]:step.offsets[0][k] + a.size] += a.ravel()
            for li, r in enumerate(refs, start=1):
                flat[step.offsets[li][0]:step.offsets[li][0] + r.shape[1]] += c_ref @ r
        assert min(clipped) < 1.0                                      # the clip acts
        acc = to_np(step.acc)
        assert rel_l2(acc, flat) <= (2e-2 if dtype == torch.bfloat16 else 1e-4)
        for li in range(1, 4):                                         # rows are summed in fp32 whatever the dtype
            off, n = step.offsets[li][0], math.prod(step.shapes[li][0])
            assert rel_l2(acc[off:off + n], flat[off:off + n]) <= 2e-3
        step.finish_macro_batch()
        g = O.add_noise_and_scale(acc, hp["sigma"], hp["C"], 2 * B, seed=9, step=t, elem_offset=0)
        real = np.concatenate([np.arange(o, o + math.prod(s)) for offs, shps in zip(step.offsets, step.shapes)
                               for o, s in zip(offs, shps)])
        norm = np.linalg.norm(g[real])
        f = 1.0
        if max_grad_norm is not None:
            assert norm > max_grad_norm                                # the global clip acts too
            f = max_grad_norm / norm
            assert step.grad_norm() == pytest.approx(norm, rel=1e-5)
        new = O.adamw_step(r_th, r_m, r_v, g * f, hp["lr"], hp["beta1"], hp["beta2"], hp["xi"], hp["weight_decay"], t)
        assert_update_close(to_np(step.theta), r_th, new[0], new[2])
        assert rel_l2(to_np(step.m), new[1]) <= 1e-4 and float(step.acc.abs().max()) == 0.0
        r_th, r_m, r_v = to_np(step.theta), to_np(step.m), to_np(step.v)
    assert b.dp_poll_status() == 0


def test_an_example_contributes_at_most_the_clip_norm():
    """One example's clipped contribution over all tensors, rows included, has norm C."""
    grads, refs = per_example(1, torch.float32)
    step = DPStep(SPECS[1:], DEV, C=1e-3, sigma=0.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0)
    for i in range(B):
        step.acc.zero_()
        data = [synth.LayerData(sp, G=gr[i:i + 1].contiguous()) for sp, gr in zip(SPECS[1:], grads)]
        step.accumulate_microbatch([], rows=step.row_list(data))
        assert float(step.acc.double().norm()) == pytest.approx(1e-3, rel=1e-5)


def test_row_list_of_another_microbatch_size_is_refused():
    grads, _ = per_example(2, torch.float32)
    with pytest.raises(ValueError):
        RowList([(grads[0], None), (grads[1][:3], None)])
    with pytest.raises(ValueError):
        RowList([(grads[0], torch.zeros(D + 1, device=DEV))])
    with pytest.raises(ValueError):
        RowList([(grads[0].to(torch.bfloat16), None)])
    assert NONE.numel() == 0
