"""The vocabulary head's losses as they are used: a masked-LM head that shares its table with the token embedding, beside other
tensors, through DPStep; distillation whose gradient is a layer's G; captured, replayed and concurrent calls."""
import math

import pytest
import torch

import paper_2108_01624_b200 as dp
from paper_2108_01624_b200 import synth
from paper_2108_01624_b200.synth import EMBEDDING, HEAD, LAYERNORM, LINEAR, ROWS, LayerData, LayerSpec

pytestmark = pytest.mark.gpu
DEV = "cuda"


def work(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def new_step(specs, **kw):
    return dp.DPStep(specs, DEV, C=0.7, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.1, **kw)


class Model:
    """Embedding table V x d shared with the head, a linear layer, a norm, a small table: inputs of one microbatch."""

    def __init__(self, dtype, B=6, T=13, Tm=4, d=40, V=211, seed=0):
        self.B, self.T, self.Tm, self.d, self.V, self.dtype = B, T, Tm, d, V, dtype
        self.specs = [LayerSpec(EMBEDDING, V, d, False, "emb"), LayerSpec(LINEAR, d, 24, True, "fc"), LayerSpec(LAYERNORM, d, d, False, "ln"),
                      LayerSpec(ROWS, 4, 3, False, "relpos"), LayerSpec(HEAD, V, d, True, "mlm")]
        self.draw(seed)

    def draw(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        B, T, Tm, d, V = self.B, self.T, self.Tm, self.d, self.V

        def normal(*s, scale=1.0):
            return torch.randn(*s, generator=g, device=DEV) * scale
        self.ids = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
        self.labels = self.ids[:, :Tm].clone()
        self.labels[0, 1:] = -1
        G = [normal(B, T, d, scale=0.05), normal(B, T, 24, scale=0.02), normal(B, T, d, scale=0.05)]
        A = [None, normal(B, T, d), normal(B, T, d)]
        self.data = [LayerData(self.specs[k], G=G[k].to(self.dtype), A=None if A[k] is None else A[k].to(self.dtype),
                               ids=self.ids if k == 0 else None) for k in range(3)]
        self.data += [LayerData(self.specs[3], G=normal(B, 4, 3, scale=0.1)), None]
        self.x, self.weight = normal(B, Tm, d).to(self.dtype), normal(V, d, scale=0.2).to(self.dtype)
        self.bias, self.tw = normal(V, scale=0.1), torch.rand(B, Tm, generator=g, device=DEV)

    def gradients(self):
        """Every example's gradients in 64 bits: table, linear weight and bias, norm gain and bias, rows, head bias."""
        B, V, d = self.B, self.V, self.d
        emb, fc, ln = (self.data[k] for k in range(3))
        table = torch.zeros(B, V, d, dtype=torch.float64, device=DEV)
        table.scatter_add_(1, self.ids.long()[..., None].expand(-1, -1, d), emb.G.double())
        z = self.x.double() @ self.weight.double().t() + self.bias.double()
        p = torch.softmax(z, -1)
        live = (self.labels >= 0).double()[..., None]
        p = (p - torch.nn.functional.one_hot(self.labels.clamp(min=0).long(), V)) * live * self.tw.double()[..., None]
        table += p.transpose(1, 2) @ self.x.double()
        return [table, fc.A.double().transpose(1, 2) @ fc.G.double(), fc.G.double().sum(1), (ln.A.double() * ln.G.double()).sum(1),
                ln.G.double().sum(1), self.data[3].G.double(), p.sum(1)]


def run_microbatch(step, m, head, loss, lse, dx, ws):
    dp.dp_vocab_loss(head, loss, lse, workspace=ws)
    step.head_backward(4, head, lse, dx)
    return step.accumulate_microbatch(step.layer_list(m.data), rows=step.row_list(m.data))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_shared_head_in_the_privatised_step(dtype):
    m = Model(dtype)
    step = new_step(m.specs, shared_tables={4: 0})
    refs = [torch.zeros_like(g[0]) for g in m.gradients()]
    for seed in (0, 1):
        m.draw(seed)
        head = dp.VocabHead(m.x, m.weight, m.labels, bias=m.bias, token_weights=m.tw)
        loss, lse = torch.empty(m.B, m.Tm, device=DEV), torch.empty(m.B, m.Tm, device=DEV)
        dx = torch.empty_like(m.x)
        sq, clip = run_microbatch(step, m, head, loss, lse, dx, work(dp.dp_vocab_workspace_bytes(head)))
        grads = m.gradients()
        n = sum(g.flatten(1).pow(2).sum(1) for g in grads)
        # norms: bf16 activations and gradients are exact inputs, the products' sums fp32 (2^-15 of absolute sums, cancellation
        # between the parts below 16); factors follow with half of it
        assert bool(((sq.double() - n).abs() <= 2.0 ** -11 * n).all())
        c = torch.clamp(0.7 / n.sqrt(), max=1.0)
        assert bool((c < 1).any()) and bool(((clip.double() - c).abs() <= 2.0 ** -11 * c).all())
        for r, g in zip(refs, grads):
            r += torch.einsum("b...,b->...", g, c)
    got = [step.view(step.acc, 0, 0), step.view(step.acc, 1, 0), step.view(step.acc, 1, 1), step.view(step.acc, 2, 0), step.view(step.acc, 2, 1),
           step.view(step.acc, 3, 0), step.view(step.acc, 4, 1)]
    assert step.view(step.acc, 4, 0).data_ptr() == got[0].data_ptr()
    for a, r in zip(got, refs):      # the linear layer's G is rounded to bf16 after it is scaled: 2^-8 of absolute sums, in norm less
        assert float((a.double() - r).norm()) <= (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11) * float(r.norm())
    theta = step.theta.clone()
    step.finish_macro_batch()
    assert dp.dp_poll_status() == 0 and not torch.equal(theta, step.theta) and bool(step.theta.isfinite().all())


def test_the_head_equals_a_projection_that_is_given_its_logits_gradient():
    """The same microbatch through a LINEAR projection whose A is dlogits: norms and sums agree to what bf16 dlogits lose."""
    m = Model(torch.bfloat16, V=208)
    head = dp.VocabHead(m.x, m.weight, m.labels, bias=None, token_weights=m.tw)
    loss, lse, dx = torch.empty(m.B, m.Tm, device=DEV), torch.empty(m.B, m.Tm, device=DEV), torch.empty_like(m.x)
    a = new_step(m.specs[:1] + [LayerSpec(HEAD, m.V, m.d, False)], shared_tables={1: 0})
    dp.dp_vocab_loss(head, loss, lse, workspace=work(dp.dp_vocab_workspace_bytes(head)))
    a.head_backward(1, head, lse, dx)
    sq, _ = a.accumulate_microbatch(a.layer_list(m.data[:1] + [None]))
    z = m.x.float() @ m.weight.float().t()
    G = (z - lse[..., None]).exp() - torch.nn.functional.one_hot(m.labels.clamp(min=0).long(), m.V)
    G = (G * torch.where(m.labels >= 0, m.tw, 0.0)[..., None]).bfloat16()
    spec = LayerSpec(LINEAR, m.V, m.d, False)
    p = new_step(m.specs[:1] + [spec], shared_tables={1: 0})
    sq2, _ = p.accumulate_microbatch(p.layer_lists([m.data[0], LayerData(spec, G=m.x, A=G)]))
    assert bool(((sq - sq2).abs() <= 2.0 ** -7 * sq2).all())
    assert float((a.acc - p.acc).norm()) <= 2.0 ** -7 * float(p.acc.norm())


def test_distilled_gradients_train_a_layer():
    """Teacher's top logits to dlogits in place, then the projection's norms, clip and sum; the dlogits in 64 bits as the oracle."""
    B, T, d, V, K = 5, 6, 64, 512, 8
    g = torch.Generator(device=DEV).manual_seed(0)
    x, w = torch.randn(B, T, d, generator=g, device=DEV).bfloat16(), (torch.randn(d, V, generator=g, device=DEV) * 0.3).bfloat16()
    logits = (x.float() @ w.float()).bfloat16()
    top, ids = (logits.float() + torch.randn(B, T, V, generator=g, device=DEV)).topk(K, -1)
    zd = logits.double() / 2.0
    q = torch.softmax(top.double() / 2.0, -1)
    G = 2.0 * torch.softmax(zd, -1).scatter_add(-1, ids, -q)
    loss = torch.empty(B, T, device=DEV)
    dp.dp_distill_loss(logits, ids.int(), top, 2.0, loss, logits)
    assert bool(((logits.double() - G).abs() <= 2.0 ** -8 * G.abs() + 2.0 ** -16 * (G.abs() + 2.0 * torch.zeros_like(G).scatter_add(-1, ids, q))).all())
    step = new_step([LayerSpec(LINEAR, d, V, False)])
    sq, clip = step.accumulate_microbatch(step.layer_list([LayerData(step.specs[0], G=logits, A=x)]))
    per = x.double().transpose(1, 2) @ G
    n = per.flatten(1).pow(2).sum(1)
    assert bool(((sq.double() - n).abs() <= 2.0 ** -6 * n).all())           # dlogits to 2^-8, squared
    ref = torch.einsum("bij,b->ij", per, torch.clamp(0.7 / n.sqrt(), max=1.0))
    assert float((step.view(step.acc, 0, 0).double() - ref).norm()) <= 2.0 ** -6 * float(ref.norm())


def chain(m, head, out, ws, stream=None):
    dp.dp_vocab_loss(head, out["loss"], out["lse"], workspace=ws, stream=stream)
    dp.dp_vocab_loss_backward(head, out["lse"], out["dx"], out["sq"], workspace=ws, stream=stream)
    dp.dp_vocab_loss_cross_sqnorms(head, out["lse"], m.ids, m.data[0].G, out["sq"], workspace=ws, stream=stream)
    dp.dp_clip_factors(out["sq"], 0.7, out["clip"], stream=stream)
    out["acc_w"].zero_()
    out["acc_b"].zero_()
    dp.dp_vocab_loss_clipped_accumulate(head, out["lse"], out["clip"], out["acc_w"], out["acc_b"], workspace=ws, stream=stream)


def outputs(m):
    e = dict(device=DEV)
    return {"loss": torch.empty(m.B, m.Tm, **e), "lse": torch.empty(m.B, m.Tm, **e), "dx": torch.empty_like(m.x), "sq": torch.empty(m.B, **e),
            "clip": torch.empty(m.B, **e), "acc_w": torch.empty(m.V, m.d, **e), "acc_b": torch.empty(m.V, **e)}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_captured_chain_replays_with_new_inputs(dtype):
    m = Model(dtype, B=9, V=700)
    head = dp.VocabHead(m.x, m.weight, m.labels, bias=m.bias, token_weights=m.tw)
    ws, out = work(dp.dp_vocab_workspace_bytes(head)), outputs(m)
    chain(m, head, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(m, head, out, ws)
    for seed in (5, 6):
        other = Model(dtype, B=9, V=700, seed=seed)
        for name in ("x", "weight", "labels", "bias", "tw", "ids"):
            getattr(m, name).copy_(getattr(other, name))
        m.data[0].G.copy_(other.data[0].G)
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        replayed = {k: t.clone() for k, t in out.items()}
        chain(m, head, out, ws)
        assert all(torch.equal(replayed[k], out[k]) and bool(out[k].isfinite().all()) for k in out)
    # distillation, captured on rows that come from a kernel before it
    z0 = torch.randn(3, 5, 901, device=DEV).to(dtype)
    z, ids, t = torch.empty_like(z0), torch.randint(0, 901, (3, 5, 6), device=DEV, dtype=torch.int32), torch.randn(3, 5, 6, device=DEV)
    loss = torch.empty(3, 5, device=DEV)
    graph = torch.cuda.CUDAGraph()
    dp.dp_distill_loss(z0, ids, t, 2.0, loss, z)
    want, first = z.clone(), loss.clone()
    with torch.cuda.graph(graph):
        z.copy_(z0)
        dp.dp_distill_loss(z, ids, t, 2.0, loss, z)
    for _ in range(3):
        loss.zero_()
        graph.replay()
        assert torch.equal(z, want) and torch.equal(loss, first)


def test_two_streams_with_workspaces_of_their_own():
    models = [Model(torch.bfloat16, B=30, T=20, V=3000, seed=s) for s in (1, 2)]
    heads = [dp.VocabHead(m.x, m.weight, m.labels, bias=m.bias, token_weights=m.tw) for m in models]
    want = []
    for m, h in zip(models, heads):
        out = outputs(m)
        chain(m, h, out, work(dp.dp_vocab_workspace_bytes(h)))
        want.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs, spaces = [outputs(m) for m in models], [work(dp.dp_vocab_workspace_bytes(h)) for h in heads]
    torch.cuda.synchronize()
    for _ in range(4):
        for m, h, out, ws, s in zip(models, heads, outs, spaces, streams):
            with torch.cuda.stream(s):
                chain(m, h, out, ws, stream=s)
    torch.cuda.synchronize()
    for out, ref in zip(outs, want):
        assert all(torch.equal(out[k], ref[k]) for k in out)


def test_a_microbatch_of_the_encoder_stack_with_its_head():
    """Two encoder blocks, the word-piece table and the head that shares it: the step runs and every clipped contribution stays
    within C (one example a microbatch: the accumulator's norm)."""
    specs = synth.encoder_layer_specs(128, 256, "l0.") + [LayerSpec(EMBEDDING, 3001, 128, False, "tok_emb")]
    wl = synth.Workload("stack", 1, 32, torch.bfloat16, specs)
    step = new_step(specs + [LayerSpec(HEAD, 3001, 128, True, "mlm")], shared_tables={7: 6})
    for seed in range(3):
        data = synth.generate(wl, seed=seed, device=DEV) + [None]
        g = torch.Generator(device=DEV).manual_seed(seed)
        x = torch.randn(1, 5, 128, generator=g, device=DEV).bfloat16()
        w = (torch.randn(3001, 128, generator=g, device=DEV) * 0.1).bfloat16()
        y = torch.randint(0, 3001, (1, 5), generator=g, device=DEV, dtype=torch.int32)
        head = dp.VocabHead(x, w, y, bias=torch.zeros(3001, device=DEV))
        loss, lse = torch.empty(1, 5, device=DEV), torch.empty(1, 5, device=DEV)
        dp.dp_vocab_loss(head, loss, lse, workspace=work(dp.dp_vocab_workspace_bytes(head)))
        step.head_backward(7, head, lse, None)
        sq, clip = step.accumulate_microbatch(step.layer_list(data))
        assert float(clip) < 1.0
        # the linear layers' G is rounded to bf16 after it is scaled (2^-8)
        assert abs(math.sqrt(float(step.acc.double().pow(2).sum())) - 0.7) <= 2.0 ** -8 * 0.7
        step.discard_macro_batch()
