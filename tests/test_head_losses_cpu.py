"""Host side, without a GPU, of the vocabulary head's losses: struct layouts, what the calls refuse, workspace sizes, what the
binding and DPStep check before the library is called."""
import ctypes as C

import pytest
import torch

from paper_2108_01624_b200 import binding as b
from paper_2108_01624_b200 import build as builder
from paper_2108_01624_b200 import step as step_module
from paper_2108_01624_b200.synth import EMBEDDING, HEAD, LINEAR, ROWS, LayerSpec, Workload, generate, kappa

ARG, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -6
P = 4096          # an aligned address that nothing is read from


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return b.lib()


def head(**kw):
    f = dict(dtype=1, B=4, T=8, d=64, V=1000, X=P, ldx=64, W=P, ldw=64, bias=P, labels=P, weights=P)
    f.update(kw)
    return b.dp_vocab_head(*f.values())


def calls(lib, h, ws=P, n=1 << 45):
    """The four calls on a head with everything else in order."""
    r = C.byref(h)
    return {"loss": lib.dp_vocab_loss(r, P, P, ws, n, None),
            "backward": lib.dp_vocab_loss_backward(r, P, P, max(h.d, 1), P, 0, ws, n, None),
            "sum": lib.dp_vocab_loss_clipped_accumulate(r, P, P, P, P, ws, n, None),
            "cross": lib.dp_vocab_loss_cross_sqnorms(r, P, P, P, max(h.d, 1), 5, P, ws, n, None)}


def test_struct_layouts():
    assert C.sizeof(b.dp_vocab_head) == 80 and b.dp_vocab_head.X.offset == 24 and b.dp_vocab_head.weights.offset == 72
    assert C.sizeof(b.dp_distill) == 72 and b.dp_distill.temperature.offset == 24 and b.dp_distill.weights.offset == 64


@pytest.mark.parametrize("change, code", [
    (dict(X=None), ARG), (dict(W=None), ARG), (dict(labels=None), ARG), (dict(dtype=2), ARG), (dict(B=0), ARG), (dict(T=-1), ARG),
    (dict(d=0), ARG), (dict(V=0), ARG), (dict(ldx=63), ARG), (dict(ldw=0), ARG),
    (dict(X=P + 1), ALIGN), (dict(W=P + 1), ALIGN), (dict(labels=P + 2), ALIGN), (dict(bias=P + 2), ALIGN), (dict(weights=P + 1), ALIGN),
    (dict(dtype=0, X=P + 2), ALIGN), (dict(V=(1 << 26) + 1), UNSUPPORTED), (dict(B=1 << 20, T=128), UNSUPPORTED),
    (dict(d=(1 << 16) + 1, ldx=1 << 20, ldw=1 << 20), UNSUPPORTED)])
def test_heads_that_are_refused(lib, change, code):
    h = head(**change)
    assert set(calls(lib, h).values()) == {code}
    assert lib.dp_vocab_workspace_bytes(C.byref(h)) == 0


def test_arguments_that_are_refused(lib):
    h = head()
    r, n = C.byref(h), 1 << 45
    assert lib.dp_vocab_loss(None, P, P, P, n, None) == ARG
    assert lib.dp_vocab_loss(r, None, P, P, n, None) == ARG and lib.dp_vocab_loss(r, P, None, P, n, None) == ARG
    assert lib.dp_vocab_loss(r, P + 2, P, P, n, None) == ALIGN and lib.dp_vocab_loss(r, P, P + 1, P, n, None) == ALIGN
    bw = lib.dp_vocab_loss_backward
    assert bw(r, None, P, 64, P, 0, P, n, None) == ARG and bw(r, P, None, 64, None, 0, P, n, None) == ARG
    assert bw(r, P, P, 63, P, 0, P, n, None) == ARG and bw(r, P, P + 1, 64, P, 0, P, n, None) == ALIGN
    assert bw(r, P, P, 64, P + 2, 0, P, n, None) == ALIGN
    su = lib.dp_vocab_loss_clipped_accumulate
    assert su(r, None, P, P, P, P, n, None) == ARG and su(r, P, None, P, P, P, n, None) == ARG
    assert su(r, P, P, None, P, P, n, None) == ARG and su(r, P, P, P, None, P, n, None) == ARG
    assert su(r, P, P, P + 2, P, P, n, None) == ALIGN
    cr = lib.dp_vocab_loss_cross_sqnorms
    assert cr(r, P, None, P, 64, 5, P, P, n, None) == ARG and cr(r, P, P, P, 64, 0, P, P, n, None) == ARG
    assert cr(r, P, P, P, 63, 5, P, P, n, None) == ARG and cr(r, P, P, P + 1, 64, 5, P, P, n, None) == ALIGN
    assert cr(r, P, P, P, 64, 1 << 27, P, P, n, None) == UNSUPPORTED
    need = lib.dp_vocab_workspace_bytes(r)
    assert need > 0
    for ws, size in ((None, n), (P + 128, n), (P, 16)):
        assert set(calls(lib, h, ws, size).values()) == {WORKSPACE}
    no_bias = head(bias=None)
    assert lib.dp_vocab_loss_clipped_accumulate(C.byref(no_bias), P, P, P, None, None, 0, None) == WORKSPACE   # acc_b is not asked for


def test_the_workspace_is_bounded(lib):
    """G takes at most 1 GiB, or one block of 2048 columns; the rest are token rows, shared tiles and small sums."""
    def size(B, T, d, V, dtype=1):
        return lib.dp_vocab_workspace_bytes(C.byref(head(B=B, T=T, d=d, V=V, ldx=d, ldw=d, dtype=dtype)))
    gib = 1 << 30
    assert size(256, 20, 1024, 30522) < gib
    for V in (30522, 250000, 1 << 24):
        assert size(256, 128, 1024, V) < 2 * gib + 8 * V             # the bias, padded, comes with V
    assert size(256, 20, 1024, 30522, dtype=0) < 2 * gib
    assert size(1, 1, 8, 1) < 64 << 20


@pytest.mark.parametrize("change, code", [
    (dict(logits=None), ARG), (dict(top_ids=None), ARG), (dict(top_logits=None), ARG), (dict(dtype=3), ARG), (dict(teacher_dtype=-1), ARG),
    (dict(N=0), ARG), (dict(V=0), ARG), (dict(K=0), ARG), (dict(temperature=0.0), ARG), (dict(temperature=-1.0), ARG),
    (dict(temperature=float("nan")), ARG), (dict(temperature=float("inf")), ARG), (dict(temperature=1e-40), ARG), (dict(ld=499), ARG),
    (dict(K=1025), UNSUPPORTED), (dict(V=(1 << 30) + 1, ld=1 << 31), UNSUPPORTED), (dict(logits=P + 1), ALIGN), (dict(top_ids=P + 2), ALIGN),
    (dict(top_logits=P + 2), ALIGN), (dict(weights=P + 1), ALIGN)])
def test_distillations_that_are_refused(lib, change, code):
    f = dict(dtype=1, teacher_dtype=0, N=6, V=500, K=8, temperature=2.0, logits=P, ld=500, top_ids=P, top_logits=P, weights=P)
    f.update(change)
    assert lib.dp_distill_loss(C.byref(b.dp_distill(*f.values())), P, 2 * P, max(f["ld"], f["V"]), None) == code


def test_distillation_outputs_that_are_refused(lib):
    p = b.dp_distill(1, 0, 6, 500, 8, 2.0, P, 500, P, P, P)
    r = C.byref(p)
    assert lib.dp_distill_loss(None, P, P, 500, None) == ARG and lib.dp_distill_loss(r, None, P, 500, None) == ARG
    assert lib.dp_distill_loss(r, P, 2 * P, 499, None) == ARG
    assert lib.dp_distill_loss(r, P, P, 512, None) == ARG            # in place with other rows
    assert lib.dp_distill_loss(r, P, P + 1, 500, None) == ALIGN and lib.dp_distill_loss(r, P + 2, 2 * P, 500, None) == ALIGN


def test_binding_checks_tensors_before_the_library_is_called(lib):
    x, w, y = torch.zeros(2, 3, 8), torch.zeros(5, 8), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        b.VocabHead(x, w, y)
    with pytest.raises(ValueError, match="device tensor"):
        b.dp_distill_loss(torch.zeros(1, 2, 8), torch.zeros(1, 2, 3, dtype=torch.int32), torch.zeros(1, 2, 3), 1.0, torch.zeros(1, 2), None)
    with pytest.raises(ValueError, match="tensor expected"):
        b.VocabHead(3, w, y)
    for bad in (None, (0,), (0, b"short")):
        with pytest.raises(ValueError, match="vocabulary head expected"):
            b._native().vocab_workspace_bytes(bad)


class FakeHead:
    def __init__(self, B, V, d, bias=True):
        self.B, self.weight, self.bias = B, torch.zeros(V, d), torch.zeros(V) if bias else None


def dp_step(specs, **kw):
    return step_module.DPStep(specs, "cpu", C=1.0, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0, **kw)


def test_a_heads_place_among_the_parameters():
    specs = [LayerSpec(EMBEDDING, 50, 8, False, "emb"), LayerSpec(LINEAR, 8, 6, True, "fc"), LayerSpec(HEAD, 50, 8, True, "mlm")]
    own = dp_step(specs)
    assert own.n_flat == 400 + 48 + 8 + 400 + 52 and own.shapes[2] == [(50, 8), (50,)]
    shared = dp_step(specs, shared_tables={2: 0})
    assert shared.offsets[2] == [0, 456] and shared.n_flat == 456 + 52           # the table is the embedding's, the bias its own
    flat = torch.arange(shared.n_flat, dtype=torch.float32)
    assert [p.numel() for p in shared.tensor_pieces(flat)] == [400, 48, 6, 50]
    assert [p.numel() for p in shared.tensor_pieces(flat[450:], 450)] == [4, 50]
    assert sum(s.n_params() for s in specs) == 400 + 54 + 450
    assert kappa(specs, 4) == kappa(specs[:2], 4)
    for bad in ({2: 1}, {0: 2}):
        with pytest.raises(ValueError):
            dp_step(specs, shared_tables=bad)
    with pytest.raises(ValueError, match="only one"):
        dp_step([specs[0], specs[2], specs[2]], shared_tables={1: 0, 2: 0})
    with pytest.raises(ValueError, match="not drawn"):
        generate(Workload("w", 2, 4, torch.float32, specs), specs=specs[2:])


def test_a_microbatch_wants_every_head(monkeypatch):
    """Norms begin with the heads', in the order of their calls; one left out, or of another microbatch, is refused."""
    said = []
    monkeypatch.setattr(step_module.b, "dp_vocab_workspace_bytes", lambda h: 256)
    monkeypatch.setattr(step_module.b, "dp_vocab_loss_backward", lambda h, lse, dx, sq, add, ws, s: said.append(("norm", h.B, add)))
    monkeypatch.setattr(step_module.b, "dp_clip_factors", lambda *a: said.append("clip"))
    monkeypatch.setattr(step_module.b, "dp_vocab_loss_clipped_accumulate", lambda h, lse, c, w, bias, ws, s: said.append(("sum", tuple(w.shape), bias is not None)))
    specs = [LayerSpec(HEAD, 50, 8, True, "a"), LayerSpec(HEAD, 20, 8, False, "b")]
    step = dp_step(specs)
    a, c = FakeHead(4, 50, 8), FakeHead(4, 20, 8, bias=False)
    with pytest.raises(ValueError, match="every HEAD"):
        step.accumulate_microbatch([])
    step.head_backward(1, c, None, None)
    with pytest.raises(ValueError, match="every HEAD"):
        step.accumulate_microbatch([])
    step.head_backward(0, a, None, None)
    step.accumulate_microbatch([])
    assert said == [("norm", 4, False), ("norm", 4, True), "clip", ("sum", (50, 8), True), ("sum", (20, 8), False)]
    assert step.examples_seen == 4
    with pytest.raises(ValueError, match="every HEAD"):
        step.accumulate_microbatch([])                               # the next microbatch wants them again
    said.clear()
    step.head_backward(0, a, None, None)
    step.head_backward(0, a, None, None)                             # begins anew
    step.head_backward(1, FakeHead(3, 20, 8, bias=False), None, None)    # another microbatch
    assert said == [("norm", 4, False), ("norm", 4, False), ("norm", 3, False)]
    for li, h in ((0, c), (0, FakeHead(4, 50, 8, bias=False)), (1, FakeHead(4, 20, 8))):
        with pytest.raises(ValueError, match="expected"):
            step.head_backward(li, h, None, None)
    with pytest.raises(ValueError, match="no HEAD"):
        dp_step([LayerSpec(ROWS, 1, 8)]).head_backward(0, a, None, None)
    step.discard_macro_batch()
    assert step.examples_seen == 0
    with pytest.raises(ValueError, match="every HEAD"):
        step.accumulate_microbatch([])


def test_a_heads_outgrown_workspace_outlives_the_stream_that_uses_it(monkeypatch):
    """Calls on a stream of the caller's may still be at work in a workspace when a larger microbatch replaces it."""
    step = dp_step([LayerSpec(HEAD, 20, 8, False, "mlm")])
    recorded = []

    class Buffer:
        def numel(self):
            return 256

        def record_stream(self, stream):
            recorded.append(stream)

    step._head_ws = Buffer()
    monkeypatch.setattr(step_module.b, "dp_vocab_workspace_bytes", lambda head: 256)
    step._head_workspace(None, "side")
    assert recorded == []
    monkeypatch.setattr(step_module.b, "dp_vocab_workspace_bytes", lambda head: 512)
    assert step._head_workspace(None, "side").numel() == 512
    assert recorded == ["side"]
