"""DPStep with a vocabulary head, without a GPU: a microbatch that is refused or fails leaves no norms behind that a later one
would add to.  The library's calls are stand-ins that do their sums on the host."""
import pytest
import torch

from paper_2108_01624_b200 import step as step_module
from paper_2108_01624_b200.binding import Layer
from paper_2108_01624_b200.parallel import ShardedUpdate
from paper_2108_01624_b200.synth import EMBEDDING, HEAD, LINEAR, LayerSpec

SPECS = [LayerSpec(EMBEDDING, 50, 8, False, "emb"), LayerSpec(LINEAR, 8, 6, False, "fc"), LayerSpec(HEAD, 50, 8, False, "mlm")]


class Head:
    def __init__(self, B=4, V=50, d=8):
        self.B, self.weight, self.bias, self.x = B, torch.zeros(V, d), None, torch.zeros(B, 3, d)


class Layers:
    def __init__(self, layers, B=4):
        self.layers, self.B = layers, B

    def __len__(self):
        return len(self.layers)


class Calls:
    """Layers' norms of 10 an example, a head's of 1, a cross term of -2; clip factors keep what they were given."""

    def __init__(self, monkeypatch):
        self.names, self.fails, self.seen = [], None, None
        for name in ("dp_workspace_bytes", "dp_vocab_workspace_bytes"):
            monkeypatch.setattr(step_module.b, name, lambda x: 256)
        monkeypatch.setattr(step_module.b, "LayerList", Layers)
        norms = lambda value: lambda a, sq, add, *rest: sq.copy_(sq * bool(add) + value)
        self.put(monkeypatch, "dp_per_example_sqnorms", norms(10.0))
        self.put(monkeypatch, "dp_vocab_loss_backward", lambda h, lse, dx, sq, add, *rest: sq.copy_(sq * bool(add) + 1.0))
        self.put(monkeypatch, "dp_vocab_loss_cross_sqnorms", lambda h, lse, ids, g, sq, *rest: sq.sub_(2.0))
        self.put(monkeypatch, "dp_clip_factors", lambda sq, *rest: setattr(self, "seen", sq.clone()))
        for name in ("dp_clipped_accumulate_after_sqnorms", "dp_vocab_loss_clipped_accumulate"):
            self.put(monkeypatch, name, lambda *a: None)

    def put(self, monkeypatch, name, act):
        def call(*a):
            self.names.append(name)
            act(*a)
            if name == self.fails:
                raise RuntimeError(name)
        monkeypatch.setattr(step_module.b, name, call)


def make(monkeypatch):
    calls = Calls(monkeypatch)
    step = step_module.DPStep(SPECS, "cpu", C=1.0, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0, shared_tables={2: 0})
    emb = Layer(kind=EMBEDDING, G=torch.zeros(4, 5, 8), ids=torch.zeros(4, 5, dtype=torch.int32), acc_w=step.view(step.acc, 0, 0))
    fc = Layer(kind=LINEAR, G=torch.zeros(4, 5, 6), A=torch.zeros(4, 5, 8), acc_w=step.view(step.acc, 1, 0))
    return step, calls, emb, fc


def begun_anew(step, calls, layers, norm=9.0):
    """The microbatch, whole: head 1, layers 10, cross term -2."""
    step.head_backward(2, Head(), None, None)
    step.accumulate_microbatch(layers)
    return torch.equal(calls.seen, torch.full((4,), norm))


def test_what_is_refused_is_refused_before_the_first_norm(monkeypatch):
    step, calls, emb, fc = make(monkeypatch)
    step.head_backward(2, Head(), None, None)
    calls.names.clear()
    other = Layer(kind=EMBEDDING, G=emb.G.bfloat16(), ids=emb.ids, acc_w=emb.acc_w)
    wide = Layer(kind=EMBEDDING, G=torch.zeros(4, 5, 16), ids=emb.ids, acc_w=emb.acc_w)
    for bad in (Layers([fc]), Layers([other, fc]), Layers([wide, fc]), Layers([emb, emb, fc]), [Layers([emb]), Layers([fc], B=5)]):
        with pytest.raises(ValueError):
            step.accumulate_microbatch(bad)
    assert calls.names == [] and step.examples_seen == 0
    step.accumulate_microbatch(Layers([emb, fc]))              # corrected, the head's norms still there
    assert torch.equal(calls.seen, torch.full((4,), 9.0)) and step.examples_seen == 4


@pytest.mark.parametrize("name", ["dp_per_example_sqnorms", "dp_vocab_loss_cross_sqnorms", "dp_clip_factors"])
def test_a_microbatch_that_fails_midway_wants_its_heads_again(monkeypatch, name):
    step, calls, emb, fc = make(monkeypatch)
    step.head_backward(2, Head(), None, None)
    calls.fails = name
    with pytest.raises(RuntimeError, match=name):
        step.accumulate_microbatch(Layers([emb, fc]))
    calls.fails = None
    with pytest.raises(ValueError, match="every HEAD"):
        step.accumulate_microbatch(Layers([emb, fc]))
    assert begun_anew(step, calls, Layers([emb, fc]))


def test_a_heads_backward_that_fails_drops_the_heads_before_it(monkeypatch):
    specs = [LayerSpec(HEAD, 50, 8, False, "a"), LayerSpec(HEAD, 50, 8, False, "b")]
    calls = Calls(monkeypatch)
    step = step_module.DPStep(specs, "cpu", C=1.0, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0)
    step.head_backward(0, Head(), None, None)
    calls.fails = "dp_vocab_loss_backward"                     # after it has added to the norms
    with pytest.raises(RuntimeError):
        step.head_backward(1, Head(), None, None)
    calls.fails = None
    step.head_backward(1, Head(), None, None)
    with pytest.raises(ValueError, match="every HEAD"):
        step.accumulate_microbatch([])
    step.head_backward(0, Head(), None, None)
    step.accumulate_microbatch([])
    assert torch.equal(calls.seen, torch.full((4,), 2.0))


def test_a_macro_batch_that_the_ranks_discard_takes_its_heads_along(monkeypatch):
    """The status that made them discard it may be that of a head's norms."""
    class Dist:
        ReduceOp = torch.distributed.ReduceOp

        def get_backend(self):
            return "gloo"

        def all_reduce(self, t, op=None):
            return None
    step, calls, emb, fc = make(monkeypatch)
    step.acc.fill_(1.0)
    update = ShardedUpdate(step, Dist(), 1, 0, poll_fn=lambda: -5)
    step.head_backward(2, Head(), None, None)
    step.examples_seen = 4
    with pytest.raises(step_module.DeviceStatusError):
        update.finish_macro_batch()
    assert step.examples_seen == 0 and not step.acc.any()
    with pytest.raises(ValueError, match="every HEAD"):
        step.accumulate_microbatch(Layers([emb, fc]))


class Buffer:
    """Stands for a buffer on the device: its size, and the streams that it was recorded for."""

    def __init__(self, n):
        self.n, self.recorded = n, []

    def numel(self):
        return self.n

    def record_stream(self, stream):
        self.recorded.append(stream)


def test_buffers_that_are_replaced_outlive_every_stream_that_used_them(monkeypatch):
    for name in ("dp_workspace_bytes", "dp_vocab_workspace_bytes"):
        monkeypatch.setattr(step_module.b, name, lambda x: x.B * 64)
    monkeypatch.setattr(step_module.b, "LayerList", Layers)
    for name in ("dp_per_example_sqnorms", "dp_vocab_loss_backward", "dp_clip_factors", "dp_clipped_accumulate_after_sqnorms",
                 "dp_vocab_loss_clipped_accumulate"):
        monkeypatch.setattr(step_module.b, name, lambda *a: None)
    step = step_module.DPStep(SPECS[1:], "cpu", C=1.0, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0)

    def microbatch(B, stream, lists=1):
        step.head_backward(1, Head(B=B), None, None, stream=stream)
        step.accumulate_microbatch([Layers([None], B=B)] * lists, stream=stream)
    old = step._sqnorm, step._clip, step._ws, step._head_ws = Buffer(4), Buffer(4), [Buffer(256)], Buffer(256)
    microbatch(4, "a")
    microbatch(4, "b")
    assert all(t.recorded == [] for t in (old[0], old[1], old[2][0], old[3]))
    ws = old[2][0]
    microbatch(5, "c")                                         # more of everything
    for t in (old[0], old[1], ws, old[3]):
        assert {"a", "b"} <= set(t.recorded) <= {"a", "b", "c"}
    assert step._sqnorm.numel() == step._clip.numel() == 5 and step._ws[0].numel() == step._head_ws.numel() == 320
    step._sqnorm, step._clip, step._ws, step._head_ws = new = Buffer(5), Buffer(5), [Buffer(320)], Buffer(320)
    microbatch(5, "d")
    other = new[2][0]
    microbatch(3, "d", lists=2)                                # fewer examples, another number of lists
    assert set(new[0].recorded) == set(new[1].recorded) == {"c", "d"} and set(other.recorded) == {"c", "d"}
    assert new[3].recorded == [] and step._head_ws is new[3]   # large enough


def test_buffers_are_allocated_for_the_stream_that_uses_them(monkeypatch):
    """What torch allocates or fills for a call on a stream of the caller's goes to that stream."""
    calls = Calls(monkeypatch)
    entered = []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream)

        def __exit__(self, *a):
            entered.append(None)
    empty = torch.empty

    def watched(*a, **k):
        assert entered and entered[-1] == "s"
        return empty(*a, **k)
    step = step_module.DPStep(SPECS[1:], "cpu", C=1.0, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0)
    monkeypatch.setattr(step, "_on", On, raising=False)
    monkeypatch.setattr(step_module.torch, "empty", watched)
    step.head_backward(1, Head(), None, None, stream="s")
    step.accumulate_microbatch([Layers([None])], stream="s")
    assert entered.count("s") >= 3 and calls.seen is not None


def test_what_ends_a_macro_batch_stays_on_its_stream(monkeypatch):
    """Fills by torch, of the accumulator, the sums of squares and what is allocated for them, are in the order of the calls' stream."""
    inside, outside = [], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            inside.append(self.stream)

        def __exit__(self, *a):
            inside.pop()
    zero, zeros = torch.Tensor.zero_, torch.zeros

    def watched(act):
        def call(*a, **k):
            if inside != ["s"]:
                outside.append(act)
            return act(*a, **k)
        return call
    for name in ("dp_noise_scale_adamw_step_snr", "dp_add_noise_and_scale", "dp_adamw_step", "dp_global_sqnorm", "dp_clip_adamw_step"):
        monkeypatch.setattr(step_module.b, name, lambda *a: None)
    monkeypatch.setattr(step_module.b, "dp_global_norm_workspace_bytes", lambda: 256)
    monkeypatch.setattr(step_module.b, "dp_poll_status", lambda stream: -5 if stream == "s" and failing else 0)
    failing = False
    hyper = dict(C=1.0, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.0)
    steps = [step_module.DPStep(SPECS, "cpu", track_snr=True, **hyper), step_module.DPStep(SPECS, "cpu", **hyper),
             step_module.DPStep(SPECS, "cpu", max_grad_norm=1.0, **hyper)]
    monkeypatch.setattr(step_module.DPStep, "_on", lambda self, stream: On(stream))
    monkeypatch.setattr(torch.Tensor, "zero_", watched(zero))
    monkeypatch.setattr(step_module.torch, "zeros", watched(zeros))
    for step, fused in zip(steps, (True, False, True)):
        step.finish_macro_batch(4, fused=fused, stream="s")
    failing = True
    with pytest.raises(step_module.DeviceStatusError):
        steps[0].finish_macro_batch(4, stream="s")
    assert outside == []


def test_a_microbatch_that_fails_while_its_sums_are_added_spoils_the_macro_batch(monkeypatch):
    """Some of its contributions are in the accumulator: passed again they would be there twice, beyond C."""
    step, calls, emb, fc = make(monkeypatch)
    for name in ("dp_clipped_accumulate_after_sqnorms", "dp_vocab_loss_clipped_accumulate"):
        step.head_backward(2, Head(), None, None)
        calls.fails = name
        with pytest.raises(RuntimeError, match=name):
            step.accumulate_microbatch(Layers([emb, fc]))
        calls.fails = None
        with pytest.raises(RuntimeError, match="discard_macro_batch"):
            step.head_backward(2, Head(), None, None)
        with pytest.raises(RuntimeError, match="discard_macro_batch"):
            step.accumulate_microbatch(Layers([emb, fc]))
        with pytest.raises(RuntimeError, match="discard_macro_batch"):
            step.finish_macro_batch(4, check_status=False)
        assert step.t == 0
        step.discard_macro_batch()
        assert begun_anew(step, calls, Layers([emb, fc])) and step.examples_seen == 4


def test_ranks_discard_a_macro_batch_that_one_of_them_has_spoilt(monkeypatch):
    agreed = []

    class Dist:
        ReduceOp = torch.distributed.ReduceOp

        def get_backend(self):
            return "gloo"

        def all_reduce(self, t, op=None):
            agreed.append(int(t))
    step, calls, emb, fc = make(monkeypatch)
    update = ShardedUpdate(step, Dist(), 1, 0, poll_fn=lambda: 0)
    step.head_backward(2, Head(), None, None)
    calls.fails = "dp_vocab_loss_clipped_accumulate"
    with pytest.raises(RuntimeError):
        step.accumulate_microbatch(Layers([emb, fc]))
    calls.fails = None
    with pytest.raises(step_module.DeviceStatusError):
        update.finish_macro_batch()
    assert agreed and agreed[0] < 0 and step.t == 0
    assert begun_anew(step, calls, Layers([emb, fc]))
