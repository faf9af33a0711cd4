"""Host logic, without a GPU, of DPStep with tensors whose per-example gradients are given (ROWS) and with a global-norm
clip of the noised mean gradient, alone and across ranks."""
import math
import os
import sys

import numpy as np
import pytest
import torch
import torch.multiprocessing as mp

from paper_2108_01624_b200 import binding, synth
from paper_2108_01624_b200 import step as step_mod
from paper_2108_01624_b200.synth import EMBEDDING, LINEAR, ROWS, LayerData, LayerSpec

from .test_parallel_cpu import _free_port

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HP = dict(C=1.0, sigma=1.0, lr=1e-3, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.1)


class _FakeList:
    def __init__(self, entries):
        self.entries, self.B = list(entries), 4

    def __len__(self):
        return len(self.entries)


class _FakeBinding:
    """Records the order of the calls; the lists are stand-ins, since no device is there."""
    DP_OK, DP_PATH_AUTO = 0, 0
    LayerList = RowList = _FakeList
    Layer = binding.Layer

    def __init__(self):
        self.calls = []

    def dp_workspace_bytes(self, ll):
        return 0

    def dp_global_norm_workspace_bytes(self):
        return 256

    def dp_poll_status(self, stream=None):
        return 0

    def __getattr__(self, name):
        def call(*a, **k):
            self.calls.append((name, a, k))
        return call


SPECS = [LayerSpec(LINEAR, 8, 4, True, "fc"), *synth.attention_param_specs(2, 6, 8)]


def make(monkeypatch, specs=SPECS, **kw):
    fake = _FakeBinding()
    monkeypatch.setattr(step_mod, "b", fake)
    return step_mod.DPStep(specs, "cpu", **HP, **kw), fake


def test_rows_specs_and_their_place_in_the_flat_vector(monkeypatch):
    st, _ = make(monkeypatch)
    assert [s.kind for s in SPECS] == [LINEAR, ROWS, ROWS, ROWS]
    assert st.shapes == [[(8, 4), (4,)], [(1, 6)], [(1, 6)], [(8, 2)]]
    assert st.offsets == [[0, 32], [36], [44], [52]] and st.n_flat == 68           # starts at multiples of 4
    assert sum(s.n_params() for s in SPECS) == 36 + 6 + 6 + 16
    data = synth.generate(synth.Workload("w", 4, 3, torch.float32, SPECS), seed=1)
    assert [tuple(d.G.shape) for d in data] == [(4, 3, 4), (4, 1, 6), (4, 1, 6), (4, 8, 2)]
    assert data[1].A is None and data[1].G.dtype == torch.float32
    assert len(st.layer_list(data)) == 1
    rows = st.row_list(data)
    assert len(rows) == 3 and rows.entries[2][1].shape == (8, 2) and rows.entries[2][0] is not None
    assert rows.entries[0][1].data_ptr() == st.acc[36:].data_ptr()
    assert make(monkeypatch, [SPECS[0]])[0].row_list(data[:1]) is None


def test_an_example_norm_never_misses_a_rows_tensor(monkeypatch):
    st, fake = make(monkeypatch)
    layers, rows = _FakeList(["fc"]), _FakeList(["q", "k", "table"])
    for bad in (None, _FakeList(["q", "k"])):
        with pytest.raises(ValueError):
            st.accumulate_microbatch(layers, rows=bad)
    other = _FakeList(["q", "k", "table"])
    other.B = 5
    with pytest.raises(ValueError):
        st.accumulate_microbatch(layers, rows=other)
    assert fake.calls == [] and st.examples_seen == 0
    st.accumulate_microbatch(layers, rows=rows)
    names = [c[0] for c in fake.calls]
    assert names == ["dp_per_example_sqnorms", "dp_rows_sqnorms", "dp_clip_factors", "dp_clipped_accumulate_after_sqnorms",
                     "dp_rows_clipped_accumulate"]
    assert fake.calls[1][1][2] is True and st.examples_seen == 4       # added to the layers' norms
    # a model of rows alone: its norms start the sum
    st, fake = make(monkeypatch, SPECS[1:])
    st.accumulate_microbatch(_FakeList([]), rows=rows)
    assert [c[0] for c in fake.calls] == ["dp_rows_sqnorms", "dp_clip_factors", "dp_rows_clipped_accumulate"]
    assert fake.calls[0][1][2] is False
    # and one without rows refuses them
    st, _ = make(monkeypatch, SPECS[:1])
    with pytest.raises(ValueError):
        st.accumulate_microbatch(layers, rows=rows)


def test_pieces_leave_out_padding_and_aliases(monkeypatch):
    st, _ = make(monkeypatch)
    whole = st.tensor_pieces(st.acc)
    assert [p.numel() for p in whole] == [32, 4, 6, 6, 16]
    got = st.tensor_pieces(st.acc[34:50], 34, 50)                      # a shard that cuts the bias and a gain
    assert [(p.data_ptr() - st.acc.data_ptr()) // 4 for p in got] == [34, 36, 44] and [p.numel() for p in got] == [2, 6, 6]
    assert sum(p.numel() for lo in range(0, 68, 4) for p in st.tensor_pieces(st.acc[lo:lo + 4], lo, lo + 4)) == 64
    tied = [LayerSpec(EMBEDDING, 10, 4, False, "emb"), LayerSpec(LINEAR, 10, 4, False, "out")]
    st, _ = make(monkeypatch, tied, shared_tables={1: 0})
    assert [p.numel() for p in st.tensor_pieces(st.acc)] == [40]


def test_global_clip_comes_between_noise_and_update(monkeypatch):
    st, fake = make(monkeypatch, max_grad_norm=0.5)
    st.examples_seen = 12
    st.finish_macro_batch()
    assert [c[0] for c in fake.calls] == ["dp_add_noise_and_scale", "dp_global_sqnorm", "dp_clip_adamw_step"]
    noise, norm, update = (c[1] for c in fake.calls)
    assert noise[3] == 12 and noise[6] == 0 and len(norm[0]) == 5 and norm[1] is update[5] is st.grad_sqsum
    assert update[4] is True and update[6] == 0.5 and update[-2] == 1 and st.t == 1 and st.examples_seen == 0
    st.grad_sqsum.fill_(9.0)
    assert st.grad_norm() == 3.0
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(ValueError):
            make(monkeypatch, max_grad_norm=bad)
    with pytest.raises(ValueError):
        make(monkeypatch, max_grad_norm=1.0, track_snr=True)
    with pytest.raises(RuntimeError):
        make(monkeypatch)[0].grad_norm()


# ---- across ranks ---------------------------------------------------------------------------------------------------
class _State:
    def __init__(self, n, acc, max_grad_norm):
        self.acc, self.max_grad_norm = acc.clone(), max_grad_norm
        self.theta = torch.linspace(-1, 1, n, dtype=torch.float64)
        self.m, self.v = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
        self.t, self.examples_seen, self.grad_sqsum = 0, 0, None

    def noised_sqnorm(self, acc, elem_offset, batch_size):
        from oracle import dp_oracle as O
        acc.copy_(torch.from_numpy(O.add_noise_and_scale(acc.numpy(), 1.3, 0.5, batch_size, 11, self.t, elem_offset)))
        self.grad_sqsum = acc.square().sum().view(1)
        return self.grad_sqsum

    def clipped_update(self, theta, m, v, acc):
        from oracle import dp_oracle as O
        f = min(1.0, self.max_grad_norm / math.sqrt(float(self.grad_sqsum)))
        new = O.adamw_step(theta.numpy(), m.numpy(), v.numpy(), acc.numpy() * f, 1e-2, 0.9, 0.999, 1e-11, 0.5, self.t)
        for t, x in zip((theta, m, v), new):
            t.copy_(torch.from_numpy(x))
        acc.zero_()


def _local(rank, n):
    return torch.randn(n, generator=torch.Generator().manual_seed(100 + rank), dtype=torch.float64)


def _worker(rank, world, port, n, out_dir):
    sys.path.insert(0, ROOT)
    import torch.distributed as dist
    from paper_2108_01624_b200.parallel import ShardedUpdate
    os.environ["MASTER_ADDR"], os.environ["MASTER_PORT"] = "127.0.0.1", str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    st = _State(n, _local(rank, n), 0.01)
    with pytest.raises(ValueError):
        ShardedUpdate(st, dist, world, rank, poll_fn=lambda: 0, peer_acc=[st.acc] * world, peer_theta=[st.theta] * world)
    sh = ShardedUpdate(st, dist, world, rank, poll_fn=lambda: 0)
    for _ in range(2):
        st.acc.copy_(_local(rank, n))
        st.examples_seen = 64
        sh.finish_macro_batch()
    torch.save({"theta": st.theta, "acc": st.acc, "sq": st.grad_sqsum}, f"{out_dir}/r{rank}.pt")
    dist.destroy_process_group()


@pytest.mark.parametrize("world,n", [(2, 1003), (3, 4)])                # with 4 elements two of three shards are empty
def test_ranks_share_one_factor(world, n, tmp_path):
    mp.spawn(_worker, args=(world, _free_port(), n, str(tmp_path)), nprocs=world, join=True)
    st = _State(n, sum(_local(r, n) for r in range(world)), 0.01)
    for _ in range(2):
        st.t += 1
        acc = sum(_local(r, n) for r in range(world))
        st.noised_sqnorm(acc, 0, 64)
        assert float(st.grad_sqsum) > 0.01 ** 2                        # the clip acts
        st.clipped_update(st.theta, st.m, st.v, acc)
    for r in range(world):
        o = torch.load(f"{tmp_path}/r{r}.pt")
        np.testing.assert_allclose(o["theta"].numpy(), st.theta.numpy(), rtol=1e-12, atol=1e-14)
        assert float(o["sq"]) == pytest.approx(float(st.grad_sqsum), rel=1e-12) and float(o["acc"].abs().max()) == 0.0
