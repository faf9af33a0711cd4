"""GPU: the calls on small tensors as programs use them side by side -- streams with workspaces of their own, long inputs
that split into many units, extents of one with odd strides, a data-parallel end of a macro-batch with the global clip."""
import os

import pytest
import torch

from paper_2108_01624_b200 import DPStep, synth
from paper_2108_01624_b200 import binding as b
from paper_2108_01624_b200.synth import LINEAR, LayerSpec

from .test_attention_params_gpu import (BF16, DEV, F32, HALF, NONE, QK_REL, bucket_map, gen, randn, relpos_rows, rotate64, within)
from .test_parallel_cpu import _free_port

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)


def work(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_scores_of_one_example(dtype):
    """Many tiles per head, causal and cut by both lengths inside a tile."""
    g = gen(1)
    T = 2300
    G = randn(g, 1, 1, T, T, dtype=dtype)
    ql, kl = (torch.tensor([n], dtype=torch.int32, device=DEV) for n in (2111, 1999))
    for causal in (False, True):
        ref, mag = relpos_rows(G, 32, 128, True, 0, causal, ql, kl)
        rows = torch.empty(1, 32, 1, device=DEV)
        b.dp_relpos_bias_grad(G, rows, causal=causal, q_len=ql, k_len=kl, workspace=work(b.dp_relpos_workspace_bytes(G, 32)))
        within(rows, ref, mag * (32 + 130 + 600) * HALF[F32])          # a strand's rows, a tile's diagonals, the tiles


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,hq,hk,D", [(1, 5000, 2, 1, 64), (2, 3, 200, 1, 32), (70, 2, 1, 1, 128)])
def test_backward_over_many_units(dtype, B, T, hq, hk, D):
    g = gen(2)
    q, k = randn(g, B, T, hq, D, dtype=dtype), randn(g, B, T, hk, D, dtype=dtype)
    dq, dk = randn(g, B, T, hq, D, dtype=dtype), randn(g, B, T, hk, D, dtype=dtype)
    gain, freq = 1 + 0.1 * randn(g, D), b.rope_frequencies(D)
    pos = torch.arange(T, device=DEV).expand(B, T)
    oq, ok, rq, rk = torch.empty_like(q), torch.empty_like(k), torch.empty(B, D, device=DEV), torch.empty(B, D, device=DEV)
    b.dp_qknorm_rope_backward(q, k, dq, dk, oq, ok, gain, gain, rq, rk, 1e-6, freq, workspace=work(b.dp_qknorm_workspace_bytes(q, k)))
    for x, dy, rows in ((q, dq, rq), (k, dk, rk)):
        xd = x.double()
        hat = xd * (xd.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        u = rotate64(dy.double(), pos, freq, False, -1.0)
        length = torch.linalg.vector_norm(torch.stack([u[..., :D // 2], u[..., D // 2:]]), dim=0).repeat(1, 1, 1, 2)
        terms = (length * hat.abs()).sum((1, 2))
        within(rows, (u * hat).sum((1, 2)), terms * (2 * QK_REL + 600 * HALF[F32]))
    # heads of one token in place of an extent of one: strides that nothing depends on may be odd
    if B == 1:
        one = q.as_strided((1, T, hq, D), (12345, hq * D, D, 1))
        o1, o2 = torch.empty_like(q), torch.empty_like(q)
        b.dp_qknorm_rope(q, None, o1, None, gain, None, 1e-6, freq)
        b.dp_qknorm_rope(one, None, o2, None, gain, None, 1e-6, freq)
        assert torch.equal(o1, o2)


def test_forward_skips_padding_of_single_tokens():
    """Tokens of all examples share warps; those behind an example's length stay as they were."""
    g = gen(3)
    B, H, D = 37, 5, 64
    lengths = (torch.arange(B, device=DEV) % 3 > 0).to(torch.int32)
    x = randn(g, B, 1, H, D, dtype=BF16)
    out = torch.full_like(x, 4.0)
    pos = torch.randint(0, 1 << 20, (B, 1), generator=g, device=DEV, dtype=torch.int32)
    freq = b.rope_frequencies(D)
    b.dp_qknorm_rope(x, None, out, None, None, None, 1e-6, freq, pos, lengths)
    xd = x.double()
    ref = rotate64(xd * (xd.square().mean(-1, keepdim=True) + 1e-6).rsqrt(), pos, freq, False)
    assert bool((out[lengths == 0] == 4).all())
    keep = lengths > 0
    within(out[keep], ref[keep], ref[keep].abs() * HALF[BF16] * 1.001 + 4 * QK_REL * 3)      # a pair is shorter than 4


def test_two_streams_with_workspaces_of_their_own():
    g = gen(4)
    B, H, T, D, nb = 5, 3, 300, 64, 32
    data = []
    for _ in range(2):
        G, x, dy = randn(g, B, H, T, T, dtype=BF16), randn(g, B, T, H, D, dtype=BF16), randn(g, B, T, H, D, dtype=BF16)
        data.append(dict(G=G, x=x, dy=dy, t=[randn(g, 100003), randn(g, 77)], rows=torch.empty(B, nb, H, device=DEV),
                         dx=torch.empty_like(x), gr=torch.empty(B, D, device=DEV),
                         sq=torch.empty(1, dtype=torch.float64, device=DEV), w1=work(b.dp_relpos_workspace_bytes(G, nb)),
                         w2=work(b.dp_qknorm_workspace_bytes(x, None)), w3=work(b.dp_global_norm_workspace_bytes())))
    freq = b.rope_frequencies(D)

    def chain(d, stream=None):
        b.dp_relpos_bias_grad(d["G"], d["rows"], workspace=d["w1"], stream=stream)
        b.dp_qknorm_rope_backward(d["x"], None, d["dy"], None, d["dx"], None, None, None, d["gr"], None, 1e-6, freq,
                                  workspace=d["w2"], stream=stream)
        b.dp_global_sqnorm(d["t"], d["sq"], False, d["w3"], stream)
    want = []
    for d in data:
        chain(d)
        want.append([d[k].clone() for k in ("rows", "dx", "gr", "sq")])
        for k in ("rows", "dx", "gr", "sq"):
            d[k].zero_()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for d, s in zip(data, streams):
            chain(d, s)
    torch.cuda.synchronize()
    for d, w in zip(data, want):
        assert all(torch.equal(d[k], v) for k, v in zip(("rows", "dx", "gr", "sq"), w))


def test_gradient_of_shared_scores_views():
    """One gradient of the scores given for every head and example through strides of 0 (a bias broadcast over both)."""
    g = gen(5)
    one = randn(g, 1, 1, 64, 96)
    G = one.expand(3, 4, 64, 96)
    rows = torch.empty(3, 32, 4, device=DEV)
    b.dp_relpos_bias_grad(G, rows, workspace=work(b.dp_relpos_workspace_bytes(G, 32)))
    assert torch.equal(rows, rows[:1, :, :1].expand(3, 32, 4))
    bucket, _ = bucket_map(32, 128, True, 64, 96, 0)
    ref = torch.zeros(32, dtype=torch.float64, device=DEV).index_add_(0, bucket.reshape(-1), one.double().reshape(-1))
    mag = torch.zeros(32, dtype=torch.float64, device=DEV).index_add_(0, bucket.reshape(-1), one.double().abs().reshape(-1))
    within(rows[0, :, 0], ref, mag * 200 * HALF[F32])
    assert NONE.numel() == 0


def test_sharded_end_with_the_global_clip_equals_the_single_one(tmp_path):
    """ShardedUpdate's default functions over the library's kernels, in a process group of one."""
    import torch.distributed as dist

    from paper_2108_01624_b200.parallel import ShardedUpdate
    os.environ["MASTER_ADDR"], os.environ["MASTER_PORT"] = "127.0.0.1", str(_free_port())
    dist.init_process_group("gloo", rank=0, world_size=1)
    try:
        specs = [LayerSpec(LINEAR, 33, 21, True, "fc")] + synth.attention_param_specs(3, 10, 16)
        steps = [DPStep(specs, DEV, C=1.0, sigma=0.7, lr=1e-2, beta1=0.9, beta2=0.999, xi=1e-11, weight_decay=0.1, seed=4,
                        max_grad_norm=1e-2) for _ in range(2)]
        acc = randn(gen(6), steps[0].n_flat)
        sharded = ShardedUpdate(steps[1], dist, 1, 0)
        for t in range(2):
            for st in steps:
                st.acc.copy_(acc * (t + 1))
                st.examples_seen = 64
            steps[0].finish_macro_batch()
            sharded.finish_macro_batch()
            assert steps[0].grad_norm() > 1e-2 and steps[0].grad_norm() == steps[1].grad_norm()
            for name in ("theta", "m", "v", "acc"):
                assert torch.equal(getattr(steps[0], name), getattr(steps[1], name)), name
        assert float(steps[1].acc.abs().max()) == 0.0 and float(steps[1].theta.abs().max()) > 0
    finally:
        dist.destroy_process_group()


def test_captured_calls_behind_copies_and_fills():
    """The calls' kernels may be set up before their predecessors end: behind copies, fills and torch's own kernels, eager
    and in a replayed graph, they still see what those wrote."""
    g = gen(7)
    B, P, n = 64, 512, 3_000_000
    src, grad, clip = randn(g, P), randn(g, B, P), torch.rand(B, generator=g, device=DEV)
    acc, sq, total = torch.empty(P, device=DEV), torch.empty(B, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
    big, out, t = randn(g, n), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    x, y = randn(g, 32, 64, 8, 64, dtype=BF16), torch.empty(32, 64, 8, 64, dtype=BF16, device=DEV)
    w, freq = work(b.dp_global_norm_workspace_bytes()), b.rope_frequencies(64)
    rl = b.RowList([(grad, acc)])

    def chain():
        acc.copy_(src)                                                 # a copy, then the call that adds to it
        b.dp_rows_clipped_accumulate(rl, clip)
        sq.zero_()
        b.dp_rows_sqnorms(rl, sq, True)
        t.copy_(big)
        t.mul_(2.0)                                                    # a kernel of torch's, then the norm of what it wrote
        b.dp_global_sqnorm([t], total, False, w)
        b.dp_clip_by_global_norm([t], [out], total, 1.0)
        y.zero_()
        b.dp_qknorm_rope(x, None, y, None, None, None, 1e-6, freq)
        y.add_(1.0)

    def check():
        terms = grad.double() * clip.double()[:, None]
        within(acc, src.double() + terms.sum(0), (terms.abs().sum(0) + src.double().abs()) * 40 * HALF[F32])
        ref = grad.double().square().sum(1)
        within(sq, ref, ref * 40 * HALF[F32])
        norm2 = float((big.double() * 2).square().sum())
        assert float(total) == pytest.approx(norm2, rel=34 * 2.0 ** -24)
        want = big.double() * 2 / norm2 ** 0.5
        within(out, want, want.abs() * 40 * HALF[F32])
        z = torch.empty_like(y)
        b.dp_qknorm_rope(x, None, z, None, None, None, 1e-6, freq)
        torch.cuda.synchronize()
        assert torch.equal(y, z + 1.0)
    for _ in range(20):
        chain()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for seed in range(3):
        h = gen(70 + seed)
        src.copy_(randn(h, P)), grad.copy_(randn(h, B, P)), big.copy_(randn(h, n)), x.copy_(randn(h, 32, 64, 8, 64, dtype=BF16))
        for _ in range(10):
            graph.replay()
        check()
