"""Host side of the calls for the global norm, per-example rows, the relative position bias and the query/key norms:
struct layouts, bucket borders, refusals before any launch.  No GPU."""
import ctypes as C

import pytest
import torch

from paper_2108_01624_b200 import binding as b
from paper_2108_01624_b200 import build as builder

ARG, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -6


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return b.lib()


def test_struct_layouts():
    assert C.sizeof(b.dp_rows) == 24 and b.dp_rows.width.offset == 16
    assert C.sizeof(b.dp_relpos) == 32 and b.dp_relpos.offset.offset == 24
    assert C.sizeof(b.dp_qknorm) == 8 * 4 + 8 + 5 * 8 and b.dp_qknorm.inv_freq.offset == 72
    assert C.sizeof(b.dp_heads) == 32


def whole_number_starts(num_buckets, max_distance, both):
    """Bucket borders from the definition, in Python's whole numbers."""
    half = num_buckets // 2 if both else num_buckets
    exact = half // 2
    rest = half - exact
    starts = list(range(exact + 1))
    for j in range(1, rest):
        lo, hi = 1, max_distance
        while lo < hi:                                   # smallest n with (n / exact)^rest >= (distance / exact)^j
            mid = (lo + hi) // 2
            if mid ** rest * exact ** j >= max_distance ** j * exact ** rest:
                hi = mid
            else:
                lo = mid + 1
        starts.append(lo)
    return starts[:half]


@pytest.mark.parametrize("both", [False, True])
def test_bucket_borders_are_exact(lib, both):
    for half in list(range(2, 41)) + [64, 97, 128]:
        for distance in {half // 2 + 1, half, half + 1, 2 * half, 64, 100, 128, 129, 256, 1000, 4096, 46341, 1 << 24}:
            if distance <= half // 2:
                continue
            nb = 2 * half if both else half
            assert b.dp_relpos_bucket_starts(nb, distance, both) == whole_number_starts(nb, distance, both), (nb, distance)
    # the classic 32 buckets over 128 positions: borders that are whole powers of two exactly
    assert b.dp_relpos_bucket_starts(32, 128, True) == [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]


def test_bucket_arguments_are_refused(lib):
    out = (C.c_int32 * 256)()
    call = lambda *a: lib.dp_relpos_bucket_starts(*a, C.cast(out, C.c_void_p))  # noqa: E731
    assert call(32, 128, 1) == 0
    assert call(1, 128, 0) == ARG and call(257, 128, 0) == ARG        # too few, too many
    assert call(33, 128, 1) == ARG                                    # odd, both sides
    assert call(2, 128, 1) == ARG                                     # one bucket a side
    assert call(32, 8, 1) == ARG and call(32, 9, 1) == 0              # the log part needs room
    assert call(32, 0, 0) == ARG and call(32, (1 << 24) + 1, 0) == ARG
    assert lib.dp_relpos_bucket_starts(32, 128, 1, None) == ARG


def test_global_norm_refusals(lib):
    n = int(lib.dp_global_norm_workspace_bytes())
    assert n == 65536
    ptrs, sizes = (C.c_void_p * 2)(4096, 8192), (C.c_int64 * 2)(4, 4)
    call = lambda p=ptrs, s=sizes, k=2, dt=0, out=256, ws=256, wn=n: lib.dp_global_sqnorm(  # noqa: E731
        p, s, k, dt, 0, out, ws, wn, None)
    assert call(p=None) == ARG and call(s=None) == ARG and call(k=-1) == ARG and call(dt=2) == ARG
    assert call(out=None) == ARG and call(out=260) == ALIGN
    assert call(ws=None) == WORKSPACE and call(wn=n - 1) == WORKSPACE and call(ws=128) == WORKSPACE
    assert call(p=(C.c_void_p * 2)(4096, None)) == ARG
    assert call(p=(C.c_void_p * 2)(4096, 8194)) == ALIGN              # fp32
    assert call(s=(C.c_int64 * 2)(4, -1)) == ARG
    clip = lambda p=ptrs, o=ptrs, s=sizes, sq=256, m=1.0, told=None: lib.dp_clip_by_global_norm(  # noqa: E731
        p, o, s, 2, 0, sq, m, told, None)
    assert clip(o=None) == ARG and clip(sq=None) == ARG and clip(sq=260) == ALIGN and clip(told=258) == ALIGN
    assert clip(m=0.0) == ARG and clip(m=-1.0) == ARG and clip(m=float("nan")) == ARG and clip(m=float("inf")) == ARG
    assert clip(o=(C.c_void_p * 2)(4096, None)) == ARG and clip(o=(C.c_void_p * 2)(4096, 8193)) == ALIGN
    step = lambda th=256, n=8, sq=256, m=1.0, lr=1e-3, t=1: lib.dp_clip_adamw_step(  # noqa: E731
        th, 512, 768, 1024, 0, n, sq, m, lr, 0.9, 0.999, 1e-11, 0.0, t, None)
    assert step(th=None) == ARG and step(n=-1) == ARG and step(sq=None) == ARG and step(m=0.0) == ARG
    assert step(t=0) == ARG and step(lr=float("nan")) == ARG and step(th=258) == ALIGN and step(sq=260) == ALIGN
    assert step(n=0) == 0


def test_rows_refusals(lib):
    r = (b.dp_rows * 2)()
    for k in range(2):
        r[k].grad, r[k].acc, r[k].width = 4096, 8192, 16
    p = C.cast(r, C.c_void_p)
    assert lib.dp_rows_sqnorms(None, 2, 4, 256, 0, None) == ARG
    assert lib.dp_rows_sqnorms(p, 0, 4, 256, 0, None) == ARG and lib.dp_rows_sqnorms(p, 2, 0, 256, 0, None) == ARG
    assert lib.dp_rows_sqnorms(p, 2, 4, None, 0, None) == ARG and lib.dp_rows_sqnorms(p, 2, 4, 258, 0, None) == ALIGN
    assert lib.dp_rows_clipped_accumulate(p, 2, 4, None, None) == ARG
    assert lib.dp_rows_clipped_accumulate(p, 2, 4, 258, None) == ALIGN
    r[1].acc = None
    assert lib.dp_rows_clipped_accumulate(p, 2, 4, 256, None) == ARG
    r[1].acc, r[1].width = 8192, 0
    assert lib.dp_rows_sqnorms(p, 2, 4, 256, 0, None) == ARG
    r[1].width, r[1].grad = 16, 4098
    assert lib.dp_rows_sqnorms(p, 2, 4, 256, 0, None) == ALIGN
    r[1].grad = None
    assert lib.dp_rows_sqnorms(p, 2, 4, 256, 0, None) == ARG


def test_relpos_refusals(lib):
    def p(nb=32, dist=128, both=1, H=4, Tq=512, Tk=512, off=0):
        return C.byref(b.dp_relpos(nb, dist, both, H, Tq, Tk, off))
    fwd = lambda q=p(), table=4096, td=0, out=8192, od=1, sh=512 * 512, sq=512: lib.dp_relpos_bias(  # noqa: E731
        q, table, td, out, od, sh, sq, None)
    assert fwd(q=None) == ARG and fwd(table=None) == ARG and fwd(out=None) == ARG
    assert fwd(td=2) == ARG and fwd(od=-1) == ARG and fwd(sq=511) == ARG and fwd(sh=-1) == ARG
    assert fwd(table=4098) == ALIGN and fwd(out=8193) == ALIGN
    for bad in (p(nb=31), p(dist=4), p(H=0), p(Tq=0), p(Tk=0), p(Tk=(1 << 24) + 1), p(off=1 << 40), p(off=-(1 << 40))):
        assert fwd(q=bad) == ARG
        assert lib.dp_relpos_workspace_bytes(bad, 4) == 0
    assert fwd(q=p(H=70000)) == UNSUPPORTED
    grad = lambda q=p(), B=2, G=4096, dt=1, s=(4 << 18, 1 << 18, 512), ql=None, rows=8192, ws=None, wn=0: (  # noqa: E731
        lib.dp_relpos_bias_grad(q, B, 0, G, dt, *s, ql, None, rows, 0, ws, wn, None))
    assert grad(q=None) == ARG and grad(B=0) == ARG and grad(G=None) == ARG and grad(rows=None) == ARG and grad(dt=2) == ARG
    assert grad(s=(-1, 0, 0)) == ARG and grad(G=4097) == ALIGN and grad(rows=8194) == ALIGN and grad(ql=258) == ALIGN
    need = lib.dp_relpos_workspace_bytes(p(), 2)
    assert need > 0 and grad() == WORKSPACE                           # several units per head: partial sums
    assert grad(ws=256, wn=64) == WORKSPACE and grad(ws=128, wn=need) == WORKSPACE


def test_qknorm_refusals(lib):
    freq = (C.c_double * 32)(*[0.5] * 32)
    nan = (C.c_double * 32)(*[float("nan")] * 32)

    def p(dtype=1, B=2, T=8, n_q=4, n_k=2, dim=64, rot=64, eps=1e-6, gain=None, f=freq):
        return C.byref(b.dp_qknorm(dtype, B, T, n_q, n_k, dim, rot, 0, eps, gain, None, None, None,
                                   C.cast(f, C.c_void_p) if f is not None else None))
    h = lambda ptr=4096, s=64: C.byref(b.dp_heads(ptr, 8 * 4 * s, 4 * s, s))  # noqa: E731
    fwd = lambda q=p(), x=h(), y=h(), ox=h(), oy=h(): lib.dp_qknorm_rope(q, x, y, ox, oy, None)  # noqa: E731
    for bad in (None, p(dtype=2), p(B=0), p(T=0), p(n_q=-1), p(n_q=0, n_k=0), p(dim=0), p(dim=63), p(rot=66), p(rot=-2),
                p(rot=3), p(eps=-1.0), p(eps=float("nan")), p(f=None), p(f=nan)):
        assert fwd(q=bad) == ARG
        assert lib.dp_qknorm_workspace_bytes(bad) == 0
    assert fwd(q=p(dim=514, rot=0)) == UNSUPPORTED and fwd(q=p(T=(1 << 24) + 1)) == UNSUPPORTED
    assert fwd(q=p(gain=258)) == ALIGN
    assert fwd(x=None) == ARG and fwd(oy=None) == ARG and fwd(x=h(None)) == ARG and fwd(x=h(4096, -1)) == ARG
    assert fwd(x=h(4097)) == ALIGN
    bwd = lambda q=p(), g=h(), rq=8192, ws=None, wn=0: lib.dp_qknorm_rope_backward(  # noqa: E731
        q, h(), h(), g, h(), h(), h(), rq, None, 0, ws, wn, None)
    assert bwd(q=p(dim=63)) == ARG and bwd(g=None) == ARG and bwd(rq=8194) == ALIGN
    need = lib.dp_qknorm_workspace_bytes(p())
    assert need > 0 and bwd() == WORKSPACE and bwd(ws=256, wn=need - 1) == WORKSPACE and bwd(ws=128, wn=need) == WORKSPACE


def test_binding_checks_tensors_before_the_library_is_called(lib):
    x = torch.zeros(2, 3, 4, 8)
    with pytest.raises(ValueError):
        b.dp_global_sqnorm([torch.zeros(4)], torch.zeros(1, dtype=torch.float64))           # host tensors
    with pytest.raises(ValueError):
        b.dp_clip_by_global_norm([], None, torch.zeros(1, dtype=torch.float64), 1.0)
    with pytest.raises(ValueError):
        b.RowList([])
    with pytest.raises(ValueError):
        b.RowList([(torch.zeros(2, 3), None)])                                              # host tensors
    with pytest.raises(ValueError):
        b.dp_relpos_bias_grad(x, torch.zeros(2, 32, 3))
    with pytest.raises(ValueError):
        b.dp_qknorm_rope(x, None, x, None, None, None, 1e-6, None)
    with pytest.raises(ValueError):
        b.dp_qknorm_rope(None, None, None, None, None, None, 1e-6, None)


def test_rope_frequencies():
    f = b.rope_frequencies(8, 10000.0)
    assert f.dtype == torch.float64
    torch.testing.assert_close(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14, atol=0)
    assert b.rope_frequencies(0).numel() == 0


def test_missing_module_fails_loudly(lib, monkeypatch, tmp_path):
    monkeypatch.setattr(b, "_module", None)
    monkeypatch.setattr(b, "MODULE_PATH", str(tmp_path / "nope.so"))
    with pytest.raises(ImportError):
        b.RowList([(torch.zeros(2, 3), None)])


def test_module_refuses_what_is_no_tensor_or_number(lib):
    with pytest.raises(ValueError):
        b.dp_global_sqnorm([1.0], torch.zeros(1, dtype=torch.float64))
    with pytest.raises(TypeError):
        b.dp_global_sqnorm(3, torch.zeros(1, dtype=torch.float64))
    with pytest.raises(ValueError):
        b.RowList([torch.zeros(2, 3)])
    with pytest.raises(TypeError):
        b._native().global_sqnorm(1)
    with pytest.raises(TypeError):
        b._native().bind(1)
    with pytest.raises(ValueError):
        b.dp_relpos_workspace_bytes(torch.zeros(2, 3), 32)
    assert b.dp_relpos_workspace_bytes(torch.empty(2, 4, 512, 512), 32) >= 256          # host arithmetic: any device
