"""Host side, without a GPU, of what the calls for the global norm, rows, relative position bias and query/key norms
promise at their limits: which calls they refuse, and the rules that their kernels' sources keep."""
import ctypes as C
import os
import re

import pytest

from paper_2108_01624_b200 import binding as b
from paper_2108_01624_b200 import build as builder

ARG, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -6


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return b.lib()


def closing(text, at, pair):
    """Index behind the bracket that closes the one at text[at]."""
    depth = 0
    for i in range(at, len(text)):
        depth += (text[i] == pair[0]) - (text[i] == pair[1])
        if depth == 0:
            return i + 1
    raise AssertionError("unbalanced")


def kernels():
    """(file, name, parameters, body) of every kernel of the library, comments left out."""
    for f in sorted(os.listdir(builder.CSRC)):
        if not f.endswith((".cu", ".cuh")):
            continue
        text = re.sub(r"//[^\n]*", "", open(os.path.join(builder.CSRC, f)).read())
        for m in re.finditer(r"__global__\s+void\s+", text):
            at = m.end()
            if text.startswith("__launch_bounds__", at):
                at = closing(text, text.index("(", at), "()")
            name = re.compile(r"\s*(\w+)\s*\(").match(text, at)
            end = closing(text, name.end() - 1, "()")
            body = text.index("{", end)
            yield f, name.group(1), text[name.end():end - 1], text[body:closing(text, body, "{}")]


def test_kernels_that_start_early_promise_nothing_about_their_pointers():
    """A kernel launched with launch_chained starts while its predecessor still writes, so none of its pointers may be
    __restrict__ (for a const one that says the data do not change during the kernel; a load could then move before the wait),
    none of its loads non-coherent, and it waits before anything else."""
    found = list(kernels())
    chained = {name for f in os.listdir(builder.CSRC) if f.endswith(".cu")
               for call in re.findall(r"launch_chained\(([^,]*(?:<[^>]*>[^,]*)*),", open(os.path.join(builder.CSRC, f)).read())
               for name in re.findall(r"\bk_\w+", call)}
    waiting = {name for _, name, _, body in found if "wait_for_predecessor()" in body}
    assert len(found) > 20 and len(waiting) >= 9 and chained == waiting
    for f, name, params, body in found:
        if name in waiting:
            assert "__restrict__" not in params, (f, name)
            assert "__ldg" not in body and ".nc." not in body and "__restrict__" not in body, (f, name)
            before = body[1:body.index("wait_for_predecessor()")]
            assert all(re.match(r"(constexpr|(extern\s+)?__shared__)\b", s.strip()) for s in before.split(";") if s.strip()), (f, name)


# An accepted layout is recognised by the next check's answer: its pointer is off the grid, so that nothing is launched.
def test_a_bias_that_would_overlap_itself_is_refused(lib):
    def bias(sh, sq, H=4, Tq=16, Tk=24):
        return lib.dp_relpos_bias(C.byref(b.dp_relpos(32, 128, 1, H, Tq, Tk, 0)), 4096, 0, 8193, 1, sh, sq, None)
    assert bias(16 * 24, 24) == ALIGN and bias(24, 4 * 24) == ALIGN                  # heads outside, queries outside
    assert bias(1 << 40, 24) == ALIGN and bias(30, 4 * 30) == ALIGN and bias(16 * 24 + 5, 24) == ALIGN      # with gaps
    assert bias(16 * 30 - 6, 30) == ALIGN                                            # no gap behind a head's last row
    for sh, sq in ((0, 24), (23, 4 * 24), (24, 24), (16 * 24 - 1, 24), (24, 4 * 24 - 1), (96, 24), (0, 1 << 40)):
        assert bias(sh, sq) == ARG, (sh, sq)
    assert bias(0, 24, H=1) == ALIGN and bias(24, 24, Tq=1) == ALIGN                 # the stride of an extent of one


def test_heads_that_would_overlap_themselves_are_refused(lib):
    B, T, H, D = 2, 8, 4, 64

    def heads(ptr, sb, st, sh):
        return C.byref(b.dp_heads(ptr, sb, st, sh))
    good = heads(4096, T * H * D, H * D, D)

    def p(B=B, T=T, H=H):
        return C.byref(b.dp_qknorm(1, B, T, H, 0, D, 0, 0, 1e-6, None, None, None, None, None))

    def fwd(strides, x=good, **k):
        return lib.dp_qknorm_rope(p(**k), x, None, heads(8193, *strides), None, None)

    def bwd(strides, x=good, g=good, **k):
        return lib.dp_qknorm_rope_backward(p(**k), x, None, g, None, heads(8193, *strides), None, None, None, 0, None, 0, None)
    for call in (fwd, bwd):
        for strides in ((T * H * D, H * D, D), (T * H * D, D, T * D), (D, B * H * D, B * D), (3 * T * H * D, 3 * H * D, 3 * D),
                        (T * (H * D + 1), H * D + 1, D), (1 << 50, 1 << 30, 1 << 20)):
            assert call(strides) == ALIGN, strides
        for strides in ((0, H * D, D), (T * H * D, 0, D), (T * H * D, H * D, 0), (0, 0, 0), (T * H * D, H * D, D - 1),
                        (T * H * D, H * D - 1, D), (T * H * D - 1, H * D, D), (H * D, H * D, D), (D, H * D, D)):
            assert call(strides) == ARG, strides
        assert call((0, H * D, D), B=1) == ALIGN and call((H * D, 0, D), T=1) == ALIGN and call((T * D, D, 0), H=1) == ALIGN
        # inputs may be read several times
        wide = heads(4096, 0, 0, 0)
        assert call((T * H * D, H * D, D), x=wide) == ALIGN
    assert bwd((T * H * D, H * D, D), g=heads(4096, 0, H * D, 0)) == ALIGN


# ---- what the module was built for --------------------------------------------------------------------------------
def test_a_module_built_for_another_torch_is_rebuilt_and_never_loaded(lib, monkeypatch, tmp_path):
    import torch
    assert not builder.needs_module() and b._native().built_for == builder.module_key()
    assert torch.__version__ in builder.module_key()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0.1+other")
        assert builder.needs_module() and builder.needs_build() and not builder.needs_library()
        m.setattr(b, "_module", None)
        with pytest.raises(ImportError, match="another torch"):
            b.dp_relpos_workspace_bytes(torch.empty(1, 1, 4, 4), 32)
        assert b._module is None
    # the commands that build count as sources
    with monkeypatch.context() as m:
        later = tmp_path / "build.py"
        later.write_text("")
        os.utime(later, (1 << 33, 1 << 33))
        m.setattr(builder, "__file__", str(later))
        assert builder.needs_library() and builder.needs_module()


def test_the_library_is_built_where_the_module_cannot_be(lib, monkeypatch, tmp_path):
    """The C ABI and the calls bound by ctypes need neither Python's headers nor torch's."""
    import torch
    module = tmp_path / "_dp_tensors.so"
    module.write_bytes(b"left by an earlier build, of other sources")
    monkeypatch.setattr(builder, "MODULE", str(module))
    monkeypatch.setenv("CXX", str(tmp_path / "no compiler"))
    with pytest.warns(RuntimeWarning, match="_dp_tensors"):
        assert builder.build() == builder.LIB
    assert not module.exists()                                        # nothing that does not fit the library is left
    with pytest.raises(RuntimeError):                                 # asked for by itself it fails
        builder.build_module()
    monkeypatch.setattr(b, "MODULE_PATH", str(module))
    monkeypatch.setattr(b, "_module", None)
    with pytest.raises(ImportError):
        b.dp_relpos_workspace_bytes(torch.empty(1, 1, 4, 4), 32)
    assert b.dp_version() >= 100


# ---- the clip of a macro-batch across ranks -------------------------------------------------------------------------
class _OneRankOfMany:
    """Collectives as a rank sees them whose peers add nothing."""
    class ReduceOp:
        MIN = "min"

    def get_backend(self):
        return "gloo"

    def all_reduce(self, t, op=None):
        pass

    def all_gather(self, out, mine):
        pass


def test_a_rank_whose_shard_was_empty_can_finish_a_macro_batch_alone(monkeypatch):
    from paper_2108_01624_b200.parallel import ShardedUpdate
    from paper_2108_01624_b200.synth import LINEAR, LayerSpec

    from .test_step_rows_cpu import make
    st, fake = make(monkeypatch, [LayerSpec(LINEAR, 2, 2, False, "fc")], shard_world=3, max_grad_norm=0.5)
    sharded = ShardedUpdate(st, _OneRankOfMany(), 3, 2, poll_fn=lambda: 0)
    assert sharded.lo == sharded.hi
    st.examples_seen = 8
    sharded.finish_macro_batch()                                       # nothing of its own to sum or update
    assert fake.calls == [] and float(st.grad_sqsum) == 0.0
    st.examples_seen = 8
    st.finish_macro_batch()                                            # the job goes on with one rank
    norm = [a for name, a, _ in fake.calls if name == "dp_global_sqnorm"]
    assert len(norm) == 1 and norm[0][1] is st.grad_sqsum and norm[0][3] is not None


# ---- eps ----------------------------------------------------------------------------------------------------------
def test_an_eps_that_fp32_cannot_hold_is_refused(lib):
    """The kernels add eps in fp32: one that is lost there would turn a head of zeros into NaN, one beyond it any head into 0."""
    h = C.byref(b.dp_heads(4096, 8 * 4 * 64, 4 * 64, 64))
    off = C.byref(b.dp_heads(8193, 8 * 4 * 64, 4 * 64, 64))            # misaligned: the call ends before a launch

    def call(eps):
        p = C.byref(b.dp_qknorm(1, 2, 8, 4, 0, 64, 0, 0, eps, None, None, None, None, None))
        a = lib.dp_qknorm_rope(p, h, None, off, None, None)
        z = lib.dp_qknorm_rope_backward(p, h, None, h, None, off, None, None, None, 0, None, 0, None)
        assert a == z
        return a
    for eps in (0.0, 1e-6, 1.0, 2.0 ** -126, 3e38):
        assert call(eps) == ALIGN, eps
    for eps in (1e-39, 1e-50, 5e-324, 1e39, float("inf"), -1e-6, float("nan")):
        assert call(eps) == ARG, eps
