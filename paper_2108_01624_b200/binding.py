"""ctypes binding of libdp_b200.so: the same entry points as include/dp.h, taking torch tensors.

Argument marshalling only -- every step runs in the library's CUDA kernels.  There is no CPU or
PyTorch fallback: if the shared library is missing or a call fails, an exception is raised.  The calls for small
tensors marshal through a CPython module (_dp_tensors.so) instead of ctypes.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# DP_B200_LIB selects another build of the library (e.g. one compiled with experimental -D flags).
LIB_PATH = os.environ.get("DP_B200_LIB") or os.path.join(_HERE, "libdp_b200.so")

DP_OK = 0
DP_LINEAR, DP_LAYERNORM, DP_EMBEDDING = 0, 1, 2
DP_F32, DP_BF16 = 0, 1
DP_PATH_AUTO, DP_PATH_GRAM, DP_PATH_MATERIALIZED = 0, 1, 2
_KINDS = {"linear": DP_LINEAR, "layernorm": DP_LAYERNORM, "embedding": DP_EMBEDDING}

EXPORTS = ["dp_workspace_bytes", "dp_per_example_sqnorms", "dp_clip_factors", "dp_clipped_accumulate", "dp_clipped_accumulate_after_sqnorms", "dp_accumulate_schedule", "dp_reduce_noise_adamw_step",
           "dp_add_noise_and_scale", "dp_adamw_step", "dp_noise_scale_adamw_step", "dp_noise_scale_adamw_step_snr",
           "dp_clip_stats", "dp_philox_u32", "dp_shared_table_cross_sqnorms",
           "dp_token_equality_mask", "dp_layernorm_sqnorms_static", "dp_poll_status", "dp_last_timeout_info", "dp_launch_count",
           "dp_set_wait_limit_cycles", "dp_selftest_wait_timeout",
           "dp_status_string", "dp_version",
           "dp_global_norm_workspace_bytes", "dp_global_sqnorm", "dp_clip_by_global_norm", "dp_clip_adamw_step",
           "dp_rows_sqnorms", "dp_rows_clipped_accumulate",
           "dp_relpos_bucket_starts", "dp_relpos_bias", "dp_relpos_workspace_bytes", "dp_relpos_bias_grad",
           "dp_qknorm_rope", "dp_qknorm_workspace_bytes", "dp_qknorm_rope_backward",
           "dp_vocab_workspace_bytes", "dp_vocab_loss", "dp_vocab_loss_backward", "dp_vocab_loss_clipped_accumulate",
           "dp_vocab_loss_cross_sqnorms", "dp_distill_loss"]


class dp_layer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("dtype", C.c_int32), ("path", C.c_int32), ("has_bias", C.c_int32),
                ("B", C.c_int32), ("T", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32),
                ("A", C.c_void_p), ("ids", C.c_void_p), ("G", C.c_void_p),
                ("acc_w", C.c_void_p), ("acc_b", C.c_void_p)]


class dp_rows(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("acc", C.c_void_p), ("width", C.c_int64)]


class dp_relpos(C.Structure):
    _fields_ = [("num_buckets", C.c_int32), ("max_distance", C.c_int32), ("bidirectional", C.c_int32),
                ("n_heads", C.c_int32), ("Tq", C.c_int32), ("Tk", C.c_int32), ("offset", C.c_int64)]


class dp_qknorm(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("T", C.c_int32), ("n_q", C.c_int32), ("n_k", C.c_int32),
                ("dim", C.c_int32), ("rot", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_double),
                ("gain_q", C.c_void_p), ("gain_k", C.c_void_p), ("positions", C.c_void_p), ("lengths", C.c_void_p),
                ("inv_freq", C.c_void_p)]


class dp_heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_b", C.c_int64), ("stride_t", C.c_int64), ("stride_h", C.c_int64)]


class dp_vocab_head(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("T", C.c_int32), ("d", C.c_int32), ("V", C.c_int32),
                ("X", C.c_void_p), ("ldx", C.c_int64), ("W", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p),
                ("labels", C.c_void_p), ("weights", C.c_void_p)]


class dp_distill(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("teacher_dtype", C.c_int32), ("N", C.c_int32), ("V", C.c_int32), ("K", C.c_int32),
                ("temperature", C.c_double), ("logits", C.c_void_p), ("ld", C.c_int64), ("top_ids", C.c_void_p),
                ("top_logits", C.c_void_p), ("weights", C.c_void_p)]


class DpError(RuntimeError):
    def __init__(self, fn: str, code: int):
        self.code = code
        super().__init__(f"{fn} failed: {code} ({status_string(code)})")


_lib = None


def lib() -> C.CDLL:
    """Load the shared library (built by paper_2108_01624_b200.build); fails loudly when absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found: run `python -m paper_2108_01624_b200.build` (needs nvcc). "
                              "There is no fallback implementation.")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64, f32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_uint64, C.c_double, C.c_size_t
        L.dp_workspace_bytes.restype = sz
        L.dp_workspace_bytes.argtypes = [vp, i32]
        L.dp_per_example_sqnorms.argtypes = [vp, i32, vp, i32, vp, sz, vp]
        L.dp_clip_factors.argtypes = [vp, i32, f32, vp, vp]
        L.dp_clipped_accumulate.argtypes = [vp, i32, vp, vp, sz, vp]
        L.dp_clipped_accumulate_after_sqnorms.argtypes = [vp, i32, vp, vp, sz, vp]
        L.dp_accumulate_schedule.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32]
        L.dp_add_noise_and_scale.argtypes = [vp, i64, i64, f32, f32, i64, u64, u64, vp]
        L.dp_adamw_step.argtypes = [vp, vp, vp, vp, i64, f32, f32, f32, f32, f32, i64, vp]
        L.dp_noise_scale_adamw_step.argtypes = [vp, vp, vp, vp, i32, i64, i64, f32, f32, i64, u64, u64,
                                                f32, f32, f32, f32, f32, i64, vp]
        L.dp_reduce_noise_adamw_step.argtypes = [vp, vp, vp, vp, vp, i32, i32, i64, i64, f32, f32, i64, u64, u64,
                                                 f32, f32, f32, f32, f32, i64, vp]
        L.dp_noise_scale_adamw_step_snr.argtypes = [vp, vp, vp, vp, i32, i64, i64, f32, f32, i64, u64, u64,
                                                    f32, f32, f32, f32, f32, i64, vp, vp]
        L.dp_clip_stats.argtypes = [vp, i32, vp, vp]
        L.dp_philox_u32.argtypes = [vp, i64, i64, u64, u64, vp]
        L.dp_token_equality_mask.argtypes = [vp, i32, i32, vp, vp]
        L.dp_shared_table_cross_sqnorms.argtypes = [vp, vp, i32, i32, vp, vp, i32, i32, i32, i32, vp, vp]
        L.dp_layernorm_sqnorms_static.argtypes = [vp, vp, i32, vp]
        L.dp_global_norm_workspace_bytes.restype = sz
        L.dp_global_norm_workspace_bytes.argtypes = []
        L.dp_global_sqnorm.argtypes = [vp, vp, i32, i32, i32, vp, vp, sz, vp]
        L.dp_clip_by_global_norm.argtypes = [vp, vp, vp, i32, i32, vp, f32, vp, vp]
        L.dp_clip_adamw_step.argtypes = [vp, vp, vp, vp, i32, i64, vp, f32, f32, f32, f32, f32, f32, i64, vp]
        L.dp_rows_sqnorms.argtypes = [vp, i32, i32, vp, i32, vp]
        L.dp_rows_clipped_accumulate.argtypes = [vp, i32, i32, vp, vp]
        L.dp_relpos_bucket_starts.argtypes = [i32, i32, i32, vp]
        L.dp_relpos_bias.argtypes = [vp, vp, i32, vp, i32, i64, i64, vp]
        L.dp_relpos_workspace_bytes.restype = sz
        L.dp_relpos_workspace_bytes.argtypes = [vp, i32]
        L.dp_relpos_bias_grad.argtypes = [vp, i32, i32, vp, i32, i64, i64, i64, vp, vp, vp, i32, vp, sz, vp]
        L.dp_qknorm_rope.argtypes = [vp, vp, vp, vp, vp, vp]
        L.dp_qknorm_workspace_bytes.restype = sz
        L.dp_qknorm_workspace_bytes.argtypes = [vp]
        L.dp_qknorm_rope_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.dp_vocab_workspace_bytes.restype = sz
        L.dp_vocab_workspace_bytes.argtypes = [vp]
        L.dp_vocab_loss.argtypes = [vp, vp, vp, vp, sz, vp]
        L.dp_vocab_loss_backward.argtypes = [vp, vp, vp, i64, vp, i32, vp, sz, vp]
        L.dp_vocab_loss_clipped_accumulate.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
        L.dp_vocab_loss_cross_sqnorms.argtypes = [vp, vp, vp, vp, i64, i32, vp, vp, sz, vp]
        L.dp_distill_loss.argtypes = [vp, vp, vp, i64, vp]
        L.dp_poll_status.argtypes = [vp]
        L.dp_set_wait_limit_cycles.argtypes = [C.c_longlong]
        L.dp_selftest_wait_timeout.argtypes = [vp]
        L.dp_status_string.restype = C.c_char_p
        L.dp_status_string.argtypes = [i32]
        L.dp_version.restype = i32
        L.dp_launch_count.restype = C.c_longlong
        for name in EXPORTS:
            getattr(L, name)          # AttributeError if the library does not export it
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().dp_status_string(int(code)).decode()


def _check(fn: str, code: int):
    if code != DP_OK:
        raise DpError(fn, code)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return t.data_ptr()


def _stream(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


@dataclass
class Layer:
    """Python-side layer description; tensors live on the GPU."""
    kind: str
    G: torch.Tensor
    A: Optional[torch.Tensor] = None
    ids: Optional[torch.Tensor] = None
    acc_w: Optional[torch.Tensor] = None
    acc_b: Optional[torch.Tensor] = None
    has_bias: bool = False
    vocab: int = 0
    path: int = DP_PATH_AUTO


class LayerList:
    """A HOST array of dp_layer descriptors plus references that keep the tensors alive."""

    def __init__(self, layers: Sequence[Layer]):
        self.layers = list(layers)
        self.array = (dp_layer * len(self.layers))()
        for k, L in enumerate(self.layers):
            d = self.array[k]
            B, T, d_out = L.G.shape
            if L.G.dtype not in (torch.float32, torch.bfloat16):
                raise ValueError("A and G must be fp32 or bf16")
            d.kind = _KINDS[L.kind]
            d.dtype = DP_F32 if L.G.dtype == torch.float32 else DP_BF16
            d.path = int(L.path)
            d.has_bias = int(bool(L.has_bias))
            d.B, d.T, d.d_out = B, T, d_out
            if L.kind == "embedding":
                if L.ids is None or L.ids.dtype != torch.int32:
                    raise ValueError("embedding needs int32 ids")
                d.d_in = int(L.vocab)
            else:
                if L.A is None or L.A.dtype != L.G.dtype:
                    raise ValueError("A must have G's dtype")
                d.d_in = L.A.shape[2]
            d.A, d.ids, d.G = _ptr(L.A), _ptr(L.ids), _ptr(L.G)
            d.acc_w, d.acc_b = _ptr(L.acc_w), _ptr(L.acc_b)
            for acc in (L.acc_w, L.acc_b):
                if acc is not None and acc.dtype != torch.float32:
                    raise ValueError("accumulators are fp32")

    @property
    def ptr(self):
        return C.cast(self.array, C.c_void_p)

    def __len__(self):
        return len(self.layers)

    @property
    def B(self) -> int:
        return int(self.array[0].B)


def dp_version() -> int:
    return lib().dp_version()


def dp_workspace_bytes(layers: LayerList) -> int:
    return int(lib().dp_workspace_bytes(layers.ptr, len(layers)))


def alloc_workspace(layers: LayerList) -> Optional[torch.Tensor]:
    """Caller-owned scratch for the two layer-list calls (torch's allocator aligns to 512 bytes)."""
    n = dp_workspace_bytes(layers)
    dev = layers.layers[0].G.device
    return torch.empty(max(n, 256), dtype=torch.uint8, device=dev)


def dp_per_example_sqnorms(layers: LayerList, sqnorm: torch.Tensor, accumulate_into: bool = False,
                           workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    ws_p, ws_n = (_ptr(workspace), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    _check("dp_per_example_sqnorms",
           lib().dp_per_example_sqnorms(layers.ptr, len(layers), _ptr(sqnorm), int(accumulate_into), ws_p, ws_n,
                                        _stream(stream)))
    return sqnorm


def dp_shared_table_cross_sqnorms(emb: Layer, proj: Layer, sqnorm: torch.Tensor, stream=None) -> torch.Tensor:
    """sqnorm[i] += 2 <scatter_i, dlogits_i^T h_i> for a table trained through the embedding layer `emb` and the
    output projection `proj` (a linear layer whose A is dlogits [B, T_out, V] and whose G is h [B, T_out, d])."""
    B, T, d = emb.G.shape
    _, T_out, V = proj.A.shape
    if emb.ids is None or emb.ids.dtype != torch.int32 or proj.A.dtype != emb.G.dtype or proj.G.dtype != emb.G.dtype:
        raise ValueError("embedding ids (int32) and one dtype for G_emb, dlogits and h expected")
    if proj.G.shape != (B, T_out, d) or int(emb.vocab) != V:
        raise ValueError("the projection must map [B, T_out, V] x [B, T_out, d] onto the embedding's [V, d] table")
    dtype = DP_F32 if emb.G.dtype == torch.float32 else DP_BF16
    _check("dp_shared_table_cross_sqnorms",
           lib().dp_shared_table_cross_sqnorms(_ptr(emb.ids), _ptr(emb.G), B, T, _ptr(proj.A), _ptr(proj.G), T_out, d, V,
                                               dtype, _ptr(sqnorm), _stream(stream)))
    return sqnorm


def dp_clip_factors(sqnorm: torch.Tensor, C_: float, clip: torch.Tensor, stream=None) -> torch.Tensor:
    _check("dp_clip_factors", lib().dp_clip_factors(_ptr(sqnorm), sqnorm.numel(), float(C_), _ptr(clip), _stream(stream)))
    return clip


def dp_clipped_accumulate(layers: LayerList, clip: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    ws_p, ws_n = (_ptr(workspace), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    _check("dp_clipped_accumulate",
           lib().dp_clipped_accumulate(layers.ptr, len(layers), _ptr(clip), ws_p, ws_n, _stream(stream)))


def dp_clipped_accumulate_after_sqnorms(layers: LayerList, clip: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                                        stream=None) -> None:
    """dp_clipped_accumulate for the call that directly follows dp_per_example_sqnorms over the same `layers`
    and `workspace`: the LayerNorm column sums left there are reused instead of being recomputed."""
    ws_p, ws_n = (_ptr(workspace), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    _check("dp_clipped_accumulate_after_sqnorms",
           lib().dp_clipped_accumulate_after_sqnorms(layers.ptr, len(layers), _ptr(clip), ws_p, ws_n, _stream(stream)))


def dp_accumulate_schedule(layers: LayerList, units: int, max_launches: int = 16) -> dict:
    """Host-only view of the accumulate GEMM's work schedule on a device with `units` CTA pairs: per layer the first
    work item and the launch it belongs to (-1: the layer takes another path), per launch the number of example
    ranges a tile is split into and the number of item slots."""
    n = len(layers)
    start, launch = (C.c_int64 * n)(), (C.c_int32 * n)()
    splits, slots = (C.c_int32 * max_launches)(), (C.c_int64 * max_launches)()
    rc = lib().dp_accumulate_schedule(layers.ptr, n, int(units), C.cast(start, C.c_void_p), C.cast(launch, C.c_void_p),
                                      C.cast(splits, C.c_void_p), C.cast(slots, C.c_void_p), max_launches)
    if rc < 0:
        raise DpError("dp_accumulate_schedule", rc)
    return {"item_start": list(start), "launch": list(launch), "splits": list(splits)[:rc], "slots": list(slots)[:rc]}


def dp_add_noise_and_scale(acc: torch.Tensor, sigma: float, C_: float, batch_size: int, seed: int, step: int,
                           elem_offset: int = 0, stream=None) -> torch.Tensor:
    _check("dp_add_noise_and_scale",
           lib().dp_add_noise_and_scale(_ptr(acc), acc.numel(), int(elem_offset), float(sigma), float(C_),
                                        int(batch_size), int(seed), int(step), _stream(stream)))
    return acc


def dp_adamw_step(theta, m, v, g, lr, beta1, beta2, xi, weight_decay, t, stream=None) -> None:
    _check("dp_adamw_step",
           lib().dp_adamw_step(_ptr(theta), _ptr(m), _ptr(v), _ptr(g), theta.numel(), float(lr), float(beta1),
                               float(beta2), float(xi), float(weight_decay), int(t), _stream(stream)))


def dp_noise_scale_adamw_step(theta, m, v, acc, zero_acc, sigma, C_, batch_size, seed, step, lr, beta1, beta2,
                              xi, weight_decay, t, elem_offset: int = 0, stream=None) -> None:
    _check("dp_noise_scale_adamw_step",
           lib().dp_noise_scale_adamw_step(_ptr(theta), _ptr(m), _ptr(v), _ptr(acc), int(bool(zero_acc)),
                                           theta.numel(), int(elem_offset), float(sigma), float(C_),
                                           int(batch_size), int(seed), int(step), float(lr), float(beta1),
                                           float(beta2), float(xi), float(weight_decay), int(t), _stream(stream)))


def dp_noise_scale_adamw_step_snr(theta, m, v, acc, zero_acc, sigma, C_, batch_size, seed, step, lr, beta1, beta2,
                                  xi, weight_decay, t, sq_sums: torch.Tensor, elem_offset: int = 0, stream=None) -> None:
    """sq_sums: float64 device tensor [2], accumulated into (sum acc^2, sum (sigma C z)^2)."""
    if sq_sums.dtype != torch.float64 or sq_sums.numel() != 2:
        raise ValueError("sq_sums must be a float64 tensor with 2 elements")
    _check("dp_noise_scale_adamw_step_snr",
           lib().dp_noise_scale_adamw_step_snr(_ptr(theta), _ptr(m), _ptr(v), _ptr(acc), int(bool(zero_acc)),
                                               theta.numel(), int(elem_offset), float(sigma), float(C_),
                                               int(batch_size), int(seed), int(step), float(lr), float(beta1),
                                               float(beta2), float(xi), float(weight_decay), int(t),
                                               _ptr(sq_sums), _stream(stream)))


def dp_reduce_noise_adamw_step(theta, m, v, acc_shards, theta_shards, zero_acc, sigma, C_, batch_size, seed, step, lr,
                               beta1, beta2, xi, weight_decay, t, elem_offset: int = 0, stream=None) -> None:
    """Fused cross-rank sum + noise + AdamW on one shard.  acc_shards: one entry per rank, the shard inside that
    rank's accumulator (a tensor, or a raw device address for peer-mapped memory); theta_shards: the shard inside
    every rank's replica of theta, entries may be None (or the whole argument None) to skip the write."""
    def addr(x):
        return 0 if x is None else (int(x) if isinstance(x, int) else x.data_ptr())
    R = len(acc_shards)
    acc_arr = (C.c_void_p * R)(*[addr(a) for a in acc_shards])
    th_arr = None if theta_shards is None else (C.c_void_p * R)(*[addr(x) for x in theta_shards])
    _check("dp_reduce_noise_adamw_step",
           lib().dp_reduce_noise_adamw_step(_ptr(theta), _ptr(m), _ptr(v), C.cast(acc_arr, C.c_void_p),
                                            None if th_arr is None else C.cast(th_arr, C.c_void_p), R,
                                            int(bool(zero_acc)), theta.numel(), int(elem_offset), float(sigma),
                                            float(C_), int(batch_size), int(seed), int(step), float(lr), float(beta1),
                                            float(beta2), float(xi), float(weight_decay), int(t), _stream(stream)))


def dp_clip_stats(clip: torch.Tensor, out: torch.Tensor, stream=None) -> torch.Tensor:
    _check("dp_clip_stats", lib().dp_clip_stats(_ptr(clip), clip.numel(), _ptr(out), _stream(stream)))
    return out


def dp_philox_u32(out: torch.Tensor, elem_offset: int, seed: int, step: int, stream=None) -> torch.Tensor:
    """out: int32 tensor (bit pattern of the uint32 words)."""
    _check("dp_philox_u32", lib().dp_philox_u32(_ptr(out), out.numel(), int(elem_offset), int(seed), int(step),
                                                _stream(stream)))
    return out


def dp_token_equality_mask(ids: torch.Tensor, mask: torch.Tensor, stream=None) -> torch.Tensor:
    B, T = ids.shape
    _check("dp_token_equality_mask", lib().dp_token_equality_mask(_ptr(ids), B, T, _ptr(mask), _stream(stream)))
    return mask


STATIC_SCRATCH_FLOATS = 1 << 20


def dp_layernorm_sqnorms_static(layers: LayerList, sqnorm: torch.Tensor, accumulate_into: bool = False,
                                stream=None) -> torch.Tensor:
    """Norms of the single LayerNorm layer in `layers` with the library's fixed scratch (no workspace)."""
    if len(layers) != 1:
        raise ValueError("exactly one LayerNorm layer expected")
    _check("dp_layernorm_sqnorms_static",
           lib().dp_layernorm_sqnorms_static(layers.ptr, _ptr(sqnorm), int(accumulate_into), _stream(stream)))
    return sqnorm


def dp_last_timeout_info():
    info = (C.c_int * 5)()
    _check("dp_last_timeout_info", lib().dp_last_timeout_info(info))
    return list(info)


def dp_launch_count() -> int:
    return int(lib().dp_launch_count())


def dp_poll_status(stream=None) -> int:
    return int(lib().dp_poll_status(_stream(stream)))


def dp_set_wait_limit_cycles(cycles: int) -> None:
    """Limit of every bounded device-side wait on the current device (<= 0: the default of 4e9 SM cycles)."""
    _check("dp_set_wait_limit_cycles", lib().dp_set_wait_limit_cycles(int(cycles)))


def dp_selftest_wait_timeout(stream=None) -> None:
    """Enqueues the kernel whose waits nobody satisfies; dp_poll_status reports DP_ERR_TIMEOUT afterwards."""
    _check("dp_selftest_wait_timeout", lib().dp_selftest_wait_timeout(_stream(stream)))



# ---- global norm over many tensors, rows, relative position bias, query/key norms, losses of a vocabulary head ---------
# These calls serve small tensors too, where the host side of a call is most of its time: the CPython module _dp_tensors
# (csrc/dp_tensors.cpp) checks the tensors, fills the descriptors and calls the library's entry points.  It takes what the
# functions below take, in their order, and returns the status; a tensor that does not fit raises ValueError.
MODULE_PATH = os.path.join(_HERE, "_dp_tensors.so")
_BOUND = ["dp_global_sqnorm", "dp_clip_by_global_norm", "dp_clip_adamw_step", "dp_rows_sqnorms", "dp_rows_clipped_accumulate",
          "dp_relpos_bias", "dp_relpos_workspace_bytes", "dp_relpos_bias_grad", "dp_qknorm_rope",
          "dp_qknorm_workspace_bytes", "dp_qknorm_rope_backward", "dp_vocab_workspace_bytes", "dp_vocab_loss",
          "dp_vocab_loss_backward", "dp_vocab_loss_clipped_accumulate", "dp_vocab_loss_cross_sqnorms",
          "dp_distill_loss"]       # in the order of its bind()
_module = None


def _native():
    global _module
    if _module is None:
        if not os.path.exists(MODULE_PATH):
            raise ImportError(f"{MODULE_PATH} not found: run `python -m paper_2108_01624_b200.build` (needs nvcc and g++). "
                              "There is no fallback implementation.")
        from . import build as builder
        if not builder.module_fits(MODULE_PATH):          # before it is loaded: its view of a tensor may be another
            raise ImportError(f"{MODULE_PATH} was built for another torch or Python than this one ({builder.module_key()}): "
                              "run `python -m paper_2108_01624_b200.build`.")
        spec = importlib.util.spec_from_file_location("_dp_tensors", MODULE_PATH)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        m.bind(*[C.cast(getattr(lib(), name), C.c_void_p).value for name in _BOUND])
        _module = m
    return _module


def dp_global_norm_workspace_bytes() -> int:
    return int(lib().dp_global_norm_workspace_bytes())


def dp_global_sqnorm(tensors: Sequence[torch.Tensor], sqsum: torch.Tensor, accumulate_into: bool = False,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """sqsum (float64, one element) = or += the sum of squares over all tensors of the list (one dtype, fp32 or bf16)."""
    rc = (_module or _native()).global_sqnorm(tensors, sqsum, accumulate_into, workspace,
                                              None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_global_sqnorm", rc)
    return sqsum


def dp_clip_by_global_norm(tensors: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]], sqsum: torch.Tensor,
                           max_norm: float, norm_and_factor: Optional[torch.Tensor] = None, stream=None) -> None:
    """outs[k] = tensors[k] * min(1, max_norm / sqrt(sqsum)); outs=None scales in place.  norm_and_factor: optional
    float32 tensor with 2 elements that receives the norm and the factor."""
    rc = (_module or _native()).clip_by_global_norm(tensors, outs, sqsum, max_norm, norm_and_factor,
                                                    None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_clip_by_global_norm", rc)


def dp_clip_adamw_step(theta, m, v, g, zero_g, sqsum: torch.Tensor, max_norm: float, lr, beta1, beta2, xi, weight_decay,
                       t, stream=None) -> None:
    """dp_adamw_step on g * min(1, max_norm / sqrt(sqsum)); zero_g clears g in the same pass."""
    rc = (_module or _native()).clip_adamw_step(theta, m, v, g, zero_g, sqsum, max_norm, lr, beta1, beta2, xi, weight_decay,
                                                t, None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_clip_adamw_step", rc)


class RowList:
    """A HOST array of dp_rows descriptors: (per-example gradients [B, ...], accumulator [...]) pairs, fp32, plus
    references that keep the tensors alive.  The accumulator may be None where only the norms are wanted."""

    def __init__(self, pairs: Sequence[tuple]):
        self.pairs = list(pairs)
        self.native = (_module or _native()).rows_list(self.pairs)

    @property
    def B(self) -> int:
        return self.native[1]

    def __len__(self):
        return len(self.pairs)


def dp_rows_sqnorms(rows: RowList, sqnorm: torch.Tensor, accumulate_into: bool = False, stream=None) -> torch.Tensor:
    rc = (_module or _native()).rows_sqnorms(rows.native, sqnorm, accumulate_into,
                                             None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_rows_sqnorms", rc)
    return sqnorm


def dp_rows_clipped_accumulate(rows: RowList, clip: torch.Tensor, stream=None) -> None:
    rc = (_module or _native()).rows_clipped_accumulate(rows.native, clip, None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_rows_clipped_accumulate", rc)


def dp_relpos_bucket_starts(num_buckets: int, max_distance: int, bidirectional: bool) -> List[int]:
    """Smallest distance of each bucket of one side (host only)."""
    half = num_buckets // 2 if bidirectional else num_buckets
    out = (C.c_int32 * max(half, 1))()
    _check("dp_relpos_bucket_starts",
           lib().dp_relpos_bucket_starts(int(num_buckets), int(max_distance), int(bool(bidirectional)),
                                         C.cast(out, C.c_void_p)))
    return list(out)


def dp_relpos_bias(table: torch.Tensor, out: torch.Tensor, max_distance: int = 128, bidirectional: bool = True,
                   offset: int = 0, stream=None) -> torch.Tensor:
    """out[h, q, k] = table[bucket(k - q - offset), h]; table [num_buckets, heads], out [heads, Tq, Tk] with unit stride
    along the keys and rows that do not overlap (fp32 or bf16 each)."""
    rc = (_module or _native()).relpos_bias(table, out, max_distance, bidirectional, offset,
                                            None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_relpos_bias", rc)
    return out


def dp_relpos_workspace_bytes(G: torch.Tensor, num_buckets: int) -> int:
    """Scratch for dp_relpos_bias_grad over G [B, heads, Tq, Tk] (at least 256, so that it can be allocated)."""
    return (_module or _native()).relpos_workspace_bytes(G, num_buckets)


def dp_relpos_bias_grad(G: torch.Tensor, rows: torch.Tensor, max_distance: int = 128, bidirectional: bool = True,
                        offset: int = 0, causal: bool = False, q_len: Optional[torch.Tensor] = None,
                        k_len: Optional[torch.Tensor] = None, accumulate_into: bool = False,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """rows[b, n, h] = or += sum over the (q, k) of bucket n of G[b, h, q, k]: every example's gradient of the table.
    G [B, heads, Tq, Tk] (fp32 or bf16) with unit stride along the keys, rows fp32 [B, num_buckets, heads]; q_len, k_len
    int32 [B]."""
    rc = (_module or _native()).relpos_bias_grad(G, rows, max_distance, bidirectional, offset, causal, q_len, k_len,
                                                 accumulate_into, workspace, None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_relpos_bias_grad", rc)
    return rows


def rope_frequencies(rot: int, base: float = 10000.0) -> torch.Tensor:
    """inv_freq[j] = base^(-2j / rot), float64 on the host: radians per position of pair j."""
    return float(base) ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))


def dp_qknorm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], out_q: Optional[torch.Tensor],
                   out_k: Optional[torch.Tensor], gain_q: Optional[torch.Tensor], gain_k: Optional[torch.Tensor],
                   eps: float, inv_freq: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                   lengths: Optional[torch.Tensor] = None, interleaved: bool = False, stream=None) -> None:
    """RMS norm per head with gain, then the position rotation.  q, k [B, T, heads, dim] (any strides, unit along dim;
    the outputs' heads do not overlap), either None; gains fp32 [dim] or None; inv_freq float64 on the host
    (rope_frequencies), its length is rot / 2, None for no rotation; positions int32 [B, T], lengths int32 [B]."""
    rc = (_module or _native()).qknorm_rope(q, k, out_q, out_k, gain_q, gain_k, eps, inv_freq, positions, lengths,
                                            interleaved, None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_qknorm_rope", rc)


def dp_qknorm_workspace_bytes(q: Optional[torch.Tensor], k: Optional[torch.Tensor]) -> int:
    """Scratch for dp_qknorm_rope_backward (at least 256, so that it can be allocated)."""
    return (_module or _native()).qknorm_workspace_bytes(q, k)


def dp_qknorm_rope_backward(q, k, dout_q, dout_k, dq, dk, gain_q: Optional[torch.Tensor], gain_k: Optional[torch.Tensor],
                            rows_q: Optional[torch.Tensor], rows_k: Optional[torch.Tensor], eps: float,
                            inv_freq: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                            lengths: Optional[torch.Tensor] = None, interleaved: bool = False,
                            accumulate_into: bool = False, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dq, dk and every example's gradients of the gains (rows_q, rows_k fp32 [B, dim], or None) from the inputs of
    dp_qknorm_rope and the gradients of its outputs."""
    rc = (_module or _native()).qknorm_rope_backward(q, k, dout_q, dout_k, dq, dk, gain_q, gain_k, rows_q, rows_k, eps,
                                                     inv_freq, positions, lengths, interleaved, accumulate_into, workspace,
                                                     None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_qknorm_rope_backward", rc)


class VocabHead:
    """A softmax head over a vocabulary: tokens x [B, T, d] (evenly spaced rows), table weight [V, d] of the same dtype
    (fp32 or bf16), labels int32 [B, T] (negative: no loss), bias fp32 [V] or None, token_weights fp32 [B, T] or None for
    ones.  A HOST descriptor plus references that keep the tensors alive."""

    def __init__(self, x: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 token_weights: Optional[torch.Tensor] = None):
        self.x, self.weight, self.labels, self.bias, self.token_weights = x, weight, labels, bias, token_weights
        self.native = (_module or _native()).vocab_head(x, weight, labels, bias, token_weights)

    @property
    def B(self) -> int:
        return self.x.shape[0]


def dp_vocab_workspace_bytes(head: VocabHead) -> int:
    """Scratch for the calls on this head (at least 256, so that it can be allocated)."""
    return (_module or _native()).vocab_workspace_bytes(head.native)


def dp_vocab_loss(head: VocabHead, loss: torch.Tensor, lse: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """loss, lse [B, T] fp32: weighted cross entropy of every token and the log-sum-exp of its logits, which are not kept."""
    rc = (_module or _native()).vocab_loss(head.native, loss, lse, workspace, None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_vocab_loss", rc)
    return loss


def dp_vocab_loss_backward(head: VocabHead, lse: torch.Tensor, dx: Optional[torch.Tensor], sqnorm: Optional[torch.Tensor],
                           accumulate_into: bool = False, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dx like x (may be a view with evenly spaced rows, but not lie over x) and sqnorm [B] = or += every example's squared norm of the gradients
    of table and bias; either may be None."""
    rc = (_module or _native()).vocab_loss_backward(head.native, lse, dx, sqnorm, accumulate_into, workspace,
                                                    None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_vocab_loss_backward", rc)


def dp_vocab_loss_clipped_accumulate(head: VocabHead, lse: torch.Tensor, clip: torch.Tensor, acc_w: torch.Tensor,
                                     acc_b: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                     stream=None) -> None:
    """acc_w [V, d] and, with a bias, acc_b [V] += the clipped sum over the examples of their gradients."""
    rc = (_module or _native()).vocab_loss_clipped_accumulate(head.native, lse, clip, acc_w, acc_b, workspace,
                                                              None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_vocab_loss_clipped_accumulate", rc)


def dp_vocab_loss_cross_sqnorms(head: VocabHead, lse: torch.Tensor, ids: torch.Tensor, g_emb: torch.Tensor,
                                sqnorm: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """sqnorm[i] += twice the inner product of the two parts of example i's gradient of a table that the head shares with
    the token embedding: ids int32 [B, inputs], g_emb [B, inputs, d] the gradient of the embedding's output."""
    rc = (_module or _native()).vocab_loss_cross_sqnorms(head.native, lse, ids, g_emb, sqnorm, workspace,
                                                         None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_vocab_loss_cross_sqnorms", rc)
    return sqnorm


def dp_distill_loss(logits: torch.Tensor, top_ids: torch.Tensor, top_logits: torch.Tensor, temperature: float,
                    loss: torch.Tensor, dlogits: Optional[torch.Tensor], token_weights: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """Distillation of logits [B, T, V] from the teacher's K top logits (top_ids int32, top_logits fp32 or bf16, [B, T, K];
    negative ids are empty places): loss [B, T] fp32 and, unless None, dlogits like logits (which may be logits itself, but not overlap it otherwise)."""
    rc = (_module or _native()).distill_loss(logits, top_ids, top_logits, temperature, loss, dlogits, token_weights,
                                             None if stream is None else stream.cuda_stream)
    if rc:
        raise DpError("dp_distill_loss", rc)
    return loss
