"""Host-side sequencing of one DP-SGD macro-step over the C ABI (no arithmetic here).

Algorithm 1's g_t needs, per microbatch, the per-example norms over ALL layers before any layer can be
scaled, hence two passes over (A, G): norms -> clip factors -> clipped accumulate.  Noise, the division by
the macro-batch size and the AdamW update run once per macro-batch (Section 5.3) as one fused pass.
"""
from __future__ import annotations

import math
from typing import List, Optional, Sequence

import torch

from . import binding as b
from .synth import EMBEDDING, LAYERNORM, LINEAR, ROWS, LayerData, LayerSpec


class DeviceStatusError(RuntimeError):
    """The library's device-side status word was not clean when a macro-batch was about to be applied."""

    def __init__(self, code: int):
        self.code = int(code)
        try:
            what = b.status_string(self.code)
        except Exception:          # the library itself is missing
            what = "?"
        super().__init__(f"device status {self.code} ({what}): the macro-batch was discarded, "
                         "parameters and optimizer state are unchanged")


class DPStep:
    """Owns the flat fp32 state (theta, m, v, accumulator) for a list of layer specs.

    Tensors are laid end to end in spec order (weight then bias), each start rounded up to a multiple of
    4 elements so that every tensor is 16-byte aligned and one fused launch covers the whole vector.  The
    flat index of an element is also its Philox element index.
    """

    def __init__(self, specs: Sequence[LayerSpec], device, C: float, sigma: float, lr: float, beta1: float,
                 beta2: float, xi: float, weight_decay: float, seed: int = 0, theta: Optional[torch.Tensor] = None,
                 track_snr: bool = False, shared_tables: Optional[dict] = None, shard_world: int = 1,
                 max_grad_norm: Optional[float] = None):
        """shard_world: number of data-parallel ranks the macro-batch will be finished across (parallel.ShardedUpdate).
        The accumulator and theta are then allocated with room for `shard_world` equal shards (acc_store,
        theta_store; acc and theta are their first n_flat elements), so that the reduce-scatter and the all-gather
        of a macro-batch's end run in place.

        shared_tables maps the index of an output-projection spec (a bias-free LINEAR layer with d_in = V whose
        A is dlogits and whose G is the projection's input) to the index of the EMBEDDING spec whose [V, d] table it
        also trains (BERT's masked-LM decoder): the projection gets no storage of its own, both layers accumulate into
        the table, and the per-example norm includes the inner product of their two contributions.

        max_grad_norm clips the noised mean gradient of a macro-batch to this global L2 norm, over all tensors, before
        the AdamW update (post-processing of Algorithm 1's g_t, so it changes nothing about the privacy of a step).

        A ROWS spec [d_in, d_out] is a tensor whose per-example gradients are formed elsewhere (dp_relpos_bias_grad,
        dp_qknorm_rope_backward): pass them with every microbatch, accumulate_microbatch(..., rows=row_list(data))."""
        if max_grad_norm is not None:
            if not (max_grad_norm > 0.0 and math.isfinite(max_grad_norm)):
                raise ValueError("max_grad_norm must be positive and finite")
            if track_snr:
                raise ValueError("track_snr reads its sums from the fused update, which max_grad_norm does not use")
        self.max_grad_norm = max_grad_norm
        self.grad_sqsum = None          # float64 [1]: squared norm of the last macro-batch's noised mean gradient
        self._norm_ws = None
        self.specs = list(specs)
        self.shared_tables = dict(shared_tables or {})
        for p_li, e_li in self.shared_tables.items():
            sp, se = self.specs[p_li], self.specs[e_li]
            if not (e_li < p_li and se.kind == EMBEDDING and sp.kind == LINEAR and not sp.has_bias
                    and sp.d_in == se.d_in and sp.d_out == se.d_out):
                raise ValueError("a shared table needs an EMBEDDING [V, d] listed before a bias-free LINEAR V -> d")
        self.device = torch.device(device)
        self.C, self.sigma, self.lr, self.beta1, self.beta2 = C, sigma, lr, beta1, beta2
        self.xi, self.weight_decay, self.seed = xi, weight_decay, seed
        self.offsets: List[List[int]] = []
        self.shapes: List[List[tuple]] = []
        pos = 0
        for li, sp in enumerate(self.specs):
            if li in self.shared_tables:              # alias of the embedding's table
                e_li = self.shared_tables[li]
                self.offsets.append(list(self.offsets[e_li]))
                self.shapes.append(list(self.shapes[e_li]))
                continue
            if sp.kind == LINEAR:
                shp = [(sp.d_in, sp.d_out)] + ([(sp.d_out,)] if sp.has_bias else [])
            elif sp.kind == LAYERNORM:
                shp = [(sp.d_out,), (sp.d_out,)]
            else:
                shp = [(sp.d_in, sp.d_out)]
            offs = []
            for s in shp:
                offs.append(pos)
                n = 1
                for x in s:
                    n *= x
                pos += (n + 3) // 4 * 4
            self.offsets.append(offs)
            self.shapes.append(shp)
        self.n_flat = pos
        from .parallel import padded_length
        cap = padded_length(pos, shard_world)
        self.acc_store = torch.zeros(cap, dtype=torch.float32, device=self.device)
        self.acc = self.acc_store[:pos]
        self.m = torch.zeros(pos, dtype=torch.float32, device=self.device)
        self.v = torch.zeros_like(self.m)
        self.theta_store = torch.zeros_like(self.acc_store) if theta is None else None
        self.theta = self.theta_store[:pos] if theta is None else theta
        self.t = 0
        self.examples_seen = 0
        # gradient-SNR of Section 5.2.1: (sum acc^2, sum noise^2) of the last macro-batch, filled by the fused pass
        self.sq_sums = torch.zeros(2, dtype=torch.float64, device=self.device) if track_snr else None
        self._ws = None
        self._sqnorm = None
        self._clip = None

    def view(self, flat: torch.Tensor, li: int, k: int) -> torch.Tensor:
        shp = self.shapes[li][k]
        n = 1
        for x in shp:
            n *= x
        off = self.offsets[li][k]
        return flat[off:off + n].view(*shp)

    def layer_list(self, data: Sequence[LayerData], paths: Optional[Sequence[int]] = None) -> b.LayerList:
        """Descriptors for one microbatch; data[k] must correspond to specs[k].  ROWS entries are left to row_list."""
        out = []
        for li, ld in enumerate(data):
            sp = self.specs[li]
            assert ld.spec.kind == sp.kind and ld.spec.d_out == sp.d_out
            if sp.kind == ROWS:
                continue
            acc_w = self.view(self.acc, li, 0)
            acc_b = self.view(self.acc, li, 1) if len(self.shapes[li]) > 1 else None
            out.append(b.Layer(kind=sp.kind, G=ld.G, A=ld.A, ids=ld.ids, acc_w=acc_w, acc_b=acc_b,
                               has_bias=sp.has_bias, vocab=sp.d_in if sp.kind == EMBEDDING else 0,
                               path=b.DP_PATH_AUTO if paths is None else paths[li]))
        return b.LayerList(out)

    def row_list(self, data: Sequence[LayerData]) -> Optional[b.RowList]:
        """Descriptors of the ROWS entries of one microbatch (None if there are none); data[k] corresponds to specs[k]."""
        pairs = [(ld.G.view(ld.G.shape[0], sp.d_in, sp.d_out), self.view(self.acc, li, 0))
                 for li, (sp, ld) in enumerate(zip(self.specs, data)) if sp.kind == ROWS]
        return b.RowList(pairs) if pairs else None

    def tensor_pieces(self, flat: torch.Tensor, lo: int = 0, hi: Optional[int] = None) -> List[torch.Tensor]:
        """The tensors' elements among [lo, hi) of the flat vector, whose element lo is flat[0]: one 1-D view per tensor,
        without the padding between tensors.  A shared table counts once."""
        hi = self.n_flat if hi is None else hi
        out = []
        for li in range(len(self.specs)):
            if li in self.shared_tables:
                continue
            for off, shp in zip(self.offsets[li], self.shapes[li]):
                a, z = max(off, lo), min(off + math.prod(shp), hi)
                if a < z:
                    out.append(flat[a - lo:z - lo])
        return out

    def layer_lists(self, data: Sequence[LayerData], paths: Optional[Sequence[int]] = None) -> List[b.LayerList]:
        """Descriptors for one microbatch whose layers do not all see the same number of tokens (encoder layers per
        token, the masked-LM head per masked position, pooler and sentence classifier per example): one list per
        token count, in order of first appearance; accumulate_microbatch takes the result."""
        whole = self.layer_list(data, paths)
        groups: dict = {}
        for L in whole.layers:
            groups.setdefault(int(L.G.shape[1]), []).append(L)
        return [b.LayerList(ls) for ls in groups.values()]

    def accumulate_microbatch(self, layers, stream=None, rows=None):
        """norms -> clip factors -> clipped accumulate for one microbatch (all enqueued, no sync).
        `layers` is a LayerList, or a list of them (layer_lists) when token counts differ between layers; `rows` is the
        row_list of the microbatch, needed exactly when there are ROWS specs (an example's norm runs over ALL its
        tensors: one left out would break the bound that the noise is calibrated to)."""
        lists = [layers] if isinstance(layers, b.LayerList) else list(layers)
        lists = [ll for ll in lists if len(ll)]
        n_rows = sum(sp.kind == ROWS for sp in self.specs)
        if (0 if rows is None else len(rows)) != n_rows:
            raise ValueError(f"the model has {n_rows} ROWS tensors: pass row_list(data) of this microbatch as rows")
        if not lists and rows is None:
            raise ValueError("no layers")
        B = lists[0].B if lists else rows.B
        if rows is not None and rows.B != B:
            raise ValueError(f"rows of {rows.B} examples, layers of {B}")
        if self._sqnorm is None or self._sqnorm.numel() != B:
            self._sqnorm = torch.empty(B, dtype=torch.float32, device=self.device)
            self._clip = torch.empty(B, dtype=torch.float32, device=self.device)
        if self._ws is None or len(self._ws) != len(lists):
            self._ws = [None] * len(lists)
        for k, ll in enumerate(lists):
            need = b.dp_workspace_bytes(ll)
            if self._ws[k] is None or self._ws[k].numel() < need:
                self._ws[k] = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
            b.dp_per_example_sqnorms(ll, self._sqnorm, k > 0, self._ws[k], stream)
        if self.shared_tables:
            by_acc = {}
            for ll in lists:
                for L in ll.layers:
                    by_acc.setdefault(L.acc_w.data_ptr(), []).append(L)
            for pair in by_acc.values():          # an embedding and the projection that shares its accumulator
                if len(pair) == 2:
                    emb, proj = (pair[0], pair[1]) if pair[0].kind == EMBEDDING else (pair[1], pair[0])
                    b.dp_shared_table_cross_sqnorms(emb, proj, self._sqnorm, stream)
        if rows is not None:
            b.dp_rows_sqnorms(rows, self._sqnorm, bool(lists), stream)
        b.dp_clip_factors(self._sqnorm, self.C, self._clip, stream)
        for k, ll in enumerate(lists):
            b.dp_clipped_accumulate_after_sqnorms(ll, self._clip, self._ws[k], stream)
        if rows is not None:
            b.dp_rows_clipped_accumulate(rows, self._clip, stream)
        self.examples_seen += B
        return self._sqnorm, self._clip

    def discard_macro_batch(self) -> None:
        """Drops the partly accumulated macro-batch: the accumulator is cleared, theta, m, v and t stay as they are."""
        self.acc.zero_()
        self.examples_seen = 0

    def check_device_status(self, stream=None) -> None:
        """Waits for the stream and reads the library's sticky status word.  A bounded wait that ran out or a token
        id out of range makes the kernels skip the offending work, so a squared norm may be wrong and the factor
        min(1, C/||g_i||) would no longer bound that example's contribution by C -- the sensitivity that the noise of
        Algorithm 1 is calibrated to.  In that case the macro-batch is discarded and DeviceStatusError raised."""
        code = b.dp_poll_status(stream)
        if code != b.DP_OK:
            self.discard_macro_batch()
            raise DeviceStatusError(code)

    def finish_macro_batch(self, batch_size: Optional[int] = None, fused: bool = True, stream=None,
                           check_status: bool = True):
        """Noise, division by the macro-batch size and the AdamW update; clears the accumulator.
        With check_status (one host synchronisation per macro-batch) a device-side error reported since the last
        poll raises DeviceStatusError BEFORE anything is applied: theta, m, v and t are untouched and the
        accumulator is cleared."""
        if check_status:
            self.check_device_status(stream)
        N = self.examples_seen if batch_size is None else batch_size
        self.t += 1
        if self.max_grad_norm is not None:
            self.noised_sqnorm(self.acc, 0, N, stream)
            self.clipped_update(self.theta, self.m, self.v, self.acc, stream)
        elif fused and self.sq_sums is not None:
            self.sq_sums.zero_()
            b.dp_noise_scale_adamw_step_snr(self.theta, self.m, self.v, self.acc, True, self.sigma, self.C, N,
                                            self.seed, self.t, self.lr, self.beta1, self.beta2, self.xi,
                                            self.weight_decay, self.t, self.sq_sums, 0, stream)
        elif fused:
            b.dp_noise_scale_adamw_step(self.theta, self.m, self.v, self.acc, True, self.sigma, self.C, N, self.seed,
                                        self.t, self.lr, self.beta1, self.beta2, self.xi, self.weight_decay, self.t,
                                        0, stream)
        else:
            b.dp_add_noise_and_scale(self.acc, self.sigma, self.C, N, self.seed, self.t, 0, stream)
            b.dp_adamw_step(self.theta, self.m, self.v, self.acc, self.lr, self.beta1, self.beta2, self.xi,
                            self.weight_decay, self.t, stream)
            self.acc.zero_()
        self.examples_seen = 0

    def noised_sqnorm(self, acc: torch.Tensor, elem_offset: int, batch_size: int, stream=None) -> torch.Tensor:
        """acc (the flat vector from element elem_offset on) <- (acc + noise) / batch_size in place; returns the squared
        norm of its tensors' elements in grad_sqsum."""
        if self.grad_sqsum is None:
            self.grad_sqsum = torch.zeros(1, dtype=torch.float64, device=self.device)
        if self._norm_ws is None:       # after an end of a macro-batch with an empty shard there is a sum, but no workspace
            self._norm_ws = torch.empty(b.dp_global_norm_workspace_bytes(), dtype=torch.uint8, device=self.device)
        b.dp_add_noise_and_scale(acc, self.sigma, self.C, batch_size, self.seed, self.t, elem_offset, stream)
        b.dp_global_sqnorm(self.tensor_pieces(acc, elem_offset, elem_offset + acc.numel()), self.grad_sqsum, False,
                           self._norm_ws, stream)
        return self.grad_sqsum

    def clipped_update(self, theta, m, v, acc, stream=None) -> None:
        """AdamW on acc, clipped to max_grad_norm by the squared norm in grad_sqsum; acc is cleared."""
        b.dp_clip_adamw_step(theta, m, v, acc, True, self.grad_sqsum, self.max_grad_norm, self.lr, self.beta1, self.beta2,
                             self.xi, self.weight_decay, self.t, stream)

    def grad_norm(self) -> float:
        """Global norm of the last finished macro-batch's noised mean gradient before its clip (host sync)."""
        if self.grad_sqsum is None:
            raise RuntimeError("construct DPStep with max_grad_norm and finish a macro-batch")
        return math.sqrt(float(self.grad_sqsum.item()))

    def state_dict(self) -> dict:
        """Everything a run needs to resume in the middle of a macro-batch: parameters, Adam moments, the partly
        filled accumulator, the macro-step counter (which also keys the noise) and the examples seen so far.
        The noise generator is counter-based, so a resumed run draws exactly the noise the original would have."""
        return {"theta": self.theta.clone(), "m": self.m.clone(), "v": self.v.clone(), "acc": self.acc.clone(),
                "t": self.t, "examples_seen": self.examples_seen, "seed": self.seed, "n_flat": self.n_flat}

    def load_state_dict(self, state: dict) -> None:
        if int(state["n_flat"]) != self.n_flat:
            raise ValueError("state belongs to another parameter layout")
        for name in ("theta", "m", "v", "acc"):
            getattr(self, name).copy_(state[name])
        self.t, self.examples_seen, self.seed = int(state["t"]), int(state["examples_seen"]), int(state["seed"])

    def gradient_snr(self) -> float:
        """||aggregated clipped gradient|| / ||noise vector|| of the last finished macro-batch (host sync)."""
        if self.sq_sums is None:
            raise RuntimeError("construct DPStep with track_snr=True")
        s = self.sq_sums.cpu()
        return float((s[0] / s[1]).sqrt()) if float(s[1]) > 0 else float("inf")
