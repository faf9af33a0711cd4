"""Host-side sequencing of one DP-SGD macro-step over the C ABI (no arithmetic here).

Algorithm 1's g_t needs, per microbatch, the per-example norms over ALL layers before any layer can be
scaled, hence two passes over (A, G): norms -> clip factors -> clipped accumulate.  Noise, the division by
the macro-batch size and the AdamW update run once per macro-batch (Section 5.3) as one fused pass.
"""
from __future__ import annotations

import contextlib
import math
from typing import List, Optional, Sequence

import torch

from . import binding as b
from .synth import EMBEDDING, HEAD, LAYERNORM, LINEAR, ROWS, LayerData, LayerSpec


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

        A HEAD spec [V, d] is a softmax head whose logits and their gradients are not kept (binding.VocabHead).  Its turn in a
        microbatch: head_backward(li, head, lse, dx) in the backward pass, accumulate_microbatch after it.  It may share the table
        of an EMBEDDING spec through shared_tables too, with a bias of its own.

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
            if not (e_li < p_li and se.kind == EMBEDDING and (sp.kind == HEAD or sp.kind == LINEAR and not sp.has_bias)
                    and sp.d_in == se.d_in and sp.d_out == se.d_out):
                raise ValueError("a shared table needs an EMBEDDING [V, d] listed before a bias-free LINEAR V -> d or a HEAD")
            if sp.kind == HEAD and list(self.shared_tables.values()).count(e_li) > 1:
                raise ValueError("a HEAD that shares a table is the only one that does")
        self.device = torch.device(device)
        self.C, self.sigma, self.lr, self.beta1, self.beta2 = C, sigma, lr, beta1, beta2
        self.xi, self.weight_decay, self.seed = xi, weight_decay, seed
        self.offsets: List[List[int]] = []
        self.shapes: List[List[tuple]] = []
        pos = 0
        for li, sp in enumerate(self.specs):
            if sp.kind == LINEAR:
                shp = [(sp.d_in, sp.d_out)] + ([(sp.d_out,)] if sp.has_bias else [])
            elif sp.kind == LAYERNORM:
                shp = [(sp.d_out,), (sp.d_out,)]
            elif sp.kind == HEAD:
                shp = [(sp.d_in, sp.d_out)] + ([(sp.d_in,)] if sp.has_bias else [])
            else:
                shp = [(sp.d_in, sp.d_out)]
            offs = []
            for k, s in enumerate(shp):
                if k == 0 and li in self.shared_tables:              # alias of the embedding's table
                    offs.append(self.offsets[self.shared_tables[li]][0])
                    continue
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
        self.spoilt = False             # a microbatch failed while its clipped sums were added: some are in acc
        # gradient-SNR of Section 5.2.1: (sum acc^2, sum noise^2) of the last macro-batch, filled by the fused pass
        self.sq_sums = torch.zeros(2, dtype=torch.float64, device=self.device) if track_snr else None
        self._ws = None
        self._sqnorm = None
        self._clip = None
        self._heads: dict = {}          # heads of the microbatch under way: spec index -> (head, lse)
        self._head_ws = None
        self._streams: dict = {}        # buffers -> the streams whose calls have used them

    def view(self, flat: torch.Tensor, li: int, k: int) -> torch.Tensor:
        shp = self.shapes[li][k]
        n = 1
        for x in shp:
            n *= x
        off = self.offsets[li][k]
        return flat[off:off + n].view(*shp)

    def layer_list(self, data: Sequence[LayerData], paths: Optional[Sequence[int]] = None) -> b.LayerList:
        """Descriptors for one microbatch; data[k] must correspond to specs[k].  ROWS entries are left to row_list, HEAD
        entries (None) to head_backward."""
        out = []
        for li, ld in enumerate(data):
            sp = self.specs[li]
            if sp.kind == HEAD:
                continue
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
            own = slice(1 if li in self.shared_tables else 0, None)
            for off, shp in zip(self.offsets[li][own], self.shapes[li][own]):
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

    # Buffers of the calls.  Each is allocated for the stream of the calls that use it (the one they are given, or else the current
    # one), and one that is replaced is kept from the allocator until every stream that used it is past it.
    def _on(self, stream):
        return torch.cuda.stream(stream) if stream is not None and self.device.type == "cuda" else contextlib.nullcontext()

    def _used(self, what, stream) -> None:
        """A call on `stream` is about to use the buffers `what`."""
        if stream is None and self.device.type == "cuda":
            stream = torch.cuda.current_stream(self.device)
        if stream is not None:
            self._streams.setdefault(what, set()).add(stream)

    def _replaced(self, what, *buffers) -> None:
        for stream in self._streams.pop(what, ()):
            for t in buffers:
                t.record_stream(stream)

    def _batch(self, B: int, stream=None) -> None:
        """Norms and factors of a microbatch of B examples."""
        if self._sqnorm is None or self._sqnorm.numel() != B:
            if self._sqnorm is not None:
                self._replaced("batch", self._sqnorm, self._clip)
            with self._on(stream):
                self._sqnorm, self._clip = (torch.empty(B, dtype=torch.float32, device=self.device) for _ in range(2))
        self._used("batch", stream)

    def _at_least(self, old: Optional[torch.Tensor], need: int, what, stream) -> torch.Tensor:
        """A workspace of `need` bytes or more: the old one, or another in its place."""
        if old is None or old.numel() < need:
            if old is not None:
                self._replaced(what, old)
            with self._on(stream):
                old = torch.empty(need, dtype=torch.uint8, device=self.device)
        self._used(what, stream)
        return old

    def _workspaces(self, lists, stream=None) -> None:
        """A workspace for each of the microbatch's lists of layers."""
        if self._ws is None or len(self._ws) != len(lists):
            for k, ws in enumerate(self._ws or ()):
                self._replaced(k, ws)
            self._ws = [None] * len(lists)
        for k, ll in enumerate(lists):
            self._ws[k] = self._at_least(self._ws[k], max(b.dp_workspace_bytes(ll), 256), k, stream)

    def _head_workspace(self, head: b.VocabHead, stream=None) -> torch.Tensor:
        self._head_ws = self._at_least(self._head_ws, b.dp_vocab_workspace_bytes(head), "head", stream)
        return self._head_ws

    def head_backward(self, li: int, head: b.VocabHead, lse: torch.Tensor, dx: Optional[torch.Tensor], stream=None) -> None:
        """Backward pass of the HEAD spec `li` for the microbatch under way, from dp_vocab_loss's lse: dx, and the norms of its
        gradients for the clip.  accumulate_microbatch, which wants every HEAD spec's call before it, adds its clipped sum, so
        the head's tensors and lse stay as they are until then.  Again for the same spec, or with another number of examples: the
        microbatch begins anew."""
        self.refuse_if_spoilt()
        sp = self.specs[li]
        if sp.kind != HEAD:
            raise ValueError(f"spec {li} is no HEAD")
        if tuple(head.weight.shape) != (sp.d_in, sp.d_out) or (head.bias is not None) != sp.has_bias:
            raise ValueError(f"spec {li}: a head [{sp.d_in}, {sp.d_out}] {'with' if sp.has_bias else 'without'} bias expected")
        begun, self._heads = self._heads, {}          # norms that a call fails to add to are not added to again
        if li in begun or any(h.B != head.B for h, _ in begun.values()):
            begun = {}
        self._batch(head.B, stream)
        b.dp_vocab_loss_backward(head, lse, dx, self._sqnorm, bool(begun), self._head_workspace(head, stream), stream)
        self._heads = {**begun, li: (head, lse)}

    def accumulate_microbatch(self, layers, stream=None, rows=None):
        """norms -> clip factors -> clipped accumulate for one microbatch (all enqueued, no sync).
        `layers` is a LayerList, or a list of them (layer_lists) when token counts differ between layers; `rows` is the
        row_list of the microbatch, needed exactly when there are ROWS specs (an example's norm runs over ALL its
        tensors: one left out would break the bound that the noise is calibrated to).
        What does not fit together is refused before the first norm, and can be passed again corrected.  A call that fails later
        leaves norms half summed: the microbatch begins anew with the HEAD specs' head_backward.  One that fails among the clipped
        sums leaves some of them in the accumulator, where a second try would add them again, beyond C: nothing but
        discard_macro_batch is taken then."""
        self.refuse_if_spoilt()
        lists = [layers] if isinstance(layers, b.LayerList) else list(layers)
        lists = [ll for ll in lists if len(ll)]
        heads = dict(sorted(self._heads.items()))
        if len(heads) != sum(sp.kind == HEAD for sp in self.specs):
            raise ValueError("every HEAD spec needs its head_backward before accumulate_microbatch")
        n_rows = sum(sp.kind == ROWS for sp in self.specs)
        if (0 if rows is None else len(rows)) != n_rows:
            raise ValueError(f"the model has {n_rows} ROWS tensors: pass row_list(data) of this microbatch as rows")
        if not lists and rows is None and not heads:
            raise ValueError("no layers")
        B = lists[0].B if lists else rows.B if rows is not None else next(iter(heads.values()))[0].B
        if any(h.B != B for h, _ in heads.values()):
            raise ValueError(f"heads of other numbers of examples than {B}")
        if rows is not None and rows.B != B:
            raise ValueError(f"rows of {rows.B} examples, layers of {B}")
        if any(ll.B != B for ll in lists):
            raise ValueError(f"layers of other numbers of examples than {B}")
        by_acc = {}                                   # layers by the accumulator of their weight
        for ll in lists if self.shared_tables else ():
            for L in ll.layers:
                by_acc.setdefault(L.acc_w.data_ptr(), []).append(L)
        tables = {}                                   # the embedding that shares its table with a head
        for li, (head, _) in heads.items():
            if li in self.shared_tables:
                emb = by_acc.get(self.view(self.acc, li, 0).data_ptr(), [])
                if len(emb) != 1 or emb[0].kind != EMBEDDING:
                    raise ValueError(f"the embedding that shares its table with head {li} is missing")
                if emb[0].G.dtype != head.x.dtype or emb[0].G.shape[2] != head.x.shape[2]:
                    raise ValueError(f"the embedding's G and the states of head {li} that shares its table differ in dtype or width")
                tables[li] = emb[0]
        self._heads = {}                              # what follows adds to their norms: after a failure they are wanted anew
        self._batch(B, stream)
        self._workspaces(lists, stream)
        for k, ll in enumerate(lists):
            b.dp_per_example_sqnorms(ll, self._sqnorm, k > 0 or bool(heads), self._ws[k], stream)
        for pair in by_acc.values():                  # an embedding and the projection that shares its accumulator
            if len(pair) == 2:
                emb, proj = (pair[0], pair[1]) if pair[0].kind == EMBEDDING else (pair[1], pair[0])
                b.dp_shared_table_cross_sqnorms(emb, proj, self._sqnorm, stream)
        for li, emb in tables.items():
            head, lse = heads[li]
            b.dp_vocab_loss_cross_sqnorms(head, lse, emb.ids, emb.G, self._sqnorm, self._head_workspace(head, stream), stream)
        if rows is not None:
            b.dp_rows_sqnorms(rows, self._sqnorm, bool(lists) or bool(heads), stream)
        b.dp_clip_factors(self._sqnorm, self.C, self._clip, stream)
        self.spoilt = True                            # until all of the sums are added
        for k, ll in enumerate(lists):
            b.dp_clipped_accumulate_after_sqnorms(ll, self._clip, self._ws[k], stream)
        for li, (head, lse) in heads.items():
            b.dp_vocab_loss_clipped_accumulate(head, lse, self._clip, self.view(self.acc, li, 0),
                                               self.view(self.acc, li, 1) if head.bias is not None else None,
                                               self._head_workspace(head, stream), stream)
        if rows is not None:
            b.dp_rows_clipped_accumulate(rows, self._clip, stream)
        self.spoilt = False
        self.examples_seen += B
        return self._sqnorm, self._clip

    def discard_macro_batch(self, stream=None) -> None:
        """Drops the partly accumulated macro-batch: the accumulator is cleared, theta, m, v and t stay as they are."""
        with self._on(stream):
            self.acc.zero_()
        self._heads = {}
        self.examples_seen = 0
        self.spoilt = False

    def refuse_if_spoilt(self) -> None:
        if self.spoilt:
            raise RuntimeError("a microbatch failed while its clipped sums were added to the accumulator: discard_macro_batch() first")

    def check_device_status(self, stream=None) -> None:
        """Waits for the stream and reads the library's sticky status word.  A bounded wait that ran out or a token
        id out of range makes the kernels skip the offending work, so a squared norm may be wrong and the factor
        min(1, C/||g_i||) would no longer bound that example's contribution by C -- the sensitivity that the noise of
        Algorithm 1 is calibrated to.  In that case the macro-batch is discarded and DeviceStatusError raised."""
        code = b.dp_poll_status(stream)
        if code != b.DP_OK:
            self.discard_macro_batch(stream)
            raise DeviceStatusError(code)

    def finish_macro_batch(self, batch_size: Optional[int] = None, fused: bool = True, stream=None,
                           check_status: bool = True):
        """Noise, division by the macro-batch size and the AdamW update; clears the accumulator.
        With check_status (one host synchronisation per macro-batch) a device-side error reported since the last
        poll raises DeviceStatusError BEFORE anything is applied: theta, m, v and t are untouched and the
        accumulator is cleared."""
        if check_status:
            self.check_device_status(stream)
        self.refuse_if_spoilt()
        N = self.examples_seen if batch_size is None else batch_size
        self.t += 1
        if self.max_grad_norm is not None:
            self.noised_sqnorm(self.acc, 0, N, stream)
            self.clipped_update(self.theta, self.m, self.v, self.acc, stream)
        elif fused and self.sq_sums is not None:
            with self._on(stream):
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
            with self._on(stream):
                self.acc.zero_()
        self.examples_seen = 0

    def noised_sqnorm(self, acc: torch.Tensor, elem_offset: int, batch_size: int, stream=None) -> torch.Tensor:
        """acc (the flat vector from element elem_offset on) <- (acc + noise) / batch_size in place; returns the squared
        norm of its tensors' elements in grad_sqsum."""
        with self._on(stream):
            if self.grad_sqsum is None:
                self.grad_sqsum = torch.zeros(1, dtype=torch.float64, device=self.device)
            if self._norm_ws is None:   # after an end of a macro-batch with an empty shard there is a sum, but no workspace
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
