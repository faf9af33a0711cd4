"""The operators that a transformer trained under DP-SGD needs beside the layer kinds of the privatised step, with
their plain forms.

  clip       a list of gradient tensors scaled to a global L2 norm of at most max_norm
  adamw      the same clip folded into an AdamW step over flat fp32 state
  bias       the learned relative position bias of an attention layer, [heads, queries, keys], from its bucket table
  bias_grad  every example's gradient of that table from the gradient of the scores, its norm, clip factor and the
             clipped sum over the microbatch
  qk         RMS norm of every query and key head, with a learned gain, and the position rotation, in one pass
  qk_grad    its backward pass: gradients of queries and keys, and every example's gradients of the two gains

`run` computes them in elementary torch operations, or, where `own` is true, through the package's calls.  `exact` is
the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6                                     # of the RMS norm
LR, BETA1, BETA2, XI, DECAY = 6.0902e-4, 0.9, 0.999, 1e-11, 0.5


def listed():
    return [
        # the gradients of one narrow encoder block: a call that is all latency
        {"name": "clip one small block", "op": "clip", "dtype": "fp32", "hidden": 64, "ffn": 256, "blocks": 1, "vocab": 0,
         "max_norm": 1.0},
        # the bf16 gradients of the whole BERT-Large stack with its word-piece table
        {"name": "clip BERT-Large bf16", "op": "clip", "dtype": "bf16", "hidden": 1024, "ffn": 4096, "blocks": 24,
         "vocab": 30522, "max_norm": 1.0},
        # one linear layer of 64 x 64 with bias: the smallest model that the repository trains
        {"name": "adamw one small layer", "op": "adamw", "n": 4160, "max_norm": 1.0, "t": 3},
        # every parameter of the BERT-Large stack, as one flat vector
        {"name": "adamw BERT-Large", "op": "adamw", "n": 333563904, "max_norm": 1.0, "t": 100},
        # one query against a long context: the bias row of a token that is being generated
        {"name": "bias one query", "op": "bias", "dtype": "bf16", "heads": 16, "tq": 1, "tk": 8191, "buckets": 32,
         "distance": 128, "both": False, "offset": 8190},
        # a long document, every query against every key
        {"name": "bias long document", "op": "bias", "dtype": "bf16", "heads": 16, "tq": 4096, "tk": 4096, "buckets": 32,
         "distance": 128, "both": True, "offset": 0},
        # one layer of the BERT-Large microbatch
        {"name": "bias_grad T=128", "op": "bias_grad", "dtype": "bf16", "batch": 256, "heads": 16, "tq": 128, "tk": 128,
         "buckets": 32, "distance": 128, "both": True, "offset": 0, "causal": False, "ragged": False},
        # the long-sequence microbatch, examples padded to 512 tokens
        {"name": "bias_grad T=512 padded", "op": "bias_grad", "dtype": "bf16", "batch": 64, "heads": 16, "tq": 512,
         "tk": 512, "buckets": 32, "distance": 128, "both": True, "offset": 0, "causal": False, "ragged": True},
        # one new token for each of 64 sequences, grouped heads
        {"name": "qk one token", "op": "qk", "dtype": "bf16", "batch": 64, "tokens": 1, "hq": 32, "hk": 8, "dim": 128,
         "rot": 128, "pairs": "halves", "first": 32767, "fused": True},
        # the BERT-Large microbatch: 16 heads of 64 out of the fused projection
        {"name": "qk BERT-Large", "op": "qk", "dtype": "bf16", "batch": 256, "tokens": 128, "hq": 16, "hk": 16, "dim": 64,
         "rot": 64, "pairs": "halves", "first": 0, "fused": True},
        # its backward pass
        {"name": "qk_grad BERT-Large", "op": "qk_grad", "dtype": "bf16", "batch": 256, "tokens": 128, "hq": 16, "hk": 16,
         "dim": 64, "rot": 64, "pairs": "halves", "first": 0, "fused": True},
        # few examples of odd length in fp32, neighbouring pairs, a part of the head rotated, heads before tokens
        {"name": "qk_grad odd fp32", "op": "qk_grad", "dtype": "fp32", "batch": 3, "tokens": 515, "hq": 9, "hk": 3,
         "dim": 80, "rot": 32, "pairs": "neighbours", "first": 100003, "fused": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("clip", "adamw", "bias", "bias_grad", "qk", "qk_grad"))
    dtype = rng.choice(("fp32", "bf16"))
    if op == "clip":
        return {"op": op, "dtype": dtype, "hidden": _log_int(rng, 17, 1024), "ffn": _log_int(rng, 33, 4096),
                "blocks": rng.randint(1, 24), "vocab": rng.choice((0, _log_int(rng, 100, 30522))),
                "max_norm": round(10.0 ** rng.uniform(-2, 5), 4)}
    if op == "adamw":
        return {"op": op, "n": _log_int(rng, 1, 333563904), "max_norm": round(10.0 ** rng.uniform(-2, 5), 4),
                "t": _log_int(rng, 1, 20000)}
    if op in ("bias", "bias_grad"):
        half = rng.choice((4, 8, 16, 32))
        both = rng.random() < 0.5
        c = {"op": op, "dtype": dtype, "heads": rng.randint(1, 24), "buckets": 2 * half if both else half,
             "distance": rng.choice((half + 1, 64, 128, 129, 256, 1000)), "both": both}
        if op == "bias":
            c.update(tq=rng.choice((1, _log_int(rng, 2, 4096))), tk=_log_int(rng, 1, 4096))
            c["offset"] = rng.choice((0, c["tk"] - 1, rng.randint(-50, 5000)))
            return c
        c.update(tq=_log_int(rng, 1, 1100), tk=_log_int(rng, 1, 1100))
        c["batch"] = _log_int(rng, 1, max(1, min(256, 100_000_000 // (c["heads"] * c["tq"] * c["tk"]))))
        c["offset"] = rng.choice((0, max(0, c["tk"] - c["tq"])))
        c["causal"], c["ragged"] = rng.random() < 0.5, rng.random() < 0.5
        return c
    dim = rng.choice((32, 64, 80, 96, 128, 192, 256, 6, 50))
    hk = rng.randint(1, 8)
    c = {"op": op, "dtype": dtype, "hq": hk * rng.randint(1, 6), "hk": hk, "dim": dim,
         "rot": rng.choice((dim, dim // 4 * 2)), "pairs": rng.choice(("halves", "neighbours")),
         "first": rng.choice((0, rng.randint(0, 1000000))), "fused": rng.random() < 0.5}
    c["tokens"] = rng.choice((1, _log_int(rng, 2, 4096)))
    c["batch"] = _log_int(rng, 1, max(1, min(256, 60_000_000 // (c["tokens"] * (c["hq"] + hk) * dim))))
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _shapes(case):
    """The tensors of `blocks` encoder blocks (weights, biases, norms) and of the word-piece table."""
    h, f = case["hidden"], case["ffn"]
    block = [(h, 3 * h), (3 * h,), (h, h), (h,), (h,), (h,), (h, f), (f,), (f, h), (h,), (h,), (h,)]
    return block * case["blocks"] + ([(case["vocab"], h)] if case["vocab"] else [])


def _views(flat, shapes):
    """Tensors end to end in one flat vector, each start at a multiple of 16 bytes."""
    step, out, pos = 16 // flat.element_size(), [], 0
    for s in shapes:
        n = math.prod(s)
        out.append(flat[pos:pos + n].view(s))
        pos += -(-n // step) * step
    return out


def _flat_length(shapes, dtype):
    step = 16 // dtype.itemsize
    return sum(-(-math.prod(s) // step) * step for s in shapes)


def _lengths(case, g, most):
    return torch.randint(max(1, most // 4), most + 1, (case["batch"],), generator=g, device=DEV, dtype=torch.int32)


def _inv_freq(case):
    r = case["rot"] // 2
    return 10000.0 ** (-torch.arange(r, dtype=torch.float64) / max(r, 1))      # radians a token, on the host


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    op = case["op"]
    s = {"case": case}
    if op == "clip":
        dtype, shapes = DTYPES[case["dtype"]], _shapes(case)
        n = _flat_length(shapes, dtype)
        flat, out = torch.zeros(n, dtype=dtype, device=DEV), torch.zeros(n, dtype=dtype, device=DEV)
        grads = _views(flat, shapes)
        for x in grads:
            x.normal_(0.0, 0.01, generator=g)
        s.update(flat=flat, grads=grads, out=out, outs=_views(out, shapes),
                 work=torch.empty(65536, dtype=torch.uint8, device=DEV))
    elif op == "adamw":
        n = case["n"]
        s.update(theta=normal(n).mul_(0.02), m=normal(n).mul_(1e-4), v=normal(n).square_().mul_(1e-8),
                 g=normal(n).mul_(1e-3), work=torch.empty(65536, dtype=torch.uint8, device=DEV))
    elif op == "bias":
        s.update(table=normal(case["buckets"], case["heads"]))
    elif op == "bias_grad":
        B, H, tq, tk = case["batch"], case["heads"], case["tq"], case["tk"]
        scale = torch.pow(10.0, 2.0 * torch.rand(B, generator=g, device=DEV) - 1.0) / math.sqrt(H * tq * tk)
        G = torch.empty(B, H, tq, tk, dtype=DTYPES[case["dtype"]], device=DEV)
        for i in range(B):
            G[i] = normal(H, tq, tk) * scale[i]
        s.update(q_len=None, k_len=None)
        if case["ragged"]:                     # what lies beyond an example's lengths was never written
            s.update(q_len=_lengths(case, g, tq), k_len=_lengths(case, g, tk))
            away = torch.arange(tq, device=DEV)[None, :, None] >= s["q_len"][:, None, None]
            away = away | (torch.arange(tk, device=DEV)[None, None, :] >= s["k_len"][:, None, None])
            G.masked_fill_(away[:, None], float("nan"))
        s.update(G=G, acc=normal(case["buckets"], H))
    else:
        B, T, hq, hk, D = (case[k] for k in ("batch", "tokens", "hq", "hk", "dim"))
        dtype = DTYPES[case["dtype"]]
        if case["fused"]:                      # queries, keys and values side by side, as one projection writes them
            x = normal(B, T, (hq + 2 * hk) * D).to(dtype)
            s.update(q=x[..., :hq * D].unflatten(-1, (hq, D)), k=x[..., hq * D:(hq + hk) * D].unflatten(-1, (hk, D)))
        else:                                  # heads before tokens
            s.update(q=normal(B, hq, T, D).to(dtype).transpose(1, 2), k=normal(B, hk, T, D).to(dtype).transpose(1, 2))
        s.update(gain_q=1.0 + 0.1 * normal(D), gain_k=1.0 + 0.1 * normal(D), inv_freq=_inv_freq(case),
                 pos=torch.arange(T, dtype=torch.int32, device=DEV).add_(case["first"]).expand(B, T).contiguous())
        if op == "qk_grad":
            s.update(gq=normal(B, T, hq, D).to(dtype), gk=normal(B, T, hk, D).to(dtype))
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_clip(s):
    x = s["flat"].float()                      # the tensors lie end to end, zeros between them change nothing
    norm = x.double().square().sum().sqrt()
    factor = torch.where(norm > 0, (s["case"]["max_norm"] / norm).clamp(max=1.0), torch.ones_like(norm))
    return {"grads": (x * factor.float()).to(s["flat"].dtype), "norm": norm.float(), "factor": factor.float()}


def _plain_adamw(s):
    c, g = s["case"], s["g"]
    norm = g.double().square().sum().sqrt()
    factor = torch.where(norm > 0, (c["max_norm"] / norm).clamp(max=1.0), torch.ones_like(norm))
    g = g * factor.float()
    s["m"].mul_(BETA1).add_(g * (1.0 - BETA1))
    s["v"].mul_(BETA2).add_(g * g * (1.0 - BETA2))
    root = (s["v"] * (1.0 / (1.0 - BETA2 ** c["t"]))).sqrt_().add_(XI)
    step = (s["m"] * (1.0 / (1.0 - BETA1 ** c["t"]))).div_(root).add_(s["theta"] * DECAY)
    s["theta"].sub_(step.mul_(LR))
    return {"theta": s["theta"], "m": s["m"], "v": s["v"]}


def _plain_buckets(c):
    """[tq, tk] bucket of (query, key).  Distances below `exact` have a bucket each; the others are spaced by their
    logarithm, so bucket exact + j starts at exact * (distance / exact)^(j / rest), taken to the next whole number."""
    half = c["buckets"] // 2 if c["both"] else c["buckets"]
    exact = half // 2
    j = torch.arange(1, half - exact, dtype=torch.float64, device=DEV)
    start = exact * (c["distance"] / exact) ** (j / (half - exact))
    start = torch.ceil(start * (1.0 - 1e-11)).long()
    start = torch.cat([torch.arange(1, exact + 1, device=DEV), start])
    rel = torch.arange(c["tk"], device=DEV)[None, :] - (torch.arange(c["tq"], device=DEV) + c["offset"])[:, None]
    far = rel.abs() if c["both"] else (-rel).clamp(min=0)
    bucket = torch.searchsorted(start, far, right=True)
    return bucket + half * (rel > 0) if c["both"] else bucket


def _plain_bias(s):
    c = s["case"]
    return s["table"].t()[:, _plain_buckets(c)].to(DTYPES[c["dtype"]])


def _plain_bias_grad(s):
    c = s["case"]
    B, H, tq, tk = (c[k] for k in ("batch", "heads", "tq", "tk"))
    keep = torch.ones(1, tq, tk, dtype=torch.bool, device=DEV)
    row, col = torch.arange(tq, device=DEV)[:, None], torch.arange(tk, device=DEV)[None, :]
    if c["causal"]:
        keep = keep & (col <= row + c["offset"])
    if c["ragged"]:
        keep = keep & (row < s["q_len"][:, None, None]) & (col < s["k_len"][:, None, None])
    G = torch.where(keep[:, None], s["G"].double(), 0.0)
    member = torch.nn.functional.one_hot(_plain_buckets(c).view(-1), c["buckets"]).double()
    rows = (G.view(B * H, tq * tk) @ member).view(B, H, -1).transpose(1, 2).contiguous()
    square = rows.square().sum((1, 2))
    clip = torch.where(square > 0, square.rsqrt().clamp(max=1.0), torch.ones_like(square))
    acc = s["acc"].double() + (rows * clip[:, None, None]).sum(0)
    return {"rows": rows.float(), "square": square.float(), "clip": clip.float(), "acc": acc.float()}


def _plain_angles(s):
    angle = s["pos"].double()[..., None, None] * s["inv_freq"].to(DEV)         # [B, T, 1, rot / 2]
    return angle.cos().float(), angle.sin().float()


def _plain_rotate(x, cos, sin, c):
    r = c["rot"]
    a, rest = x[..., :r], x[..., r:]
    if c["pairs"] == "halves":
        u, v = a[..., :r // 2], a[..., r // 2:]
        return torch.cat([u * cos - v * sin, v * cos + u * sin, rest], -1)
    u, v = a[..., 0::2], a[..., 1::2]
    return torch.cat([torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2), rest], -1)


def _plain_qk(s):
    c, (cos, sin) = s["case"], _plain_angles(s)

    def one(x, gain):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
        return _plain_rotate(x, cos, sin, c).to(DTYPES[c["dtype"]])

    return {"q": one(s["q"], s["gain_q"]), "k": one(s["k"], s["gain_k"])}


def _plain_qk_grad(s):
    c, (cos, sin) = s["case"], _plain_angles(s)

    def one(x, gain, dy):
        x, u = x.float(), _plain_rotate(dy.float(), cos, -sin, c)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        hat, w = x * r, u * gain
        dx = r * (w - hat * (w * hat).mean(-1, keepdim=True))
        return dx.to(DTYPES[c["dtype"]]), (u * hat).sum((1, 2))

    dq, rows_q = one(s["q"], s["gain_q"], s["gq"])
    dk, rows_k = one(s["k"], s["gain_k"], s["gk"])
    return {"dq": dq, "dk": dk, "rows_q": rows_q, "rows_k": rows_k}


_PLAIN = {"clip": _plain_clip, "adamw": _plain_adamw, "bias": _plain_bias, "bias_grad": _plain_bias_grad,
          "qk": _plain_qk, "qk_grad": _plain_qk_grad}


# ---- the package's calls --------------------------------------------------------------------------------------------
def _own_clip(s):
    import paper_2108_01624_b200 as dp
    square = torch.empty(1, dtype=torch.float64, device=DEV)
    told = torch.empty(2, dtype=torch.float32, device=DEV)
    dp.dp_global_sqnorm(s["grads"], square, workspace=s["work"])
    dp.dp_clip_by_global_norm(s["grads"], s["outs"], square, s["case"]["max_norm"], told)
    return {"grads": s["out"], "norm": told[0], "factor": told[1]}


def _own_adamw(s):
    import paper_2108_01624_b200 as dp
    square = torch.empty(1, dtype=torch.float64, device=DEV)
    dp.dp_global_sqnorm([s["g"]], square, workspace=s["work"])
    dp.dp_clip_adamw_step(s["theta"], s["m"], s["v"], s["g"], False, square, s["case"]["max_norm"], LR, BETA1, BETA2, XI,
                          DECAY, s["case"]["t"])
    return {"theta": s["theta"], "m": s["m"], "v": s["v"]}


def _own_bias(s):
    import paper_2108_01624_b200 as dp
    c = s["case"]
    out = torch.empty(c["heads"], c["tq"], c["tk"], dtype=DTYPES[c["dtype"]], device=DEV)
    return dp.dp_relpos_bias(s["table"], out, max_distance=c["distance"], bidirectional=c["both"], offset=c["offset"])


def _own_bias_grad(s):
    import paper_2108_01624_b200 as dp
    c = s["case"]
    B, H = c["batch"], c["heads"]
    rows = torch.empty(B, c["buckets"], H, dtype=torch.float32, device=DEV)
    square, clip = torch.empty(B, dtype=torch.float32, device=DEV), torch.empty(B, dtype=torch.float32, device=DEV)
    work = torch.empty(dp.dp_relpos_workspace_bytes(s["G"], c["buckets"]), dtype=torch.uint8, device=DEV)
    dp.dp_relpos_bias_grad(s["G"], rows, max_distance=c["distance"], bidirectional=c["both"], offset=c["offset"],
                           causal=c["causal"], q_len=s["q_len"], k_len=s["k_len"], workspace=work)
    acc = s["acc"].clone()
    table = dp.RowList([(rows, acc)])
    dp.dp_rows_sqnorms(table, square)
    dp.dp_clip_factors(square, 1.0, clip)
    dp.dp_rows_clipped_accumulate(table, clip)
    return {"rows": rows, "square": square, "clip": clip, "acc": acc}


def _own_qk(s):
    import paper_2108_01624_b200 as dp
    c, q, k = s["case"], s["q"], s["k"]
    out_q, out_k = (torch.empty(x.shape, dtype=x.dtype, device=DEV) for x in (q, k))
    dp.dp_qknorm_rope(q, k, out_q, out_k, s["gain_q"], s["gain_k"], EPS, s["inv_freq"], positions=s["pos"],
                      interleaved=c["pairs"] == "neighbours")
    return {"q": out_q, "k": out_k}


def _own_qk_grad(s):
    import paper_2108_01624_b200 as dp
    c, q, k = s["case"], s["q"], s["k"]
    dq, dk = (torch.empty(x.shape, dtype=x.dtype, device=DEV) for x in (q, k))
    rows_q, rows_k = (torch.empty(c["batch"], c["dim"], dtype=torch.float32, device=DEV) for _ in range(2))
    work = torch.empty(dp.dp_qknorm_workspace_bytes(q, k), dtype=torch.uint8, device=DEV)
    dp.dp_qknorm_rope_backward(q, k, s["gq"], s["gk"], dq, dk, s["gain_q"], s["gain_k"], rows_q, rows_k, EPS,
                               s["inv_freq"], positions=s["pos"], interleaved=c["pairs"] == "neighbours", workspace=work)
    return {"dq": dq, "dk": dk, "rows_q": rows_q, "rows_k": rows_k}


_OWN = {"clip": _own_clip, "adamw": _own_adamw, "bias": _own_bias, "bias_grad": _own_bias_grad, "qk": _own_qk,
        "qk_grad": _own_qk_grad}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    size = DTYPES[case["dtype"]].itemsize if "dtype" in case else 4
    if op == "clip":
        n = sum(math.prod(s) for s in _shapes(case))
        return {"bytes": 2 * size * n, "flops": 3 * n}
    if op == "adamw":
        return {"bytes": 28 * case["n"], "flops": 16 * case["n"]}
    if op == "bias":
        n = case["heads"] * case["tq"] * case["tk"]
        return {"bytes": size * n + 4 * case["heads"] * case["buckets"], "flops": 0}
    if op == "bias_grad":
        B, P, tq, tk = case["batch"], case["buckets"] * case["heads"], case["tq"], case["tk"]
        n = tq * tk
        if case["causal"]:
            seen = np.clip(np.arange(tq) + case["offset"] + 1, 0, tk)
            n = int(seen.sum())
        n *= B * case["heads"]
        if case["ragged"]:
            n = n * 25 // 64                   # mean share of lengths between a quarter and the whole, both ways
        return {"bytes": size * n + 4 * B * P + 8 * P + 8 * B, "flops": n + 4 * B * P}
    B, T, hq, hk, D = (case[k] for k in ("batch", "tokens", "hq", "hk", "dim"))
    n = B * T * (hq + hk) * D
    if op == "qk":
        return {"bytes": 2 * size * n + 4 * B * T + 8 * D, "flops": 7 * n}
    return {"bytes": 3 * size * n + 4 * B * T + 8 * D + 8 * B * D, "flops": 15 * n}


# ---- definitions in 64 bits -----------------------------------------------------------------------------------------
def _bucket_of(c, rel):
    """Bucket of key position minus query position, in whole numbers: bucket exact + j holds the distances n with
    (n / exact)^rest >= (distance / exact)^j, the last bucket all beyond."""
    base, half = 0, c["buckets"]
    if c["both"]:
        half //= 2
        base = half if rel > 0 else 0
        n = abs(rel)
    else:
        n = max(0, -rel)
    exact = half // 2
    if n < exact:
        return base + n
    rest, far = half - exact, c["distance"]
    j = 0
    while j + 1 < rest and n ** rest * exact ** (j + 1) >= far ** (j + 1) * exact ** rest:
        j += 1
    return base + exact + j


def _buckets_by_diagonal(c):
    """Of rel = -(tq - 1) - offset ... tk - 1 - offset; far ones are alike, so they are looked up at `most`."""
    most = 2 * c["distance"]
    rels = range(-(c["tq"] - 1) - c["offset"], c["tk"] - c["offset"])
    known = {r: _bucket_of(c, r) for r in range(-most, most + 1)}
    return [known[max(-most, min(most, r))] for r in rels]


def exact(case, seed):
    s, op, c = prepare(case, seed), case["op"], case
    if op == "clip":
        total = sum(float(torch.linalg.vector_norm(x.double())) ** 2 for x in s["grads"])
        norm = math.sqrt(total)
        factor = 1.0 if norm == 0.0 else min(1.0, c["max_norm"] / norm)
        return {"grads": s["flat"].double() * factor, "norm": norm, "factor": factor}
    if op == "adamw":
        total = sum(float(x.double().pow(2).sum()) for x in s["g"].split(1 << 24))
        factor = 1.0 if total == 0.0 else min(1.0, c["max_norm"] / math.sqrt(total))
        new = {"theta": [], "m": [], "v": []}
        for theta, m, v, g in zip(*(s[k].split(1 << 24) for k in ("theta", "m", "v", "g"))):
            theta, m, v, g = theta.double(), m.double(), v.double(), g.double() * factor
            m = BETA1 * m + (1 - BETA1) * g
            v = BETA2 * v + (1 - BETA2) * g ** 2
            hat = (m / (1 - BETA1 ** c["t"])) / ((v / (1 - BETA2 ** c["t"])) ** 0.5 + XI)
            for k, x in (("theta", theta - LR * (hat + DECAY * theta)), ("m", m), ("v", v)):
                new[k].append(x)
        return {k: torch.cat(x) for k, x in new.items()}
    if op == "bias":
        line = s["table"].double()[torch.tensor(_buckets_by_diagonal(c), device=DEV)]          # [diagonals, heads]
        out = torch.empty(c["heads"], c["tq"], c["tk"], dtype=torch.float64, device=DEV)
        for q in range(c["tq"]):
            first = c["tq"] - 1 - q
            out[:, q] = line[first:first + c["tk"]].t()
        return out
    if op == "bias_grad":
        B, H, tq, tk = (c[k] for k in ("batch", "heads", "tq", "tk"))
        of = torch.tensor(_buckets_by_diagonal(c), device=DEV)
        rows = torch.zeros(B, c["buckets"], H, dtype=torch.float64, device=DEV)
        wide = tq + tk
        for i in range(B):
            nq, nk = (tq, tk) if not c["ragged"] else (int(s["q_len"][i]), int(s["k_len"][i]))
            G = torch.zeros(H, tq, wide, dtype=torch.float64, device=DEV)
            G[:, tq - nq:, :nk] = s["G"][i, :, :nq, :nk].double().flip(1)
            # read with rows shorter by one, each row moves one to the right: column = key - query + tq - 1
            line = G.view(H, -1)[:, :tq * (wide - 1)].view(H, tq, wide - 1).sum(1)
            if c["causal"]:
                line[:, max(0, tq + c["offset"]):] = 0.0
            rows[i].index_add_(0, of, line.t())
        square = rows.pow(2).sum((1, 2))
        clip = torch.tensor([1.0 if n == 0.0 else min(1.0, 1.0 / math.sqrt(n)) for n in square.tolist()],
                            dtype=torch.float64, device=DEV)
        acc = s["acc"].double() + torch.einsum("b,bnh->nh", clip, rows)
        return {"rows": rows, "square": square, "clip": clip, "acc": acc}
    r, D = c["rot"], c["dim"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       (s["pos"].double()[..., None] * s["inv_freq"].to(DEV)))[:, :, None]   # [B, T, 1, rot / 2]
    places = torch.arange(r, device=DEV)
    places = places.view(2, r // 2).t() if c["pairs"] == "halves" else places.view(r // 2, 2)  # [pair, 2]

    def rotated(x, by):
        y = x.clone()
        z = torch.complex(x[..., places[:, 0]], x[..., places[:, 1]]) * by
        y[..., places[:, 0]], y[..., places[:, 1]] = z.real, z.imag
        return y

    out = {}
    for name in ("q", "k"):
        x, gain = s[name].double(), s["gain_" + name].double()
        rms = (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt()
        if op == "qk":
            out[name] = rotated(x / rms * gain, turn)
            continue
        dy = rotated(s["g" + name].double(), turn.conj())
        out["rows_" + name] = torch.einsum("bthd,bthd->bd", dy, x / rms)
        dy = dy * gain
        out["d" + name] = dy / rms - x * (dy * x).sum(-1, keepdim=True) / (D * rms ** 3)
    return out
