"""The losses of a masked-LM head trained under DP-SGD, and what the clip needs of them, with their plain forms.

  loss       softmax cross entropy of the tokens X [B, T, d] against the vocabulary table W [V, d] and a bias, with the
             log-sum-exp of every token's logits, which are not kept
  loss_grad  its gradient for X, and every example's squared norm of the gradients of table and bias
  loss_sum   its clipped sum: the table's and the bias' accumulators += sum over the examples of clip_i times their
             gradients
  cross      what the norm of a table shared with the token embedding needs besides: twice the inner product of the
             two parts of an example's gradient
  distill    distillation of full logits from a teacher's top logits at a temperature, loss and gradient

`run` computes them in elementary torch operations, or, where `own` is true, through the package's calls.  `exact` is
the definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of one example over a small vocabulary: a call that is all latency
        {"name": "loss one token", "op": "loss", "dtype": "bf16", "batch": 1, "tokens": 1, "d": 64, "vocab": 1000,
         "bias": True, "ragged": False},
        # the microbatch of the BERT-Large stack: 20 masked positions of 128, the whole word-piece table
        {"name": "loss BERT-Large", "op": "loss", "dtype": "bf16", "batch": 256, "tokens": 20, "d": 1024, "vocab": 30522,
         "bias": True, "ragged": False},
        # a small fp32 model of odd sizes, examples with different numbers of masked positions
        {"name": "loss odd fp32", "op": "loss", "dtype": "fp32", "batch": 7, "tokens": 37, "d": 100, "vocab": 5003,
         "bias": True, "ragged": True},
        # the same microbatch, backward
        {"name": "loss_grad BERT-Large", "op": "loss_grad", "dtype": "bf16", "batch": 256, "tokens": 20, "d": 1024,
         "vocab": 30522, "bias": True, "ragged": False},
        {"name": "loss_grad odd fp32", "op": "loss_grad", "dtype": "fp32", "batch": 7, "tokens": 37, "d": 100,
         "vocab": 5003, "bias": True, "ragged": True},
        # its clipped sum into the accumulators
        {"name": "loss_sum BERT-Large", "op": "loss_sum", "dtype": "bf16", "batch": 256, "tokens": 20, "d": 1024,
         "vocab": 30522, "bias": True, "ragged": False},
        # a few long examples with a loss at every position, padded, at BERT-Base's width
        {"name": "loss_sum long ragged", "op": "loss_sum", "dtype": "bf16", "batch": 4, "tokens": 512, "d": 768,
         "vocab": 30522, "bias": False, "ragged": True},
        # the shared table's cross term of a small model, and of the BERT-Large microbatch
        {"name": "cross small", "op": "cross", "dtype": "fp32", "batch": 8, "tokens": 5, "inputs": 33, "d": 64,
         "vocab": 1000, "bias": True, "ragged": True},
        {"name": "cross BERT-Large", "op": "cross", "dtype": "bf16", "batch": 256, "tokens": 20, "inputs": 128, "d": 1024,
         "vocab": 30522, "bias": True, "ragged": False},
        # the masked positions of one example
        {"name": "distill one example", "op": "distill", "dtype": "bf16", "batch": 1, "tokens": 20, "vocab": 30522, "k": 32,
         "temperature": 2.0, "ragged": False},
        # odd sizes in fp32
        {"name": "distill odd fp32", "op": "distill", "dtype": "fp32", "batch": 13, "tokens": 77, "vocab": 5003, "k": 7,
         "temperature": 1.0, "ragged": True},
        # every position of the long-sequence microbatch
        {"name": "distill every position", "op": "distill", "dtype": "bf16", "batch": 64, "tokens": 512, "vocab": 30522,
         "k": 64, "temperature": 2.0, "ragged": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("loss", "loss_grad", "loss_sum", "cross", "distill"))
    c = {"op": op, "dtype": rng.choice(("fp32", "bf16")), "vocab": _log_int(rng, 40, 50000), "ragged": rng.random() < 0.5}
    if op == "distill":
        c["tokens"] = _log_int(rng, 1, 512)
        c["batch"] = _log_int(rng, 1, max(1, min(256, 400_000_000 // (c["tokens"] * c["vocab"]))))
        c["k"] = rng.choice((1, 2, _log_int(rng, 3, 32), rng.randint(33, 128)))
        c["k"] = min(c["k"], c["vocab"])
        c["temperature"] = rng.choice((1.0, 2.0, round(rng.uniform(0.5, 8.0), 3)))
        return c
    c["d"] = rng.choice((_log_int(rng, 8, 1024), 8 * _log_int(rng, 1, 128), 64 * rng.randint(1, 16)))
    c["bias"] = rng.random() < 0.5
    c["tokens"] = rng.choice((1, 20, _log_int(rng, 2, 300)))
    most = 5120 * 1024 * 30522 // (c["d"] * c["vocab"] * (6 if c["dtype"] == "fp32" else 1))
    c["batch"] = _log_int(rng, 1, max(1, min(256, most // c["tokens"], 8192 // c["tokens"])))
    if op == "cross":
        c["inputs"] = rng.choice((c["tokens"], _log_int(rng, 1, 512)))
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _lse(x, weight, bias):
    z = x.double() @ weight.double().t()
    return torch.logsumexp(z if bias is None else z + bias, -1).float()


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def ids(*shape):                           # word-pieces, the frequent ones first
        return (case["vocab"] ** torch.rand(*shape, generator=g, device=DEV, dtype=torch.float64)).int() - 1

    op, B, T, V = (case[k] for k in ("op", "batch", "tokens", "vocab"))
    dtype = DTYPES[case["dtype"]]
    s = {"case": case}
    # masked positions of each example, and the weights that make an example's loss their mean
    count = torch.full((B, 1), T, device=DEV)
    if case["ragged"]:
        count = torch.randint(max(1, T // 4), T + 1, (B, 1), generator=g, device=DEV)
    live = torch.arange(T, device=DEV) < count
    s["token_weights"] = (1.0 / count.float()).expand(B, T).contiguous()
    if op == "distill":
        k = case["k"]
        logits = torch.empty(B, T, V, dtype=dtype, device=DEV)
        s["top_ids"] = torch.empty(B, T, k, dtype=torch.int32, device=DEV)
        s["top_logits"] = torch.empty(B, T, k, device=DEV)
        for i in range(B):                     # the teacher agrees with the student in part
            z = 2.0 * normal(T, V)
            logits[i] = z
            top, at = (z + 2.0 * normal(T, V)).topk(k, -1)
            s["top_logits"][i], s["top_ids"][i] = top, at.int()
        if case["ragged"]:                     # positions without a teacher were never written
            s["top_ids"].masked_fill_(~live[..., None], -1)
            logits.masked_fill_(~live[..., None], float("nan"))
        s["logits"] = logits
        return s
    d = case["d"]
    s["weight"] = (normal(V, d) * (2.0 / math.sqrt(d))).to(dtype)
    s["bias"] = normal(V) if case["bias"] else None
    s["labels"] = ids(B, T)
    # the better the model knows a position, the more its state points along its word-piece's row
    known = 4.0 * torch.rand(B, T, 1, generator=g, device=DEV)
    s["x"] = (normal(B, T, d) + known * s["weight"].float()[s["labels"].long()]).to(dtype)
    s["lse"] = None if op == "loss" else _lse(s["x"].view(B * T, d), s["weight"], s["bias"]).view(B, T)
    if case["ragged"]:
        s["labels"].masked_fill_(~live, -1)
        s["x"].masked_fill_(~live[..., None], float("nan"))
    if op == "loss_sum":
        s["clip"] = torch.rand(B, generator=g, device=DEV)
        s["acc_w"], s["acc_b"] = 1e-3 * normal(V, d), 1e-3 * normal(V)
    if op == "cross":
        s["ids"] = ids(B, case["inputs"])
        s["g_emb"] = (normal(B, case["inputs"], d) * (0.3 / math.sqrt(d))).to(dtype)
        s["sqnorm"] = 1.0 + torch.rand(B, generator=g, device=DEV)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_logits(s):
    """X in 32 bits with zeros at the positions without a label, which of them have one, and the logits [B, T, V]."""
    live = s["labels"] >= 0
    x = torch.where(live[..., None], s["x"].float(), 0.0)
    z = x @ s["weight"].float().t()
    return x, live, z if s["bias"] is None else z.add_(s["bias"])


def _plain_loss(s):
    _, live, z = _plain_logits(s)
    most = z.amax(-1, keepdim=True)
    lse = (z - most).exp_().sum(-1).log() + most[..., 0]
    at = z.gather(-1, s["labels"].clamp(min=0).long()[..., None])[..., 0]
    return {"loss": torch.where(live, s["token_weights"] * (lse - at), 0.0), "lse": torch.where(live, lse, 0.0)}


def _plain_gradient(s):
    """X and the gradient of the logits, [B, T, V]."""
    x, live, z = _plain_logits(s)
    G = z.sub_(s["lse"][..., None]).exp_()
    at = s["labels"].clamp(min=0).long()[..., None]
    G.scatter_add_(-1, at, torch.full(at.shape, -1.0, device=DEV))
    return x, G.mul_(torch.where(live, s["token_weights"], 0.0)[..., None])


def _plain_loss_grad(s):
    x, G = _plain_gradient(s)
    dx = (G @ s["weight"].float()).to(s["x"].dtype)
    x, G = x.double(), G.double()              # one large square and a vocabulary of small ones in each sum
    both = (x @ x.transpose(1, 2) + (0.0 if s["bias"] is None else 1.0)) * (G @ G.transpose(1, 2))
    return {"dx": dx, "sqnorm": both.sum((1, 2)).float()}


def _plain_loss_sum(s):
    x, G = _plain_gradient(s)
    G = G.mul_(s["clip"][:, None, None]).flatten(0, 1)
    s["acc_w"].addmm_(G.t(), x.flatten(0, 1))
    if s["bias"] is not None:
        s["acc_b"].add_(G.sum(0))
    return {"acc_w": s["acc_w"], "acc_b": s["acc_b"]}


def _plain_cross(s):
    live = s["labels"] >= 0
    x = torch.where(live[..., None], s["x"].float(), 0.0)
    z = x @ s["weight"][s["ids"].long()].float().transpose(1, 2)              # [B, T, inputs]
    if s["bias"] is not None:
        z = z + s["bias"][s["ids"].long()][:, None]
    G = (z - s["lse"][..., None]).exp() - (s["labels"][..., None] == s["ids"][:, None]).float()
    G = G * torch.where(live, s["token_weights"], 0.0)[..., None]
    return s["sqnorm"] + 2.0 * (G * (x @ s["g_emb"].float().transpose(1, 2))).sum((1, 2))


def _plain_distill(s):
    c, tau = s["case"], s["case"]["temperature"]
    given = s["top_ids"] >= 0
    live = given.any(-1, keepdim=True)
    z = torch.where(live, s["logits"].float() / tau, 0.0)
    most = z.amax(-1, keepdim=True)
    p = (z - most).exp_()
    total = p.sum(-1, keepdim=True)
    t = torch.where(given, s["top_logits"] / tau, float("-inf"))
    t = torch.where(live, t - t.amax(-1, keepdim=True), float("-inf"))
    q = t.exp()
    mass = q.sum(-1, keepdim=True).clamp(min=1.0)                              # at least exp(0); 1 where there is none
    q = q / mass
    at = s["top_ids"].clamp(min=0).long()
    gap = torch.where(q > 0, t - mass.log() - z.gather(-1, at) + most + total.log(), 0.0)
    w = torch.where(live[..., 0], s["token_weights"], 0.0)
    dz = (p.div_(total)).scatter_add_(-1, at, -q).mul_(w[..., None] * tau)
    return {"loss": w * (tau * tau) * (q * gap).sum(-1), "dlogits": dz.to(DTYPES[c["dtype"]])}


_PLAIN = {"loss": _plain_loss, "loss_grad": _plain_loss_grad, "loss_sum": _plain_loss_sum, "cross": _plain_cross,
          "distill": _plain_distill}


# ---- the package's calls --------------------------------------------------------------------------------------------
def _own_head(dp, s):
    head = dp.VocabHead(s["x"], s["weight"], s["labels"], bias=s["bias"], token_weights=s["token_weights"])
    return head, torch.empty(dp.dp_vocab_workspace_bytes(head), dtype=torch.uint8, device=DEV)


def _own_loss(s):
    import paper_2108_01624_b200 as dp
    head, work = _own_head(dp, s)
    loss, lse = (torch.empty(s["labels"].shape, dtype=torch.float32, device=DEV) for _ in range(2))
    dp.dp_vocab_loss(head, loss, lse, workspace=work)
    return {"loss": loss, "lse": lse}


def _own_loss_grad(s):
    import paper_2108_01624_b200 as dp
    head, work = _own_head(dp, s)
    dx = torch.empty(s["x"].shape, dtype=s["x"].dtype, device=DEV)
    sqnorm = torch.empty(s["case"]["batch"], dtype=torch.float32, device=DEV)
    dp.dp_vocab_loss_backward(head, s["lse"], dx, sqnorm, workspace=work)
    return {"dx": dx, "sqnorm": sqnorm}


def _own_loss_sum(s):
    import paper_2108_01624_b200 as dp
    head, work = _own_head(dp, s)
    dp.dp_vocab_loss_clipped_accumulate(head, s["lse"], s["clip"], s["acc_w"], s["acc_b"] if s["case"]["bias"] else None,
                                        workspace=work)
    return {"acc_w": s["acc_w"], "acc_b": s["acc_b"]}


def _own_cross(s):
    import paper_2108_01624_b200 as dp
    head, work = _own_head(dp, s)
    sqnorm = s["sqnorm"].clone()
    dp.dp_vocab_loss_cross_sqnorms(head, s["lse"], s["ids"], s["g_emb"], sqnorm, workspace=work)
    return sqnorm


def _own_distill(s):
    import paper_2108_01624_b200 as dp
    loss = torch.empty(s["top_ids"].shape[:2], dtype=torch.float32, device=DEV)
    dlogits = torch.empty(s["logits"].shape, dtype=s["logits"].dtype, device=DEV)
    dp.dp_distill_loss(s["logits"], s["top_ids"], s["top_logits"], s["case"]["temperature"], loss, dlogits,
                       token_weights=s["token_weights"])
    return {"loss": loss, "dlogits": dlogits}


_OWN = {"loss": _own_loss, "loss_grad": _own_loss_grad, "loss_sum": _own_loss_sum, "cross": _own_cross,
        "distill": _own_distill}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    op, V, size = case["op"], case["vocab"], DTYPES[case["dtype"]].itemsize
    n = case["batch"] * case["tokens"]
    if case["ragged"]:
        n = max(1, n * 5 // 8)                 # mean share of counts between a quarter and the whole
    if op == "distill":
        return {"bytes": 2 * size * n * V + 8 * n * case["k"] + 8 * n, "flops": 4 * n * V}
    d, B = case["d"], case["batch"]
    inputs = size * (n * d + V * d) + (4 * V if case["bias"] else 0) + 8 * n
    product = 2 * n * V * d
    if op == "loss":
        return {"bytes": inputs + 8 * n, "flops": product}
    if op == "loss_grad":                      # the logits again, the gradient of X, and the products of an example's tokens
        return {"bytes": inputs + 4 * n + size * n * d + 4 * B, "flops": 2 * product + 2 * n * (V + d)}
    if op == "loss_sum":                       # the logits again, and the sum
        return {"bytes": inputs + 4 * n + 4 * B + 8 * V * (d + (1 if case["bias"] else 0)), "flops": 2 * product}
    m = B * case["inputs"]
    rows = min(V, m)                           # rows of the table that the inputs name, at most
    return {"bytes": size * (n * d + rows * d + m * d) + 4 * m + 12 * n + 8 * B, "flops": 4 * n * case["inputs"] * d}


# ---- definitions in 64 bits -----------------------------------------------------------------------------------------
def _exact_head(s):
    """Tokens with a label as rows: their states, examples, weights, labels, logits."""
    B, T = s["labels"].shape
    rows = torch.nonzero(s["labels"].flatten() >= 0)[:, 0]
    x = s["x"].flatten(0, 1)[rows].double()
    z = torch.einsum("nd,vd->nv", x, s["weight"].double())
    if s["bias"] is not None:
        z += s["bias"].double()
    return rows, rows // T, x, s["token_weights"].flatten()[rows].double(), s["labels"].flatten()[rows].long(), z


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    B, T = case["batch"], case["tokens"]
    if op == "distill":
        tau = case["temperature"]
        if B * T * case["vocab"] > 400_000_000:
            return None
        loss = torch.zeros(B, T, dtype=torch.float64, device=DEV)
        dz = torch.zeros(s["logits"].shape, dtype=torch.float64, device=DEV)
        for i in range(B):
            rows = torch.nonzero((s["top_ids"][i] >= 0).any(-1))[:, 0]
            logp = torch.log_softmax(s["logits"][i, rows].double() / tau, -1)
            logq = torch.log_softmax(s["top_logits"][i, rows].double() / tau, -1)
            at, w = s["top_ids"][i, rows].long(), s["token_weights"][i, rows].double()
            loss[i, rows] = w * tau ** 2 * (logq.exp() * (logq - torch.take_along_dim(logp, at, -1))).sum(-1)
            q = torch.zeros_like(logp).scatter_(-1, at, logq.exp())
            dz[i, rows] = (w * tau)[:, None] * (logp.exp() - q)
        return {"loss": loss, "dlogits": dz}
    rows, of, x, w, labels, z = _exact_head(s)
    if op == "loss":
        lse = torch.logsumexp(z, -1)
        out = {k: torch.zeros(B * T, dtype=torch.float64, device=DEV) for k in ("loss", "lse")}
        out["lse"][rows] = lse
        out["loss"][rows] = w * (lse - torch.take_along_dim(z, labels[:, None], -1)[:, 0])
        return {k: v.view(B, T) for k, v in out.items()}
    lse = s["lse"].flatten()[rows].double()
    if op == "cross":
        sqnorm = s["sqnorm"].double()
        for i in range(B):
            mine = torch.nonzero(of == i)[:, 0]
            at = s["ids"][i].long()
            G = (z[mine][:, at] - lse[mine, None]).exp() - (labels[mine, None] == at).double()
            table = (G * w[mine, None]).t() @ x[mine]                          # what the projection adds to the inputs' rows
            sqnorm[i] += 2.0 * (table * s["g_emb"][i].double()).sum()
        return sqnorm
    G = (z - lse[:, None]).exp()
    G[torch.arange(len(rows), device=DEV), labels] -= 1.0
    G *= w[:, None]
    if op == "loss_sum":
        c = s["clip"].double()[of]
        acc_w = s["acc_w"].double() + torch.einsum("nv,nd->vd", G, x * c[:, None])
        acc_b = s["acc_b"].double()
        return {"acc_w": acc_w, "acc_b": acc_b + torch.einsum("nv,n->v", G, c) if case["bias"] else acc_b}
    dx = torch.zeros(B * T, case["d"], dtype=torch.float64, device=DEV)
    dx[rows] = G @ s["weight"].double()
    sqnorm = torch.zeros(B, dtype=torch.float64, device=DEV)
    for i in range(B):
        mine = torch.nonzero(of == i)[:, 0]
        sqnorm[i] = (G[mine].t() @ x[mine]).pow(2).sum()
        if case["bias"]:
            sqnorm[i] += G[mine].sum(0).pow(2).sum()
    return {"dx": dx.view(B, T, -1), "sqnorm": sqnorm}
