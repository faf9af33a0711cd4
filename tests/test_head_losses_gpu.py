"""The vocabulary head's losses on the GPU against their definitions in 64 bits, with bounds from the arithmetic:
  a product of bf16 numbers is exact in fp32; the tensor cores' sums drop less than 2^-23 of the terms' absolute sum at each step
  of 16, so a logit is off by dz = (steps + 4) 2^-23 sum |x w| (fp32: six products' steps, and 2^-22 for what three bf16 numbers leave);
  an exponential is off by dz + 2^-20 of itself; G at the label, formed in fp64, by 2^-20 of itself;
  G is read as hi + lo (2^-16 of it), as hi alone for a bf16 dX (2^-8); fp32 X and W as two numbers there (2^-16);
  sums of G take at most 2^-15 of their absolute sum (a part of 128 steps, then fp32); results are rounded once."""
import math

import pytest
import torch

import paper_2108_01624_b200 as dp

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def workspace(head):
    """All bytes 255: what is read before it is written shows as NaN."""
    return torch.full((dp.dp_vocab_workspace_bytes(head),), 255, dtype=torch.uint8, device=DEV)


class Case:
    """A head, what the calls need, and the definition in 64 bits with the bounds above."""

    def __init__(self, B, T, d, V, dtype, bias=True, weights=True, dead=0.3, seed=0, sure=0.0, pad_x=0, pad_w=0, scale=2.0):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def normal(*s):
            return torch.randn(*s, generator=g, device=DEV)
        self.B, self.T, self.d, self.V, self.dtype = B, T, d, V, dtype
        self.weight = torch.zeros(V, d + pad_w, dtype=dtype, device=DEV)[:, :d]
        self.weight.copy_(normal(V, d) * (scale / math.sqrt(d)))
        self.labels = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
        self.x = torch.zeros(B, T, d + pad_x, dtype=dtype, device=DEV)[..., :d]
        self.x.copy_(normal(B, T, d) + sure * self.weight.float()[self.labels.long()])
        self.live = torch.rand(B, T, generator=g, device=DEV) >= dead
        self.labels[~self.live] = -1
        self.x[~self.live] = float("nan")
        self.bias = normal(V) if bias else None
        self.tw = torch.rand(B, T, generator=g, device=DEV) + 0.1 if weights else None
        self.clip = torch.rand(B, generator=g, device=DEV)
        self.define()

    def define(self):
        f32 = self.dtype == F32
        self.xd = torch.where(self.live[..., None], self.x.double(), 0.0)
        w = self.weight.double()
        self.z = self.xd @ w.t()
        steps = (6 if f32 else 1) * -(-self.d // 16) + 4
        size = self.xd.abs() @ w.abs().t()
        self.dz = steps * 2.0 ** -23 * size + (2.0 ** -22 * size if f32 else 0.0)
        if self.bias is not None:
            self.z = self.z + self.bias.double()
            self.dz = self.dz + 2.0 ** -23 * self.bias.double().abs().nan_to_num(posinf=0.0)
        self.lse64 = torch.logsumexp(self.z, -1)
        self.lse = torch.where(self.live, self.lse64, 0.0).float()
        at = self.labels.clamp(min=0).long()[..., None]
        self.w = torch.where(self.live, torch.ones_like(self.lse64) if self.tw is None else self.tw.double(), 0.0)
        others = torch.logsumexp(self.z.scatter(-1, at, float("-inf")), -1)
        self.loss = torch.where(self.live, self.w * torch.nn.functional.softplus(others - self.z.gather(-1, at)[..., 0], threshold=1e6), 0.0)
        p = (self.z - self.lse.double()[..., None]).exp()
        y = torch.zeros_like(p).scatter_(-1, at, 1.0)
        self.G = self.w[..., None] * (p - y)
        self.dG = torch.where(y > 0, self.G.abs() * 2.0 ** -20, self.w[..., None] * p * (self.dz.expm1() + 2.0 ** -20))

    def head(self, **kw):
        return dp.VocabHead(kw.get("x", self.x), self.weight, self.labels, bias=self.bias, token_weights=self.tw)

    def check_loss(self):
        head = self.head()
        loss, lse = (torch.full((self.B, self.T), float("nan"), device=DEV) for _ in range(2))
        dp.dp_vocab_loss(head, loss, lse, workspace=workspace(head))
        dz = torch.where(self.live[..., None], self.dz, 0.0).amax(-1)
        assert torch.equal(loss[~self.live], torch.zeros_like(loss[~self.live])) and torch.equal(lse[~self.live], torch.zeros_like(lse[~self.live]))
        err = (lse.double() - torch.where(self.live, self.lse64, 0.0)).abs()
        assert bool((err <= torch.where(self.live, dz + 2.0 ** -20 + 2.0 ** -23 * self.lse64.abs(), 0.0)).all()), float(err.max())
        err = (loss.double() - self.loss).abs()                        # relative to the loss, however small: softplus' <= softplus
        assert bool((err <= self.loss * (1.01 * dz + 2.0 ** -19) + 1e-37).all()), float((err / self.loss).nan_to_num().max())

    def check_backward(self, sq0=None, out=None):
        head, f32 = self.head(), self.dtype == F32
        dx = torch.full_like(self.x, float("nan")) if out is None else out
        sq = torch.full((self.B,), float("nan"), device=DEV) if sq0 is None else sq0.clone()
        dp.dp_vocab_loss_backward(head, self.lse, dx, sq, accumulate_into=sq0 is not None, workspace=workspace(head))
        w, G = self.weight.double(), self.G
        ref = G @ w
        r = 2 * 2.0 ** -16 if f32 else 2.0 ** -8
        tol = self.dG @ w.abs() + (r + 2.0 ** -15) * (G.abs() @ w.abs()) + (2.0 ** -24 if f32 else 2.0 ** -8) * ref.abs()
        err = (dx.double() - ref).abs()
        assert bool((err <= 1.02 * tol + 1e-37).all()), float((err / tol).nan_to_num().max())
        one = 0.0 if self.bias is None else 1.0
        K, Ka = self.xd @ self.xd.transpose(1, 2) + one, self.xd.abs() @ self.xd.abs().transpose(1, 2) + one
        Q, Qa = G @ G.transpose(1, 2), G.abs() @ G.abs().transpose(1, 2)
        ref = (K * Q).sum((1, 2)) + (0.0 if sq0 is None else sq0.double())
        half = self.dG @ G.abs().transpose(1, 2)
        tol = (Ka * (half + half.transpose(1, 2)) + ((4 if f32 else 2) * 2.0 ** -16 + 2.0 ** -14) * Ka * Qa).sum((1, 2)) + 2.0 ** -22 * ref
        err = (sq.double() - ref).abs()
        assert bool((err <= 1.02 * tol + 1e-37).all()), float((err / tol).nan_to_num().max())
        return dx, sq

    def check_sum(self):
        head, f32 = self.head(), self.dtype == F32
        g = torch.Generator(device=DEV).manual_seed(9)
        acc_w, acc_b = torch.randn(self.V, self.d, generator=g, device=DEV), torch.randn(self.V, generator=g, device=DEV)
        w0, b0 = acc_w.double(), acc_b.double()
        dp.dp_vocab_loss_clipped_accumulate(head, self.lse, self.clip, acc_w, acc_b if self.bias is not None else None, workspace=workspace(head))
        c = self.clip.double()[:, None, None]
        G, dG, x = (c * self.G).flatten(0, 1), (c * self.dG).flatten(0, 1), self.xd.flatten(0, 1)
        ref = w0 + G.t() @ x
        tol = dG.t() @ x.abs() + ((2 if f32 else 1) * 2.0 ** -16 + 2.0 ** -15) * (G.abs().t() @ x.abs()) + 2.0 ** -23 * (w0.abs() + ref.abs())
        err = (acc_w.double() - ref).abs()
        assert bool((err <= 1.02 * tol).all()), float((err / tol).max())
        ref, tol = b0, torch.zeros_like(b0)
        if self.bias is not None:
            ref = b0 + G.sum(0)
            tol = dG.sum(0) + 2.0 ** -18 * G.abs().sum(0) + 2.0 ** -23 * (b0.abs() + ref.abs())
        err = (acc_b.double() - ref).abs()
        assert bool((err <= 1.02 * tol).all()), float((err / tol).nan_to_num().max())
        return acc_w, acc_b

    def check_cross(self, Tu, seed=3):
        g = torch.Generator(device=DEV).manual_seed(seed)
        ids = torch.randint(0, self.V, (self.B, Tu), generator=g, device=DEV, dtype=torch.int32)
        ids[:, :min(Tu, self.T)] = torch.where(self.labels >= 0, self.labels, 0)[:, :min(Tu, self.T)]     # words that are labels too
        e = torch.randn(self.B, Tu, self.d, generator=g, device=DEV).to(self.dtype)
        sq0 = torch.rand(self.B, generator=g, device=DEV)
        sq, head = sq0.clone(), self.head()
        dp.dp_vocab_loss_cross_sqnorms(head, self.lse, ids, e, sq, workspace=workspace(head))
        at = ids.long()[:, None].expand(self.B, self.T, Tu)
        G, dG = self.G.gather(-1, at), self.dG.gather(-1, at)
        # here z at a label is a tensor-core sum like the others
        dG = torch.maximum(dG, self.w[..., None] * (self.z.gather(-1, at) - self.lse.double()[..., None]).exp() * (self.dz.gather(-1, at).expm1() + 2.0 ** -20))
        k, ka = self.xd @ e.double().transpose(1, 2), self.xd.abs() @ e.double().abs().transpose(1, 2)
        dk = ((6 if self.dtype == F32 else 1) * -(-self.d // 16) + 8) * 2.0 ** -23 * ka
        ref = sq0.double() + 2.0 * (G * k).sum((1, 2))
        tol = 2.0 * (dG * k.abs() + (G.abs() + dG) * dk + 2.0 ** -19 * (G * k).abs()).sum((1, 2)) + 2.0 ** -22 * (sq0.double() + ref.abs())
        err = (sq.double() - ref).abs()
        assert bool((err <= 1.02 * tol).all()), float((err / tol).max())


# one word, one token; words that do not fill a tile; rows that do not fill 16 bytes; 3 blocks of G; examples of 41 tokens (82 rows of
# planes: one a CTA), 70 (140 rows: the layers' kernels), a long one (their tiles, and column sums for the bias); many tiles;
# one tile of two K blocks left over for eleven pairs
SHAPES = [(1, 1, 8, 1), (1, 1, 64, 1000), (2, 3, 17, 5), (3, 20, 64, 257), (7, 20, 128, 511), (4, 5, 200, 7), (5, 41, 72, 4500),
          (2, 70, 40, 300), (2, 700, 64, 300), (40, 20, 264, 2050), (3, 2, 1024, 777), (6, 20, 16, 5821)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_loss_gradient_sum_and_cross_term(shape, dtype):
    c = Case(*shape, dtype, bias=shape[2] != 40, weights=shape[3] != 5)
    c.check_loss()
    c.check_backward()
    c.check_sum()
    c.check_cross(9)
    c.check_cross(150, seed=4)
    assert dp.dp_poll_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_token_dead_and_every_token_alive(dtype):
    for dead in (1.1, 0.0):
        c = Case(3, 7, 48, 100, dtype, dead=dead)
        c.check_loss()
        dx, sq = c.check_backward(sq0=torch.rand(3, device=DEV) if dead else None)
        acc_w, acc_b = c.check_sum()
        if dead > 1.0:
            assert bool((dx == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sure_tokens_keep_their_relative_error(dtype):
    """Losses of 1e-3 to 1e-12, and gradients as small beside the ones they are differences of."""
    c = Case(4, 16, 256, 500, dtype, sure=6.0, dead=0.1, bias=False)
    assert 0 < float(c.loss[c.live].min()) < 1e-6
    c.check_loss()
    c.check_backward()
    c.check_sum()


@pytest.mark.parametrize("dtype, pad_x, pad_w", [(BF16, 8, 16), (BF16, 3, 0), (BF16, 0, 5), (F32, 4, 4), (F32, 1, 3)])
def test_rows_with_gaps(dtype, pad_x, pad_w):
    c = Case(3, 9, 64, 300, dtype, pad_x=pad_x, pad_w=pad_w)
    c.check_loss()
    wide = torch.full((3, 9, 64 + 5), 7.0, dtype=dtype, device=DEV)
    c.check_backward(out=wide[..., 2:66])
    assert bool((wide[..., :2] == 7).all()) and bool((wide[..., 66:] == 7).all())
    c.check_sum()
    c.check_cross(4)
    # a view that starts anywhere
    x = torch.zeros(3 * 9 * 64 + 1, dtype=dtype, device=DEV)[1:].view(3, 9, 64)
    x.copy_(c.x)
    loss, lse = torch.empty(3, 9, device=DEV), torch.empty(3, 9, device=DEV)
    again = torch.empty(3, 9, device=DEV)
    h1, h2 = c.head(), c.head(x=x)
    dp.dp_vocab_loss(h1, again, lse, workspace=workspace(h1))
    dp.dp_vocab_loss(h2, loss, lse, workspace=workspace(h2))
    assert torch.allclose(loss, again, rtol=1e-5)


def test_words_that_cannot_occur():
    c = Case(2, 9, 64, 700, BF16, dead=0.2)
    banned = torch.arange(700, device=DEV) % 3 == 0
    banned[256:512] = True                        # a whole tile of them
    c.bias[banned] = float("-inf")
    free = (~banned).nonzero()[:, 0]
    c.labels = torch.where(c.live, free[torch.randint(0, len(free), c.labels.shape, device=DEV)].int(), -1)
    c.define()
    c.dz = torch.where(banned, 0.0, c.dz)
    c.dG = torch.where(banned, 0.0, c.dG)
    c.check_loss()
    c.check_backward()
    acc_w, acc_b = c.check_sum()
    # a label that cannot occur: an infinite loss, and still finite gradients (p = 0, G = -w)
    i, t = c.live.nonzero()[0].tolist()
    c.labels[i, t] = 0
    loss, lse = torch.empty(2, 9, device=DEV), torch.empty(2, 9, device=DEV)
    head = c.head()
    ws = workspace(head)
    dp.dp_vocab_loss(head, loss, lse, workspace=ws)
    assert float(loss[i, t]) == math.inf and bool(lse.isfinite().all()) and bool(loss.flatten().isinf().sum() == 1)
    dx = torch.empty_like(c.x)
    dp.dp_vocab_loss_backward(head, lse, dx, None, workspace=ws)
    assert bool(dx.isfinite().all())


def test_values_that_are_not_numbers_show_and_stay_with_their_token():
    c = Case(2, 5, 64, 300, BF16, dead=0.0)
    c.x[0, 1, 3], c.x[1, 2, 0] = float("nan"), float("inf")
    head = c.head()
    ws, loss, lse = workspace(head), torch.empty(2, 5, device=DEV), torch.empty(2, 5, device=DEV)
    dp.dp_vocab_loss(head, loss, lse, workspace=ws)
    bad = torch.zeros(2, 5, dtype=torch.bool, device=DEV)
    bad[0, 1] = bad[1, 2] = True
    assert bool((loss.isnan() == bad).all()) and bool((lse.isnan() == bad).all())
    dx, sq = torch.empty_like(c.x), torch.empty(2, device=DEV)
    dp.dp_vocab_loss_backward(head, lse, dx, sq, workspace=ws)
    assert bool((dx.isnan().all(-1) == bad).all()) and bool(sq.isnan().all())


def test_labels_and_ids_beyond_the_vocabulary_are_reported_and_left_out():
    c = Case(2, 6, 64, 300, F32, dead=0.0)
    c.labels[0, 2], c.live[0, 2] = -1, False
    c.x[0, 2] = float("nan")
    c.define()
    c.labels[0, 2] = 300
    assert dp.dp_poll_status() == 0
    c.check_loss()
    assert dp.dp_poll_status() == -7
    c.check_backward()
    assert dp.dp_poll_status() == -7
    c.check_sum()
    assert dp.dp_poll_status() == -7
    c.labels[0, 2] = -1
    head, e, sq = c.head(), torch.randn(2, 4, 64, device=DEV), torch.zeros(2, device=DEV)
    ids = torch.tensor([[1, -1, 2, 300], [3, 4, 5, 6]], dtype=torch.int32, device=DEV)
    e[0, 1] = e[0, 3] = float("nan")
    dp.dp_vocab_loss_cross_sqnorms(head, c.lse, ids, e, sq, workspace=workspace(head))
    assert dp.dp_poll_status() == -7 and bool(sq.isfinite().all())
    good, sq2 = ids.clone(), torch.zeros(2, device=DEV)
    good[0, 1] = good[0, 3] = 0
    e[0, 1] = e[0, 3] = 0.0
    dp.dp_vocab_loss_cross_sqnorms(head, c.lse, good, e, sq2, workspace=workspace(head))
    assert dp.dp_poll_status() == 0 and torch.allclose(sq, sq2, rtol=1e-5, atol=1e-6)


def test_gradient_against_differences_of_the_loss():
    c = Case(2, 6, 40, 90, F32, dead=0.2, seed=5)
    x0 = torch.where(c.live[..., None], c.x, 0.0)
    c.x.copy_(x0)
    head = c.head()
    ws, loss, lse, dx = workspace(head), torch.empty(2, 6, device=DEV), torch.empty(2, 6, device=DEV), torch.empty_like(c.x)

    def total(x):
        c.x.copy_(x)
        dp.dp_vocab_loss(head, loss, lse, workspace=ws)
        return float(loss.double().sum())
    total(x0)
    dp.dp_vocab_loss_backward(head, lse, dx, None, workspace=ws)
    g = torch.Generator(device=DEV).manual_seed(1)
    for _ in range(4):
        u = torch.randn(x0.shape, generator=g, device=DEV)
        h = 2.0 ** -6
        num, ana = (total(x0 + h * u) - total(x0 - h * u)) / (2 * h), float((dx.double() * u.double()).sum())
        # third differences h^2/6 |u|^3-ish (below 2^-12 of the scale) and losses to 2^-19 of theirs over 2 h
        scale = float((dx.double().abs() * u.double().abs()).sum())
        assert abs(num - ana) <= 2.0 ** -8 * scale + 2.0 ** -19 * float(loss.double().sum()) / h


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norms_are_those_of_single_examples_sums(dtype):
    """|c_i g_i| from the clipped sum of one example alone, against sqrt(sqnorm_i): what the clip relies on."""
    c = Case(3, 11, 72, 600, dtype)
    _, sq = c.check_backward()
    for i in range(3):
        head = dp.VocabHead(c.x[i:i + 1], c.weight, c.labels[i:i + 1], bias=c.bias, token_weights=c.tw[i:i + 1])
        acc_w, acc_b = torch.zeros(600, 72, device=DEV), torch.zeros(600, device=DEV)
        dp.dp_vocab_loss_clipped_accumulate(head, c.lse[i:i + 1], torch.ones(1, device=DEV), acc_w, acc_b, workspace=workspace(head))
        n = float(acc_w.double().pow(2).sum() + acc_b.double().pow(2).sum())
        assert abs(n - float(sq[i])) <= 2.0 ** -12 * n


def test_runs_repeat_bit_by_bit():
    c = Case(40, 20, 264, 2050, BF16)
    first = None
    for _ in range(3):
        head = c.head()
        ws = workspace(head)
        ws.random_()
        loss, lse = torch.empty(40, 20, device=DEV), torch.empty(40, 20, device=DEV)
        dx, sq = torch.empty_like(c.x), torch.empty(40, device=DEV)
        acc_w, acc_b = torch.ones(2050, 264, device=DEV), torch.ones(2050, device=DEV)
        dp.dp_vocab_loss(head, loss, lse, workspace=ws)
        dp.dp_vocab_loss_backward(head, lse, dx, sq, workspace=ws)
        dp.dp_vocab_loss_clipped_accumulate(head, lse, c.clip, acc_w, acc_b, workspace=ws)
        now = [t.clone() for t in (loss, lse, dx, sq, acc_w, acc_b)]
        assert first is None or all(torch.equal(p, q) for p, q in zip(first, now))
        first = now


def test_several_pieces_of_the_vocabulary():
    """140800 tokens: a block of G is larger than half of what one piece holds, so that two pieces share dX, norms and sums."""
    c = Case(2200, 64, 16, 2100, BF16, dead=0.2)
    c.check_backward()
    c.check_sum()


@pytest.mark.parametrize("d", [64, 24])
def test_cross_term_of_many_examples(d):
    Case(70001, 1, d, 50, BF16, dead=0.2).check_cross(2)


# the widest rows and rows of one element; many short examples, one long; few words and very many; one example a microbatch
EXTREMES = [(2, 3, 65536, 40), (2, 70, 65536, 5), (3, 5, 1, 300), (70000, 1, 8, 9), (9000, 3, 24, 33), (1, 5000, 16, 40), (2, 3, 8, 200003),
            (1, 257, 72, 2049)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", EXTREMES)
def test_the_largest_and_the_smallest_sizes(shape, dtype):
    c = Case(*shape, dtype)
    c.check_loss()
    c.check_backward()
    c.check_sum()
    c.check_cross(5)
    assert dp.dp_poll_status() == 0


def test_a_gradient_without_norms_and_norms_without_a_gradient():
    c = Case(5, 20, 200, 3000, BF16)
    head = c.head()
    dx, sq = c.check_backward()
    one, two = torch.full_like(dx, float("nan")), torch.full_like(sq, float("nan"))
    dp.dp_vocab_loss_backward(head, c.lse, one, None, workspace=workspace(head))
    dp.dp_vocab_loss_backward(head, c.lse, None, two, workspace=workspace(head))
    assert torch.equal(one, dx) and torch.equal(two, sq)


def test_rows_around_a_strided_gradient_stay_as_they_were():
    c = Case(3, 7, 40, 300, BF16)
    whole = torch.full((3, 7, 64), 5.0, dtype=BF16, device=DEV)
    c.check_backward(out=whole[..., 8:48])
    assert bool((whole[..., :8] == 5.0).all()) and bool((whole[..., 48:] == 5.0).all())


def test_parts_of_the_log_sum_exp_are_joined_in_pieces():
    B, T, d, V = 700, 100, 8, 70000
    g = torch.Generator(device=DEV).manual_seed(0)
    x, w = torch.randn(B, T, d, generator=g, device=DEV).bfloat16(), torch.randn(V, d, generator=g, device=DEV).bfloat16()
    y = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
    head = dp.VocabHead(x, w, y)
    loss, lse = torch.empty(B, T, device=DEV), torch.empty(B, T, device=DEV)
    dp.dp_vocab_loss(head, loss, lse, workspace=workspace(head))
    for i in range(0, B, 35):
        z = x[i].double() @ w.double().t()
        ref = torch.logsumexp(z, -1)
        tol = 5 * 2.0 ** -23 * (x[i].double().abs() @ w.double().abs().t()).amax(-1) + 2.0 ** -20 + 2.0 ** -23 * ref.abs()
        assert bool(((lse[i].double() - ref).abs() <= tol).all())
        want = ref - z.gather(-1, y[i].long()[:, None])[:, 0]
        assert bool(((loss[i].double() - want).abs() <= want * (1.01 * tol + 2.0 ** -19)).all())


# ---- distillation -----------------------------------------------------------------------------------------------------
def distill_reference(z, ids, t, tau, w):
    """Loss, gradient, and bounds: exponents to 2^-22 of their size, exponentials to 2^-21, sums of fp32."""
    N, V = z.shape
    given = (ids >= 0) & (t > float("-inf"))
    live = given.any(-1)
    zd = torch.where(live[:, None], z.double() / tau, 0.0)
    logp = torch.log_softmax(zd, -1)
    logq = torch.log_softmax(torch.where(given, t.double() / tau, float("-inf")), -1)
    logq = torch.where(live[:, None], logq, float("-inf"))
    q, at = torch.where(given, logq.exp(), 0.0), ids.clamp(min=0).long()
    gap = torch.where(q > 0, logq - logp.gather(-1, at), 0.0)
    w = torch.where(live, w.double(), 0.0)
    loss = w * tau ** 2 * (q * gap).sum(-1)
    p, scattered = logp.exp(), torch.zeros_like(logp).scatter_add_(-1, at, q)
    c = (w * tau)[:, None]
    size = torch.where(q > 0, logq.abs() + logp.gather(-1, at).abs(), 0.0)
    far = (zd.amax(-1, keepdim=True) - zd).nan_to_num(posinf=0.0)
    tol_loss = w * tau ** 2 * 2.0 ** -18 * (1.0 + (q * size).sum(-1))
    tol = c * (p * (2.0 ** -18 + 2.0 ** -22 * far) + scattered * (2.0 ** -18 + 2.0 ** -22 * size.amax(-1, keepdim=True)))
    return loss, torch.where(live[:, None], c * (p - scattered), 0.0), tol_loss, torch.where(live[:, None], tol, 0.0)


def check_distill(z, ids, t, tau, w, dz):
    N = z.shape[0] * z.shape[1]
    # both are read before the call: it may write in place
    ref = distill_reference(z.reshape(N, -1), ids.reshape(N, -1), t.reshape(N, -1).float(), tau, torch.ones(N, device=DEV) if w is None else w.reshape(N))
    loss = torch.full(z.shape[:2], float("nan"), device=DEV)
    dp.dp_distill_loss(z, ids, t, tau, loss, dz, token_weights=w)
    err = (loss.view(N).double() - ref[0]).abs()
    assert bool((err <= ref[2]).all()), float((err / ref[2]).nan_to_num().max())
    if dz is not None:
        tol = ref[3] + (2.0 ** -24 if z.dtype == F32 else 2.0 ** -8) * ref[1].abs() + 1e-37
        err = (dz.reshape(N, -1).double() - ref[1]).abs()
        assert bool((err <= tol).all()), float((err / tol).max())


def distill_case(B, T, V, K, dtype, teacher=F32, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = (3.0 * torch.randn(B, T, V, generator=g, device=DEV)).to(dtype)
    t = (3.0 * torch.randn(B, T, K, generator=g, device=DEV)).to(teacher)
    ids = torch.randint(0, V, (B, T, K), generator=g, device=DEV, dtype=torch.int32)     # with repetitions
    ids[torch.rand(B, T, K, generator=g, device=DEV) < 0.2] = -1
    ids[0, 0] = -1                                                                        # no teacher at all
    z[0, 0] = float("nan")
    return z, ids, t, torch.rand(B, T, generator=g, device=DEV) + 0.1


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B, T, V, K, tau", [(1, 2, 1, 1, 1.0), (1, 3, 2, 5, 2.0), (5, 7, 40, 3, 1.0), (2, 65, 511, 33, 0.5), (3, 5, 2049, 64, 2.0),
                                             (2, 9, 5003, 7, 4.0), (2, 3, 30522, 128, 2.0), (1, 3, 50001, 1024, 1.5), (1, 2, 130001, 16, 1.0)])
def test_distillation(B, T, V, K, tau, dtype):
    z, ids, t, w = distill_case(B, T, V, K, dtype)
    dz = torch.full_like(z, float("nan"))
    check_distill(z, ids, t, tau, w, dz)
    check_distill(z, ids, t.bfloat16(), tau, None, dz)
    check_distill(z, ids, t, tau, w, None)
    check_distill(z, ids, t, tau, w, z)              # in place
    assert dp.dp_poll_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [37, 3001, 130001])
def test_distillation_of_rows_that_start_anywhere(V, dtype):
    z, ids, t, w = distill_case(3, 4, V, 9, dtype)
    for lead, gap, lead2, gap2 in ((1, 0, 1, 0), (3, 5, 3, 5), (0, 2, 1, 1), (0, 8, 0, 16)):
        a = torch.full((12 * (V + gap) + lead,), float("inf"), dtype=dtype, device=DEV)      # what lies beside the rows must not show
        zv = a[lead:].view(12, V + gap)[:, :V].view(3, 4, V)
        zv.copy_(z)
        o = torch.full((12 * (V + gap2) + lead2,), 5.0, dtype=dtype, device=DEV)
        ov = o[lead2:].view(12, V + gap2)[:, :V].view(3, 4, V)
        check_distill(zv, ids, t, 2.0, w, ov)
        beside = torch.ones_like(o, dtype=torch.bool)
        beside[lead2:].view(12, V + gap2)[:, :V] = False
        assert bool((o[beside] == 5.0).all())


@pytest.mark.parametrize("V", [300, 6000, 130001])
def test_distillation_special_values(V):
    z, ids, t, w = distill_case(1, 6, V, 5, F32)
    ids[0, 1:] = torch.arange(5, dtype=torch.int32, device=DEV)
    t[0, 1] = float("-inf")                                   # a teacher that gives nothing any weight
    t[0, 2, 1:] = float("-inf")                               # one word alone
    z[0, 3, 3] = float("-inf")                                # a word of the teacher's that the student cannot say
    z[0, 4, 100:] = float("-inf")                             # words that cannot occur
    t[0, 5, 2] = float("nan")
    loss, dz = torch.empty(1, 6, device=DEV), torch.empty_like(z)
    dp.dp_distill_loss(z, ids, t, 1.0, loss, dz, token_weights=w)
    assert float(loss[0, 1]) == 0.0 and bool((dz[0, 1] == 0).all())
    assert float(loss[0, 3]) == math.inf and bool(dz[0, 3].isfinite().all())
    assert math.isnan(float(loss[0, 5])) and bool(dz[0, 5, :5].isnan().all())
    keep = [2, 4]
    ref = distill_reference(z[0, keep], ids[0, keep], t[0, keep], 1.0, w[0, keep])
    assert bool(((loss[0, keep].double() - ref[0]).abs() <= ref[2]).all())
    assert bool(((dz[0, keep].double() - ref[1]).abs() <= ref[3] + 2.0 ** -24 * ref[1].abs()).all())
    ids[0, 2, 4] = V                                          # beyond the vocabulary: an empty place, reported
    assert dp.dp_poll_status() == 0
    dp.dp_distill_loss(z, ids, t, 1.0, loss, dz, token_weights=w)
    assert dp.dp_poll_status() == -7
    assert bool(((dz[0, 2].double() - ref[1][0]).abs() <= ref[3][0] + 2.0 ** -24 * ref[1][0].abs()).all())


def test_distillation_gradient_against_differences():
    z, ids, t, w = distill_case(1, 4, 60, 6, F32)
    z[0, 0] = 0.0
    loss, dz = torch.empty(1, 4, device=DEV), torch.empty_like(z)
    dp.dp_distill_loss(z, ids, t, 2.0, loss, dz, token_weights=w)
    g = torch.Generator(device=DEV).manual_seed(2)
    for _ in range(4):
        u, h = torch.randn(z.shape, generator=g, device=DEV), 2.0 ** -5
        up, down = torch.empty(1, 4, device=DEV), torch.empty(1, 4, device=DEV)
        dp.dp_distill_loss(z + h * u, ids, t, 2.0, up, None, token_weights=w)
        dp.dp_distill_loss(z - h * u, ids, t, 2.0, down, None, token_weights=w)
        num, ana = float((up.double() - down.double()).sum()) / (2 * h), float((dz.double() * u.double()).sum())
        assert abs(num - ana) <= 2.0 ** -9 * float((dz.abs() * u.abs()).double().sum()) + 2.0 ** -18 * float(loss.double().sum() + 8) / h


def test_distillation_beyond_32_bits():
    """72000 rows of 30001 words: the last rows lie behind 2^31 elements."""
    N, V = 72000, 30001
    z = torch.empty(1, N, V, dtype=BF16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(0))
    ids = torch.randint(0, V, (1, N, 4), device=DEV, dtype=torch.int32)
    t, loss = torch.randn(1, N, 4, device=DEV), torch.empty(1, N, device=DEV)
    rows = [0, 1, 35000, N - 2, N - 1]
    ref = distill_reference(z[0, rows], ids[0, rows], t[0, rows], 1.0, torch.ones(5, device=DEV))
    dp.dp_distill_loss(z, ids, t, 1.0, loss, z)
    assert bool(((loss[0, rows].double() - ref[0]).abs() <= ref[2]).all())
    assert bool(((z[0, rows].double() - ref[1]).abs() <= ref[3] + 2.0 ** -8 * ref[1].abs() + 1e-37).all())
