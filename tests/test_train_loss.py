"""The loss over a vocabulary against its formula in 64 bits.

Tolerances.  Products of 16-bit values are exact in 32 bits; a logit's sum over D terms is off by at most D 2^-24 of the sum of the
terms' sizes, in practice by a few times its root.  exp of it and the sum over the vocabulary pass that error on as it stands.
G is rounded to the operands' type (half a step each), so that a gradient is off by half a step of the sum of its terms' sizes
(roundings of either sign: far less), and by half a step of itself."""
import ctypes as C

import pytest
import torch

from test_train_norm_recurrence import HALF, U32, near, train  # noqa: F401

gpu = pytest.mark.gpu


def test_refusals_need_no_gpu(train):  # noqa: F811
    L = train.load()
    p = C.c_void_p(0x1000)
    big = 1 << 60
    fwd = lambda x=p, xs=64, ws=64, n=4, d=64, v=100, kind=2, t=p, w=p, work=p, nb=big: L.ones_cross_entropy_forward(  # noqa: E731
        x, xs, w, ws, n, d, v, kind, t, p, p, work, nb, None)
    assert fwd(x=None) == fwd(t=None) == fwd(w=None) == fwd(xs=63) == fwd(ws=63) == fwd(n=-1) == fwd(d=0) == fwd(v=0) == -1
    assert fwd(kind=0) == fwd(kind=7) == fwd(work=None) == -1               # products of 32-bit operands are not offered
    assert fwd(nb=16) == fwd(work=C.c_void_p(0x1001)) == -5
    assert fwd(n=(1 << 24) + 1) == fwd(v=(1 << 24) + 1) == fwd(d=65537, xs=65537, ws=65537) == fwd(n=1 << 24, v=1 << 24) == -3
    assert fwd(n=1 << 24, d=65536, xs=65536, ws=65536, v=1) == -3
    assert fwd(n=0, x=None, t=None, work=None, nb=0) == 0
    bwd = lambda dl=p, w=p, dw=p, work=p, nb=big, n=4: L.ones_cross_entropy_backward(  # noqa: E731
        dl, p, 64, w, 64, n, 64, 100, 1, p, p, p, dw, work, nb, None)
    assert bwd(dl=None) == bwd(w=None) == bwd(dw=None) == bwd(work=None) == -1 and bwd(nb=100) == -5
    for f in (L.ones_cross_entropy_forward_workspace_bytes, L.ones_cross_entropy_backward_workspace_bytes):
        assert f(4, 0, 5, 0) == f(-1, 4, 5, 0) == f(4, 4, 0, 1) == 0 and f(100, 64, 1000, 0) > f(100, 64, 1000, 1) > 0
    # the gradients of the logits are held piece by piece
    assert L.ones_cross_entropy_backward_workspace_bytes(16384, 512, 131072, 1) < (128 << 20) + 16384 * 512 * 6 + (1 << 20)


def test_rows_far_apart_are_copied(train):  # noqa: F811
    """A workgroup's loads lie up to 63 rows beside each other at offsets of 32 bits: rows further apart need the copies' workspace."""
    L = train.load()
    p = C.c_void_p(0x1000)
    for size, call in ((L.ones_cross_entropy_forward_workspace_bytes, lambda xs, ws, nb: L.ones_cross_entropy_forward(
            p, xs, p, ws, 4, 64, 100, 2, p, p, p, p, nb, None)),
            (L.ones_cross_entropy_backward_workspace_bytes, lambda xs, ws, nb: L.ones_cross_entropy_backward(
                p, p, xs, p, ws, 4, 64, 100, 2, p, p, p, p, p, nb, None))):
        assert call(64, (1 << 24) + 8, size(4, 64, 100, 1)) == -5


def test_the_binding_refuses_wrong_shapes(train):  # noqa: F811
    x, w, t = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(train.OnesError):
        train.linear_cross_entropy_forward(x, w, t)
    with pytest.raises(TypeError):
        train.linear_cross_entropy_forward(x.float(), w.float(), t)


def loss64(x, w, t, dloss):
    x, w, dloss = x.double(), w.double(), dloss.double()
    skip = t < 0
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    at = t.clamp(min=0).long()[:, None]
    loss = torch.where(skip, torch.zeros_like(lse), lse - z.gather(1, at)[:, 0])
    p = torch.exp(z - lse[:, None])
    g = p.clone()
    g.scatter_add_(1, at, -torch.ones_like(lse)[:, None])
    scale = torch.where(skip, torch.zeros_like(lse), dloss)[:, None]
    return loss, lse, g * scale, p * scale.abs(), x, w


def check(train, x, w, t, dloss):  # noqa: F811
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    dx, dw = train.linear_cross_entropy_backward(dloss, x, w, t, lse)
    clean = torch.where((t < 0)[:, None], torch.zeros_like(x), x)
    wloss, wlse, g, p, cx, cw = loss64(clean, w, t, dloss)
    valid = t >= 0
    size = (cx.abs() @ cw.abs().t()).amax(1)                              # of the terms of the row's logits
    d, v, n = x.shape[1], w.shape[0], x.shape[0]
    many = 16 + 4 * d ** 0.5 + v / 64
    near(lse[valid], wlse[valid], (size + wlse.abs() + 1)[valid], many, "lse")
    near(loss, wloss, torch.where(valid, 2 * size + wlse.abs() + 1, torch.zeros_like(size)), many, "loss")
    half = HALF[x.dtype]
    # G: half a step of itself, the error of its logit and lse (which its probability has as a factor), and fp16's smallest
    # steps (2^-24 under a scale of 2^14 / dloss)
    soft = many * U32 * (size + 2 + wlse.abs())[:, None] * p + 2.0 ** -36 * dloss.abs().max().item() * valid[:, None]
    dg = half * g.abs() + soft
    for got, want, error, small, terms, k, what in (
            (dx, g @ cw, dg @ cw.abs(), soft @ cw.abs(), g.abs() @ cw.abs(), v, "dx"),
            (dw, g.t() @ cx, dg.t() @ cx.abs(), soft.t() @ cx.abs(), g.abs().t() @ cx.abs(), n, "dweight")):
        sums = U32 * (16 + 4 * k ** 0.5) * terms
        bound = error + sums + half * want.abs() * (1 + 2.0 ** -7) + (2.0 ** -24 if x.dtype == torch.float16 else 1e-37)
        off = (got.double() - want).abs()
        assert (off <= bound).all(), f"{what}: {(off - bound).max().item()} beyond the bound"
        # half steps of either sign: the whole is off by less than the sum of the bounds
        assert off.norm() <= half * want.norm() + (small + sums).norm() + (off.numel() ** 0.5) * 2.0 ** -25, what
    assert not dx[~valid].any()
    again = train.linear_cross_entropy_backward(dloss, x, w, t, lse)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


SIZES = [(1, 8, 1), (1, 1, 3), (2, 7, 129), (64, 256, 1000), (130, 64, 257), (300, 100, 513), (257, 514, 2049), (33, 136, 5000),
         (1000, 72, 8200), (128, 1024, 128)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,vocabulary", SIZES)
def test_loss_and_gradients(train, rows, cols, vocabulary, dtype):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(rows + vocabulary)
    x = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(vocabulary, cols, generator=gen, device="cuda") * 1.5 / cols ** 0.5).to(dtype)
    t = torch.randint(0, vocabulary, (rows,), generator=gen, device="cuda")
    if rows > 2:
        t[torch.rand(rows, generator=gen, device="cuda") < 0.3] = -100
        t[0], t[-1] = vocabulary - 1, -1
        x[t < 0] = float("nan")                                       # padding may hold anything
    dloss = torch.rand(rows, generator=gen, device="cuda") / rows
    check(train, x, w, t, dloss)


@gpu
def test_loss_in_several_pieces_and_large_tiles(train):  # noqa: F811
    """2304 rows of 40001 words: 184 MB of logits' gradients, so two pieces, the second of a ragged end; large tiles."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(2304, 384, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(40001, 384, generator=gen, device="cuda") * 0.08).bfloat16()
    t = torch.randint(0, 40001, (2304,), generator=gen, device="cuda")
    t[5:50] = -100
    check(train, x, w, t, torch.full((2304,), 1 / 2259, device="cuda"))


@gpu
def test_loss_of_strided_unaligned_and_extreme_inputs(train):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(3)
    wide = torch.randn(90, 300, generator=gen, device="cuda").half()
    table = (torch.randn(260, 300, generator=gen, device="cuda") * 0.2).half()
    t = torch.randint(0, 260, (90,), generator=gen, device="cuda")
    dloss = torch.randn(90, generator=gen, device="cuda")
    for lo, hi in ((0, 64), (8, 72), (3, 67), (1, 72)):
        check(train, wide[:, lo:hi], table[:, lo:hi], t, dloss)
    check(train, wide[:64, :90].t(), table[:, :64], t.int(), dloss * 0)
    check(train, wide[:, :64], table[:, :64], torch.full_like(t, -100), dloss)        # every row ignored
    check(train, wide[:, :64], table[:, :64], t, dloss * 1e-7)                        # fp16: gradients of the smallest sizes
    # one logit far above all others, and a table whose logits are all far below zero
    x = torch.zeros(3, 16, device="cuda", dtype=torch.bfloat16)
    x[:, 0] = 100
    w = torch.zeros(200, 16, device="cuda", dtype=torch.bfloat16)
    w[7, 0] = 100
    t = torch.tensor([7, 8, -1], device="cuda")
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    assert lse.tolist() == [1e4] * 3 and loss.tolist() == [0, 1e4, 0]
    w[:, 0] = -100
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    want = -1e4 + torch.tensor(200.0).log().item()
    assert (lse - want).abs().max() < 1e-2 and abs(loss[0].item() - 5.298) < 1e-2
    # NaN in one row stays in that row's loss
    x[1, 3] = float("nan")
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    assert loss[0].isfinite() and loss[1].isnan() and lse[1].isnan() and loss[2] == 0


@gpu
def test_loss_of_rows_that_lie_gigabytes_apart(train):  # noqa: F811
    """Row 16 begins 2^32 bytes behind row 0: what a 32-bit offset loses."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    apart = torch.empty(40 << 27, dtype=torch.bfloat16, device="cuda").as_strided((40, 64), (1 << 27, 1))
    apart.copy_(torch.randn(40, 64, generator=gen, device="cuda"))
    other = torch.randn(70, 64, generator=gen, device="cuda").bfloat16() * 0.2
    target = torch.randint(0, 40, (70,), generator=gen, device="cuda")
    check(train, other, apart, target, torch.rand(70, generator=gen, device="cuda"))
    check(train, apart, other, target[:40], torch.rand(40, generator=gen, device="cuda"))


@gpu
def test_a_target_beyond_the_vocabulary_is_not_read_and_shows(train):  # noqa: F811
    x, w = torch.randn(4, 32, device="cuda").bfloat16(), torch.randn(70, 32, device="cuda").bfloat16()
    t = torch.tensor([3, 70, 1 << 40, 5], device="cuda")
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    assert loss.isnan().tolist() == [False, True, True, False] and lse.isfinite().all()
    dx, dw = train.linear_cross_entropy_backward(torch.ones(4, device="cuda"), x, w, t, lse)
    assert dx.isnan().any(1).tolist() == [False, True, True, False] and dw.isnan().all()


@gpu
def test_loss_of_no_rows(train):  # noqa: F811
    w = torch.randn(50, 24, device="cuda").bfloat16()
    x, t = w[:0], torch.zeros(0, dtype=torch.int64, device="cuda")
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    dx, dw = train.linear_cross_entropy_backward(loss, x, w, t, lse)
    assert loss.shape == (0,) and dx.shape == (0, 24) and not dw.any() and dw.shape == w.shape


@gpu
def test_gradients_under_autograd_against_differences(train):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(20, 40, generator=gen, device="cuda").half().requires_grad_()
    w = (torch.randn(60, 40, generator=gen, device="cuda") * 0.2).half().requires_grad_()
    t = torch.randint(-1, 60, (20,), generator=gen, device="cuda")
    weights = torch.rand(20, generator=gen, device="cuda")
    (train.linear_cross_entropy(x, w, t) * weights).sum().backward()
    f = lambda a, b: (loss64(a, b, t, weights)[0] * weights.double()).sum()  # noqa: E731
    for u in (x, w):
        direction = torch.randn(u.shape, generator=gen, device="cuda").double()
        moved = [[q.detach().double() + (s * 1e-4 * direction if q is u else 0) for q in (x, w)] for s in (1, -1)]
        difference = (f(*moved[0]) - f(*moved[1])) / 2e-4
        size = (u.grad.double() * direction).abs().sum()
        assert abs((u.grad.double() * direction).sum() - difference) <= 2 * HALF[torch.float16] * size


@gpu
def test_loss_in_a_graph_and_on_another_stream(train):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(200, 128, generator=gen, device="cuda").half()
    w = torch.randn(3001, 128, generator=gen, device="cuda").half() * 0.1
    t = torch.randint(-1, 3001, (200,), generator=gen, device="cuda")
    dloss = torch.rand(200, generator=gen, device="cuda")

    def both():
        loss, lse = train.linear_cross_entropy_forward(x, w, t)
        return [loss, lse, *train.linear_cross_entropy_backward(dloss, x, w, t, lse)]

    want = [q.clone() for q in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        for q in got:
            q.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)) and all(torch.equal(p, q) for p, q in zip(both(), want))


@gpu
@pytest.mark.parametrize("rows", [4095, 4097])
def test_loss_where_the_parts_are_joined_otherwise(train, rows):  # noqa: F811
    """Few rows are joined eight at a time, many 64 at a time; an ignored, an unknown and a NaN row among them."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, 64, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(3001, 64, generator=gen, device="cuda") * 0.2).bfloat16()
    t = torch.randint(0, 3001, (rows,), generator=gen, device="cuda")
    t[7], t[rows - 2], x[rows - 1, 5] = -100, 3001, float("nan")
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    fine = torch.ones(rows, dtype=torch.bool, device="cuda")
    fine[[7, rows - 2, rows - 1]] = False
    want, wlse, *_ = loss64(x[fine], w, t[fine], torch.ones(rows - 3, device="cuda"))
    size = (x[fine].double().abs() @ w.double().abs().t()).amax(1)
    many = 16 + 4 * 64 ** 0.5 + 3001 / 64
    near(lse[fine], wlse, size + wlse.abs() + 1, many, "lse")
    near(loss[fine], want, 2 * size + wlse.abs() + 1, many, "loss")
    assert loss[7] == 0 and loss[rows - 2].isnan() and lse[rows - 2].isfinite() and loss[rows - 1].isnan() and lse[rows - 1].isnan()


def test_the_outputs_under_autograd_can_be_changed_in_place(train, monkeypatch):  # noqa: F811
    """What the binding itself hands out, without a GPU: the library's call is left out, so the values are whatever memory held."""
    monkeypatch.setattr(train, "_check", lambda *a, **k: None)
    monkeypatch.setattr(train, "_call", lambda *a: None)
    x, w = torch.zeros(6, 8).bfloat16().requires_grad_(), torch.zeros(5, 8).bfloat16().requires_grad_()
    t = torch.tensor([0, 1, -1, 4, 2, -1])
    loss = train.linear_cross_entropy(x, w, t)
    loss[t < 0] = 0
    loss.mul_(0.5)
    loss.sum().backward()
    assert x.grad.shape == x.shape and w.grad.shape == w.shape
    u = torch.zeros(2, 3, 4).requires_grad_()
    for outputs in ((train.layer_norm(u),), train.gated_recurrence(u, u)):
        for q in outputs:
            q.mul_(2)
        sum(q.sum() for q in outputs).backward()


@gpu
def test_a_loss_changed_in_place_has_the_changed_gradient(train):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn(40, 64, generator=gen, device="cuda").bfloat16().requires_grad_()
    w = (torch.randn(90, 64, generator=gen, device="cuda") * 0.2).bfloat16().requires_grad_()
    t = torch.randint(-1, 90, (40,), generator=gen, device="cuda")
    weights = torch.rand(40, generator=gen, device="cuda")
    loss = train.linear_cross_entropy(x, w, t)
    loss.mul_(weights)
    loss[:5] = 0
    loss.sum().backward()
    weights[:5] = 0
    _, lse = train.linear_cross_entropy_forward(x.detach(), w.detach(), t)
    dx, dw = train.linear_cross_entropy_backward(weights, x.detach(), w.detach(), t, lse)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw)


def row_errors(train, x, w, t, dloss):  # noqa: F811
    """Per row, what dx is off by and what G's rounding (half a step each, of either sign) and dx's own make of it, as norms; dx, dweight."""
    loss, lse = train.linear_cross_entropy_forward(x, w, t)
    dx, dw = train.linear_cross_entropy_backward(dloss, x, w, t, lse)
    rows = dloss.isfinite()
    _, wlse, g, p, cx, cw = loss64(x, w, t, torch.where(rows, dloss, torch.zeros_like(dloss)))
    want, half = g @ cw, HALF[x.dtype]
    # a logit's error goes into its probability, and with that into all of the row's terms
    logits = (16 + 4 * x.shape[1] ** 0.5 + w.shape[0] / 64) * U32 * ((cx.abs() @ cw.abs().t()).amax(1) + 2 + wlse.abs())
    allowed = 2 * half * (g.square() @ cw.square()).sum(1).sqrt() + half * want.norm(dim=1) + logits * (p @ cw.abs()).norm(dim=1)
    allowed = allowed + (2.0 ** -24 * x.shape[1] ** 0.5 if x.dtype == torch.float16 else 0.0)
    return (dx.double() - want).norm(dim=1), allowed, dx, dw


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_an_infinite_gradient_of_a_loss_stays_in_its_row_of_dx(train, dtype):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(37)
    x = (torch.randn(70, 64, generator=gen, device="cuda") * 0.3).to(dtype)
    w = (torch.randn(30000, 64, generator=gen, device="cuda") * 0.2 + 0.1).to(dtype)
    t = torch.randint(0, 30000, (70,), generator=gen, device="cuda")
    dloss = torch.full((70,), 1e-3, device="cuda")
    dloss[3], dloss[66] = float("inf"), float("nan")
    off, allowed, dx, dw = row_errors(train, x, w, t, dloss)
    assert not dx[[3, 66]].isfinite().any() and not dw.isfinite().any()
    off[[3, 66]] = 0
    assert (off <= allowed).all(), (off / allowed).max().item()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,words", [(140, 64, 30000), (140, 33, 131072), (1329, 2774, 1593), (4103, 250, 12267)])
def test_rows_of_small_gradients_next_to_large_ones(train, rows, cols, words, dtype):  # noqa: F811
    """dloss from 2^13 down to 2^-13: dx of every row is right for itself, and dW for words that only a small row has as its target."""
    gen = torch.Generator(device="cuda").manual_seed(41)
    x = (torch.randn(rows, cols, generator=gen, device="cuda") * 0.3).to(dtype)
    w = (torch.randn(words, cols, generator=gen, device="cuda") * 1.6 + 0.8).div(cols ** 0.5).to(dtype)
    t = torch.randperm(words, generator=gen, device="cuda")[:rows]
    dloss = 2.0 ** (13 - torch.arange(rows, device="cuda") % 27) * (1 + torch.rand(rows, generator=gen, device="cuda"))
    t[7] = -1
    off, allowed, dx, dw = row_errors(train, x, w, t, dloss)
    off[7] = 0
    assert (off <= allowed).all(), (off / allowed).max().item()
    _, _, g, p, cx, _ = loss64(x, w, t, dloss)
    want, at = g.t() @ cx, t.clamp(min=0)
    error = (dw.double() - want).norm(dim=1)
    # G's roundings of either sign, and x's in units of the largest dloss
    mine = 2 * HALF[dtype] * (g.t().square() @ cx.square()).sum(1).sqrt() + HALF[dtype] * want.norm(dim=1) + 2.0 ** -24 * cols ** 0.5
    soft = (16 + 4 * cols ** 0.5 + words / 64) * U32 * 8 * (p.t() @ cx.abs()).norm(dim=1)
    assert (error <= mine + soft)[at].all(), (error / (mine + soft))[at].max().item()
