"""Norms of queries and keys for each head with their rotation against the formulas in 64 bits.

Tolerances: an output is rounded once (half a step of its type); the arithmetic of 32 bits before it, of the sums of squares and of the angles,
is off by some 2^-24 of the terms, taken as so many of them."""
import ctypes as C

import pytest
import torch

from test_train_norm_recurrence import HALF, U32, near, train  # noqa: F401

gpu = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def pairs_of(x, f, interleaved):
    r = 2 * f
    return (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :f], x[..., f:r])


def turned(x, cos, sin, interleaved):
    f = cos.shape[-1]
    a, b = pairs_of(x, f, interleaved)
    y = x.clone()
    c, d = pairs_of(y, f, interleaved)
    c.copy_(a * cos - b * sin)
    d.copy_(b * cos + a * sin)
    return y


def rotation64(x, w, positions, frequencies, eps, interleaved, dy):
    x, w, dy = x.double(), w.double(), dy.double()
    angle = positions.double()[:, None, None] * frequencies.double()
    cos, sin = angle.cos(), angle.sin()
    r = (x.pow(2).mean(-1, keepdim=True) + eps) ** -0.5
    y = turned(x * r * w, cos, sin, interleaved)
    g = turned(dy, cos, -sin, interleaved)
    u = g * w
    dx = r * (u - x * r * (u * x * r).mean(-1, keepdim=True))
    # of a pair both elements' sizes
    size = lambda t: turned(t.abs(), torch.ones_like(cos), -torch.ones_like(sin), interleaved).abs() + turned(t.abs(), torch.ones_like(cos), torch.ones_like(sin), interleaved).abs()  # noqa: E731
    su = size(dy) * w.abs()
    return y, dx, (g * x * r).sum((0, 1)), size(x * r * w), r * (su + (x * r).abs() * (su * (x * r).abs()).mean(-1, keepdim=True)), (size(dy) * (x * r).abs()).sum((0, 1))


def test_refusals_need_no_gpu(train):
    L = train.load()
    p = C.c_void_p(0x1000)
    fwd = lambda q=p, qs=128, qh=64, tokens=3, heads=2, kv=1, dim=64, kind=2, qw=p, wk=0, eps=1e-6, pos=p, fr=p, pairs=32, out=p: L.ones_head_norm_rotation_forward(  # noqa: E731
        q, qs, qh, p, 64, 64, tokens, heads, kv, dim, kind, qw, p, wk, eps, pos, fr, pairs, 0, out, p, None)
    for bad in (fwd(q=None), fwd(qs=-1), fwd(qh=-1), fwd(tokens=-1), fwd(heads=-1), fwd(dim=0, pairs=0), fwd(kind=3), fwd(qw=None), fwd(wk=1), fwd(eps=-1.0),
                fwd(eps=float("nan")), fwd(pos=None), fwd(fr=None), fwd(pairs=33), fwd(pairs=-1), fwd(out=None)):
        assert bad == -1
    assert fwd(tokens=(1 << 30) + 1) == fwd(heads=1025) == fwd(dim=513) == fwd(qs=1 << 33) == -3
    assert fwd(tokens=0, q=None, out=None, pos=None) == 0
    need = L.ones_head_norm_rotation_workspace_bytes(10, 2, 1, 64)
    assert need > 0 and L.ones_head_norm_rotation_workspace_bytes(10, 2, 1, 0) == 0
    back = lambda ws=p, n=need, dq=p, g=p: L.ones_head_norm_rotation_backward(  # noqa: E731
        g, 128, 64, p, 64, 64, p, 128, 64, p, 64, 64, 10, 2, 1, 64, 0, p, p, 0, 1e-6, p, p, 32, 0, dq, p, p, p, ws, n, None)
    assert back(ws=None) == back(dq=None) == back(g=None) == -1 and back(n=need - 1) == -5
    x = torch.zeros(4, 2, 8)
    with pytest.raises(train.OnesError):
        train.head_norm_rotation_forward(x, x, x[0, 0], x[0, 0], torch.zeros(4, dtype=torch.int32), torch.zeros(4))
    with pytest.raises(TypeError):
        train.head_norm_rotation_forward(x.double(), x, x[0, 0], x[0, 0], torch.zeros(4, dtype=torch.int32), torch.zeros(4))


CASES = [(1, 1, 1, 2, 1, False), (5, 3, 2, 64, 32, False), (7, 16, 2, 128, 64, True), (33, 5, 5, 80, 20, False), (9, 12, 4, 80, 20, True), (4, 2, 1, 17, 8, False),
         (4, 2, 1, 17, 5, True), (6, 2, 2, 256, 128, False), (3, 1, 1, 512, 256, True), (3, 1, 1, 511, 100, False), (2100, 4, 1, 96, 48, False), (11, 3, 1, 32, 0, False),
         (50, 7, 3, 100, 50, True), (5000, 2, 2, 64, 16, True), (8, 40, 1, 16, 8, False), (3, 2, 1, 1, 0, False), (70, 0, 3, 64, 32, False), (2, 1, 1, 300, 150, False)]


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("tokens,heads,kv,dim,pairs,interleaved", CASES)
def test_head_norm_rotation(train, tokens, heads, kv, dim, pairs, interleaved, dtype):
    gen = torch.Generator(device="cuda").manual_seed(tokens * 1000 + dim)
    make = lambda *s, std=1.0, mean=0.0: torch.randn(*s, generator=gen, device="cuda") * std + mean  # noqa: E731
    kind = dtype if dim % 3 else FP32
    q, k, dq, dk = (make(tokens, h, dim, std=1.5).to(dtype) for h in (heads, kv, heads, kv))
    qw, kw = make(dim, std=0.2, mean=1).to(kind), make(dim, std=0.2, mean=1).to(kind)
    positions = torch.randint(-5000, 1 << 20, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    frequencies = 10000.0 ** (-torch.arange(pairs, device="cuda") / max(pairs, 1))
    args = (positions, frequencies.float(), 1e-5, interleaved)
    got = train.head_norm_rotation_forward(q, k, qw, kw, *args)
    back = train.head_norm_rotation_backward(dq, dk, q, k, qw, kw, *args)
    for x, w, dy, y, dx, dw in ((q, qw, dq, got[0], back[0], back[2]), (k, kw, dk, got[1], back[1], back[3])):
        assert (y.dtype, dx.dtype, dw.dtype, y.shape, dx.shape) == (dtype, dtype, kind, x.shape, x.shape)
        wy, wdx, wdw, sy, sdx, sdw = rotation64(x, w, *args, dy)
        near(y, wy, sy, 32 + dim // 16, "y")
        near(dx, wdx, sdx, 64 + dim // 8, "dx")
        near(dw, wdw, sdw, 64 + tokens // 16, "dweight")
    again = train.head_norm_rotation_backward(dq, dk, q, k, qw, kw, *args)
    assert all(torch.equal(a, b) for a, b in zip(again, back))


@gpu
def test_strides_and_positions_of_other_kinds(train):
    gen = torch.Generator(device="cuda").manual_seed(4)
    rows = torch.randn(60, 6 * 64 + 1, generator=gen, device="cuda").to(BF16)
    w = torch.rand(64, generator=gen, device="cuda") + 0.5
    fr = 100.0 ** (-torch.arange(32, device="cuda") / 32.0)
    long_positions = torch.arange(60, device="cuda") * 3
    heads_first = torch.randn(4, 60, 64, generator=gen, device="cuda").to(BF16)
    for q, k in ((rows[:, :256].unflatten(1, (4, 64)), rows[:, 256:384].unflatten(1, (2, 64))), (rows[:, 1:257].unflatten(1, (4, 64)), rows[:, 257:].unflatten(1, (2, 64))),
                 (heads_first.transpose(0, 1), heads_first[:1].transpose(0, 1)), (heads_first[:1].transpose(0, 1).expand(60, 4, 64), heads_first.transpose(0, 1).flip(2))):
        got = train.head_norm_rotation_forward(q, k, w, w, long_positions, fr)
        want = train.head_norm_rotation_forward(q.contiguous(), k.contiguous(), w, w, long_positions.int(), fr)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        one = torch.ones((), device="cuda", dtype=BF16)
        got = train.head_norm_rotation_backward(one.expand(q.shape), one.expand(k.shape), q, k, w, w, long_positions, fr)
        want = train.head_norm_rotation_backward(torch.ones_like(q).contiguous(), torch.ones_like(k).contiguous(), q.contiguous(), k.contiguous(), w, w, long_positions, fr)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_rows_of_nothing_of_zeros_and_of_nan(train):
    w, fr = torch.ones(64, device="cuda"), torch.ones(32, device="cuda")
    none = torch.empty(0, 2, 64, device="cuda", dtype=BF16)
    positions = torch.zeros(0, device="cuda", dtype=torch.int32)
    q, k = train.head_norm_rotation_forward(none, none, w, w, positions, fr)
    dq, dk, dqw, dkw = train.head_norm_rotation_backward(none, none, none, none, w, w, positions, fr)
    assert q.shape == dq.shape == (0, 2, 64) and not dqw.any() and not dkw.any()
    x = torch.zeros(3, 2, 64, device="cuda", dtype=BF16)
    x[1, 1, 7] = float("nan")
    x[2, 0, 9] = float("inf")
    q, k = train.head_norm_rotation_forward(x, x, w, w, torch.arange(3, device="cuda", dtype=torch.int32), fr)
    assert not q[0].any() and not q[1, 0].any() and q[1, 1].isnan().all() and q[2, 0].isnan().any() and not q[2, 1].any()
    # the largest positions: the angle keeps its place
    far = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1], device="cuda", dtype=torch.int32)
    x = torch.randn(3, 1, 64, device="cuda")
    fr = 10000.0 ** (-torch.arange(32, device="cuda") / 32.0)
    q, _ = train.head_norm_rotation_forward(x, x, w, w, far, fr)
    y, _, _, size, _, _ = rotation64(x, w, far, fr, 1e-6, False, x)
    near(q, y, size, 64, "far")
    with pytest.raises(ValueError):
        train.head_norm_rotation_forward(x, x, w, w, far, torch.ones(33, device="cuda"))
    with pytest.raises(TypeError):
        train.head_norm_rotation_forward(x, x, w, None, far, fr)
    with pytest.raises(ValueError):
        train.head_norm_rotation_forward(x, x[:2], w, w, far, fr)


@gpu
def test_norms_alone_need_no_positions(train):
    x, w = torch.randn(9, 2, 40, device="cuda"), torch.rand(40, device="cuda") + 0.5
    y, z = torch.empty_like(x), torch.empty_like(x)
    rc = train.load().ones_head_norm_rotation_forward(x.data_ptr(), 80, 40, x.data_ptr(), 80, 40, 9, 2, 2, 40, 0, w.data_ptr(), w.data_ptr(), 0, 1e-6, None, None, 0, 0,
                                                      y.data_ptr(), z.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(y, z)
    near(y, x.double() * (x.double().pow(2).mean(-1, keepdim=True) + 1e-6) ** -0.5 * w.double(), x.double().abs() * 2, 64, "y")


@gpu
def test_gradients_under_autograd_against_differences(train):
    gen = torch.Generator(device="cuda").manual_seed(6)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda", requires_grad=True)  # noqa: E731
    q, k, qw, kw = make(5, 3, 24), make(5, 2, 24), make(24), make(24)
    positions, fr = torch.tensor([0, 7, 3, 900, -4], device="cuda", dtype=torch.int32), torch.tensor([1.0, 0.3, 0.01, 0.002], device="cuda")
    vq, vk = torch.randn(5, 3, 24, generator=gen, device="cuda"), torch.randn(5, 2, 24, generator=gen, device="cuda")
    a, b = train.head_norm_rotation(q, k, qw, kw, positions, fr, 1e-6, True)
    ((a * vq).sum() + (b * vk).sum()).backward()
    f = lambda q, k, qw, kw: sum((rotation64(x, w, positions, fr, 1e-6, True, x)[0] * g.double()).sum() for x, w, g in ((q, qw, vq), (k, kw, vk)))  # noqa: E731
    for t in (q, k, qw, kw):
        direction = torch.randn(t.shape, generator=gen, device="cuda").double()
        moved = [[u.detach().double() + (s * 1e-4 * direction if u is t else 0) for u in (q, k, qw, kw)] for s in (1, -1)]
        difference = (f(*moved[0]) - f(*moved[1])) / 2e-4
        assert abs((t.grad.double() * direction).sum() - difference) < 1e-4 * (1 + abs(difference))


@gpu
def test_a_stream_and_a_captured_graph_give_the_same(train):
    gen = torch.Generator(device="cuda").manual_seed(7)
    q, k = (torch.randn(3000, h, 128, generator=gen, device="cuda").bfloat16() for h in (4, 2))
    w, fr, positions = torch.rand(128, generator=gen, device="cuda"), 100.0 ** (-torch.arange(64, device="cuda") / 64.0), torch.arange(3000, device="cuda", dtype=torch.int32)

    def both(q=q):
        return (*train.head_norm_rotation_forward(q, k, w, w, positions, fr), *train.head_norm_rotation_backward(q, k, q, k, w, w, positions, fr))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph, q2 = torch.cuda.CUDAGraph(), q.clone()
    with torch.cuda.graph(graph):
        found = both(q2)
    for i in range(3):
        q2.copy_(q + i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(found, both(q + i))), i


def both_ways(train, q, k, qw, kw, dq, dk, *args):
    """Forward and backward against the formulas, equal bits from call to call."""
    tokens, _, dim = q.shape
    y = train.head_norm_rotation_forward(q, k, qw, kw, *args)
    back = train.head_norm_rotation_backward(dq, dk, q, k, qw, kw, *args)
    for x, w, dy, got, dx, dw in ((q, qw, dq, y[0], back[0], back[2]), (k, kw, dk, y[1], back[1], back[3])):
        wy, wdx, wdw, sy, sdx, sdw = rotation64(x, w, *args, dy)
        near(got, wy, sy, 32 + dim // 16, "y")
        near(dx, wdx, sdx, 64 + dim // 8, "dx")
        near(dw, wdw, sdw, 64 + tokens // 16, "dweight")
    again = train.head_norm_rotation_backward(dq, dk, q, k, qw, kw, *args)
    assert all(torch.equal(a, b) for a, b in zip(again, back))


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("tokens,heads,kv,dim,pairs", [(33, 16, 2, 128, 64), (40, 16, 2, 64, 32), (5, 3, 1, 80, 20), (4, 2, 1, 17, 8), (2100, 5, 1, 96, 48), (9, 1, 1, 512, 256)])
def test_norms_without_eps(train, tokens, heads, kv, dim, pairs, dtype):
    """eps 0, and heads that do not fill the last rows of a wave: what is not there has no norm, and no part in the weights' gradients."""
    gen = torch.Generator(device="cuda").manual_seed(tokens + dim)
    make = lambda *s, std=1.0, mean=0.0: torch.randn(*s, generator=gen, device="cuda") * std + mean  # noqa: E731
    q, k, dq, dk = (make(tokens, h, dim, std=1.5).to(dtype) for h in (heads, kv, heads, kv))
    w = [make(dim, std=0.2, mean=1) for _ in range(2)]
    positions = torch.arange(tokens, device="cuda", dtype=torch.int32)
    both_ways(train, q, k, *w, dq, dk, positions, 100.0 ** (-torch.arange(pairs, device="cuda") / pairs), 0.0, False)


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dim,interleaved", [(128, False), (80, True), (17, False), (512, False)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_whose_squares_are_no_floats(train, dim, interleaved, dtype, eps):
    """Elements of 1e21 and 1e30, and without eps of 1e-21 and 1e-30, beside ordinary ones: norms as of all others."""
    gen = torch.Generator(device="cuda").manual_seed(dim)
    make = lambda *s, std=1.0, mean=0.0: torch.randn(*s, generator=gen, device="cuda") * std + mean  # noqa: E731
    size = torch.tensor([1.0, 1e21, 1e30, 1e19] + ([1e-21, 1e-30, 1e-19] if eps == 0 else []), device="cuda")[:, None, None]
    n = len(size)
    q, k = (make(n, h, dim).mul(size).to(dtype) for h in (5, 2))
    q[1, 0, 1:], k[2, 1, 2:] = 0, 0                                  # most of a row nothing
    # gradients of the sizes that such rows give and take: dx stays within the type
    dq, dk = (make(n, h, dim).mul(size.clamp(1e-3, 1e3)).to(dtype) for h in (5, 2))
    w = [make(dim, std=0.2, mean=1) for _ in range(2)]
    positions = torch.arange(n, device="cuda", dtype=torch.int32)
    both_ways(train, q, k, *w, dq, dk, positions, 100.0 ** (-torch.arange(dim // 4, device="cuda") / (dim // 4)), eps, interleaved)
