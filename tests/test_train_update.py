"""The orthogonalised update against its formula in 64 bits.

Tolerances.  Each step rounds X, A and B to fp16 (half a step, 2^-11 of an element, of either sign: 2^-11 / sqrt(3) of the whole at
most) once each, and the result once to its own type.  A step's products pass an error of X on times the polynomial's slope, at most 3.5
relative to a value that grows as much where singular values are small, and below 2.2 where they are near 1; the errors of A and B
enter with the weights |b| + 2 |c| and 1.  Over five steps: a sum of five errors of at most (1 + 7 + 1) 2^-11 / sqrt(3), each kept, not
amplified, relative to the whole: 45 * 2.8e-4 = 1.3e-2 at the very worst, the root of the sum of squares 1.4e-2 / sqrt(5): 5.7e-3."""
import ctypes as C

import pytest
import torch

from test_train_norm_recurrence import HALF, U32, train  # noqa: F401

gpu = pytest.mark.gpu
ABC = (3.4445, -4.7750, 2.0315)


def test_refusals_need_no_gpu(train):  # noqa: F811
    L = train.load()
    p = C.c_void_p(0x1000)
    ok = (C.c_float * 3)(*ABC)
    call = lambda g=p, n=1, m=64, c=64, kind=2, beta=0.9, steps=5, abc=ok, eps=1e-7, out=p, okind=2, ws=p, nb=1 << 40: (  # noqa: E731
        L.ones_orthogonal_update(g, None, n, m, c, kind, beta, 1, steps, abc, eps, out, okind, ws, nb, None))
    assert call(g=None) == call(out=None) == call(n=-1) == call(m=-1) == call(c=-1) == call(kind=5) == call(okind=0) == -1
    assert call(beta=-0.1) == call(beta=1.5) == call(beta=float("nan")) == call(steps=0) == call(steps=101) == call(abc=None) == -1
    assert call(eps=-1.0) == call(ws=None) == -1 and call(nb=10) == call(ws=C.c_void_p(0x1008)) == -5
    assert call(m=65537) == call(c=65537) == call(n=65536) == call(abc=(C.c_float * 3)(17, 0, 0)) == call(abc=(C.c_float * 3)(float("nan"), 0, 0)) == -3
    assert call(n=0, g=None) == call(m=0, g=None) == call(c=0, out=None) == 0
    assert L.ones_orthogonal_update_workspace_bytes(1, 0, 5) == L.ones_orthogonal_update_workspace_bytes(-1, 5, 5) == 0
    assert L.ones_orthogonal_update_workspace_bytes(2, 100, 50) == L.ones_orthogonal_update_workspace_bytes(2, 50, 100) > 0


def test_the_binding_refuses_on_the_cpu(train):  # noqa: F811
    g = torch.zeros(4, 4)
    with pytest.raises(train.OnesError):
        train.orthogonal_update(g)


def update64(g, m, beta, nesterov, steps, abc, eps):
    g = g.double()
    if m is not None:
        m = beta * m.double() + g
    u = g if m is None else g + beta * m if nesterov else m
    x = u / (u.pow(2).sum((-2, -1), keepdim=True).sqrt() + eps)
    tall = x.shape[-2] > x.shape[-1]
    x = x.transpose(-2, -1) if tall else x
    for _ in range(steps):
        q = x @ x.transpose(-2, -1)
        x = abc[0] * x + (abc[1] * q + abc[2] * q @ q) @ x
    return (x.transpose(-2, -1) if tall else x), m


SIZES = [(1, 1, 1), (1, 1, 9), (3, 5, 2), (1, 64, 64), (2, 65, 130), (5, 128, 100), (1, 300, 70), (1, 257, 513), (1, 520, 129), (40, 33, 47),
         (1, 1100, 1300), (20, 384, 512), (1, 2600, 1100)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("count,rows,cols", SIZES)
def test_update(train, count, rows, cols, dtype):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    g = (torch.randn(count, rows, cols, generator=gen, device="cuda") * 1e-2).to(dtype)
    m = torch.randn(count, rows, cols, generator=gen, device="cuda") * 0.1 if rows % 2 == 0 or cols % 2 else None
    nesterov = cols % 3 != 0
    held = None if m is None else m.clone()
    got = train.orthogonal_update(g, m, 0.95, nesterov, 5, ABC, 1e-7)
    want, moved = update64(g, held, 0.95, nesterov, 5, ABC, 1e-7)
    kind = torch.bfloat16 if dtype == torch.float32 else dtype
    assert got.dtype == kind and got.shape == g.shape
    off = (got.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert off.max() <= 5.7e-3 + HALF[kind], off.max().item()
    if m is not None:
        assert ((m.double() - moved).abs() <= 3 * U32 * (held.double().abs() + g.double().abs())).all()
    values = torch.linalg.svdvals(got.double())
    assert values.max() < 1.3
    if m is not None:
        m.copy_(held)
    assert torch.equal(train.orthogonal_update(g, m, 0.95, nesterov, 5, ABC, 1e-7), got)


@gpu
def test_update_of_a_single_matrix_of_other_scales_and_layouts(train):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(6)
    g = torch.randn(200, 136, generator=gen, device="cuda")
    want, _ = update64(g, None, 0, False, 5, ABC, 0.0)
    for scale in (1e-15, 1.0, 1e12):                                   # the norm is taken out first
        got = train.orthogonal_update(g * scale, eps=0.0)
        assert (got.double() - want).norm() <= (5.7e-3 + HALF[torch.bfloat16]) * want.norm()
    turned = train.orthogonal_update(g.t(), eps=0.0)                   # the shorter side first, either way
    assert (turned.double() - want.t()).norm() <= (5.7e-3 + HALF[torch.bfloat16]) * want.norm()
    half = train.orthogonal_update(g, steps=1, dtype=torch.float16)
    one, _ = update64(g, None, 0, False, 1, ABC, 1e-7)
    assert (half.double() - one).norm() <= 3e-3 * one.norm()
    # a classical cubic step converges to the orthogonal factor
    near = train.orthogonal_update(g, steps=25, coefficients=(1.5, -0.5, 0.0), dtype=torch.float16)
    u, _, v = torch.linalg.svd(g.double(), full_matrices=False)
    assert (near.double() - u @ v).norm() <= 5.7e-3 * (136 ** 0.5)


@gpu
def test_update_of_zeros_of_low_rank_and_of_nan(train):  # noqa: F811
    zero = torch.zeros(3, 70, 40, device="cuda")
    assert not train.orthogonal_update(zero).any()
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = torch.randn(70, 3, generator=gen, device="cuda") @ torch.randn(3, 90, generator=gen, device="cuda")
    got = train.orthogonal_update(g.half())
    want, _ = update64(g.half(), None, 0, False, 5, ABC, 1e-7)
    u, _, v = torch.linalg.svd(g.half().double(), full_matrices=False)
    u, v = u[:, :3], v[:3]
    core, whole = u.t() @ got.double() @ v.t(), u.t() @ want @ v.t()
    assert (core - whole).norm() <= (5.7e-3 + HALF[torch.float16]) * whole.norm()
    # the rounding noise of X, whose elements are about (70 * 90)^-1/2, grows by 3.4445 a step where there is no signal: 485
    # in all, and half as much again from the later steps
    rest = torch.linalg.matrix_norm(got.double() - u @ core @ v, 2)
    assert rest <= 2 * 485 * HALF[torch.float16] * (70 ** 0.5 + 90 ** 0.5) / (70 * 90) ** 0.5
    zero[1, 2, 3] = float("nan")
    got = train.orthogonal_update(zero)
    assert got[1].isnan().all() and not got[0].any() and not got[2].any()


@gpu
def test_refusals_of_the_binding(train):  # noqa: F811
    g = torch.zeros(6, 4, device="cuda")
    for bad in (lambda: train.orthogonal_update(g, torch.zeros(4, 6, device="cuda").t()), lambda: train.orthogonal_update(g[0]),
                lambda: train.orthogonal_update(g, torch.zeros(6, 5, device="cuda")), lambda: train.orthogonal_update(g, coefficients=(1, 2))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: train.orthogonal_update(g, dtype=torch.float32), lambda: train.orthogonal_update(g, g.half()),
                lambda: train.orthogonal_update(g.int())):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(train.OnesError):
        train.orthogonal_update(g, steps=0)
    assert train.orthogonal_update(g[:0]).shape == (0, 4)


@gpu
def test_update_in_a_graph(train):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(2)
    g, m = torch.randn(2, 96, 160, generator=gen, device="cuda").bfloat16(), torch.zeros(2, 96, 160, device="cuda")
    first = train.orthogonal_update(g, m)
    second = train.orthogonal_update(g, m)
    end = m.clone()
    m.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = train.orthogonal_update(g, m)
    for _ in range(2):
        m.zero_()
        graph.replay()
        assert torch.equal(got, first)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, second) and torch.equal(m, end)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("scale", [1e-37, 1e-30, 1e-24, 1e20, 1e30, 1e37])
@pytest.mark.parametrize("rows,cols", [(200, 136), (33, 71)])
def test_update_of_gradients_whose_squares_leave_32_bits(train, rows, cols, scale, dtype):  # noqa: F811
    """Finite gradients of any size: the norm is the root of a sum of squares that 32 bits do not hold."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    g = (torch.randn(2, rows, cols, generator=gen, device="cuda").double() * scale).to(dtype)
    m = (torch.randn(2, rows, cols, generator=gen, device="cuda").double() * scale).float()
    eps = 1e-7 if scale > 1 else 0.0
    for momentum in (None, m):
        want, _ = update64(g, momentum, 0.95, True, 5, ABC, eps)
        got = train.orthogonal_update(g, momentum, 0.95, True, 5, ABC, eps, dtype=torch.bfloat16)
        off = (got.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
        assert off.max() <= 5.7e-3 + HALF[torch.bfloat16], off.max().item()


@gpu
def test_update_of_one_small_matrix_among_large_ones(train):  # noqa: F811
    """Every matrix has a norm of its own; an infinity makes its own matrix NaN, zeros stay zeros."""
    gen = torch.Generator(device="cuda").manual_seed(31)
    one = torch.randn(64, 96, generator=gen, device="cuda")
    g = torch.stack([one * 1e30, one * 1e-30, one * 0, one])
    g[3, 5, 6] = float("inf")
    got = train.orthogonal_update(g, eps=1e-37)
    want, _ = update64(one, None, 0, False, 5, ABC, 0.0)
    for k in (0, 1):
        assert (got[k].double() - want).norm() <= (5.7e-3 + HALF[torch.bfloat16]) * want.norm()
    assert not got[2].any() and got[3].isnan().all()


# What products of pairs and sums of 32 bits make of the whole over five steps: 45 (see the top of the file) times half a step of 22 bits
# and, for up to 4096 terms of either sign, 2^-24 times a quarter of the root of their number.
IN_PAIRS = 45 * (2.0 ** -22 + 16 * U32)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("count,rows,cols", SIZES)
def test_an_fp16_result_has_the_precision_of_fp16(train, count, rows, cols, dtype):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    rank = max(1, min(rows, cols) // 8)
    signal = torch.randn(count, rows, rank, generator=gen, device="cuda").double() @ torch.randn(count, rank, cols, generator=gen, device="cuda").double()
    g = ((signal / rank ** 0.5 + torch.randn(count, rows, cols, generator=gen, device="cuda")) * 1e-3).to(dtype)
    m = ((signal * 8 / rank ** 0.5 + 3 * torch.randn(count, rows, cols, generator=gen, device="cuda")) * 1e-3).float() if rows % 3 else None
    want, _ = update64(g, m, 0.95, True, 5, ABC, 1e-7)
    got = train.orthogonal_update(g, m, 0.95, True, 5, ABC, 1e-7, dtype=torch.float16)
    off = (got.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert off.max() <= HALF[torch.float16] + IN_PAIRS, off.max().item()
