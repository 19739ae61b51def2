"""Clipping of gradients by their global norm against the formula in 64 bits.

Tolerances: the norm is summed in 64 bits and rounded to 32 once; a clipped element is a product of 32 bits with a factor of 32 bits, rounded to
the gradient's type."""
import ctypes as C
import math

import pytest
import torch

from test_train_norm_recurrence import HALF, U32, train  # noqa: F401

gpu = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def test_refusals_need_no_gpu(train):
    L = train.load()
    p = C.c_void_p(0x1000)

    def clip(at=(0x1000, 0x2000), counts=(8, 8), types=(0, 2), n=None, limit=1.0, eps=1e-6, norm=p, ws=p, nbytes=1 << 20):
        k = len(at)
        return L.ones_clip_gradients((C.c_void_p * k)(*at), (C.c_int64 * k)(*counts), (C.c_int32 * k)(*types), k if n is None else n, limit, eps, norm, ws, nbytes, None)

    for bad in (clip(at=(0, 0x2000)), clip(counts=(-1, 8)), clip(types=(0, 3)), clip(n=-1), clip(limit=-1.0), clip(limit=float("nan")), clip(eps=-1.0), clip(norm=None),
                clip(ws=None), clip(at=(0x1002, 0x2000)), clip(at=(0x1000, 0x2001)),
                clip(at=(0x1000, 0x1000)), clip(at=(0x2000, 0x1000), counts=(8, 0x801)), clip(at=(0x101e, 0x1000), types=(2, 0))):       # one twice, overlaps
        assert bad == -1
    assert clip(counts=(8, (1 << 46) + 1)) == clip(n=(1 << 20) + 1) == -3 and clip(nbytes=100) == clip(ws=C.c_void_p(0x1010)) == -5
    assert L.ones_clip_gradients(None, None, None, 3, 1.0, 0.0, p, p, 1 << 20, None) == -1
    assert L.ones_clip_gradients_workspace_bytes(-1) == 0 and L.ones_clip_gradients_workspace_bytes(1000) >= 8 * 1024
    with pytest.raises(train.OnesError):
        train.clip_gradients([torch.zeros(4)], 1.0)
    with pytest.raises(ValueError):
        train.clip_gradients([], 1.0)
    with pytest.raises(TypeError):
        train.clip_gradients([torch.zeros(4).double()], 1.0)


def check(train, gradients, limit, eps=1e-6):
    exact = [g.double().clone() for g in gradients]
    want = math.sqrt(sum(g.pow(2).sum().item() for g in exact))
    factor = min(1.0, limit / (want + eps)) if want + eps > 0 else 1.0
    norm = train.clip_gradients(gradients, limit, eps)
    assert norm.dtype == FP32 and norm.dim() == 0 and abs(norm.item() - want) <= 2 * U32 * want + 1e-45
    for g, e in zip(gradients, exact):
        if factor == 1.0:
            assert torch.equal(g.double(), e)
        else:
            tiny = {BF16: 1e-38, FP16: 2.0 ** -25, FP32: 1e-38}[g.dtype]
            assert ((g.double() - e * factor).abs() <= (HALF[g.dtype] + 4 * U32) * (e * factor).abs() * (1 + 2.0 ** -6) + tiny).all()
    return norm


SIZES = [[1], [7], [8191], [8192], [8193], [0, 5, 0], [100, 1, 3000, 77777], [3] * 257, [1000003], [11] * 400 + [50000], [0] * 260 + [9]]


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32, None], ids=["bf16", "fp16", "fp32", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=[f"{len(s)}x{max(s)}" for s in SIZES])
def test_clip_gradients(train, sizes, dtype):
    gen = torch.Generator(device="cuda").manual_seed(sum(sizes))
    make = lambda: [torch.randn(n, generator=gen, device="cuda").to(dtype or (BF16, FP32, FP16)[i % 3]) for i, n in enumerate(sizes)]  # noqa: E731
    for limit in (0.25, 1e9, float("inf"), 0.0):
        check(train, make(), limit)


@gpu
def test_sizes_that_32_bits_do_not_square(train):
    """1e-30 and 1e30: their squares are no floats."""
    for size in (1e-30, 1e30):
        g = [torch.full((1000,), size, device="cuda"), torch.full((30,), -size, device="cuda")]
        check(train, [t.clone() for t in g], size * 3, eps=0.0)
        check(train, [t.bfloat16() for t in g], size * 3, eps=0.0)


@gpu
def test_a_norm_that_is_not_finite_changes_nothing(train):
    for bad in (float("nan"), float("inf"), -float("inf")):
        g = [torch.randn(5000, device="cuda"), torch.randn(20, device="cuda").bfloat16()]
        g[0][4321] = bad
        before = [t.clone() for t in g]
        norm = train.clip_gradients(g, 0.1)
        assert not norm.isfinite() and all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(g, before))
    g = [torch.full((4,), 3e38, device="cuda")]                      # the norm is no float, yet a number
    assert train.clip_gradients(g, 1.0).isinf() and (g[0] - 0.5).abs().max() < 1e-6


@gpu
def test_orders_of_dimensions_strides_and_none(train):
    gen = torch.Generator(device="cuda").manual_seed(3)
    base = torch.randn(7, 40, 11, generator=gen, device="cuda")
    flat = torch.randn(5000, generator=gen, device="cuda").bfloat16()
    g = [base.permute(2, 0, 1), flat[1:999], flat[1001:4001].view(-1, 1, 3), torch.randn((), generator=gen, device="cuda"), None, torch.randn(2, 3, 4, 4, generator=gen, device="cuda").to(memory_format=torch.channels_last)]
    edge = flat[[0, 999, 1000, 4001]].clone()
    given = [t for t in g if t is not None]
    exact = [t.double().clone() for t in given]
    norm = train.clip_gradients(g, 1.0)
    factor = 1.0 / math.sqrt(sum(t.pow(2).sum().item() for t in exact))
    for t, e in zip(given, exact):
        assert ((t.double() - e * factor).abs() <= (HALF[t.dtype] + 4 * U32) * (e * factor).abs() * (1 + 2.0 ** -6) + 1e-12).all()
    assert torch.equal(flat[[0, 999, 1000, 4001]], edge) and norm > 1
    for bad in ([base[:, ::2]], [flat[:10], flat[:10]], [flat[:10], flat[9:20]], [torch.ones((), device="cuda").expand(5)]):
        with pytest.raises((ValueError, train.OnesError)):
            train.clip_gradients(bad, 1.0)


@gpu
def test_equal_bits_streams_and_graphs(train):
    gen = torch.Generator(device="cuda").manual_seed(5)
    fresh = [torch.randn(n, generator=gen, device="cuda").bfloat16() for n in (300000, 17, 70001)]
    one, two = [t.clone() for t in fresh], [t.clone() for t in fresh]
    want = train.clip_gradients(one, 1.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = train.clip_gradients(two, 1.5)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(one, two))
    graph, held = torch.cuda.CUDAGraph(), [t.clone() for t in fresh]
    with torch.cuda.graph(graph):
        found = train.clip_gradients(held, 1.5)
    for i in range(3):
        for t, f in zip(held, fresh):
            t.copy_(f * (1 + i))
        eager = [t.clone() for t in held]
        graph.replay()
        torch.cuda.synchronize()
        norm = train.clip_gradients(eager, 1.5)
        assert torch.equal(found, norm) and all(torch.equal(a, b) for a, b in zip(held, eager)), i


@gpu
@pytest.mark.parametrize("limit", [1.0, 1e-3, 1e-6])
def test_factors_that_32_bits_do_not_hold(train, limit):
    """A million elements of 3e38 (norm 3e41): limit / norm is no normal float, every element times it is."""
    for dtype in (FP32, BF16):
        g = [torch.full((1000000,), 3e38, device="cuda", dtype=dtype), torch.full((30,), -1e37, device="cuda", dtype=dtype)]
        exact = [t.double() for t in g]
        norm = math.sqrt(sum(t.pow(2).sum().item() for t in exact))
        assert train.clip_gradients(g, limit).isinf()
        for t, e in zip(g, exact):
            want = e * (limit / (norm + 1e-6))
            assert ((t.double() - want).abs() <= (HALF[dtype] + 4 * U32) * want.abs()).all()
