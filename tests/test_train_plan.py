"""Which kernels a size reaches, asked of the plans themselves (csrc/train_plan.h, compiled here for the host), and the results of
every shape of tile of every matrix product, and of every cut of the recurrence, at sizes that reach it.

The tolerances are those of the other files.  An element of the update is held to eight times what the whole may be off by, as a share of
the elements' root mean square (the errors are sums of many roundings of either sign, so that six deviations are not passed by any of 10^7
elements): an element that is missing or out of place is off by that root mean square itself."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from test_train_loss import check
from test_train_norm_recurrence import HALF, U32, near, recurrence64, train  # noqa: F401
from test_train_update import ABC, IN_PAIRS, update64

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LARGE, MIDDLE, DEEP, SMALL, TINY = range(5)
SHIM = r"""
#include "train_plan.h"
using namespace ones::train;
extern "C" {
void loss(int64_t rows, int64_t cols, int64_t words, int64_t *to) {
  const LossPlan p = loss_plan(rows, cols, words, true, false, true);
  const int64_t out[] = {p.logits, p.logits_piece, p.gradients.tiles, p.gradients.of_dx.splits, p.gradients.of_dw.splits, p.piece, p.pieces};
  std::copy(out, out + 7, to);
}
void blocks(int64_t rows, int64_t cols, int64_t words, int64_t *to) {
  const LossPlan p = loss_plan(rows, cols, words, true, false, true);
  const int64_t out[] = {p.block, p.blocks, p.piece, static_cast<int64_t>((p.dx_sum ? p.dx_sum : p.backward) - p.g)};
  std::copy(out, out + 4, to);
}
// Threads of the largest launch of either call.
void launch(int64_t rows, int64_t cols, int64_t words, int64_t *to) {
  *to = 0;
  if (check_loss(rows, cols, words, cols, cols, ONES_BF16) != ONES_OK) return;
  const LossPlan p = loss_plan(rows, cols, words, true, true, true);
  const int64_t some = std::min(rows, p.block), piece = std::min(p.piece, words);
  const Split dx = p.gradients.of_dx, dw = p.gradients.of_dw;
  const TileCost &c = kTileCosts[p.gradients.tiles], &f = kTileCosts[p.logits];
  const int64_t threads = p.gradients.tiles == kTiny ? 256 : 512;
  const int64_t products = ceil_div(cols, c.bm) * (ceil_div(some, c.bn) * dx.splits + ceil_div(piece, c.bn) * dw.splits) * threads;
  const int64_t finish = (dx.splits > 1 ? some * cols : 0) + (p.blocks > 1 || dw.splits > 1 ? piece * cols : 0);
  *to = std::max({products, finish, 2 * ceil_div(words, f.bm) * ceil_div(rows, f.bn), rows * 128});      // the logits' tiles have 31 bits; 8 rows a join
}
void update(int64_t count, int64_t rows, int64_t cols, int64_t *to) {
  const UpdateTiles t = update_tiles(count, std::min(rows, cols), std::max(rows, cols), false);
  to[0] = t.gram; to[1] = t.poly; to[2] = t.apply;
}
void update_in_pairs(int64_t count, int64_t rows, int64_t cols, int64_t *to) {
  const UpdateTiles t = update_tiles(count, std::min(rows, cols), std::max(rows, cols), true);
  to[0] = t.gram; to[1] = t.poly; to[2] = t.apply;
}
void recurrence(int64_t batch, int64_t steps, int64_t channels, int64_t backward, int64_t *to) {
  const Cut c = cut_of(batch, steps, channels, backward != 0);
  to[0] = c.lanes; to[1] = c.segments;
}
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("plan")
    (at / "shim.cpp").write_text(SHIM)
    subprocess.check_call([gxx, "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", f"-I{ROOT}/include", f"-I{ROOT}/paper_2108_03645_amd/csrc",
                           str(at / "shim.cpp"), "-o", str(at / "shim.so")])
    L = C.CDLL(str(at / "shim.so"))

    def ask(name, n, *sizes):
        out = (C.c_int64 * n)()
        getattr(L, name)(*(C.c_int64(s) for s in sizes), out)
        return tuple(out)

    return ask


# (rows, cols, words): tiles of the logits forward, of a piece's logits, of the gradients; parts of k of dx and of dW; pieces
LOSSES = {
    (100, 16, 17081): (DEEP, DEEP, TINY, 30, 1, 1),
    (149, 40, 17081): (SMALL, SMALL, TINY, 30, 1, 1),
    (17081, 24, 101): (DEEP, SMALL, TINY, 1, 30, 1),
    (146, 24, 35423): (LARGE, LARGE, TINY, 31, 1, 1),
    (101, 547, 2755): (TINY, TINY, DEEP, 15, 1, 1),
    (4765, 550, 99): (TINY, TINY, SMALL, 1, 25, 1),
    (767, 162, 29519): (SMALL, SMALL, LARGE, 31, 1, 1),
    (1329, 2774, 1593): (DEEP, DEEP, LARGE, 1, 1, 1),
    (2035, 770, 32799): (LARGE, SMALL, DEEP, 1, 1, 2),
    (4103, 250, 12267): (LARGE, LARGE, DEEP, 1, 1, 2),
    (17083, 71, 3971): (LARGE, LARGE, SMALL, 1, 8, 2),
    (11861, 546, 8237): (SMALL, SMALL, LARGE, 1, 2, 2),
    (8191, 1022, 16999): (LARGE, LARGE, LARGE, 1, 1, 3),
    (6001, 1030, 24001): (LARGE, LARGE, SMALL, 1, 1, 3),
}
# (count, rows, cols): tiles of A, of B, of X
UPDATES = {
    (40, 267, 269): (DEEP, DEEP, SMALL),
    (40, 415, 417): (SMALL, SMALL, LARGE),
    (5, 3287, 70): (TINY, TINY, DEEP),
    (8, 4177, 131): (TINY, TINY, LARGE),
    (1, 1083, 3679): (TINY, TINY, MIDDLE),
    (16, 1049, 643): (MIDDLE, SMALL, LARGE),
    (40, 541, 543): (LARGE, LARGE, SMALL),
    (2, 65, 131): (TINY, TINY, TINY),
    (1, 2999, 2047): (DEEP, DEEP, SMALL),
    (1, 3001, 2999): (MIDDLE, MIDDLE, LARGE),
    (2, 4101, 2047): (MIDDLE, MIDDLE, MIDDLE),
}
# the same where the operands are held in pairs (fp16 results)
PAIRS = {
    (2, 131, 65): (TINY, TINY, TINY),
    (40, 267, 269): (DEEP, DEEP, SMALL),
    (40, 415, 417): (SMALL, SMALL, LARGE),
    (5, 3287, 70): (TINY, TINY, DEEP),
    (8, 4177, 131): (TINY, TINY, LARGE),
    (3, 3599, 349): (TINY, TINY, MIDDLE),
    (16, 643, 645): (MIDDLE, MIDDLE, LARGE),
    (40, 541, 543): (LARGE, LARGE, SMALL),
    (2, 4101, 2047): (MIDDLE, MIDDLE, MIDDLE),
}
# (batch, steps, channels): lanes and segments forward, and backward
RECURRENCES = {
    (96, 1101, 130): (8, 1, 16, 1),
    (48, 1030, 256): (8, 1, 16, 1),
    (200, 1101, 160): (8, 1, 16, 1),
    (200, 1100, 161): (8, 1, 16, 1),
    (1, 8301, 4100): (16, 8, 16, 8),
    (1, 8300, 4098): (16, 8, 16, 8),
}


@pytest.mark.parametrize("sizes", LOSSES, ids=str)
def test_tiles_of_the_loss(plans, sizes):
    *found, _, pieces = plans("loss", 7, *sizes)
    assert (*found, pieces) == LOSSES[sizes]


@pytest.mark.parametrize("sizes", UPDATES, ids=str)
def test_tiles_of_the_update(plans, sizes):
    assert plans("update", 3, *sizes) == UPDATES[sizes]


@pytest.mark.parametrize("sizes", PAIRS, ids=str)
def test_tiles_of_the_update_in_pairs(plans, sizes):
    assert plans("update_in_pairs", 3, *sizes) == PAIRS[sizes]


@pytest.mark.parametrize("sizes", RECURRENCES, ids=str)
def test_cuts_of_the_recurrence(plans, sizes):
    assert plans("recurrence", 2, *sizes, 0) + plans("recurrence", 2, *sizes, 1) == RECURRENCES[sizes]


def test_the_sizes_reach_every_shape_of_every_product():
    for shapes, of in (((LARGE, DEEP, SMALL, TINY), [[p[k] for p in LOSSES.values()] for k in range(3)]),
                       (range(5), [[p[k] for p in UPDATES.values()] for k in range(3)]), (range(5), [[p[k] for p in PAIRS.values()] for k in range(3)])):
        assert all(set(shapes) == set(reached) for reached in of)
    # dx added up over pieces of the vocabulary and rounded behind the last, by each of the tiles that large calls take
    assert {p[2] for p in LOSSES.values() if p[3] == 1 and p[5] > 1} == {LARGE, DEEP, SMALL}


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("sizes", LOSSES, ids=str)
def test_loss_of_every_shape(train, sizes, dtype):  # noqa: F811
    rows, cols, words = sizes
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(words, cols, generator=gen, device="cuda") * 1.5 / cols ** 0.5).to(dtype)
    t = torch.randint(0, words, (rows,), generator=gen, device="cuda")
    t[torch.rand(rows, generator=gen, device="cuda") < 0.1] = -100
    t[0], t[-1] = words - 1, -1
    x[t < 0] = float("nan")
    check(train, x, w, t, torch.rand(rows, generator=gen, device="cuda") / rows)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("sizes", UPDATES, ids=str)
def test_update_of_every_shape(train, sizes, dtype):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(sum(sizes))
    g = (torch.randn(*sizes, generator=gen, device="cuda") * 1e-2).to(dtype)
    m = torch.randn(*sizes, generator=gen, device="cuda") * 0.1
    held = m.clone()
    got = train.orthogonal_update(g, m, 0.95, True, 5, ABC, 1e-7)
    want, moved = update64(g, held, 0.95, True, 5, ABC, 1e-7)
    off = (got.double() - want).abs()
    whole = want.flatten(1).norm(dim=1)
    assert (off.flatten(1).norm(dim=1) <= (5.7e-3 + HALF[dtype]) * whole).all()
    mean = (whole / (sizes[1] * sizes[2]) ** 0.5)[:, None, None]
    assert (off <= 8 * 5.7e-3 * mean + HALF[dtype] * want.abs() * (1 + 2.0 ** -7)).all()
    assert ((m.double() - moved).abs() <= 3 * U32 * (held.double().abs() + g.double().abs())).all()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("sizes", RECURRENCES, ids=str)
def test_recurrence_of_every_cut(train, sizes, dtype):  # noqa: F811
    batch, steps, channels = sizes
    gen = torch.Generator(device="cuda").manual_seed(steps + channels)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    gate, x, dh = ((make(batch, steps, channels) * k).to(dtype) for k in (3, 1, 1))
    state, dlast, lengths = make(batch, channels), make(batch, channels), None
    if steps % 2:
        lengths = torch.randint(0, steps + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
        lengths[-1] = steps // 2
        past = torch.arange(steps, device="cuda")[None, :] >= lengths[:, None]
        gate[past], x[past], dh[past] = float("nan"), float("inf"), float("nan")
    h, last, carry = train.gated_recurrence_forward(gate, x, state, lengths)
    dgate, dx, dstate = train.gated_recurrence_backward(dh, dlast, gate, x, carry, lengths)
    if lengths is not None:
        gate[past], x[past], dh[past] = 0, 0, 0
        assert not h[past].any() and not dgate[past].any() and not dx[past].any()
    wh, wlast, wdgate, wdx, wdstate = recurrence64(gate, x, state, lengths, dh, dlast)
    # an error of a step (six roundings) is passed on for 1 / (1 - a) steps at most, and composed runs add as many again
    keep = torch.sigmoid(-gate.double())
    slow = torch.clamp(1 / keep.amin((0, 1)), max=float(steps)) + 8
    top = wh.abs().amax((0, 1)) + x.double().abs().amax((0, 1)) + state.double().abs().amax(0)
    lam = (wdx.abs() / keep).amax((0, 1)) + dh.double().abs().amax((0, 1)) + dlast.double().abs().amax(0)
    near(h, wh, (top * slow).expand_as(wh), 16, "h")
    near(last, wlast, (top * slow).expand_as(wlast), 16, "last")
    near(dx, wdx, (lam * slow).expand_as(wdx), 16, "dx")
    near(dgate, wdgate, (lam * top * slow * 2).expand_as(wdgate), 16, "dgate")
    near(dstate, wdstate, (lam * slow).expand_as(wdstate), 16, "dstate")


def test_the_logits_gradients_lie_no_further_apart_than_the_products_load(plans, train):  # noqa: F811
    """Rows of what the products load lie 2^20 elements apart at most: 256 rows at offsets of 32 bits."""
    for rows, cols, words in ((1, 8, 1 << 24), (3, 24, (1 << 20) + 1), (2, 8, 1 << 20), (63, 64, 1 << 21), (500, 8, 1 << 24)):
        *_, piece, pieces = plans("loss", 7, rows, cols, words)
        assert piece <= 1 << 20 and (pieces - 1) * piece < words <= pieces * piece
    L, p = train.load(), C.c_void_p(0x1000)
    wide = L.ones_cross_entropy_forward_workspace_bytes(4, 64, 100, 1)
    for xs, ws in ((64, (1 << 20) + 8), ((1 << 20) + 8, 64)):
        assert L.ones_cross_entropy_forward(p, xs, p, ws, 4, 64, 100, 2, p, p, p, p, wide, None) == -5
    wide = L.ones_cross_entropy_backward_workspace_bytes(4, 64, 100, 1)
    assert L.ones_cross_entropy_backward(p, p, 64, p, (1 << 20) + 8, 4, 64, 100, 2, p, p, p, p, p, wide, None) == -5


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_loss_of_few_rows_over_a_vocabulary_of_millions(train, dtype):  # noqa: F811
    words = (1 << 20) + 300
    gen = torch.Generator(device="cuda").manual_seed(23)
    x = torch.randn(3, 24, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(words, 24, generator=gen, device="cuda") * 0.3).to(dtype)
    check(train, x, w, torch.tensor([words - 1, 5, 1 << 19], device="cuda"), torch.rand(3, generator=gen, device="cuda"))


@gpu
def test_loss_of_rows_as_far_apart_as_the_products_load(train):  # noqa: F811
    """2^20 elements: loaded as they lie, with the workspace that has no room for copies; eight more: copied."""
    gen = torch.Generator(device="cuda").manual_seed(29)
    for stride in (1 << 20, (1 << 20) + 8):
        apart = torch.empty(300 * stride, dtype=torch.bfloat16, device="cuda").as_strided((300, 64), (stride, 1))
        apart.copy_(torch.randn(300, 64, generator=gen, device="cuda"))
        other = (torch.randn(270, 64, generator=gen, device="cuda") * 0.2).bfloat16()
        check(train, other, apart, torch.randint(0, 300, (270,), generator=gen, device="cuda"), torch.rand(270, generator=gen, device="cuda"))
        check(train, apart, other, torch.randint(0, 270, (300,), generator=gen, device="cuda"), torch.rand(300, generator=gen, device="cuda"))


def test_the_logits_gradients_that_are_held_stay_below_128_mib(plans, train):  # noqa: F811
    """Whatever the rows: x's copy and the 32-bit sum of dx grow with them, nothing else of the workspace."""
    size = train.load().ones_cross_entropy_backward_workspace_bytes
    for rows, cols, words in ((1 << 18, 8, 1000), ((1 << 18) + 1, 8, 1000), (300000, 64, 500), (524288, 8, 1000), (1 << 20, 24, 5000), (1 << 24, 8, 1000),
                              (1 << 24, 128, 17)):
        block, blocks, piece, held = plans("blocks", 4, rows, cols, words)
        assert held <= 128 << 20 and block * piece * 2 <= 128 << 20 and (blocks - 1) * block < rows <= blocks * block
        assert size(rows, cols, words, 1) <= rows * cols * 6 + (256 << 20)
    assert plans("blocks", 4, 1 << 18, 8, 1000)[1] == 1 and plans("blocks", 4, (1 << 18) + 1, 8, 1000)[1] == 2


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("cols,words", [(24, 700), (33, 90)])
def test_loss_of_rows_in_blocks(train, cols, words, dtype):  # noqa: F811
    """Two blocks of rows with two pieces of the vocabulary, or one; the second block is shorter, a run of ignored rows reaches over both."""
    rows = (1 << 18) + 301
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(words, cols, generator=gen, device="cuda") * 1.5 / cols ** 0.5).to(dtype)
    t = torch.randint(0, words, (rows,), generator=gen, device="cuda")
    t[131000:131500], t[-1] = -100, words - 1
    x[t < 0] = float("nan")
    check(train, x, w, t, torch.rand(rows, generator=gen, device="cuda") / rows)


def test_launches_of_every_accepted_size_of_the_loss_fit(plans):
    """A grid has less than 2^32 threads: at the corners of what is accepted, and between them."""
    largest = 0
    sizes = lambda top: [v for k in range(0, top + 1, 2) for v in (1 << k, (1 << k) * 3 // 2 + 1) if v <= 1 << top]  # noqa: E731
    for rows in sizes(24):
        for cols in sizes(16):
            for words in sizes(24):
                largest = max(largest, *plans("launch", 1, rows, cols, words))
    assert 1 << 28 < largest < 1 << 32


@gpu
@pytest.mark.parametrize("sizes", PAIRS, ids=str)
def test_update_of_every_shape_in_pairs(train, sizes):  # noqa: F811
    """Element by element: half a step of fp16, and eight times (as above) what 22 bits leave of the whole."""
    gen = torch.Generator(device="cuda").manual_seed(sum(sizes))
    g = torch.randn(*sizes, generator=gen, device="cuda") * 1e-2
    m = torch.randn(*sizes, generator=gen, device="cuda") * 0.1
    want, _ = update64(g, m, 0.95, True, 5, ABC, 1e-7)
    got = train.orthogonal_update(g, m, 0.95, True, 5, ABC, 1e-7, dtype=torch.float16)
    off, mean = (got.double() - want).abs(), want.square().mean((1, 2), keepdim=True).sqrt()
    assert (off <= HALF[torch.float16] * want.abs() * (1 + 2.0 ** -7) + 8 * IN_PAIRS * mean + 2.0 ** -24).all(), (off / mean).max().item()
