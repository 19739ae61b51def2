"""Layer norm and the gated recurrence against their formulas in 64 bits.

Tolerances.  An output of a 16-bit or 32-bit type is rounded once, by eps / 2 of its value; the 32-bit arithmetic before it has an error of
a few 2^-24 per operation on terms of the sizes that are summed, taken as so many 2^-24 of the largest such term."""
import ctypes as C

import numpy as np
import pytest
import torch

HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
U32 = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def train():
    import os

    from paper_2108_03645_amd import ones
    if not os.path.exists(ones.library_path()):
        pytest.skip("libones.so not built here")
    from paper_2108_03645_amd import train as binding
    binding.load()
    return binding


def near(got, want, terms, operations, what):
    """|got - want| <= half a step of the type at want + operations * 2^-24 * the size of the terms (16-bit denormals: a step)."""
    want = want.double()
    tiny = 2.0 ** -24 if got.dtype == torch.float16 else 0.0
    bound = HALF[got.dtype] * want.abs() * (1 + 2.0 ** -7) + operations * U32 * terms.double() + tiny + 1e-37
    off = (got.double() - want).abs()
    worst = (off - bound).max().item() if off.numel() else 0.0
    assert worst <= 0, f"{what}: {worst} beyond the bound; off by {off.max().item()}"


# ---------------------------------------------------------------- refusals (CPU) ------
def test_refusals_need_no_gpu(train):
    L = train.load()
    p = C.c_void_p(0x1000)
    norm = lambda x=p, stride=8, rows=2, cols=8, kind=2, wkind=0, eps=1e-5, y=p: L.ones_layer_norm_forward(  # noqa: E731
        x, stride, rows, cols, kind, None, None, wkind, eps, y, p, p, None)
    assert norm(x=None) == norm(y=None) == norm(stride=7) == norm(rows=-1) == norm(cols=0, stride=0) == norm(kind=3) == -1
    assert norm(kind=2, wkind=1) == norm(eps=-1.0) == norm(eps=float("nan")) == -1
    assert norm(cols=32769, stride=32769) == norm(rows=1 << 40, stride=1 << 20) == -3
    assert norm(rows=0, x=None, y=None) == 0                       # nothing to do, nothing launched
    need = L.ones_layer_norm_workspace_bytes(100, 1000)
    assert need >= 2 * 1000 * 4 and L.ones_layer_norm_workspace_bytes(1, 0) == 0 and L.ones_layer_norm_workspace_bytes(-1, 5) == 0
    back = lambda ws, n, dy=p, rows=100: L.ones_layer_norm_backward(dy, 1000, p, 1000, rows, 1000, 0, None, 0, p, p, p, p, p, ws, n, None)  # noqa: E731
    assert back(None, need) == back(p, need, dy=None) == -1
    assert back(p, need - 1) == back(C.c_void_p(0x1010), need) == -5

    rec = lambda g=p, b=2, t=5, c=7, kind=2, h=p, step=7: L.ones_recurrence_forward(  # noqa: E731
        g, 35, step, p, 35, 7, b, t, c, kind, None, None, h, None, None, None, 0, None)
    assert rec(g=None) == rec(h=None) == rec(b=-1) == rec(t=-1) == rec(c=-1) == rec(kind=9) == rec(step=-7) == -1
    assert rec(b=65536) == rec(t=(1 << 30) + 1) == rec(c=(1 << 24) + 1) == rec(step=1 << 33) == rec(b=65535, t=1 << 30, c=1 << 24) == -3
    assert rec(b=0, g=None) == rec(c=0, g=None) == 0
    assert L.ones_recurrence_carry_bytes(2, 129, 7) == 2 * 2 * 7 * 4 and L.ones_recurrence_carry_bytes(-1, 1, 1) == 0
    assert L.ones_recurrence_workspace_bytes(512, 100000, 64) == 0      # enough sequences: the steps are not split
    need = L.ones_recurrence_workspace_bytes(1, 100000, 64)
    assert need > 0
    long = lambda ws, n: L.ones_recurrence_forward(p, 0, 64, p, 0, 64, 1, 100000, 64, 0, None, None, p, None, None, ws, n, None)  # noqa: E731
    assert long(None, 0) == -1 and long(p, need - 1) == -5
    assert L.ones_recurrence_backward(None, 1, 1, None, p, 1, 1, p, 1, 1, 1, 1, 1, 0, p, None, p, p, None, None, 0, None) == -1
    assert L.ones_recurrence_backward(p, 1, 1, None, p, 1, 1, p, 1, 1, 1, 1, 1, 0, None, None, p, p, None, None, 0, None) == -1
    assert L.ones_recurrence_step(p, 8, p, 8, 1, 8, 0, None, p, None) == L.ones_recurrence_step(p, -8, p, 8, 1, 8, 0, p, p, None) == -1
    assert L.ones_recurrence_step(None, 8, None, 8, 0, 8, 0, None, None, None) == 0


def test_the_header_and_the_binding_name_the_same_functions(train):
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "ones_train.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(ones_[a-z_]+)\s*\(", text)))
    assert declared == sorted(train.EXPORTS) == sorted(train._ARGUMENTS)
    assert all(hasattr(train.load(), name) for name in declared)


def test_the_binding_refuses_on_the_cpu(train):
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(train.OnesError):
        train.layer_norm_forward(x)
    with pytest.raises(TypeError):
        train.layer_norm_forward(x.double())
    with pytest.raises(TypeError):
        train.layer_norm_forward(3.0)
    with pytest.raises(TypeError):
        train.gated_recurrence_forward(x, x.int())


# --------------------------------------------------------------------- layer norm ------
def norm64(x, w, b, eps, dy):
    x, dy = x.double(), dy.double()
    d = x.shape[-1]
    mean = x.mean(-1)
    c = x - mean[..., None]
    rstd = (c.pow(2).mean(-1) + eps) ** -0.5
    xh = c * rstd[..., None]
    w = torch.ones(d, device=x.device).double() if w is None else w.double()
    b = torch.zeros(d, device=x.device).double() if b is None else b.double()
    g = dy * w
    dx = rstd[..., None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    lead = tuple(range(x.dim() - 1))
    return xh * w + b, mean, rstd, dx, (dy * xh).sum(lead), dy.sum(lead), xh


NORMS = [(1, 1), (1, 2), (3, 7), (5, 64), (2, 513), (67, 1001), (130, 1024), (9, 2048), (9, 2049), (21, 4096), (3, 8191), (6, 8200),
         (2, 32768), (2, 32767), (1, 8), (5000, 40)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,cols", NORMS)
def test_layer_norm(train, rows, cols, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows * 40000 + cols)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    kind = dtype if cols % 2 else torch.float32
    x, dy = (make(rows, cols) * 1.5 + 3).to(dtype), make(rows, cols).to(dtype)
    w, b = (make(cols) * 0.2 + 1).to(kind), make(cols).to(kind)
    y, mean, rstd = train.layer_norm_forward(x, w, b, 1e-5)
    dx, dw, db = train.layer_norm_backward(dy, x, w, mean, rstd)
    wy, wm, wr, wdx, wdw, wdb, xh = norm64(x, w, b, 1e-5, dy)
    assert (y.dtype, dx.dtype, dw.dtype, db.dtype) == (dtype, dtype, kind, kind)
    size = x.double().abs().amax(-1, keepdim=True)
    # the mean of so many values: pairwise in effect (a run in registers, then a tree): 32 + log2 of the threads
    near(mean, wm, size[:, 0], 48, "mean")
    near(rstd, wr, wr * (1 + size[:, 0] ** 2 * wr ** 2), 64, "rstd")
    off = 1 + size * wr[:, None]                                  # what an error of the mean becomes in xh, and of rstd
    amplified = off * (1 + size * wr[:, None])
    near(y, wy, amplified * w.double().abs() * (1 + xh.abs()) + b.double().abs(), 80, "y")
    g = (dy.double() * w.double()).abs()
    near(dx, wdx, wr[:, None] * amplified * (g + g.mean(-1, keepdim=True) * (1 + xh.abs()) ** 2), 200, "dx")
    near(dw, wdw, (dy.double().abs() * amplified * (1 + xh.abs())).sum(0), 200, "dweight")
    near(db, wdb, dy.double().abs().sum(0), 64 + rows // 256, "dbias")
    again = train.layer_norm_backward(dy, x, w, mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))


@gpu
def test_layer_norm_strides_shapes_and_missing_weights(train):
    gen = torch.Generator(device="cuda").manual_seed(5)
    wide = torch.randn(40, 3 * 96 + 5, generator=gen, device="cuda").to(torch.bfloat16)
    for x in (wide[:, 96:192], wide[:, 1:97], wide[::3, :96], wide.t()[:64, :33], wide[:36, :96].reshape(4, 9, 96), wide[0, :96], torch.randn(96, generator=gen, device="cuda").bfloat16().expand(7, 96)):
        dy = torch.randn(x.shape, generator=gen, device="cuda").to(torch.bfloat16)
        y, mean, rstd = train.layer_norm_forward(x)
        flat, flat_dy = x.reshape(-1, x.shape[-1]), dy.reshape(-1, x.shape[-1])
        wy, wm, _, wdx, wdw, wdb, _ = norm64(flat, None, None, 1e-5, flat_dy)
        assert y.shape == x.shape and mean.shape == rstd.shape == x.shape[:-1]
        near(y.reshape(wy.shape), wy, wy.abs() + 1, 300, "y")
        dx, dw, db = train.layer_norm_backward(dy, x, None, mean, rstd, want_bias=False)
        assert db is None and dw.dtype == torch.float32
        near(dx.reshape(wdx.shape), wdx, wdx.abs() + 20, 300, "dx")
        near(dw, wdw, flat_dy.double().abs().sum(0) * 4, 300, "dweight")
        # a gradient that is one number everywhere, as sum() leaves it
        one = torch.ones((), device="cuda", dtype=torch.bfloat16).expand(x.shape)
        _, _, ones_db = train.layer_norm_backward(one, x, None, mean, rstd)
        assert torch.equal(ones_db, torch.full_like(ones_db, flat.shape[0]))


@gpu
def test_layer_norm_of_nothing_and_of_rows_without_spread(train):
    w = torch.ones(24, device="cuda")
    x = torch.zeros(0, 24, device="cuda", dtype=torch.float16)
    y, mean, rstd = train.layer_norm_forward(x, w, w)
    dx, dw, db = train.layer_norm_backward(x, x, w, mean, rstd)
    assert y.shape == dx.shape == (0, 24) and torch.equal(dw, torch.zeros_like(w)) and torch.equal(db, torch.zeros_like(w))
    flat = torch.full((3, 24), 7.0, device="cuda")
    flat[1, 5] = float("nan")
    flat[2, 3] = float("inf")
    y, mean, rstd = train.layer_norm_forward(flat, w, w * 2)
    assert torch.equal(y[0], torch.full_like(y[0], 2.0)) and abs(rstd[0].item() - 1e-5 ** -0.5) < 1e-3
    assert y[1].isnan().all() and y[2].isnan().all()
    # a large common offset: the centred sum of squares keeps what x - mean has
    x = torch.randn(4, 1000, device="cuda") + 4096
    y, mean, rstd = train.layer_norm_forward(x)
    wy, _, wr, *_ = norm64(x, None, None, 1e-5, x)
    assert ((rstd.double() - wr).abs() / wr).max() < 1e-6
    assert (y.double() - wy).abs().max() < 4096 * 16 * U32


@gpu
def test_layer_norm_gradients_under_autograd_against_differences(train):
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(3, 50, generator=gen, device="cuda", requires_grad=True)
    w = torch.randn(50, generator=gen, device="cuda", requires_grad=True)
    b = torch.randn(50, generator=gen, device="cuda", requires_grad=True)
    v = torch.randn(3, 50, generator=gen, device="cuda")
    (train.layer_norm(x, w, b) * v).sum().backward()

    def f(x, w, b):
        return (norm64(x, w, b, 1e-5, x)[0] * v.double()).sum()

    for t in (x, w, b):
        direction = torch.randn(t.shape, generator=gen, device="cuda").double()
        h = 1e-4
        moved = [[u.detach().double() + (s * h * direction if u is t else 0) for u in (x, w, b)] for s in (1, -1)]
        difference = (f(*moved[0]) - f(*moved[1])) / (2 * h)
        assert abs((t.grad.double() * direction).sum() - difference) < 1e-4 * (1 + abs(difference))   # h^2 and 2^-24 of the sums


# ---------------------------------------------------------------------- recurrence ------
def recurrence64(gate, x, state, lengths, dh, dlast):
    b, t, c = x.shape
    gate, x, dh = gate.double(), x.double(), dh.double()
    a, keep = torch.sigmoid(gate), torch.sigmoid(-gate)
    h = torch.zeros(b, c, device=x.device, dtype=torch.float64) if state is None else state.double()
    lengths = torch.full((b,), t, device=x.device) if lengths is None else lengths.long().clamp(0, t)
    hs, before = torch.zeros_like(x), torch.zeros_like(x)
    for i in range(t):
        live = (i < lengths)[:, None]
        before[:, i] = h
        h = torch.where(live, a[:, i] * h + keep[:, i] * x[:, i], h)
        hs[:, i] = torch.where(live, h, torch.zeros_like(h))
    dgate, dx = torch.zeros_like(x), torch.zeros_like(x)
    back = torch.zeros(b, c, device=x.device, dtype=torch.float64) if dlast is None else dlast.double()
    for i in range(t - 1, -1, -1):
        live = (i < lengths)[:, None]
        lam = dh[:, i] + back
        zero = torch.zeros_like(lam)
        dx[:, i] = torch.where(live, keep[:, i] * lam, zero)
        dgate[:, i] = torch.where(live, lam * (before[:, i] - x[:, i]) * a[:, i] * keep[:, i], zero)
        back = torch.where(live, a[:, i] * lam, back)
    return hs, h, dgate, dx, back


RUNS = [(1, 1, 1), (2, 3, 5), (1, 127, 64), (3, 128, 65), (2, 129, 66), (4, 300, 128), (1, 2000, 40), (1, 1500, 61), (2, 700, 4),
        (200, 20, 68), (1, 5003, 8)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("batch,steps,channels", RUNS)
def test_recurrence(train, batch, steps, channels, dtype):
    gen = torch.Generator(device="cuda").manual_seed(steps * 1000 + channels)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    gate, x, dh = ((make(batch, steps, channels) * k).to(dtype) for k in (3, 1, 1))
    state, dlast, lengths = make(batch, channels), make(batch, channels), None
    if steps % 2:
        lengths = torch.randint(0, steps + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
        lengths[-1] = 0 if batch > 1 else steps // 2
        # what lies past the length is not read
        for i, n in enumerate(lengths.tolist()):
            gate[i, n:], x[i, n:], dh[i, n:] = float("nan"), float("inf"), float("nan")
    if channels % 3 == 0:
        state = dlast = None
    h, last, carry = train.gated_recurrence_forward(gate, x, state, lengths)
    dgate, dx, dstate = train.gated_recurrence_backward(dh, dlast, gate, x, carry, lengths)
    clean = [torch.nan_to_num(v, 0.0, 0.0, 0.0) for v in (gate, x, dh)]
    wh, wlast, wdgate, wdx, wdstate = recurrence64(clean[0], clean[1], state, lengths, clean[2], dlast)
    # every product of gates is at most 1 and (1 - a) sums to 1 - A: an error of one step (six roundings: exp, sum, quotient,
    # product, sum) is passed on with weight a; the sums that the weights make are 1 / (1 - a) steps long, and one composed
    # run adds as many again.  Sizes: the largest state, the largest lambda.
    a = torch.sigmoid(clean[0].double())
    reach = torch.clamp(1 / (1 - a).mean((0, 1)).clamp(min=1e-9), max=float(steps)) + 8   # per channel, in steps
    slow = torch.clamp(1 / (1 - a).amin((0, 1)).clamp(min=1e-9), max=float(steps)) + 8
    top = wh.abs().amax((0, 1)) + clean[1].double().abs().amax((0, 1)) + (0 if state is None else state.double().abs().amax(0))
    lam = (wdx.abs() / (1 - a).clamp(min=1e-30)).amax((0, 1)) + clean[2].double().abs().amax((0, 1)) + (0 if dlast is None else dlast.double().abs().amax(0))
    n = 16
    near(h, wh, (top * slow).expand_as(wh), n, "h")
    near(last, wlast, (top * slow).expand_as(wlast), n, "last")
    near(dx, wdx, (lam * slow).expand_as(wdx), n, "dx")
    near(dgate, wdgate, (lam * top * slow * 2).expand_as(wdgate), n, "dgate")
    near(dstate, wdstate, (lam * slow).expand_as(wdstate), n, "dstate")
    assert reach.isfinite().all()
    if lengths is not None:
        for i, k in enumerate(lengths.tolist()):
            assert not h[i, k:].any() and not dgate[i, k:].any() and not dx[i, k:].any()


@gpu
def test_recurrence_steps_equal_the_scan_and_update_the_state_in_place(train):
    gen = torch.Generator(device="cuda").manual_seed(3)
    for channels, dtype in ((64, torch.bfloat16), (33, torch.float16), (8, torch.float32)):
        gate, x = (torch.randn(5, 40, channels, generator=gen, device="cuda").to(dtype) for _ in range(2))
        state = torch.randn(5, channels, generator=gen, device="cuda")
        want, wlast, *_ = recurrence64(gate, x, state, None, x, None)
        at = state.data_ptr()
        for t in range(40):
            g, u = (gate[:, t], x[:, t]) if t % 2 else (gate[:, t:t + 1], x[:, t:t + 1])     # rows of a longer array
            h = train.gated_recurrence_step(g, u, state)
            assert h.shape == u.shape
            near(h.reshape(5, channels), want[:, t], torch.full_like(want[:, t], 4.0), 16 * 40, f"step {t}")
        assert state.data_ptr() == at
        near(state, wlast, torch.full_like(wlast, 4.0), 16 * 40, "state")
    with pytest.raises(ValueError):
        train.gated_recurrence_step(x[:, 0], x[:, 0], torch.zeros(8, 5, device="cuda").t())


@gpu
def test_recurrence_of_no_steps_and_saturated_gates(train):
    state = torch.randn(3, 10, device="cuda")
    none = torch.zeros(3, 0, 10, device="cuda")
    h, last, carry = train.gated_recurrence_forward(none, none, state)
    assert h.shape == (3, 0, 10) and torch.equal(last, state)
    dgate, dx, dstate = train.gated_recurrence_backward(none, state * 2, none, none, carry)
    assert dgate.shape == (3, 0, 10) and torch.equal(dstate, state * 2)
    for value, dtype in ((200.0, torch.float32), (-200.0, torch.float32), (float("inf"), torch.bfloat16), (float("-inf"), torch.float16)):
        gate = torch.full((3, 150, 10), value, device="cuda", dtype=dtype)
        x = torch.randn(3, 150, 10, device="cuda").to(dtype)
        h, last, carry = train.gated_recurrence_forward(gate, x, state)
        want = state[:, None].expand(3, 150, 10) if value > 0 else x.float()
        assert torch.equal(h.float(), want.to(dtype).float()) and torch.equal(last, want[:, -1].float())
        dgate, dx, dstate = train.gated_recurrence_backward(x, None, gate, x, carry)
        assert not dgate.float().abs().gt(1e-30).any() and dx.isfinite().all()
        if value < 0:
            assert torch.equal(dx, x)


@gpu
def test_recurrence_strides_autograd_and_differences(train):
    gen = torch.Generator(device="cuda").manual_seed(12)
    both = torch.randn(2, 37, 2, 24, generator=gen, device="cuda")
    gate = both[:, :, 0].requires_grad_(False)
    x = both[:, :, 1]
    state = torch.randn(2, 24, generator=gen, device="cuda")
    dh, dlast = torch.randn(2, 37, 24, generator=gen, device="cuda"), torch.randn(2, 24, generator=gen, device="cuda")
    plain = train.gated_recurrence_forward(gate.contiguous(), x.contiguous(), state)
    strided = train.gated_recurrence_forward(gate, x, state)
    turned = train.gated_recurrence_forward(gate.transpose(0, 1).contiguous().transpose(0, 1), x.transpose(1, 2).contiguous().transpose(1, 2), state)
    for p, q, r in zip(plain, strided, turned):
        assert torch.equal(p, q) and torch.equal(p, r)
    leaves = [gate.clone().requires_grad_(), x.clone().requires_grad_(), state.clone().requires_grad_()]
    h, last = train.gated_recurrence(*leaves)
    ((h * dh).sum() + (last * dlast).sum()).backward()

    def f(g, u, s):
        hs, end, *_ = recurrence64(g, u, s, None, u, None)
        return (hs * dh.double()).sum() + (end * dlast.double()).sum()

    for t in leaves:
        direction = torch.randn(t.shape, generator=gen, device="cuda").double()
        moved = [[u.detach().double() + (s * 1e-4 * direction if u is t else 0) for u in leaves] for s in (1, -1)]
        difference = (f(*moved[0]) - f(*moved[1])) / 2e-4
        assert abs((t.grad.double() * direction).sum() - difference) < 1e-4 * (1 + abs(difference))
    # only one of the outputs is used, with a gradient that is one number
    g2 = gate.clone().requires_grad_()
    train.gated_recurrence(g2, x)[1].sum().backward()
    want = recurrence64(gate, x, None, None, torch.zeros_like(x), torch.ones_like(state))[2]
    near(g2.grad, want, want.abs() + 1, 300, "dgate from the last state")
    wide = torch.zeros(2, 1, 24, device="cuda").expand(2, 37, 24)              # one gate for all steps
    h, _, _ = train.gated_recurrence_forward(wide, x, None)
    near(h, recurrence64(wide, x, None, None, x, None)[0], torch.full_like(h, 4.0), 300, "repeated gate")


@gpu
def test_another_stream_and_a_captured_graph_give_the_same(train):
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn(300, 520, generator=gen, device="cuda").bfloat16() for _ in range(2))
    seq = torch.randn(1, 3000, 64, generator=gen, device="cuda").bfloat16()

    def all_of_it():
        y, mean, rstd = train.layer_norm_forward(x)
        got = [y, *train.layer_norm_backward(dy, x, None, mean, rstd)]
        h, last, carry = train.gated_recurrence_forward(seq, seq)
        return got + [h, last, *train.gated_recurrence_backward(seq, last, seq, seq, carry)]

    want = [t.clone() for t in all_of_it()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_of_it()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_it()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        assert all(torch.equal(p, q) for p, q in zip(all_of_it(), want))
    assert np.isfinite(want[0].float().sum().item())


@gpu
@pytest.mark.parametrize("rows,cols,kind", [(1, 512, torch.float16), (16, 37, torch.float32), (17, 511, torch.float16), (64, 256, torch.float32),
                                            (64, 512, torch.float16), (65, 512, torch.float16), (64, 513, torch.float16)])
def test_layer_norm_of_few_rows_sums_its_weights_gradients(train, rows, cols, kind):
    """Around the sizes that one workgroup takes alone; without weights, and with one of the two gradients only."""
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    x, dy = (torch.randn(rows, cols, generator=gen, device="cuda").half() for _ in range(2))
    w = (torch.randn(cols, generator=gen, device="cuda") + 2).to(kind)
    y, mean, rstd = train.layer_norm_forward(x, w)
    *_, wdx, wdw, wdb, xh = norm64(x, w, None, 1e-5, dy)
    dx, dw, db = train.layer_norm_backward(dy, x, w, mean, rstd)
    assert dw.dtype == db.dtype == kind
    near(dx, wdx, wdx.abs() + 20, 300, "dx")
    near(dw, wdw, (dy.double().abs() * (1 + xh.abs())).sum(0), 300, "dweight")
    near(db, wdb, dy.double().abs().sum(0), 128, "dbias")
    again = train.layer_norm_backward(dy, x, w, mean, rstd, want_bias=False)
    assert again[2] is None and torch.equal(again[0], dx) and torch.equal(again[1], dw)
    assert torch.equal(train.layer_norm_backward(dy, x, None, mean, rstd)[2].to(kind), db)


@gpu
def test_results_that_go_past_the_caches_are_the_same(train):
    """Results of 64 MiB and more are written with a hint: the same rows in a smaller call give the same bits, odd columns too."""
    gen = torch.Generator(device="cuda").manual_seed(21)
    for cols in (1024, 1027):
        x = torch.randn(33000, cols, generator=gen, device="cuda").bfloat16()
        y, mean, rstd = train.layer_norm_forward(x)
        few = train.layer_norm_forward(x[-300:])
        assert all(torch.equal(p[-300:], q) for p, q in zip((y, mean, rstd), few))
        dx = train.layer_norm_backward(x, x, None, mean, rstd)[0]
        assert torch.equal(dx[-300:], train.layer_norm_backward(x[-300:], x[-300:], None, mean[-300:], rstd[-300:])[0])
    for channels in (256, 259):
        gate, x, dh = (torch.randn(200, 700, channels, generator=gen, device="cuda").bfloat16() for _ in range(3))
        lengths = torch.randint(0, 701, (200,), generator=gen, device="cuda", dtype=torch.int32)
        h, last, carry = train.gated_recurrence_forward(gate, x, None, lengths)
        back = train.gated_recurrence_backward(dh, None, gate, x, carry, lengths)
        want, want_last, few = train.gated_recurrence_forward(gate[:50], x[:50], None, lengths[:50])
        bound = 2 * HALF[torch.bfloat16] * (want.double().abs() + 2.0 ** -8)          # other segments: other roundings of 32 bits
        assert ((h[:50].double() - want.double()).abs() <= bound).all() and torch.allclose(last[:50], want_last, rtol=1e-4, atol=1e-5)
        for got, one in zip(back, train.gated_recurrence_backward(dh[:50], None, gate[:50], x[:50], few, lengths[:50])):
            assert ((got[:50].double() - one.double()).abs() <= 2 * HALF[torch.bfloat16] * (one.double().abs() + 2.0 ** -8)).all()


def test_a_single_token_of_any_size_is_not_refused(train):
    """Up to the limits of batch and channels; a state that is missing shows that the sizes were taken."""
    L, p = train.load(), C.c_void_p(0x1000)
    step = lambda b, c: L.ones_recurrence_step(p, c, p, c, b, c, 2, None, p, None)  # noqa: E731
    assert step(65535, 8192) == step(65535, 1 << 24) == step(1, 1 << 24) == -1
    assert step(65536, 8) == step(1, (1 << 24) + 1) == -3


@gpu
@pytest.mark.parametrize("batch,channels", [(65535, 8192), (65535, 1031)])
def test_a_single_token_of_many_sequences(train, batch, channels):
    """More than 2^16 workgroups' worth: a thread takes several runs of channels."""
    gen = torch.Generator(device="cuda").manual_seed(channels)
    gate, x = (torch.randn(batch, channels, generator=gen, device="cuda").bfloat16() for _ in range(2))
    state = torch.randn(batch, channels, generator=gen, device="cuda")
    parts = [slice(0, 300), slice(40000, 40300), slice(batch - 300, batch)]
    held = [state[rows].clone() for rows in parts]
    h = train.gated_recurrence_step(gate, x, state)
    for rows, old in zip(parts, held):
        want, end, *_ = recurrence64(gate[rows, None], x[rows, None], old, None, x[rows, None], None)
        near(h[rows], want[:, 0], torch.full_like(end, 8.0), 16, "h")
        near(state[rows], end, torch.full_like(end, 8.0), 16, "state")


def test_many_sequences_of_few_steps_are_not_refused(train):
    L, p = train.load(), C.c_void_p(0x1000)
    run = lambda b, t, c: L.ones_recurrence_forward(p, t * c, c, p, t * c, c, b, t, c, 2, None, None, None, None, None, None, 0, None)  # noqa: E731
    assert run(65535, 2, 8192) == run(4096, 1, 1 << 24) == run(65535, 300, 1 << 20) == -1       # taken, but h is missing
    assert run(4097, 1, 1 << 24) == -3


@gpu
@pytest.mark.parametrize("channels", [8192, 8190])
def test_recurrence_of_many_sequences_of_few_steps(train, channels):
    """2^24 workgroups, more than one dimension of a launch takes; every third sequence has one step only."""
    batch, steps = 65535, 2
    gen = torch.Generator(device="cuda").manual_seed(channels)
    gate, x, dh = (torch.randn(batch, steps, channels, generator=gen, device="cuda").bfloat16() for _ in range(3))
    lengths = torch.full((batch,), steps, device="cuda", dtype=torch.int32)
    lengths[::3] = 1
    state = torch.randn(batch, channels, generator=gen, device="cuda")
    h, last, carry = train.gated_recurrence_forward(gate, x, state, lengths)
    dgate, dx, dstate = train.gated_recurrence_backward(dh, state, gate, x, carry, lengths)
    for rows in (slice(0, 300), slice(32700, 33000), slice(batch - 300, batch)):
        want = recurrence64(gate[rows], x[rows], state[rows], lengths[rows], dh[rows], state[rows])
        for got, one, what in zip((h, last, dgate, dx, dstate), want, ("h", "last", "dgate", "dx", "dstate")):
            near(got[rows], one, torch.full_like(one, 64.0), 32, what)


def test_what_is_updated_in_place_is_known_to_autograd(train, monkeypatch):
    """A backward pass that needs the old state or momentum raises, as behind torch's own in-place operators; no GPU: the call is left out."""
    monkeypatch.setattr(train, "_check", lambda *a, **k: None)
    monkeypatch.setattr(train, "_call", lambda *a: None)
    x = torch.zeros(2, 8)
    for shape, change in (((2, 8), lambda t: train.gated_recurrence_step(x, x, t)), ((8, 8), lambda t: train.orthogonal_update(torch.zeros(8, 8), t))):
        leaf = torch.ones(shape, requires_grad=True)
        held = leaf * 2
        loss = held.square().sum()                                    # keeps held
        with torch.no_grad():
            change(held)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        with torch.inference_mode():
            change(torch.ones(shape))
