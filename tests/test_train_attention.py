"""Causal attention over packed sequences and its single-token form against their formulas in 64 bits.

Tolerances.  A rounding to 16 bits is off by up to half a step, h = eps / 2 of the value.  The forward call rounds the exponentials (numerator
and denominator alike) and the result; scores, sums and exponentials of 32 bits are off by some 2^-24 of the terms that they are made of, which
moves an exponential by that much of itself.  Backward, p or ds are rounded and the result, and delta carries what the forward's
exponentials were rounded by.  Every bound below adds these up, term by term, for the worst signs; beside it, over a thousand elements and more, the
root mean square of the error is held to h: it is made of up to three roundings with an rms of h / 3^0.5 each."""
import ctypes as C

import pytest
import torch

from test_train_norm_recurrence import HALF, U32, train  # noqa: F401

gpu = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


def offsets_of(lengths, front=0):
    ends = [front]
    for n in lengths:
        ends.append(ends[-1] + n)
    return ends


def attention64(q, k, v, ends, scale, do=None):
    """The formulas, one head of one sequence after another, and beside every result the sum of its terms' sizes."""
    n, h, d = q.shape
    kv = k.shape[1]
    new = lambda *s: torch.zeros(*s, device=q.device, dtype=torch.float64)  # noqa: E731
    r = {"o": new(n, h, d), "lse": torch.full((h, n), -float("inf"), device=q.device, dtype=torch.float64), "z": new(h, n), "so": new(n, h, d)}
    if do is not None:
        r.update({name: new(n, h if name.endswith("q") else kv, d) for name in ("dq", "dk", "dv", "sdq", "sdk", "sdv", "edq", "edk")})
    for lo, hi in zip(ends, ends[1:]):
        for head in range(h if hi > lo else 0):
            of = head // (h // kv)
            qs, ks, vs = q[lo:hi, head].double(), k[lo:hi, of].double(), v[lo:hi, of].double()
            live = torch.ones(hi - lo, hi - lo, device=q.device, dtype=torch.bool).tril()
            z = (torch.mm(qs, ks.t()) * scale).masked_fill(~live, -float("inf"))
            p = torch.softmax(z, 1)
            r["lse"][head, lo:hi] = torch.logsumexp(z, 1)
            r["z"][head, lo:hi] = (torch.mm(qs.abs(), ks.abs().t()) * scale).masked_fill(~live, 0).amax(1)
            r["o"][lo:hi, head] = torch.mm(p, vs)
            r["so"][lo:hi, head] = torch.mm(p, vs.abs())
            if do is not None:
                g = do[lo:hi, head].double()
                dp = torch.mm(g, vs.t())
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                # what an error of delta or of dp, relative to the terms they are sums of, becomes
                each = torch.mm(g.abs(), vs.abs().t()) * live
                loose = p * (each + (p * each).sum(1, keepdim=True))
                r["dq"][lo:hi, head] = torch.mm(ds, ks) * scale
                r["sdq"][lo:hi, head] = torch.mm(ds.abs(), ks.abs()) * scale
                r["edq"][lo:hi, head] = torch.mm(loose, ks.abs()) * scale
                r["dk"][lo:hi, of] += torch.mm(ds.t(), qs) * scale
                r["sdk"][lo:hi, of] += torch.mm(ds.abs().t(), qs.abs()) * scale
                r["edk"][lo:hi, of] += torch.mm(loose.t(), qs.abs()) * scale
                r["dv"][lo:hi, of] += torch.mm(p.t(), g)
                r["sdv"][lo:hi, of] += torch.mm(p.t(), g.abs())
    return r


def held(got, want, bound, what, rms=True):
    h = HALF[got.dtype]
    off = (got.double() - want).abs()
    tiny = 2.0 ** -24 if got.dtype == FP16 else 1e-37
    over = off - bound - h * want.abs() * (1 + 2.0 ** -7) - tiny
    assert not off.isnan().any(), f"{what}: NaN"
    assert over.numel() == 0 or over.max() <= 0, f"{what}: {over.max().item()} beyond the bound, off by {off.max().item()}"
    if rms and got.numel() >= 1000 and want.norm() > 0 and got.dtype in (BF16, FP16):
        share = ((got.double() - want).norm() / want.norm()).item()
        assert share <= h, f"{what}: off by {share:.2e} of its norm, {h:.2e} is held"


def check(train, q, k, v, ends, do=None, scale=None, rms=True):
    h = HALF[q.dtype]
    s = q.shape[2] ** -0.5 if scale is None else scale
    offsets = torch.tensor(ends, device=q.device, dtype=torch.int32)
    r = attention64(q, k, v, ends, s, do)
    o, lse, rest = train.attention_forward(q, k, v, offsets, scale, keep_rest=do is not None)
    longest = max([b - a for a, b in zip(ends, ends[1:])] + [1])
    e = (q.shape[2] + 32) * U32 * r["z"]                            # of a score: relative, of its exponential
    few = (longest + 64) * U32                                       # of a sum over keys
    inside = torch.zeros(q.shape[0], dtype=torch.bool, device=q.device)
    inside[ends[0]:ends[-1]] = True
    rows = e.t()[..., None]
    held(o, r["o"], r["so"] * (2 * h + 2 * rows + few), "o", rms)
    assert torch.equal(o[~inside], torch.zeros_like(o[~inside])) and torch.isneginf(lse[:, ~inside]).all()
    held(lse[:, inside], r["lse"][:, inside], (e + few + 2.0 ** -20 + 4 * U32 * r["lse"].abs())[:, inside], "lse")
    if do is None:
        return (o, lse)
    assert rest.shape == o.shape and torch.equal(rest[~inside], torch.zeros_like(rest[~inside]))
    held((o.float() + rest.float()), r["o"], r["so"] * (2 * h + 2 * rows + few) + h * h * r["o"].abs() + 2.0 ** -24, "o and rest")
    dq, dk, dv = train.attention_backward(do, q, k, v, o, lse, rest, offsets, scale)
    loose = 2 * h + 4 * e.max() + 2 * few
    held(dq, r["dq"], r["sdq"] * (h + 2 * e.max() + few) + r["edq"] * loose, "dq", rms)
    held(dk, r["dk"], r["sdk"] * (h + 2 * e.max() + few) + r["edk"] * loose, "dk", rms)
    held(dv, r["dv"], r["sdv"] * (h + 2 * e.max() + few), "dv", rms)
    for t in (dq, dk, dv):
        assert torch.equal(t[~inside], torch.zeros_like(t[~inside]))
    again = train.attention_backward(do, q, k, v, o, lse, rest, offsets, scale)
    assert all(torch.equal(x, y) for x, y in zip(again, (dq, dk, dv)))
    return o, lse, rest, dq, dk, dv


def inputs(seed, n, heads, kv, dim, dtype, std=1.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda h, s: (torch.randn(n, h, dim, generator=g, device="cuda") * s).to(dtype)  # noqa: E731
    return make(heads, std), make(kv, std), make(kv, 1.0), make(heads, 0.05)


# ---------------------------------------------------------------- refusals (CPU) ------
def test_refusals_need_no_gpu(train):
    L = train.load()
    p = C.c_void_p(0x1000)
    fwd = lambda q=p, qs=128, qh=64, tokens=5, heads=2, kv=1, dim=64, kind=2, off=p, seqs=1, scale=0.1, o=p, lse=p, ks=64: L.ones_attention_forward(  # noqa: E731
        q, qs, qh, p, ks, 64, p, 64, 64, tokens, heads, kv, dim, kind, off, seqs, scale, o, None, lse, None)
    for bad in (fwd(q=None), fwd(q=C.c_void_p(0x1008)), fwd(qs=100), fwd(qs=32), fwd(qh=4), fwd(tokens=-1), fwd(heads=3, kv=2), fwd(heads=0), fwd(kv=0),
                fwd(dim=60), fwd(dim=0), fwd(kind=0), fwd(kind=7), fwd(off=None), fwd(seqs=-1), fwd(scale=0.0), fwd(scale=-1.0), fwd(scale=float("nan")),
                fwd(scale=float("inf")), fwd(o=None), fwd(lse=None), fwd(o=C.c_void_p(0x1002))):
        assert bad == -1
    assert fwd(dim=136) == fwd(tokens=(1 << 30) + 1) == fwd(heads=2048) == fwd(qs=(1 << 20) + 8) == fwd(tokens=1 << 30, heads=8) == -3
    assert fwd(tokens=0, q=None, off=None, o=None, lse=None) == 0
    need = L.ones_attention_workspace_bytes(1000, 3, 4, 2, 64)
    assert need >= 4 * 1000 * 4 and L.ones_attention_workspace_bytes(1000, 3, 4, 3, 64) == 0
    back = lambda ws=p, n=need, do=p, dq=p, o=p: L.ones_attention_backward(  # noqa: E731
        do, 256, 64, p, 256, 64, p, 128, 64, p, 128, 64, 1000, 4, 2, 64, 1, p, 3, 0.1, o, None, p, dq, p, p, ws, n, None)
    assert back(do=None) == back(dq=None) == back(o=None) == back(ws=None) == -1
    assert back(n=need - 1) == back(ws=C.c_void_p(0x1010)) == -5
    step = lambda q=p, keys=p, b=2, cap=9, heads=4, kv=2, dim=64, kind=1, kb=9 * 128, ks=128, kh=64, lengths=p, scale=0.1, o=p: L.ones_attention_step(  # noqa: E731
        q, 256, 64, p, 128, 64, p, 128, 64, keys, kb, ks, kh, p, 9 * 128, 128, 64, lengths, b, cap, heads, kv, dim, kind, scale, o, None, 0, None)
    for bad in (step(q=None), step(keys=None), step(b=-1), step(cap=-1), step(heads=3), step(dim=12), step(kind=0), step(kb=-8), step(kb=9), step(ks=32),
                step(lengths=None), step(scale=0.0), step(o=None), step(keys=C.c_void_p(0x1008))):
        assert bad == -1
    assert step(b=65536) == step(cap=(1 << 30) + 1) == step(ks=(1 << 20) + 8) == step(b=60000, heads=128, kv=128) == step(kb=1 << 50) == -3
    assert step(b=0, q=None, keys=None, o=None) == 0
    assert L.ones_attention_step_workspace_bytes(1, 100000, 8, 2, 64) > 0 and L.ones_attention_step_workspace_bytes(1, 100, 8, 2, 64) == 0
    assert step(kb=0) == step(kb=56) == step(kh=0) == step(kh=56) == -1     # two places of a cache in one
    assert step(b=1, cap=100000) == -1                               # split over the keys: a workspace is needed


def test_the_binding_refuses_on_the_cpu(train):
    q, k = torch.zeros(4, 2, 8, dtype=BF16), torch.zeros(4, 1, 8, dtype=BF16)
    with pytest.raises(train.OnesError):
        train.attention_forward(q, k, k)
    with pytest.raises(TypeError):
        train.attention_forward(q.float(), k, k)
    with pytest.raises(TypeError):
        train.attention_forward(None, k, k)
    with pytest.raises(train.OnesError):
        train.attention_step(q, k, k, torch.zeros(4, 9, 1, 8, dtype=BF16), torch.zeros(4, 9, 1, 8, dtype=BF16), torch.zeros(4, dtype=torch.int32))


# ------------------------------------------------------------- packed sequences ------
SHAPES = [([1], 1, 1, 8), ([2], 2, 1, 64), ([0, 1, 0, 5, 0], 4, 2, 40), ([127, 128, 129], 3, 3, 64), ([300, 0, 1, 64, 65], 6, 2, 80), ([1000], 4, 1, 128),
          ([5] * 70 + [0] * 3 + [33], 2, 2, 72), ([31, 32, 33, 63, 64, 65, 95, 96, 97], 8, 2, 128), ([257, 2], 16, 2, 96), ([513], 7, 7, 16), ([1, 1, 1], 1, 1, 128)]


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("lengths,heads,kv,dim", SHAPES, ids=[f"{len(s[0])}x{sum(s[0])}-{s[1]}-{s[2]}-{s[3]}" for s in SHAPES])
def test_attention(train, lengths, heads, kv, dim, dtype):
    n = sum(lengths)
    check(train, *inputs(n * 131 + dim, n, heads, kv, dim, dtype)[:3], offsets_of(lengths))
    q, k, v, do = inputs(n * 131 + dim, n, heads, kv, dim, dtype)
    check(train, q, k, v, offsets_of(lengths), do, rms=max(lengths) >= 64)


# enough rows for workgroups of 128 queries; key heads of one and of more query heads (the parts of a group are summed behind, or there is one)
LARGE = [([5000, 3001, 333], 16, 2, 128, BF16), ([4099, 0, 4100], 16, 16, 64, FP16), ([8222], 16, 1, 96, FP16), ([1] * 50 + [4200, 3983], 32, 16, 32, BF16)]


@gpu
@pytest.mark.parametrize("lengths,heads,kv,dim,dtype", LARGE, ids=["128", "64", "96", "32"])
def test_attention_of_many_rows(train, lengths, heads, kv, dim, dtype):
    n = sum(lengths) + 3
    q, k, v, do = inputs(n + dim, n, heads, kv, dim, dtype)
    check(train, q, k, v, offsets_of(lengths), do)
    check(train, q, k, v, offsets_of(lengths))


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_rows_outside_all_sequences(train, dtype):
    """In front of the first and behind the last; what they hold is not read."""
    q, k, v, do = inputs(5, 400, 4, 2, 64, dtype)
    for t in (q, k, v, do):
        t[:37] = float("nan")
        t[37 + 250:] = float("inf")
    check(train, q, k, v, offsets_of([130, 0, 120], front=37), do)
    o, lse, _ = train.attention_forward(q, k, v, torch.zeros(1, device="cuda", dtype=torch.int32))      # no sequence at all
    assert not o.any() and torch.isneginf(lse).all()


@gpu
def test_a_sequence_does_not_see_its_neighbours(train):
    q, k, v, do = inputs(6, 300, 2, 1, 128, BF16)
    ends = offsets_of([100, 90, 110])
    want = check(train, q, k, v, ends, do)
    for t in (q, k, v, do):
        t[100:190] = float("nan")
    offsets = torch.tensor(ends, device="cuda", dtype=torch.int32)
    o, lse, rest = train.attention_forward(q, k, v, offsets, keep_rest=True)
    got = (o, lse.t(), rest, *train.attention_backward(do, q, k, v, o, lse, rest, offsets))
    want = (want[0], want[1].t(), *want[2:])
    for a, b in zip(got, want):
        assert torch.equal(a[:100], b[:100]) and torch.equal(a[190:], b[190:]) and a[100:190].isnan().all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("bad,n,heads", [(float("nan"), 200, 2), (float("inf"), 200, 2), (-float("inf"), 200, 2), (float("nan"), 200, 1), (float("nan"), 2310, 64)])
def test_a_row_does_not_see_what_comes_behind_it(train, bad, n, heads, dtype):
    """Infinities and NaN of a token reach its own row of o and dq and those behind it, its own of dk and dv and those before it, and no other.
    Rows that share a step with it are summed another way: either way is off by a share of h, so they differ by up to two (rest: by as much as o)."""
    def alike(got, right, what):
        size = want[0].float().norm() if what[1] == "rest" else right.float().norm()
        assert got.isfinite().all() and (got.float() - right.float()).norm() <= 2 * HALF[dtype] * size, what

    at = 77
    clean = inputs(30, n, heads, 1, 128, dtype)
    ends = offsets_of([n])
    offsets = torch.tensor(ends, device="cuda", dtype=torch.int32)
    want = check(train, *clean[:3], ends, clean[3])
    for which in range(4):                                           # q, k, v, do
        t = [x.clone() for x in clean]
        t[which][at, 0, 5:7] = bad
        o, lse, rest = train.attention_forward(*t[:3], offsets, keep_rest=True)
        dq, dk, dv = train.attention_backward(t[3], *t[:3], o, lse, rest, offsets)
        for name, got, right in (("o", o, want[0]), ("lse", lse.t(), want[1].t()), ("rest", rest, want[2]), ("dq", dq, want[3])):
            same = [i for i in range(n) if i < at or (which in (0, 3) and i != at)]
            alike(got[same], right[same], (which, name))
        if which in (0, 3):                                          # of a query: only the keys up to it
            alike(dk[at + 1:], want[4][at + 1:], (which, "dk"))
            alike(dv[at + 1:], want[5][at + 1:], (which, "dv"))
        if which == 2:
            assert not o[at:, 0, 5:7].isfinite().any() and o[at:, 0, 7:].isfinite().all()
        elif which == 3:
            assert not dv[:at + 1, 0, 5:7].isfinite().any() and dv[:, 0, 7:].isfinite().all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,heads,kv", [(200, 2, 1), (200, 1, 1), (2310, 64, 8)])
def test_what_keys_see_behind_what_they_do_not(train, n, heads, kv, bad, dtype):
    """Infinities and NaN in gradients at places that share a step with keys behind them, and at later ones that these keys see: dv holds what is seen, in
    that element and no other, and keys behind all of it are as they were."""
    q, k, v, do = inputs(33, n, heads, kv, 128, dtype)
    offsets = torch.tensor([0, n], device="cuda", dtype=torch.int32)
    o, lse, rest = train.attention_forward(q, k, v, offsets, keep_rest=True)
    clean = train.attention_backward(do, q, k, v, o, lse, rest, offsets)
    up = float("inf")
    for first, then in ((70, 90), (70, 150), (64, 127)):             # in one step of 32, in another tile, at a tile's ends
        g = do.clone()
        g[first, 0, 5], g[then, 0, 5], g[then, 0, 9] = bad, up, -up
        _, dk, dv = train.attention_backward(g, q, k, v, o, lse, rest, offsets)
        before = dv[:first + 1, 0, 5]
        assert (before == up).all() if bad == up else before.isnan().all()
        assert (dv[first + 1:then + 1, 0, 5] == up).all() and (dv[:then + 1, 0, 9] == -up).all()
        others = [d for d in range(128) if d not in (5, 9)]
        assert dv[:, 0, others].isfinite().all() and torch.equal(dv[:, 1:], clean[2][:, 1:]) and torch.equal(dk[:, 1:], clean[1][:, 1:])
        for got, right in ((dv[:, 0, others], clean[2][:, 0, others]), (dv[then + 1:], clean[2][then + 1:]), (dk[then + 1:], clean[1][then + 1:])):
            assert (got.float() - right.float()).norm() <= 2 * HALF[dtype] * right.float().norm()
    # in every step of 32: every key sees some, most do not see one of their own step
    for t, which in ((do, 0), (q, 1)):
        bads = t.clone()
        bads[::32, 0, 5] = bad
        last = (n - 1) // 32 * 32
        if which == 0:
            _, dk, dv = train.attention_backward(bads, q, k, v, o, lse, rest, offsets)
            seen = dv[:last + 1, 0, 5]
            assert (seen.isnan() if bad != bad else seen == bad).all() and dv[:, 0, others].isfinite().all()
        else:
            _, dk, dv = train.attention_backward(do, bads, k, v, *train.attention_forward(bads, k, v, offsets, keep_rest=True), offsets)
            assert not dk[:last + 1, 0].isfinite().any() and not dv[:last + 1, 0].isfinite().any()
        assert dk[last + 1:].isfinite().all() and dv[last + 1:].isfinite().all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_infinite_results_have_no_rest(train, dtype):
    """Nothing is rounded off infinity: o + rest is o there, in rows that saw it in a product and in rows that are summed again."""
    q, k, v, do = inputs(34, 300, 2, 1, 64, dtype)
    v[100, 0, 3], v[40, 0, 7] = float("inf"), -float("inf")
    k[40] = -30 * q[40:41, :1].sign()                                 # and one that most weights are small for
    o, _, rest = train.attention_forward(q, k, v, torch.tensor([0, 300], device="cuda", dtype=torch.int32), keep_rest=True)
    assert (o[100:, :, 3] == float("inf")).all() and (o[40:, :, 7] == -float("inf")).all()
    assert not rest[100:, :, 3].any() and not rest[40:, :, 7].any() and rest.isfinite().all() and rest.any()


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("n", [128, 130, 159, 300])
def test_keys_of_minus_infinity_have_no_weight(train, n, dtype):
    """A score of -infinity is a weight of 0: nothing of the key reaches o, its dk and dv are 0, whatever the length leaves of the last step."""
    q, k, v, do = inputs(36, n, 2, 1, 64, dtype)
    q = q.abs() + 1
    k[[5, 70, n - 1], 0, 3] = -float("inf")
    offsets = torch.tensor([0, n], device="cuda", dtype=torch.int32)
    o, lse, rest = train.attention_forward(q, k, v, offsets, keep_rest=True)
    _, dk, dv = train.attention_backward(do, q, k, v, o, lse, rest, offsets)
    assert all(t.isfinite().all() for t in (o, lse, rest, dk, dv))
    for key in (5, 70, n - 1):
        assert not dk[key].any() and not dv[key].any()
    assert dv[6].any() and dk[6].any()


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("n,heads", [(128, 1), (300, 1), (300, 4)])
def test_keys_far_below_the_largest_score_see_infinities(train, n, heads, dtype):
    """Weights of e^-200 are 0 in 32 bits: infinities in o's gradient reach dv, and those of values o, all the same."""
    q, do = torch.ones(n, heads, 64, device="cuda", dtype=dtype), torch.ones(n, heads, 64, device="cuda", dtype=dtype)
    k, v = torch.ones(n, 1, 64, device="cuda", dtype=dtype), torch.ones(n, 1, 64, device="cuda", dtype=dtype)
    k[10] = -24                                                      # scores 8 and -192
    offsets = torch.tensor([0, n], device="cuda", dtype=torch.int32)
    o, lse, rest = train.attention_forward(q, k, v, offsets, keep_rest=True)
    do[50, 0, 5], do[60, 0, 6], do[70, 0, 7], do[80, 0, 7] = float("inf"), -float("inf"), float("inf"), -float("inf")
    dv = train.attention_backward(do, q, k, v, o, lse, rest, offsets)[2]
    for key in (0, 10):
        assert dv[key, 0, 5] == float("inf") and dv[key, 0, 6] == -float("inf") and dv[key, 0, 7].isnan()
        assert dv[key, 0, 8:].isfinite().all() and dv[key, 0, :5].isfinite().all()
    assert dv[90:].isfinite().all() and not dv[10, 0, 8:].any()
    v[10, 0, 3] = float("inf")
    o = train.attention_forward(q, k, v, offsets)[0]
    assert (o[10:, :, 3] == float("inf")).all() and torch.equal(o[:10], q[:10]) and torch.equal(o[..., 4:], q[..., 4:])


@gpu
def test_what_every_row_sees_is_not_looked_for_again(train):
    """NaN that belongs in a row: the first token's value, every value, and every row at once; a long sequence takes no longer for it."""
    q, k, v, do = inputs(31, 30000, 1, 1, 64, BF16)
    offsets = torch.tensor([0, 30000], device="cuda", dtype=torch.int32)

    def timed():
        begun, ended = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begun.record()
        o, lse, rest = train.attention_forward(q, k, v, offsets, keep_rest=True)
        grads = train.attention_backward(do, q, k, v, o, lse, rest, offsets)
        ended.record()
        ended.synchronize()
        return o, grads, begun.elapsed_time(ended)

    timed()
    clean = timed()[2]
    v[0, 0, 3] = float("nan")
    o, (dq, dk, dv), took = timed()
    assert o[:, 0, 3].isnan().all() and o[:, 0, 4:].isfinite().all() and dq.isnan().any() and took < 20 * clean + 5
    v[0, 0, 3], v[20, 0, 3], v[40, 0, 3] = float("inf"), float("nan"), float("nan")
    o, _, took = timed()
    assert (o[:20, 0, 3] == float("inf")).all() and o[20:, 0, 3].isnan().all() and took < 20 * clean + 5
    v[20, 0, 3], v[40, 0, 3] = 1, -float("inf")
    o, _, took = timed()
    assert (o[:40, 0, 3] == float("inf")).all() and o[40:, 0, 3].isnan().all() and o[:, 0, 4:].isfinite().all() and took < 20 * clean + 5
    v[:] = float("nan")
    assert timed()[2] < 20 * clean + 5
    q[:], k[:], do[:] = (float("nan"),) * 3
    assert timed()[2] < 20 * clean + 5


@gpu
def test_many_sequences_and_offsets_that_do_not_rise(train):
    lengths = [(i * 7) % 4 for i in range(9001)]
    q, k, v, do = inputs(7, sum(lengths), 1, 1, 8, FP16)
    ends = offsets_of(lengths)
    o, lse, _ = train.attention_forward(q, k, v, torch.tensor(ends, device="cuda", dtype=torch.int32))
    # every sequence has up to three rows: the formula over its rows by their distance
    first = torch.tensor([e for e, m in zip(ends, lengths) for _ in range(m)], device="cuda")
    z = torch.full((len(first), 3), -float("inf"), device="cuda", dtype=torch.float64)
    at = torch.arange(len(first), device="cuda")
    for back in range(3):
        j = (at - back).clamp(min=0)
        z[:, back] = torch.where(at - back >= first, (q[:, 0].double() * k[j, 0].double()).sum(1) * 8 ** -0.5, z[:, back])
    p = torch.softmax(z, 1)
    want = sum(p[:, back, None] * v[(at - back).clamp(min=0), 0].double() for back in range(3))
    assert (o[:, 0].double() - want).abs().max() < 6 * 2.0 ** -11 * v.abs().max().item()
    assert (lse[0].double() - torch.logsumexp(z, 1)).abs().max() < 1e-4
    # offsets out of range or falling are pulled in: nothing outside is read or written
    for bad in ([0, 90, 40, 10 ** 9], [-5, 50, 60, 2 ** 31 - 1], [70, 10, 30, 20]):
        o, lse, rest = train.attention_forward(q[:100], k[:100], v[:100], torch.tensor(bad, device="cuda", dtype=torch.int32), keep_rest=True)
        train.attention_backward(do[:100], q[:100], k[:100], v[:100], o, lse, rest, torch.tensor(bad, device="cuda", dtype=torch.int32))
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_strides_and_alignments(train, dim):
    g = torch.Generator(device="cuda").manual_seed(8)
    rows = torch.randn(200, 8 * dim + 3, generator=g, device="cuda").to(BF16)
    heads_first = torch.randn(4, 200, dim, generator=g, device="cuda").to(BF16)
    do = torch.randn(200, 4, dim, generator=g, device="cuda").to(BF16) * 0.1
    packed = rows[:, :8 * dim].contiguous()
    for q, k, v in ((packed[:, :4 * dim].view(200, 4, dim), packed[:, 4 * dim:6 * dim].view(200, 2, dim), packed[:, 6 * dim:].view(200, 2, dim)),
                    (heads_first.transpose(0, 1), heads_first[1:3].transpose(0, 1), heads_first[2:].transpose(0, 1)),
                    (rows[:, 3:3 + 4 * dim].unflatten(1, (4, dim)), rows[:, 1:1 + dim].unflatten(1, (1, dim)), rows[:, 2:2 + dim].unflatten(1, (1, dim))),
                    (heads_first.permute(1, 0, 2).flip(2), heads_first[:1].transpose(0, 1), heads_first[3:].transpose(0, 1))):
        check(train, q, k, v, offsets_of([120, 80]), do)
    one = torch.full((), 0.5, device="cuda", dtype=BF16).expand(200, 4, dim)                    # a gradient that sum() leaves
    check(train, q, k, v, offsets_of([200]), one, rms=False)


@gpu
def test_rows_that_lie_far_apart(train):
    """Offsets beyond 2^31 elements."""
    base = torch.zeros(2200 << 20, device="cuda", dtype=BF16)
    far = base.view(2200, 1 << 20)
    g = torch.Generator(device="cuda").manual_seed(9)
    q, k, v, do = (torch.randn(2200, 1, 64, generator=g, device="cuda").to(BF16) for _ in range(4))
    for i, t in enumerate((q, k, v, do)):
        far[:, 64 * i:64 * i + 64] = t[:, 0]
    parts = [far[:, 64 * i:64 * i + 64].unsqueeze(1) for i in range(4)]
    offsets = torch.tensor([0, 2200], device="cuda", dtype=torch.int32)
    want = train.attention_forward(q, k, v, offsets, keep_rest=True)
    got = train.attention_forward(*parts[:3], offsets, keep_rest=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(train.attention_backward(parts[3], *parts[:3], *got, offsets), train.attention_backward(do, q, k, v, *want, offsets)))


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_large_and_small_scores(train, dtype):
    """Rows whose largest score comes late, all alike, far below zero, and a scale of its own."""
    q, k, v, do = inputs(10, 260, 2, 2, 64, dtype)
    rising = (torch.arange(260, device="cuda", dtype=torch.float32) / 26).to(dtype)
    check(train, q * 0 + 1, k * 0 + rising[:, None, None], v, offsets_of([260]), do, rms=False)
    check(train, q * 0 + 1, k * 0 - rising[:, None, None], v, offsets_of([260]), do, rms=False)
    check(train, q * 0, k, v, offsets_of([260]), do, rms=False)
    check(train, q, k, v, offsets_of([200, 60]), do, scale=0.37, rms=False)


@gpu
def test_fp16_gradients_of_very_different_sizes(train):
    """ds is held in units of its own: gradients of 2^-20 and rows of 2^-12 beside rows of 1 keep fp16's precision."""
    q, k, v, do = inputs(11, 700, 4, 2, 64, FP16)
    do = (do.float() * 20).half()
    do[300:] *= 2.0 ** -12                                           # a second sequence of small gradients
    ends = offsets_of([300, 400])
    check(train, q, k, v, ends, do)
    offsets = torch.tensor(ends, device="cuda", dtype=torch.int32)
    r = attention64(q, k, v, ends, 0.125, do)
    got = train.attention_backward(do, q, k, v, *train.attention_forward(q, k, v, offsets, keep_rest=True), offsets)
    for name, t in zip(("dq", "dk", "dv"), got):                     # as a share of the small ones alone; their own rounding: fp16's smallest
        want, part = r[name][300:], t[300:].double()
        assert (part - want).norm() <= HALF[FP16] * want.norm() + 2.0 ** -25 * want.numel() ** 0.5, name


@gpu
def test_fp16_gradients_far_below_those_in_front(train):
    """Units go by what a tile's rows see: keys whose queries all have gradients of 2^-15 keep fp16's precision behind queries with gradients of 2^14, and
    queries whose values are of 2^-12 in front of values of 2^12."""
    q, k, v, do = inputs(35, 900, 4, 2, 64, FP16)
    offsets = torch.tensor([0, 900], device="cuda", dtype=torch.int32)
    for which in ("dk", "dv", "dq"):
        g, u = do.float() / 0.05, v.float()
        if which == "dq":
            u[:512], u[512:] = u[:512] * 2.0 ** -12, u[512:] * 2.0 ** 12
            rows = slice(0, 512)
        else:
            g[:512], g[512:] = (g[:512] * 2.0 ** 14).clamp(-60000, 60000), g[512:] * 2.0 ** -15
            rows = slice(512, 900)
        t = q, k, u.half()
        g = g.half()
        r = attention64(*t, [0, 900], 0.125, g)
        got = dict(zip(("dq", "dk", "dv"), train.attention_backward(g, *t, *train.attention_forward(*t, offsets, keep_rest=True), offsets)))[which]
        want, part = r[which][rows], got[rows].double()
        # as above: of its norm the products' roundings, and its own where that is fp16's smallest
        assert (part - want).norm() <= HALF[FP16] * want.norm() + 2.0 ** -25 * want.numel() ** 0.5, which


@gpu
def test_gradients_under_autograd_against_differences(train):
    q, k, v, do = inputs(12, 90, 4, 2, 32, FP16, std=0.5)
    q, k, v = (t.requires_grad_() for t in (q, k, v))
    ends = offsets_of([50, 40])
    offsets = torch.tensor(ends, device="cuda", dtype=torch.int32)
    (train.attention(q, k, v, offsets).float() * do.float()).sum().backward()
    f = lambda *t: (attention64(*t, ends, 32 ** -0.5)["o"] * do.double()).sum()  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(13)
    for t in (q, k, v):
        direction = torch.randn(t.shape, generator=g, device="cuda").double()
        eps = 1e-3
        moved = [[u.detach().double() + (s * eps * direction if u is t else 0) for u in (q, k, v)] for s in (1, -1)]
        difference = (f(*moved[0]) - f(*moved[1])) / (2 * eps)
        # 2^-11 of the gradient's elements, in a random direction
        assert abs((t.grad.double() * direction).sum() - difference) < 6 * 2.0 ** -11 * t.grad.double().norm() + 1e-5 * (1 + abs(difference))


@gpu
def test_streams_graphs_and_two_calls_at_once(train):
    q, k, v, do = inputs(14, 900, 4, 2, 64, FP16)
    offsets = torch.tensor(offsets_of([500, 0, 380]), device="cuda", dtype=torch.int32)

    def both(q=q, do=do):
        o, lse, rest = train.attention_forward(q, k, v, offsets, keep_rest=True)
        return (o, lse, rest, *train.attention_backward(do, q, k, v, o, lse, rest, offsets))

    want = both()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for side in sides:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got.append(both())
    for side, one in zip(sides, got):
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(one, want))
    graph = torch.cuda.CUDAGraph()
    q2 = q.clone()
    with torch.cuda.graph(graph):
        found = both(q2)
    for i in range(3):
        q2.copy_(q * (1 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(found, both(q * (1 + i)))), i


@gpu
def test_the_binding_refuses(train):
    q, k, v, do = inputs(15, 10, 4, 2, 64, BF16)
    with pytest.raises(ValueError):
        train.attention_forward(q, k, v[:, :1])
    with pytest.raises(ValueError):
        train.attention_forward(q[:, :3], k, v)
    with pytest.raises(ValueError):
        train.attention_forward(q, k[:9], v)
    with pytest.raises(ValueError):
        train.attention_forward(q[..., :60], k[..., :60], v[..., :60])
    with pytest.raises(TypeError):
        train.attention_forward(q, k.half(), v)
    with pytest.raises(TypeError):
        train.attention_forward(q, k, v, torch.zeros(2, device="cuda", dtype=torch.int64))
    with pytest.raises(train.OnesError):
        train.attention_forward(q, k, v, scale=-1.0)
    wide = torch.zeros(10, 1, 136, device="cuda", dtype=BF16)
    with pytest.raises(train.OnesError):
        train.attention_forward(wide, wide, wide)


# -------------------------------------------------------------- single tokens ------
def step64(q, keys, values, k, v, lengths, scale):
    b, h, d = q.shape
    kv = k.shape[1]
    o, sizes, z_most = (torch.zeros(b, h, d, device=q.device, dtype=torch.float64) for _ in range(3))
    for i, n in enumerate(lengths):
        if n < 0:
            continue
        for head in range(h):
            of = head // (h // kv)
            ks, vs = torch.cat([keys[i, :n, of], k[i, of:of + 1]]).double(), torch.cat([values[i, :n, of], v[i, of:of + 1]]).double()
            p = torch.softmax(ks @ q[i, head].double() * scale, 0)
            o[i, head], sizes[i, head] = p @ vs, p @ vs.abs()
            z_most[i, head] = ((ks.abs() @ q[i, head].double().abs()) * scale).max()
    return o, sizes, z_most


STEPS = [([0], 1, 1, 1, 8), ([0, 1, 2, 5], 6, 4, 2, 64), ([31, 32, 33, 127, 128, 129, -1, 130], 131, 8, 8, 40), ([700, 3, 699], 800, 16, 1, 128),
         ([5000], 5001, 6, 2, 80), ([2000, 64], 2100, 34, 2, 64), ([300], 1 << 16, 20, 1, 128), ([255, 256, 257], 300, 3, 1, 72)]


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("lengths,capacity,heads,kv,dim", STEPS, ids=[f"{len(s[0])}x{max(s[0])}of{s[1]}-{s[2]}-{s[3]}-{s[4]}" for s in STEPS])
def test_attention_step(train, lengths, capacity, heads, kv, dim, dtype):
    b = len(lengths)
    g = torch.Generator(device="cuda").manual_seed(max(lengths) + dim)
    make = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).to(dtype)  # noqa: E731
    q, k, v, keys, values = make(b, heads, dim, std=1.3), make(b, kv, dim, std=1.3), make(b, kv, dim), make(b, capacity, kv, dim, std=1.3), make(b, capacity, kv, dim)
    for i, n in enumerate(lengths):                                  # what lies behind does not matter
        keys[i, max(n, 0):], values[i, max(n, 0):] = float("nan"), float("nan")
    before = keys.clone(), values.clone()
    o = train.attention_step(q, k, v, keys, values, torch.tensor(lengths, device="cuda", dtype=torch.int32))
    want, sizes, z = step64(q, *before, k, v, lengths, dim ** -0.5)
    held(o, want, sizes * (2 * HALF[dtype] + 2 * (dim + 32) * U32 * z + (max(lengths) + 64) * U32), "o")
    for cache, old, new in ((keys, before[0], k), (values, before[1], v)):
        for i, n in enumerate(lengths):
            if n >= 0:
                old[i, n] = new[i]
        assert torch.equal(cache.view(torch.int16), old.view(torch.int16))


SEEN = [(40, [39, 20]), (700, [65, 300]), (2048, [2000, 700]), (8192, [513, 65]), (1024, [65, 1023])]


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("capacity,lengths", SEEN, ids=[f"{s[1][0]}of{s[0]}" for s in SEEN])
def test_a_step_keeps_the_nan_and_infinities_that_it_sees(train, capacity, lengths, dtype):
    """In a key or a value of the first sequence's first key head: of the first place, the last one (alone in its part in some), many, the new token.  o is
    what the formula gives, and the other sequence and key head keep their bits."""
    b, heads, kv, dim = 2, 6, 2, 64
    g = torch.Generator(device="cuda").manual_seed(capacity)
    make = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).to(dtype)  # noqa: E731
    clean = make(b, heads, dim, std=1.3), make(b, kv, dim, std=1.3), make(b, kv, dim), make(b, capacity, kv, dim, std=1.3), make(b, capacity, kv, dim)
    at = torch.tensor(lengths, device="cuda", dtype=torch.int32)
    right = train.attention_step(*(t.clone() for t in clean), at)
    n = lengths[0]
    z = step64(clean[0], *clean[3:], *clean[1:3], lengths, dim ** -0.5)[2]
    for which in (0, 1):                                             # keys, values
        for bad in (float("nan"), float("inf"), -float("inf")):
            for places in (slice(0, 1), slice(n - 1, n), slice(n // 2, n), slice(0, n), None):
                t = [x.clone() for x in clean]
                (t[1 + which][0, 0] if places is None else t[3 + which][0, places, 0])[..., 5:7] = bad
                want, sizes, _ = step64(t[0], *t[3:], *t[1:3], lengths, dim ** -0.5)
                o = train.attention_step(*t, at)
                what = f"{('keys', 'values')[which]} {bad} {places}"
                assert torch.equal(o.isnan(), want.isnan()), what
                assert torch.equal(o.double()[want.isinf()], want[want.isinf()]), what
                good = want.isfinite()
                assert good.any(), what
                bound = sizes * (2 * HALF[dtype] + 2 * (dim + 32) * U32 * z + (n + 64) * U32)
                held(o[good], want[good], bound[good], what, rms=False)
                assert torch.equal(o[1], right[1]) and torch.equal(o[0, 3:], right[0, 3:]), what


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("capacity", [900, 4096])
def test_a_step_keeps_what_it_sees_far_below_the_largest_score(train, capacity, dtype):
    """Weights of e^-200 are 0 in 32 bits: what they stand for is seen all the same."""
    n, dim = 700, 64
    q, k, v = (torch.ones(1, h, dim, device="cuda", dtype=dtype) for h in (2, 1, 1))
    keys, values = torch.ones(1, capacity, 1, dim, device="cuda", dtype=dtype), torch.ones(1, capacity, 1, dim, device="cuda", dtype=dtype)
    keys[:, 300:] = -24                                              # scores 8 and -192
    at = torch.tensor([n], device="cuda", dtype=torch.int32)
    step = lambda: train.attention_step(q, k, v, keys, values, at)  # noqa: E731
    assert torch.equal(step(), q)
    values[0, 650, 0, 5], values[0, 651, 0, 6], values[0, 652, 0, 7] = float("inf"), -float("inf"), float("nan")
    values[0, 660, 0, 8], values[0, 310, 0, 8] = float("inf"), -float("inf")
    o = step()
    assert (o[..., 5] == float("inf")).all() and (o[..., 6] == -float("inf")).all() and o[..., 7:9].isnan().all()
    assert torch.equal(o[..., :5], q[..., :5]) and torch.equal(o[..., 9:], q[..., 9:])
    k[:], v[0, 0, 9] = -24, -float("inf")                            # the new token's
    assert (step()[..., 9] == -float("inf")).all() and torch.equal(step()[..., :5], q[..., :5])
    keys[0, 690, 0, 3] = float("nan")
    assert step().isnan().all()


@gpu
def test_a_step_without_room(train):
    g = torch.Generator(device="cuda").manual_seed(2)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    q, k, v, keys, values = make(4, 2, 64), make(4, 1, 64), make(4, 1, 64), make(4, 40, 1, 64), make(4, 40, 1, 64)
    before = keys.clone()
    o = train.attention_step(q, k, v, keys, values, torch.tensor([39, 40, 2 ** 31 - 1, -2 ** 31], device="cuda", dtype=torch.int32))
    assert o[0].isfinite().all() and o[1:3].isnan().all() and not o[3].any()
    before[0, 39] = k[0]
    assert torch.equal(keys, before)
    with pytest.raises(ValueError):
        train.attention_step(q, k, v, keys[..., :63], values, torch.zeros(4, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        train.attention_step(q, k, v, keys, values.permute(3, 0, 1, 2).contiguous().permute(1, 2, 3, 0), torch.zeros(4, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):                                  # one cache for all sequences: two would write one place
        train.attention_step(q, k, v, keys[:1].expand(4, 40, 1, 64), values, torch.zeros(4, device="cuda", dtype=torch.int32))
    empty = torch.empty(4, 0, 1, 64, device="cuda", dtype=torch.bfloat16)
    assert train.attention_step(q, k, v, empty, empty, torch.zeros(4, device="cuda", dtype=torch.int32)).isnan().all()
    none = torch.empty(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    assert train.attention_step(none, none[:, :1], none[:, :1], empty[:0], empty[:0], torch.zeros(0, device="cuda", dtype=torch.int32)).shape == (0, 2, 64)


@gpu
def test_steps_continue_like_the_whole_sequence(train):
    """Token after token, from nothing, in a graph that is replayed; the cache's heads lie first."""
    n, heads, kv, dim, b = 150, 4, 2, 64, 3
    q, k, v, _ = inputs(21, b * n, heads, kv, dim, FP16)
    whole, _, _ = train.attention_forward(q, k, v, torch.arange(0, b * n + 1, n, device="cuda", dtype=torch.int32))
    keys, values = (torch.zeros(b, kv, n, dim, device="cuda", dtype=FP16).transpose(1, 2) for _ in range(2))
    lengths = torch.zeros(b, device="cuda", dtype=torch.int32)
    now = [torch.empty(b, h, dim, device="cuda", dtype=FP16) for h in (heads, kv, kv)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = train.attention_step(*now, keys, values, lengths)
        lengths += 1
    for t in range(n):
        for to, of in zip(now, (q, k, v)):
            to.copy_(of.view(b, n, *of.shape[1:])[:, t])
        graph.replay()
        # either is off by its roundings: of exponentials and of itself
        assert (out.float() - whole.view(b, n, heads, dim)[:, t].float()).abs().max() < 6 * 2.0 ** -11 * v.abs().max(), t
    assert lengths.tolist() == [n] * b and torch.equal(keys.reshape(-1), k.view(b, n, kv, dim).reshape(-1))


@gpu
def test_a_cache_beyond_32_bits_of_offsets(train):
    keys, values = (torch.zeros(2, 2100, 8, 1 << 17, device="cuda", dtype=BF16)[..., :64] for _ in range(2))      # 2^31.04 elements a sequence
    g = torch.Generator(device="cuda").manual_seed(3)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    near_k, near_v = make(2, 2100, 8, 64), make(2, 2100, 8, 64)
    keys.copy_(near_k)
    values.copy_(near_v)
    q, k, v = make(2, 8, 64), make(2, 8, 64), make(2, 8, 64)
    lengths = torch.tensor([2099, 2090], device="cuda", dtype=torch.int32)
    want = train.attention_step(q, k, v, near_k, near_v, lengths)
    got = train.attention_step(q, k, v, keys, values, lengths)
    assert torch.equal(got, want) and torch.equal(keys, near_k) and torch.equal(values, near_v)


SHIM = r"""
#include "train_plan.h"
using namespace ones::train;
extern "C" {
void attention(int64_t tokens, int64_t sequences, int64_t heads, int64_t kv, int64_t dim, int64_t *to) {
  const AttentionPlan p = attention_plan(tokens, sequences, heads, kv, dim);
  to[0] = attention_few(tokens, heads); to[1] = p.parts; to[2] = static_cast<int64_t>(p.bytes);
}
void step(int64_t batch, int64_t capacity, int64_t heads, int64_t kv, int64_t dim, int64_t *to) {
  const StepPlan p = step_plan(batch, capacity, heads, kv, dim);
  to[0] = p.splits; to[1] = p.blocks_of_heads; to[2] = static_cast<int64_t>(p.bytes);
}
void rotation(int64_t tokens, int64_t heads, int64_t kv, int64_t dim, int64_t pairs, int64_t bytes, int64_t backward, int64_t *to) {
  const RotationPlan p = rotation_plan(tokens, heads, kv, dim, pairs, bytes, backward != 0);
  to[0] = p.vec; to[1] = p.lanes; to[2] = p.per; to[3] = p.parts; to[4] = p.blocks;
}
void apart(int64_t batch, int64_t batch_stride, int64_t stride, int64_t head_stride, int64_t capacity, int64_t kv, int64_t dim, int64_t *to) {
  to[0] = Places(batch, batch_stride, stride, head_stride, capacity, kv, dim).apart();
}
void meets(int64_t batch, int64_t batch_stride, int64_t stride, int64_t head_stride, int64_t capacity, int64_t kv, int64_t dim, int64_t delta, int64_t *to) {
  to[0] = Places(batch, batch_stride, stride, head_stride, capacity, kv, dim).meets(delta);
}
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    import os
    import shutil
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("no g++")
    at = tmp_path_factory.mktemp("plans")
    (at / "shim.cpp").write_text(SHIM)
    subprocess.check_call([compiler, "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{root}/include", f"-I{root}/paper_2108_03645_amd/csrc", str(at / "shim.cpp"),
                           "-o", str(at / "shim.so")])
    lib = C.CDLL(str(at / "shim.so"))

    def ask(name, *sizes):
        to = (C.c_int64 * 8)()
        getattr(lib, name)(*[C.c_int64(v) for v in sizes], to)
        return list(to)

    return ask


def test_caches_whose_places_are_shared_are_refused(train, plans):
    """By the C entry too: two places of a cache, or of the two caches, in one would be written and read in the same launch."""
    L, p = train.load(), C.c_void_p(0x1000)

    def step(b=2, cap=9, kv=2, keys=(9 * 128, 128, 64), values=(9 * 128, 128, 64), at=0x1000, to=0x100000):
        return L.ones_attention_step(p, 256, 64, p, 128, 64, p, 128, 64, C.c_void_p(at), *keys, C.c_void_p(to), *values, p, b, cap, 2 * kv, kv, 64, 1, 0.1, p, None, 0, None)

    shared = [(9 * 128, 64, 64), (128, 128, 64), (64, 64, 9 * 64), (8 * 128, 128, 64), (9 * 128, 128, 128), (64 * 9, 128, 64), (9 * 128, 120, 64), (9 * 128, 128, 72), (72, 144, 8 * 144 + 64)]
    for layout in shared:
        assert step(keys=layout) == step(values=layout) == -1, layout
        assert not plans("apart", 2, *layout, 9, 2, 64)[0], layout
    for layout in [(9 * 128, 128, 64), (9 * 128, 64, 9 * 64), (128, 256, 64), (64, 256, 128), (64, 128, 9 * 128), (1 << 20, 1 << 10, 1 << 15)]:
        assert plans("apart", 2, *layout, 9, 2, 64)[0], layout
    assert plans("apart", 1, 0, 64, 0, 9, 1, 64)[0] and plans("apart", 1, 0, 64, 64, 1, 2, 64)[0] and plans("apart", 5, 64, 0, 64, 1, 1, 64)[0]
    # the largest that is taken does not wrap
    assert plans("apart", 65535, 1 << 30, 1 << 20, 1 << 40, 1 << 30, 1024, 128)[0] == 0


def test_keys_and_values_that_share_places_are_refused(train, plans):
    """One tensor for both, or values that begin inside the keys; places that lie between each other are two."""
    L, p = train.load(), C.c_void_p(0x1000)

    def step(keys, values, at, to, b=2, cap=9, kv=2):
        return L.ones_attention_step(p, 256, 64, p, 128, 64, p, 128, 64, C.c_void_p(at), *keys, C.c_void_p(to), *values, p, b, cap, 2 * kv, kv, 64, 1, 0.1, p, None, 0, None)

    dense, at = (9 * 128, 128, 64), 1 << 20
    for behind in (0, 8, 64, -64, 128, 9 * 128, -9 * 128, 17 * 128, -(17 * 128 + 64)):
        assert step(dense, dense, at, at + 2 * behind) == -1, behind
    between = (2 * 9 * 128, 128, 64)
    assert step(between, between, at, at + 2 * 128) == step(between, dense, at, at) == -1
    import itertools
    import random
    rng = random.Random(1)
    for _ in range(300):                                             # against the elements themselves
        sizes, dim = [rng.randint(1, 3) for _ in range(3)], rng.choice([8, 16])
        order, strides, reach = rng.sample(range(3), 3), [0] * 3, dim
        for axis in order:
            strides[axis] = reach + 8 * rng.choice([0, 0, 1, 2, 5])
            reach += strides[axis] * (sizes[axis] - 1)
        places = {sum(i * s for i, s in zip(at, strides)) + d for at in itertools.product(*map(range, sizes)) for d in range(dim)}
        layout = (sizes[0], *strides, *sizes[1:], dim)
        assert plans("apart", *layout)[0] == 1
        for delta in [8 * rng.randint(-reach // 8 - 1, reach // 8 + 1) for _ in range(30)]:
            assert plans("meets", *layout, delta)[0] == any(x + delta in places for x in places), (layout, delta)


def test_the_sizes_above_reach_every_kernel_and_cut(plans):
    """Workgroups of 64 and of 128 queries, one part of a group's heads and more, keys in one part and in more, loads of 16, 8 and less bytes."""
    few = {(plans("attention", sum(s[0]), len(s[0]), *s[1:4])[0], (s[3] + 31) // 32) for s in SHAPES + LARGE}
    assert few == {(a, b) for a in (0, 1) for b in (1, 2, 3, 4)}
    parts = {(plans("attention", sum(s[0]), len(s[0]), *s[1:4])[1] > 1) for s in LARGE}
    assert parts == {False, True}
    assert {plans("step", len(s[0]), *s[1:])[0] > 1 for s in STEPS} == {False, True} == {plans("step", len(s[0]), *s[1:])[1] > 1 for s in STEPS}
    from test_train_rotation import CASES
    lanes = {(plans("rotation", *c[:5], b, back)[0] * b, back) for c in CASES for b in (2, 4) for back in (0, 1)}
    assert lanes >= {(16, 0), (8, 0), (16, 1), (8, 1)} and any(plans("rotation", *c[:5], 2, 0)[0] == 1 for c in CASES)
    assert {plans("rotation", *c[:5], 2, 1)[3] > 1 for c in CASES} == {False, True}


def test_parts_and_splits_stay_within_bounds(plans):
    import random
    rng = random.Random(4)
    for _ in range(3000):
        kv, group, tokens = rng.randint(1, 64), rng.choice([1, 2, 3, 7, 16]), int(2 ** rng.uniform(0, 24))
        _, parts, *_ = plans("attention", tokens, rng.randint(0, 100), kv * group, kv, 64)
        assert 1 <= parts <= group and -(-group // -(-group // parts)) == parts          # no part without a head
        splits, blocks, *_ = plans("step", rng.randint(1, 3000), int(2 ** rng.uniform(0, 26)), kv * group, kv, 64)
        assert 1 <= splits <= 512 and (blocks - 1) * 16 < group <= blocks * 16
        dim = rng.randint(1, 512)
        vec, lanes, per, _, n, *_ = plans("rotation", tokens, kv * group, kv, dim, rng.randint(0, dim // 2), rng.choice([2, 4]), rng.randint(0, 1))
        assert vec * lanes * per >= (dim + 1) // 2 and lanes in (4, 8, 16, 32, 64) and 1 <= n <= 2048 and (vec > 1 or (lanes == 16 and per <= 16))
