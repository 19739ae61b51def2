"""The operators of a scheduled language-model job's training step, as cases that can be timed and compared.

The search decides at which batch a job trains; these are the parts of that job's step.  Layer norm, the gated linear
recurrence and the loss over the vocabulary work per sample (the slope of the job's iteration time over its batch), the
orthogonalised update works per step (its offset).  A pass is one call, forward and backward where the operator has both.
"""
import math

import torch

own = False

COEFFICIENTS = (3.4445, -4.7750, 2.0315)          # of the Newton-Schulz products
EPS_NORM, EPS_UPDATE, BETA = 1e-5, 1e-7, 0.95
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MOST = {"norm": 32768 * 2048, "recurrence": 131072 * 512, "loss": 8192 * 32000 * 1024, "update": 4096 ** 3}


def _norm(name, rows, cols, dtype, weights="fp32"):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "weights": weights}


def _recurrence(name, batch, steps, channels, dtype, ragged=False, state=False):
    return {"name": name, "op": "recurrence", "batch": batch, "steps": steps, "channels": channels, "dtype": dtype,
            "ragged": ragged, "state": state}


def _loss(name, rows, cols, vocabulary, dtype, backward=True, ignored=0.0):
    return {"name": name, "op": "loss", "rows": rows, "cols": cols, "vocabulary": vocabulary, "dtype": dtype,
            "backward": backward, "ignored": ignored}


def _update(name, count, rows, cols, dtype, nesterov=True):
    return {"name": name, "op": "update", "count": count, "rows": rows, "cols": cols, "dtype": dtype, "nesterov": nesterov}


def listed():
    return [
        # one GPU's share of a small job: 64 tokens of a narrow model, forward and backward; latency counts
        _norm("norm_small", 64, 256, "bf16"),
        # columns that fit no vector width, in 16 bits with 16-bit weights
        _norm("norm_odd", 5003, 1001, "fp16", weights="fp16"),
        # the largest: 32768 tokens (a local batch of 16 sequences of 2048) of 2048 channels
        _norm("norm_large", 32768, 2048, "bf16"),
        # one new token for each of 64 sequences that a job's model is answering
        _recurrence("recurrence_token", 64, 1, 1024, "bf16", state=True),
        # an ordinary training step's mixer: 16 sequences of 2048 steps
        _recurrence("recurrence_train", 16, 2048, 1024, "bf16"),
        # few and long sequences of different lengths: the work has to be split over the time
        _recurrence("recurrence_long", 2, 65521, 512, "fp16", ragged=True, state=True),
        # the smallest loss: a local batch of 64 tokens, a small vocabulary
        _loss("loss_small", 64, 256, 1000, "bf16"),
        # odd sizes, a fifth of the targets padding
        _loss("loss_odd", 1003, 514, 10007, "fp16", ignored=0.2),
        # evaluation: the loss alone, more rows
        _loss("loss_forward", 16384, 512, 32000, "bf16", backward=False),
        # the largest: 8192 tokens, 32000 words, with both gradients
        _loss("loss_large", 8192, 1024, 32000, "bf16", ignored=0.05),
        # the updates of eight small square matrices of a model in one call
        _update("update_small", 8, 256, 256, "bf16"),
        # one large matrix, tall, odd sides
        _update("update_large", 1, 4100, 3000, "bf16"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def side(lo, hi):                             # mostly multiples of 64, some of 8, some odd
        n = spread(lo, hi)
        step = rng.choice([64, 64, 8, 1])
        return max(lo, n // step * step)

    op = rng.choice(["norm", "recurrence", "loss", "update"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "norm":
        cols = side(64, 8192)
        rows = min(spread(1, 65536), MOST[op] // cols)
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        case = _norm(None, rows, cols, dtype, weights=rng.choice(["fp32", dtype]))
    elif op == "recurrence":
        channels, batch = side(64, 4096), spread(1, 128)
        steps = min(rng.choice([1, spread(2, 131072), spread(128, 8192)]), max(1, MOST[op] // (channels * batch)))
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        case = _recurrence(None, batch, steps, channels, dtype, ragged=steps > 1 and rng.random() < 0.4,
                           state=steps == 1 or rng.random() < 0.5)
    elif op == "loss":
        cols, vocabulary = side(64, 4096), side(100, 131072)
        rows = min(spread(1, 16384), MOST[op] // (cols * vocabulary) or 1)
        case = _loss(None, rows, cols, vocabulary, dtype, backward=rng.random() < 0.75, ignored=rng.choice([0.0, 0.0, 0.3]))
    else:
        rows, cols = side(32, 4096), side(32, 8192)
        small, large = min(rows, cols), max(rows, cols)
        if small * small * large > MOST[op]:
            cols = rows = min(small, 4096)
            small = large = rows
        count = max(1, min(rng.choice([1, 1, 4, 16]), MOST[op] // (small * small * large)))
        case = _update(None, count, rows, cols, dtype, nesterov=rng.random() < 0.7)
    del case["name"]
    return case


# ------------------------------------------------------------------- inputs --------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def prepare(case, seed):
    g, dtype = _generator(seed), _TYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, to=dtype):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).add_(mean).to(to)

    state = {"case": dict(case)}
    if case["op"] == "norm":
        n, d, weights = case["rows"], case["cols"], _TYPES[case["weights"]]
        state.update(x=normal(n, d, std=1.5, mean=0.3), dy=normal(n, d, std=0.1),
                     weight=normal(d, std=0.2, mean=1.0, to=weights), bias=normal(d, std=0.2, to=weights))
    elif case["op"] == "recurrence":
        b, t, c = case["batch"], case["steps"], case["channels"]
        state.update(gate=normal(b, t, c, std=1.5, mean=2.0), x=normal(b, t, c), lengths=None, state=None)
        if case["ragged"]:
            state["lengths"] = torch.randint(0, t + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
            state["lengths"][0] = t
        if case["state"]:
            state["state"] = normal(b, c, to=torch.float32)
        if t > 1:
            state.update(dh=normal(b, t, c, std=0.1), dlast=normal(b, c, std=0.1, to=torch.float32))
    elif case["op"] == "loss":
        n, d, v = case["rows"], case["cols"], case["vocabulary"]
        target = torch.randint(0, v, (n,), generator=g, device="cuda")
        if case["ignored"]:
            target[torch.rand(n, generator=g, device="cuda") < case["ignored"]] = -100
        valid = (target >= 0).sum().clamp(min=1)
        state.update(x=normal(n, d), weight=normal(v, d, std=1.5 / math.sqrt(d)), target=target,
                     dloss=torch.full((n,), 1.0, device="cuda") / valid)
    else:
        k, m, n = case["count"], case["rows"], case["cols"]
        # a gradient of a low-rank signal and noise, as gradients are, and the momentum of earlier ones
        rank = max(1, min(m, n) // 8)
        signal = torch.matmul(normal(k, m, rank, to=torch.float32), normal(k, rank, n, to=torch.float32))
        state.update(grad=((signal / math.sqrt(rank) + normal(k, m, n, to=torch.float32)) * 1e-3).to(dtype),
                     momentum=(signal / math.sqrt(rank) * 8 + normal(k, m, n, std=3.0, to=torch.float32)) * 1e-3)
    return state


# -------------------------------------------------------------- plain forms --------
def _plain_norm(s):
    x, dy, w, b = s["x"].float(), s["dy"].float(), s["weight"].float(), s["bias"].float()
    mean = x.mean(1)
    centred = x - mean[:, None]
    rstd = torch.rsqrt(centred.square().mean(1) + EPS_NORM)
    xh = centred * rstd[:, None]
    y = xh * w + b
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    to = s["weight"].dtype
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd, "dx": dx.to(s["x"].dtype),
            "dweight": (dy * xh).sum(0).to(to), "dbias": dy.sum(0).to(to)}


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t along dimension 1 from zero, by doubling."""
    shift = 1
    while shift < u.shape[1]:
        u = torch.cat([u[:, :shift], u[:, shift:] + a[:, shift:] * u[:, :-shift]], 1)
        a = torch.cat([a[:, :shift], a[:, shift:] * a[:, :-shift]], 1)
        shift *= 2
    return a, u


def _plain_recurrence(s):
    gate, x, dtype = s["gate"].float(), s["x"].float(), s["x"].dtype
    b, t, c = x.shape
    h0 = s["state"] if s["state"] is not None else torch.zeros(b, c, device=x.device)
    a, keep = torch.sigmoid(gate), torch.sigmoid(-gate)
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(t, device=x.device)[None, :] < s["lengths"][:, None])[..., None]
        a, keep = torch.where(live, a, torch.ones_like(a)), torch.where(live, keep, torch.zeros_like(keep))
    through, h = _scan(a, keep * x)
    h = h + through * h0[:, None]
    last = h[:, -1].clone()
    out = h if live is None else torch.where(live, h, torch.zeros_like(h))
    if t == 1:
        s["state"].copy_(last)
        return {"h": out.to(dtype), "state": s["state"]}
    dh = s["dh"].float() if live is None else torch.where(live, s["dh"].float(), torch.zeros_like(h))
    before = torch.cat([h0[:, None], h[:, :-1]], 1)
    back = dh.flip(1).clone()
    back[:, 0] += s["dlast"]
    gates = a.flip(1)
    _, lam = _scan(torch.cat([torch.zeros_like(gates[:, :1]), gates[:, :-1]], 1), back)
    lam = lam.flip(1)
    dx = keep * lam
    dgate = lam * (before - x) * a * keep
    return {"h": out.to(dtype), "last": last, "dgate": dgate.to(dtype), "dx": dx.to(dtype), "dstate": a[:, 0] * lam[:, 0]}


def _plain_loss(s):
    x, w, target = s["x"].float(), s["weight"].float(), s["target"]
    z = x @ w.t()
    top = z.max(1).values
    p = torch.exp(z - top[:, None])
    total = p.sum(1)
    lse = top + torch.log(total)
    valid = target >= 0
    at = target.clamp(min=0)[:, None]
    loss = torch.where(valid, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    if not s["case"]["backward"]:
        return {"loss": loss, "lse": lse}
    scale = torch.where(valid, s["dloss"], torch.zeros_like(lse))
    p *= (scale / total)[:, None]
    p.scatter_add_(1, at, -scale[:, None])
    return {"loss": loss, "lse": lse, "dx": (p @ w).to(s["x"].dtype), "dweight": (p.t() @ x).to(s["x"].dtype)}


def _plain_update(s):
    g = s["grad"].float()
    m = BETA * s["momentum"] + g
    u = g + BETA * m if s["case"]["nesterov"] else m
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS_UPDATE)
    a, b, c = COEFFICIENTS
    for _ in range(5):
        q = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * q + c * torch.matmul(q, q), x)
    x = x.transpose(1, 2) if tall else x
    s["momentum"].copy_(m)
    return {"update": x.contiguous().to(s["grad"].dtype), "momentum": s["momentum"]}


# -------------------------------------------------------- framework's calls --------
def _own(s):
    from paper_2108_03645_amd import train

    case = s["case"]
    if case["op"] == "norm":
        y, mean, rstd = train.layer_norm_forward(s["x"], s["weight"], s["bias"], EPS_NORM)
        dx, dweight, dbias = train.layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd)
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dweight": dweight, "dbias": dbias}
    if case["op"] == "recurrence":
        if case["steps"] == 1:
            h = train.gated_recurrence_step(s["gate"], s["x"], s["state"])
            return {"h": h, "state": s["state"]}
        h, last, carry = train.gated_recurrence_forward(s["gate"], s["x"], s["state"], s["lengths"])
        dgate, dx, dstate = train.gated_recurrence_backward(s["dh"], s["dlast"], s["gate"], s["x"], carry, s["lengths"])
        return {"h": h, "last": last, "dgate": dgate, "dx": dx, "dstate": dstate}
    if case["op"] == "loss":
        loss, lse = train.linear_cross_entropy_forward(s["x"], s["weight"], s["target"])
        if not case["backward"]:
            return {"loss": loss, "lse": lse}
        dx, dweight = train.linear_cross_entropy_backward(s["dloss"], s["x"], s["weight"], s["target"], lse)
        return {"loss": loss, "lse": lse, "dx": dx, "dweight": dweight}
    update = train.orthogonal_update(s["grad"], s["momentum"], BETA, case["nesterov"], 5, COEFFICIENTS, EPS_UPDATE)
    return {"update": update, "momentum": s["momentum"]}


def run(state):
    # the momentum, and the state of a token's step, advance with every pass, as in a program's loop
    if own:
        return _own(state)
    return {"norm": _plain_norm, "recurrence": _plain_recurrence, "loss": _plain_loss,
            "update": _plain_update}[state["case"]["op"]](state)


# --------------------------------------------------------------------- work --------
def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "norm":
        n, d = case["rows"], case["cols"]
        f = 4 if case["weights"] == "fp32" else 2
        # x, y, dy, dx; mean and rstd; weight, bias and their gradients
        return {"bytes": 4 * n * d * e + 8 * n + 4 * d * f, "flops": 22 * n * d}
    if case["op"] == "recurrence":
        b, t, c = case["batch"], case["steps"], case["channels"]
        if t == 1:
            return {"bytes": 3 * b * c * e + 8 * b * c, "flops": 10 * b * c}
        # gate, x, dh; h, dgate, dx; states
        return {"bytes": 6 * b * t * c * e + 4 * b * c * (3 + case["state"]), "flops": 30 * b * t * c}
    if case["op"] == "loss":
        n, d, v = case["rows"], case["cols"], case["vocabulary"]
        both = 2 if case["backward"] else 1
        # the products forward; backward the two of the gradients, and the logits' again since they are not kept
        return {"bytes": both * (n + v) * d * e + 16 * n, "flops": (8 if case["backward"] else 2) * n * v * d}
    k, small, large = case["count"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    return {"bytes": k * small * large * (2 * e + 8), "flops": 5 * k * (3 * small * small * large + small ** 3)}


# ----------------------------------------------------- the definition, 64 bits -----
def _exact_norm(s):
    x, dy = s["x"].double(), s["dy"].double()
    w, b, d = s["weight"].double(), s["bias"].double(), x.shape[1]
    mean = x.sum(1) / d
    var = ((x - mean[:, None]) ** 2).sum(1) / d
    rstd = (var + EPS_NORM) ** -0.5
    xh = torch.einsum("nd,n->nd", x - mean[:, None], rstd)
    g = dy * w
    along = (g * xh).sum(1) / d
    dx = (g - (g.sum(1) / d)[:, None] - along[:, None] * xh) * rstd[:, None]
    return {"y": xh * w + b, "mean": mean, "rstd": rstd, "dx": dx, "dweight": torch.einsum("nd,nd->d", dy, xh),
            "dbias": torch.einsum("nd->d", dy)}


def _exact_recurrence(s):
    """One step after another."""
    b, t, c = s["x"].shape
    h = s["state"].double().clone() if s["state"] is not None else torch.zeros(b, c, device="cuda", dtype=torch.float64)
    lengths = s["lengths"].long() if s["lengths"] is not None else torch.full((b,), t, device="cuda")
    a = 1.0 / (1.0 + torch.exp(-s["gate"].double().transpose(0, 1)))          # [t, b, c], a step's entries together
    u = s["x"].double().transpose(0, 1) / (1.0 + torch.exp(s["gate"].double().transpose(0, 1)))
    past = (torch.arange(t, device="cuda")[:, None] >= lengths[None, :])[..., None].expand(t, b, c)
    a, u = a.masked_fill(past, 1.0), u.masked_fill(past, 0.0)
    hs = torch.empty(t + 1, b, c, device="cuda", dtype=torch.float64)
    hs[0] = h
    for i in range(t):
        torch.addcmul(u[i], a[i], hs[i], out=hs[i + 1])
    last = hs[t].clone()
    h = hs[1:].masked_fill(past, 0.0).transpose(0, 1)
    if t == 1:
        return {"h": h, "state": last}
    lam = s["dh"].double().transpose(0, 1).masked_fill(past, 0.0).contiguous()
    lam[t - 1] += s["dlast"].double()
    for i in range(t - 2, -1, -1):
        lam[i].addcmul_(a[i + 1], lam[i + 1])
    dstate = a[0] * lam[0]
    x, keep = s["x"].double().transpose(0, 1), (1.0 / (1.0 + torch.exp(s["gate"].double().transpose(0, 1)))).masked_fill(past, 0.0)
    dx = (lam * keep).transpose(0, 1)
    dgate = (lam * keep * a * (hs[:-1] - x)).transpose(0, 1)
    return {"h": h, "last": last, "dgate": dgate, "dx": dx, "dstate": dstate}


def _exact_loss(s):
    x, w, target = s["x"].double(), s["weight"].double(), s["target"]
    n = x.shape[0]
    loss, lse, dx = [], [], []
    dweight = torch.zeros_like(w)
    for lo in range(0, n, 2048):                  # some rows at a time
        xs, ts, ds = x[lo:lo + 2048], target[lo:lo + 2048], s["dloss"][lo:lo + 2048].double()
        z = torch.mm(xs, w.t())
        one = torch.logsumexp(z, 1)
        skip = ts < 0
        index = torch.arange(len(ts), device="cuda")
        loss.append((one - z[index, ts.masked_fill(skip, 0)]).masked_fill(skip, 0.0))
        lse.append(one)
        if s["case"]["backward"]:
            grad = torch.exp(z - one[:, None])
            grad[index, ts.masked_fill(skip, 0)] -= 1.0
            grad *= ds.masked_fill(skip, 0.0)[:, None]
            dx.append(torch.mm(grad, w))
            dweight.addmm_(grad.t(), xs)
    found = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    return {**found, "dx": torch.cat(dx), "dweight": dweight} if s["case"]["backward"] else found


def _exact_update(s):
    """The products of the wide matrix, with a I + b Q + c Q^2 formed first."""
    g, m = s["grad"].double(), s["momentum"].double()
    m = m * BETA + g
    u = m * BETA + g if s["case"]["nesterov"] else m
    a, b, c = COEFFICIENTS
    out = []
    for one in u:
        wide = one if one.shape[0] <= one.shape[1] else one.t().contiguous()
        wide = wide / (torch.linalg.vector_norm(wide) + EPS_UPDATE)
        for _ in range(5):
            gram = torch.mm(wide, wide.t())
            poly = torch.addmm(gram, gram, gram, beta=b, alpha=c)
            poly.diagonal().add_(a)
            wide = torch.mm(poly, wide)
        out.append(wide if one.shape[0] <= one.shape[1] else wide.t())
    return {"update": torch.stack(out), "momentum": m}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "recurrence": _exact_recurrence, "loss": _exact_loss, "update": _exact_update}[case["op"]](s)
