"""The operators of a scheduled job whose model attends, as cases that can be timed and compared.

Queries and keys are normed for each head and turned by their positions, a whole batch of packed sequences attends causally (forward, and
backward where the job trains), a sequence is continued token by token over its cache, and the gradients of a step are clipped by
their global norm.  A pass is one operator, forward and backward where the case has both.
"""
import math
import random

import torch

own = False

EPS_NORM, EPS_CLIP, BASE = 1e-6, 1e-6, 10000.0
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# of a drawn case, as the largest listed one: elements of queries and keys, of a cache, of gradients; attention's operations and bytes
MOST = {"rotation": 32768 * 18 * 128, "attention": (962542436352, 606076928), "step": 32 * 8192 * 4 * 128, "clip": 1 << 27}


def _rotation(name, tokens, heads, kv_heads, dim, dtype, backward=True, rotary=None, interleaved=False, weights="fp32", far=False):
    return {"name": name, "op": "rotation", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "backward": backward, "rotary": rotary or dim // 2 * 2, "interleaved": interleaved, "weights": weights, "far": far}


def _attention(name, tokens, sequences, heads, kv_heads, dim, dtype, backward=True, ragged=False, behind=0):
    return {"name": name, "op": "attention", "tokens": tokens, "sequences": sequences, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "backward": backward, "ragged": ragged, "behind": behind}


def _step(name, batch, longest, heads, kv_heads, dim, dtype, ragged=True):
    return {"name": name, "op": "step", "batch": batch, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "ragged": ragged}


def _clip(name, tensors, elements, dtype, clips=True):
    return {"name": name, "op": "clip", "tensors": tensors, "elements": elements, "dtype": dtype, "clips": clips}


def listed():
    return [
        # one new token for each of 64 sequences that a job's model is answering; latency counts
        _rotation("rotation_token", 64, 16, 2, 64, "bf16", backward=False, far=True),
        # rows that fill no power of two, half of each turned, neighbours in pairs, 16-bit weights
        _rotation("rotation_odd", 5003, 12, 4, 80, "fp16", rotary=40, interleaved=True, weights="fp16"),
        # the largest: 32768 tokens (a local batch of 16 sequences of 2048) of 16 heads over 2
        _rotation("rotation_large", 32768, 16, 2, 128, "bf16"),
        # a small job's step: four sequences of 64 tokens, a narrow model; latency counts
        _attention("attention_small", 256, 4, 4, 4, 64, "bf16"),
        # packed sequences of very different lengths, one and none among them, rows of padding behind the last
        _attention("attention_ragged", 6007, 19, 12, 4, 80, "fp16", ragged=True, behind=57),
        # a long prompt, forward only
        _attention("attention_prompt", 16384, 1, 16, 2, 128, "bf16", backward=False),
        # the largest: an ordinary training step's mixer, 16 sequences of 2048 tokens
        _attention("attention_large", 32768, 16, 16, 2, 128, "bf16"),
        # eight short sequences continued: latency counts
        _step("step_small", 8, 200, 8, 8, 64, "bf16"),
        # one long sequence: its cache has to be split over the card
        _step("step_long", 1, 100003, 16, 2, 128, "fp16", ragged=False),
        # a batch of sequences, half a gigabyte of cache
        _step("step_large", 32, 8192, 32, 4, 128, "bf16", ragged=False),
        # the gradients of a small model, below the limit, as in most steps
        _clip("clip_small", 12, 1100003, "mixed", clips=False),
        # the gradients of a larger one, clipped
        _clip("clip_large", 148, 1 << 27, "bf16"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotation", "attention", "attention", "step", "clip"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    dim = rng.choice([64, 64, 128, 128, 8 * rng.randint(1, 16)])
    if op == "rotation":
        dim = rng.choice([64, 128, 256, 8 * rng.randint(1, 32), rng.randint(2, 256)])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        tokens = max(1, min(spread(1, 65536), MOST[op] // ((heads + kv_heads) * dim * (2 if dtype == "fp32" else 1))))
        case = _rotation(None, tokens, heads, kv_heads, dim, dtype, rng.random() < 0.75, max(2, dim // rng.choice([2, 2, 2, 4]) // 2 * 2)
                         if rng.random() < 0.3 else None, rng.random() < 0.4, rng.choice(["fp32", dtype]), rng.random() < 0.3)
    elif op == "attention":
        sequences, longest = spread(1, 64), spread(1, 16384)
        case = _attention(None, min(32768, sequences * longest), sequences, heads, kv_heads, dim, dtype, rng.random() < 0.7, rng.random() < 0.6,
                          rng.choice([0, 0, rng.randint(1, 63)]))
        if case["tokens"] > 64:
            case["tokens"] -= rng.randint(0, 7)
        while any(work(case)[k] > most for k, most in zip(("flops", "bytes"), MOST[op])):
            case["tokens"] //= 2
        if max(_lengths(case)) < 2:
            case["backward"] = False              # a row with one key has no gradient but rounding
    elif op == "step":
        batch = spread(1, 256)
        longest = max(1, min(spread(1, 131072), MOST[op] // (batch * kv_heads * dim)))
        case = _step(None, batch, longest, heads, kv_heads, dim, dtype, rng.random() < 0.7)
    else:
        tensors = spread(1, 400)
        case = _clip(None, tensors, max(tensors, spread(1000, MOST[op])), rng.choice(["bf16", "fp16", "fp32", "mixed"]), rng.random() < 0.5)
        if case["dtype"] in ("fp32", "mixed"):
            case["elements"] = max(tensors, case["elements"] // 2)
    del case["name"]
    return case


def _lengths(case):
    """The lengths of the sequences, by the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    if case["op"] == "step":
        n = case["longest"]
        return [n if i == 0 or not case["ragged"] else int(n * rng.random() ** 2) for i in range(case["batch"])]
    rest, count = case["tokens"] - min(case["behind"], case["tokens"] - 1), case["sequences"]
    if not case["ragged"]:
        return [rest * (i + 1) // count - rest * i // count for i in range(count)]
    weights = [0.0 if i % 7 == 3 and count > 4 else rng.random() ** 3 for i in range(count)]
    total = sum(weights) or 1.0
    lengths = [int(rest * w / total) for w in weights]
    lengths[lengths.index(max(lengths))] += rest - sum(lengths)
    return lengths


def _sizes(case):
    """The sizes of a step's gradients: matrices, vectors, and an odd one or two, by the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    weights = [rng.choice([1.0, 1.0, 1.0, 4.0, 0.001]) for _ in range(case["tensors"])]
    total = sum(weights)
    return [max(1, int(case["elements"] * w / total)) for w in weights]


# ------------------------------------------------------------------- inputs --------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def prepare(case, seed):
    g, dtype = _generator(seed), _TYPES.get(case["dtype"])

    def normal(*shape, std=1.0, mean=0.0, to=dtype):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).add_(mean).to(to)

    state = {"case": dict(case)}
    if case["op"] == "clip":
        kinds = [dtype or (torch.bfloat16, torch.float32)[i % 2] for i in range(case["tensors"])]
        # the gradients of a type as views of one buffer, each from a multiple of 64 elements on, zeros between them
        buffers, gradients = {}, []
        for kind in dict.fromkeys(kinds):
            buffers[kind] = torch.zeros(sum((n + 63) // 64 * 64 for n, of in zip(_sizes(case), kinds) if of == kind), device="cuda", dtype=kind)
        begin = dict.fromkeys(buffers, 0)
        for i, (n, kind) in enumerate(zip(_sizes(case), kinds)):
            gradients.append(buffers[kind][begin[kind]:begin[kind] + n])
            gradients[-1].copy_(normal(n, std=1e-3 * (1 + i % 5), to=kind))
            begin[kind] += (n + 63) // 64 * 64
        norm = math.sqrt(sum(t.double().square().sum().item() for t in buffers.values()))
        state.update(gradients=gradients, buffers=list(buffers.values()), limit=norm * (0.4 if case["clips"] else 3.0))
        return state
    h, k, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotation":
        n = case["tokens"]
        # queries and keys as they lie in the rows of one projection, in front of the values
        rows = normal(n, (h + 2 * k) * d, std=1.5)
        state.update(q=rows[:, :h * d].view(n, h, d), k=rows[:, h * d:(h + k) * d].view(n, k, d),
                     qw=normal(d, std=0.2, mean=1.0, to=_TYPES[case["weights"]]), kw=normal(d, std=0.2, mean=1.0, to=_TYPES[case["weights"]]),
                     positions=torch.arange(n, device="cuda", dtype=torch.int32) % 2048,
                     frequencies=BASE ** (-torch.arange(0, case["rotary"], 2, device="cuda", dtype=torch.float64) / case["rotary"]).float())
        if case["far"]:
            state["positions"] = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda", dtype=torch.int32)
        if case["backward"]:
            state.update(dq=normal(n, h, d, std=0.1), dk=normal(n, k, d, std=0.1))
    elif case["op"] == "attention":
        n, lengths = case["tokens"], _lengths(case)
        ends = [0]
        for one in lengths:
            ends.append(ends[-1] + one)
        # queries and keys as the rotation leaves them; the values in the rows of the projection
        rows = normal(n, (h + 2 * k) * d)
        state.update(q=normal(n, h, d, std=1.4), k=normal(n, k, d, std=1.4), v=rows[:, (h + k) * d:].view(n, k, d), ends=ends,
                     offsets=torch.tensor(ends, device="cuda", dtype=torch.int32))
        if case["backward"]:
            state["do"] = normal(n, h, d, std=0.05)
    else:
        b, lengths = case["batch"], _lengths(case)
        room = case["longest"] + 1
        state.update(q=normal(b, h, d, std=1.4), k=normal(b, k, d, std=1.4), v=normal(b, k, d), host=lengths,
                     keys=torch.empty(b, room, k, d, device="cuda", dtype=dtype), values=torch.empty(b, room, k, d, device="cuda", dtype=dtype),
                     lengths=torch.tensor(lengths, device="cuda", dtype=torch.int32))
        for i in range(b):
            state["keys"][i], state["values"][i] = normal(room, k, d, std=1.4), normal(room, k, d)
    return state


# -------------------------------------------------------------- plain forms --------
def _turned(x, cos, sin, interleaved):
    """The first 2 * cos.shape[-1] elements of the last dimension turned in pairs."""
    r = 2 * cos.shape[-1]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    first, second = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([first, second], -1).flatten(-2) if interleaved else torch.cat([first, second], -1)
    return torch.cat([both, x[..., r:]], -1)


def _plain_rotation(s):
    angle = s["positions"].double()[:, None] * s["frequencies"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    style, found = s["case"]["interleaved"], {}
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "w"].float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS_NORM)
        xh = x * r
        found[name] = _turned(xh * w, cos, sin, style).to(s[name].dtype)
        if s["case"]["backward"]:
            g = _turned(s["d" + name].float(), cos, -sin, style)
            u = g * w
            found["d" + name] = (r * (u - xh * (u * xh).mean(-1, keepdim=True))).to(s[name].dtype)
            found["d" + name + "w"] = (g * xh).sum((0, 1)).to(s[name + "w"].dtype)
    return found


def _plain_attention(s):
    case, dtype = s["case"], s["q"].dtype
    n, h, d = s["q"].shape
    kv, back = case["kv_heads"], case["backward"]
    group, scale = h // kv, d ** -0.5
    o = torch.zeros(n, h, d, device="cuda", dtype=dtype)
    lse = torch.full((h, n), -math.inf, device="cuda")
    dq, dk, dv = (torch.zeros(n, heads, d, device="cuda", dtype=dtype) for heads in (h, kv, kv)) if back else (None,) * 3
    for lo, hi in zip(s["ends"], s["ends"][1:]):
        m = hi - lo
        if m == 0:
            continue
        q = s["q"][lo:hi].float().view(m, kv, group, d).permute(1, 2, 0, 3).contiguous()          # [kv, group, m, d]
        k, v = s["k"][lo:hi].float().transpose(0, 1).contiguous(), s["v"][lo:hi].float().transpose(0, 1).contiguous()
        kt, vt = k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()
        if back:
            do = s["do"][lo:hi].float().view(m, kv, group, d).permute(1, 2, 0, 3).contiguous()
            sum_k, sum_v = torch.zeros_like(k), torch.zeros_like(v)
        step = max(1, min(m, (1 << 29) // (h * m)))                       # rows at a time
        for at in range(0, m, step):
            c, end = min(step, m - at), min(m, at + step)
            qs = q[:, :, at:end].reshape(kv, group * c, d)
            z = torch.matmul(qs, kt[:, :, :end].contiguous()).view(kv, group, c, end) * scale
            z.masked_fill_(torch.arange(end, device="cuda")[None, :] > torch.arange(at, end, device="cuda")[:, None], -math.inf)
            top = z.max(-1, keepdim=True).values
            p = torch.exp(z - top)
            total = p.sum(-1, keepdim=True)
            p = (p / total).view(kv, group * c, end)
            out = torch.matmul(p, v[:, :end].contiguous())
            lse[:, lo + at:lo + end] = (top + torch.log(total)).view(h, c)
            o[lo + at:lo + end] = out.view(kv, group, c, d).permute(2, 0, 1, 3).reshape(c, h, d).to(dtype)
            if back:
                dos = do[:, :, at:end].reshape(kv, group * c, d)
                ds = p * (torch.matmul(dos, vt[:, :, :end].contiguous()) - (dos * out).sum(-1, keepdim=True)) * scale
                dq[lo + at:lo + end] = torch.matmul(ds, k[:, :end].contiguous()).view(kv, group, c, d).permute(2, 0, 1, 3).reshape(c, h, d).to(dtype)
                sum_k[:, :end] += torch.matmul(ds.transpose(1, 2).contiguous(), qs)
                sum_v[:, :end] += torch.matmul(p.transpose(1, 2).contiguous(), dos)
        if back:
            dk[lo:hi], dv[lo:hi] = sum_k.transpose(0, 1).to(dtype), sum_v.transpose(0, 1).to(dtype)
    return {"o": o, "lse": lse, **({"dq": dq, "dk": dk, "dv": dv} if back else {})}


def _plain_step(s):
    q, keys, values, lengths = s["q"], s["keys"], s["values"], s["lengths"].long()
    b, h, d = q.shape
    kv = keys.shape[2]
    rows = torch.arange(b, device="cuda")
    keys[rows, lengths], values[rows, lengths] = s["k"], s["v"]
    out = torch.empty_like(q)
    most = max(1, (1 << 28) // (keys.shape[1] * kv * d))                  # sequences at a time
    for lo in range(0, b, most):
        part = slice(lo, min(b, lo + most))
        n = max(s["host"][part]) + 1
        qs = q[part].float().view(-1, kv, h // kv, d)
        kt = keys[part, :n].float().permute(0, 2, 3, 1).contiguous()      # [b, kv, d, n]
        z = torch.matmul(qs, kt) * d ** -0.5
        z.masked_fill_((torch.arange(n, device="cuda")[None, :] > lengths[part, None])[:, None, None], -math.inf)
        p = torch.exp(z - z.max(-1, keepdim=True).values)
        p = p / p.sum(-1, keepdim=True)
        out[part] = torch.matmul(p, values[part, :n].float().permute(0, 2, 1, 3).contiguous()).reshape(-1, h, d).to(q.dtype)
    return {"o": out, "keys": keys, "values": values}


def _plain_clip(s):
    squares = [t.double().square().sum() for t in s["gradients"]]
    norm = torch.stack(squares).sum().sqrt()
    factor = torch.clamp(_limit(s) / (norm + EPS_CLIP), max=1.0)
    if s["case"]["clips"]:
        for t in s["gradients"]:
            t.copy_(t.float() * factor.float())
    return {"norm": norm.float(), "gradients": s["buffers"]}


def _limit(s):
    """The limit of this pass.  The gradients are those that the last pass left; where a step's would be new ones, and above the limit
    again, the limit falls by a little from pass to pass."""
    limit = s["limit"]
    if s["case"]["clips"]:
        s["limit"] = limit * 0.999
    return limit


# -------------------------------------------------------- framework's calls --------
def _own(s):
    from paper_2108_03645_amd import train

    case = s["case"]
    if case["op"] == "rotation":
        common = (s["qw"], s["kw"], s["positions"], s["frequencies"], EPS_NORM, case["interleaved"])
        q, k = train.head_norm_rotation_forward(s["q"], s["k"], *common)
        if not case["backward"]:
            return {"q": q, "k": k}
        dq, dk, dqw, dkw = train.head_norm_rotation_backward(s["dq"], s["dk"], s["q"], s["k"], *common)
        return {"q": q, "dq": dq, "dqw": dqw, "k": k, "dk": dk, "dkw": dkw}
    if case["op"] == "attention":
        o, lse, rest = train.attention_forward(s["q"], s["k"], s["v"], s["offsets"], keep_rest=case["backward"])
        if not case["backward"]:
            return {"o": o, "lse": lse}
        dq, dk, dv = train.attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, rest, s["offsets"])
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    if case["op"] == "step":
        o = train.attention_step(s["q"], s["k"], s["v"], s["keys"], s["values"], s["lengths"])
        return {"o": o, "keys": s["keys"], "values": s["values"]}
    norm = train.clip_gradients(s["gradients"], _limit(s), EPS_CLIP)
    return {"norm": norm, "gradients": s["buffers"]}


def run(state):
    # a step writes its token to the place behind the cache's last every time; clipped gradients stay clipped (see _limit)
    if own:
        return _own(state)
    return {"rotation": _plain_rotation, "attention": _plain_attention, "step": _plain_step, "clip": _plain_clip}[state["case"]["op"]](state)


# --------------------------------------------------------------------- work --------
def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "clip":
        sizes = _sizes(case)
        nbytes = sum(n * (e if case["dtype"] != "mixed" else (2, 4)[i % 2]) for i, n in enumerate(sizes))
        # read; and what is clipped written
        return {"bytes": (2 if case["clips"] else 1) * nbytes, "flops": (3 if case["clips"] else 2) * sum(sizes)}
    h, k, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotation":
        each = case["tokens"] * (h + k) * d
        # q, k and what becomes of them; backward their gradients both ways; positions
        return {"bytes": each * e * (4 if case["backward"] else 2) + 4 * case["tokens"], "flops": each * (37 if case["backward"] else 12)}
    lengths = _lengths(case)
    if case["op"] == "attention":
        pairs, n = sum(m * (m + 1) // 2 for m in lengths), case["tokens"]
        # q, o; k, v; lse; backward do, dq; dk, dv.  Two products forward, five backward
        return {"bytes": n * (h + k) * d * e * (4 if case["backward"] else 2) + 4 * n * h, "flops": pairs * h * d * (14 if case["backward"] else 4)}
    total = sum(m + 1 for m in lengths)
    return {"bytes": 2 * total * k * d * e + case["batch"] * (2 * h + 2 * k) * d * e, "flops": 4 * total * h * d}


# ----------------------------------------------------- the definition, 64 bits -----
def _exact_rotation(s):
    """Pairs as complex numbers."""
    case, found = s["case"], {}
    r = case["rotary"]
    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), s["positions"].double()[:, None] * s["frequencies"].double())[:, None]

    def pairs(x):
        return torch.complex(x[..., 0:r:2].contiguous(), x[..., 1:r:2].contiguous()) if case["interleaved"] else torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous())

    def back(x, z):
        y = x.clone()
        if case["interleaved"]:
            y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
        else:
            y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
        return y

    for name in ("q", "k"):
        x, w = s[name].double(), s[name + "w"].double()
        rms = ((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS_NORM) ** 0.5
        y = x / rms * w
        found[name] = back(y, pairs(y) * turn)
        if case["backward"]:
            dy = s["d" + name].double()
            g = back(dy, pairs(dy) * turn.conj())
            found["d" + name] = g * w / rms - x * (g * w * x).sum(-1, keepdim=True) / (x.shape[-1] * rms ** 3)
            found["d" + name + "w"] = torch.einsum("thd,thd->d", g, x / rms)
    return found


def _exact_attention(s):
    """One head of one sequence after another."""
    n, h, d = s["q"].shape
    kv, back = s["k"].shape[1], s["case"]["backward"]
    zeros = lambda heads: torch.zeros(n, heads, d, device="cuda", dtype=torch.float64)  # noqa: E731
    found = {"o": zeros(h), "lse": torch.full((h, n), -math.inf, device="cuda", dtype=torch.float64)}
    if back:
        found.update(dq=zeros(h), dk=zeros(kv), dv=zeros(kv))
    for lo, hi in zip(s["ends"], s["ends"][1:]):
        for head in range(h if hi > lo else 0):
            of = head // (h // kv)
            q, k, v = s["q"][lo:hi, head].double(), s["k"][lo:hi, of].double(), s["v"][lo:hi, of].double()
            z = torch.mm(q, k.t()) / math.sqrt(d)
            z = torch.where(torch.ones_like(z, dtype=torch.bool).tril_(), z, -math.inf)
            p = torch.softmax(z, 1)
            found["lse"][head, lo:hi] = torch.logsumexp(z, 1)
            found["o"][lo:hi, head] = torch.mm(p, v)
            if back:
                do = s["do"][lo:hi, head].double()
                found["dv"][lo:hi, of] += torch.mm(p.t(), do)
                dp = torch.mm(do, v.t())
                dz = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                found["dq"][lo:hi, head] = torch.mm(dz, k)
                found["dk"][lo:hi, of] += torch.mm(dz.t(), q)
    return found


def _exact_step(s):
    b, h, d = s["q"].shape
    kv = s["k"].shape[1]
    out = torch.empty(b, h, d, device="cuda", dtype=torch.float64)
    for i, n in enumerate(s["host"]):
        for of in range(kv):
            k = torch.cat([s["keys"][i, :n, of], s["k"][i, of:of + 1]]).double()
            v = torch.cat([s["values"][i, :n, of], s["v"][i, of:of + 1]]).double()
            heads = slice(of * (h // kv), (of + 1) * (h // kv))
            out[i, heads] = torch.mm(torch.softmax(torch.mm(s["q"][i, heads].double(), k.t()) / math.sqrt(d), 1), v)
    return {"o": out, "keys": None, "values": None}


def _exact_clip(s):
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t.double()) for t in s["gradients"]]))
    factor = min(1.0, s["limit"] / (norm.item() + EPS_CLIP))
    return {"norm": norm, "gradients": [t.double() * factor for t in s["buffers"]]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotation": _exact_rotation, "attention": _exact_attention, "step": _exact_step, "clip": _exact_clip}[case["op"]](s)
