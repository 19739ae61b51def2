"""A job for the search: a small language model that trains at whatever local batch the winning schedule gives it.

    python -m paper_2108_03645_amd.elastic_job [--mixer recurrence|attention] [--clip LIMIT]

One pass of the paper's loop (Section 3.1) with a real worker on one GPU: the job's steps are timed at a few local batches, a line
through them gives the slope a and the offset d of its iteration time t(B, g) = a*B/g + c*log2(g) + d ("profiled online",
Section 3.2.1), the search places it among other jobs, and the worker trains on at its share of the batch, with the learning rate
scaled by the batch (Section 3.3.2).  Layer norm, recurrence or attention, and loss are ``train``'s and make a; the clipping of the gradients and
the update of the matrices are ``train``'s as well and belong to d.  At the end the model continues a sequence token by token.

Data: a synthetic language, in which every word has one usual successor."""
from __future__ import annotations

import time

import numpy as np
import torch

from . import train, workloads


class Model:
    """Embedding, blocks of (layer norm, a mixer between projections), layer norm, output table.  The mixer is the gated recurrence, or causal
    attention with two query heads of `dim` elements to a key head, their norms and the rotation by positions."""

    def __init__(self, vocabulary=1000, width=256, blocks=2, device="cuda:0", seed=0, mixer="recurrence", dim=64):
        if mixer not in ("recurrence", "attention"):
            raise ValueError(f"mixer: recurrence or attention, not {mixer!r}")
        if mixer == "attention" and width % (2 * dim):
            raise ValueError(f"width: a multiple of {2 * dim} is wanted, got {width}")
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *shape, std: (torch.randn(*shape, generator=g, device=device) * std).requires_grad_()  # noqa: E731
        self.vocabulary, self.width, self.blocks = vocabulary, width, blocks
        self.embedding = normal(vocabulary, width, std=1.0)
        self.output = normal(vocabulary, width, std=width ** -0.5)
        # the matrices of all blocks in one tensor (of each: gate, value, out; or queries, keys over values, out), so that one call updates them all
        self.matrices = normal(3 * blocks, width, width, std=width ** -0.5)
        self.norms = torch.ones(blocks + 1, 2, width, device=device)
        self.norms[:, 1] = 0
        self.norms.requires_grad_()
        self.mixer, self.dim, self.heads = mixer, dim, width // dim
        if mixer == "attention":
            self.head_norms = torch.ones(blocks, 2, dim, device=device, requires_grad=True)
            self.frequencies = 10000.0 ** (-torch.arange(0, dim, 2, device=device) / dim)

    def parameters(self):
        """The tensors that learn beside the matrices."""
        return [self.embedding, self.output, self.norms] + ([self.head_norms] if self.mixer == "attention" else [])

    def projected(self, k, y, positions, matrices):
        """Queries, keys (normed and turned) and values of the rows y [tokens, width] in block k."""
        queries, keys_values = matrices
        q = (y @ queries.t()).view(-1, self.heads, self.dim)
        keys, values = (y @ keys_values.t()).view(-1, 2, self.heads // 2, self.dim).unbind(1)
        q, keys = train.head_norm_rotation(q, keys, self.head_norms[k, 0], self.head_norms[k, 1], positions, self.frequencies)
        return q, keys, values

    def hidden(self, tokens, states=None):
        """[batch, steps, width] after the last norm, and the blocks' states behind the last step: of the recurrence, or the keys and values
        [batch, steps, heads, dim] that attention met.  states: what the recurrence goes on from."""
        if self.mixer == "attention":
            if states is not None:
                raise ValueError("states: attention begins a sequence anew; attention_step continues one")
            return self.attended(tokens)
        x = self.embedding[tokens].bfloat16()
        ends = []
        for k in range(self.blocks):
            gate, value, out = self.matrices[3 * k:3 * k + 3].bfloat16()
            y = train.layer_norm(x, self.norms[k, 0], self.norms[k, 1])
            h, end = train.gated_recurrence(y @ gate.t(), y @ value.t(), None if states is None else states[k])
            x = x + h @ out.t()
            ends.append(end)
        return train.layer_norm(x, self.norms[-1, 0], self.norms[-1, 1]), ends

    def attended(self, tokens):
        batch, steps = tokens.shape
        x = self.embedding[tokens.reshape(-1)].bfloat16()
        offsets = torch.arange(batch + 1, device=x.device, dtype=torch.int32) * steps
        positions = torch.arange(steps, device=x.device, dtype=torch.int32).repeat(batch)
        ends = []
        for k in range(self.blocks):
            *inner, out = self.matrices[3 * k:3 * k + 3].bfloat16()
            y = train.layer_norm(x, self.norms[k, 0], self.norms[k, 1])
            q, keys, values = self.projected(k, y, positions, inner)
            x = x + train.attention(q, keys, values, offsets).flatten(1) @ out.t()
            ends.append([t.unflatten(0, (batch, steps)) for t in (keys, values)])
        return train.layer_norm(x, self.norms[-1, 0], self.norms[-1, 1]).view(batch, steps, -1), ends

    def loss(self, tokens):
        """The mean loss of every next token; tokens below 0 are padding."""
        y, _ = self.hidden(tokens[:, :-1].clamp(min=0))
        target = tokens[:, 1:].reshape(-1)
        loss = train.linear_cross_entropy(y.reshape(-1, self.width), self.output.bfloat16(), target)
        return loss.sum() / (target >= 0).sum().clamp(min=1)

    @torch.no_grad()
    def continue_from(self, tokens, n):
        """The n likeliest next tokens one after another, by the mixer's single steps: [batch, n]."""
        y, states = self.hidden(tokens)
        y, found = y[:, -1], []
        weights = self.matrices.bfloat16()
        output = self.output.bfloat16()
        if self.mixer == "attention":             # caches with room for what comes
            batch, steps = tokens.shape
            lengths = torch.full((batch,), steps, device=y.device, dtype=torch.int32)
            states = [[torch.cat([t, t.new_empty(batch, n, *t.shape[2:])], 1) for t in state] for state in states]
        for _ in range(n):
            token = (y @ output.t()).argmax(1)
            found.append(token)
            x = self.embedding[token].bfloat16()
            for k in range(self.blocks):
                y = train.layer_norm(x, self.norms[k, 0], self.norms[k, 1])
                if self.mixer == "attention":
                    h = train.attention_step(*self.projected(k, y, lengths, weights[3 * k:3 * k + 2]), *states[k], lengths).flatten(1)
                else:
                    h = train.gated_recurrence_step(y @ weights[3 * k].t(), y @ weights[3 * k + 1].t(), states[k])
                x = x + h @ weights[3 * k + 2].t()
            if self.mixer == "attention":
                lengths += 1
            y = train.layer_norm(x, self.norms[-1, 0], self.norms[-1, 1])
        return torch.stack(found, 1)


class Worker:
    """Trains a model at a local batch that may change between any two steps.  The learning rate is proportional to the batch: `rate` at
    `per_sample_rate_at` sequences.  clip: the norm that all gradients together are clipped to; None: they are not."""

    def __init__(self, model, rate=0.02, per_sample_rate_at=512, clip=None):
        self.model, self.rate, self.at, self.clip = model, rate, per_sample_rate_at, clip
        self.momentum = torch.zeros_like(model.matrices)
        self.others = torch.optim.AdamW(model.parameters(), lr=rate / 4, weight_decay=0.0)

    def rate_of(self, batch):
        return self.rate * batch / self.at

    def step(self, tokens):
        model, rate = self.model, self.rate_of(tokens.shape[0])
        model.matrices.grad = None
        self.others.zero_grad(set_to_none=True)
        loss = model.loss(tokens)
        loss.backward()
        if self.clip is not None:
            train.clip_gradients([model.matrices.grad] + [p.grad for p in model.parameters()], self.clip)
        update = train.orthogonal_update(model.matrices.grad, self.momentum)
        with torch.no_grad():
            model.matrices.add_(update, alpha=-rate)
        for group in self.others.param_groups:
            group["lr"] = rate / 4
        self.others.step()
        return loss.detach()


class Language:
    """Sequences over a vocabulary in which every word has one successor, taken with a probability of 0.9."""

    def __init__(self, vocabulary, steps, device="cuda:0", seed=0):
        self.g = torch.Generator(device=device).manual_seed(seed)
        self.vocabulary, self.steps, self.device = vocabulary, steps, device
        self.successor = torch.randperm(vocabulary, generator=self.g, device=device)

    def batch(self, n):
        words = torch.randint(0, self.vocabulary, (n, self.steps + 1), generator=self.g, device=self.device)
        usual = torch.rand(n, self.steps, generator=self.g, device=self.device) < 0.9
        for t in range(self.steps):
            words[:, t + 1] = torch.where(usual[:, t], self.successor[words[:, t]], words[:, t + 1])
        return words


def fit(batches, seconds):
    """(a, d) of seconds = a * batch + d by least squares, neither below 0 (what ones_jobs takes)."""
    b, t = np.asarray(batches, np.float64), np.asarray(seconds, np.float64)
    a = max(0.0, float(((b - b.mean()) * (t - t.mean())).sum() / max(((b - b.mean()) ** 2).sum(), 1e-300)))
    return a, max(0.0, float((t - a * b).mean()))


def local_batch(slot, slot_of_gpu, batch_of_gpu):
    """The samples that a worker of the job in `slot` processes a step, by ones_placement's map (0: the job waits)."""
    mine = np.flatnonzero(np.asarray(slot_of_gpu) == slot)
    return int(np.asarray(batch_of_gpu)[mine[0]]) if mine.size else 0


def measure(worker, language, batches, repeats=3):
    """Seconds a step at each local batch: the median of `repeats`, behind a first step that is not counted."""
    seconds = []
    for n in batches:
        tokens, times = language.batch(n), []
        for _ in range(repeats + 1):
            torch.cuda.synchronize()
            begun = time.perf_counter()
            worker.step(tokens)
            torch.cuda.synchronize()
            times.append(time.perf_counter() - begun)
        seconds.append(float(np.median(times[1:])))
    return seconds


def place(a, d, batches, generations=20, slot=0):
    """The local batch that the search gives a job with these figures, its samples and GPUs, and the cluster's GPUs.  The cluster runs
    other jobs when this one arrives in `slot`; arrivals are served first.  Raises RuntimeError if the winning schedule lets it wait."""
    from . import ones

    cluster, jobs = workloads.paper_scale()
    jobs.active[slot] = 0
    search = ones.Search(cluster, jobs)
    try:
        search.generation(generations)
        jobs.active[slot], jobs.job_id[slot] = 1, jobs.job_id.max() + 1
        jobs.a[slot], jobs.d[slot], jobs.gpu_max_batch[slot] = a, d, batches[-1]
        jobs.bmin[slot], jobs.bmax[slot], jobs.remaining[slot] = batches[0], 1024, 1e6
        search.set_new_jobs_first(True)
        search.set_jobs(jobs)
        search.generation(1)
        batch, (samples, gpus, _) = local_batch(slot, *search.placement()), search.best()
    finally:
        search.close()
    if not batch:
        raise RuntimeError("the winning schedule lets the job wait")
    return batch, int(samples[slot]), int(gpus[slot]), cluster.n_gpus


def main(steps=60, generations=20, slot=0, mixer="recurrence", clip=None):
    model = Model(vocabulary=4000, width=512, mixer=mixer)
    worker, language = Worker(model, clip=clip) if clip is not None else Worker(model), Language(model.vocabulary, 256)
    first = worker.step(language.batch(32)).item()
    batches = [32, 64, 128, 256, 512]
    seconds = measure(worker, language, batches)
    a, d = fit(batches, seconds)
    print("steps at local batches", ", ".join(f"{n}: {1e3 * t:.2f} ms" for n, t in zip(batches, seconds)),
          f"-> a = {1e6 * a:.2f} us a sample, d = {1e3 * d:.2f} ms")

    batch, samples, gpus, of = place(a, d, batches, generations, slot)
    print(f"the winning schedule gives the job {samples} samples on {gpus} of {of} GPUs: {batch} a worker")

    losses = [first] + [worker.step(language.batch(batch)).item() for _ in range(steps)]
    print(f"loss {losses[0]:.3f} at first, {losses[1]:.3f} -> {losses[-1]:.3f} in {steps} steps")
    prompt = language.batch(4)[:, :16]
    answer = model.continue_from(prompt, 8)
    want, last = [], prompt[:, -1]
    for _ in range(8):
        last = language.successor[last]
        want.append(last)
    right = (answer == torch.stack(want, 1)).float().mean().item()
    print(f"continues four sequences by eight words, {100 * right:.0f} % the usual ones")
    return losses, right


if __name__ == "__main__":
    import argparse

    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--mixer", choices=("recurrence", "attention"), default="recurrence")
    parser.add_argument("--clip", type=float, metavar="LIMIT", help="clip the gradients to this norm")
    main(**vars(parser.parse_args()))
