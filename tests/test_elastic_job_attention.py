"""The scheduled job's model with attention as its mixer: the operators together, as a training step and a continuation use them."""
import pytest
import torch

from paper_2108_03645_amd import elastic_job

gpu = pytest.mark.gpu


def test_mixers_are_checked():
    with pytest.raises(ValueError):
        elastic_job.Model(mixer="convolution", device="cpu")
    with pytest.raises(ValueError):
        elastic_job.Model(mixer="attention", width=192, device="cpu")
    assert len(elastic_job.Model(7, 128, 1, device="cpu", mixer="attention").parameters()) == 4
    assert len(elastic_job.Model(7, 128, 1, device="cpu").parameters()) == 3


def plain_loss(model, tokens):
    """The model in torch's operations of 32 bits."""
    p = {n: getattr(model, n).detach().clone().requires_grad_() for n in ("embedding", "output", "matrices", "norms", "head_norms")}
    ids, target = tokens[:, :-1], tokens[:, 1:].reshape(-1)
    b, n = ids.shape
    norm = torch.nn.functional.layer_norm
    angle = torch.arange(n, device=tokens.device)[:, None] * model.frequencies
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turned(x, w):
        x = x * (x.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * w
        u, v = x.chunk(2, -1)
        return torch.cat([u * cos - v * sin, v * cos + u * sin], -1)

    x = p["embedding"][ids]
    for k in range(model.blocks):
        queries, keys_values, out = p["matrices"][3 * k:3 * k + 3]
        y = norm(x, (model.width,), p["norms"][k, 0], p["norms"][k, 1])
        q = turned((y @ queries.t()).view(b, n, model.heads, model.dim), p["head_norms"][k, 0])
        keys, values = (y @ keys_values.t()).view(b, n, 2, model.heads // 2, model.dim).unbind(2)
        keys, values = (t.repeat_interleave(2, 2).transpose(1, 2).contiguous() for t in (turned(keys, p["head_norms"][k, 1]), values))
        z = q.transpose(1, 2).contiguous() @ keys.transpose(2, 3).contiguous() * model.dim ** -0.5
        z = z.masked_fill(torch.ones(n, n, device=z.device, dtype=torch.bool).triu(1), -float("inf"))
        x = x + (torch.softmax(z, -1) @ values).transpose(1, 2).reshape(b, n, -1) @ out.t()
    y = norm(x, (model.width,), p["norms"][-1, 0], p["norms"][-1, 1])
    z = y.reshape(-1, model.width) @ p["output"].t()
    return torch.nn.functional.cross_entropy(z, target), p


@gpu
def test_the_gradients_are_those_of_the_model_in_32_bits():
    model = elastic_job.Model(vocabulary=300, width=128, blocks=2, seed=2, mixer="attention", dim=32)
    tokens = torch.randint(0, 300, (6, 90), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    loss = model.loss(tokens)
    loss.backward()
    want, p = plain_loss(model, tokens)
    want.backward()
    # some twenty roundings to bfloat16 one behind the other in either direction, 2^-8 / 3^0.5 of a value each: 2 %; norms may double them
    assert abs(loss - want) < 0.04 * want
    for name, q in p.items():
        assert (getattr(model, name).grad - q.grad).norm() < 0.04 * q.grad.norm(), name


@gpu
@pytest.mark.parametrize("clip", [None, 0.5, 1e9])
def test_steps_at_changing_batches_run(clip):
    model = elastic_job.Model(vocabulary=200, width=128, blocks=1, mixer="attention")
    worker, language = elastic_job.Worker(model, clip=clip), elastic_job.Language(200, 24)
    for n in (1, 7, 32, 3):
        before = [t.detach().clone() for t in [model.matrices] + model.parameters()]
        assert worker.step(language.batch(n)).isfinite()
        assert all((a != b.detach()).any() and b.isfinite().all() for a, b in zip(before, [model.matrices] + model.parameters()))
        if clip == 0.5:
            norm = torch.stack([t.grad.norm() for t in [model.matrices] + model.parameters()]).norm()
            assert norm <= 0.5 * (1 + 1e-5)


@gpu
def test_single_steps_continue_like_the_whole_sequence():
    model = elastic_job.Model(vocabulary=300, width=128, blocks=2, seed=3, mixer="attention")
    tokens = torch.randint(0, 300, (5, 21), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    answer = model.continue_from(tokens, 6)
    for n in range(6):
        with torch.no_grad():
            y, _ = model.hidden(torch.cat([tokens, answer[:, :n]], 1))
            z = y[:, -1].float() @ model.output.float().t()
        chosen = z.gather(1, answer[:, n:n + 1])[:, 0]
        # the step's choice is the likeliest word up to the roundings of 16 bits on the way
        assert (z.max(1).values - chosen).max() < 0.25, n


@gpu
def test_the_job_runs_with_attention(capsys):
    losses, right = elastic_job.main(steps=3, generations=2, mixer="attention", clip=1.0)
    print(capsys.readouterr().out)
    assert all(loss == loss and abs(loss) < 100 for loss in losses) and 0 <= right <= 1


def test_states_of_another_kind_are_refused():
    """Attention begins a sequence anew: what the recurrence would go on from has no place in it."""
    model = elastic_job.Model(7, 128, 1, device="cpu", mixer="attention")
    with pytest.raises(ValueError):
        model.hidden(torch.zeros(1, 3, dtype=torch.int64), [torch.zeros(1, 128)])
