"""The job that trains at the local batch the search gives it (paper_2108_03645_amd/elastic_job.py)."""
import numpy as np
import pytest
import torch

from paper_2108_03645_amd import elastic_job


def test_a_line_through_step_times():
    a, d = elastic_job.fit([16, 32, 64], [0.010 + 16e-5, 0.010 + 32e-5, 0.010 + 64e-5])
    assert abs(a - 1e-5) < 1e-12 and abs(d - 0.010) < 1e-12
    assert elastic_job.fit([8, 16], [2.0, 1.0]) == (0.0, 1.5)         # a falling line: no slope, the mean
    assert elastic_job.fit([8], [2.0]) == (0.0, 2.0)


def test_local_batch_of_a_placement():
    slots, batches = np.array([2, 2, 0, -1]), np.array([64, 64, 128, 0])
    assert [elastic_job.local_batch(s, slots, batches) for s in (0, 1, 2)] == [128, 0, 64]


@pytest.mark.gpu
def test_the_model_learns_the_language_and_continues_it(capsys):
    losses, right = elastic_job.main(steps=60, generations=5)
    print(capsys.readouterr().out)
    # a uniform guess costs log 4000 = 8.3, the language itself 0.9 log(1 / 0.9) + 0.1 log(4000 / 0.1) = 1.2
    assert losses[0] > 7 and losses[-1] < 4 and right > 0.5
    assert np.isfinite(losses).all()


@pytest.mark.gpu
def test_single_steps_continue_like_the_whole_sequence():
    model = elastic_job.Model(vocabulary=300, width=64, blocks=2, seed=3)
    tokens = torch.randint(0, 300, (5, 21), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    answer = model.continue_from(tokens, 6)
    for n in range(6):
        with torch.no_grad():
            y, _ = model.hidden(torch.cat([tokens, answer[:, :n]], 1))
            z = y[:, -1].float() @ model.output.float().t()
        # the step's choice is the likeliest word up to the roundings of 16 bits on the way
        chosen = z.gather(1, answer[:, n:n + 1])[:, 0]
        assert (z.max(1).values - chosen).max() < 0.25, n


@pytest.mark.gpu
def test_the_batch_may_change_and_padding_does_not_count():
    model = elastic_job.Model(vocabulary=200, width=64, blocks=1)
    worker, language = elastic_job.Worker(model), elastic_job.Language(200, 24)
    for n in (1, 7, 32, 3):
        assert worker.step(language.batch(n)).isfinite()
    tokens = language.batch(4)
    padded = torch.cat([tokens, torch.full((4, 5), -1, device="cuda")], 1)
    with torch.no_grad():
        whole, short = model.loss(padded), model.loss(tokens)
    assert abs(whole - short) < 1e-5 * short


def test_the_learning_rate_is_proportional_to_the_batch(monkeypatch):
    """At every batch the search may give, for the matrices and for the rest; the operators are stood in for, so no GPU is needed."""
    monkeypatch.setattr(elastic_job.train, "orthogonal_update", lambda grad, momentum: torch.ones_like(grad))
    model = elastic_job.Model(vocabulary=7, width=4, blocks=1, device="cpu")
    monkeypatch.setattr(model, "loss", lambda tokens: sum(p.sum() for p in (model.matrices, model.embedding, model.output, model.norms)))
    worker = elastic_job.Worker(model)
    moved, rates = [], []
    for n in (32, 64, 512, 1024):
        before = model.matrices.detach().clone()
        worker.step(torch.zeros(n, 3, dtype=torch.int64))
        moved.append((before - model.matrices.detach()).mean().item())
        rates.append(worker.others.param_groups[0]["lr"])
    assert np.allclose(np.array(moved) / moved[0], [1, 2, 16, 32], rtol=1e-4) and np.allclose(np.array(rates) / rates[0], [1, 2, 16, 32])
    assert np.allclose(moved, [worker.rate_of(n) for n in (32, 64, 512, 1024)], rtol=1e-4)


class Waiting:
    """A search whose winner has no GPU for the job."""
    closed = False

    def __init__(self, cluster, jobs):
        self.jobs, self.gpus = len(jobs.active), cluster.n_gpus

    def generation(self, n):
        pass

    set_jobs = set_new_jobs_first = generation

    def placement(self):
        return np.full(self.gpus, 1), np.full(self.gpus, 64)

    def best(self):
        return np.zeros(self.jobs, int), np.zeros(self.jobs, int), 0.0

    def close(self):
        Waiting.closed = True


def test_a_job_that_waits_is_not_trained(monkeypatch):
    from paper_2108_03645_amd import ones
    monkeypatch.setattr(ones, "Search", Waiting)
    monkeypatch.setattr(elastic_job, "Model", lambda **k: type("M", (), {"vocabulary": 4}))
    monkeypatch.setattr(elastic_job, "Worker", lambda model: type("W", (), {"step": staticmethod(lambda tokens: torch.zeros(()))}))
    monkeypatch.setattr(elastic_job, "Language", lambda *a: type("L", (), {"batch": staticmethod(lambda n: None)}))
    monkeypatch.setattr(elastic_job, "measure", lambda *a: [1, 2, 3, 4, 5])
    with pytest.raises(RuntimeError, match="wait"):
        elastic_job.main()
    assert Waiting.closed


@pytest.mark.gpu
@pytest.mark.parametrize("a,d", [(2e-5, 1e-3), (1e-4, 2e-2)])
def test_the_search_gives_the_job_a_batch(a, d):
    batch, samples, gpus, of = elastic_job.place(a, d, [32, 64, 128, 256, 512], generations=5)
    assert 0 < batch <= 512 and 1 <= gpus <= of and 32 <= samples <= 1024 and batch * gpus >= samples
