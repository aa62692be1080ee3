"""The worker's operators on torch's current stream and the job on its own, ordered
on the GPU alone: by streams that wait for each other, and by events given with the
pushes.  Delays in front of either side's work show an order that is missing."""

import math

import pytest

from test_gpu_worker_pass import COLS, EPS, KEYS, ROWS, STEPS, VOCAB, WORKERS, _program

pytestmark = pytest.mark.gpu

DELAY = 4_000_000  # clock ticks: some milliseconds


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


@pytest.mark.parametrize("by", ["streams", "events"])
def test_steps_without_waiting_on_the_host(torch, by):
    from paper_1805_07891_amd import layers
    from paper_1805_07891_amd.job import TorchJob
    from paper_1805_07891_amd.workloads import Job
    lr = 0.5
    g = torch.Generator(device="cuda").manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    job = TorchJob(Job("head", WORKERS, KEYS, lr=lr, weight_decay=0.0), "cuda:0", optimizer="sgd")
    assert job.stream != torch.cuda.current_stream()
    w0 = torch.zeros(job.arena_elems, device="cuda")
    init = (1.0 + 0.1 * r(COLS), 0.1 * r(COLS), r(VOCAB, COLS) / math.sqrt(COLS))
    for o, t in zip(job.offsets, init):
        w0[o:o + t.numel()] = t.flatten()
    job.set_weights(w0)
    for i in range(WORKERS):
        job.attach_grads(i, torch.zeros(job.arena_elems, device="cuda"))
    x = [r(ROWS, COLS) * 2.0 + 0.5 for _ in range(WORKERS)]
    targets = [torch.randint(-1, VOCAB, (ROWS,), generator=g, device="cuda") for _ in range(WORKERS)]
    dloss = torch.full((ROWS,), 1.0 / ROWS, device="cuda")
    weight, bias, w = job.weights(0), job.weights(1), job.weights(2, VOCAB, COLS)
    losses = []
    for step in range(STEPS):
        print("step", step, by, flush=True)
        here = torch.cuda.current_stream()
        here.wait_stream(job.stream)  # the weights of the step before, which has read the arenas
        for i in range(WORKERS):
            y, mean, rstd = layers.layer_norm(x[i], weight, bias, EPS)
            loss, lse = layers.vocab_loss(y, w, targets[i])
            torch.cuda._sleep(DELAY)
            dy = layers.vocab_loss_grad(y, w, targets[i], lse, dloss, job.gradient(i, 2, VOCAB, COLS))
            layers.layer_norm_grad(dy, x[i], weight, mean, rstd, job.gradient(i, 0),
                                   job.gradient(i, 1))
            losses.append(loss)
            if by == "events":
                ready = torch.cuda.Event()
                ready.record(here)
                job.push_bucket(i, job.bucket(i, range(len(KEYS))), ready)
        if by == "streams":
            job.stream.wait_stream(here)
            job.push_all()
        with torch.cuda.stream(job.stream):
            torch.cuda._sleep(DELAY)
        job.step()
    job.sync()
    torch.cuda.synchronize()
    want = [t.double() for t in init]
    for step in range(STEPS):
        ref, want = _program(torch, [t.double() for t in x], targets, *want, lr, False)
        for a, b in zip(losses[step * WORKERS:], ref):
            # a loss of about 6 from logits of some 64 terms: 2^-24 times a few hundred
            assert bool(((a.double() - b).abs() <= 3e-5 * (1.0 + b.abs())).all())
    for k, b in enumerate(want):
        a = job.weights(k).double().view(b.shape)
        # weights of about 1 rounded to fp32 at each step, gradients right to about 1e-5
        moved = (b - init[k].double()).abs().max()
        assert bool(((a - b).abs() <= 1e-4 * moved + 2.0 ** -22 * b.abs()).all()), k
    job.destroy()
