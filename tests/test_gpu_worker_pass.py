"""The worker's operators together, as a training program uses them: two
workers with rows of their own run layer norm, the cross entropy over the
vocabulary and its gradients from the weights that the job hands out, write
the weight gradients into the arenas that they push, and the job steps.
Every step's loss and the weights after it are compared with the same program
in 64 bits."""

import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


ROWS, COLS, VOCAB, WORKERS, STEPS, EPS = 96, 64, 500, 2, 3, 1e-5
KEYS = (COLS, COLS, VOCAB * COLS)  # the norm's weight and bias, the vocabulary's weights


def _program(torch, x, targets, weight, bias, w, lr, distill):
    """One step in 64 bits: (losses, new weights); plain SGD on the workers' sum."""
    gw, gb, gv, losses = 0, 0, 0, []
    for xi, t in zip(x, targets):
        mean = xi.mean(1, keepdim=True)
        c = xi - mean
        h = c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
        y = h * weight + bias
        temp = 2.0 if distill else 1.0
        z = y @ w.t() / temp
        lse = torch.logsumexp(z, 1, keepdim=True)
        q = torch.zeros_like(z)
        if distill:
            q.scatter_add_(1, t[0], torch.softmax(t[1].double() / temp, 1))
        else:
            q[t >= 0, t[t >= 0]] = 1.0
        live = q.sum(1) > 0
        losses.append((temp * temp * (torch.xlogy(q, q) + q * (lse - z)).sum(1)))
        G = torch.where(live[:, None], temp * (torch.exp(z - lse) - q), 0.0) / ROWS
        dy = G @ w
        gv = gv + G.t() @ y
        gw, gb = gw + (dy * h).sum(0), gb + dy.sum(0)
    return losses, (weight - lr * gw, bias - lr * gb, w - lr * gv)


@pytest.mark.parametrize("distill", [False, True])
def test_two_workers_train(torch, distill):
    from paper_1805_07891_amd import layers
    from paper_1805_07891_amd.job import TorchJob
    from paper_1805_07891_amd.workloads import Job
    lr = 0.5
    g = torch.Generator(device="cuda").manual_seed(7)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    spec = Job("head", WORKERS, KEYS, lr=lr, weight_decay=0.0)
    job = TorchJob(spec, "cuda:0", optimizer="sgd")
    w0 = torch.zeros(job.arena_elems, device="cuda")
    init = (1.0 + 0.1 * r(COLS), 0.1 * r(COLS), r(VOCAB, COLS) / math.sqrt(COLS))
    for o, t in zip(job.offsets, init):
        w0[o:o + t.numel()] = t.flatten()
    job.set_weights(w0)
    arenas = [torch.zeros(job.arena_elems, device="cuda") for _ in range(WORKERS)]
    for i, a in enumerate(arenas):
        job.attach_grads(i, a)
    x = [r(ROWS, COLS) * 2.0 + 0.5 for _ in range(WORKERS)]
    if distill:
        targets = [(torch.stack([torch.randperm(VOCAB, generator=g, device="cuda")[:9]
                                 for _ in range(ROWS)]), 2.0 * r(ROWS, 9)) for _ in range(WORKERS)]
    else:
        targets = [torch.randint(-1, VOCAB, (ROWS,), generator=g, device="cuda")
                   for _ in range(WORKERS)]
    dloss = torch.full((ROWS,), 1.0 / ROWS, device="cuda")
    want = [t.double() for t in init]
    for step in range(STEPS):
        print("step", step, "distill", distill, flush=True)
        job.sync()
        weight, bias, w = job.weights(0), job.weights(1), job.weights(2, VOCAB, COLS)
        got = []
        for i in range(WORKERS):
            y, mean, rstd = layers.layer_norm(x[i], weight, bias, EPS)
            dw = job.gradient(i, 2, VOCAB, COLS)
            if distill:
                loss, lse = layers.distill_loss(y, w, *targets[i], 2.0)
                dy = layers.distill_loss_grad(y, w, *targets[i], 2.0, lse, dloss, dw)
            else:
                loss, lse = layers.vocab_loss(y, w, targets[i])
                dy = layers.vocab_loss_grad(y, w, targets[i], lse, dloss, dw)
            layers.layer_norm_grad(dy, x[i], weight, mean, rstd, job.gradient(i, 0),
                                   job.gradient(i, 1))
            got.append(loss)
        torch.cuda.synchronize()
        losses, want = _program(torch, [t.double() for t in x], targets, *want, lr, distill)
        job.push_and_step()
        job.sync()
        for a, b in zip(got, losses):
            # a loss of about 6 from logits of some 64 terms: 2^-24 times a few hundred
            assert bool(((a.double() - b).abs() <= 3e-5 * (1.0 + b.abs())).all())
        for k, b in enumerate(want):
            a = job.weights(k).double().view(b.shape)
            # weights of about 1 rounded to fp32 at each step, gradients right to about 1e-5
            moved = (b - init[k].double()).abs().max()
            assert bool(((a - b).abs() <= 1e-4 * moved + 2.0 ** -22 * b.abs()).all()), (step, k)
    job.destroy()
