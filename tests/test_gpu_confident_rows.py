"""Rows whose target has nearly all of the softmax: losses near 0, of small and
of very large logits, against 64 bits.

The logits are exact: each row of x picks one column, where w holds them.  With the
largest logit as the reference its own term is 1, and the loss is log(1 + s) plus
the target's distance from it.  Bounds, with u = 2^-24: a lane adds n terms to a sum of 1
to 2, each addition off by u, never by more than the terms themselves; the terms, the
logarithm and the distance are off by a few u of themselves.
"""

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


TARGETS = [10.0, 12.0, 20.0, 50.0, 100.0, 500.0]  # logits; exact in every type


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows, cols, vocab", [(12, 64, 8), (1100, 96, 4100), (2100, 72, 8200)])
def test_losses_near_zero(torch, rows, cols, vocab, dtype):
    """Logits of the target from 10 to 500, the others 0 (64, 128 and 256 rows a tile)."""
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x = torch.zeros(rows, cols, device="cuda", dtype=dtype)
    w = torch.zeros(vocab, cols, device="cuda", dtype=dtype)
    # column c of w: 1 at one entry of the vocabulary, whose logit a row of x chooses
    size = torch.tensor(TARGETS, device="cuda")[torch.arange(rows, device="cuda") % len(TARGETS)]
    column = torch.arange(rows, device="cuda") % cols
    entry = torch.arange(cols, device="cuda") * 37 % vocab
    if vocab < cols:
        column %= vocab
        entry = torch.arange(cols, device="cuda")
        w[torch.arange(vocab), torch.arange(vocab)] = 1.0
    else:
        w[entry, torch.arange(cols, device="cuda")] = 1.0
    target = entry[column]
    x[torch.arange(rows, device="cuda"), column] = size.to(dtype)
    print("confident rows", rows, cols, vocab, dtype, flush=True)
    loss, lse = layers.vocab_loss(x, w, target)
    rest = (vocab - 1) * torch.exp(-size.double())
    want = torch.log1p(rest)
    adds = min(vocab, 128)
    off = torch.minimum(rest, torch.tensor(adds * U, device="cuda", dtype=torch.float64))
    bound = off + 4 * U * (want + U)
    assert bool((loss >= 0).all()), loss.min().item()
    worst = ((loss.double() - want).abs() / (bound + 2 * U)).max().item()
    assert worst <= 1.0, f"{worst:.3g} times the bound"
    # a teacher with this one entry is the same loss
    one, _ = layers.distill_loss(x, w, target[:, None].contiguous(), torch.zeros(rows, 1, device="cuda"))
    assert bool((one >= 0).all()) and bool(((one.double() - want).abs() <= bound + 2 * U).all())


@pytest.mark.parametrize("dtype, size", [("bfloat16", 2.0 ** 20), ("float16", 2.0 ** 15),
                                         ("float32", 2.0 ** 60)])
def test_very_large_logits(torch, dtype, size):
    """Logits up to ``size`` squared: softmax is one entry, losses are differences."""
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    rows, cols, vocab = 16, 64, 200
    x = torch.zeros(rows, cols, device="cuda", dtype=dtype)
    w = torch.zeros(vocab, cols, device="cuda", dtype=dtype)
    # products of few digits: exact in fp32
    x[:, 0] = (size * (1.0 - torch.arange(rows, device="cuda") / 32)).to(dtype)
    w[:, 0] = (size * (torch.arange(vocab, device="cuda") % 100 + 1) / 128).to(dtype)
    w[99, 0] = w[199, 0] = size  # the largest twice
    w[50, 0] = size * 1.25
    target = torch.arange(rows, device="cuda") * 10
    target[::2] = 50
    print("very large logits", dtype, flush=True)
    loss, lse = layers.vocab_loss(x, w, target)
    z = x.double() @ w.double().t()
    want_lse = torch.logsumexp(z, 1)
    want = want_lse - z.gather(1, target[:, None])[:, 0]
    assert bool(((lse.double() - want_lse).abs() <= 2 * U * want_lse).all())
    assert bool(((loss.double() - want).abs() <= 2 * U * want).all())
    dw = torch.full((vocab, cols), 7.0, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, None, dw)
    G = torch.exp(z - want_lse[:, None])
    G[torch.arange(rows), target] -= 1.0
    half = torch.finfo(dtype).eps / 2
    wdx, wdw = G @ w.double(), G.t() @ x.double()
    assert bool(((dx.double() - wdx).abs() <= (half + 4 * U) * wdx.abs()).all())
    # sums of up to 16 products of 22 bits and more
    size_dw = G.abs().t() @ x.double().abs()
    assert bool(((dw.double() - wdw).abs() <= (2.0 ** -21 + 32 * U) * size_dw).all())
