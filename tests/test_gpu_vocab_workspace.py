"""Losses over a vocabulary in the smallest workspaces, which one allocation for
both passes is: every piece's sums carried to the next."""

import pytest

from test_gpu_vocab_loss import _check_grad, _check_loss, _definition, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows, cols, vocab, top", [(64, 64, 30000, 0), (300, 72, 9001, 0),
                                                    (5, 2100, 5000, 0), (70, 100, 9001, 21)])
def test_a_small_workspace_for_both_passes(torch, rows, cols, vocab, top, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, w, *target, dloss = _inputs(torch, rows, cols, vocab, dtype, top)
    t = 1.5 if top else 1.0
    loss = layers.distill_loss if top else layers.vocab_loss
    grad = layers.distill_loss_grad if top else layers.vocab_loss_grad
    args = (*target, t) if top else target
    d = _definition(torch, x, w, target[0], target[1] if top else None, t, dloss)
    most = layers.vocab_workspace(x, w, top).numel()
    for n in (0, most // 50, most // 7, most // 2):
        print("workspace", n, "of", most, rows, cols, vocab, top, dtype, flush=True)
        space = layers.vocab_workspace(x, w, top, most=n)
        behind = torch.full((space.numel() + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        out, lse = loss(x, w, *args, workspace=behind[:space.numel()])
        _check_loss(d, out, lse)
        dw = torch.full((vocab, cols), 7.0, device="cuda")
        dx = grad(x, w, *args, lse, dloss, dw, workspace=behind[:space.numel()])
        _check_grad(torch, d, dx, dw, dtype, pieces=vocab / 256)
        assert bool((behind[space.numel():] == 0x5a).all())
        # the loss alone, in what it needs alone
        alone = layers.vocab_workspace(x, w, top, grad=False, most=0)
        again, _ = loss(x, w, *args, workspace=alone)
        _check_loss(d, again, lse)


def test_a_row_of_infinities_and_absent_pieces(torch):
    """Pieces whose logits are all -inf leave no reference to the next."""
    from paper_1805_07891_amd import layers
    import math
    x = torch.zeros(3, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(2000, 64, device="cuda", dtype=torch.bfloat16)
    x[:, 0], x[:, 1] = 1.0, torch.tensor([1.0, 2.0, 3.0])
    w[:, 1] = torch.arange(2000, device="cuda") % 7
    w[:600, 0] = w[1500:, 0] = -math.inf
    target = torch.tensor([700, 1499, 900], device="cuda")
    space = layers.vocab_workspace(x, w, grad=False, most=0)
    whole, whole_lse = layers.vocab_loss(x, w, target)
    loss, lse = layers.vocab_loss(x, w, target, workspace=space)
    z = x.double().cpu()[:, 1:] @ w.double().cpu()[600:1500, 1:].t()
    want_lse = torch.logsumexp(z, 1)
    want = want_lse - z.gather(1, target.cpu()[:, None] - 600)[:, 0]
    for got, got_lse in ((whole, whole_lse), (loss, lse)):
        assert bool(((got_lse.double().cpu() - want_lse).abs() <= 2e-6 * want_lse).all())
        assert bool(((got.double().cpu() - want).abs() <= 2e-6 * want_lse).all())
