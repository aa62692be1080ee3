"""A teacher's entries found by the epilogue of 256 x 256 tiles, which the forward pass
takes where gathering them would cost more: 2100 rows by 8200 entries fill one round
of those tiles (and a rest of smaller ones), and 64 entries of 200 columns for each row are
4 + 2100 * 64 * 200 * 2 / 7e6 = 12 us to gather against 1.5 + 64 * 0.1 = 8."""

import pytest

from test_gpu_vocab_loss import _check_grad, _check_loss, _definition, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows, cols, vocab, top", [(2100, 200, 8200, 64), (2051, 193, 8192, 101)])
def test_entries_of_large_tiles(torch, rows, cols, vocab, top, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, w, index, logits, dloss = _inputs(torch, rows, cols, vocab, dtype, top)
    print("teacher's entries", rows, cols, vocab, top, dtype, flush=True)
    d = _definition(torch, x, w, index, logits, 1.5, dloss)
    loss, lse = layers.distill_loss(x, w, index, logits, 1.5)
    torch.cuda.synchronize()
    _check_loss(d, loss, lse)
    dw = torch.full((vocab, cols), 7.0, device="cuda")
    dx = layers.distill_loss_grad(x, w, index, logits, 1.5, lse, dloss, dw)
    torch.cuda.synchronize()
    _check_grad(torch, d, dx, dw, dtype)
