"""Rows of zeros among small ones: a padded vocabulary, hidden states that were
cleared.  They have no size of their own, so they may not set the scale at which the
others' gradients are held.  Against 64 bits: every entry of P and Q keeps 22 bits down to
2^-38 of the largest there is; the products add (k / 16 + 24) roundings of 2^-23.
"""

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("power", [0, -6, -12, -20])
def test_zero_rows_among_small_ones(torch, power, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    if dtype == torch.float16 and power < -8:
        pytest.skip("fp16 itself has no digits left there")
    rows, cols, vocab = 130, 64, 5000
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, w = (r(rows, cols) * 2.0 ** power).to(dtype), (r(vocab, cols) * 2.0 ** power).to(dtype)
    x[7] = 0.0
    x[8] = 0.0
    w[vocab - 100:] = 0.0  # padding of the vocabulary
    w[11] = 0.0
    target = torch.randint(vocab - 100, (rows,), generator=g, device="cuda")
    target[8] = -1
    dloss = 0.5 + torch.rand(rows, generator=g, device="cuda")
    print("zero rows", power, dtype, flush=True)
    loss, lse = layers.vocab_loss(x, w, target)
    dw = torch.full((vocab, cols), 7.0, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, dloss, dw)
    xd, wd = x.double(), w.double()
    z, size = xd @ wd.t(), xd.abs() @ wd.abs().t()
    want = torch.logsumexp(z, 1)
    p = torch.exp(z - want[:, None])
    live = target >= 0
    q = torch.zeros_like(z)
    q[live.nonzero()[:, 0], target[live]] = 1.0
    f = torch.where(live, dloss.double(), 0.0)[:, None]
    G = f * (p - q)
    # of softmax: logits, lse (its sum: fewer than 100 roundings and the partial sums), exp
    z_off = (cols / 16 + 24) * U * size
    lse_off = z_off.max(1).values + (100 + vocab / 512) * U + 4 * U * want.abs()
    G_off = f * p * (z_off + lse_off[:, None] + 4 * U * (1 + (z - want[:, None]).abs())) + U * G.abs()
    half = torch.finfo(dtype).eps / 2
    plane = 2.0 ** -22 if dtype == torch.float32 else half
    off = (G_off + plane * 1.01 * G.abs()) @ wd.abs() + f * vocab * 2.0 ** -38 * wd.abs().max()
    off = off + (vocab / 16 * 1.1 + 40) * U * 1.1 * (G.abs() @ wd.abs())
    wdx, wdw = G @ wd, G.t() @ xd
    worst = ((dx.double() - wdx).abs() / (off + half * 1.01 * wdx.abs() + torch.finfo(dtype).tiny)).max()
    assert worst <= 1.0, f"dx: {worst.item():.3g} times the bound"
    most = (f[:, 0] * xd.abs().max(1).values).max()
    off = (G_off + 2.0 ** -21 * G.abs()).t() @ xd.abs() + rows * 2.0 ** -38 * most
    off = off + (rows / 16 * 2.2 + 24) * U * 1.1 * (G.abs().t() @ xd.abs())
    worst = ((dw.double() - wdw).abs() / (off + 1e-30)).max()
    assert worst <= 1.0, f"dw: {worst.item():.3g} times the bound"


def test_nothing_but_zeros(torch):
    from paper_1805_07891_amd import layers
    for dtype in (torch.float32, torch.bfloat16):
        x, w = torch.zeros(70, 64, device="cuda", dtype=dtype), torch.zeros(300, 64, device="cuda", dtype=dtype)
        target = torch.arange(70, device="cuda")
        loss, lse = layers.vocab_loss(x, w, target)
        assert bool(((loss - torch.tensor(300.0).log().item()).abs() <= 1e-6).all())
        dw = torch.full((300, 64), 7.0, device="cuda")
        assert not layers.vocab_loss_grad(x, w, target, lse, None, dw).any() and not dw.any()
