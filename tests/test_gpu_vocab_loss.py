"""The losses over a vocabulary and their gradients against 64 bits.

Bounds, with u = 2^-23 for a sum in the matrix cores (16 products at once, then
one addition to the fp32 sum; truncation counted as two roundings) and t the
type's half step.  A logit is wrong by at most (D / 16 + 24) u times its sum
of magnitudes; the logarithm of the sum of exponentials by the largest such
error and the roundings of exponentials and their sums (fewer than 100 u and
the partial sums' number over 16); softmax - q by that times the softmax.
P is rounded to the type (fp32: 22 bits), Q to two fp16 planes (22 bits),
both down to 2^-39 of their largest; the products add (k / 16 + 24) u of their
sums of magnitudes.
"""

import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


def _inputs(torch, rows, cols, vocab, dtype, top=0, seed=1, peak=8.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w = r(vocab, cols) / math.sqrt(cols)
    to = torch.randint(vocab, (rows,), generator=g, device="cuda")
    x = r(rows, cols) + peak * torch.rand(rows, 1, generator=g, device="cuda") * w[to]
    dloss = 0.2 + torch.rand(rows, generator=g, device="cuda")
    if not top:
        to[::7] = -100
        if rows > 1:
            to[-1] = vocab
        return x.to(dtype), w.to(dtype), to, dloss
    index = torch.randint(-1, vocab + 1, (rows, top), generator=g, device="cuda")
    logits = 3.0 * r(rows, top)
    logits[torch.rand(rows, top, generator=g, device="cuda") < 0.05] = -math.inf
    index[::7] = -1
    return x.to(dtype), w.to(dtype), index, logits, dloss


def _definition(torch, x, w, target, logits, t, dloss):
    """Everything in 64 bits, and the bounds of what may be off."""
    x, w = x.double(), w.double()
    rows, vocab, d = x.shape[0], w.shape[0], x.shape[1]
    z, size = x @ w.t() / t, x.abs() @ w.t().abs() / t
    lse = torch.logsumexp(z, 1)
    q = torch.zeros_like(z)
    if logits is None:
        live = (target >= 0) & (target < vocab)
        q[live.nonzero()[:, 0], target[live]] = 1.0
    else:
        in_ = (target >= 0) & (target < vocab) & (logits != -math.inf)
        live = in_.any(1)
        v = torch.where(in_, logits.double() / t, -math.inf)
        v[~live] = 0.0
        v = torch.softmax(v, 1)
        v[~in_] = 0.0
        q.scatter_add_(1, target.clamp(0, vocab - 1), v)
    p = torch.exp(z - lse[:, None])
    loss = t * t * (torch.xlogy(q, q) + q * (lse[:, None] - z)).sum(1)
    dl = torch.ones(rows, device=x.device) if dloss is None else dloss
    f = torch.where(live, dl.double() * t, 0.0)[:, None]
    # where a row is not live its hidden states may hold anything
    zero = lambda m: torch.where(live[:, None], m, 0.0)  # noqa: E731
    p, z, size, xl = zero(p), zero(z), zero(size), zero(x)
    ends = torch.where(live, lse, 0.0)
    G = f * (p - q)
    z_off = (d / 16 + 24) * U * size
    lse_off = z_off.max(1).values + (100 + vocab / 512) * U + 4 * U * ends.abs()
    p_off = p * (z_off + lse_off[:, None] + 4 * U * (1 + (z - ends[:, None]).abs()))
    q_off = 4 * U * q * (1 + (0 if logits is None else logits.abs().clamp(max=1e4).max().item() / t))
    out = dict(loss=loss, lse=lse, dx=G @ w, dw=G.t() @ xl, live=live)
    terms = q * (z_off + lse_off[:, None] + 8 * U * (1 + (z - ends[:, None]).abs())) + q_off * 30
    out["loss_off"] = t * t * (terms.sum(1) + 4 * U * (q * (ends[:, None] - z).abs()).sum(1)) + 1e-30
    out["lse_off"] = lse_off
    out["G_off"], out["G"] = f.abs() * (p_off + q_off + U * (p - q).abs()), G.abs()
    out["f"], out["x"], out["w"] = f.abs(), xl.abs(), w.abs()
    return out


def _within(got, want, bound, what):
    off = (got.double() - want).abs()
    assert bool(got.isfinite().all()), what
    worst = (off / bound).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"


def _check_loss(d, loss, lse):
    live = d["live"]
    assert not loss[~live].any()
    _within(loss[live], d["loss"][live], d["loss_off"][live], "loss")
    _within(lse[live], d["lse"][live], d["lse_off"][live], "lse")


def _check_grad(torch, d, dx, dw, dtype, pieces=1):
    rows, vocab = d["G"].shape
    if dx is not None:
        assert not dx[~d["live"]].any()
        half = torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 2.0 ** -22
        low = d["f"] * 2.0 ** -39 * d["w"].max()
        off = (d["G_off"] + half * 1.01 * d["G"] + low) @ d["w"]
        off = off + (vocab / 16 * 1.1 + 24 + 16 + pieces) * U * 1.1 * (d["G"] @ d["w"])
        t = torch.finfo(dtype).eps / 2
        _within(dx, d["dx"], off + t * 1.01 * d["dx"].abs() + torch.finfo(dtype).tiny, "dx")
    if dw is not None:
        most = (d["f"][:, 0] * d["x"].max(1).values).max() if rows else 0.0
        off = (d["G_off"] + 2.0 ** -21 * d["G"]).t() @ d["x"] + rows * 2.0 ** -36 * most
        off = off + (rows / 16 * 2.2 + 24) * U * 1.1 * (d["G"].t() @ d["x"])
        _within(dw, d["dw"], off + 1e-30, "dw")


# (rows, columns, vocabulary): one of each, odd ones, rows and columns that end inside a
# tile, products of enough tiles for each of the tile shapes, and of a little more than a
# whole round of tiles (of the logits, of dw, of dx)
SHAPES = [(1, 8, 1), (1, 1, 3), (2, 64, 1000), (5, 40, 300), (64, 128, 257), (100, 100, 1000),
          (257, 72, 513), (300, 512, 2000), (513, 203, 777), (1100, 96, 4100), (2100, 72, 8200),
          (600, 1100, 13100), (13100, 1100, 600)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows, cols, vocab", SHAPES)
def test_cross_entropy(torch, rows, cols, vocab, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, w, target, dloss = _inputs(torch, rows, cols, vocab, dtype)
    if rows > 1:
        x[0] = math.nan  # padding: target -100
    print("cross entropy", rows, cols, vocab, dtype, flush=True)
    d = _definition(torch, x, w, target, None, 1.0, dloss)
    loss, lse = layers.vocab_loss(x, w, target)
    torch.cuda.synchronize()
    _check_loss(d, loss, lse)
    dw = torch.full((vocab, cols), 7.0, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, dloss, dw)
    torch.cuda.synchronize()
    _check_grad(torch, d, dx, dw, dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows, cols, vocab, top, t", [
    (1, 8, 5, 1, 1.0), (3, 64, 1000, 5, 2.0), (70, 100, 300, 128, 0.5), (260, 128, 513, 17, 3.0),
    (40, 72, 100, 1024, 2.0), (1100, 64, 4100, 33, 2.0), (2100, 40, 8200, 64, 1.5)])
def test_distillation(torch, rows, cols, vocab, top, t, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, w, index, logits, dloss = _inputs(torch, rows, cols, vocab, dtype, top)
    print("distillation", rows, cols, vocab, top, t, dtype, flush=True)
    d = _definition(torch, x, w, index, logits, t, dloss)
    loss, lse = layers.distill_loss(x, w, index, logits, t)
    torch.cuda.synchronize()
    _check_loss(d, loss, lse)
    dw = torch.full((vocab, cols), 7.0, device="cuda")
    dx = layers.distill_loss_grad(x, w, index, logits, t, lse, dloss, dw)
    torch.cuda.synchronize()
    _check_grad(torch, d, dx, dw, dtype)


def test_a_teacher_of_one_entry_is_a_target(torch):
    from paper_1805_07891_amd import layers
    x, w, target, dloss = _inputs(torch, 50, 64, 400, torch.bfloat16)
    loss, lse = layers.vocab_loss(x, w, target)
    index, logits = target[:, None].contiguous(), torch.full((50, 1), -3.5, device="cuda")
    loss2, lse2 = layers.distill_loss(x, w, index, logits, 1.0)
    assert torch.equal(lse, lse2) and torch.equal(loss, loss2)
    a, b = torch.empty(400, 64, device="cuda"), torch.empty(400, 64, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, dloss, a)
    dx2 = layers.distill_loss_grad(x, w, index, logits, 1.0, lse2, dloss, b)
    assert torch.equal(dx, dx2) and torch.equal(a, b)


def test_the_same_index_twice_and_absent_entries(torch):
    from paper_1805_07891_amd import layers
    x, w, _, _ = _inputs(torch, 6, 48, 200, torch.float32)
    index = torch.tensor([[3, 3, 9], [5, -1, 5], [-1, -7, 200], [7, 8, 7], [199, 0, 199], [1, 2, 3]],
                         device="cuda")
    logits = torch.tensor([[1.0, 1.0, 0.0], [0.5, 9.0, 0.5], [1.0, 2.0, 3.0],
                           [-math.inf, 2.0, 1.0], [-math.inf, -math.inf, -math.inf],
                           [30.0, -90.0, 0.0]], device="cuda")
    d = _definition(torch, x, w, index, logits, 2.0, None)
    assert d["live"].tolist() == [True, True, False, True, False, True]
    loss, lse = layers.distill_loss(x, w, index, logits, 2.0)
    _check_loss(d, loss, lse)
    dw = torch.empty(200, 48, device="cuda")
    dx = layers.distill_loss_grad(x, w, index, logits, 2.0, lse, None, dw)
    _check_grad(torch, d, dx, dw, torch.float32)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_pieces_of_the_vocabulary(torch, dtype):
    """Any workspace from the least to the best gives results within the same
    bounds, and never touches what lies behind it."""
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    rows, cols, vocab = 150, 96, 1900
    x, w, target, dloss = _inputs(torch, rows, cols, vocab, dtype)
    d = _definition(torch, x, w, target, None, 1.0, dloss)
    lib = layers.load_library()
    sizes = layers._sizes(x, w)
    for grad in (False, True):
        least, best = lib.phub_vocab_bytes(*sizes, 0, int(grad))
        for n in sorted({least, (2 * least + best) // 3, (least + best) // 2, best}):
            space = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
            if not grad:
                loss, lse = layers.vocab_loss(x, w, target, workspace=space[:n])
                _check_loss(d, loss, lse)
            else:
                dw = torch.full((vocab, cols), 7.0, device="cuda")
                dx = layers.vocab_loss_grad(x, w, target, lse, dloss, dw, workspace=space[:n])
                _check_grad(torch, d, dx, dw, dtype, pieces=8)
            assert bool((space[n:] == 0x5a).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_strides_alignment_and_what_lies_between_rows(torch, dtype):
    from paper_1805_07891_amd import layers, phub
    dtype = getattr(torch, dtype)
    for rows, cols, vocab, gap, shift in ((70, 64, 300, 8, 8), (33, 65, 200, 7, 3), (20, 128, 130, 4, 1)):
        x0, w0, target, dloss = _inputs(torch, rows, cols, vocab, dtype)
        x = torch.full((rows, cols + gap + shift), math.nan, dtype=dtype, device="cuda")[:, shift:shift + cols]
        w = torch.full((vocab, cols + gap + shift), math.nan, dtype=dtype, device="cuda")[:, shift:shift + cols]
        x.copy_(x0)
        w.copy_(w0)
        d = _definition(torch, x, w, target, None, 1.0, dloss)
        loss, lse = layers.vocab_loss(x, w, target)
        _check_loss(d, loss, lse)
        dwb = torch.full((vocab, cols + gap), 7.0, device="cuda")
        dxb = torch.full((rows, cols + gap), 7.0, dtype=dtype, device="cuda")
        lib, space = layers.load_library(), layers.vocab_workspace(x, w)
        lib.phub_vocab_loss_grad(*layers._sizes(x, w), target.data_ptr(), lse.data_ptr(),
                                 dloss.data_ptr(), dxb.data_ptr(), cols + gap, dwb.data_ptr(),
                                 cols + gap, 0, space.data_ptr(), space.numel(),
                                 torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        _check_grad(torch, d, dxb[:, :cols], dwb[:, :cols], dtype)
        assert bool((dwb[:, cols:] == 7.0).all()) and bool((dxb[:, cols:] == 7.0).all())
    assert phub.PHUB_BF16 == 1


def test_accumulate_either_gradient_alone_and_repeats(torch):
    from paper_1805_07891_amd import layers
    x, w, target, dloss = _inputs(torch, 200, 80, 1200, torch.bfloat16)
    loss, lse = layers.vocab_loss(x, w, target)
    dw = torch.empty(1200, 80, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, dloss, dw)
    again = torch.empty_like(dw)
    assert layers.vocab_loss_grad(x, w, target, lse, dloss, again, want_dx=False) is None
    assert torch.equal(again, dw)
    assert torch.equal(layers.vocab_loss_grad(x, w, target, lse, dloss), dx)
    summed = torch.full_like(dw, 0.5)
    layers.vocab_loss_grad(x, w, target, lse, dloss, summed, accumulate=True)
    assert torch.equal(summed, dw + 0.5)
    l2, _ = layers.vocab_loss(x, w, target)
    assert torch.equal(loss, l2)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows, cols, vocab, top", [(5, 40, 300, 0), (1100, 96, 4100, 0),
                                                    (2100, 72, 8200, 0), (1100, 64, 4100, 33)])
def test_either_gradient_alone_has_the_same_bits(torch, rows, cols, vocab, top, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, w, *target, dloss = _inputs(torch, rows, cols, vocab, dtype, top)
    loss = layers.distill_loss if top else layers.vocab_loss
    grad = layers.distill_loss_grad if top else layers.vocab_loss_grad
    args = (*target, 2.0) if top else target
    _, lse = loss(x, w, *args)
    dw, alone = torch.empty(vocab, cols, device="cuda"), torch.empty(vocab, cols, device="cuda")
    dx = grad(x, w, *args, lse, dloss, dw)
    assert grad(x, w, *args, lse, dloss, alone, want_dx=False) is None
    assert torch.equal(alone, dw)
    assert torch.equal(grad(x, w, *args, lse, dloss), dx)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_pieces_of_the_vocabulary_with_a_teacher(torch, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    rows, cols, vocab, top, t = 130, 72, 1500, 21, 1.5
    x, w, index, logits, dloss = _inputs(torch, rows, cols, vocab, dtype, top)
    d = _definition(torch, x, w, index, logits, t, dloss)
    for most in (0, 1 << 20, None):
        space = layers.vocab_workspace(x, w, top, most=most)
        loss, lse = layers.distill_loss(x, w, index, logits, t, workspace=space)
        _check_loss(d, loss, lse)
        dw = torch.full((vocab, cols), 7.0, device="cuda")
        dx = layers.distill_loss_grad(x, w, index, logits, t, lse, dloss, dw, workspace=space)
        _check_grad(torch, d, dx, dw, dtype, pieces=8)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_many_rows_few_entries_and_accumulation(torch, dtype):
    """The weights' gradient in parts over the rows, added to what is there."""
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, w, target, dloss = _inputs(torch, 5000, 64, 100, dtype)
    d = _definition(torch, x, w, target, None, 1.0, dloss)
    loss, lse = layers.vocab_loss(x, w, target)
    _check_loss(d, loss, lse)
    dw = torch.full((100, 64), 7.0, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, dloss, dw)
    _check_grad(torch, d, dx, dw, dtype)
    twice = dw.clone()
    layers.vocab_loss_grad(x, w, target, lse, dloss, twice, accumulate=True)
    assert torch.equal(twice, dw + dw)


def test_a_teachers_largest_logits(torch):
    """Logits near the ends of fp32, which no temperature may carry beyond them."""
    from paper_1805_07891_amd import layers
    x, w, _, _ = _inputs(torch, 4, 48, 200, torch.float32)
    index = torch.tensor([[3, 4], [5, 6], [7, -1], [8, 9]], device="cuda")
    logits = torch.tensor([[3e38, 3e38], [-3e38, 3e38], [-3e38, 1.0], [-3e38, -3e38]], device="cuda")
    for t in (1e-3, 0.5, 2.0):
        # the same distributions from logits of ordinary size
        plain = torch.tensor([[0.0, 0.0], [-1e4, 0.0], [0.0, 0.0], [0.0, 0.0]], device="cuda")
        d = _definition(torch, x, w, index, plain, t, None)
        loss, lse = layers.distill_loss(x, w, index, logits, t)
        _check_loss(d, loss, lse)
        dw = torch.empty(200, 48, device="cuda")
        dx = layers.distill_loss_grad(x, w, index, logits, t, lse, None, dw)
        _check_grad(torch, d, dx, dw, torch.float32)


def test_no_live_rows_and_no_rows(torch):
    from paper_1805_07891_amd import layers
    x, w, target, dloss = _inputs(torch, 40, 64, 300, torch.bfloat16)
    x.fill_(math.nan)
    target.fill_(-1)
    loss, lse = layers.vocab_loss(x, w, target)
    assert not loss.any()
    dw = torch.full((300, 64), 7.0, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, dloss, dw)
    assert not dx.any() and not dw.any()
    dw.fill_(7.0)
    e = torch.empty(0, device="cuda")
    layers.vocab_loss_grad(x[:0], w, target[:0], e, None, dw, accumulate=True)
    assert bool((dw == 7.0).all())
    dx = layers.vocab_loss_grad(x[:0], w, target[:0], e, None, dw)
    assert dx.shape == (0, 64) and not dw.any()
    loss, lse = layers.vocab_loss(x[:0], w, target[:0])
    assert loss.shape == (0,)


def test_rows_of_unequal_size_and_zero_weights_of_rows(torch):
    """Hidden states over many powers of two, rows' gradients from 1e-6 to 1e4
    and zeros: each gradient within its bound."""
    from paper_1805_07891_amd import layers
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        x, w, target, dloss = _inputs(torch, 120, 64, 500, dtype)
        scale = 2.0 ** torch.randint(-6, 4, (120, 1), device="cuda",
                                     generator=torch.Generator(device="cuda").manual_seed(5))
        x = (x.float() * scale).to(dtype)
        x[8] = 0.0
        w[3] = 0.0
        dloss = dloss * 10.0 ** torch.linspace(-6, 1, 120, device="cuda")
        dloss[5::11] = 0.0
        d = _definition(torch, x, w, target, None, 1.0, dloss)
        loss, lse = layers.vocab_loss(x, w, target)
        _check_loss(d, loss, lse)
        dw = torch.empty(500, 64, device="cuda")
        dx = layers.vocab_loss_grad(x, w, target, lse, dloss, dw)
        _check_grad(torch, d, dx, dw, dtype)


def test_a_live_row_that_is_not_finite_shows(torch):
    from paper_1805_07891_amd import layers
    x, w, target, _ = _inputs(torch, 30, 64, 300, torch.float32)
    x[4, 7] = math.nan
    loss, lse = layers.vocab_loss(x, w, target)
    bad = loss.isnan()
    assert bad.nonzero()[:, 0].tolist() == [4]
    dw = torch.empty(300, 64, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, None, dw)
    assert bool(dx[4].isnan().all()) and bool(dx[:4].isfinite().all()) and bool(dw.isnan().all())


def test_gradient_against_differences(torch):
    """(loss(a + e d) - loss(a - e d)) / 2e in 64 bits against the fp32 gradients."""
    from paper_1805_07891_amd import layers
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w, index, logits, dloss = _inputs(torch, 24, 40, 90, torch.float32, top=6)
    _, lse = layers.distill_loss(x, w, index, logits, 2.0)
    dw = torch.empty(90, 40, device="cuda")
    dx = layers.distill_loss_grad(x, w, index, logits, 2.0, lse, dloss, dw)

    def loss(x, w):
        return (_definition(torch, x, w, index, logits, 2.0, dloss)["loss"] * dloss.double()).sum()

    e = 1e-4
    for grad, a, b in ((dx, x, w), (dw, w, x)):
        a, b = a.double(), b.double()
        d = torch.randn(a.shape, generator=g, device="cuda").double()
        pair = (lambda v: (v, b)) if grad is dx else (lambda v: (b, v))
        slope = (loss(*pair(a + e * d)) - loss(*pair(a - e * d))) / (2 * e)
        size = (grad.double() * d).abs().sum()
        assert abs(slope - (grad.double() * d).sum()) <= 1e-4 * size


def test_captured_and_replayed(torch):
    from paper_1805_07891_amd import layers
    for dtype in (torch.bfloat16, torch.float32):
        x, w, target, dloss = _inputs(torch, 200, 72, 900, dtype)
        space = layers.vocab_workspace(x, w)
        dw = torch.empty(900, 72, device="cuda")

        def passes():
            loss, lse = layers.vocab_loss(x, w, target, workspace=space)
            return loss, layers.vocab_loss_grad(x, w, target, lse, dloss, dw, workspace=space)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            passes()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            loss, dx = passes()
        for turn in range(3):
            nx, nw, nt, _ = _inputs(torch, 200, 72, 900, dtype, seed=20 + turn)
            x.copy_(nx)
            w.copy_(nw)
            target.copy_(nt)
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (loss, dx, dw)]
            el, edx = passes()
            torch.cuda.synchronize()
            for a, b in zip(got, (el, edx, dw)):
                assert torch.equal(a, b)


def test_two_graphs_share_a_workspace(torch):
    from paper_1805_07891_amd import layers
    first = _inputs(torch, 150, 72, 900, torch.float32)
    second = _inputs(torch, 90, 40, 700, torch.bfloat16, top=11, seed=2)
    space = layers.vocab_workspace(*first[:2])
    assert space.numel() >= layers.vocab_workspace(*second[:2], 11).numel()
    dws = [torch.empty(900, 72, device="cuda"), torch.empty(700, 40, device="cuda")]

    def cross_entropy():
        x, w, target, dloss = first
        loss, lse = layers.vocab_loss(x, w, target, workspace=space)
        return loss, layers.vocab_loss_grad(x, w, target, lse, dloss, dws[0], workspace=space), dws[0]

    def distill():
        x, w, index, logits, dloss = second
        loss, lse = layers.distill_loss(x, w, index, logits, 2.0, workspace=space)
        return loss, layers.distill_loss_grad(x, w, index, logits, 2.0, lse, dloss, dws[1],
                                              workspace=space), dws[1]

    want = [[t.clone() for t in run()] for run in (cross_entropy, distill)]
    graphs, got = [], []
    for run in (cross_entropy, distill):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(run())
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (0, 1)):
        for out in got:
            for t in out:
                t.fill_(7.0)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
        assert torch.equal(cross_entropy()[0], want[0][0])


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows, cols, vocab, top", [(1, 4096, 100, 0), (40, 2100, 200, 0),
                                                    (130, 6000, 500, 0), (33, 3000, 300, 20)])
def test_long_rows_of_few_tiles(torch, rows, cols, vocab, top, dtype):
    """The logits' sums in parts: right, and the same bits every time."""
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, w, *target, dloss = _inputs(torch, rows, cols, vocab, dtype, top)
    if rows == 1:
        target = [torch.full_like(target[0], 5)]
    loss = layers.distill_loss if top else layers.vocab_loss
    grad = layers.distill_loss_grad if top else layers.vocab_loss_grad
    args = (*target, 2.0) if top else target
    d = _definition(torch, x, w, target[0], target[1] if top else None, 2.0 if top else 1.0, dloss)
    first = None
    for _ in range(20):
        out, lse = loss(x, w, *args)
        dw = torch.full((vocab, cols), 7.0, device="cuda")
        dx = grad(x, w, *args, lse, dloss, dw)
        now = (out, lse, dx, dw)
        if first is None:
            first = now
            _check_loss(d, out, lse)
            _check_grad(torch, d, dx, dw, dtype)
        live = d["live"]
        assert torch.equal(lse[live], first[1][live])
        assert all(torch.equal(a, b) for a, b in zip(now[::2] + now[3:], first[::2] + first[3:]))


def test_two_streams_at_once(torch):
    from paper_1805_07891_amd import layers
    sets = [_inputs(torch, 300, 64, 2000, torch.bfloat16, seed=s) for s in (1, 2)]
    want = []
    for x, w, target, dloss in sets:
        loss, lse = layers.vocab_loss(x, w, target)
        dw = torch.empty(2000, 64, device="cuda")
        want.append((loss, layers.vocab_loss_grad(x, w, target, lse, dloss, dw), dw))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], []
    for (x, w, target, dloss), s in zip(sets, streams):
        with torch.cuda.stream(s):
            loss, lse = layers.vocab_loss(x, w, target)
            dw = torch.empty(2000, 64, device="cuda")
            got.append((loss, layers.vocab_loss_grad(x, w, target, lse, dloss, dw), dw))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_offsets_beyond_32_bits(torch):
    """Weights and their gradient of more than 2^32 bytes and elements."""
    from paper_1805_07891_amd import layers
    rows, cols, vocab = 3, 4096, 1_100_000
    w = torch.empty(vocab, cols, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02)
    x = torch.randn(rows, cols, device="cuda").to(torch.bfloat16)
    target = torch.tensor([vocab - 1, 5, 600_000], device="cuda")
    loss, lse = layers.vocab_loss(x, w, target)
    dw = torch.full((vocab, cols), 7.0, device="cuda")
    dx = layers.vocab_loss_grad(x, w, target, lse, None, dw)
    torch.cuda.synchronize()
    z = torch.cat([x.double() @ c.double().t() for c in w.split(100_000)], 1)
    want = torch.logsumexp(z, 1)
    assert bool(((lse.double() - want).abs() <= 1e-4).all())
    assert bool((loss.double() - (want - z.gather(1, target[:, None])[:, 0])).abs().max() <= 1e-4)
    G = torch.exp(z - want[:, None])
    G[torch.arange(3), target] -= 1.0
    want_dx = sum(g @ c.double() for g, c in zip(G.split(100_000, 1), w.split(100_000)))
    assert bool((dx.double() - want_dx).norm() <= 2.0 ** -7 * want_dx.norm())
    for v in (0, 5, 600_000, 1_048_575, 1_048_576, vocab - 1):
        e = G[:, v] @ x.double()
        # p is right to 1e-4 of itself
        assert bool(((dw[v].double() - e).abs() <= 2e-4 * (G[:, v].abs() @ x.double().abs()) + 1e-12).all())


def test_the_binding_refuses(torch):
    from paper_1805_07891_amd import layers, phub
    x, w, target, dloss = _inputs(torch, 20, 64, 100, torch.bfloat16)
    loss, lse = layers.vocab_loss(x, w, target)
    index, logits = target[:, None].contiguous(), torch.zeros(20, 1, device="cuda")
    for bad in (lambda: layers.vocab_loss(x, w[:, :60], target), lambda: layers.vocab_loss(x, w.float(), target),
                lambda: layers.vocab_loss(x, w, target.int()), lambda: layers.vocab_loss(x, w, target[:5]),
                lambda: layers.vocab_loss(x, w.cpu(), target), lambda: layers.vocab_loss(x.t(), w, target),
                lambda: layers.vocab_loss_grad(x, w, target, lse, dloss.double()),
                lambda: layers.vocab_loss_grad(x, w, target, lse, dloss, torch.empty(100, 64, device="cuda").half()),
                lambda: layers.vocab_loss(x, w, target, workspace=torch.empty(9, device="cuda")),
                lambda: layers.distill_loss(x, w, index, logits.double()),
                lambda: layers.distill_loss(x, w, index[:3], logits)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(phub.PhubError):
        layers.vocab_loss(x, w, target, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(phub.PhubError):
        layers.distill_loss(x, w, index, logits, 0.0)
