"""Layer norm and its backward pass against 64 bits.

Bounds, with u = 2^-24 and t the type's half step: a mean or sum over a row
is at most 32 additions in a thread, 6 in a wave and 16 over waves, so wrong
by at most 56 u times the sum of magnitudes (rows beyond the registers: cols /
1024 more); everything after it is a handful of roundings.  Sums over rows
add at most rows / 256 + 72 terms in turn.
"""

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    return torch


def _half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def _inputs(torch, rows, cols, dtype, seed=1, affine=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = (r(rows, cols) * 2.0 + r(rows, 1)).to(dtype)
    dy = (r(rows, cols) * 0.1).to(dtype)
    return x, dy, (1.0 + 0.3 * r(cols) if affine else None), (0.2 * r(cols) if affine else None)


def _definition(torch, x, dy, weight, bias):
    x, dy = x.double(), dy.double()
    w = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + EPS)
    h = c * rstd[:, None]
    dh = dy * w
    dx = rstd[:, None] * (dh - dh.mean(1, keepdim=True) - h * (dh * h).mean(1, keepdim=True))
    return dict(y=h * w + b, mean=mean, rstd=rstd, dx=dx, dw=(dy * h).sum(0), db=dy.sum(0), h=h, w=w)


def _within(got, want, bound):
    off = (got.double() - want).abs()
    worst = (off / bound).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"{worst:.3g} times the bound"


def _check(torch, x, dy, weight, bias, got, d):
    rows, cols = x.shape
    t = _half_step(torch, x.dtype)
    n = 56 + cols / 1024
    m1 = x.double().abs().mean(1, keepdim=True)
    rstd = d["rstd"][:, None]
    # of h: the mean's error, that of x - mean, and rstd's (half its sum's, and 4 roundings)
    h_off = U * ((n + 2) * m1 * rstd + (n / 2 + 8) * d["h"].abs())
    _within(got["mean"], d["mean"], U * (n + 1) * m1[:, 0] + 1e-30)
    _within(got["rstd"], d["rstd"], U * (n / 2 + 6) * d["rstd"] + U * (n + 2) * m1[:, 0] * d["rstd"] ** 2)
    out = d["y"].abs()
    _within(got["y"], d["y"], t * out * 1.01 + h_off * d["w"].abs() + 4 * U * (out + (d["h"] * d["w"]).abs())
            + torch.finfo(x.dtype).tiny)
    if "dx" in got:
        dh = (dy.double() * d["w"]).abs()
        a, b = dh.mean(1, keepdim=True), (dh * d["h"].abs()).mean(1, keepdim=True)
        off = rstd * ((n + 4) * U * (dh + a + d["h"].abs() * b)
                      + d["h"].abs() * (dh * h_off).mean(1, keepdim=True) + h_off * b)
        off = off + d["dx"].abs() * (n / 2 + 8) * U
        _within(got["dx"], d["dx"], t * d["dx"].abs() * 1.01 + off + torch.finfo(x.dtype).tiny)
    k = rows / 256 + 72
    dya = dy.double().abs()
    if "dw" in got:
        _within(got["dw"], d["dw"], (k + 4) * U * (dya * d["h"].abs()).sum(0)
                + (dya * h_off).sum(0) + 1e-30)
    if "db" in got:
        _within(got["db"], d["db"], (k + 2) * U * dya.sum(0) + 1e-30)


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 64), (130, 100), (7, 513), (33, 1000), (600, 1001), (9, 2047),
          (64, 2048), (17, 4095), (5, 8192), (3, 8200), (4, 16384), (2, 16400), (3, 40001), (2000, 256)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_both_passes(torch, rows, cols, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    x, dy, w, b = _inputs(torch, rows, cols, dtype)
    print("layer norm", rows, cols, dtype, flush=True)
    y, mean, rstd = layers.layer_norm(x, w, b, EPS)
    dw, db = torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    dx = layers.layer_norm_grad(dy, x, w, mean, rstd, dw, db)
    _check(torch, x, dy, w, b, dict(y=y, mean=mean, rstd=rstd, dx=dx, dw=dw, db=db),
           _definition(torch, x, dy, w, b))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_offsets_and_no_weights(torch, dtype):
    from paper_1805_07891_amd import layers
    dtype = getattr(torch, dtype)
    for rows, cols in ((37, 130), (6, 3001), (3, 17000)):
        big, dyb, _, _ = _inputs(torch, rows + 1, cols + 11, dtype, seed=2)
        x, dy = big[1:, 3:3 + cols], dyb[1:, 5:5 + cols]
        y, mean, rstd = layers.layer_norm(x, None, None, EPS)
        dw = torch.zeros(cols + 1, device="cuda")[1:]
        dx = layers.layer_norm_grad(dy, x, None, mean, rstd, dw, None)
        _check(torch, x, dy, None, None, dict(y=y, mean=mean, rstd=rstd, dx=dx, dw=dw),
               _definition(torch, x, dy, None, None))


def test_rows_of_dx_and_y_keep_what_lies_between_them(torch):
    from paper_1805_07891_amd import layers, phub
    rows, cols, stride = 5, 77, 100
    x, dy, w, b = _inputs(torch, rows, cols, torch.float16)
    lib = layers.load_library()
    y = torch.full((rows, stride), 3.0, dtype=torch.float16, device="cuda")
    dx = torch.full((rows, stride), 3.0, dtype=torch.float16, device="cuda")
    stats = torch.empty(2, rows, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    lib.phub_layer_norm(phub.PHUB_F16, rows, cols, x.data_ptr(), cols, w.data_ptr(), b.data_ptr(), EPS,
                        y.data_ptr(), stride, stats[0].data_ptr(), stats[1].data_ptr(), st)
    lib.phub_layer_norm_grad(phub.PHUB_F16, rows, cols, dy.data_ptr(), cols, x.data_ptr(), cols,
                             w.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), dx.data_ptr(),
                             stride, None, None, 0, None, 0, st)
    d = _definition(torch, x, dy, w, b)
    _check(torch, x, dy, w, b, dict(y=y[:, :cols], mean=stats[0], rstd=stats[1], dx=dx[:, :cols]), d)
    assert bool((y[:, cols:] == 3.0).all()) and bool((dx[:, cols:] == 3.0).all())
    # statistics are not wanted: the same y
    y2 = torch.empty(rows, cols, dtype=torch.float16, device="cuda")
    lib.phub_layer_norm(phub.PHUB_F16, rows, cols, x.data_ptr(), cols, w.data_ptr(), b.data_ptr(), EPS,
                        y2.data_ptr(), cols, None, None, st)
    assert torch.equal(y2, y[:, :cols])


def test_accumulate_adds_and_parts_can_be_left_out(torch):
    from paper_1805_07891_amd import layers
    x, dy, w, b = _inputs(torch, 700, 300, torch.bfloat16)
    _, mean, rstd = layers.layer_norm(x, w, b, EPS)
    one_w, one_b = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    layers.layer_norm_grad(dy, x, w, mean, rstd, one_w, one_b)
    dw, db = torch.full((300,), 0.5, device="cuda"), torch.full((300,), -0.25, device="cuda")
    assert layers.layer_norm_grad(dy, x, w, mean, rstd, dw, db, accumulate=True, want_dx=False) is None
    assert torch.equal(dw, 0.5 + one_w) and torch.equal(db, -0.25 + one_b)
    only = torch.empty(300, device="cuda")
    layers.layer_norm_grad(dy, x, w, mean, rstd, None, only)
    assert torch.equal(only, one_b)


def test_no_rows(torch):
    from paper_1805_07891_amd import layers
    x = torch.empty(0, 50, device="cuda")
    y, mean, rstd = layers.layer_norm(x)
    assert y.shape == (0, 50) and mean.shape == (0,)
    dw, db = torch.ones(50, device="cuda"), torch.ones(50, device="cuda")
    layers.layer_norm_grad(x, x, None, mean, rstd, dw, db, accumulate=True)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    layers.layer_norm_grad(x, x, None, mean, rstd, dw, db)
    assert not dw.any() and not db.any()


def test_more_rows_than_one_launch_takes(torch):
    from paper_1805_07891_amd import layers
    for cols in (24, 5):
        x, dy, w, b = _inputs(torch, (1 << 20) + 77, cols, torch.bfloat16, seed=4)
        y, mean, rstd = layers.layer_norm(x, w, b, EPS)
        dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        dx = layers.layer_norm_grad(dy, x, w, mean, rstd, dw, db)
        d = _definition(torch, x, dy, w, b)
        _check(torch, x, dy, w, b, dict(y=y, mean=mean, rstd=rstd, dx=dx, dw=dw, db=db), d)


def test_a_row_of_one_value_and_large_offsets(torch):
    from paper_1805_07891_amd import layers
    x = torch.full((4, 1000), 1e4, device="cuda")
    x[1] += torch.arange(1000, device="cuda") * 0.01
    x[2] = 0.0
    x[3, 5] = float("nan")
    y, mean, rstd = layers.layer_norm(x, None, None, EPS)
    assert not y[2].any() and mean[2] == 0.0
    assert bool(y[3].isnan().all()) and bool(y[:3].isfinite().all())
    d = _definition(torch, x[:3], x[:3], None, None)
    # the mean is taken first and exactly enough: offsets cost u |x| rstd and no more
    _within(y[1], d["y"][1], U * 60 * 1e4 * d["rstd"][1])


def test_gradient_against_differences(torch):
    """(loss(x + e d) - loss(x - e d)) / 2e in 64 bits, loss = sum dy y."""
    from paper_1805_07891_amd import layers
    x, dy, w, b = _inputs(torch, 6, 90, torch.float32)
    _, mean, rstd = layers.layer_norm(x, w, b, EPS)
    dw, db = torch.empty(90, device="cuda"), torch.empty(90, device="cuda")
    dx = layers.layer_norm_grad(dy, x, w, mean, rstd, dw, db)
    g = torch.Generator(device="cuda").manual_seed(3)
    e = 1e-5

    def loss(x, w, b):
        c = x - x.mean(1, keepdim=True)
        return (dy.double() * (c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * w + b)).sum()

    args = [x.double(), w.double(), b.double()]
    for i, grad in enumerate((dx, dw, db)):
        d = torch.randn(args[i].shape, generator=g, device="cuda").double()
        up = [a + e * d if j == i else a for j, a in enumerate(args)]
        down = [a - e * d if j == i else a for j, a in enumerate(args)]
        slope = (loss(*up) - loss(*down)) / (2 * e)
        # e^2 of the third derivative, and the gradient's 1e-5 of the terms' size
        size = (grad.double() * d).abs().sum()
        assert abs(slope - (grad.double() * d).sum()) <= 1e-5 * size


def test_captured_and_replayed(torch):
    from paper_1805_07891_amd import layers
    x, dy, w, b = _inputs(torch, 300, 513, torch.bfloat16)
    dw, db = torch.empty(513, device="cuda"), torch.empty(513, device="cuda")

    def passes():
        y, mean, rstd = layers.layer_norm(x, w, b, EPS)
        return y, layers.layer_norm_grad(dy, x, w, mean, rstd, dw, db)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        passes()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = passes()
    for turn in range(3):
        nx, ndy, _, _ = _inputs(torch, 300, 513, torch.bfloat16, seed=10 + turn)
        x.copy_(nx)
        dy.copy_(ndy)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw, db)]
        ey, edx = passes()
        torch.cuda.synchronize()
        for a, b_ in zip(got, (ey, edx, dw, db)):
            assert torch.equal(a, b_)


def test_another_stream_and_refusals_of_the_binding(torch):
    from paper_1805_07891_amd import layers
    x, dy, w, b = _inputs(torch, 64, 128, torch.float32)
    y, mean, rstd = layers.layer_norm(x, w, b, EPS)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2, _, _ = layers.layer_norm(x, w, b, EPS)
    side.synchronize()
    assert torch.equal(y, y2)
    for bad in (lambda: layers.layer_norm(x.double()), lambda: layers.layer_norm(x.t()),
                lambda: layers.layer_norm(x[0]), lambda: layers.layer_norm(x.cpu()),
                lambda: layers.layer_norm(x, w[:5]), lambda: layers.layer_norm(x, w.double()),
                lambda: layers.layer_norm_grad(dy[:5], x, w, mean, rstd),
                lambda: layers.layer_norm_grad(dy.half(), x, w, mean, rstd),
                lambda: layers.layer_norm_grad(dy, x, w, mean, rstd, w[::2])):
        with pytest.raises(ValueError):
            bad()
