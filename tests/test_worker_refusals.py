"""Argument checks of the worker's operators (CPU: a refused call returns its
code and a message before it touches the GPU; the pointers are made up)."""

import os

import pytest

from paper_1805_07891_amd import phub

P = 1 << 20  # a pointer that no accepted call reaches the GPU with


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(phub.DEFAULT_LIB):
        from paper_1805_07891_amd import build
        build.build()
    return phub.load()


def _refused(lib, call, args, word):
    assert call(*args, check=False) == phub.PHUB_EINVAL
    assert word in lib.last_error()


NORM = dict(type=0, rows=4, cols=8, x=P, xs=8, w=P, b=P, eps=1e-5, y=P, ys=8, mean=P, rstd=P,
            stream=None)


@pytest.mark.parametrize("change, word", [
    (dict(type=3), "type"), (dict(type=-1), "type"), (dict(rows=-1), "rows"),
    (dict(rows=1 << 30), "rows"), (dict(cols=0), "cols"), (dict(cols=(1 << 20) + 1), "cols"),
    (dict(x=None), "x is NULL"), (dict(x=P + 2), "aligned"), (dict(type=1, x=P + 1), "aligned"),
    (dict(xs=7), "apart"), (dict(ys=7), "apart"), (dict(y=None), "y is NULL"),
    (dict(w=P + 1), "weight"), (dict(b=P + 2), "bias"), (dict(mean=P + 2), "mean"),
    (dict(rstd=P + 2), "rstd"), (dict(eps=-1e-5), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps")])
def test_layer_norm_refuses(lib, change, word):
    _refused(lib, lib.phub_layer_norm, {**NORM, **change}.values(), word)


NORM_GRAD = dict(type=0, rows=4, cols=8, dy=P, dys=8, x=P, xs=8, w=P, mean=P, rstd=P, dx=P, dxs=8,
                 dw=P, db=P, acc=0, ws=P, n=1 << 20, stream=None)


@pytest.mark.parametrize("change, word", [
    (dict(type=9), "type"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"),
    (dict(dy=None), "dy is NULL"), (dict(dys=3), "dy"), (dict(x=None), "x is NULL"),
    (dict(xs=0), "apart"), (dict(mean=None), "mean is NULL"), (dict(rstd=None), "rstd is NULL"),
    (dict(dx=P + 1), "dx"), (dict(dxs=7), "dx"), (dict(dw=P + 1), "dweight"),
    (dict(db=P + 3), "dbias"), (dict(ws=None), "workspace is NULL"), (dict(ws=P + 16), "workspace"),
    (dict(n=2 * 4 * 8 * 4 - 1), "bytes")])
def test_layer_norm_grad_refuses(lib, change, word):
    _refused(lib, lib.phub_layer_norm_grad, {**NORM_GRAD, **change}.values(), word)


def test_nothing_wanted_or_no_rows_needs_no_pointers(lib):
    none = {**NORM_GRAD, **dict(dx=None, dw=None, db=None, ws=None, n=0)}
    assert lib.phub_layer_norm_grad(*none.values()) == 0
    assert lib.phub_layer_norm(*{**NORM, **dict(rows=0, x=None, y=None)}.values()) == 0
    assert lib.phub_vocab_loss(*{**LOSS, **dict(rows=0, x=None, w=None, target=None, loss=None,
                                                lse=None, ws=None, n=0)}.values()) == 0
    assert lib.phub_vocab_loss_grad(*{**LOSS_GRAD, **dict(dx=None, dw=None, ws=None,
                                                          n=0)}.values()) == 0


LOSS = dict(type=0, rows=4, cols=8, vocab=10, x=P, xs=8, w=P, ws_=8, target=P, loss=P, lse=P, ws=P,
            n=1 << 30, stream=None)


@pytest.mark.parametrize("change, word", [
    (dict(type=3), "type"), (dict(rows=-1), "rows"), (dict(rows=(1 << 21) + 1), "rows"),
    (dict(cols=0), "cols"), (dict(cols=(1 << 16) + 1), "cols"), (dict(vocab=0), "vocab"),
    (dict(vocab=(1 << 24) + 1), "vocab"), (dict(x=None), "x is NULL"), (dict(x=P + 1), "x"),
    (dict(xs=7), "x"), (dict(xs=(1 << 21) + 1), "x"), (dict(w=None), "w is NULL"),
    (dict(ws_=7), "w"), (dict(target=None), "target"), (dict(target=P + 4), "target"),
    (dict(loss=None), "loss"), (dict(lse=P + 2), "lse"), (dict(ws=None), "workspace"),
    (dict(ws=P + 128), "workspace"), (dict(n=1000), "needed")])
def test_vocab_loss_refuses(lib, change, word):
    _refused(lib, lib.phub_vocab_loss, {**LOSS, **change}.values(), word)


LOSS_GRAD = dict(type=0, rows=4, cols=8, vocab=10, x=P, xs=8, w=P, ws_=8, target=P, lse=P, dloss=P,
                 dx=P, dxs=8, dw=P, dws=8, acc=0, ws=P, n=1 << 30, stream=None)


@pytest.mark.parametrize("change, word", [
    (dict(type=3), "type"), (dict(vocab=-5), "vocab"), (dict(lse=None), "lse"),
    (dict(dloss=P + 2), "dloss"), (dict(dx=P + 1), "dx"), (dict(dxs=4), "dx"),
    (dict(dw=P + 2), "dw"), (dict(dws=7), "dw"), (dict(ws=P + 8), "workspace"),
    (dict(n=0), "needed")])
def test_vocab_loss_grad_refuses(lib, change, word):
    _refused(lib, lib.phub_vocab_loss_grad, {**LOSS_GRAD, **change}.values(), word)


DISTILL = dict(type=0, rows=4, cols=8, vocab=10, x=P, xs=8, w=P, ws_=8, top=3, index=P, logit=P,
               t=2.0, loss=P, lse=P, ws=P, n=1 << 30, stream=None)
DISTILL_GRAD = dict(type=0, rows=4, cols=8, vocab=10, x=P, xs=8, w=P, ws_=8, top=3, index=P, logit=P,
                    t=2.0, lse=P, dloss=P, dx=P, dxs=8, dw=P, dws=8, acc=0, ws=P, n=1 << 30,
                    stream=None)


@pytest.mark.parametrize("change, word", [
    (dict(top=0), "top"), (dict(top=1025), "top"), (dict(index=None), "index"),
    (dict(logit=None), "logit"), (dict(logit=P + 2), "logit"), (dict(t=0.0), "temperature"),
    (dict(t=-1.0), "temperature"), (dict(t=float("nan")), "temperature"),
    (dict(t=float("inf")), "temperature"), (dict(t=1e-7), "temperature"),
    (dict(t=1e7), "temperature"), (dict(rows=(1 << 20) + 1, top=1024), "entries"),
    (dict(n=1000), "needed")])
def test_distill_refuses(lib, change, word):
    _refused(lib, lib.phub_distill_loss, {**DISTILL, **change}.values(), word)
    _refused(lib, lib.phub_distill_loss_grad, {**DISTILL_GRAD, **change}.values(), word)


def test_workspace_sizes(lib):
    sizes = (1, 512, 256, 5000, P, 256, P, 256)
    least, best = lib.phub_vocab_bytes(*sizes, 0, 1)
    assert 0 < least < best and best % 256 == 0 and least % 256 == 0
    # an odd width and fp32 need room for copies; entries of a teacher too
    assert lib.phub_vocab_bytes(1, 512, 255, 5000, P, 256, P, 256, 0, 0) > \
        lib.phub_vocab_bytes(*sizes, 0, 0)
    assert lib.phub_vocab_bytes(*sizes, 64, 1)[0] > least
    for bad in ((4, 512, 256, 5000, P, 256, P, 256, 0, 1), (1, -1, 256, 5000, P, 256, P, 256, 0, 1),
                (1, 512, 256, 5000, P, 256, P, 256, 2000, 1)):
        with pytest.raises(phub.PhubError):
            lib.phub_vocab_bytes(*bad)
    assert lib.phub_vocab_bytes(1, 0, 256, 5000, P, 256, P, 256, 0, 1) == (0, 0)
    assert lib.phub_layer_norm_grad_bytes(3, 100) == 2 * 3 * 100 * 4
    with pytest.raises(phub.PhubError):
        lib.phub_layer_norm_grad_bytes(3, 0)
