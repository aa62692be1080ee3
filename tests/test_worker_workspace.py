"""Workspace sizes of the losses over a vocabulary (CPU: phub_vocab_bytes only)."""

import os
import random

import pytest

from paper_1805_07891_amd import phub

P = 1 << 20  # only its alignment counts


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(phub.DEFAULT_LIB):
        from paper_1805_07891_amd import build
        build.build()
    return phub.load()


def _bytes(lib, kind, rows, cols, vocab, top, grad):
    return lib.phub_vocab_bytes(kind, rows, cols, vocab, P, cols, P, cols, top, grad)


def test_a_loss_alone_needs_little(lib):
    # a row leaves at most two fp32 values for each 32 entries of a piece, besides its logit
    # and what pieces before it came to
    least, best = _bytes(lib, phub.PHUB_BF16, 4096, 4096, 131072, 0, 0)
    assert least <= 4096 * (8 * 256 // 32 + 8 + 4) + 1024
    # and in tiles of 256 two for each 128
    assert least < best <= 4096 * (8 * 131072 // 128 + 8 + 4) + 1024
    least, best = _bytes(lib, phub.PHUB_BF16, 5, 4096, 32768, 0, 0)
    assert least <= best <= 5 * (8 * 32768 // 32 + 4) + 1024


def test_one_workspace_serves_both_passes(lib):
    rng = random.Random(1)
    for _ in range(300):
        spread = lambda n: int(n ** rng.random())  # noqa: E731
        kind, top = rng.randrange(3), rng.choice([0, 0, 1, 33, 1024])
        rows, cols, vocab = spread(1 << 20), spread(1 << 16), spread(1 << 24)
        forward = _bytes(lib, kind, rows, cols, vocab, top, 0)
        backward = _bytes(lib, kind, rows, cols, vocab, top, 1)
        what = (kind, rows, cols, vocab, top)
        assert 0 < forward[0] <= forward[1] and 0 < backward[0] <= backward[1], what
        assert forward[0] <= backward[0], what
        assert all(n % 256 == 0 for n in forward + backward), what


def test_the_largest_sizes_fit_a_gpu(lib):
    for kind in (phub.PHUB_F32, phub.PHUB_BF16):
        for top in (0, 32):
            least, _ = _bytes(lib, kind, 1 << 21, 4096, 1 << 24, top, 0)
            assert least < 64 << 30
