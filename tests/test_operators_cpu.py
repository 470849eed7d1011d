"""The language-model operators' host side, without a GPU."""
import ctypes

import pytest

from paper_2102_02888_amd import _native


@pytest.fixture(scope="module")
def lib():
    return _native.lib()


def _workspace(lib, tokens, vocab, width):
    n = ctypes.c_size_t()
    assert lib.onebit_embedding_grad_workspace(tokens, vocab, width, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("vocab", [1, 30522])
def test_gradient_workspace_serves_every_shorter_and_narrower_call(lib, vocab):
    """The size for (tokens, width) covers every call of at most as many tokens and
    columns: it falls nowhere as either grows.  Looked at around every number of
    tokens and of columns where the pieces of the list may change their length."""
    widths = sorted({max(1, (1 << e) + d) for e in range(0, 15) for d in (-8, -5, -1, 0, 1, 4, 9)} |
                    {768, 771, 1016, 1020, 3000})
    tokens = {0, 1, 131072, 130000}
    for e in range(3, 24):
        tokens |= {(1 << e) + d for d in (-129, -16, -8, -1, 0, 1, 7, 128)}
    for w in (96, 193, 771, 1000):  # threads of a row that are no power of two
        for piece in (8, 16, 32, 64):
            first = -(-(1 << 18) // w) * 2 * piece
            tokens |= {first - 1, first, first + 1}
    tokens = sorted(t for t in tokens if t >= 0)
    below = [0] * len(tokens)  # the largest size of any narrower call, by tokens
    for w in widths:
        most = 0
        for k, t in enumerate(tokens):
            size = _workspace(lib, t, vocab, w)
            assert size >= most, (t, w)
            assert size >= below[k], (t, w)
            most, below[k] = size, size
