"""The host side of layer norm, attention and the losses, without a GPU: what their
entry points refuse (the pointers are not read), and their workspaces."""
import ctypes

import pytest

from paper_2102_02888_amd import _native

P = 4096  # an address, for arguments that are looked at but not read


@pytest.fixture(scope="module")
def lib():
    return _native.lib()


def _refused(lib, name, args, at, bad, status):
    for value in bad:
        given = list(args)
        given[at] = value
        assert getattr(lib, name)(*given) == status, (name, at, value)


def test_layer_norm_refusals(lib):
    fwd = [P, 0, 8, 5, 8, P, P, 0, 1e-5, P, 0, 8, None]
    for at, bad, status in ((0, [None], -1), (0, [P + 2], -2), (1, [3, -1], -1), (2, [7, 1 << 41], -1),
                            (3, [-1, 1 << 31], -1), (4, [-1, 16385], -1), (5, [P + 2], -2),
                            (6, [P + 1], -2), (7, [9], -1), (8, [-1.0, float("nan"), float("inf")], -1),
                            (9, [None], -1), (10, [4], -1), (11, [7], -1)):
        _refused(lib, "onebit_layer_norm_forward", fwd, at, bad, status)
    bwd = [P, 0, 8, P, 0, 8, 5, 8, P, 0, 1e-5, P, 8, P, P, 0, 0, P, None]
    for at, bad, status in ((0, [None], -1), (3, [None], -1), (4, [3], -1), (7, [16385], -1),
                            (11, [P + 2], -2), (12, [7], -1), (13, [P + 2], -2), (15, [7], -1),
                            (17, [None], -1), (17, [P + 8], -2)):
        _refused(lib, "onebit_layer_norm_grad", bwd, at, bad, status)
    # nothing to do: nothing is launched
    assert lib.onebit_layer_norm_forward(None, 0, 0, 0, 8, None, None, 0, 1e-5, None, 0, 0, None) == 0
    assert lib.onebit_layer_norm_forward(None, 0, 0, 5, 0, None, None, 0, 1e-5, None, 0, 0, None) == 0


def test_workspaces_serve_smaller_calls(lib):
    n = ctypes.c_size_t()
    for rows in (0, 1, 3, 700, 1024, 5000, 131072):
        for width in (0, 1, 64, 65, 1024, 1025, 16384):
            assert lib.onebit_layer_norm_grad_workspace(rows, width, ctypes.byref(n)) == 0
            most = n.value
            for r, w in ((rows // 2, width), (rows, width // 2), (max(rows - 1, 0), max(width - 1, 0))):
                assert lib.onebit_layer_norm_grad_workspace(r, w, ctypes.byref(n)) == 0
                assert n.value <= most
    assert lib.onebit_layer_norm_grad_workspace(5, 5, None) == -1
    assert lib.onebit_layer_norm_grad_workspace(-1, 5, ctypes.byref(n)) == -1
    assert lib.onebit_attention_grad_workspace(1 << 20, 64, ctypes.byref(n)) == 0
    assert n.value >= (1 << 26) * 4
    for tokens, heads in ((-1, 4), (4, 0), ((1 << 30) + 1, 4), (4, 1 << 15)):
        assert lib.onebit_attention_grad_workspace(tokens, heads, ctypes.byref(n)) == -1


def test_attention_refusals(lib):
    #      q  ld  k  ld  v  ld  type tokens heads kv dim starts seq causal scale out ld lse stream
    fwd = [P, 64, P, 32, P, 32, 1, 10, 4, 2, 16, P, 2, 1, 0.25, P, 64, P, None]
    for at, bad, status in ((0, [None], -1), (0, [P + 1], -2), (1, [63], -1), (3, [31], -1), (5, [31], -1),
                            (6, [0, 3, -1], -1), (7, [-1, (1 << 30) + 1], -1), (8, [0, 3, 1 << 15], -1),
                            (9, [0, 3, -1], -1), (10, [0, 129], -1), (11, [None], -1), (11, [P + 2], -2),
                            (12, [-1, (1 << 30) + 1, 1 << 24], -1), (14, [0.0, -1.0, float("nan")], -1),
                            (15, [None], -1), (16, [63], -1), (17, [P + 2], -2)):
        _refused(lib, "onebit_attention_forward", fwd, at, bad, status)
    bwd = [P, 64, P, 64, P, 32, P, 32, P, 64, P, 1, 10, 4, 2, 16, P, 2, 1, 0.25, P, 64, P, 32, P, 32, P, None]
    for at, bad, status in ((0, [None], -1), (8, [None], -1), (10, [None], -1), (10, [P + 2], -2),
                            (20, [None], -1), (21, [63], -1), (23, [31], -1), (24, [P + 1], -2),
                            (26, [None], -1), (26, [P + 8], -2)):
        _refused(lib, "onebit_attention_grad", bwd, at, bad, status)
    fwd[7] = 0
    assert lib.onebit_attention_forward(*fwd) == 0
    fwd[7], fwd[12] = 10, 0
    assert lib.onebit_attention_forward(*fwd) == 0


def test_loss_refusals(lib):
    fwd = [P, 0, 8, 5, 8, P, 8, 1.0, P, P, 3, P, P, None]
    for at, bad, status in ((0, [None], -1), (0, [P + 2], -2), (1, [3], -1), (2, [7], -1), (3, [-1, 1 << 31], -1),
                            (4, [-1, (1 << 30) + 1], -1), (5, [None], -1), (5, [P + 4], -2), (6, [2, 0], -1),
                            (7, [0.0, -1.0, float("nan"), float("inf")], -1), (8, [P + 2], -2), (9, [P + 1], -2),
                            (10, [-1, 65], -1), (11, [P + 4], -2), (12, [P + 2], -2)):
        _refused(lib, "onebit_logprobs_forward", fwd, at, bad, status)
    bwd = [P, 0, 8, 5, 8, P, 8, 1.0, P, P, P, 8, P, P, None]
    for at, bad, status in ((0, [None], -1), (5, [None], -1), (8, [P + 2], -2), (9, [P + 2], -2), (10, [None], -1),
                            (11, [7], -1), (12, [P + 2], -2), (13, [P + 2], -2)):
        _refused(lib, "onebit_logprobs_grad", bwd, at, bad, status)
    one = [P, 0, 8, 5, 8, P, 8, P, 0, 3, 3, 1.0, P, None]
    for at, bad, status in ((5, [None], -1), (6, [3], -1), (7, [None], -1), (8, [3], -1), (9, [2], -1),
                            (10, [0, 257], -1), (11, [0.0], -1), (12, [None], -1), (12, [P + 2], -2)):
        _refused(lib, "onebit_distill_forward", one, at, bad, status)
    two = [P, 0, 8, 5, 8, P, 8, P, 0, 3, 3, 1.0, P, P, 8, P, None]
    for at, bad, status in ((12, [None], -1), (13, [None], -1), (14, [7], -1), (15, [P + 2], -2)):
        _refused(lib, "onebit_distill_grad", two, at, bad, status)
    assert lib.onebit_logprobs_forward(None, 0, 0, 0, 8, None, 8, 1.0, None, None, 0, None, None, None) == 0
