"""The language-model operators' host side, without a GPU."""
import ctypes
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2102_02888_amd import _native
from paper_2102_02888_amd.build import LIB
from paper_2102_02888_amd.muon import PRODUCTS_F16, PRODUCTS_F32, matrices_kernels
from matrix_lists import KERNEL_LISTS

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


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


def _kernels(tmp_path):
    """{kernel symbol: its instructions} of the built library's gfx950 code."""
    shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True,
                   stdout=subprocess.DEVNULL)
    out = {}
    for part in glob.glob(str(tmp_path / "lib.so.*gfx950")):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part], check=True,
                              stdout=subprocess.PIPE, text=True).stdout
        for line in text.splitlines():
            name = re.match(r"[0-9a-f]+ <(.*)>:$", line)
            if name:
                now = out.setdefault(name.group(1), [])
            elif line.startswith("\t"):
                now.append(line.split("//")[0].strip())
    return out


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler for the built kernels")
def test_every_wave_waits_for_its_stores_before_a_workgroup_publishes_them(tmp_path):
    """Where one thread releases a whole workgroup's sums to other workgroups (the
    write-back of the L2, then the counter's increment), every wave has to have
    waited for its own stores before the barrier that the thread comes from, which
    does not wait for them by itself; the thread has to wait for the write-back
    before it counts, and for the count before it discards what its caches hold."""
    found = 0

    def waits(code):
        return any(l.startswith("s_waitcnt") and "vmcnt(0)" in l for l in code)

    for name, code in _kernels(tmp_path).items():
        for k, line in enumerate(code):
            if not line.startswith("buffer_wbl2"):
                continue
            found += 1
            barrier = max(i for i in range(k) if code[i].startswith("s_barrier"))
            store = max(i for i in range(barrier) if "global_store" in code[i])
            count = min(i for i in range(k, len(code)) if "atomic_add" in code[i])
            discard = min(i for i in range(count, len(code)) if code[i].startswith("buffer_inv"))
            after = min(i for i in range(count, len(code)) if code[i].startswith("s_barrier"))
            assert waits(code[store:barrier]), (name, code[store:barrier + 1])
            assert waits(code[k:count]), (name, code[k:count + 1])
            assert waits(code[count:discard]) and discard < after, (name, code[count:after + 1])
    assert found  # the parts of a Gram sum


def test_tested_lists_take_every_kernel():
    """Each product (the last one is next's other epilogue) by each of the four
    kernels, for both kinds of products; and sums in parts, for both."""
    want = {(name, kernel) for name in ("gram", "poly", "next")
            for kernel in ((64, 2), (64, 4), (128, 1), (256, 1))}
    for products, at in ((PRODUCTS_F32, 1), (PRODUCTS_F16, 2)):
        seen, parts = set(), 0
        for case, entry in KERNEL_LISTS.items():
            got = matrices_kernels(entry[0], products)
            assert got == entry[at], case
            parts = max(parts, got.pop("parts"))
            seen |= set(got.items())
        assert seen == want and parts > 1


def test_matrices_kernels_refusals_and_empty_lists(lib):
    empty = dict(gram=(0, 0), poly=(0, 0), next=(0, 0), parts=0)
    assert matrices_kernels([(0, 5), (7, 0)]) == empty
    one = (ctypes.c_int64 * 1)(4)
    assert lib.onebit_matrices_kernels(one, one, 1, 0, None, None, None) == 0
    assert lib.onebit_matrices_kernels(None, one, 1, 0, None, None, None) == -1
    assert lib.onebit_matrices_kernels(one, one, 0, 0, None, None, None) == -1
    assert lib.onebit_matrices_kernels(one, one, 1, 2, None, None, None) == -1
    for bad in ((-1, 4), (4, (1 << 20) + 1), (1 << 16, 1 << 16)):
        with pytest.raises(_native.OnebitError):
            matrices_kernels([(4, 4), bad])


def test_gradient_too_large_for_a_launch_is_refused_before_it(lib):
    """(The pointers are not read: nothing is launched.)"""
    for tokens, width, dtype in ((1 << 30, 257, 0), ((1 << 31) - 1, 1, 0), (1 << 29, 513, 1),
                                 (1, (1 << 31) - 1, 0)):
        assert lib.onebit_embedding_grad(4096, dtype, width, 4096, 4, tokens, 10, width, -1, 1.0,
                                         4096, 0, width, 0, 4096, None) == -1, (tokens, width)
        assert b"too many" in lib.onebit_last_error()
