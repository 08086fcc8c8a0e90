"""Calls that the paged cache's entry points refuse, as far as they can be told without a device: nothing is launched and
no pointer followed before the arguments have passed."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2508_17892_b200 import build, recall
    build.build()
    return recall.load_library()


def _shares(a, b, n, row_a, row_b):
    """Do n rows at a = (address, stride) and at b share a byte?  By counting, strides and rows in elements of 2 bytes."""
    cells = lambda p, s, r: {p + 2 * (i * s + j) for i in range(n) for j in range(r)}  # noqa: E731
    return bool(cells(*a, row_a) & cells(*b, row_b))


@pytest.mark.skipif(torch.cuda.is_available(), reason="what is not refused would be launched on these addresses")
def test_rope_refuses_rows_that_are_read_and_written(lib):
    """Rows of 16 elements at every distance on both sides, slices of one tensor among them; -6 (no device) is what a call
    gets that has passed."""
    from paper_2508_17892_b200.paged import IlreRopeSpec
    spec = IlreRopeSpec(10000.0, 16, 0, 0, 1.0, 0.0, 0.0, 0.0, 0.0)
    x = 1 << 20
    passed = set()
    for n, xs, os_ in ((1, 16, 16), (1, 16, 48), (2, 16, 16), (3, 48, 48), (4, 56, 56), (3, 16, 48), (4, 48, 16)):
        for step in range(-40, 41):
            out = x + 16 * step
            code = lib.ilre_rope(ctypes.byref(spec), x, xs, out, os_, 4096, n, 1, 16, 0, 0, None)
            shared = _shares((x, xs), (out, os_), n, 16, 16)
            if out == x:
                assert (code == -1) == (n > 1 and xs != os_)
            elif xs == os_ or n == 1:
                assert (code == -1) == shared, (n, xs, step)
            else:                                            # two strides: refused where the spans meet
                assert code == -1 or not shared
                assert code != -1 or -((n - 1) * os_ + 16) * 2 < out - x < ((n - 1) * xs + 16) * 2
            if code != -1:
                passed.add(code)
    assert passed == {-6}
