"""Sizes of the layers' workspaces at the largest arguments, without a GPU."""
import ctypes

import pytest

from paper_2412_18052_b200 import binding
from paper_2412_18052_b200.build import build

MOST = (1 << 31) - 65           # largest number of tokens, columns, rows
OK, TOO_LARGE = 0, 8
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def L():
    build()
    return binding.lib()


def test_no_size_wraps_around(L):
    """A workspace is never smaller than one for less; what no 64-bit number of bytes holds is refused."""
    out = ctypes.c_size_t()
    for dtype, terms in ((F32, 3), (BF16, 1)):
        for V in (0, MOST):
            sizes = {}
            for T in (1, 1000, 1 << 20, 1 << 26, 1 << 29, 1 << 30, MOST):
                for width in (1, 1000, 1 << 20, 1 << 26, 1 << 29, 1 << 30, MOST):
                    rc = L.gaf_layer_workspace_bytes(T, width, V, dtype, ctypes.byref(out))
                    rows = terms * ((T + 127) // 128 * 128) * ((width + 7) // 8 * 8) * 2       # dy laid out anew: the largest part of it
                    assert rc == (OK if rows < 1 << 63 else TOO_LARGE), (T, width)
                    if rc == OK:
                        assert out.value >= rows
                        sizes[T, width] = out.value
            assert all(sizes[a] <= sizes[b] for a in sizes for b in sizes if a[0] <= b[0] and a[1] <= b[1])
