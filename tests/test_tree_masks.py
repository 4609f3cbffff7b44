"""Which mask words the attention kernels read, and what they make of them (CPU:
the device code run on the host)."""
import ctypes

import numpy as np
import pytest

from oracle import spec_decode as S
from tests import _hip_host


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return _hip_host.compile_host("tree", tmp_path_factory.mktemp("hip_host"))


def _p(a):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


@pytest.mark.parametrize("unit", [32, 64])
@pytest.mark.parametrize("words,sizes", [(1, (1, 7, 32, 33, 40, 63, 64)), (2, (64, 65, 97, 128)),
                                         (3, (130, 192)), (0, (1, 31, 64, 200))])
def test_every_word_read_is_one_of_the_row(lib, words, sizes, unit):
    """Every alignment of the context to tiles of 32 and of 64 positions (a
    tile of 64 is asked for in halves, the second of which may lie past the
    last node)."""
    rng = np.random.default_rng(words)
    for n in sizes:
        for L in range(0, 130):
            node = int(rng.integers(0, n))
            row = rng.integers(0, 2 ** 64, words, dtype=np.uint64) if words else None
            bits = np.full(L + n + 64, 9, np.uint8)
            outside = lib.seen(_p(row), words, node, n, L, unit, _p(bits))
            assert outside == 0, (n, L)
            want = np.zeros_like(bits)
            want[S.positions_seen(L, n, node, S.mask_bits(row) if words else None)] = 1
            end = -(-(L + n) // unit) * unit
            assert np.array_equal(bits[:end], want[:end]), (n, L)
