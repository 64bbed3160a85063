"""The dropout generator of the kernels (csrc/philox.h), built for the host, against the oracle's and the published vectors."""
import ctypes

import numpy as np
import pytest

from host_build import CXX, library
from oracle import block_oracle as bo

pytestmark = pytest.mark.skipif(CXX is None, reason="needs a host C++ compiler")


def _philox(counter, key):
    c, k, out = (ctypes.c_uint32 * 4)(*counter), (ctypes.c_uint32 * 2)(*key), (ctypes.c_uint32 * 4)()
    library("philox.cpp").philox(c, k, out)
    return tuple(out)


def test_known_answer_and_random_counters():
    assert _philox((0, 0, 0, 0), (0, 0)) == (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)
    r = np.random.default_rng(3)
    for _ in range(200):
        c, k = [int(v) for v in r.integers(0, 2 ** 32, 4)], [int(v) for v in r.integers(0, 2 ** 32, 2)]
        assert _philox(c, k) == tuple(int(v) for v in bo.philox4x32_10(c, k))
