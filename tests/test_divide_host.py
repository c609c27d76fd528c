"""The division by page sizes and group sizes that the kernels use, compiled for the host.  No GPU."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2510_24606_amd import build

SOURCE = r"""
#include "divide.h"
extern "C" long check(uint32_t d, const int32_t *x, long n) {      // the first x that comes out wrong, or -1
    uint32_t mul; int shift;
    dhsa::set_divisor(d, &mul, &shift);
    for (long i = 0; i < n; ++i)
        if (dhsa::divided(x[i], mul, shift) != (int)((uint32_t)x[i] / d)) return x[i];
    return -1;
}
"""


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    where = tmp_path_factory.mktemp("divide")
    (where / "divide.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-shared", "-fPIC", "-I", os.path.join(build.HERE, "csrc"), "-o", str(where / "divide.so"), str(where / "divide.cpp")],
                   check=True)
    f = C.CDLL(str(where / "divide.so")).check
    f.argtypes, f.restype = [C.c_uint32, C.c_void_p, C.c_long], C.c_long
    return f


def test_every_small_divisor_and_the_ends_of_the_range(check):
    rng = np.random.default_rng(1)
    top = (1 << 31) - 1
    sizes = np.unique(np.concatenate([np.arange(1, 3000), 2 ** np.arange(31), 2 ** np.arange(2, 31) - 1, 2 ** np.arange(30) + 1,
                                      rng.integers(1, 1 << 30, 3000), np.arange((1 << 30) - 20, (1 << 30) + 1)]))
    anywhere = np.concatenate([np.arange(2000), top - np.arange(2000), rng.integers(0, top, 2000, endpoint=True)])
    for d in (int(x) for x in sizes):
        k = np.concatenate([rng.integers(0, top // d, 300, endpoint=True), top // d - np.arange(min(20, top // d + 1))])
        x = np.ascontiguousarray(np.clip(np.concatenate([anywhere, k * d, k * d + d - 1, k * d - 1]), 0, top).astype(np.int32))
        assert check(d, x.ctypes.data, len(x)) == -1, d
