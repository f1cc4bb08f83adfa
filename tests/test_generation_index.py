"""The index arithmetic of the generation kernels at the largest sizes that the entry points accept, against Python's integers: host
code, no GPU."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
TOP = 2**31 - 1


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("index") / "libgeneration_index.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fwrapv", "-shared", "-fPIC",
                    os.path.join(HERE, "generation_index.cpp"), "-o", out], check=True)
    return ctypes.CDLL(out)


@pytest.mark.parametrize("n", [1, 2, 1000, 2**30, 2**30 + 1, 1_200_000_000, 1_500_000_000, TOP])
def test_the_first_entry_of_a_ring(index, n):
    """A ring of pages of one token has up to 2^31 - 1 entries."""
    for first in (0, 1, n - 1, n // 2 + 1, n // 2 - 1, 1_100_000_000, TOP, -1, -n, 1 - n, -TOP - 1):
        assert index.ring_first(first, n) == first % n, first
