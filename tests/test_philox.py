"""The dropout's generator against the published vectors of Philox4x32-10 (the header compiled for the CPU), and the
fp64 oracle's mask against it."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import block as O

SOURCE = r"""
#define __device__
#define __forceinline__ inline
#include "lx_philox.h"
extern "C" unsigned kept(unsigned group, unsigned token, const unsigned* q, unsigned below) {
  lx::Dropout d{nullptr, below, 1.f};
  return lx::dropout_kept(d, lx::DropoutKeys{q[0], q[1], q[2], q[3]}, group, token);
}
"""


@pytest.fixture(scope="module")
def kept(root, tmp_path_factory):
    at = tmp_path_factory.mktemp("philox")
    (at / "k.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(root, "paper_2608_07814_amd", "csrc"), "-o", at / "k.so", at / "k.cpp"],
                   check=True)
    f = ctypes.CDLL(str(at / "k.so")).kept
    f.restype, f.argtypes = ctypes.c_uint32, [ctypes.c_uint32, ctypes.c_uint32, ctypes.POINTER(ctypes.c_uint32), ctypes.c_uint32]
    return lambda group, token, key, offset, below: f(group, token, (ctypes.c_uint32 * 4)(*key, *offset), below)


ONES = 0xFFFFFFFF


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((ONES,) * 4, (ONES,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_published_vectors(kept, counter, key, words):
    """A column is kept exactly as long as its 16 bits are not below the border: that gives them all."""
    for c, u in enumerate(h for w in words for h in (w & 0xFFFF, w >> 16)):
        assert kept(*counter[:2], key, counter[2:], u) >> c & 1 and not kept(*counter[:2], key, counter[2:], u + 1) >> c & 1, c


@pytest.mark.parametrize("seed,offset,p", [(0, 0, 0.5), (0xFFFFFFFFFFFFFFFF, 0xFFFFFFFFFFFFFFFF, 0.3), (0x1234567890ABCDEF, (7 << 32) + 11, 0.9)])
def test_oracle_draws_the_same(kept, seed, offset, p):
    low = 0xFFFFFFFF
    mask = O.dropout_keep(5, 40, p, seed, offset) > 0
    got = [[kept(c // 8, t, (seed & low, seed >> 32), (offset & low, offset >> 32), int(p * 65536 + 0.5)) >> c % 8 & 1 for c in range(40)] for t in range(5)]
    assert np.array_equal(mask, np.array(got, bool))
