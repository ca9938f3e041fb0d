"""Registers of the 4-bit product and norm kernels, read from the gfx950 assembly that
the sources compile to (no GPU needed)."""
import os
import re
import subprocess
import tempfile

from paper_2608_07814_amd import build as B


def _asm(src):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, src + ".s")
        subprocess.run([B.HIPCC, *B.CFLAGS, "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", out],
                       check=True, stderr=subprocess.DEVNULL)
        return open(out).read()


def _sizes(asm, what, name):
    return {m[0]: int(m[1]) for m in re.findall(r"\.set (_Z\w*%s\w*)\.%s, (\d+)" % (name, what), asm)}


def test_products_keep_everything_in_registers():
    """A tile's accumulators and fragments stay in registers, and as many
    workgroups as the tile's size plans for fit on a compute unit: 64 x 64 four
    (at most 128 registers a lane of 512), 128 x 128 two (256); one of 256 x 256
    has two wavefronts per SIMD (256)."""
    asm = _asm("k_mx4.hip")
    scratch, vgpr, agpr = (_sizes(asm, w, "k_mx4_gemm") for w in ("private_seg_size", "num_vgpr", "num_agpr"))
    assert len(scratch) >= 6 and max(scratch.values()) == 0, scratch
    for n in vgpr:
        most = 128 if "ILi64ELi64E" in n else 256 if "gemm_tile" in n else 512
        assert vgpr[n] + agpr[n] <= most, (n, vgpr[n], agpr[n])


def test_no_packed_fp32():
    for src in ("k_mx4.hip", "k_norm.hip", "k_balance.hip"):
        assert not re.search(r"\bv_pk_(add|mul|fma)_f32", _asm(src)), src
