"""Refusals of the norms with an 8-bit output, the 8-bit rounding and the dropout, on
the CPU. No call here reaches a kernel launch."""
import ctypes
import os

import pytest
import torch

from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx

FAKE = 0x10000  # a 256-byte-aligned address that is never dereferenced
BAD, UNS, SMALL, OK = lx.LX_ERR_INVALID_ARGUMENT, lx.LX_ERR_UNSUPPORTED, lx.LX_ERR_WORKSPACE_TOO_SMALL, lx.LX_OK


@pytest.fixture(scope="module")
def L(root):
    if not os.path.exists(lx.LIB_PATH):
        from paper_2608_07814_amd import build
        build.build()
    return lb.lib()


def layer(**kw):
    s = lb.LxNormLayer()
    a = dict(d=64, h_dtype=lx.LX_BF16, y_dtype=lx.LX_F32, x_dtype=lx.LX_BF16, w_dtype=lx.LX_BF16, residual_scale=1.0,
             eps=1e-6, w_pre=FAKE, w_post=FAKE, scale=FAKE, gate=FAKE)
    for n, v in dict(a, **kw).items():
        setattr(s, n, v)
    return s


NORM = dict(T=4, h=FAKE, y=FAKE, y_rows=4, k=2, slot_row=FAKE, slot_weights=FAKE, h_out=FAKE, x=None, codes=FAKE, scales=FAKE)


@pytest.mark.parametrize("over,call,code", [
    (dict(d=60), {}, UNS), (dict(d=lb.NORM_MAX_D + 8), {}, UNS), (dict(eps=-1.0), {}, BAD), ({}, dict(T=-1), BAD),
    ({}, dict(h=None), BAD), ({}, dict(h_out=None), BAD), ({}, dict(codes=None), BAD), ({}, dict(codes=FAKE + 8), BAD),
    ({}, dict(scales=None), BAD), ({}, dict(scales=FAKE + 2), BAD), ({}, dict(x=FAKE, codes=None), BAD), ({}, dict(x=FAKE + 8), BAD),
    (dict(x_dtype=7), dict(x=FAKE), BAD), (dict(w_pre=None), dict(x=FAKE), BAD), (dict(w_pre=None), dict(codes=None), BAD), ({}, dict(k=33), BAD),
    ({}, dict(slot_row=None), BAD), ({}, dict(y=None), BAD), ({}, dict(T=0, h=None, codes=None, scales=None), OK),
])
def test_norm_mx8(L, over, call, code):
    a = dict(NORM, **call)
    st = L.lx_block_norm_mx8(ctypes.byref(layer(**over)), *a.values(), None)
    assert st == code, L.lx_last_error()
    assert bool(L.lx_last_error()) == (code != OK)


def test_null_structures(L):
    drop = ctypes.byref(lb.LxDropout(0.5, FAKE))
    assert L.lx_block_norm_mx8(None, *NORM.values(), None) == BAD
    assert L.lx_block_norm_dropout(None, drop, 1, FAKE, FAKE, FAKE, FAKE, None) == BAD
    assert L.lx_block_norm_dropout(ctypes.byref(layer()), None, 1, FAKE, FAKE, FAKE, FAKE, None) == BAD
    assert L.lx_block_norm_dropout_backward(ctypes.byref(layer()), None, 1, *[FAKE] * 11, 1 << 30, None) == BAD


@pytest.mark.parametrize("p,rng,call,code", [
    (-0.1, FAKE, {}, BAD), (1.0, FAKE, {}, BAD), (1 - 2.0 ** -17, FAKE, {}, BAD), (float("nan"), FAKE, {}, BAD), (0.5, None, {}, BAD),
    (0.5, FAKE + 4, {}, BAD), (0.5, FAKE, dict(y=None, h_out=None), BAD), (0.5, FAKE, dict(h=None), BAD), (0.5, FAKE, dict(x=None), BAD),
    (0.5, FAKE, dict(T=0, h=None, x=None), OK), (0.0, None, {}, BAD),
])
def test_dropout(L, p, rng, call, code):
    a = dict(dict(T=4, h=FAKE, y=FAKE, h_out=FAKE, x=FAKE), **call)
    st = L.lx_block_norm_dropout(ctypes.byref(layer()), ctypes.byref(lb.LxDropout(p, rng)), *a.values(), None)
    assert st == code, L.lx_last_error()


GRAD = dict(T=4, h_out=FAKE, y=FAKE, dx=FAKE, dh_out=FAKE, dh=FAKE, dy=FAKE, dgate=FAKE, dw_pre=FAKE, dw_post=FAKE,
            dscale=FAKE, ws=FAKE, n=1 << 40)


@pytest.mark.parametrize("p,rng,call,code", [
    (1.0, FAKE, {}, BAD), (0.5, None, {}, BAD), (0.5, FAKE + 4, {}, BAD), (0.5, FAKE, dict(y=None), BAD), (0.5, FAKE, dict(dh=None), BAD),
    (0.5, FAKE, dict(dy=None), BAD), (0.5, FAKE, dict(dgate=None), BAD), (0.5, FAKE, dict(dw_post=None), BAD), (0.5, FAKE, dict(ws=None), BAD),
    (0.5, FAKE, dict(n=16), SMALL), (0.5, FAKE, dict(dx=None), BAD),
])
def test_dropout_backward(L, p, rng, call, code):
    a = dict(GRAD, **call)
    st = L.lx_block_norm_dropout_backward(ctypes.byref(layer()), ctypes.byref(lb.LxDropout(p, rng)), *a.values(), None)
    assert st == code, L.lx_last_error()


@pytest.mark.parametrize("call,code", [
    (dict(rows=-1), BAD), (dict(K=0), BAD), (dict(K=60), UNS), (dict(rows=1 << 36), UNS), (dict(dt=3), BAD),
    (dict(act=2), BAD), (dict(x=None), BAD), (dict(x=FAKE + 8), BAD), (dict(codes=FAKE + 8), BAD), (dict(codes=None), BAD),
    (dict(scales=FAKE + 2), BAD), (dict(scales=None), BAD), (dict(rows=0, x=None), OK),
])
def test_mx8_quantize_and_dequantize(L, call, code):
    a = dict(dict(x=FAKE, dt=lx.LX_F32, rows=4, K=64, act=0, codes=FAKE, scales=FAKE), **call)
    assert L.lx_mx8_quantize(a["x"], a["dt"], a["rows"], a["K"], a["act"], a["codes"], a["scales"], None) == code
    if "act" not in call:
        assert L.lx_mx8_dequantize(a["codes"], a["scales"], a["rows"], a["K"], a["x"], a["dt"], None) == code


FEW = dict(x=FAKE, dt=lx.LX_BF16, T=4, d=64, ids=FAKE, w=FAKE, k=2, E=8, f=32, gu=FAKE, gus=FAKE, dn=FAKE, dns=FAKE, out=FAKE, odt=lx.LX_F32,
           ws=FAKE, n=1 << 40)


@pytest.mark.parametrize("call,code", [
    (dict(T=-1), BAD), (dict(T=65), UNS), (dict(d=0), BAD), (dict(d=60), UNS), (dict(f=20), UNS), (dict(f=0), BAD), (dict(d=1 << 21), UNS),
    (dict(E=0), UNS), (dict(E=8193), UNS), (dict(k=0), UNS), (dict(k=33), UNS), (dict(dt=2), BAD), (dict(odt=-1), BAD), (dict(x=None), BAD),
    (dict(x=FAKE + 8), BAD), (dict(ids=None), BAD), (dict(ids=FAKE + 2), BAD), (dict(w=None), BAD), (dict(gu=FAKE + 4), BAD), (dict(gus=None), BAD),
    (dict(dn=None), BAD), (dict(dns=FAKE + 1), BAD), (dict(out=None), BAD), (dict(out=FAKE + 8), BAD), (dict(ws=None), BAD),
    (dict(ws=FAKE + 128), BAD), (dict(n=64), SMALL), (dict(T=0, x=None, ws=None), OK),
])
def test_moe_few(L, call, code):
    a = dict(FEW, **call)
    st = L.lx_mx4_moe_few(*a.values(), None)
    assert st == code, L.lx_last_error()
    n = L.lx_mx4_moe_few_workspace_bytes(a["T"], a["k"], a["E"], a["d"], a["f"])
    assert (n == 0) == (any(v in call for v in ("T", "d", "f", "E", "k"))), n


GEMM = dict(a=FAKE, as_=FAKE, ar=4, rm=FAKE, b=FAKE, bs=FAKE, off=FAKE, G=2, M=4, N=16, K=64)


@pytest.mark.parametrize("call,epi,to,code", [
    (dict(M=-1), {}, {}, BAD), (dict(N=0), {}, {}, BAD), (dict(K=0), {}, {}, BAD), (dict(K=60), {}, {}, UNS), (dict(G=0), {}, {}, BAD),
    (dict(G=8193), {}, {}, UNS), (dict(M=(1 << 31) - 255, ar=(1 << 31) - 1), {}, {}, UNS), (dict(N=(1 << 31) - 255), {}, {}, UNS),
    (dict(M=1 << 30, N=1 << 11, ar=1 << 30), {}, {}, UNS), (dict(ar=3, rm=None), {}, {}, BAD), (dict(ar=-1), {}, {}, BAD), (dict(off=None), {}, {}, BAD),
    (dict(a=None), {}, {}, BAD), (dict(a=FAKE + 8), {}, {}, BAD), (dict(as_=FAKE + 2), {}, {}, BAD), (dict(b=FAKE + 4), {}, {}, BAD),
    (dict(bs=None), {}, {}, BAD), (dict(rm=FAKE + 2), {}, {}, BAD), (dict(off=FAKE + 1), {}, {}, BAD),
    ({}, dict(act=4), {}, BAD), ({}, dict(act=-1), {}, BAD), ({}, dict(bias_dtype=2), {}, BAD), ({}, dict(residual_dtype=3), {}, BAD),
    ({}, dict(bias=FAKE + 2), {}, BAD), ({}, dict(bias=FAKE + 1, bias_dtype=1), {}, BAD), ({}, dict(residual=FAKE + 2), {}, BAD),
    (dict(N=17), dict(act=3), {}, BAD), ({}, {}, dict(out=None), BAD), ({}, {}, dict(out=FAKE + 8), BAD), ({}, {}, dict(dt=2), BAD),
    ({}, {}, dict(scales=FAKE + 2), BAD), (dict(N=20), {}, dict(scales=FAKE), UNS), (dict(N=24), dict(act=3), dict(scales=FAKE), UNS),
    (dict(M=0, a=None), {}, dict(out=None), OK),
])
def test_mx8_gemm(L, call, epi, to, code):
    e = lb.LxEpilogue()
    for n, v in dict(dict(act=0, bias_dtype=0, residual_dtype=0, bias=FAKE, residual=FAKE), **epi).items():
        setattr(e, n, v)
    t = dict(dict(out=FAKE, dt=lx.LX_F32, scales=None), **to)
    st = L.lx_mx8_gemm(*dict(GEMM, **call).values(), ctypes.byref(e), *t.values(), FAKE, 1 << 60, None)
    assert st == code, L.lx_last_error()
    assert bool(L.lx_last_error()) == (code != OK)


def test_the_largest_products_are_taken(L):
    most = (1 << 31) - 256
    for M, N in ((most, 1), (most, 8), (1, most), (8, most)):
        L.lx_mx8_gemm_workspace_bytes(M, N, 64, 1, 0)
        assert not L.lx_last_error()
    assert L.lx_mx8_gemm_workspace_bytes(4, 8, 64, 1, 9) == 0 and L.lx_last_error()


def test_wrappers_refuse_cpu_tensors():
    h, w = torch.zeros(2, 8), torch.zeros(8)
    rng = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: lb.block_norm_mx8(h, w_pre=w), lambda: lb.block_norm_dropout(h, h, 0.5, rng, w_pre=w),
                 lambda: lb.block_norm_dropout_backward(h, h, h, None, 0.5, rng, w_pre=w), lambda: lb.mx8_quantize(h),
                 lambda: lb.mx8_dequantize(lb.Mx8(torch.zeros(2, 128, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.uint8), 128))):
        with pytest.raises(ValueError):
            call()


def test_fp8_oracle_rounds_as_defined():
    """Ties to the even code, subnormal codes, and scales under which nothing saturates."""
    import numpy as np
    from oracle import block as O
    x = np.zeros((1, 128))
    x[0, :6] = [448, 17, 19, 2.0 ** -9, 1.5 * 2.0 ** -9, 2.0 ** -10]
    x[0, 32:34] = [449, 1]
    codes, scales, _ = O.quantize8(x)
    v = O.dequantize8(codes, scales, 128)[0]
    assert scales[0].tolist() == [127, 128, 0, 0]
    assert v[:6].tolist() == [448, 16, 20, 2.0 ** -9, 2.0 ** -8, 0] and v[32:34].tolist() == [448, 1]
    # the published test vector of the generator: key and counter of zeros and of ones
    assert [int(b) for b in (O.dropout_keep(1, 8, 0.5, 0, 0) > 0)[0]] == [
        h >= 0x8000 for w in (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8) for h in (w & 0xFFFF, w >> 16)]
