"""The C ABI of the operators around the expert layer on the CPU: every
declared entry point is exported, and arguments are refused as documented. No
call here reaches a kernel launch."""
import ctypes
import os
import re

import pytest

from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx

FAKE = 0x10000  # a 256-byte-aligned address that is never dereferenced
BAD, UNS, SMALL = lx.LX_ERR_INVALID_ARGUMENT, lx.LX_ERR_UNSUPPORTED, lx.LX_ERR_WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def L(root):
    if not os.path.exists(lx.LIB_PATH):
        from paper_2608_07814_amd import build
        build.build()
    return lb.lib()


def test_every_declared_symbol_is_bound(L, root):
    src = open(os.path.join(root, "include", "lorex_block.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(lx_[a-z0-9_]+)\s*\(", src)))
    assert names == sorted(lb.EXPORTS)
    for n in names:
        assert hasattr(L, n)


def _layer(**kw):
    s = lb.LxNormLayer()
    a = dict(d=64, h_dtype=lx.LX_BF16, y_dtype=lx.LX_F32, x_dtype=lx.LX_BF16, w_dtype=lx.LX_BF16, residual_scale=1.0,
             eps=1e-6, w_pre=FAKE, w_post=FAKE, scale=FAKE, gate=FAKE)
    a.update(kw)
    for n, v in a.items():
        setattr(s, n, v)
    return s


NORM = dict(T=4, h=FAKE, y=FAKE, y_rows=4, k=2, slot_row=FAKE, slot_weights=FAKE, h_out=FAKE, x=FAKE)


@pytest.mark.parametrize("layer,call,code", [
    (dict(d=60), {}, UNS), (dict(d=lb.NORM_MAX_D + 8), {}, UNS), (dict(d=0), {}, BAD), (dict(h_dtype=2), {}, BAD),
    (dict(w_dtype=-1), {}, BAD), (dict(eps=-1.0), {}, BAD), (dict(eps=float("nan")), {}, BAD),
    (dict(w_pre=FAKE + 8), {}, BAD), (dict(w_post=FAKE + 2), {}, BAD), (dict(scale=FAKE + 4), {}, BAD),
    (dict(gate=FAKE + 2), {}, BAD), ({}, dict(T=-1), BAD), ({}, dict(h=None), BAD), ({}, dict(h=FAKE + 8), BAD),
    ({}, dict(y=FAKE + 4), BAD), ({}, dict(h_out=None), BAD), ({}, dict(x=None), BAD),
    (dict(w_pre=None), {}, BAD),                                   # x without w_pre
    ({}, dict(slot_row=None), BAD), ({}, dict(slot_weights=None), BAD), ({}, dict(k=0), BAD), ({}, dict(k=33), BAD),
    ({}, dict(y_rows=-1), BAD), ({}, dict(T=1 << 30, k=32), UNS), ({}, dict(slot_row=FAKE + 2), BAD),
    ({}, dict(y=None), BAD),                                       # slots and h_out without y
    (dict(w_pre=None), dict(y=None, h_out=None, slot_row=None, slot_weights=None, x=None), BAD),
    ({}, dict(T=0, h=None, x=None, h_out=None), lx.LX_OK),
])
def test_block_norm_refusals(L, layer, call, code):
    s, a = _layer(**layer), dict(NORM, **call)
    st = L.lx_block_norm(ctypes.byref(s), a["T"], a["h"], a["y"], a["y_rows"], a["k"], a["slot_row"], a["slot_weights"],
                         a["h_out"], a["x"], None)
    assert st == code, L.lx_last_error()
    assert bool(L.lx_last_error()) == (code != lx.LX_OK)


GRAD = dict(T=4, h_out=FAKE, y=FAKE, dx=FAKE, dh_out=FAKE, dh=FAKE, dy=FAKE, dgate=FAKE, dw_pre=FAKE, dw_post=FAKE,
            dscale=FAKE, ws=FAKE, n=1 << 40)


@pytest.mark.parametrize("layer,call,code", [
    (dict(d=60), {}, UNS), ({}, dict(T=-1), BAD), ({}, dict(h_out=None), BAD), ({}, dict(dh=None), BAD),
    ({}, dict(dx=None), BAD), ({}, dict(dy=None), BAD), ({}, dict(y=None), BAD), ({}, dict(dgate=None), BAD),
    ({}, dict(dw_pre=None), BAD), ({}, dict(dw_post=None), BAD), ({}, dict(dscale=None), BAD),
    (dict(scale=None), {}, BAD), (dict(w_pre=None), {}, BAD), ({}, dict(dy=FAKE + 8), BAD), ({}, dict(ws=None), BAD),
    ({}, dict(ws=FAKE + 128), BAD), ({}, dict(n=16), SMALL), ({}, dict(dw_pre=FAKE + 4), BAD),
    (dict(w_pre=None), dict(y=None, dx=None, dy=None, dw_pre=None, dw_post=None, dscale=None, dgate=None), BAD),
])
def test_block_norm_backward_refusals(L, layer, call, code):
    s, a = _layer(**layer), dict(GRAD, **call)
    st = L.lx_block_norm_backward(ctypes.byref(s), *[a[n] for n in ("T", "h_out", "y", "dx", "dh_out", "dh", "dy", "dgate",
                                                                    "dw_pre", "dw_post", "dscale", "ws", "n")], None)
    assert st == code, L.lx_last_error()
    assert L.lx_last_error()


def test_null_layer(L):
    assert L.lx_block_norm(None, 1, FAKE, None, 0, 0, None, None, None, FAKE, None) == BAD
    assert L.lx_block_norm_backward(None, 1, *[FAKE] * 11, 1 << 30, None) == BAD


BAL = dict(logits=FAKE, dt=lx.LX_F32, T=5000, E=64, ids=FAKE, k=8, mask=None, loss=FAKE, counts=FAKE, prob=FAKE, n_tok=FAKE,
           ws=FAKE, n=1 << 40)


@pytest.mark.parametrize("call,code", [
    (dict(E=0), UNS), (dict(E=1025), UNS), (dict(T=-1), BAD), (dict(k=0), BAD), (dict(k=33), BAD), (dict(dt=2), BAD),
    (dict(T=1 << 27, k=16), UNS), (dict(logits=None), BAD), (dict(logits=FAKE + 4), BAD), (dict(ids=None), BAD),
    (dict(ids=FAKE + 1), BAD), (dict(loss=None), BAD), (dict(counts=None), BAD), (dict(prob=FAKE + 2), BAD),
    (dict(n_tok=None), BAD), (dict(ws=None), BAD), (dict(ws=FAKE + 64), BAD), (dict(n=16), SMALL),
])
def test_balance_refusals(L, call, code):
    a = dict(BAL, **call)
    st = L.lx_balance_loss(a["logits"], a["dt"], a["T"], a["E"], a["ids"], a["k"], a["mask"], 1.0, a["loss"], a["counts"],
                           a["prob"], a["n_tok"], a["ws"], a["n"], None)
    assert st == code, L.lx_last_error()
    assert L.lx_last_error()


@pytest.mark.parametrize("call,code", [
    (dict(E=2000), UNS), (dict(T=-1), BAD), (dict(k=0), BAD), (dict(dt=2), BAD), (dict(logits=None), BAD),
    (dict(counts=None), BAD), (dict(n_tok=None), BAD), (dict(dlogits=None), BAD), (dict(dlogits=FAKE + 8), BAD),
    (dict(dloss=FAKE + 2), BAD), (dict(T=0, logits=None), lx.LX_OK),
])
def test_balance_backward_refusals(L, call, code):
    a = dict(BAL, dloss=FAKE, dlogits=FAKE, **call) if "dloss" not in call and "dlogits" not in call \
        else dict(dict(BAL, dloss=FAKE, dlogits=FAKE), **call)
    st = L.lx_balance_loss_backward(a["logits"], a["dt"], a["T"], a["E"], a["k"], a["mask"], a["counts"], a["n_tok"], 1.0,
                                    a["dloss"], a["dlogits"], None)
    assert st == code, L.lx_last_error()


@pytest.mark.parametrize("call,code", [
    (dict(rows=-1), BAD), (dict(K=0), BAD), (dict(K=60), UNS), (dict(rows=1 << 36), UNS), (dict(dt=3), BAD),
    (dict(act=2), BAD), (dict(x=None), BAD), (dict(x=FAKE + 8), BAD), (dict(codes=FAKE + 8), BAD), (dict(codes=None), BAD),
    (dict(scales=FAKE + 2), BAD), (dict(scales=None), BAD), (dict(rows=0, x=None), lx.LX_OK),
])
def test_mx4_quantize_and_dequantize_refusals(L, call, code):
    a = dict(dict(x=FAKE, dt=lx.LX_F32, rows=4, K=64, act=0, codes=FAKE, scales=FAKE), **call)
    assert L.lx_mx4_quantize(a["x"], a["dt"], a["rows"], a["K"], a["act"], a["codes"], a["scales"], None) == code
    if "act" not in call:
        assert L.lx_mx4_dequantize(a["codes"], a["scales"], a["rows"], a["K"], a["x"], a["dt"], None) == code


@pytest.mark.parametrize("call,code", [
    (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(K=60), UNS), (dict(G=0), BAD), (dict(G=8193), UNS),
    (dict(M=1 << 30, N=1 << 11, ar=1 << 30), UNS), (dict(dt=2), BAD), (dict(ar=3, rm=None), BAD), (dict(ar=-1), BAD),
    (dict(off=None), BAD),                                         # several groups without offsets
    (dict(a=None), BAD), (dict(a=FAKE + 8), BAD), (dict(as_=FAKE + 2), BAD), (dict(b=FAKE + 4), BAD), (dict(bs=None), BAD),
    (dict(rm=FAKE + 2), BAD), (dict(off=FAKE + 1), BAD), (dict(out=None), BAD), (dict(out=FAKE + 8), BAD),
    (dict(M=0, a=None, out=None), lx.LX_OK),
])
def test_mx4_gemm_refusals(L, call, code):
    a = dict(dict(a=FAKE, as_=FAKE, ar=4, rm=FAKE, b=FAKE, bs=FAKE, off=FAKE, G=2, M=4, N=8, K=64, out=FAKE, dt=lx.LX_F32), **call)
    n = L.lx_mx4_gemm_workspace_bytes(a["M"], a["N"], a["K"], a["G"])
    st = L.lx_mx4_gemm(a["a"], a["as_"], a["ar"], a["rm"], a["b"], a["bs"], a["off"], a["G"], a["M"], a["N"], a["K"], a["out"],
                       a["dt"], FAKE, n, None)
    assert st == code, L.lx_last_error()


def test_wrappers_refuse_cpu_tensors():
    import torch
    with pytest.raises(ValueError):
        lb.block_norm(torch.zeros(2, 8), w_pre=torch.zeros(8))
    with pytest.raises(ValueError):
        lb.balance_loss(torch.zeros(2, 8), torch.zeros(2, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        lb.mx4_quantize(torch.zeros(2, 32))


def test_fp4_oracle_rounds_as_defined():
    """The oracle's rounding against a search over all codes, ties included."""
    import numpy as np
    from oracle import block as O
    x = np.array([[0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7.9, -0.25, -0.75, -5, 4.0, 0.2500001, 0.74] + [0.0] * 16])
    codes, scales, _ = O.quantize(x)
    assert scales[0, 0] == 127
    v = O.dequantize(codes, scales, 32)[0]
    assert v[:16].tolist() == [0, 0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -1, -4, 4, 0.5, 0.5]
    assert scales[0, 1:].tolist() == [0, 0, 0] and codes[0, 16:].max() == 0
