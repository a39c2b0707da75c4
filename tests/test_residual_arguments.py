"""The argument checks of the root-mean-square norm and of the AdamW step: synchronous, before anything touches a device,
so they are tested without one.  Pointers are made-up addresses that no call may follow."""
import ctypes

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

vp = ctypes.c_void_p
P, Q, R, S = 0x10000, 0x20000, 0x30000, 0x40000           # 32-byte aligned, never read
NULL, ARG, DTYPE, ALIGN, WORKSPACE, TOO_LARGE = (hb.HAG_ERR_NULL, hb.HAG_ERR_ARG, hb.HAG_ERR_DTYPE, hb.HAG_ERR_ALIGN, hb.HAG_ERR_WORKSPACE,
                                                 hb.HAG_ERR_TOO_LARGE)
F32, BF16 = hb.HAG_F32, hb.HAG_BF16
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    build_library()
    return hb.load_library()


def _fwd(lib, **k):
    a = dict(n=4, d=8, x=P, xdt=F32, ldx=8, r=Q, sdt=F32, ldr=8, w=None, wdt=F32, eps=1e-5, y=R, ydt=F32, ldy=8, t=S, ldt=8, rstd=None) | k
    return lib.hag_rms_norm_fwd(a["n"], a["d"], a["x"], a["xdt"], a["ldx"], a["r"], a["sdt"], a["ldr"], a["w"], a["wdt"], a["eps"], a["y"], a["ydt"],
                                a["ldy"], a["t"], a["ldt"], a["rstd"], None)


def _quant(lib, **k):
    a = dict(n=4, d=64, x=P, xdt=F32, ldx=64, r=Q, sdt=F32, ldr=64, w=None, wdt=F32, eps=1e-5, kind=hb.HAG_E4M3, block=32, q=R, ldq=64, s=P, t=S, ldt=64,
             rstd=None) | k
    return lib.hag_rms_norm_quant_fwd(a["n"], a["d"], a["x"], a["xdt"], a["ldx"], a["r"], a["sdt"], a["ldr"], a["w"], a["wdt"], a["eps"], a["kind"],
                                      a["block"], a["q"], a["ldq"], a["s"], a["t"], a["ldt"], a["rstd"], None)


def _bwd(lib, **k):
    a = dict(n=4, d=8, g=P, ydt=F32, ldg=8, t=Q, sdt=F32, ldt=8, rstd=P, w=None, wdt=F32, a=None, lda=8, out=R, ldo=8, x=None, ldx=8, gw=P, ws=P) | k
    return lib.hag_rms_norm_bwd(a["n"], a["d"], a["g"], a["ydt"], a["ldg"], a["t"], a["sdt"], a["ldt"], a["rstd"], a["w"], a["wdt"], a["a"], a["lda"],
                                a["out"], a["ldo"], a["x"], a["ldx"], a["gw"], a["ws"], None)


BF = dict(xdt=BF16, sdt=BF16, ydt=BF16)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(n=-1), ARG), (dict(d=0), ARG), (dict(eps=-1.0), ARG), (dict(eps=NAN), ARG), (dict(ldy=7), ARG),
    (dict(ldt=7), ARG), (dict(ldx=-1), ARG), (dict(ldr=-8), ARG), (dict(y=P, ldy=9), ARG), (dict(t=Q, ldt=16), ARG), (dict(y=S), ARG), (dict(y=P, ydt=BF16), ARG),
    (dict(xdt=2), DTYPE), (dict(sdt=-1), DTYPE), (dict(ydt=3), DTYPE), (dict(wdt=2), DTYPE), (dict(xdt=BF16), DTYPE), (dict(sdt=BF16), DTYPE),
    (dict(xdt=BF16, ydt=BF16, r=None), DTYPE), (dict(xdt=BF16, sdt=BF16), DTYPE), (dict(x=P + 2), ALIGN), (dict(r=Q + 2), ALIGN), (dict(y=R + 1), ALIGN),
    (dict(t=S + 2), ALIGN), (dict(w=P + 2), ALIGN), (dict(w=P + 1, wdt=BF16), ALIGN), (dict(rstd=P + 2), ALIGN), (BF | dict(x=P + 1), ALIGN),
    (dict(d=(1 << 30) + 1, ldy=1 << 31, ldt=1 << 31), TOO_LARGE), (dict(n=0, x=None, y=None, r=None, t=None), 0), (dict(n=0, sdt=BF16, xdt=BF16, ydt=BF16), 0)])
def test_forward(lib, change, status):
    assert _fwd(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(x=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL), (dict(n=-1), ARG), (dict(block=16), ARG), (dict(block=-32), ARG), (dict(block=256), ARG),
    (dict(eps=NAN), ARG), (dict(ldq=63), ARG), (dict(ldt=63), ARG), (dict(q=P), ARG), (dict(q=S), ARG), (dict(kind=2), DTYPE), (dict(xdt=BF16, r=None), DTYPE),
    (dict(sdt=BF16), DTYPE), (dict(s=P + 2), ALIGN), (dict(t=S + 1), ALIGN), (dict(n=0, x=None, q=None, s=None), 0)])
def test_quantised(lib, change, status):
    assert _quant(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(g=None), NULL), (dict(t=None), NULL), (dict(out=None), NULL), (dict(rstd=None), NULL), (dict(n=-1), ARG), (dict(d=-3), ARG), (dict(ldo=7), ARG),
    (dict(ldg=-1), ARG), (dict(a=S, lda=-1), ARG), (dict(out=P, ldo=9), ARG), (dict(x=R, ydt=BF16), ARG), (dict(x=S, ldx=7), ARG), (dict(ydt=2), DTYPE),
    (dict(sdt=2), DTYPE), (dict(wdt=-1), DTYPE), (dict(sdt=BF16), DTYPE), (dict(sdt=BF16, ydt=BF16, x=S), DTYPE), (dict(out=R + 2), ALIGN), (dict(x=S + 1), ALIGN),
    (dict(gw=P + 2), ALIGN), (dict(rstd=P + 1), ALIGN), (dict(a=S + 2), ALIGN), (dict(ws=P + 4), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(d=(1 << 30) + 1, ldo=1 << 31), TOO_LARGE), (dict(n=0, g=None, t=None, out=None, rstd=None, gw=None, ws=None), 0)])
def test_backward(lib, change, status):
    assert _bwd(lib, **change) == status


def test_backward_workspace(lib):
    size = lib.hag_rms_norm_bwd_workspace_bytes
    assert size(-1, 8) == 0 and size(5, 0) == 0 and size(0, 8) > 0 and size(1000, 8) > 0
    assert size(10, 1 << 30) == 10 * (1 << 32) and size(1 << 40, 8) == size(1 << 20, 8)


def _step(lib, count=2, params=(P, Q), pk=(0, 1), grads=(R, S), gk=(0, 1), copies=None, lens=(4, 4), decays=(0.0, 0.1), kind=0, mean=P, square=Q, scales=R,
          options=True, **o):
    arr = lambda t, v: None if v is None else (t * len(v))(*v)  # noqa: E731
    opt = hb.HagAdamwOptions(**(dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, max_norm=1.0, step=1) | o))
    return lib.hag_adamw_step(count, arr(vp, params), arr(ctypes.c_int, pk), arr(vp, grads), arr(ctypes.c_int, gk), arr(vp, copies), arr(ctypes.c_int64, lens),
                              arr(ctypes.c_double, decays), kind, mean, square, scales, ctypes.byref(opt) if options else None, None)


@pytest.mark.parametrize("change,status", [
    (dict(options=False), NULL), (dict(params=None), NULL), (dict(pk=None), NULL), (dict(grads=None), NULL), (dict(gk=None), NULL), (dict(lens=None), NULL),
    (dict(decays=None), NULL), (dict(params=(None, Q)), NULL), (dict(mean=None), NULL), (dict(square=None), NULL), (dict(kind=1, scales=None), NULL),
    (dict(count=-1), ARG), (dict(lens=(4, -1)), ARG), (dict(decays=(0.0, -0.1)), ARG), (dict(decays=(NAN, 0.0)), ARG), (dict(step=0), ARG), (dict(step=-5), ARG),
    (dict(lr=-1.0), ARG), (dict(lr=NAN), ARG), (dict(beta1=1.0), ARG), (dict(beta1=-0.1), ARG), (dict(beta2=NAN), ARG), (dict(eps=-1.0), ARG),
    (dict(total_norm=P, max_norm=-1.0), ARG), (dict(total_norm=P, max_norm=NAN), ARG), (dict(kind=2), DTYPE), (dict(pk=(0, 2)), DTYPE), (dict(gk=(-1, 0)), DTYPE),
    (dict(params=(P + 2, Q)), ALIGN), (dict(grads=(R, S + 1)), ALIGN), (dict(copies=(P + 1, None)), ALIGN), (dict(mean=P + 8), ALIGN), (dict(square=Q + 4), ALIGN),
    (dict(kind=1, scales=R + 4), ALIGN), (dict(lr_device=P + 2), ALIGN), (dict(step_device=P + 4), ALIGN), (dict(total_norm=P + 1), ALIGN),
    (dict(lens=((1 << 39) - 255, 4)), TOO_LARGE), (dict(lens=((1 << 63) - 1, (1 << 63) - 1)), TOO_LARGE), (dict(lens=(0, 0), mean=None, square=None), 0),
    (dict(count=0, params=None, pk=None, grads=None, gk=None, lens=None, decays=None, mean=None, square=None), 0), (dict(grads=(None, None)), 0)])
def test_step(lib, change, status):
    assert _step(lib, **change) == status


def test_state_blocks(lib):
    blocks = lambda *lens: lib.hag_adamw_state_blocks(len(lens), (ctypes.c_int64 * len(lens))(*lens))  # noqa: E731
    assert blocks(0) == 0 and blocks(1) == 1 and blocks(256) == 1 and blocks(257, 0, 255, 512) == 5 and blocks(-1) == -1
    assert blocks((1 << 39) - 256) == (1 << 31) - 1 and blocks((1 << 39) - 255) == -1 and blocks((1 << 63) - 1) == -1
    assert lib.hag_adamw_state_blocks(-1, None) == -1 and lib.hag_adamw_state_blocks(1, None) == -1 and lib.hag_adamw_state_blocks(0, None) == 0


def test_the_block_of_the_states_is_the_headers():
    import os
    import re
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hag.h")).read()
    assert int(re.search(r"#define HAG_ADAMW_BLOCK (\d+)", header).group(1)) == hb.HAG_ADAMW_BLOCK
