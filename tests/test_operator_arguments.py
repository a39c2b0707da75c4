"""The argument checks of the embedding, layer-norm and clipping entry points: synchronous, before anything touches a
device, so they are tested without one.  Pointers are made-up addresses that no call may follow."""
import ctypes

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

vp = ctypes.c_void_p
P, Q, R = 0x10000, 0x20000, 0x30000           # 16-byte aligned, never read
NULL, ARG, DTYPE, ALIGN, WORKSPACE, TOO_LARGE = (hb.HAG_ERR_NULL, hb.HAG_ERR_ARG, hb.HAG_ERR_DTYPE, hb.HAG_ERR_ALIGN, hb.HAG_ERR_WORKSPACE,
                                                 hb.HAG_ERR_TOO_LARGE)


@pytest.fixture(scope="module")
def lib():
    build_library()
    return hb.load_library()


def _emb_fwd(lib, **k):
    a = dict(ids=P, t=0, n=4, v=9, table=Q, tdt=0, ldt=8, dt=0, d=8, out=R, ldo=8) | k
    return lib.hag_embedding_fwd(a["ids"], a["t"], a["n"], a["v"], a["table"], a["tdt"], a["ldt"], a["dt"], a["d"], 1.0, a["out"], a["ldo"], None)


def _emb_bwd(lib, **k):
    a = dict(ids=P, t=0, n=4, v=9, dt=0, d=8, g=Q, ldg=8, out=R, tdt=0, ldo=8, ws=P) | k
    return lib.hag_embedding_bwd(a["ids"], a["t"], a["n"], a["v"], a["dt"], a["d"], a["g"], a["ldg"], 1.0, a["out"], a["tdt"], a["ldo"], a["ws"], None)


@pytest.mark.parametrize("change,status", [
    (dict(ids=None), NULL), (dict(table=None), NULL), (dict(out=None), NULL), (dict(d=0), ARG), (dict(n=-1), ARG), (dict(v=-1), ARG),
    (dict(ldt=-1), ARG), (dict(ldo=7), ARG), (dict(out=Q), ARG), (dict(t=2), DTYPE), (dict(dt=2), DTYPE), (dict(tdt=-1), DTYPE),
    (dict(ids=P + 2), ALIGN), (dict(ids=P + 4, t=1), ALIGN), (dict(table=Q + 2), ALIGN), (dict(out=R + 1, dt=1), ALIGN),
    (dict(v=(1 << 31) - 1), TOO_LARGE), (dict(d=(1 << 30) + 1, ldt=1 << 31, ldo=1 << 31), TOO_LARGE), (dict(n=0, ids=None, out=None), 0)])
def test_embedding_forward(lib, change, status):
    assert _emb_fwd(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(ids=None), NULL), (dict(g=None), NULL), (dict(out=None), NULL), (dict(d=0), ARG), (dict(n=-1), ARG), (dict(v=-1), ARG),
    (dict(ldg=-1), ARG), (dict(ldo=7), ARG), (dict(out=Q), ARG), (dict(t=-1), DTYPE), (dict(dt=5), DTYPE), (dict(tdt=2), DTYPE),
    (dict(g=Q + 2), ALIGN), (dict(out=R + 2), ALIGN), (dict(ws=P + 8), ALIGN), (dict(ws=None), WORKSPACE), (dict(n=(1 << 31) - 1), TOO_LARGE),
    (dict(v=0, out=None), 0)])
def test_embedding_backward(lib, change, status):
    assert _emb_bwd(lib, **change) == status


def test_embedding_workspace(lib):
    size = lib.hag_embedding_bwd_workspace_bytes
    assert size(0, 10, 8) == 0 and size(-1, 10, 8) == 0
    assert size(1, 10, 8) > 0 and size(1 << 20, 10, 8) > size(1000, 10, 8)


def _ln_fwd(lib, **k):
    a = dict(n=4, d=8, dt=0, x=P, ldx=8, w=None, b=None, wdt=0, eps=1e-5, y=Q, ldy=8, m=None, r=None) | k
    return lib.hag_layer_norm_fwd(a["n"], a["d"], a["dt"], a["x"], a["ldx"], a["w"], a["b"], a["wdt"], a["eps"], a["y"], a["ldy"], a["m"], a["r"], None)


def _ln_bwd(lib, **k):
    a = dict(n=4, d=8, dt=0, g=P, ldg=8, x=Q, ldx=8, m=P, r=P, w=None, wdt=0, gx=R, ldgx=8, gw=P, gb=None, ws=P) | k
    return lib.hag_layer_norm_bwd(a["n"], a["d"], a["dt"], a["g"], a["ldg"], a["x"], a["ldx"], a["m"], a["r"], a["w"], a["wdt"], a["gx"], a["ldgx"],
                                  a["gw"], a["gb"], a["ws"], None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(n=-1), ARG), (dict(d=0), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG),
    (dict(ldy=7), ARG), (dict(ldx=-2), ARG), (dict(y=P, ldy=9), ARG), (dict(dt=3), DTYPE), (dict(wdt=3), DTYPE), (dict(x=P + 2), ALIGN),
    (dict(w=P + 2), ALIGN), (dict(b=P + 1, wdt=1), ALIGN), (dict(m=P + 2), ALIGN), (dict(d=(1 << 30) + 1, ldy=1 << 31), TOO_LARGE),
    (dict(n=0, x=None, y=None), 0)])
def test_layer_norm_forward(lib, change, status):
    assert _ln_fwd(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(g=None), NULL), (dict(x=None), NULL), (dict(gx=None), NULL), (dict(m=None), NULL), (dict(r=None), NULL), (dict(n=-1), ARG),
    (dict(d=-3), ARG), (dict(ldgx=7), ARG), (dict(ldg=-1), ARG), (dict(gx=P, ldgx=9), ARG), (dict(dt=2), DTYPE), (dict(wdt=2), DTYPE),
    (dict(gx=R + 2), ALIGN), (dict(gw=P + 2), ALIGN), (dict(gb=P + 1), ALIGN), (dict(r=P + 2), ALIGN), (dict(ws=P + 4), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(ws=None, gw=None, gb=Q), WORKSPACE), (dict(n=0, gw=None, ws=None, g=None, x=None, gx=None, m=None, r=None), 0)])
def test_layer_norm_backward(lib, change, status):
    assert _ln_bwd(lib, **change) == status


def test_layer_norm_workspace(lib):
    size = lib.hag_layer_norm_bwd_workspace_bytes
    assert size(-1, 8) == 0 and size(5, 0) == 0 and size(1000, 8) > 0


def _clip(lib, count=2, grads=(P, Q), out=(P, Q), lens=(4, 4), kinds=(0, 1), limit=1.0, norm=R, ws=P):
    arr = lambda kind, v: None if v is None else (kind * len(v))(*v)  # noqa: E731
    return lib.hag_clip_grad_norm(count, arr(vp, grads), arr(vp, out), arr(ctypes.c_int64, lens), arr(ctypes.c_int, kinds), limit, norm, ws, None)


@pytest.mark.parametrize("change,status", [
    (dict(count=-1), ARG), (dict(limit=-0.5), ARG), (dict(limit=float("nan")), ARG), (dict(lens=(4, -1)), ARG), (dict(grads=None), NULL),
    (dict(lens=None), NULL), (dict(kinds=None), NULL), (dict(out=None, norm=None), NULL), (dict(grads=(P, None)), NULL), (dict(out=(None, Q)), NULL),
    (dict(kinds=(0, 2)), DTYPE), (dict(grads=(P + 2, Q)), ALIGN), (dict(out=(P, Q + 1)), ALIGN), (dict(norm=R + 2), ALIGN), (dict(ws=P + 8), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(lens=(1 << 60, 4)), TOO_LARGE)])
def test_clip(lib, change, status):
    assert _clip(lib, **change) == status


def test_clip_workspace(lib):
    size = lib.hag_clip_grad_norm_workspace_bytes
    assert size(-1) == 0 and size(0) > 0 and size(10_000) > size(10)
