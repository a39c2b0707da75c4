"""The embedding, layer-norm and clipping entry points at the ends of their integers: refused before anything touches a
device, so tested without one.  Pointers are made-up addresses that no call may follow."""
import ctypes
import os
import re

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

P, Q, R = 0x10000, 0x20000, 0x30000           # 16-byte aligned, never read


@pytest.fixture(scope="module")
def lib():
    build_library()
    return hb.load_library()


def _clip(lib, lens, kinds=(0, 1), grads=(P, Q)):
    arr = lambda kind, v: (kind * len(v))(*v)  # noqa: E731
    return lib.hag_clip_grad_norm(len(lens), arr(ctypes.c_void_p, grads), arr(ctypes.c_void_p, grads), arr(ctypes.c_int64, lens),
                                  arr(ctypes.c_int, kinds), 1.0, R, P, None)


@pytest.mark.parametrize("lens", [((1 << 63) - 1, 4), (4, (1 << 63) - 1), ((1 << 63) - 1, (1 << 63) - 1), ((1 << 63) - 8191, 1), (1 << 44, 1)])
def test_clipping_refuses_any_length_it_cannot_count(lib, lens):
    """2^31 - 1 pieces of 32 KB are the most of a launch: 2^44 - 2^13 fp32 or 2^45 - 2^14 bf16 values."""
    if lens[1] >> 62:
        assert _clip(lib, lens, kinds=(1, 1)) == hb.HAG_ERR_TOO_LARGE
    assert _clip(lib, lens) == hb.HAG_ERR_TOO_LARGE


def test_clipping_refuses_more_tensors_than_it_can_count(lib):
    """2^28 tensors are the most of a call; the lists of a longer one are not read."""
    size = lib.hag_clip_grad_norm_workspace_bytes
    assert size(1 << 28) > size((1 << 28) - 200) > size(129) > size(128) and size((1 << 28) + 1) == 0 and size((1 << 31) - 1) == 0
    for count in ((1 << 28) + 1, (1 << 31) - 1):
        assert lib.hag_clip_grad_norm(count, P, P, P, P, 1.0, R, P, None) == hb.HAG_ERR_TOO_LARGE
        assert lib.hag_clip_grad_norm(count, None, P, P, P, 1.0, R, P, None) == hb.HAG_ERR_NULL


def _gradient(lib, n=4, v=9, d=8, ws=P + 8):
    """A call that, where its sizes are accepted, is refused for its workspace (not on 16 bytes)."""
    return lib.hag_embedding_bwd(P, 0, n, v, 0, d, Q, d, 1.0, R, 0, d, ws, None)


def test_embedding_gradient_takes_the_sizes_that_the_header_names(lib):
    size = lib.hag_embedding_bwd_workspace_bytes
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hag.h")).read()
    n = (1 << 31) - int(re.search(r"backward: n >= 2\^31 - (\d+)\)", header).group(1)) - 1
    v, d = (1 << 31) - 2, 1 << 20
    for ok in (dict(n=n), dict(v=v), dict(d=d), dict(n=n, v=v), dict(n=n, d=d)):
        assert _gradient(lib, **ok) == hb.HAG_ERR_ALIGN and size(*((dict(n=4, v=9, d=8) | ok).values())) > 0
    for bad in (dict(n=n + 1), dict(n=n + 4096), dict(v=v + 1), dict(d=d + 1), dict(n=1 << 62)):
        assert _gradient(lib, **bad) == hb.HAG_ERR_TOO_LARGE


def test_embedding_lookup_takes_the_sizes_that_the_header_names(lib):
    def call(v=9, d=8, ids=P + 2):                              # ids not on their element
        return lib.hag_embedding_fwd(ids, 0, 4, v, Q, 0, d, 0, d, 1.0, R, d, None)
    assert call(v=(1 << 31) - 2) == call(d=1 << 20) == hb.HAG_ERR_ALIGN
    assert call(v=(1 << 31) - 1) == call(d=(1 << 20) + 1) == hb.HAG_ERR_TOO_LARGE


def test_layer_norm_takes_the_widths_that_the_header_names(lib):
    def call(d, x=P + 2):
        return lib.hag_layer_norm_fwd(4, d, 0, x, d, None, None, 0, 1e-5, Q, d, None, None, None)
    assert call(1 << 30) == hb.HAG_ERR_ALIGN and call((1 << 30) + 1) == hb.HAG_ERR_TOO_LARGE
