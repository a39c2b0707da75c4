"""The embedding, layer-norm and clipping entry points at the ends of their integers: refused before anything touches a
device, so tested without one.  Pointers are made-up addresses that no call may follow."""
import ctypes

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
