"""GPU parity of the embedding (rows of a table by ids, and the table's gradient) against plain 64-bit forms.

Forward: the kernel rounds the product to fp32 and that to the output type, so the result is compared bit for bit.
Backward: a row of k terms passes through at most k + 2 fp32 roundings (k additions in some fixed order, the product
with the scale, the store), each at most 2^-24 of the sum of magnitudes; a bf16 result adds one rounding (2^-8).
"""
import ctypes

import numpy as np
import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ids(seed, n, v, kind="uniform", dtype=torch.int64):
    g = _gen(seed)
    if kind == "one":
        ids = torch.full((n,), v // 2, device="cuda")
    elif kind == "skewed":
        ids = (torch.rand(n, generator=g, device="cuda") ** 6 * v).long().clamp(0, v - 1)
    else:
        ids = torch.randint(0, v, (n,), generator=g, device="cuda")
    if kind == "holes":
        ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.3, torch.full_like(ids, -1), ids)
        ids[::7] = v
        ids[::11] = v + 12345
        if dtype == torch.int64:
            ids[::13] = (1 << 40) + 1
    return ids.to(dtype)


def _forward_want(ids, table, scale, dtype):
    ids = ids.long()
    ok = (ids >= 0) & (ids < table.shape[0])
    rows = table.double()[ids.clamp(0, table.shape[0] - 1)] * float(np.float32(scale))
    rows[~ok] = 0
    return rows.float().to(dtype)


def _check_backward(ids, grad, v, scale, dtype, out=None):
    got = hb.embedding_bwd(ids, grad, v, scale=scale, dtype=dtype, out=out)
    key = ids.long()
    ok = (key >= 0) & (key < v)
    key, g = key[ok], grad[ok].double() * float(np.float32(scale))
    want = torch.zeros(v, grad.shape[1], device="cuda", dtype=torch.float64).index_add_(0, key, g)
    mag = torch.zeros_like(want).index_add_(0, key, g.abs())
    k = torch.bincount(key, minlength=v).double()[:, None]
    bound = (k + 2) * U * mag
    if dtype == BF16:
        bound += 2.0 ** -8 * want.abs()
    err = (got.double() - want).abs()
    assert (err <= bound).all(), f"worst {(err - bound).max().item():.3e}"
    assert not got[(k == 0).squeeze(1)].any()
    return got


@pytest.mark.parametrize("table_dtype,dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,v,d", [(1, 5, 8), (1, 1, 4096), (1000, 1000, 16), (4099, 119, 64), (333, 7, 1), (517, 50, 33), (70, 9, 1002),
                                   (2500, 3000, 100), (65, 20, 8200)])
def test_forward_is_exact_to_its_roundings(table_dtype, dtype, n, v, d):
    table = torch.randn(v, d, generator=_gen(1), device="cuda").to(table_dtype)
    for kind, it, scale in (("uniform", torch.int64, 1.0), ("holes", torch.int32, 0.3), ("holes", torch.int64, 16.0)):
        ids = _ids(2, n, v, kind, it)
        got = hb.embedding_fwd(ids, table, scale=scale, dtype=dtype)
        assert got.dtype == dtype and torch.equal(got, _forward_want(ids, table, scale, dtype))


def test_forward_strides_offsets_and_values_behind_holes():
    wide = torch.randn(40, 200, generator=_gen(3), device="cuda")
    wide[5] = float("nan")
    wide[6, ::2] = float("inf")
    ids = torch.tensor([0, -1, 39, 7, 40, 7, 12], device="cuda")
    for lo, hi in ((0, 64), (1, 65), (2, 66), (3, 100), (4, 4 + 128)):
        table = wide[:, lo:hi]
        buf = torch.full((7, 300), 7.0, device="cuda")
        out = buf[:, 9:9 + hi - lo]
        assert hb.embedding_fwd(ids, table, scale=2.0, out=out) is out
        assert torch.equal(out, _forward_want(ids, table, 2.0, F32))
        assert (buf[:, :9] == 7).all() and (buf[:, 9 + hi - lo:] == 7).all()       # nothing beside it is touched
    bad = torch.tensor([5, -1, 6], device="cuda")
    got = hb.embedding_fwd(bad, wide, scale=1.0)
    assert got[0].isnan().all() and not got[1].any() and torch.equal(got[2], wide[6])


@pytest.mark.parametrize("kind", ["uniform", "skewed", "one", "holes"])
@pytest.mark.parametrize("n,v,d", [(1, 1, 4), (1, 300, 8), (31, 2, 1), (1000, 100, 16), (4096, 119, 64), (4097, 255, 33), (5000, 256, 24),
                                   (9001, 70000, 40), (20011, 5, 128), (300, 40, 1100)])
def test_backward_against_the_definition(kind, n, v, d):
    for it, gdt, odt, scale in ((torch.int64, F32, F32, 1.0), (torch.int32, BF16, F32, 0.3), (torch.int32, BF16, BF16, 16.0),
                                (torch.int64, F32, BF16, 2.0)):
        ids = _ids(4, n, v, kind, it)
        grad = torch.randn(n, d, generator=_gen(5), device="cuda").to(gdt)
        _check_backward(ids, grad, v, scale, odt)


@pytest.mark.parametrize("n,v,d,kind", [(300_001, 50_257, 64, "skewed"), (700_000, 3, 32, "uniform"), (1_300_000, 1 << 20, 8, "uniform"),
                                        (262_144, 119, 72, "one"), (100_003, 2000, 520, "skewed")])
def test_backward_of_long_lists(n, v, d, kind):
    """Several stretches per block, one to three digits, rows whose terms span many warps."""
    ids = _ids(6, n, v, kind, torch.int32)
    grad = torch.randn(n, d, generator=_gen(7), device="cuda").to(BF16)
    _check_backward(ids, grad, v, 1.0, F32)


def test_backward_of_integers_is_exact_and_runs_repeat():
    ids = _ids(8, 50_000, 400, "skewed", torch.int32)
    grad = torch.randint(-8, 9, (50_000, 36), generator=_gen(9), device="cuda").float()
    want = torch.zeros(400, 36, device="cuda", dtype=torch.float64).index_add_(0, ids.long(), grad.double())
    a = hb.embedding_bwd(ids, grad, 400)
    assert torch.equal(a.double(), want)
    noise = torch.randn(50_000, 36, generator=_gen(10), device="cuda")
    assert torch.equal(hb.embedding_bwd(ids, noise, 400), hb.embedding_bwd(ids, noise, 400))


def test_backward_strides_broadcast_gradient_and_rows_nobody_named():
    ids = _ids(11, 3000, 90, "holes", torch.int64)
    wide = torch.randn(3000, 101, generator=_gen(12), device="cuda")
    for lo, hi in ((0, 64), (1, 65), (3, 50), (5, 6)):
        buf = torch.full((90, 130), 3.0, device="cuda")
        out = buf[:, 7:7 + hi - lo]
        _check_backward(ids, wide[:, lo:hi], 90, 0.5, F32, out=out)
        assert (buf[:, :7] == 3).all() and (buf[:, 7 + hi - lo:] == 3).all()
    row = torch.randn(1, 48, generator=_gen(13), device="cuda")
    _check_backward(ids, row.expand(3000, 48), 90, 1.0, F32)                       # the same row for every token
    out = torch.full((1000, 16), float("nan"), device="cuda")
    hb.embedding_bwd(torch.tensor([3, -1], device="cuda"), torch.ones(2, 16, device="cuda"), 1000, out=out)
    assert (out[3] == 1).all() and out.abs().sum() == 16
    # gradients of places that hold no token are not looked at
    g = torch.randn(3000, 8, generator=_gen(14), device="cuda")
    g[(ids < 0) | (ids >= 90)] = float("nan")
    assert hb.embedding_bwd(ids, g, 90).isfinite().all()


def test_gradient_is_the_derivative_of_the_forward_call():
    """<g, f(T + h E) - f(T - h E)> / 2h for single entries E: the map is linear and the values are small integers, so
    both sides are exact."""
    ids = _ids(15, 200, 12, "holes", torch.int64)
    g = torch.randint(-4, 5, (200, 5), generator=_gen(16), device="cuda").float()
    table = torch.randint(-4, 5, (12, 5), generator=_gen(17), device="cuda").float()
    grad = hb.embedding_bwd(ids, g, 12, scale=0.5)
    for r in range(12):
        for c in (0, 4):
            up, down = table.clone(), table.clone()
            up[r, c] += 1
            down[r, c] -= 1
            diff = (hb.embedding_fwd(ids, up, 0.5).double() - hb.embedding_fwd(ids, down, 0.5).double())
            assert float((diff * g.double()).sum() / 2) == float(grad[r, c])


def test_empty_calls():
    table = torch.ones(4, 8, device="cuda")
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert hb.embedding_fwd(none, table).shape == (0, 8)
    assert not hb.embedding_bwd(none, torch.zeros(0, 8, device="cuda"), 4).any()
    ids = torch.tensor([0, 1], device="cuda")
    assert not hb.embedding_fwd(ids, torch.zeros(0, 8, device="cuda")).any()       # a table without rows: no id names one
    assert hb.embedding_bwd(ids, torch.ones(2, 8, device="cuda"), 0).shape == (0, 8)


def test_offsets_beyond_32_bits():
    n, d = 150_000, 16_384                          # 2.46e9 elements each way
    table = torch.randn(1000, d, generator=_gen(18), device="cuda").to(BF16)
    ids = _ids(19, n, 1000, "uniform", torch.int32)
    out = hb.embedding_fwd(ids, table)
    for r in (0, 131_071, 131_072, 140_001, n - 1):
        assert torch.equal(out[r], table[int(ids[r])])
    part = hb.embedding_bwd(ids, out, 1000, dtype=F32)
    counts = torch.bincount(ids.long(), minlength=1000).double()[:, None]
    want = table.double() * counts
    assert ((part.double() - want).abs() <= (counts + 2) * U * want.abs()).all()


def test_other_streams_and_graph_capture():
    ids = _ids(20, 6000, 500, "skewed", torch.int32)
    grad = torch.randn(6000, 40, generator=_gen(21), device="cuda")
    want = hb.embedding_bwd(ids, grad, 500)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        scaled = grad * 2
        got = hb.embedding_bwd(ids, scaled, 500, scale=0.5)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    ws = torch.empty(hb.load_library().hag_embedding_bwd_workspace_bytes(6000, 500, 40), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hb.embedding_bwd(ids, grad, 500, out=out, workspace=ws)
    out.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_refusals():
    lib = hb.load_library()
    vp = ctypes.c_void_p
    ids, table = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(3, 8, device="cuda")
    out = torch.full((4, 8), 5.0, device="cuda")
    with pytest.raises(ValueError):
        hb.embedding_fwd(ids, table.t())                            # rows not contiguous
    with pytest.raises(ValueError):
        hb.embedding_fwd(ids[::2], table)
    with pytest.raises(TypeError):
        hb.embedding_fwd(ids.float(), table)
    with pytest.raises(TypeError):
        hb.embedding_fwd(ids, table.half())
    with pytest.raises(ValueError):
        hb.embedding_fwd(ids, table, out=out[:3])
    with pytest.raises(ValueError):
        hb.embedding_bwd(ids, out[:3], 3)
    with pytest.raises(ValueError):
        hb.embedding_bwd(ids, out, 3, workspace=torch.empty(16, device="cuda"))
    with pytest.raises(hb.HagError) as e:
        hb.embedding_fwd(ids, table, out=torch.empty(1, 8, device="cuda").expand(4, 8))
    assert e.value.status == hb.HAG_ERR_ARG
    assert lib.hag_embedding_fwd(vp(ids.data_ptr() + 2), 0, 1, 3, vp(table.data_ptr()), 0, 8, 0, 8, 1.0, vp(out.data_ptr()), 8, None) == hb.HAG_ERR_ALIGN
    assert lib.hag_embedding_fwd(vp(ids.data_ptr()), 0, 1, 3, vp(table.data_ptr()), 0, 8, 0, 8, 1.0, vp(table.data_ptr()), 8, None) == hb.HAG_ERR_ARG
    torch.cuda.synchronize()
    assert (out == 5).all()


@pytest.mark.parametrize("n,v,d", [(40, 7, 12), (5000, 90, 33), (30_000, 40_000, 20)])
def test_a_batch_without_a_single_token(n, v, d):
    table = torch.full((v, d), float("nan"), device="cuda")
    for ids in (torch.full((n,), -1, device="cuda"), torch.full((n,), v, dtype=torch.int32, device="cuda")):
        assert not hb.embedding_fwd(ids, table).any()
        out = torch.full((v, d), float("nan"), device="cuda")
        hb.embedding_bwd(ids, torch.full((n, d), float("inf"), device="cuda"), v, out=out)
        assert not out.any()


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("n,v,d", [(200, 30, 24), (3000, 100, 72), (20_000, 9000, 65)])
def test_matrices_that_begin_anywhere(n, v, d, offset):
    ids = _ids(22, n, v, "holes", torch.int32)
    for dtype in (F32, BF16):
        grad = torch.randn(n * d + offset, generator=_gen(23), device="cuda").to(dtype)[offset:].view(n, d)
        buf = torch.full((v * d + offset + 9,), 3.0, device="cuda", dtype=dtype)
        out = buf[offset:offset + v * d].view(v, d)
        _check_backward(ids, grad, v, 0.5, dtype, out=out)
        assert (buf[:offset] == 3).all() and (buf[offset + v * d:] == 3).all()
        rows = torch.full((n * d + offset + 9,), 3.0, device="cuda", dtype=dtype)
        got = hb.embedding_fwd(ids, out, 2.0, out=rows[offset:offset + n * d].view(n, d))
        assert torch.equal(got, _forward_want(ids, out, 2.0, dtype)) and (rows[:offset] == 3).all() and (rows[offset + n * d:] == 3).all()
