"""Embedding, layer norm and clipping where sizes and values are extreme: against plain 64-bit forms, u = 2^-24."""
import ctypes

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


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [5, 20, 36, 72, 200, 333, 1433, 4100, 9001, 16383])
@pytest.mark.parametrize("pad", [0, 5])
def test_layer_norm_gradient_of_large_constant_rows(d, dtype, pad):
    """xh is exactly 0 in every column (the sum of d equal powers of two is exact), so grad_x = rstd (q - mean q): an
    error of 2 u of each q, h + 2 of the mean, h = 64 + d/256 the longest chain of additions; one rounding for bf16.
    mean * rstd is above what fp32 holds."""
    x = torch.full((5, d + pad), 2.0 ** 112, device="cuda", dtype=dtype)[:, :d]
    g, w = _randn(1, 5, d).to(dtype), 1 + 0.2 * _randn(2, d)
    y, mean, rstd = hb.layer_norm_fwd(x, w, eps=1e-11)
    assert (mean == 2.0 ** 112).all() and not y.any() and float(mean[0]) * float(rstd[0]) > 2.0 ** 128
    gx, gw, gb = hb.layer_norm_bwd(g, x, mean, rstd, w)
    rs, q = rstd.double()[:, None], g.double() * w.double()
    want = rs * (q - q.mean(1, keepdim=True))
    bound = U * rs * (4 * q.abs() + (64 + d / 256 + 4) * q.abs().mean(1, keepdim=True)) + (2.0 ** -8 * want.abs() if dtype == BF16 else 0)
    assert ((gx.double() - want).abs() <= bound).all()
    assert not gw.any() and ((gb.double() - g.double().sum(0)).abs() <= 8 * U * g.double().abs().sum(0)).all()


def test_more_columns_than_32_bits_are_refused():
    """2^32 + 8 columns are not the 8 that their lower 32 bits say."""
    x = torch.zeros(1, (1 << 32) + 8, device="cuda", dtype=BF16)
    one = torch.zeros(1, device="cuda")
    for call in (lambda: hb.layer_norm_fwd(x, out=x), lambda: hb.layer_norm_bwd(x, x, one, one, out=x, param_grads=False),
                 lambda: hb.embedding_fwd(one.int(), x), lambda: hb.embedding_bwd(one.int(), x, 1)):
        with pytest.raises(hb.HagError) as e:
            call()
        assert e.value.status == hb.HAG_ERR_TOO_LARGE


def test_clipping_refuses_outputs_that_are_other_gradients():
    a, b, c, none = _randn(3, 5000), _randn(4, 5000), _randn(5, 5000), torch.empty(0, device="cuda")
    before = [t.clone() for t in (a, b, c)]
    for grads, out in (([a, b], [b, a]), ([a, b], [c, a]), ([a, b, c], [b, c, a]), ([a, none, b], [b, none, c])):
        with pytest.raises(ValueError):
            hb.clip_grad_norm(grads, 0.1, out=out)
    torch.cuda.synchronize()
    assert all(torch.equal(t, s) for t, s in zip((a, b, c), before))
    # some in place and some not, and several empty ones, are fine
    out, norm = hb.clip_grad_norm([a, none, none, b], 0.1, out=[a, none, none, c])
    want = torch.cat(before[:2]).double()
    assert abs(float(norm) - float(want.norm())) <= 33 * U * float(want.norm())
    got = torch.cat([a, c]).double()
    want *= 0.1 / (float(want.norm()) + 1e-6)
    assert ((got - want).abs() <= 40 * U * want.abs() + 1e-45).all() and torch.equal(b, before[1])


class _KernelNode(ctypes.Structure):
    """CUDA_KERNEL_NODE_PARAMS of the driver interface."""
    _fields_ = [("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3), ("shared", ctypes.c_uint),
                ("params", ctypes.c_void_p), ("extra", ctypes.c_void_p), ("kernel", ctypes.c_void_p), ("context", ctypes.c_void_p)]


def _launches(call):
    """[(kernel name, (x, y, z) blocks)] of what the call enqueues, read from a captured graph."""
    call()                                                          # one-time setup outside the capture
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    cuda, raw, count = ctypes.CDLL("libcuda.so.1"), ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert cuda.cuGraphGetNodes(raw, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert cuda.cuGraphGetNodes(raw, nodes, ctypes.byref(count)) == 0
    out = []
    for node in nodes:
        kind, p, name = ctypes.c_int(), _KernelNode(), ctypes.c_char_p()
        assert cuda.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        if kind.value != 0:                                         # not a kernel
            continue
        assert cuda.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(node), ctypes.byref(p)) == 0
        assert cuda.cuFuncGetName(ctypes.byref(name), ctypes.c_void_p(p.func)) == 0
        out.append((name.value.decode(), tuple(p.grid)))
    return out


def _ids(seed, n, v, kind):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "one":
        return torch.full((n,), v // 2, device="cuda", dtype=torch.int32)
    if kind == "skewed":
        return (torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) ** 6 * v).long().clamp(0, v - 1)
    ids = torch.randint(0, v, (n,), generator=gen, device="cuda")
    if kind == "holes":
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.3, -1, ids)
        ids[::7] = v
        ids[::13] = (1 << 40) + 1
    return ids


def _check_embedding_gradient(ids, grad, v, dtype):
    """A row of k terms goes through at most k + 2 fp32 roundings, each 2^-24 of the sum of magnitudes; bf16 adds 2^-8."""
    got = hb.embedding_bwd(ids, grad, v, scale=0.5, dtype=dtype)
    key = ids.long()
    ok = (key >= 0) & (key < v)
    rows, place = torch.unique(key[ok], return_inverse=True)        # only the rows that are named: v may be large
    g = grad[ok].double() * 0.5
    want = torch.zeros(len(rows), grad.shape[1], device="cuda", dtype=torch.float64).index_add_(0, place, g)
    mag = torch.zeros_like(want).index_add_(0, place, g.abs())
    k = torch.bincount(place, minlength=len(rows)).double()[:, None]
    bound = (k + 2) * U * mag + (2.0 ** -8 * want.abs() if dtype == BF16 else 0)
    assert ((got[rows].double() - want).abs() <= bound).all()
    got[rows] = 0
    assert not got.any()


@pytest.mark.parametrize("n,v,d", [(1, 16_384, 64), (64, 2048, 64), (64, 2049, 64), (64, 16_384, 64), (200, 65_536, 16), (256, 1024, 1024), (700, 1024, 512),
                                   (1000, 2560, 32), (1000, 2561, 32), (2000, 16_384, 64), (2000, 1 << 20, 1), (2048, 8000, 128), (4096, 8000, 64),
                                   (4978, 400, 336), (60_000, 1500, 128)])
def test_no_block_clears_a_large_table_alone(n, v, d):
    """2^17 values at most for a block of the embedding's gradient, 5 * 2^14 for more than 256 ids, and its result on both
    sides of that."""
    ids, grad = _ids(6, n, v, "uniform"), _randn(7, n, d)
    launches = _launches(lambda: hb.embedding_bwd(ids, grad, v))
    for name, grid in launches:
        if "embedding_tile" in name:
            assert v * d <= grid[1] * (1 << 17 if n <= 256 else 5 << 14), launches
        if "sort_small" in name:
            assert grid[0] > v * d * 4 >> 15                        # 32 KB of zeros per block besides the one that sorts
    for kind, gdt, odt in (("holes", F32, F32), ("skewed", BF16, F32), ("one", F32, BF16)):
        _check_embedding_gradient(_ids(8, n, v, kind), grad.to(gdt), v, odt)


@pytest.mark.parametrize("value", [0.1, 1000.1, -3e-5])
@pytest.mark.parametrize("d", [9, 72, 100, 333, 384, 1433, 20_001])
def test_constant_rows_whose_sum_is_rounded(value, d):
    """The mean is off by at most h u |value|, h = 64 + d/256 the longest chain of additions, plus its own rounding, and all
    differences from it by as much; y is that times rstd, which is 1 / sqrt(eps) at most.  Given that mean, the variance is
    the square of the difference, and rstd good to (h/2 + 10) u."""
    x = torch.full((6, d), value, device="cuda")
    eps = 1e-5
    y, mean, rstd = hb.layer_norm_fwd(x, eps=eps)
    dm = (65 + d / 256) * U * abs(value)
    assert ((mean.double() - x[:, 0].double()).abs() <= dm).all() and (rstd <= eps ** -0.5 * (1 + 8 * U)).all()
    assert (y.double().abs() <= dm * eps ** -0.5 * (1 + 12 * U)).all()
    want = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    assert ((y.double() - want).abs() <= 4 * U * want.abs()).all()
    off = x[:, 0].double() - mean.double()
    assert ((rstd.double() * (off.square() + eps).sqrt() - 1).abs() <= (42 + d / 512) * U).all()


def test_parameter_gradients_beyond_32_bits():
    """gw and gb of 2.46e9 elements: no chain of additions over n rows is longer than k = 128 + n/32, so (4 + k) u of the
    sum of magnitudes for gw and k u for gb."""
    n, d = 150_000, 16_384
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.empty(n, d, dtype=BF16, device="cuda").normal_(generator=gen)
    g = torch.empty(n, d, dtype=BF16, device="cuda").normal_(generator=gen)
    y, mean, rstd = hb.layer_norm_fwd(x)
    gx, gw, gb = hb.layer_norm_bwd(g, x, mean, rstd, out=y)
    sums = torch.zeros(4, d, device="cuda", dtype=torch.float64)
    for a in range(0, n, 5000):
        gd = g[a:a + 5000].double()
        t = gd * (x[a:a + 5000].double() - mean[a:a + 5000].double()[:, None]) * rstd[a:a + 5000].double()[:, None]
        sums += torch.stack([t.sum(0), t.abs().sum(0), gd.sum(0), gd.abs().sum(0)])
    k = 128 + n / 32
    assert ((gw.double() - sums[0]).abs() <= (4 + k) * U * sums[1]).all() and ((gb.double() - sums[2]).abs() <= k * U * sums[3]).all()


@pytest.mark.parametrize("n,v,d,ld", [(9000, 50, 16, 300_000), (200, 30, 24, 15_000_000)])
def test_table_gradient_of_few_rows_beyond_32_bits(n, v, d, ld):
    """Gradient rows so far apart that their offsets pass 32 bits, in tiles and in one tile."""
    wide = torch.empty(n, ld, dtype=BF16, device="cuda")
    grad = wide[:, 5:5 + d]
    grad.copy_(_randn(10, n, d))
    ids = _ids(11, n, v, "uniform")
    assert any("embedding_tile" in name for name, _ in _launches(lambda: hb.embedding_bwd(ids, grad, v)))
    for kind in ("uniform", "holes"):
        _check_embedding_gradient(_ids(11, n, v, kind), grad, v, F32)


@pytest.mark.parametrize("kind", ["uniform", "one", "skewed", "holes"])
@pytest.mark.parametrize("n,v,d", [(1, 50_257, 64), (65, 50_257, 33), (300, 50_257, 96), (1024, 40_000, 40), (1025, 70_000, 20), (4096, 50_257, 128),
                                   (8192, 1 << 18, 8), (8191, 20_000, 333), (5001, 300_001, 5), (700, 1 << 21, 1)])
def test_short_lists_into_large_tables(kind, n, v, d):
    """All passes of the sort in one launch, from one key per thread to eight, one to three digits."""
    ids, grad = _ids(13, n, v, kind), _randn(12, n, d)
    assert any("sort_small" in name for name, _ in _launches(lambda: hb.embedding_bwd(ids, grad, v)))
    for gdt, odt in ((F32, F32), (BF16, F32), (F32, BF16)):
        _check_embedding_gradient(ids, grad.to(gdt), v, odt)


@pytest.mark.parametrize("n", [6000, 100_001])
def test_four_digits(n):
    """2^25 rows, 26 bits of key in four passes, in one launch and in two per pass; among the ids the first and the last."""
    v = 1 << 25
    ids = _ids(14, n, v, "uniform")
    ids[5], ids[77], ids[n - 1], ids[n - 2] = 0, v - 1, v - 1, -1
    ids[100:1100] = 1 << 24
    for d in (1, 2):
        _check_embedding_gradient(ids, _randn(15, n, d), v, F32)
