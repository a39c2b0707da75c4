"""GPU parity of layer norm, forward and backward, against plain 64-bit forms.

Bounds, with u = 2^-24, D columns and h = 64 + D/256 the longest chain of fp32 additions a row sum goes through:
  mean    |dm| <= h u mean|x|                     (plus u |mean| for the store)
  rstd    relative (h/2 + 10) u + dm^2 / (2 var): the squares' sum, the division, the 2-ulp reciprocal square root
  y       |xh w| (h/2 + 14) u + rstd |w| dm + 2 u |y|
  grad_x  u rstd [8 |q| + (h + 8) mean|q| + (h + 16) |xh| mean|q xh|]
  grad_w  (4 + k) u sum|g xh|, grad_b k u sum|g|, where no chain of additions over n rows is longer than k = 128 + n/32
bf16 results add one rounding, 2^-8 of the value.
"""
import ctypes

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def _inside(got, want, bound, what):
    if got.dtype == BF16:
        bound = bound + 2.0 ** -8 * want.abs()
    err = (got.double() - want).abs()
    assert (err <= bound + 1e-45).all(), f"{what}: worst {(err - bound).max().item():.3e}"


def _stats(x):
    x = x.double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, var, (var + EPS).rsqrt()


def _check_forward(x, w, b, out=None):
    d = x.shape[1]
    h = 64 + d / 256
    mean, var, rstd = _stats(x)
    dm = h * U * x.double().abs().mean(1)
    xh = (x.double() - mean[:, None]) * rstd[:, None]
    wd = torch.ones(d, device="cuda", dtype=torch.float64) if w is None else w.double()
    want = xh * wd + (0 if b is None else b.double())
    y, m, r = hb.layer_norm_fwd(x, w, b, eps=EPS, out=out)
    rel = (h / 2 + 10) * U + dm.square() / (2 * (var + EPS))
    _inside(m, mean, dm + U * mean.abs(), "mean")
    _inside(r, rstd, rel * rstd, "rstd")
    bound = (xh * wd).abs() * (rel[:, None] + 4 * U) + rstd[:, None] * wd.abs() * dm[:, None] + 2 * U * want.abs()
    _inside(y, want, bound, "y")
    return y, m, r


def _check_backward(g, x, w, param_dtype=None, out=None):
    n, d = x.shape
    h, k = 64 + d / 256, 128 + n / 32
    mean, _, rstd = _stats(x)
    mean, rstd = mean.float(), rstd.float()
    gd, xd = g.double().clone(), x.double().clone()
    gx, gw, gb = hb.layer_norm_bwd(g, x, mean, rstd, w, out=out, param_dtype=param_dtype)
    rs = rstd.double()[:, None]
    xh = (xd - mean.double()[:, None]) * rs
    q = gd if w is None else gd * w.double()
    aq, aqx = q.abs().mean(1, keepdim=True), (q * xh).abs().mean(1, keepdim=True)
    want = rs * (q - q.mean(1, keepdim=True) - xh * (q * xh).mean(1, keepdim=True))
    _inside(gx, want, U * rs * (8 * q.abs() + (h + 8) * aq + (h + 16) * xh.abs() * aqx), "grad_x")
    _inside(gw, (gd * xh).sum(0), (4 + k) * U * (gd * xh).abs().sum(0), "grad_weight")
    _inside(gb, gd.sum(0), k * U * gd.abs().sum(0), "grad_bias")
    return gx, gw, gb


SHAPES = [(1, 1), (1, 4096), (1, 16385), (3, 2), (1000, 16), (257, 20), (5000, 64), (1001, 128), (777, 33), (640, 256), (300, 250), (129, 515),
          (90, 1024), (66, 1433), (40, 2048), (31, 4100), (12, 8192), (9, 16384), (5, 16386), (3, 40001)]


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_forward(n, d, dtype):
    x = (_randn(1, n, d) * 1.5 + _randn(2, d)).to(dtype)
    w, b = 1 + 0.2 * _randn(3, d), 0.3 * _randn(4, d)
    _check_forward(x, w, b)
    _check_forward(x, w.to(BF16), b.to(BF16))
    _check_forward(x, None, None)
    _check_forward(x, w, None)
    _check_forward(x, None, b)


@pytest.mark.parametrize("n,d", SHAPES + [(20_011, 64), (40_000, 24), (3000, 1024), (70_001, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_backward(n, d, dtype):
    x = (_randn(5, n, d) * 1.5 + _randn(6, d)).to(dtype)
    g, w = _randn(7, n, d).to(dtype), 1 + 0.2 * _randn(8, d)
    _check_backward(g, x, w)
    _check_backward(g, x, w.to(BF16))
    _check_backward(g, x, None, param_dtype=F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_offsets_and_in_place(dtype):
    wide, gwide, params = _randn(9, 70, 700).to(dtype), _randn(10, 70, 650).to(dtype), _randn(11, 2, 701)
    for lo, d in ((0, 64), (1, 64), (2, 30), (4, 128), (8, 512), (3, 601), (5, 1)):
        x, g, w, b = wide[:, lo:lo + d], gwide[:, lo + 1:lo + 1 + d], params[0, lo:lo + d], params[1, lo:lo + d]
        buf = torch.full((70, 720), 3.0, device="cuda", dtype=dtype)
        y, m, r = _check_forward(x, w, b, out=buf[:, 9:9 + d])
        assert (buf[:, :9] == 3).all() and (buf[:, 9 + d:] == 3).all()
        _check_forward(x.contiguous(), w, b)
        xin = x.contiguous().clone()                                # the same layout: the same bits
        want = hb.layer_norm_fwd(x.contiguous(), w, b, eps=EPS)[0]
        assert hb.layer_norm_fwd(xin, w, b, eps=EPS, out=xin)[0] is xin and torch.equal(xin, want)
        buf.fill_(3.0)
        gx, gw, gb = _check_backward(g, x, w, out=buf[:, 9:9 + d])
        assert (buf[:, :9] == 3).all() and (buf[:, 9 + d:] == 3).all()
        # the result may take the place of either input
        for k in (0, 1):
            ins = [g.contiguous().clone(), x.contiguous().clone()]
            got = hb.layer_norm_bwd(ins[0], ins[1], m, r, w, out=ins[k])
            same = hb.layer_norm_bwd(g.contiguous(), x.contiguous(), m, r, w)
            assert all(torch.equal(p, q) for p, q in zip(got, same))
    row = _randn(12, 1, 96).to(dtype)                               # one gradient row for all rows, as of a sum
    _check_backward(row.expand(50, 96), wide[:50, :96], params[0, :96])
    # in place where the row is too wide to be held in registers
    x, g = _randn(13, 4, 40_000).to(dtype), _randn(14, 4, 40_000).to(dtype)
    y, m, r = hb.layer_norm_fwd(x)
    xin = x.clone()
    assert torch.equal(hb.layer_norm_fwd(xin, out=xin)[0], y)
    want = hb.layer_norm_bwd(g, x, m, r)
    for k in (0, 1):
        ins = [g.clone(), x.clone()]
        assert all(torch.equal(p, q) for p, q in zip(hb.layer_norm_bwd(*ins, m, r, out=ins[k]), want))


def test_mean_far_from_zero_and_constant_rows():
    """A spread of 1 around 1000: sums of squares would cancel; the two-step variance does not."""
    x = _randn(15, 300, 384) + 1000
    _check_forward(x, None, None)
    flat = torch.full((10, 72), 2.5, device="cuda")
    y, m, r = hb.layer_norm_fwd(flat, None, torch.ones(72, device="cuda"), eps=EPS)
    assert (y == 1).all() and (m == 2.5).all()


def test_rows_with_infinities_stay_alone():
    x = _randn(16, 40, 200)
    clean = hb.layer_norm_fwd(x)[0]
    x[7, 3], x[20, 0] = float("inf"), float("nan")
    y = hb.layer_norm_fwd(x)[0]
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[7, 20]] = False
    assert torch.equal(y[keep], clean[keep]) and y[7].isnan().any() and y[20].isnan().all()


def test_gradient_against_differences():
    """Central differences of the 64-bit loss <g, y(x, w, b)>; step 1e-4, so the third-order term is about 1e-8."""
    n, d = 6, 48
    x, g, w, b = _randn(17, n, d), _randn(18, n, d), 1 + 0.2 * _randn(19, d), 0.3 * _randn(20, d)
    y, m, r = hb.layer_norm_fwd(x, w, b, eps=EPS)
    gx, gw, gb = hb.layer_norm_bwd(g, x, m, r, w)

    def loss(x, w, b):
        mean, _, rstd = _stats(x)
        return ((((x - mean[:, None]) * rstd[:, None]) * w + b) * g.double()).sum()

    ins = [x.double(), w.double(), b.double()]
    for which, got in enumerate((gx, gw, gb)):
        for at in range(0, got.numel(), 13):
            side = []
            for s in (1e-4, -1e-4):
                moved = [t.clone() for t in ins]
                moved[which].view(-1)[at] += s
                side.append(loss(*moved))
            want = float(side[0] - side[1]) / 2e-4
            assert abs(float(got.view(-1)[at]) - want) <= 2e-5 * (1 + abs(want))


def test_runs_repeat_and_no_rows():
    x, g, w = _randn(21, 9000, 100), _randn(22, 9000, 100), _randn(23, 100)
    y, m, r = hb.layer_norm_fwd(x, w)
    a, b = hb.layer_norm_bwd(g, x, m, r, w), hb.layer_norm_bwd(g, x, m, r, w)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    gx, gw, gb = hb.layer_norm_bwd(g, x, m, r, w, param_grads=False)
    assert torch.equal(gx, a[0]) and gw is None and gb is None
    assert hb.layer_norm_fwd(x, w, stats=False)[1] is None
    empty = x[:0]
    y, m, r = hb.layer_norm_fwd(empty, w)
    assert y.shape == (0, 100) and m.shape == (0,)
    gx, gw, gb = hb.layer_norm_bwd(empty, empty, m, r, w)
    assert gx.shape == (0, 100) and not gw.any() and not gb.any()


@pytest.mark.parametrize("d", [1, 7, 100, 333, 1433, 9001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows_of_any_width(d, dtype):
    empty, w, none = torch.empty(0, d, device="cuda", dtype=dtype), _randn(31, d), torch.empty(0, device="cuda")
    y, m, r = hb.layer_norm_fwd(empty, w)
    assert y.shape == (0, d) and m.shape == (0,)
    gx, gw, gb = hb.layer_norm_bwd(empty, empty, none, none, w)
    assert gx.shape == (0, d) and not gw.any() and not gb.any()


def test_one_of_the_parameter_gradients():
    lib, vp = hb.load_library(), ctypes.c_void_p
    x, g, w = _randn(24, 500, 72), _randn(25, 500, 72), _randn(26, 72)
    y, m, r = hb.layer_norm_fwd(x, w)
    gx, gw, gb = hb.layer_norm_bwd(g, x, m, r, w)
    ws = torch.empty(lib.hag_layer_norm_bwd_workspace_bytes(500, 72), dtype=torch.uint8, device="cuda")
    for k in (0, 1):
        gx2, one = torch.empty_like(x), torch.empty_like(w)
        pair = [None, None]
        pair[k] = vp(one.data_ptr())
        st = lib.hag_layer_norm_bwd(500, 72, 0, vp(g.data_ptr()), 72, vp(x.data_ptr()), 72, vp(m.data_ptr()), vp(r.data_ptr()),
                                    vp(w.data_ptr()), 0, vp(gx2.data_ptr()), 72, pair[0], pair[1], vp(ws.data_ptr()),
                                    torch.cuda.current_stream().cuda_stream)
        assert st == 0 and torch.equal(gx2, gx) and torch.equal(one, (gw, gb)[k])


def test_offsets_beyond_32_bits():
    n, d = 150_000, 16_384
    x = torch.empty(n, d, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(27))
    y, m, r = hb.layer_norm_fwd(x)
    rows = torch.tensor([0, 131_071, 131_072, 140_001, n - 1], device="cuda")
    part = hb.layer_norm_fwd(x[rows])[0]
    assert torch.equal(y[rows], part)
    gx, _, _ = hb.layer_norm_bwd(x, x, m, r, out=y)
    assert torch.equal(gx[rows], hb.layer_norm_bwd(x[rows], x[rows], m[rows].contiguous(), r[rows].contiguous())[0])


def test_other_streams_and_graph_capture():
    x, g, w = _randn(28, 3000, 80), _randn(29, 3000, 80), _randn(30, 80)
    y, m, r = hb.layer_norm_fwd(x, w)
    want = hb.layer_norm_bwd(g, x, m, r, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x2 = x * 1
        y2, m2, r2 = hb.layer_norm_fwd(x2, w)
        got = hb.layer_norm_bwd(g, x2, m2, r2, w)
    side.synchronize()
    assert torch.equal(y2, y) and all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, m3, r3 = hb.layer_norm_fwd(x, w)
        got = hb.layer_norm_bwd(g, x, m3, r3, w)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y3, y) and all(torch.equal(p, q) for p, q in zip(got, want))


def test_refusals():
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda")
    y, m, r = hb.layer_norm_fwd(x, w)
    with pytest.raises(ValueError):
        hb.layer_norm_fwd(x.t(), None)
    with pytest.raises(ValueError):
        hb.layer_norm_fwd(x, w[:4])
    with pytest.raises(TypeError):
        hb.layer_norm_fwd(x, w, w.to(BF16))
    with pytest.raises(TypeError):
        hb.layer_norm_fwd(x.double(), None)
    with pytest.raises(TypeError):
        hb.layer_norm_bwd(x.to(BF16), x, m, r, w)
    with pytest.raises(ValueError):
        hb.layer_norm_bwd(x, x, m[:2], r, w)
    with pytest.raises(hb.HagError) as e:
        hb.layer_norm_fwd(x, w, eps=-1.0)
    assert e.value.status == hb.HAG_ERR_ARG
    with pytest.raises(hb.HagError) as e:
        hb.layer_norm_fwd(x, w, out=torch.empty(1, 8, device="cuda").expand(4, 8))
    assert e.value.status == hb.HAG_ERR_ARG


def _at(t, offset):
    """A contiguous copy of t that begins `offset` elements into its storage, with a guard value on both sides."""
    buf = torch.full((t.numel() + offset + 9,), 3.0, device="cuda", dtype=t.dtype)
    view = buf[offset:offset + t.numel()].view(t.shape)
    view.copy_(t)
    return view, buf


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d", [(1, 129), (3, 333), (77, 130), (300, 256), (41, 515), (19, 1433), (9, 5363), (5, 9999), (23, 1024)])
@pytest.mark.parametrize("x_at,g_at,y_at", [(1, 1, 1), (0, 0, 0), (5, 5, 5), (3, 11, 3), (2, 0, 7), (6, 6, 1)])
def test_matrices_that_begin_anywhere(n, d, dtype, x_at, g_at, y_at):
    """The same misalignment in all matrices (vectors with edges), and different ones (pieces); nothing outside the
    result is written."""
    x, _ = _at((_randn(32, n, d) * 1.5 + _randn(33, d)).to(dtype), x_at)
    g, _ = _at(_randn(34, n, d).to(dtype), g_at)
    w, b = 1 + 0.2 * _randn(35, d), 0.3 * _randn(36, d)
    for check in (lambda o: _check_forward(x, w, b, out=o), lambda o: _check_backward(g, x, w, out=o)):
        out, buf = _at(torch.zeros(n, d, device="cuda", dtype=dtype), y_at)
        check(out)
        assert (buf[:y_at] == 3).all() and (buf[y_at + n * d:] == 3).all()
    xin, buf = _at(x, x_at)
    want = hb.layer_norm_fwd(x, w, b, eps=EPS, out=_at(x, x_at)[0])[0]
    assert torch.equal(hb.layer_norm_fwd(xin, w, b, eps=EPS, out=xin)[0], want) and (buf[:x_at] == 3).all() and (buf[x_at + n * d:] == 3).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d", [(1, 13), (2, 2), (20_011, 5), (9001, 8), (30_005, 13), (17, 16), (7003, 17), (5001, 29), (11, 30), (4001, 33), (3001, 49), (2003, 62), (1001, 64), (907, 65)])
@pytest.mark.parametrize("x_at,g_at,y_at", [(0, 1, 2), (7, 3, 5)])
def test_narrow_rows_that_begin_anywhere(n, d, dtype, x_at, g_at, y_at):
    """Several rows to a warp, each row's pieces in a place of its own; nothing outside the result is written."""
    x, _ = _at((_randn(37, n, d) * 1.5 + _randn(38, d)).to(dtype), x_at)
    g, _ = _at(_randn(39, n, d).to(dtype), g_at)
    w, b = 1 + 0.2 * _randn(40, d), 0.3 * _randn(41, d)
    for check in (lambda o: _check_forward(x, w, b, out=o), lambda o: _check_backward(g, x, w, out=o)):
        out, buf = _at(torch.zeros(n, d, device="cuda", dtype=dtype), y_at)
        check(out)
        assert (buf[:y_at] == 3).all() and (buf[y_at + n * d:] == 3).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [1, 3, 4, 8, 12, 16, 24, 32, 36, 257, 280, 380, 384, 385, 500, 512, 513])
@pytest.mark.parametrize("n", [1, 31, 6007, 60_001])
def test_rows_per_warp(n, d, dtype):
    """Widths around each number of lanes and of vectors per lane; aligned rows, and rows five elements apart."""
    n = n if d < 64 else min(n, 6007)
    x, g = (_randn(42, n, d) * 1.5 + _randn(43, d)).to(dtype), _randn(44, n, d).to(dtype)
    w, b = 1 + 0.2 * _randn(45, d), 0.3 * _randn(46, d)
    far = torch.empty(n, d + 5, device="cuda", dtype=dtype)
    for out in (None, far[:, :d]):
        _check_forward(x, w, b, out=out)
        _check_backward(g, x, w, out=out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [66, 80, 95, 96, 97, 150, 186, 191, 192, 193, 250])
@pytest.mark.parametrize("n", [1, 7, 5003])
def test_rows_of_three_or_six_vectors_per_lane(n, d, dtype):
    x, g = (_randn(47, n, d) * 1.5 + _randn(48, d)).to(dtype), _randn(49, n, d).to(dtype)
    w, b = 1 + 0.2 * _randn(50, d), 0.3 * _randn(51, d)
    far = torch.empty(n, d + 5, device="cuda", dtype=dtype)
    for out in (None, far[:, :d]):
        _check_forward(x, w, b, out=out)
        _check_backward(g, x, w, out=out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d", [(1, 4097), (5, 6050), (301, 7944), (3, 8190), (2, 8191), (2, 8192), (2, 8193)])
def test_blocks_of_eight_or_sixteen_columns_per_thread(n, d, dtype):
    x, g = (_randn(52, n, d) * 1.5 + _randn(53, d)).to(dtype), _randn(54, n, d).to(dtype)
    w, b = 1 + 0.2 * _randn(55, d), 0.3 * _randn(56, d)
    far = torch.empty(n, d + 5, device="cuda", dtype=dtype)
    for out in (None, far[:, :d]):
        _check_forward(x, w, b, out=out)
        _check_backward(g, x, w, out=out)
