"""GPU parity of the root-mean-square norm with the residual's addition, against plain 64-bit forms.

Bounds, with u = 2^-24, D columns and h = 64 + D/256 the longest chain of fp32 additions a row sum goes through:
  total   u |x + residual| for the addition
  rstd    relative (h/2 + 10) u: the addition (2 u in a square), the squares and their sum (h + 1), the mean and eps (3), half
          of it through the root, and the 2-ulp reciprocal root
  y       relative (h/2 + 14) u: rstd, the addition and two products
  scale   relative (h/2 + 18) u: the largest |y| and the product with a rounded 1 / top
  q       q * scale is half a step of the 8-bit type from y, where y has the relative error above and the quotient one of
          8 u: e4m3 has a step of at most 2^-3 of the value or of 2^-9, int8 one of 1
  grad    u rstd [4 |t| + (h + 8) |hh| mean|t hh|] + 2 u |grad| + u |grad_total|, t = grad_y w, hh = total rstd
  grad_w  (4 + k) u sum|g hh|, where no chain of additions over n rows is longer than k = 128 + n/32
bf16 results add one rounding, 2^-8 of the value.
"""
import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, E4M3, I8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.int8
EPS = 1e-5
TYPES = {"f32": (F32, F32, F32), "bf16": (BF16, BF16, BF16), "mixed": (BF16, F32, BF16)}       # x, stream, y


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


def _definition(x, w, residual, eps=EPS):
    total = x.double() if residual is None else x.double() + residual.double()
    rstd = (total.square().mean(1) + eps).rsqrt()
    return total, rstd, total * rstd[:, None] * (1 if w is None else w.double())


def _check_forward(x, w, residual, eps=EPS, **more):
    h = 64 + x.shape[1] / 256
    total, rstd, y = _definition(x, w, residual, eps)
    got, t, r = hb.rms_norm_fwd(x, w, residual=residual, eps=eps, **more)
    _inside(r, rstd, (h / 2 + 10) * U * rstd, "rstd")
    _inside(got, y, (h / 2 + 14) * U * y.abs(), "y")
    if residual is None:
        assert t is x
    else:
        assert t.dtype == residual.dtype
        _inside(t, total, U * total.abs(), "total")
    return got, t, r


def _check_quant(x, w, residual, block, kind, **more):
    n, d = x.shape
    rel = (32 + d / 512 + 18) * U
    total, rstd, y = _definition(x, w, residual)
    q, scales, t, r = hb.rms_norm_quant_fwd(x, w, residual=residual, eps=EPS, block=block, dtype=kind, **more)
    width, top = block or d, 448.0 if kind is E4M3 else 127.0
    assert q.dtype is kind and scales.shape == (n, -(-d // width)) and (scales > 0).all()
    parts = torch.nn.functional.pad(y, (0, -d % width)).view(n, -1, width)
    want = (parts.abs().amax(2) / top).clamp(min=2.0 ** -126)
    assert ((scales.double() - want).abs() <= rel * want).all(), "scale"
    each = scales.double().repeat_interleave(width, 1)[:, :d]
    t64 = y.abs() / each
    half = torch.maximum(2.0 ** -4 * t64, torch.full_like(t64, 2.0 ** -10)) if kind is E4M3 else torch.full_like(t64, 0.5)
    err = (q.double() * each - y).abs()
    assert (err <= each * half + (rel + 8 * U) * 1.125 * y.abs()).all(), "q"
    h = 64 + d / 256
    _inside(r, rstd, (h / 2 + 10) * U * rstd, "rstd")
    if residual is not None:
        _inside(t, total, U * total.abs(), "total")
    return q, scales, t, r


def _check_backward(g, total, w, along, x_dtype=None, out=None, param_dtype=None):
    n, d = total.shape
    h, k = 64 + d / 256, 128 + n / 32
    rstd = (total.double().square().mean(1) + EPS).rsqrt().float()
    rs = rstd.double()[:, None]
    gd, hh = g.double(), total.double() * rs
    t = gd if w is None else gd * w.double()
    want = rs * (t - hh * (t * hh).mean(1, keepdim=True)) + (0 if along is None else along.double())
    bound = U * rs * (4 * t.abs() + (h + 8) * hh.abs() * (t * hh).abs().mean(1, keepdim=True)) + 2 * U * want.abs()
    if along is not None:
        bound = bound + U * along.double().abs()
    gw64, gw_mag = (gd * hh).sum(0), (gd * hh).abs().sum(0)
    gx, gr, gw = hb.rms_norm_bwd(g, total, rstd, w, grad_total=along, x_dtype=x_dtype, out=out, param_dtype=param_dtype)
    assert gr.dtype == total.dtype and (gx is gr) == (x_dtype in (None, total.dtype)) and gx.dtype == (x_dtype or total.dtype)
    _inside(gr, want, bound, "grad_residual")
    _inside(gx, want, bound, "grad_x")
    _inside(gw, gw64, (4 + k) * U * gw_mag, "grad_weight")
    return gx, gr, gw


def _inputs(seed, n, d, types):
    tx, ts, ty = TYPES[types]
    return _randn(seed, n, d).to(tx), (2 * _randn(seed + 1, n, d)).to(ts), 1 + 0.2 * _randn(seed + 2, d)


SHAPES = [(1, 1), (1, 4096), (1, 8193), (3, 2), (1000, 16), (257, 20), (5000, 64), (1001, 128), (777, 33), (640, 256), (300, 250), (129, 515),
          (90, 1024), (66, 1433), (40, 2048), (31, 4100), (12, 8192), (9, 16384), (5, 16386), (3, 50001), (2, 49153), (700, 8), (611, 31), (2, 70_001), (3, 131_072),
          (4, 12_000), (300, 9999), (7, 32_800), (5, 65_536),
          (6, 8191), (6, 11_501), (161, 13_001), (155, 14_337), (4, 16_383)]


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("types", TYPES)
def test_forward(n, d, types):
    x, residual, w = _inputs(1, n, d, types)
    _check_forward(x, w, residual)
    _check_forward(x, w.to(BF16), residual)
    _check_forward(x, None, residual, stats=True)
    if types != "mixed":
        _check_forward(x, w, None)
    if types == "f32":
        _check_forward(x, w, None, dtype=BF16)
        _check_forward(x, w.to(BF16), residual, dtype=BF16)


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("kind", [E4M3, I8])
def test_quantised(n, d, types, kind):
    x, residual, w = _inputs(4, n, d, types)
    for block in (0, 32, 64, 128):
        _check_quant(x, w, residual, block, kind)
    _check_quant(x, w.to(BF16), residual, 64, kind)
    if types != "mixed":
        _check_quant(x, None, None, 32, kind)
        _check_quant(x, w, None, 0, kind)


@pytest.mark.parametrize("n,d", SHAPES + [(20_011, 64), (40_000, 24), (3000, 1024), (70_001, 1), (4000, 9001)])
@pytest.mark.parametrize("types", TYPES)
def test_backward(n, d, types):
    x, total, w = _inputs(7, n, d, types)
    g, along = _randn(10, n, d).to(TYPES[types][2]), _randn(11, n, d).to(TYPES[types][1])
    _check_backward(g, total, w, along, x_dtype=TYPES[types][0])
    _check_backward(g, total, w.to(BF16), None)
    _check_backward(g, total, None, along, param_dtype=F32)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("pad", [0, 3])
def test_every_width(types, pad):
    """All widths up to 700 and every 31st up to 9000: neighbours of every change of the kernel, each row's end guarded."""
    for d in [*range(1, 701), *range(701, 9000, 31)]:
        x, residual, w = _inputs(50, 3, d + pad, types)
        x, residual, w = x[:, :d], residual[:, :d], w[:d]
        guard = {t: torch.full((5, d + pad), 3.0, device="cuda", dtype=t) for t in {TYPES[types][1], TYPES[types][2]}}
        for t, out in guard.items():
            inside = out[1:4, :d]
            if t is TYPES[types][2]:
                _check_forward(x, w, residual, out=inside)
            if t is TYPES[types][1]:
                _check_backward(x if types == "mixed" else residual, residual, w, residual, out=inside)
            inside.fill_(3.0)
            assert (out == 3).all(), d
        if d % 3 == 0:
            codes = torch.full((5, d + pad), 3, device="cuda", dtype=I8)
            _check_quant(x, w, residual, (32, 64, 128, 0)[d // 3 % 4], I8, out=codes[1:4, :d])
            codes[1:4, :d] = 3
            assert (codes == 3).all(), d


@pytest.mark.parametrize("types", TYPES)
def test_strides_offsets_and_in_place(types):
    tx, ts, ty = TYPES[types]
    a, b, c, e = _randn(12, 70, 700).to(tx), _randn(13, 70, 650).to(ts), _randn(14, 70, 670).to(ty), _randn(15, 70, 690).to(ts)
    weights = 1 + 0.2 * _randn(16, 701)
    for lo, d in ((0, 64), (1, 64), (2, 30), (4, 128), (8, 512), (3, 601), (5, 1), (4, 20)):
        x, residual, g, along, w = a[:, lo:lo + d], b[:, lo:lo + d], c[:, lo + 1:lo + 1 + d], e[:, 3:3 + d], weights[lo:lo + d]
        bufs = {t: torch.full((70, 720), 3.0, device="cuda", dtype=t) for t in {ty, ts}}
        y, total, rstd = _check_forward(x, w, residual, out=bufs[ty][:, 9:9 + d])
        assert (bufs[ty][:, :9] == 3).all() and (bufs[ty][:, 9 + d:] == 3).all()
        sums = torch.full((70, 720), 3.0, device="cuda", dtype=ts)
        _check_forward(x, w, residual, total_out=sums[:, 7:7 + d])
        assert (sums[:, :7] == 3).all() and (sums[:, 7 + d:] == 3).all()
        codes = torch.full((70, 720), 3, device="cuda", dtype=I8)
        _check_quant(x, w, residual, 32, I8, out=codes[:, 5:5 + d])
        assert (codes[:, :5] == 3).all() and (codes[:, 5 + d:] == 3).all()
        # in the place of the inputs, of the same layout: the same bits
        xc, rc = x.contiguous(), residual.contiguous()
        want = hb.rms_norm_fwd(xc, w, residual=rc, eps=EPS)
        xin, rin = xc.clone(), rc.clone()
        got = hb.rms_norm_fwd(xin, w, residual=rin, eps=EPS, out=xin, total_out=rin)
        assert got[0] is xin and got[1] is rin and all(torch.equal(p, q) for p, q in zip(got, want))
        if tx == ts:
            xin, rin = xc.clone(), rc.clone()
            got = hb.rms_norm_fwd(xin, w, residual=rin, eps=EPS, out=rin, total_out=xin)
            assert all(torch.equal(p, q) for p, q in zip(got, want))
        bufs[ts].fill_(3.0)
        _check_backward(g, b[:, lo:lo + d], w, along, out=bufs[ts][:, 9:9 + d])
        assert (bufs[ts][:, :9] == 3).all() and (bufs[ts][:, 9 + d:] == 3).all()
        ins = [g.contiguous(), total.contiguous(), along.contiguous()]
        same = hb.rms_norm_bwd(ins[0], ins[1], rstd, w, grad_total=ins[2])
        for k in (0, 1, 2):
            if ins[k].dtype == ts:
                here = [t.clone() for t in ins]
                got = hb.rms_norm_bwd(here[0], here[1], rstd, w, grad_total=here[2], out=here[k])
                assert all(torch.equal(p, q) for p, q in zip(got, same))
    row = _randn(17, 1, 96)                                          # one row for all, as of a sum or a shared bias
    _check_forward(row.to(tx).expand(50, 96), weights[:96], row.to(ts).expand(50, 96))
    _check_backward(row.to(ty).expand(50, 96), b[:50, :96], weights[:96], None)


@pytest.mark.parametrize("d", [9001, 20_000, 50_000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_where_rows_are_read_again(d, dtype):
    x, residual, g = (_randn(18 + k, 4, d).to(dtype) for k in range(3))
    y, total, rstd = want = hb.rms_norm_fwd(x, None, residual=residual)
    xin, rin = x.clone(), residual.clone()
    assert all(torch.equal(p, q) for p, q in zip(hb.rms_norm_fwd(xin, None, residual=rin, out=xin, total_out=rin), want))
    same = hb.rms_norm_bwd(g, total, rstd, grad_total=residual)
    for k in range(3):
        ins = [g.clone(), total.clone(), residual.clone()]
        got = hb.rms_norm_bwd(ins[0], ins[1], rstd, grad_total=ins[2], out=ins[k])
        assert all(torch.equal(p, q) for p, q in zip(got, same))
    want = hb.rms_norm_quant_fwd(x, None, residual=residual, block=32)
    rin = residual.clone()
    got = hb.rms_norm_quant_fwd(x, None, residual=rin, block=32, total_out=rin)
    assert all(torch.equal(p.float(), q.float()) for p, q in zip(got, want))


def test_zero_rows_and_values_that_are_not_finite():
    x, residual = _randn(21, 40, 200), _randn(22, 40, 200)
    x[3], residual[3] = 0, 0
    w = 1 + 0.2 * _randn(23, 200)
    clean = hb.rms_norm_fwd(x, w, residual=residual, eps=EPS)
    q0 = hb.rms_norm_quant_fwd(x, w, residual=residual, eps=EPS, block=64)
    assert not clean[0][3].any() and not q0[0][3].float().any() and (q0[1][3] == 2.0 ** -126).all()
    x[7, 3], x[20, 0], residual[30, 199] = float("inf"), float("nan"), float("-inf")
    y, total, rstd = hb.rms_norm_fwd(x, w, residual=residual, eps=EPS)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[7, 20, 30]] = False
    assert torch.equal(y[keep], clean[0][keep]) and torch.equal(rstd[keep], clean[2][keep])
    assert y[7, 3].isnan() and not y[7, 4:].any() and y[20].isnan().all() and y[30, 199].isnan() and not y[30, :199].any()
    for block in (0, 64):
        for kind in (E4M3, I8):
            want = hb.rms_norm_quant_fwd(torch.where(keep[:, None], x, 0.0), w, residual=torch.where(keep[:, None], residual, 0.0), eps=EPS, block=block, dtype=kind)
            q, scales, _, _ = hb.rms_norm_quant_fwd(x, w, residual=residual, eps=EPS, block=block, dtype=kind)
            assert torch.equal(q[keep].float(), want[0][keep].float()) and torch.equal(scales[keep], want[1][keep])
            assert not scales[20].isfinite().any() and not scales[7, 0].isfinite()
            assert (q[20].double() * scales[20].double().repeat_interleave(block or 200)[:200]).isnan().all()
    # eps 0: a row of zeros has no direction
    assert hb.rms_norm_fwd(torch.zeros(2, 64, device="cuda"), eps=0.0)[0].isnan().all()


def test_tiny_and_large_values():
    for size in (1e-18, 1e-30, 1e15):
        x = size * _randn(24, 50, 320)
        _check_forward(x, None, None)
        _check_quant(x, None, None, 64, E4M3)
    x = _randn(25, 50, 320)
    w = torch.full((320,), 1e-38, device="cuda")                     # scales at their lower end
    q, scales, _, _ = hb.rms_norm_quant_fwd(x, w, eps=EPS)
    assert (scales == 2.0 ** -126).all()
    _, _, y = _definition(x, w, None)
    assert ((q.double() * 2.0 ** -126 - y).abs() <= 2.0 ** -126 * torch.maximum(2.0 ** -4 * y.abs() * 2.0 ** 126, torch.tensor(2.0 ** -10, device="cuda")) * 1.001).all()


def test_gradient_against_differences():
    """Central differences of the 64-bit loss <g, y> + <a, total>; step 1e-4, so the third-order term is about 1e-8."""
    n, d = 6, 48
    x, residual, g, a, w = _randn(26, n, d), _randn(27, n, d), _randn(28, n, d), _randn(29, n, d), 1 + 0.2 * _randn(30, d)
    y, total, rstd = hb.rms_norm_fwd(x, w, residual=residual, eps=EPS)
    gx, gr, gw = hb.rms_norm_bwd(g, total, rstd, w, grad_total=a)

    def loss(x, residual, w):
        total, _, y = _definition(x, w, residual)
        return (y * g.double()).sum() + (total * a.double()).sum()

    ins = [x.double(), residual.double(), w.double()]
    for which, got in enumerate((gx, gr, gw)):
        for at in range(0, got.numel(), 13):
            side = []
            for s in (1e-4, -1e-4):
                moved = [t.clone() for t in ins]
                moved[which].view(-1)[at] += s
                side.append(loss(*moved))
            want = float(side[0] - side[1]) / 2e-4
            assert abs(float(got.view(-1)[at]) - want) <= 2e-5 * (1 + abs(want))


def test_runs_repeat_and_no_rows():
    x, residual, g, w = _randn(31, 9000, 100), _randn(32, 9000, 100), _randn(33, 9000, 100), _randn(34, 100)
    y, total, rstd = hb.rms_norm_fwd(x, w, residual=residual)
    a, b = (hb.rms_norm_bwd(g, total, rstd, w, grad_total=x) for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    gx, gr, gw = hb.rms_norm_bwd(g, total, rstd, w, grad_total=x, param_grads=False)
    assert torch.equal(gx, a[0]) and gw is None
    assert hb.rms_norm_fwd(x, w, stats=False)[2] is None
    empty = x[:0]
    y, total, rstd = hb.rms_norm_fwd(empty, w, residual=empty)
    assert y.shape == (0, 100) and total.shape == (0, 100) and rstd.shape == (0,)
    q, scales, _, _ = hb.rms_norm_quant_fwd(empty, w, block=32)
    assert q.shape == (0, 100) and scales.shape == (0, 4)
    gx, gr, gw = hb.rms_norm_bwd(empty, total, rstd, w)
    assert gx.shape == (0, 100) and not gw.any()


def test_other_streams_and_graph_capture():
    x, residual, g, w = _randn(35, 3000, 136), _randn(36, 3000, 136), _randn(37, 3000, 136), _randn(38, 136)

    def calls(x, residual, g):
        y, total, rstd = hb.rms_norm_fwd(x, w, residual=residual)
        q, scales, _, _ = hb.rms_norm_quant_fwd(x, w, residual=residual, block=32)
        return [y, total, rstd, q.float(), scales, *hb.rms_norm_bwd(g, total, rstd, w, grad_total=residual)]

    want = calls(x, residual, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = calls(x * 1, residual * 1, g * 1)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    ins = [t.clone() for t in (x, residual, g)]
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls(*ins)
    with torch.cuda.graph(other):
        calls(*ins)
    for t, s in zip(ins, (g, x, residual)):
        t.copy_(s)
    other.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, calls(g, x, residual)))


def test_matrices_beyond_32_bits():
    """2.3e9 elements; rows of both ends and around 2^31 and 2^32 bytes against the definition."""
    n, d = 140_000, 16_384
    gen = torch.Generator(device="cuda").manual_seed(39)
    x, g = (torch.empty(n, d, dtype=BF16, device="cuda").normal_(generator=gen) for _ in range(2))
    rows = torch.tensor([0, 1, 65_535, 65_536, 131_071, 131_072, 131_073, n - 1], device="cuda")
    y, total, rstd = hb.rms_norm_fwd(x, residual=g)
    t64, r64, y64 = _definition(x[rows], None, g[rows])
    _inside(y[rows], y64, 100 * U * y64.abs(), "y")
    _inside(total[rows], t64, U * t64.abs(), "total")
    q, scales, _, _ = hb.rms_norm_quant_fwd(x, residual=g, block=128, total_out=total)
    some = hb.rms_norm_quant_fwd(x[rows], residual=g[rows], block=128)
    assert torch.equal(q[rows].float(), some[0].float()) and torch.equal(scales[rows], some[1])
    _, gr, _ = hb.rms_norm_bwd(g, total, rstd, grad_total=x, out=y)
    want = hb.rms_norm_bwd(g[rows], total[rows], rstd[rows], grad_total=x[rows], param_grads=False)[1]
    assert torch.equal(gr[rows], want)


def test_refusals():
    x, w = _randn(40, 8, 64), torch.ones(64, device="cuda")
    bad = torch.ones(8, 64, dtype=torch.float16, device="cuda")
    for call in (lambda: hb.rms_norm_fwd(x.cpu()), lambda: hb.rms_norm_fwd(x.t()), lambda: hb.rms_norm_fwd(x, w[:63]),
                 lambda: hb.rms_norm_fwd(x, w, residual=x[:7]), lambda: hb.rms_norm_fwd(x, w, total_out=x), lambda: hb.rms_norm_fwd(x, w, out=x[:, :63]),
                 lambda: hb.rms_norm_quant_fwd(x, w, block=16), lambda: hb.rms_norm_quant_fwd(x, w, block=32, scales=torch.empty(8, 1, device="cuda")),
                 lambda: hb.rms_norm_bwd(x, x, w[:7]), lambda: hb.rms_norm_bwd(x[:, 1:], x, w[:8]), lambda: hb.rms_norm_bwd(x, x, w[:8], workspace=w)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: hb.rms_norm_fwd(bad), lambda: hb.rms_norm_fwd(x, dtype=torch.float16), lambda: hb.rms_norm_quant_fwd(x, dtype=torch.uint8),
                 lambda: hb.rms_norm_bwd(x, x, w[:8], x_dtype=torch.float16), lambda: hb.rms_norm_bwd(x, x, w[:8], grad_total=x.bfloat16())):
        with pytest.raises(TypeError):
            call()
    for call, status in ((lambda: hb.rms_norm_fwd(x, eps=-1.0), hb.HAG_ERR_ARG), (lambda: hb.rms_norm_fwd(x.bfloat16(), dtype=F32), hb.HAG_ERR_DTYPE),
                         (lambda: hb.rms_norm_fwd(x, residual=x.bfloat16()), hb.HAG_ERR_DTYPE), (lambda: hb.rms_norm_fwd(x, residual=x, out=x, total_out=x), hb.HAG_ERR_ARG),
                         (lambda: hb.rms_norm_bwd(x, x.bfloat16(), w[:8]), hb.HAG_ERR_DTYPE)):
        with pytest.raises(hb.HagError) as e:
            call()
        assert e.value.status == status
    assert (w == 1).all()
