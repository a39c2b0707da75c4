"""Embedding, layer norm and clipping where sizes and values are extreme: against plain 64-bit forms, u = 2^-24."""
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
