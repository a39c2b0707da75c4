"""What the norm returns as its sum when y takes the place of x, and what a gradient made from it is."""
import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("n,d", [(1, 1), (3, 64), (50, 333), (2, 20_000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_without_a_residual_there_is_no_sum_left(n, d, dtype):
    """Without a residual the sum is x; once y stands there, no gradient can be made from it, so none is offered."""
    x, g = _randn(1, n, d).to(dtype), _randn(2, n, d).to(dtype)
    y, total, rstd = hb.rms_norm_fwd(x)
    assert total is x
    for where in (x.clone(), x.clone().view(n, d)):
        inside, left, same = hb.rms_norm_fwd(where, out=where)
        assert inside is where and torch.equal(inside, y) and torch.equal(same, rstd)
        assert left is None
        view = where.view(n, d)
        view.copy_(x)
        assert hb.rms_norm_fwd(where, out=view)[1] is None            # the same memory by another name
        with pytest.raises(ValueError):
            hb.rms_norm_bwd(g, left, same)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_with_a_residual_the_sum_stays(dtype):
    x, r, g = (_randn(3 + k, 40, 72).to(dtype) for k in range(3))
    want = hb.rms_norm_fwd(x, residual=r)
    grads = hb.rms_norm_bwd(g, want[1], want[2])
    for place in (0, 1):
        ins = [x.clone(), r.clone()]
        got = hb.rms_norm_fwd(ins[0], residual=ins[1], out=ins[place])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(hb.rms_norm_bwd(g, got[1], got[2]), grads))
