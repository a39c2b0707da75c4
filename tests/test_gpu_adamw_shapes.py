"""adamw_step takes gradients and copies of its parameters' shapes, not of their lengths alone."""
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


@pytest.mark.parametrize("bits", [8, 32])
def test_other_shapes_of_the_same_length_are_refused(bits):
    params = [torch.ones(20, 15, device="cuda"), torch.ones(4, 5, 6, device="cuda"), torch.ones((), device="cuda")]
    grads = [torch.ones_like(p) for p in params]
    state = hb.adamw_state(params, bits)
    a, g = torch.randn(7, 20, device="cuda"), torch.randn(7, 15, device="cuda")
    for at, wrong in ((0, g.t() @ a), (0, torch.ones(300, device="cuda")), (1, torch.ones(4, 6, 5, device="cuda")), (1, torch.ones(20, 6, device="cuda")),
                      (2, torch.ones(1, device="cuda"))):
        assert wrong.is_contiguous() and wrong.numel() == params[at].numel()
        changed = [*grads[:at], wrong, *grads[at + 1:]]
        with pytest.raises(ValueError, match="gradients"):
            hb.adamw_step(params, changed, state, 1)
        with pytest.raises(ValueError, match="gradients"):
            hb.adamw_step(params, [None if k == (at + 1) % 3 else x for k, x in enumerate(changed)], state, 1)
        with pytest.raises(ValueError, match="copies"):
            hb.adamw_step(params, grads, state, 1, copies=[x.bfloat16() if k == at else None for k, x in enumerate(changed)])
    assert all((p == 1).all() for p in params)
    copies = [torch.zeros_like(p, dtype=torch.bfloat16) for p in params]
    hb.adamw_step(params, [grads[0], None, grads[2]], state, 1, lr=0.25, weight_decay=0.0, copies=copies)
    assert all(((p - 0.75).abs() < 1e-6).all() for p in (params[0], params[2])) and (params[1] == 1).all()
    assert (copies[0] == 0.75).all() and not copies[1].any() and copies[2] == 0.75
