"""The residual example: its gradients against the same model in 64 bits under torch's own differentiation, its step against
the formula on those gradients, and that it runs in every form.

Tolerance of the gradients: every path from a parameter to the loss is some dozen fp32 operations per layer with sums of at
most a few thousand terms; 2e-4 of a gradient's norm leaves two orders of magnitude over 1000 * 2^-24 = 6e-5 relative to it
for the terms that do not cancel.  The first step from zero states is rate * g / (|g| + eps): the parameters move by less
than the rate.
"""
import importlib.util
import os

import pytest

from paper_1906_03707_b200.build import build as build_library

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    build_library()
    spec = importlib.util.spec_from_file_location("residual_adamw", os.path.join(ROOT, "examples", "residual_adamw.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _reference(model, batch):
    params = [p.detach().double().requires_grad_() for p in model.parameters()]
    n = model.layers
    table, w, gain, w2 = params[0], params[1:1 + n], params[1 + n:2 + 2 * n], params[-1]
    row_ptr, col = torch.from_numpy(batch.graph.row_ptr).cuda(), torch.from_numpy(batch.graph.col_idx).long().cuda()
    degree = row_ptr[1:] - row_ptr[:-1]
    dst = torch.repeat_interleave(torch.arange(batch.n, device="cuda"), degree)
    norm = lambda s, g: s * (s.square().mean(1, keepdim=True) + 1e-5).rsqrt() * g  # noqa: E731
    ids = batch.types.long()
    s = table[ids.clamp(min=0)] * (ids >= 0)[:, None]
    y = norm(s, gain[0])
    for k in range(n):
        a = torch.zeros_like(y).index_add(0, dst, y[col]) / degree.clamp(min=1)[:, None]
        s = s + (a @ w[k]).clamp(min=0)
        y = norm(s, gain[k + 1])
    p = y.reshape(-1, 100, y.shape[1]).mean(1)
    loss = torch.nn.functional.cross_entropy(p @ w2, batch.labels)
    return loss, torch.autograd.grad(loss, params)


def test_gradients_of_the_whole_step(example):
    batch, model = example.Batch(40), example.Model()
    loss, grads = model.loss_and_gradients(batch)
    want_loss, want = _reference(model, batch)
    assert abs(float(loss) - float(want_loss)) < 1e-5
    for k, (got, ref) in enumerate(zip(grads, want)):
        err = float((got.double() - ref).norm() / ref.norm())
        assert err < 2e-4, f"{k}: {err:.2e}"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_run_in_every_form(example, dtype, bits):
    batch, model = example.Batch(40), example.Model(dtype=dtype, bits=bits)
    before = [p.clone() for p in model.parameters()]
    grads = model.loss_and_gradients(batch)[1]
    model.step(batch, rate=1e-3)
    factor = min(1.0, 1.0 / (float(torch.cat([g.double().reshape(-1) for g in grads]).norm()) + 1e-6))
    for p, b, g, d in zip(model.parameters(), before, grads, model.decay):
        g = g.double() * factor
        want = b.double() * (1 - 1e-3 * d) - 1e-3 * g / (g.abs() + 1e-8)
        # 4 u of the parameter; the move carries the factor's 40 u and the step's 60 u, and eps hides less than that
        assert ((p.double() - want).abs() <= 2.0 ** -22 * b.double().abs() + 1e-3 * 128 * 2.0 ** -24).all()
    for _ in range(5):
        loss, norm = model.step(batch)
    assert torch.isfinite(loss) and torch.isfinite(norm) and all(p.isfinite().all() for p in model.parameters())
    if model.copies is not None:
        assert all(torch.equal(c, p.to(dtype)) for c, p in zip(model.copies, model.parameters()))
