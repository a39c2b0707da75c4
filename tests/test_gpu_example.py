"""The example trains: its gradients against the same model in 64 bits under torch's own differentiation, and a loss
that falls.

Tolerance: every path from a parameter to the loss is some dozen fp32 operations per term with sums of at most a few
thousand terms; 2e-4 of a gradient's norm leaves two orders of magnitude over 1000 * 2^-24 = 6e-5 relative to it for
the terms that do not cancel.
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
    spec = importlib.util.spec_from_file_location("graph_classification", os.path.join(ROOT, "examples", "graph_classification.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _reference(example, model, batch):
    table, w1, gain, bias, w2 = params = [p.detach().double().requires_grad_() for p in model.parameters()]
    row_ptr, col = torch.from_numpy(batch.graph.row_ptr).cuda(), torch.from_numpy(batch.graph.col_idx).long().cuda()
    degree = (row_ptr[1:] - row_ptr[:-1])
    dst = torch.repeat_interleave(torch.arange(batch.n, device="cuda"), degree)
    ids = batch.types.long()
    h = table[ids.clamp(min=0)] * (ids >= 0)[:, None]
    a = torch.zeros_like(h).index_add(0, dst, h[col]) / degree.clamp(min=1)[:, None]
    y = torch.nn.functional.layer_norm(a @ w1, (w1.shape[1],), gain, bias, 1e-5)
    r = y.clamp(min=0)
    p = r.reshape(-1, 100, r.shape[1]).mean(1)
    loss = torch.nn.functional.cross_entropy(p @ w2, batch.labels)
    return loss, torch.autograd.grad(loss, params)


def test_gradients_of_the_whole_step(example):
    batch = example.Batch(40)
    model = example.Model()
    loss, grads = model.loss_and_gradients(batch)
    want_loss, want = _reference(example, model, batch)
    assert abs(float(loss) - float(want_loss)) < 1e-5
    for name, got, ref in zip(("table", "w1", "gain", "bias", "w2"), grads, want):
        err = float((got.double() - ref).norm() / ref.norm())
        assert err < 2e-4, f"{name}: {err:.2e}"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_loss_falls(example, dtype):
    batch = example.Batch(100)
    model = example.Model(dtype=dtype)
    losses = [float(model.step(batch)[0]) for _ in range(30)]
    assert losses[-1] < 0.6 * losses[0], losses
