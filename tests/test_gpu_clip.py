"""GPU parity of the global gradient norm and of clipping by it, against plain 64-bit forms.

Bounds, u = 2^-24: a square and at most 62 fp32 additions before the sums go to fp64, so N^2 is good to 64 u and N to
33 u; the factor adds 3 roundings and the product one: 40 u of each value, and 2^-8 of it where it is stored as bf16.
"""
import math

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


def _tensors(seed, lengths, kinds, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, m in enumerate(lengths):
        k = kinds[i % len(kinds)]
        out.append((0.1 * torch.randn(m + offset, generator=gen, device="cuda")).to(k)[offset:])
    return out


def _want(grads, max_norm):
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    return norm, min(1.0, max_norm / (norm + 1e-6))


def _check(grads, max_norm, in_place=False):
    norm, c = _want(grads, max_norm)
    src = [g.double().clone() for g in grads]
    assert abs(float(hb.grad_norm(grads)) - norm) <= 33 * U * norm
    out, got = hb.clip_grad_norm(grads, max_norm, out=grads if in_place else None)
    assert abs(float(got) - norm) <= 33 * U * norm
    for g, s, o in zip(grads, src, out):
        assert (o is g) == in_place and o.dtype == g.dtype and o.shape == g.shape
        bound = 40 * U * c * s.abs() + (2.0 ** -8 * c * s.abs() if o.dtype == BF16 else 0)
        assert ((o.double() - c * s).abs() <= bound + 1e-45).all()
        if not in_place:
            assert torch.equal(g.double(), s)                       # the inputs are left alone


LISTS = [[1], [7, 0, 3], [64, 64 * 64, 1, 4097, 0, 12_289], [100_000, 5, 8192, 8193, 65_537, 31], [16] * 300,
         [int(1.7 ** k) for k in range(28)], [0, 0, 1], [3_000_001, 2]]


@pytest.mark.parametrize("lengths", LISTS)
@pytest.mark.parametrize("kinds", [(F32,), (BF16,), (F32, BF16)])
def test_lists(lengths, kinds):
    for max_norm in (0.01, 1e9):
        _check(_tensors(1, lengths, kinds), max_norm)
        _check(_tensors(2, lengths, kinds), max_norm, in_place=True)


@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_pointers_off_the_vector_boundary(offset):
    _check(_tensors(3, [10_000, 17, 4096, 1], (F32, BF16), offset), 0.5)
    _check(_tensors(4, [10_000, 17, 4096, 1], (BF16, F32), offset), 0.5, in_place=True)
    grads = _tensors(5, [5000, 333], (F32,))
    buf = torch.full((6000,), 3.0, device="cuda")
    out = [buf[offset:offset + 5000], buf[5100 + offset:5100 + offset + 333]]      # only the outputs are off
    norm, c = _want(grads, 0.5)
    hb.clip_grad_norm(grads, 0.5, out=out)
    assert torch.allclose(out[0], (grads[0].double() * c).float(), rtol=40 * U, atol=0)
    assert (buf[:offset] == 3).all() and (buf[offset + 5000:5100 + offset] == 3).all() and (buf[5433 + offset:] == 3).all()


def test_shapes_and_unclipped_in_place_keep_their_bits():
    grads = [t.view(s) for t, s in zip(_tensors(6, [120, 64, 1], (F32, BF16)), [(4, 5, 6), (8, 8), ()])]
    before = [g.clone() for g in grads]
    out, norm = hb.clip_grad_norm(grads, 1e6, out=grads)
    assert all(torch.equal(g, b) for g, b in zip(grads, before))
    out, norm = hb.clip_grad_norm(grads, 0.0)
    assert not any(o.any() for o in out)


def test_zeros_infinities_and_nan():
    zeros = [torch.zeros(100, device="cuda"), torch.zeros(5, device="cuda", dtype=BF16)]
    out, norm = hb.clip_grad_norm(zeros, 1.0)
    assert float(norm) == 0 and not any(o.any() for o in out)
    g = _tensors(7, [1000, 40], (F32,))
    g[0][10] = float("inf")
    out, norm = hb.clip_grad_norm(g, 1.0)
    assert math.isinf(float(norm)) and out[0][10].isnan() and not out[0][11:].any() and not out[1].any()
    g[1][3] = float("nan")
    out, norm = hb.clip_grad_norm(g, 1.0)
    assert math.isnan(float(norm)) and all(o.isnan().all() for o in out)
    assert math.isnan(float(hb.clip_grad_norm(g, 1.0, out=g)[1])) and all(o.isnan().all() for o in g)


def test_exact_values_and_runs_repeat():
    a, b = torch.full((30_000,), 3.0, device="cuda"), torch.full((30_000,), 4.0, device="cuda", dtype=BF16)
    assert float(hb.grad_norm([a, b])) == float(torch.tensor(5 * math.sqrt(30_000)))
    g = _tensors(8, [700_001, 3, 90_000], (F32, BF16))
    x, y = hb.clip_grad_norm(g, 0.3), hb.clip_grad_norm(g, 0.3)
    assert torch.equal(x[1], y[1]) and all(torch.equal(p, q) for p, q in zip(x[0], y[0]))


def test_a_tensor_beyond_32_bits():
    n = (1 << 31) + 10_007
    g = torch.full((n,), 0.5, dtype=BF16, device="cuda")
    g[-1] = 4096.0
    norm = math.sqrt(0.25 * (n - 1) + 4096.0 ** 2)
    out, got = hb.clip_grad_norm([g], norm / 2 + 1e-6, out=[g])
    assert abs(float(got) - norm) <= 33 * U * norm
    for i in (0, (1 << 31) - 1, 1 << 31, n - 2, n - 1):
        assert float(g[i]) == (2048.0 if i == n - 1 else 0.25)


def test_other_streams_and_graph_capture():
    g = _tensors(9, [50_000, 70, 9001], (F32, BF16))
    want, norm = hb.clip_grad_norm(g, 0.3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h = [t * 1 for t in g]
        got, n2 = hb.clip_grad_norm(h, 0.3)
    side.synchronize()
    assert torch.equal(n2, norm) and all(torch.equal(p, q) for p, q in zip(got, want))
    out = [torch.zeros_like(t) for t in g]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, n3 = hb.clip_grad_norm(g, 0.3, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(n3, norm) and all(torch.equal(p, q) for p, q in zip(out, want))


def test_refusals():
    g = [torch.ones(8, device="cuda"), torch.ones(3, 4, device="cuda")]
    for bad in ([], [g[1].t()], [g[0], g[0]], [g[0].cpu()]):
        with pytest.raises(ValueError):
            hb.clip_grad_norm(bad, 1.0)
    with pytest.raises(TypeError):
        hb.clip_grad_norm([g[0].half()], 1.0)
    with pytest.raises(ValueError):
        hb.clip_grad_norm(g, 1.0, out=g[:1])
    with pytest.raises(ValueError):
        hb.clip_grad_norm(g, 1.0, out=[g[0], g[0]])
    for limit in (-1.0, float("nan")):
        with pytest.raises(hb.HagError) as e:
            hb.clip_grad_norm(g, limit)
        assert e.value.status == hb.HAG_ERR_ARG
    assert (g[0] == 1).all()
