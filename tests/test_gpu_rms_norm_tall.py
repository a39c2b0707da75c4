"""The root-mean-square norm over more rows than a launch takes in one turn, every row against the definition (the bounds of
test_gpu_rms_norm.py).

Rows of one turn, at most, on 148 SMs: a launch has 24 blocks of 256 threads per SM where 16-byte vectors come through the ring with
more than 32 bytes per lane, 2 where they do with less, and 8 (all that fit) where vectors are narrow; a block has 256 / L rows
times the rows per turn (4 at most, of narrow vectors), L lanes sharing a row; of rows of whole blocks 6144 threads per SM, or 2048.
Each count below is more than two such turns for every type and form that its width takes, so that stages of the ring are used
again, the last turn is a part of one, and warps are left without rows.
"""
import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library
from test_gpu_rms_norm import BF16, E4M3, I8, TYPES, _check_backward, _check_forward, _check_quant, _inputs, _randn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
SHAPES = [(1_850_001, 8), (610_001, 3), (2_450_003, 4), (310_001, 13), (310_001, 20), (460_001, 32), (155_001, 33), (230_001, 64), (80_001, 100),
          (116_001, 128), (60_001, 256), (20_001, 333), (60_001, 512), (30_001, 700), (60_001, 1024), (15_001, 2048), (9_601, 3000), (7_501, 4096),
          (4_001, 8192), (449, 9999), (449, 12_000), (1_301, 20_000)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("types", TYPES)
def test_forward(n, d, types):
    x, residual, w = _inputs(60, n, d, types)
    _check_forward(x, w, residual)
    if types != "mixed":
        _check_forward(x, None, None)
    if types == "f32":
        _check_forward(x, w.to(BF16), residual, dtype=BF16)
        _check_forward(x, w, None, dtype=BF16)


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("types", TYPES)
def test_quantised(n, d, types):
    x, residual, w = _inputs(64, n, d, types)
    _check_quant(x, w, residual, 0, E4M3)
    _check_quant(x, w, residual, 32, I8)
    if types != "mixed":
        _check_quant(x, None, None, 128, E4M3)
        _check_quant(x, w, None, 0, I8)


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("types", TYPES)
def test_backward(n, d, types):
    x, total, w = _inputs(68, n, d, types)
    g, along = _randn(71, n, d).to(TYPES[types][2]), _randn(72, n, d).to(TYPES[types][1])
    _check_backward(g, total, w, along, x_dtype=TYPES[types][0])
    _check_backward(g, total, w.to(BF16), None)
