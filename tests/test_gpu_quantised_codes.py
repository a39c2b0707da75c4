"""The 8-bit outputs of the root-mean-square norm, code for code.

Rows of +1 and -1 have a mean square of exactly 1, so with eps = 0 their rstd is 1 and y is the weights with a sign, without
any rounding.  scale = max|y| (1 / top), with 1 / top rounded, and q = round(y / scale) are then what fp32 arithmetic on the
host gives, bit for bit.  The weights lie on and next to the middles between two codes, where a quotient that is off by one place gives the other code.
"""
import numpy as np
import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, E4M3, I8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.int8
TOP = {E4M3: 448.0, I8: 127.0}


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


def _middles(kind):
    if kind is I8:
        return torch.arange(0, 127) + 0.5
    codes = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).float()           # 0 to 448
    return (codes[1:] + codes[:-1]) / 2


def _weights(gen, d, block, kind):
    """Magnitudes on and next to the middles of codes, of a scale of their own per block, whose largest is top * scale."""
    width, mid = block or d, _middles(kind)
    pick = mid[torch.randint(0, mid.numel(), (d,), generator=gen)]
    size = torch.exp(3 * torch.randn(-(-d // width), generator=gen))
    each = size.repeat_interleave(width)[:d]
    w = pick * each
    w = torch.nextafter(w, w * torch.randint(0, 3, (d,), generator=gen))           # a place down, as it is, a place up
    w[torch.arange(0, d, width)] = TOP[kind] * size
    return w


@pytest.mark.parametrize("d", [8, 20, 32, 33, 64, 96, 250, 256, 333, 515, 1024, 1433, 2048, 4096, 5000, 8192, 9999, 12_000, 16_384, 16_386, 20_000, 50_001])
@pytest.mark.parametrize("kind", [E4M3, I8])
@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
def test_codes_are_the_rounded_quotients(d, kind, types):
    # the mean of d ones as the kernel takes it, a product with the rounded 1 / d, is 1 for most widths; the next such one
    while np.float32(d) * np.float32(np.float32(1) / np.float32(d)) != 1:
        d += 1
    gen, n = torch.Generator().manual_seed(d), 7
    for block in (0, 32, 64, 128):
        w = _weights(gen, d, block, kind)
        sign = torch.randint(0, 2, (n, d), generator=gen) * 2.0 - 1
        x = sign.to(F32 if types == "f32" else BF16).cuda()
        residual = torch.zeros(n, d, device="cuda") if types == "mixed" else None
        q, scales, _, rstd = hb.rms_norm_quant_fwd(x, w.cuda(), residual=residual, eps=0.0, block=block, dtype=kind)
        assert (rstd == 1).all()
        y, width = sign * w, block or d
        parts = torch.nn.functional.pad(y, (0, -d % width)).view(n, -1, width)
        want = parts.abs().amax(2) * (torch.tensor(1.0) / torch.tensor(TOP[kind]))
        assert torch.equal(scales.cpu(), want), "scales"
        quotient = (parts / want[:, :, None]).view(n, -1)[:, :d]
        codes = quotient.round().to(I8) if kind is I8 else quotient.contiguous().to(E4M3)
        assert torch.equal(q.cpu().view(torch.uint8), codes.view(torch.uint8)), f"{int((q.cpu().float() != codes.float()).sum())} codes"
