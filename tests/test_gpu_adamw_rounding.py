"""8-bit states rounded by chance: what is stored is right on average, step for step and over long runs.

Neighbouring codes differ by a fraction d of their value, d between 1/16 and 1/8.  A value with the fraction f of the way from the
lower code to the upper one is stored with the variance f (1 - f) of that gap, so over N places its mean is off by
sqrt(f (1 - f) / N) of the gap; six of those are allowed, 2^-16 of a gap for random numbers of 16 bits, and 8 u of the value for
the fp32 operations in front.

Long runs, beta2 = 0.999.  A root moves by about e = 0.0005 of itself a step, so a rounding adds a variance of e d of its square.
Where gradients keep coming it is drawn back by e a step as well, which leaves d / 2: a deviation of at most 0.25 about 1, so that
nineteen in twenty lie within exp(+-1.64 * 0.25) = 0.66 to 1.51, and the median within 0.1 (half the variance is 0.03).  Where
a root falls freely for 3000 steps the variance is 3000 e d, at most 0.19, a deviation of 0.43 of the logarithm, with a median of
exp(-0.09) since the mean is kept: bounds of exp(-0.09 +- 1.3 * 1.64 * 0.43), and 0.75 to 1.3 for the median.
"""
import math

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library
from test_gpu_adamw_large import FEW

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E4M3, BF16 = torch.float8_e4m3fn, torch.bfloat16
CODES = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).double()             # 0 to 448, ascending


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ratios(state, exact):
    stored = state.square.float() * state.scales[:, 1:]
    return (stored.double() / exact).view(state.square.shape)


@pytest.mark.parametrize("change", [1.0, 30.0, 1 / 30])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_roots_follow_gradients_that_change_unequally(change, dtype):
    """Half of each block's gradients become larger or smaller after 2000 steps; 3000 steps later every root is where it should be."""
    blocks, gen = 64, _gen(1)
    p = torch.zeros(blocks * 256, device="cuda", dtype=dtype)
    state, v, size = hb.adamw_state([p], 8), torch.zeros(blocks, 256, device="cuda", dtype=torch.float64), torch.ones(256, device="cuda")
    for t in range(1, 5001):
        if t == 2001:
            size[128:] *= change
        g = (torch.randn(blocks, 256, generator=gen, device="cuda") * size).to(dtype)
        v.mul_(0.999).addcmul_(g.double(), g.double(), value=0.001)
        hb.adamw_step([p], [g.view(-1)], state, t, lr=1e-3, betas=(0.9, 0.999), seed=7)
    ratio = _ratios(state, v.sqrt())
    for half in (0, 1):
        r = ratio[:, 128 * half:128 * half + 128].flatten()
        low, mid, high = (float(torch.quantile(r, q)) for q in (0.05, 0.5, 0.95))
        if half and change < 1:
            assert 0.75 < mid < 1.3 and low > math.exp(-0.09 - 1.3 * 1.64 * 0.43) and high < math.exp(-0.09 + 1.3 * 1.64 * 0.43), (low, mid, high)
        else:
            assert 0.9 < mid < 1.1 and low > 0.66 and high < 1.51, (low, mid, high)


class Held:
    """Blocks whose largest values stay as they are, so that all others are multiplied by beta: codes whose next quotients are known."""
    B1, B2 = 0.93, 0.97

    def __init__(self, blocks, offset=0, dtype=torch.float32):
        n, self.blocks = blocks * 256, blocks
        self.p = torch.zeros(n + offset, device="cuda", dtype=dtype)[offset:]
        self.g = torch.zeros(n + offset, device="cuda", dtype=dtype)[offset:]
        self.g.view(-1, 256)[:, 0] = 448.0
        code = torch.randint(1, 127, (blocks, 256), generator=_gen(2), device="cuda", dtype=torch.uint8)
        sign = torch.randint(0, 2, (blocks, 256), generator=_gen(3), device="cuda", dtype=torch.uint8) * 128
        code[:, 0], sign[:, 0] = 126, 0
        self.code = code.long()
        self.start = [(code + sign), code.clone(), torch.ones(blocks, 2, device="cuda")]
        self.state = hb.adamw_state([self.p], 8)

    def step(self, t, **more):
        for to, value in zip(self.state, self.start):
            (to.view(torch.uint8) if to.dtype is E4M3 else to).copy_(value)
        hb.adamw_step([self.p], [self.g], self.state, t, lr=1e-3, betas=(self.B1, self.B2), **more)
        return [t.clone().view(torch.uint8) if t.dtype is E4M3 else t.clone() for t in self.state]


@pytest.mark.parametrize("blocks", [FEW + 1003, 2000])
def test_each_code_is_right_on_average(blocks):
    held = Held(blocks)
    mean, root, scales = held.step(1, seed=11)
    assert ((scales.double() - 1).abs() <= 8 * U).all()
    codes, code = CODES.cuda(), held.code[:, 1:].flatten()
    sign = torch.where(held.start[0][:, 1:] >= 128, -1.0, 1.0).flatten().double()
    for which, (now, beta) in enumerate(((mean, held.B1), (root, math.sqrt(held.B2)))):
        value = now[:, 1:].flatten().contiguous().view(E4M3).double() * (1 if which else sign)
        want = codes[code] * beta
        upper = torch.searchsorted(codes, want).clamp(max=126)
        lo, hi = codes[upper - 1], codes[upper]
        near = 8 * U * want
        assert ((value == lo) | (value == hi) | ((want - lo <= near) & (value == codes[(upper - 2).clamp(min=0)])) | ((hi - want <= near) & (value == codes[(upper + 1).clamp(max=126)]))).all()
        if which:                                               # a positive root does not become zero
            assert (value > 0).all()
            want = want.clamp(min=2.0 ** -9)
        f = (want - lo) / (hi - lo)
        gap = hi - lo
        n = torch.zeros(127, dtype=torch.float64, device="cuda").index_add_(0, code, torch.ones_like(want))
        off = torch.zeros_like(n).index_add_(0, code, value - want) / n.clamp(min=1)
        first = torch.zeros_like(n).index_copy_(0, code, f * (1 - f))
        bound = torch.zeros_like(n).index_copy_(0, code, gap) * (6 * (first / n.clamp(min=1)).sqrt() + 2.0 ** -16) + 8 * U * codes
        if which:                                               # below the smallest code nothing is left to chance
            bound[1] = 8 * U * codes[1]
        assert (n[1:] > blocks / 30).all() and (off.abs() <= bound)[1:].all()


def test_roundings_of_different_steps_and_seeds_are_independent():
    """The average over T steps from one start has a T-th of the variance: over 255 x 200 places it is known to 6 sqrt(2 / 51 000) = 4 %."""
    held, count = Held(200), 128
    codes, code = CODES.cuda(), held.code[:, 1:]
    for steps in (True, False):
        total = torch.zeros(200, 255, dtype=torch.float64, device="cuda")
        for t in range(1, count + 1):
            _, root, _ = held.step(t if steps else 5, seed=3 if steps else t)
            total += root[:, 1:].contiguous().view(E4M3).double()
        want = codes[code] * math.sqrt(held.B2)
        upper = torch.searchsorted(codes, want)
        gap = codes[upper] - codes[upper - 1]
        f = (want - codes[upper - 1]) / gap
        use = (f * (1 - f) > 0.01) & (code > 1)
        z = ((total / count - want) / gap).square()[use] / (f * (1 - f))[use] * count
        assert int(use.sum()) > 40_000 and abs(float(z.mean()) - 1) < 0.05


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("blocks", [40, FEW + 1003])
def test_equal_calls_give_equal_bits(dtype, blocks):
    """The bits depend on seed, step and place: not on the parameters' alignment, nor on where the step's number lies."""
    held, off = Held(blocks, 0, dtype), Held(blocks, 1, dtype)
    want = held.step(9, seed=5)
    for other in (held.step(9, seed=5), off.step(9, seed=5), held.step(torch.tensor(9, device="cuda"), seed=5), held.step(9, seed=5 + (1 << 64))):
        assert all(torch.equal(a, b) for a, b in zip(want, other))
    for other in (held.step(10, seed=5), held.step(9, seed=6), held.step(9, seed=-5), held.step(9)):
        assert not torch.equal(want[0], other[0]) and not torch.equal(want[1], other[1])


@pytest.mark.parametrize("bits", [8, 32])
def test_parameters_are_those_of_the_other_rounding(bits):
    """The step uses the states before they are rounded: a seed changes what is stored in 8 bits and nothing else."""
    gen, outs = _gen(5), []
    start = [torch.randn(5000, generator=gen, device="cuda"), torch.randn(333, generator=gen, device="cuda").to(BF16)]
    grads = [0.1 * torch.randn(p.shape, generator=gen, device="cuda").to(p.dtype) for p in start]
    for seed in (None, 4):
        params = [p.clone() for p in start]
        state = hb.adamw_state(params, bits)
        hb.adamw_step(params, grads, state, 1, seed=seed)
        outs.append((params, state))
    assert all(torch.equal(a, b) for a, b in zip(outs[0][0], outs[1][0]))
    same = [torch.equal(a.float(), b.float()) for a, b in zip(outs[0][1], outs[1][1]) if a is not None]
    assert same == ([False, False, True] if bits == 8 else [True, True])


def test_replays_of_a_graph_take_the_step_from_the_device():
    held = Held(100)
    count = torch.tensor(1, device="cuda")
    held.step(count, seed=8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.adamw_step([held.p], [held.g], held.state, count, lr=1e-3, betas=(held.B1, held.B2), seed=8)
    for t in (2, 3, 100):
        want = held.step(t, seed=8)
        for to, value in zip(held.state, held.start):
            (to.view(torch.uint8) if to.dtype is E4M3 else to).copy_(value)
        count.fill_(t)
        graph.replay()
        assert all(torch.equal(a.view(torch.uint8) if a.dtype is E4M3 else a, b) for a, b in zip(held.state, want))


def test_places_behind_the_end_zeros_and_values_that_are_not_finite():
    p = torch.randn(700, generator=_gen(6), device="cuda")
    g = 0.1 * torch.randn(700, generator=_gen(7), device="cuda")
    g[300:400] = 0
    state = hb.adamw_state([p], 8)
    for x in (state.mean, state.square):
        x.view(torch.uint8).view(-1)[700:] = 77
    g[5], g[600] = float("inf"), float("nan")
    hb.adamw_step([p], [g], state, 1, seed=1)
    for x in (state.mean, state.square):
        flat = x.view(torch.uint8).view(-1)
        assert (flat[700:] == 77).all() and not (flat[300:400] & 127).any()
        nan = x.float().view(-1)[:700].isnan()
        assert nan[5] and nan[600] and int(nan.sum()) == 2
    assert state.scales.isfinite().all()
    spread = torch.logspace(-12, 2, 1280, device="cuda")
    p, state = torch.zeros(1280, device="cuda"), hb.adamw_state([torch.zeros(1280, device="cuda")], 8)
    # every root stays positive, so every step is bounded: to lr sqrt(t) of the exact states, a quarter more for codes that are off by
    # an eighth, and 10 gaps of the mean (what roundings add up to with beta1 = 0.9) over a root of one gap, whose scales are at most
    # 3.2 apart, corrected by 5.3 / 22: 7.6
    for t in range(1, 40):
        old = p.clone()
        hb.adamw_step([p], [spread * (-1) ** t], state, t, lr=1e-3, eps=1e-30, weight_decay=0.0, seed=2)
        assert (state.square.float() > 0).all() and p.isfinite().all()
        assert (p - old).abs().max() <= 1e-3 * (1.25 * math.sqrt(40) + 8)


def test_refusals():
    p = [torch.ones(10, device="cuda")]
    with pytest.raises(TypeError):
        hb.adamw_step(p, [torch.ones(10, device="cuda")], hb.adamw_state(p, 8), 1, seed=1.5)
    assert (p[0] == 1).all()
