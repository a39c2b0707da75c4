"""GPU parity of the AdamW step over a list of tensors, against the formula in 64 bits.

Bounds, u = 2^-24.  What is read of an 8-bit state carries 1 u (m) and 3 u (v); the factor of the gradient 4 u, the scaled
gradient 5 u; a coefficient rounded to fp32 1 u, each operation 1 u:
  m   u (4 b1 |m| + 12 (1 - b1) |g|)
  v   u (6 b2 v + 20 (1 - b2) g^2), so at most 20 u of the new v and 10 u of its root
  p   4 u |p| + rate / denominator (error of m + 24 u |m|): the denominator has the root's 10 u, 2 u of the approximate root,
      3 u of its product, of eps and of their sum, the quotient 4 u, the rate and the last operations the rest
8-bit states: the scale is the largest value's error and 3 u; a stored value is half a step from the new one (2^-4 of it or
2^-10 of the scale's unit), a root below the smallest code is raised to it, 2^-9.  bf16 parameters add one rounding, 2^-8.
"""
import math

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
KINDS = {"f32": (F32, F32), "bf16": (BF16, BF16), "mixed": (F32, BF16), "odd": (BF16, F32)}


@pytest.fixture(scope="module", autouse=True)
def _library():
    build_library()
    hb.load_library()
    assert torch.cuda.is_available(), "the parity tests need a CUDA device"


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


class Case:
    """Parameters, gradients and states after some steps, and the formula's answer for the next."""

    def __init__(self, seed, lengths, kinds=("f32",), bits=32, offset=0, goffset=None):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        goffset = offset if goffset is None else goffset
        self.bits, self.lengths = bits, lengths
        self.params, self.grads = [], []
        for i, m in enumerate(lengths):
            tp, tg = KINDS[kinds[i % len(kinds)]]
            self.params.append(_randn(gen, m + offset).to(tp)[offset:])
            self.grads.append((0.05 * _randn(gen, m + goffset)).to(tg)[goffset:])
        self.state = hb.adamw_state(self.params, bits)
        self.first = [0]
        for m in lengths:
            self.first.append(self.first[-1] + -(-m // 256))
        if self.state.mean.numel():
            size = 0.05 * torch.exp(_randn(gen, *self.state.mean.shape))
            mean, root = 0.3 * size * _randn(gen, *size.shape), size
            if bits == 32:
                self.state.mean.copy_(mean), self.state.square.copy_(root * root)
            else:                                               # any codes and scales are states
                self.state.mean.copy_((mean * 900).clamp(-448, 448)), self.state.square.copy_((root * 900).clamp(2.0 ** -9, 448))
                self.state.scales.copy_(torch.exp(0.3 * _randn(gen, *self.state.scales.shape)) / 900)

    def decoded(self, t):
        a, b, m = self.first[t], self.first[t + 1], self.lengths[t]
        mean, square = self.state.mean[a:b].double(), self.state.square[a:b].double()
        if self.bits == 8:
            s = self.state.scales[a:b].double()
            mean, square = mean * s[:, :1], (square * s[:, 1:]).square()
        return mean.reshape(-1)[:m], square.reshape(-1)[:m]

    def check(self, step=7, lr=3e-3, betas=(0.9, 0.99), eps=1e-8, decay=0.05, norm=None, max_norm=None, missing=(), call=None, **more):
        b1, b2 = betas
        c = 1.0 if norm is None else min(1.0, max_norm / (float(norm) + 1e-6))
        decays = decay if isinstance(decay, list) else [decay] * len(self.lengths)
        before = []
        for t, (p, g) in enumerate(zip(self.params, self.grads)):
            mean, square = self.decoded(t)
            before.append((p.double().reshape(-1).clone(), g.double().reshape(-1).clone(), mean.clone(), square.clone()))
        raw = [None if x is None else x.clone() for x in self.state]
        grads = [None if t in missing else g for t, g in enumerate(self.grads)]
        if call is None:
            got = hb.adamw_step(self.params, grads, self.state, step, lr=lr, betas=betas, eps=eps, weight_decay=decay, total_norm=norm, max_norm=max_norm, **more)
            assert got is self.params
        else:
            call()
        rate, root = lr / (1 - b1 ** step), 1 / math.sqrt(1 - b2 ** step)
        for t, (p, g, m, v) in enumerate(before):
            a, b, k = self.first[t], self.first[t + 1], self.lengths[t]
            behind = [x[a:b].reshape(-1)[k:].float() for x in (self.state.mean, self.state.square, raw[0], raw[1])]
            assert torch.equal(behind[0], behind[2]) and torch.equal(behind[1], behind[3])       # behind a tensor's end nothing changes
            if t in missing:
                assert torch.equal(self.params[t].double().reshape(-1), p)
                for x, y in zip(self.state, raw):
                    assert x is None or torch.equal(x[a:b].float(), y[a:b].float())
                continue
            if k == 0:
                continue
            g = g * c
            m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
            em = U * (4 * b1 * m.abs() + 12 * (1 - b1) * g.abs())
            ev = U * (6 * b2 * v + 20 * (1 - b2) * g * g)
            den = v1.sqrt() * root + eps
            p1 = p * (1 - lr * decays[t]) - rate * m1 / den
            bound = 4 * U * p.abs() + rate / den * (em + 24 * U * m1.abs())
            new = self.params[t].double().reshape(-1)
            rounding = 2.0 ** -8 * p1.abs() if self.params[t].dtype == BF16 else 0
            assert ((new - p1).abs() <= bound + rounding).all(), f"p[{t}]: {((new - p1).abs() - bound).max().item():.2e}"
            if "copies" in more and more["copies"] is not None and more["copies"][t] is not None:
                copy = more["copies"][t].double().reshape(-1)
                assert ((copy - p1).abs() <= bound + 2.0 ** -8 * p1.abs()).all(), "copy"
            mean, square = self.decoded(t)
            if self.bits == 32:
                assert ((mean - m1).abs() <= em).all() and ((square - v1).abs() <= ev).all()
                continue
            for which, (now, want, err) in enumerate(((mean, m1, em), (square.sqrt(), v1.sqrt(), 14 * U * v1.sqrt()))):
                pad = (b - a) * 256 - k
                scale = self.state.scales[a:b, which].double()
                blocks = torch.nn.functional.pad(want.abs(), (0, pad)).view(-1, 256)
                top = (blocks.amax(1) / 448).clamp(min=2.0 ** -126)
                slack = torch.nn.functional.pad(err, (0, pad)).view(-1, 256).amax(1) / 448 + 3 * U * top
                assert ((scale - top).abs() <= slack).all(), "scale"
                each = scale.repeat_interleave(256)[:k]
                unit = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * each)
                if which:
                    unit = torch.where(want < 2.0 ** -9 * each, 2.0 ** -9 * each, unit)
                    assert (now[want > 0] > 0).all()
                assert ((now - want).abs() <= unit * (1 + 16 * U) + err * 1.125 + 8 * U * want.abs()).all(), "code"


LISTS = [[1], [7, 0, 3], [256], [257, 255, 512], [64, 64 * 64, 1, 4097, 0, 12_289], [100_000, 5, 8192, 8193, 65_537, 31], [16] * 300,
         [int(1.7 ** k) for k in range(28)], [0, 0, 1], [3_000_001, 2]]


@pytest.mark.parametrize("lengths", LISTS)
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("kinds", [("f32",), ("bf16",), ("mixed", "f32", "odd", "bf16")])
def test_lists(lengths, bits, kinds):
    Case(1, lengths, kinds, bits).check()
    case = Case(2, lengths, kinds, bits)
    copies = [None if t % 3 == 2 else torch.empty(m, dtype=BF16, device="cuda") for t, m in enumerate(lengths)]
    norm = hb.grad_norm(case.grads)
    case.check(norm=norm, max_norm=0.3 * float(norm), decay=[0.01 * (t % 4) for t in range(len(lengths))], copies=copies, eps=1e-3)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("offset,goffset", [(1, 1), (2, 2), (3, 0), (0, 1), (4, 2), (5, 7)])
def test_pointers_off_the_vector_boundary(bits, offset, goffset):
    case = Case(3, [10_000, 17, 4096, 1, 300], ("f32", "bf16", "mixed"), bits, offset, goffset)
    wide = torch.full((5000,), 3.0, device="cuda", dtype=BF16)
    case.check(copies=[None, None, wide[offset:offset + 4096], None, None])
    assert (wide[:offset] == 3).all() and (wide[offset + 4096:] == 3).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_missing_gradients_leave_everything(bits):
    case = Case(4, [1000, 300, 0, 513, 70_000], ("f32", "bf16"), bits)
    case.check(missing=(1, 4))
    case.check(missing=(0, 1, 2, 3, 4), step=8)


@pytest.mark.parametrize("bits", [8, 32])
def test_first_step_from_zeros_and_many_steps(bits):
    """From zero states the first step is lr * g / (|g| + eps'); then twenty steps, each from the states as they are."""
    case = Case(5, [5000, 77], ("f32",), bits)
    for t in case.state:
        if t is not None:
            t.zero_()
    p, g = case.params[0].double().clone(), case.grads[0].double()
    case.check(step=1, decay=0.0, lr=1e-2, betas=(0.9, 0.999))
    want = p - 1e-2 * g / (g.abs() + 1e-8)
    assert ((case.params[0].double() - want).abs() <= 4 * U * p.abs() + 60 * U * 1e-2).all()
    for t in range(2, 22):
        case.check(step=t)


def test_eight_bits_keep_roots_positive_and_steps_bounded():
    """A block whose gradients span 14 orders of magnitude: every root stays positive, so no step exceeds lr * sqrt(t)."""
    n = 256 * 5
    g = torch.logspace(-12, 2, n, device="cuda")
    p = torch.zeros(n, device="cuda")
    state = hb.adamw_state([p], 8)
    for t in range(1, 40):
        old = p.clone()
        hb.adamw_step([p], [g * (-1) ** t], state, t, lr=1e-3, eps=1e-30, weight_decay=0.0)
        assert (p - old).abs().max() <= 1e-3 * math.sqrt(40) and p.isfinite().all()
        assert (state.square.float() > 0).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_values_that_are_not_finite_stay_alone(bits):
    case, clean = Case(6, [2000, 300], ("f32",), bits), Case(6, [2000, 300], ("f32",), bits)
    hb.adamw_step(clean.params, clean.grads, clean.state, 7)
    case.grads[0][100], case.grads[0][101], case.grads[1][299] = float("inf"), float("nan"), float("-inf")
    hb.adamw_step(case.params, case.grads, case.state, 7)
    for t, at in ((0, [100, 101]), (1, [299])):
        keep = torch.ones(case.lengths[t], dtype=torch.bool, device="cuda")
        keep[at] = False
        assert torch.equal(case.params[t][keep], clean.params[t][keep]) and not case.params[t][~keep].isfinite().any()
        if bits == 32:
            for now, then in zip(case.decoded(t), clean.decoded(t)):
                assert torch.equal(now[keep], then[keep]) and not now[~keep].isfinite().any()
        else:
            a, b = case.first[t], case.first[t + 1]
            for x in (case.state.mean, case.state.square):
                assert x[a:b].float().reshape(-1)[at].isnan().all()
                assert x[a:b].float().reshape(-1)[:case.lengths[t]].isnan().sum() == len(at)
            assert case.state.scales.isfinite().all()
    norm = torch.full((), float("nan"), device="cuda")
    hb.adamw_step(case.params, case.grads, case.state, 8, total_norm=norm, max_norm=1.0)
    assert case.params[0].isnan().all()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("norm,max_norm", [(1e38, math.inf), (3e38, math.inf), (1e38, 1e38), (2.0, math.inf), (0.0, 0.0), (0.0, 1.0), (2.0, 0.0), (1e-30, 1e-30)])
def test_ends_of_the_norm(bits, norm, max_norm):
    """min(1, max_norm / (norm + 1e-6)) where a quotient may overflow or vanish."""
    Case(10, [3000, 41], ("f32", "bf16"), bits).check(norm=torch.tensor(norm, device="cuda"), max_norm=max_norm)


@pytest.mark.parametrize("bits", [8, 32])
def test_places_without_gradient_do_not_move_but_for_decay(bits):
    """Rows of a table that no batch names: m and v stay zero, and p (1 - lr decay) is exact to 2 u and the rounding."""
    p, g = torch.randn(5000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(11)), torch.zeros(5000, device="cuda")
    g[700:900] = 0.5
    state = hb.adamw_state([p], bits)
    want = p.double()
    for t in range(1, 6):
        hb.adamw_step([p], [g], state, t, lr=1e-2, weight_decay=0.1)
        want = want * (1 - 1e-3)
    still = torch.ones(5000, dtype=torch.bool, device="cuda")
    still[700:900] = False
    assert ((p.double() - want).abs()[still] <= 5 * 3 * U * want.abs()[still]).all()
    places = still.new_zeros(state.mean.shape).view(-1)
    places[:5000] = still
    for x in (state.mean, state.square):
        assert not x.float().view(-1)[places].any() and (x.float().view(-1)[700:900] != 0).all()


def test_runs_repeat_and_shapes():
    outs = []
    for _ in range(2):
        case = Case(7, [120, 64, 1, 90_001], ("f32", "bf16"), 8)
        case.params, case.grads = ([t.view(s) for t, s in zip(x, [(4, 5, 6), (8, 8), (), (90_001, 1)])] for x in (case.params, case.grads))
        case.check()
        outs.append([*case.params, case.state.mean.float(), case.state.square.float(), case.state.scales])
    assert all(torch.equal(p, q) for p, q in zip(*outs))


@pytest.mark.parametrize("bits", [8, 32])
def test_rate_and_step_on_the_device_and_graph_capture(bits):
    case = Case(8, [50_000, 70, 9001], ("f32", "mixed"), bits)
    rate, count = torch.tensor(2e-3, device="cuda"), torch.tensor(5, device="cuda")
    lr = float(rate)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        case.check(step=5, lr=lr, call=lambda: hb.adamw_step(case.params, case.grads, case.state, count, lr=rate, betas=(0.9, 0.99), weight_decay=0.05))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = hb.grad_norm(case.grads)
        hb.adamw_step(case.params, case.grads, case.state, count, lr=rate, betas=(0.9, 0.99), weight_decay=0.05, total_norm=norm, max_norm=2.0)
    for t in (6, 7, 1_000_000):
        count.fill_(t)
        rate.fill_(1e-3 * (t % 5 + 1))
        case.grads[0].mul_(1.1)
        case.check(step=t, lr=float(rate), norm=hb.grad_norm(case.grads), max_norm=2.0, call=graph.replay)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_tensor_beyond_32_bits(bits):
    n = (1 << 31) + 10_007
    p, g = torch.full((n,), 0.5, dtype=BF16, device="cuda"), torch.full((n,), 0.25, dtype=BF16, device="cuda")
    small = torch.ones(5, device="cuda")
    state = hb.adamw_state([p, small], bits)
    g[-1] = -4.0
    hb.adamw_step([p, small], [g, torch.ones(5, device="cuda")], state, 1, lr=0.125, weight_decay=0.0)
    for i in (0, (1 << 31) - 1, 1 << 31, n - 2, n - 1):
        assert abs(float(p[i]) - (0.375 if i != n - 1 else 0.625)) <= 2.0 ** -8
    assert ((small - 0.875).abs() < 1e-6).all()
    last = state.mean[-2].float() * (1 if bits == 32 else state.scales[-2, 0])
    k = n % 256
    assert abs(float(last[k - 1]) + 0.4) < 0.03 and abs(float(last[k - 2]) - 0.025) < 0.002 and not last[k:].any()


def test_refusals():
    case = Case(9, [100, 300], ("f32",), 8)
    p, g, s = case.params, case.grads, case.state
    other = hb.adamw_state(p, 32)
    before = [t.clone() for t in p]
    one, count = torch.tensor(1e-3, device="cuda"), torch.tensor(1, device="cuda")
    for call in (lambda: hb.adamw_step([], [], s, 1), lambda: hb.adamw_step(p, g[:1], s, 1), lambda: hb.adamw_step(p, g[::-1], s, 1),
                 lambda: hb.adamw_step([p[0].cpu(), p[1]], g, s, 1), lambda: hb.adamw_step([p[0], p[0]], [g[0], g[0]], s, 1),
                 lambda: hb.adamw_step(p, p, s, 1), lambda: hb.adamw_step(p, g, s, 1, copies=[None]), lambda: hb.adamw_step(p, g, s, 1, copies=p),
                 lambda: hb.adamw_step(p, g, (other.mean, other.square, s.scales), 1), lambda: hb.adamw_step(p, g, (s.mean, s.square, None), 1),
                 lambda: hb.adamw_step(p[:1], g[:1], s, 1), lambda: hb.adamw_step(p, g, s, 1, weight_decay=[0.1]),
                 lambda: hb.adamw_step(p, g, s, 1, total_norm=one), lambda: hb.adamw_step(p, g, s, 1, max_norm=1.0),
                 lambda: hb.adamw_step(p, g, s, one), lambda: hb.adamw_step(p, g, s, 1, lr=count), lambda: hb.adamw_state(p, 16), lambda: hb.adamw_state([]),
                 lambda: hb.adamw_step([p[1].view(20, 15).t(), p[0]], g[::-1], s, 1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        hb.adamw_step([t.half() for t in p], g, s, 1)
    for more in (dict(step=0), dict(step=1, lr=-1.0), dict(step=1, betas=(1.0, 0.9)), dict(step=1, betas=(0.9, -0.1)), dict(step=1, eps=-1e-8),
                 dict(step=1, weight_decay=-0.1), dict(step=1, lr=float("nan")), dict(step=1, total_norm=one, max_norm=-1.0)):
        with pytest.raises(hb.HagError) as e:
            hb.adamw_step(p, g, s, **more)
        assert e.value.status == hb.HAG_ERR_ARG
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(p, before))


@pytest.mark.parametrize("n,d", [(1, 256), (300, 256), (40, 9000), (700, 333), (64, 9001)])
def test_steps_and_norms_behind_one_another(n, d):
    """Kernels start while those before them still run: 100 steps whose norms read the weights that the step before wrote,
    with nothing waited for, give the bits that they give with a wait after every call."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    x, start, table = _randn(gen, n, d), 1 + 0.1 * _randn(gen, d), _randn(gen, 50, d)
    ids = torch.randint(0, 50, (n,), generator=gen, device="cuda")

    def run(wait):
        wait()
        w, t, kept = start.clone(), table.clone(), []
        state = hb.adamw_state([w, t], 8)
        for k in range(1, 101):
            for call in (lambda: hb.embedding_fwd(ids, t), lambda: hb.rms_norm_fwd(kept[-1], w, residual=x),
                         lambda: hb.rms_norm_bwd(kept[-1][0], kept[-1][1], kept[-1][2], w, grad_total=x),
                         lambda: hb.adamw_step([w, t], [kept[-1][2], hb.embedding_bwd(ids, kept[-1][0], 50)], state, k, lr=0.05,
                                               total_norm=hb.grad_norm([kept[-1][2]]), max_norm=1.0)):
                kept.append(call())
                wait()
            kept[-1] = w.clone()
            wait()
        return [u for v in kept for u in (v if isinstance(v, tuple) else (v,))] + [t, *state]

    fast, slow = run(lambda: None), run(torch.cuda.synchronize)
    torch.cuda.synchronize()
    assert len(fast) == len(slow)
    for a, b in zip(fast, slow):
        assert torch.equal(a.float(), b.float())
