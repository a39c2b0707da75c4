"""The measured cases of the residual stack's norm and of the optimiser: root-mean-square norm with the residual's
addition (forward, forward with an 8-bit output, backward) and AdamW over many tensors with states in 32 or 8 bits.

A case names an operator and direction ("op"), its sizes and types.  `prepare` makes what a training or inference
program holds before the call, `run` makes one call: the plain torch form in 32 bits, or, where `own` is set, the
call of this package.  `exact` is the definition in 64 bits.
"""
import itertools
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_MOST = 256_000_000          # elements of the largest case
_EPS = 1e-5
_E4M3 = torch.float8_e4m3fn
_TOP = 448.0                 # the largest value of e4m3, and what the largest of a block is scaled to
_LEAST = 2.0 ** -126         # the smallest scale
_LOWEST = 2.0 ** -9          # the smallest positive value of e4m3
_BLOCK = 256                 # elements that share a scale of the 8-bit states
_LR, _B1, _B2, _ADAM_EPS, _DECAY, _STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 20

# types of a norm: those of x, of the residual stream, and of y
_NORM = {"f32": ("f32", "f32", "f32"), "bf16": ("bf16", "bf16", "bf16"), "mixed": ("bf16", "f32", "bf16")}
# types of a parameter, its gradient, and the copy that the next forward pass reads
_ADAM = {"f32": ("f32", "f32", None), "bf16": ("bf16", "bf16", None), "mixed": ("f32", "bf16", "bf16")}


# --------------------------------------------------------------------------- cases
def listed():
    return [
        # one node's or token's row joins the residual stream, as in inference one at a time: all latency
        dict(name="rms fwd 1x4096", op="rms_fwd", n=1, d=4096, types="bf16", weights="bf16", residual=True, pad=0),
        # a layer of a graph of 233 000 nodes
        dict(name="rms fwd 233k x128", op="rms_fwd", n=233_000, d=128, types="f32", weights="f32", residual=True, pad=0),
        # a million nodes, bf16 layers around an fp32 residual stream
        dict(name="rms fwd 1M x256 mixed", op="rms_fwd", n=1_000_000, d=256, types="mixed", weights="f32", residual=True, pad=0),
        # a small batch on its way into an 8-bit product, one scale per 128 columns
        dict(name="rms fwd8 64x4096", op="rms_fwd8", n=64, d=4096, types="bf16", weights="bf16", residual=True, block=128, pad=0),
        # the largest layer's input of an 8-bit product, one scale per row
        dict(name="rms fwd8 1M x256", op="rms_fwd8", n=1_000_000, d=256, types="bf16", weights="f32", residual=True, block=0, pad=0),
        # an odd width, rows that are part of a wider matrix, no residual stream
        dict(name="rms bwd 5001x1433", op="rms_bwd", n=5001, d=1433, types="f32", weights="f32", residual=False, pad=7),
        # the gradient of the largest layer, with what arrives along the residual stream
        dict(name="rms bwd 1M x256", op="rms_bwd", n=1_000_000, d=256, types="bf16", weights="f32", residual=True, pad=0),
        # the parameters of a small network: 12 small tensors
        dict(name="adamw 12 tensors 50k", op="adamw", bits=32, tensors=12, elements=50_000, types="f32", clip=True, shift=0),
        # a large table and 23 further tensors, bf16 gradients, fp32 parameters with their bf16 copies
        dict(name="adamw 24 tensors 200M", op="adamw", bits=32, tensors=24, elements=200_000_000, types="mixed", clip=True, shift=0),
        # the small network's with 8-bit states
        dict(name="adamw8 12 tensors 50k", op="adamw", bits=8, tensors=12, elements=50_000, types="f32", clip=True, shift=0),
        # an ordinary network: 2 million fp32 parameters
        dict(name="adamw8 30 tensors 2M", op="adamw", bits=8, tensors=30, elements=2_000_000, types="f32", clip=False, shift=0),
        # the large table and 39 further tensors in bf16: what 8-bit states are for
        dict(name="adamw8 40 tensors 200M", op="adamw", bits=8, tensors=40, elements=200_000_000, types="bf16", clip=True, shift=0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: most are multiples of 8, as feature widths are; the rest is any number."""
    d = _log(rng, lo, hi)
    return max(8, d // 8 * 8) if rng.random() < 0.65 else d


def draw(rng):
    op = rng.choice(["rms_fwd", "rms_fwd8", "rms_bwd", "adamw", "adamw"])
    if op == "adamw":
        types = rng.choice(["f32", "bf16", "mixed"])
        return dict(op=op, bits=rng.choice([8, 32]), tensors=rng.randint(1, 28), elements=_log(rng, 1000, 200_000_000), types=types,
                    clip=rng.random() < 0.5, shift=rng.choice([0, 0, 0, 1]))
    d = _width(rng, 4, 16384)
    case = dict(op=op, n=_log(rng, 1, _MOST // (2 * d)), d=d, types=rng.choice(["f32", "bf16", "mixed"]), weights=rng.choice(["f32", "bf16"]),
                residual=rng.random() < 0.75, pad=rng.choice([0, 0, 0, 8, 5]))
    if case["types"] == "mixed":
        case["residual"] = True
    if op == "rms_fwd8":
        case["block"] = rng.choice([0, 32, 64, 128])
    return case


# --------------------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _rows(gen, case, spread, dtype):
    return _normal(gen, case["n"], case["d"] + case["pad"]).mul_(spread).to(_DT[dtype])[:, :case["d"]]


def _lengths(case):
    """Lengths of the tensors: one large, the others fall off; odd numbers among them, a short one of 7."""
    t, total = case["tensors"], case["elements"]
    share = [0.5 ** min(k, 9) for k in range(t)]
    out = [max(1, int(total * s / sum(share)) - k % 2) for k, s in enumerate(share)]
    if t > 2:
        out[-1] = 7
    return out


def _first_blocks(lens):
    """Where each tensor's states begin, in blocks; the last number is that of all blocks."""
    return list(itertools.accumulate((-(-m // _BLOCK) for m in lens), initial=0))


def _inside(lens):
    """Which of the states' places belong to a tensor: True where they do, [blocks, 256]."""
    first = _first_blocks(lens)
    here = torch.zeros(first[-1] * _BLOCK, dtype=torch.bool, device="cuda")
    [here[b * _BLOCK:b * _BLOCK + m].fill_(True) for b, m in zip(first, lens)]
    return here.view(-1, _BLOCK)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "adamw":
        return _prepare_adamw(s, case, gen)
    tx, ts, ty = _NORM[case["types"]]
    d = case["d"]
    s["w"] = (1 + 0.1 * _normal(gen, d)).to(_DT[case["weights"]])
    if case["op"] == "rms_bwd":     # what the forward pass left, and what arrives from above
        s["total"] = _rows(gen, case, 2.0, ts)
        s["rstd"] = torch.rsqrt(s["total"].float().square().mean(1) + _EPS)
        s["grad"] = _normal(gen, case["n"], d).to(_DT[ty])
        s["grad_total"] = _normal(gen, case["n"], d).to(_DT[ts]) if case["residual"] else None
    else:                           # the residual stream is wider than what a layer adds to it
        s["x"] = _rows(gen, case, 1.0, tx)
        s["residual"] = _rows(gen, case, 2.0, ts) if case["residual"] else None
    return s


def _prepare_adamw(s, case, gen):
    lens = _lengths(case)
    tp, tg, tc = (_DT.get(t) for t in _ADAM[case["types"]])
    off = case["shift"]             # tensors that are parts of a flat buffer may begin anywhere
    s["params"] = [_normal(gen, m + off).to(tp)[off:] for m in lens]
    s["grads"] = [(0.01 * _normal(gen, m + off)).to(tg)[off:] for m in lens]
    s["copies"] = [torch.empty(m + off, dtype=tc, device="cuda")[off:] for m in lens] if tc else None
    # the states after some steps: a mean smaller than the root of the mean square, over a few orders of magnitude
    here = _inside(lens)
    size = torch.exp(_normal(gen, *here.shape)).mul_(0.01)
    m, root = _normal(gen, *here.shape).mul_(size).mul_(0.3 * here), size.mul_(here)
    if case["bits"] == 32:
        s["state"] = (m, root.square_(), None)
    else:
        s["state"] = _to_8_bits(m, root)
    s["norm"] = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt() if case["clip"] else None
    s["max_norm"] = 0.005 * math.sqrt(sum(lens)) if case["clip"] else None
    return s


def _to_8_bits(m, root):
    """Mean and root as e4m3 with one scale each per block: a positive root stays positive."""
    scales = torch.stack([m.abs().amax(1), root.amax(1)], 1).div_(_TOP).clamp_(min=_LEAST)
    inverse = scales.reciprocal()
    m8 = (m * inverse[:, :1]).to(_E4M3)
    root8 = torch.where(root > 0, (root * inverse[:, 1:]).clamp_(min=_LOWEST), 0.0).to(_E4M3)
    return m8, root8, scales


# --------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _run_own(s, case):
    import paper_1906_03707_b200 as hb
    op = case["op"]
    if op == "rms_fwd":
        return hb.rms_norm_fwd(s["x"], s["w"], residual=s["residual"], eps=_EPS)
    if op == "rms_fwd8":
        return hb.rms_norm_quant_fwd(s["x"], s["w"], residual=s["residual"], eps=_EPS, block=case["block"])
    if op == "rms_bwd":
        return hb.rms_norm_bwd(s["grad"], s["total"], s["rstd"], s["w"], grad_total=s["grad_total"], x_dtype=_DT[_NORM[case["types"]][0]])
    hb.adamw_step(s["params"], s["grads"], s["state"], _STEP, lr=_LR, betas=(_B1, _B2), eps=_ADAM_EPS, weight_decay=_DECAY,
                  total_norm=s["norm"], max_norm=s["max_norm"], copies=s["copies"])
    return s["params"], s["copies"], s["state"]


def _run_plain(s, case):
    op = case["op"]
    if op == "adamw":
        return _plain_adamw(s, case)
    w = s["w"].float()
    tx, ts, ty = (_DT[t] for t in _NORM[case["types"]])
    if op == "rms_bwd":
        rstd = s["rstd"][:, None]
        hat, g = s["total"].float() * rstd, s["grad"].float()
        q = g * w
        grad = (q - hat * (q * hat).mean(1, keepdim=True)) * rstd
        if s["grad_total"] is not None:
            grad += s["grad_total"].float()
        return grad.to(tx), grad.to(ts), (g * hat).sum(0).to(s["w"].dtype)
    total = s["x"].float()
    if s["residual"] is not None:
        total = total + s["residual"].float()
    rstd = torch.rsqrt(total.square().mean(1) + _EPS)
    y = total * rstd[:, None] * w
    if op == "rms_fwd":
        return y.to(ty), total.to(ts), rstd
    n, d = y.shape
    block = case["block"] or d
    parts = torch.nn.functional.pad(y, (0, -d % block)).view(n, -1, block)
    scales = (parts.abs().amax(2) / _TOP).clamp_(min=_LEAST)
    q = (parts / scales[:, :, None]).view(n, -1)[:, :d].contiguous().to(_E4M3)
    return q, scales, total.to(ts), rstd


def _plain_adamw(s, case):
    lens, state = _lengths(case), s["state"]
    first = _first_blocks(lens)
    factor = 1.0 if s["norm"] is None else (s["max_norm"] / (s["norm"] + 1e-6)).clamp(max=1.0)
    rate, root_correction = _LR / (1 - _B1 ** _STEP), math.sqrt(1 - _B2 ** _STEP)

    def one(p, g, m, v, scales):
        """One tensor: its states of whole blocks are brought up to date, behind its end they stay zero."""
        k = p.numel()
        grad = torch.zeros(m.numel(), device=p.device)
        grad[:k] = g.reshape(-1).float() * factor
        grad = grad.view(-1, _BLOCK)
        m32 = m.float() if scales is None else m.float() * scales[:, :1]
        v32 = v.float() if scales is None else (v.float() * scales[:, 1:]).square()
        m32 = m32 * _B1 + grad * (1 - _B1)
        v32 = v32 * _B2 + grad.square() * (1 - _B2)
        step = m32.view(-1)[:k] / (v32.view(-1)[:k].sqrt() / root_correction + _ADAM_EPS)
        p32 = p.reshape(-1).float() * (1 - _LR * _DECAY) - step * rate
        p.view(-1).copy_(p32)
        if scales is None:
            m.copy_(m32), v.copy_(v32)
        else:
            [old.copy_(new) for old, new in zip((m, v, scales), _to_8_bits(m32, v32.sqrt()))]
        return p32

    of = [tuple(None if t is None else t[a:b] for t in state) for a, b in zip(first, first[1:])]
    news = [one(p, g, *parts) for p, g, parts in zip(s["params"], s["grads"], of)]
    if s["copies"] is not None:
        [c.copy_(p32) for c, p32 in zip(s["copies"], news)]
    return s["params"], s["copies"], state


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "adamw":
        lens = _lengths(case)
        p, g, c = (_SIZE.get(t, 0) for t in _ADAM[case["types"]])
        state = 16 if case["bits"] == 32 else 4 + 16 / _BLOCK
        return {"bytes": sum(lens) * (2 * p + g + c + state), "flops": 20 * sum(lens)}
    n, d = case["n"], case["d"]
    x, t, y = (_SIZE[k] for k in _NORM[case["types"]])
    w, res = _SIZE[case["weights"]], case["residual"]
    if case["op"] == "rms_bwd":
        return {"bytes": n * d * (y + t + (t if res else 0) + t + (x if case["types"] == "mixed" else 0)) + 4 * n + 2 * d * w, "flops": 10 * n * d}
    out = y if case["op"] == "rms_fwd" else 1
    scales = 0 if case["op"] == "rms_fwd" else 4 * n * -(-d // (case["block"] or d))
    return {"bytes": n * d * (x + out + (2 * t if res else 0)) + 4 * n + scales + d * w, "flops": (5 if out > 1 else 8) * n * d}


# --------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "adamw":
        return _exact_adamw(s, case)
    w = s["w"].double()
    if op == "rms_bwd":
        rstd, h = s["rstd"].double(), s["total"].double()
        g = s["grad"].double()
        grad_w = torch.einsum("rd,rd,r->d", g, h, rstd)
        g *= w
        along = torch.einsum("rd,rd->r", g, h) * rstd.pow(3) / case["d"]
        g.mul_(rstd[:, None]).addcmul_(h, along[:, None], value=-1)
        if s["grad_total"] is not None:
            g += s["grad_total"]
        return g, g, grad_w
    h = s["x"].double()
    if s["residual"] is not None:
        h = h + s["residual"]
    rstd = 1.0 / torch.sqrt(torch.einsum("rd,rd->r", h, h) / case["d"] + _EPS)
    y = torch.einsum("rd,r,d->rd", h, rstd, w)
    if op == "rms_fwd":
        return y, h, rstd
    block = case["block"] or case["d"]
    pieces = y.split(block, 1)
    scales = torch.stack([torch.linalg.vector_norm(p, math.inf, dim=1) / _TOP for p in pieces], 1)
    return torch.cat([p / scales[:, k:k + 1] for k, p in enumerate(pieces)], 1), scales, h, rstd


def _exact_adamw(s, case):
    """All tensors at once, at the places of their states; the 8-bit states as the quotients before they are rounded."""
    lens, (m, v, scales) = _lengths(case), s["state"]
    here = _inside(lens)
    grad, param = torch.zeros(2, here.numel(), device="cuda", dtype=torch.float64)
    flat = here.view(-1)
    grad[flat], param[flat] = torch.cat(s["grads"]).double(), torch.cat(s["params"]).double()
    if s["norm"] is not None:
        grad *= min(1.0, s["max_norm"] / (float(s["norm"]) + 1e-6))
    grad, m, v = grad.view(-1, _BLOCK), m.double(), v.double()
    if scales is not None:
        m, v = m * scales[:, 0].double()[:, None], (v * scales[:, 1].double()[:, None]) ** 2
    m = torch.lerp(m, grad, 1 - _B1)
    v = _B2 * v + (1 - _B2) * grad * grad
    hat_m, hat_v = m / (1 - _B1 ** _STEP), v / (1 - _B2 ** _STEP)
    param -= _LR * (hat_m / (hat_v.sqrt() + _ADAM_EPS) + _DECAY * param.view(-1, _BLOCK)).view(-1)
    news = param[flat].split(lens)
    if scales is None:
        return news, None if s["copies"] is None else news, (m, v, None)
    root = v.sqrt()
    tops = torch.stack([m.abs().amax(1), root.amax(1)], 1).div(_TOP).clamp(min=_LEAST)
    return news, None if s["copies"] is None else news, (m / tops[:, :1], root / tops[:, 1:], tops)
