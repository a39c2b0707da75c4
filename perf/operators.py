"""The measured cases of the operators around the aggregation: embedding, layer norm, and clipping by the global norm.

A case names an operator and direction ("op"), its sizes and types.  `prepare` makes what a training or
inference program holds before the call, `run` makes one call: the plain torch form in 32 bits, or, where
`own` is set, the call of this package.  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_MOST = 256_000_000          # elements of the largest case
_EPS = 1e-5


# --------------------------------------------------------------------------- cases
def listed():
    return [
        # 1 000 nodes, 16 learned features each, looked up in a shuffled order: the smallest call, all latency
        dict(name="embed fwd 1000x16", op="embed_fwd", n=1000, v=1000, d=16, ids="i64", spread="perm", table="f32", rows="f32", scale=1.0),
        # a batch of 5 000 graphs of 100 nodes whose types (119 of them, a few very frequent) select the input rows
        dict(name="embed fwd 500k x64 types", op="embed_fwd", n=500_000, v=119, d=64, ids="i32", spread="zipf", table="f32", rows="f32", scale=1.0),
        # a million nodes or tokens out of a large vocabulary, scaled by sqrt(width) on the way, fp32 table and bf16 rows
        dict(name="embed fwd 1M x256", op="embed_fwd", n=1_000_000, v=50_257, d=256, ids="i64", spread="zipf", table="f32", rows="bf16", scale=16.0),
        # the gradient for the smallest batch
        dict(name="embed bwd 1000x16", op="embed_bwd", n=1000, v=100, d=16, ids="i64", spread="zipf", table="f32", rows="f32", scale=1.0),
        # the gradient of the type table: few rows, each the sum over up to 100 000 nodes
        dict(name="embed bwd 500k x64 types", op="embed_bwd", n=500_000, v=119, d=64, ids="i32", spread="zipf", table="f32", rows="f32", scale=1.0),
        # the gradient of a large vocabulary's table: many short sums, a few very long ones, rows nobody named
        dict(name="embed bwd 1M x256", op="embed_bwd", n=1_000_000, v=50_257, d=256, ids="i64", spread="zipf", table="f32", rows="bf16", scale=16.0),
        # one token's row, as in inference one node or token at a time
        dict(name="norm fwd 1x4096", op="norm_fwd", n=1, d=4096, dtype="bf16", weights="bf16", pad=0),
        # one layer's output on a graph of 233 000 nodes
        dict(name="norm fwd 233k x128", op="norm_fwd", n=233_000, d=128, dtype="f32", weights="f32", pad=0),
        # an odd width, rows that are part of a wider matrix
        dict(name="norm bwd 5001x1433", op="norm_bwd", n=5001, d=1433, dtype="f32", weights="f32", pad=7),
        # the largest layer: a million nodes, 256 features in bf16, fp32 weights
        dict(name="norm bwd 1M x256", op="norm_bwd", n=1_000_000, d=256, dtype="bf16", weights="f32", pad=0),
        # the parameters of a small network: 12 small tensors, clipped
        dict(name="clip 12 tensors 50k", op="clip", tensors=12, elements=50_000, dtype="f32", ratio=0.25),
        # a large table and 39 further tensors in both types, clipped
        dict(name="clip 40 tensors 200M", op="clip", tensors=40, elements=200_000_000, dtype="mixed", ratio=0.5),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: most are multiples of 8, as feature widths are; the rest is any number."""
    d = _log(rng, lo, hi)
    return max(8, d // 8 * 8) if rng.random() < 0.65 else d


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "clip"])
    if op.startswith("embed"):
        d = _width(rng, 4, 4096)
        n = _log(rng, 1, max(1, min(2_000_000, _MOST // (2 * d))))
        v = _log(rng, 2, max(2, min(1_000_000, _MOST // (4 * d))))
        return dict(op=op, n=n, v=v, d=d, ids=rng.choice(["i32", "i64"]), spread=rng.choice(["zipf", "uniform", "padded"]),
                    table=rng.choice(["f32", "bf16"]), rows=rng.choice(["f32", "bf16"]), scale=rng.choice([1.0, 16.0, 0.125]))
    if op.startswith("norm"):
        d = _width(rng, 4, 16384)
        n = _log(rng, 1, _MOST // (2 * d))
        return dict(op=op, n=n, d=d, dtype=rng.choice(["f32", "bf16"]), weights=rng.choice(["f32", "bf16"]),
                    pad=rng.choice([0, 0, 0, 8, 5]))
    return dict(op=op, tensors=rng.randint(1, 60), elements=_log(rng, 1000, 200_000_000), dtype=rng.choice(["f32", "bf16", "mixed"]),
                ratio=rng.choice([0.0625, 0.5, 2.0]))


# --------------------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _ids(gen, case):
    n, v = case["n"], case["v"]
    if case["spread"] == "perm":
        ids = torch.randperm(v, generator=gen, device="cuda")[:n]
    elif case["spread"] == "uniform":
        ids = torch.randint(0, v, (n,), generator=gen, device="cuda")
    else:                       # frequency falls with the rank, as of words and of atom types; ranks are shuffled over the table
        cdf = _frequencies(v).cumsum(0)
        u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
        rank = torch.searchsorted(cdf, u).clamp_(max=v - 1)
        ids = torch.randperm(v, generator=gen, device="cuda")[rank]
        if case["spread"] == "padded":   # about every eighth place of the batch holds no token
            ids = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.125, -1, ids)
    return ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _frequencies(v):
    p = 1.0 / torch.arange(1, v + 1, device="cuda" if torch.cuda.is_available() else "cpu", dtype=torch.float64)
    return p / p.sum()


def _lengths(case):
    """Lengths of the tensors: one large, the others fall off; odd numbers among them, a short one of 7."""
    t, total = case["tensors"], case["elements"]
    share = [0.5 ** min(k, 9) for k in range(t)]
    out = [max(1, int(total * s / sum(share)) - k % 2) for k, s in enumerate(share)]
    if t > 2:
        out[-1] = 7
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op == "embed_fwd":
        s["ids"] = _ids(gen, case)
        s["table"] = _normal(gen, case["v"], case["d"]).to(_DT[case["table"]])
    elif op == "embed_bwd":
        s["ids"] = _ids(gen, case)
        s["grad"] = _normal(gen, case["n"], case["d"]).to(_DT[case["rows"]])
    elif op.startswith("norm"):
        n, d = case["n"], case["d"]
        offset = _normal(gen, d)
        s["x"] = _normal(gen, n, d + case["pad"]).mul_(1.5).add_(torch.cat([offset, offset.new_zeros(case["pad"])])).to(_DT[case["dtype"]])[:, :d]
        s["w"] = (1 + 0.1 * _normal(gen, d)).to(_DT[case["weights"]])
        s["b"] = (0.1 * _normal(gen, d)).to(_DT[case["weights"]])
        if op == "norm_bwd":    # what the forward pass left
            s["grad"] = _normal(gen, n, d).to(_DT[case["dtype"]])
            s["mean"], s["rstd"] = _stats(s["x"].float())
    else:
        lens = _lengths(case)
        kinds = ["bf16" if case["dtype"] == "bf16" or (case["dtype"] == "mixed" and k % 2) else "f32" for k in range(len(lens))]
        s["grads"] = [(0.01 * _normal(gen, m)).to(_DT[k]) for m, k in zip(lens, kinds)]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]
        s["max_norm"] = case["ratio"] * 0.01 * math.sqrt(sum(lens))
    return s


def _stats(x):
    mean = x.mean(1)
    return mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + _EPS)


# --------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _run_own(s, case):
    import paper_1906_03707_b200 as hb
    op = case["op"]
    if op == "embed_fwd":
        return hb.embedding_fwd(s["ids"], s["table"], scale=case["scale"], dtype=_DT[case["rows"]])
    if op == "embed_bwd":
        return hb.embedding_bwd(s["ids"], s["grad"], case["v"], scale=case["scale"], dtype=_DT[case["table"]])
    if op == "norm_fwd":
        return hb.layer_norm_fwd(s["x"], s["w"], s["b"], eps=_EPS)
    if op == "norm_bwd":
        return hb.layer_norm_bwd(s["grad"], s["x"], s["mean"], s["rstd"], s["w"])
    out, norm = hb.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
    return out, norm


def _run_plain(s, case):
    op = case["op"]
    if op == "embed_fwd":
        ids, v = s["ids"].long(), case["v"]
        rows = s["table"][ids.clamp(0, v - 1)].float() * case["scale"]
        return rows.masked_fill_(((ids < 0) | (ids >= v))[:, None], 0.0).to(_DT[case["rows"]])
    if op == "embed_bwd":
        ids, v = s["ids"].long(), case["v"]
        ids = torch.where((ids < 0) | (ids >= v), v, ids)      # one row more than the table has takes what has no row
        total = torch.zeros(v + 1, case["d"], device=ids.device).index_add_(0, ids, s["grad"].float())
        return (total[:v] * case["scale"]).to(_DT[case["table"]])
    if op == "norm_fwd":
        x = s["x"].float()
        mean, rstd = _stats(x)
        y = (x - mean[:, None]) * rstd[:, None] * s["w"].float() + s["b"].float()
        return y.to(s["x"].dtype), mean, rstd
    if op == "norm_bwd":
        g = s["grad"].float()
        hat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        grad_b, grad_w = g.sum(0), (g * hat).sum(0)
        q = g * s["w"].float()
        gx = (q - q.mean(1, keepdim=True) - hat * (q * hat).mean(1, keepdim=True)) * s["rstd"][:, None]
        return gx.to(s["x"].dtype), grad_w.to(s["w"].dtype), grad_b.to(s["w"].dtype)
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return [(g.float() * factor).to(g.dtype) for g in s["grads"]], norm


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op.startswith("embed"):
        n, v, d = case["n"], case["v"], case["d"]
        ids = n * (4 if case["ids"] == "i32" else 8)
        named = n * (0.875 if case["spread"] == "padded" else 1.0)
        if op == "embed_bwd":
            return {"bytes": ids + named * d * _SIZE[case["rows"]] + v * d * _SIZE[case["table"]], "flops": named * d}
        if case["spread"] == "perm":
            distinct = min(n, v)
        elif case["spread"] == "uniform":
            distinct = -v * math.expm1(n * math.log1p(-1.0 / v))
        else:
            distinct = -float(torch.expm1(named * torch.log1p(-_frequencies(v).clamp(max=1 - 1e-12))).sum())
        return {"bytes": ids + distinct * d * _SIZE[case["table"]] + n * d * _SIZE[case["rows"]], "flops": n * d}
    if op.startswith("norm"):
        n, d, e, we = case["n"], case["d"], _SIZE[case["dtype"]], _SIZE[case["weights"]]
        if op == "norm_fwd":
            return {"bytes": 2 * n * d * e + 8 * n + 2 * d * we, "flops": 8 * n * d}
        return {"bytes": 3 * n * d * e + 8 * n + 3 * d * we, "flops": 14 * n * d}
    lens = _lengths(case)
    size = [2 if case["dtype"] == "bf16" or (case["dtype"] == "mixed" and k % 2) else 4 for k in range(len(lens))]
    return {"bytes": 2 * sum(m * e for m, e in zip(lens, size)), "flops": 3 * sum(lens)}


# --------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op.startswith("embed"):
        n, v, d = case["n"], case["v"], case["d"]
        ids = s["ids"].long()
        here = (ids >= 0) & (ids < v)
        if op == "embed_fwd":
            out = torch.zeros(n, d, device="cuda", dtype=torch.float64)
            out[here] = s["table"].double().index_select(0, ids[here]) * case["scale"]
            return out
        # sums over the sorted ids as differences of a running sum
        key, order = torch.sort(ids[here])
        running = torch.zeros(key.numel() + 1, d, device="cuda", dtype=torch.float64)
        torch.cumsum(s["grad"][here][order].double() * case["scale"], 0, out=running[1:])
        edge = torch.searchsorted(key, torch.arange(v + 1, device="cuda"))
        return running[edge[1:]] - running[edge[:-1]]
    if op == "norm_fwd":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1.0 / torch.sqrt(var + _EPS)
        return torch.addcmul(s["b"].double(), (x - mean[:, None]) * rstd[:, None], s["w"].double()), mean, rstd
    if op == "norm_bwd":
        d = case["d"]
        rstd = s["rstd"].double()[:, None]
        hat = s["x"].double().sub_(s["mean"].double()[:, None]).mul_(rstd)
        g = s["grad"].double()
        grad_w, grad_b = torch.einsum("rd,rd->d", g, hat), torch.einsum("rd->d", g)
        g *= s["w"].double()
        along, across = torch.einsum("rd,rd->r", g, hat) / d, torch.einsum("rd->r", g) / d
        return g.sub_(across[:, None]).addcmul_(hat, along[:, None], value=-1).mul_(rstd), grad_w, grad_b
    norm = math.sqrt(math.fsum(float(torch.dot(g.double(), g.double())) for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / (norm + 1e-6))
    return [g.double() * factor for g in s["grads"]], torch.tensor(norm, dtype=torch.float64)
