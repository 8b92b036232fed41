"""The operators of a block's training step that surround the MoE layer, as cases that can be timed and checked.

A case is a dict of plain values; `op` says which operator one pass runs:

  norm_fwd   the layer norm ahead of the gate: rows x d activations of `dtype`; `residual`: the sum with the residual stream is
             formed and kept in the same pass; `bias`: the norm has one; `stats`: mean and rstd are kept for the backward pass
  norm_bwd   its gradient: `residual`: the residual stream's own gradient is added to the input's
  muon       one update of the experts' parameters: `tensors` weight tensors of `count` matrices, the first (and third) rows x cols, the
             second cols x rows as the FFN keeps them; `dtype` that of the weights; `copy`: a bf16 copy of fp32 weights is kept beside them
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
# what Muon is run with: coefficients of the quintic, momentum, its damping of the norm
COEF, STEPS, MOMENTUM, NORM_EPS = (3.4445, -4.7750, 2.0315), 5, 0.95, 1e-7
LR, DECAY = 0.01, 0.1


def listed():
    return [
        # one token of a decoding step: the norm without anything kept for a backward pass; launch latency and nothing else
        _norm("norm_fwd", "norm_token", rows=1, d=2048, dtype="bf16", stats=False),
        # the tiny fp32 configuration
        _norm("norm_fwd", "norm_tiny_f32", rows=512, d=64, dtype="f32", residual=False),
        # a ragged prompt of a model whose width is odd: no row but the first begins at a multiple of 16 bytes
        _norm("norm_fwd", "norm_ragged", rows=7999, d=1021, dtype="bf16"),
        # a training step's forward pass at the largest configuration: residual sum and norm
        _norm("norm_fwd", "norm_wide", rows=32768, d=4096, dtype="bf16"),
        # the same four on the way back
        _norm("norm_bwd", "norm_bwd_tiny_f32", rows=512, d=64, dtype="f32", residual=False),
        _norm("norm_bwd", "norm_bwd_ragged_f32", rows=5003, d=1021, dtype="f32", bias=False),
        _norm("norm_bwd", "norm_bwd_mid", rows=16384, d=2048, dtype="bf16"),
        _norm("norm_bwd", "norm_bwd_wide", rows=32768, d=4096, dtype="bf16"),
        # the experts that one GPU owns, both matrices of each, of the tiny fp32 configuration: launches and nothing else
        _muon("muon_tiny_f32", count=2, rows=64, cols=256, tensors=2, dtype="f32"),
        # fp32 weights with a bf16 copy for the layer, sizes that fit no tile, taller than wide
        _muon("muon_odd_f32", count=3, rows=1333, cols=500, tensors=2, dtype="f32", copy=True),
        # the owned experts of the mid-size GELU configuration
        _muon("muon_gelu", count=2, rows=1024, cols=4096, tensors=2, dtype="bf16"),
        # the owned experts of the largest configuration, three matrices each
        _muon("muon_swiglu", count=2, rows=4096, cols=14336, tensors=3, dtype="bf16"),
    ]


def _norm(op, name=None, *, rows, d, dtype, residual=True, bias=True, stats=True):
    c = dict(op=op, rows=rows, d=d, dtype=dtype, residual=residual, bias=bias)
    if op == "norm_fwd":
        c["stats"] = stats
    if name is not None:
        c["name"] = name
    return c


def _muon(name=None, *, count, rows, cols, tensors, dtype, copy=False, nesterov=True):
    c = dict(op="muon", count=count, rows=rows, cols=cols, tensors=tensors, dtype=dtype, copy=copy, nesterov=nesterov)
    if name is not None:
        c["name"] = name
    return c


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case: sizes over the whole range of its operator."""
    op = rng.choice(["norm_fwd", "norm_bwd", "muon"])
    if op != "muon":
        d = int(_log(rng, 16, 8193))
        d = d if rng.random() < 0.4 else max(64, (d + 32) // 64 * 64)
        rows = int(min(_log(rng, 1, 65536), 32768 * 4096 // d))
        c = dict(rows=max(1, rows), d=d, dtype=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.6, bias=rng.random() < 0.7)
        return _norm(op, **c, stats=rng.random() < 0.7) if op == "norm_fwd" else _norm(op, **c)
    rows = int(_log(rng, 16, 4097))
    cols = int(min(_log(rng, max(16, rows / 4), rows * 5), 14336))
    if rng.random() < 0.6:
        rows, cols = max(64, (rows + 32) // 64 * 64), max(64, (cols + 32) // 64 * 64)
    tensors, dtype = rng.choice([1, 2, 3]), rng.choice(["bf16", "bf16", "f32"])
    short, long = min(rows, cols), max(rows, cols)
    most = int(2.5e13 / ((20 * long + 10 * short) * short * short * tensors))       # products of the plain form, below the largest listed
    count = max(1, min(int(_log(rng, 1, 17)), most))
    return _muon(count=count, rows=rows, cols=cols, tensors=tensors, dtype=dtype, copy=dtype == "f32" and rng.random() < 0.5, nesterov=rng.random() < 0.7)


def _shapes(case):
    a, b = (case["count"], case["rows"], case["cols"]), (case["count"], case["cols"], case["rows"])
    return [a, b, a][:case["tensors"]]


def _gradient(g, shape):
    """A weight gradient: products of activations and their gradients, whose singular values fall off, with noise below them."""
    n, r, c = shape
    k = max(1, min(r, c) // 4)
    left, right = torch.randn(n, r, k, generator=g, device=DEV), torch.randn(n, k, c, generator=g, device=DEV)
    left *= 1.0 / torch.sqrt(torch.arange(1, k + 1, device=DEV))
    return (left @ right) * 1e-3 + 2e-4 * torch.randn(n, r, c, generator=g, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    s = dict(case)
    if case["op"] == "muon":
        shapes = _shapes(case)
        s["grads"] = [_gradient(g, t) for t in shapes]
        s["momenta"] = [5.0 * _gradient(g, t) for t in shapes]
        s["weights"] = [(randn(*t) / math.sqrt(t[1])).to(TYPES[case["dtype"]]) for t in shapes]
        s["copies"] = [w.to(torch.bfloat16) for w in s["weights"]] if case["copy"] else None
        s["version"] = torch.randint(0, 100, (case["count"],), generator=g, device=DEV, dtype=torch.int32)
        return s
    rows, d, t = case["rows"], case["d"], TYPES[case["dtype"]]
    # a residual stream: channels of different size, a few of them much larger than the rest, none centred
    size, middle = torch.exp(0.4 * randn(d)), 0.3 * randn(d)
    size[torch.randint(0, d, (max(1, d // 500),), generator=g, device=DEV)] *= 20.0
    stream = lambda: randn(rows, d).mul_(size).add_(middle)  # noqa: E731
    s["gamma"] = 1.0 + 0.1 * randn(d)
    s["beta"] = 0.1 * randn(d) if case["bias"] else None
    new = lambda: torch.empty(rows, d, dtype=t, device=DEV)  # noqa: E731
    if case["op"] == "norm_fwd":
        s["X"] = stream().mul_(0.3).to(t) if case["residual"] else stream().to(t)
        s["R"] = stream().to(t) if case["residual"] else None
        s["S"], s["Y"] = (new() if case["residual"] else None), new()
        s["mean"], s["rstd"] = (torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)) if case["stats"] else (None, None)
    else:
        s["S"], s["dY"] = stream().to(t), randn(rows, d).mul_(0.02).to(t)
        s["dS"] = randn(rows, d).mul_(0.02).to(t) if case["residual"] else None
        wide = s["S"].double()
        s["mean"] = wide.mean(1).float()
        s["rstd"] = (wide.var(1, correction=0) + EPS).rsqrt().float()
        s["dX"], s["dgamma"], s["dbeta"] = new(), torch.empty(d, device=DEV), torch.empty(d, device=DEV) if case["bias"] else None
    return s


_kept = {}      # what a program makes once and keeps: the norm of a width, the update of a set of experts


def _own_norm(s):
    from paper_2411_10003_amd import binding
    key = ("norm", s["d"], s["dtype"])
    if key not in _kept:
        _kept[key] = binding.Norm(d=s["d"], dtype=s["dtype"], eps=EPS, device=DEV)
    return _kept[key]


def _own_muon(s):
    from paper_2411_10003_amd import binding
    key = ("muon", s["count"], s["rows"], s["cols"], s["tensors"], s["dtype"], s["nesterov"])
    if key not in _kept:
        _kept[key] = binding.Muon(count=s["count"], rows=s["rows"], cols=s["cols"], dtype=s["dtype"], transposed=[False, True, False][:s["tensors"]],
                                  momentum=MOMENTUM, nesterov=s["nesterov"], steps=STEPS, coefficients=COEF, eps=NORM_EPS, device=DEV)
    return _kept[key]


def _scale(s):
    return 0.2 * math.sqrt(max(s["rows"], s["cols"]))      # updates of the size that an Adam step has


def run(s):
    if s["op"] == "norm_fwd":
        if own:
            _own_norm(s).fwd(s["X"], s["gamma"], s["beta"], s["Y"], residual=s["R"], total=s["S"], mean=s["mean"], rstd=s["rstd"])
            return [s["Y"], s["S"], s["mean"], s["rstd"]]
        return _plain_norm_fwd(s)
    if s["op"] == "norm_bwd":
        if own:
            _own_norm(s).bwd(s["dY"], s["S"], s["gamma"], s["mean"], s["rstd"], s["dX"], s["dgamma"], s["dbeta"], residual_grad=s["dS"])
            return [s["dX"], s["dgamma"], s["dbeta"]]
        return _plain_norm_bwd(s)
    if own:
        _own_muon(s).step(s["grads"], s["momenta"], s["weights"], lr=LR, weight_decay=DECAY, scale=_scale(s), copies=s["copies"], version=s["version"])
        return [s["weights"], s["momenta"], s["copies"], s["version"]]
    return _plain_muon(s)


def _plain_norm_fwd(s):
    x = s["X"].float()
    total = None
    if s["residual"]:
        total = (x + s["R"].float()).to(s["X"].dtype)
        x = total.float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    y = x * rstd * s["gamma"]
    if s["bias"]:
        y = y + s["beta"]
    return [y.to(s["X"].dtype), total, mean[:, 0] if s["stats"] else None, rstd[:, 0] if s["stats"] else None]


def _plain_norm_bwd(s):
    dy, rstd = s["dY"].float(), s["rstd"][:, None]
    xh = (s["S"].float() - s["mean"][:, None]) * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if s["residual"]:
        dx = s["dS"].float() + dx
    return [dx.to(s["S"].dtype), (dy * xh).sum(0), dy.sum(0) if s["bias"] else None]


def _plain_muon(s):
    a, b, c = COEF
    for grad, momentum, weight, i in zip(s["grads"], s["momenta"], s["weights"], range(3)):
        momentum.mul_(MOMENTUM).add_(grad)
        u = grad + MOMENTUM * momentum if s["nesterov"] else momentum
        x = u / (u.double().square().sum((1, 2), keepdim=True).sqrt().float() + NORM_EPS)
        if x.shape[1] > x.shape[2]:
            x = x.transpose(1, 2).contiguous()
        for _ in range(STEPS):
            A = torch.matmul(x, x.transpose(1, 2).contiguous())
            x = a * x + torch.matmul(b * A + c * torch.matmul(A, A), x)
        if weight.shape[1] > weight.shape[2]:
            x = x.transpose(1, 2)
        new = weight.float() * (1.0 - LR * DECAY) - (LR * _scale(s)) * x
        weight.copy_(new)
        if s["copies"] is not None:
            s["copies"][i].copy_(weight)
    s["version"].add_(1)
    return [s["weights"], s["momenta"], s["copies"], s["version"]]


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "muon":
        m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        each = case["count"] * case["tensors"]
        # gradient, momentum in and out, weights in and out.  Every iterate is a polynomial in G = X X^T times the first X: one product for G, the
        # polynomial in products of symmetric matrices (half of each is the other half), one product with X.
        return {"bytes": each * m * n * (12 + 2 * size + (2 if case["copy"] else 0)) + 8 * case["count"],
                "flops": each * (m * m * n + 2 * m * m * n + (4 * STEPS - 3) * m * m * m)}
    rows, d = case["rows"], case["d"]
    vectors = 4 * d * (2 if case["bias"] else 1)
    if case["op"] == "norm_fwd":
        return {"bytes": rows * d * size * (4 if case["residual"] else 2) + vectors + (8 * rows if case["stats"] else 0), "flops": 8 * rows * d}
    return {"bytes": rows * d * size * (4 if case["residual"] else 3) + vectors + 4 * d + 8 * rows, "flops": 14 * rows * d}


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "muon":
        a, b, c = COEF
        weights, momenta, copies = [], [], []
        for grad, momentum, weight in zip(s["grads"], s["momenta"], s["weights"]):
            m = MOMENTUM * momentum.double() + grad.double()
            u = grad.double() + MOMENTUM * m if case["nesterov"] else m
            x = torch.stack([v / (torch.linalg.vector_norm(v) + NORM_EPS) for v in u])
            tall = x.shape[1] > x.shape[2]
            for _ in range(STEPS):          # x p(x^T x) or p(x x^T) x, whichever square is the smaller
                q = torch.matmul(x.mT.contiguous(), x) if tall else torch.matmul(x, x.mT.contiguous())
                p = b * q + c * torch.matmul(q, q)
                x = a * x + (torch.matmul(x, p) if tall else torch.matmul(p, x))
            weights.append(weight.double() - LR * (DECAY * weight.double() + _scale(s) * x))
            momenta.append(m)
            copies.append(weights[-1])
        return [weights, momenta, copies if case["copy"] else None, s["version"] + 1]
    t = TYPES[case["dtype"]]
    gamma = s["gamma"].double()
    beta = s["beta"].double() if case["bias"] else torch.zeros_like(gamma)
    if case["op"] == "norm_fwd":
        x = s["X"].double()
        if case["residual"]:
            x = x + s["R"].double()
        total = x
        x = x.to(t).double()                # the sum is kept, and normalised, in the type of the activations
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(beta, (x - mean[:, None]) * rstd[:, None], gamma)
        return [y, total if case["residual"] else None, mean if case["stats"] else None, rstd if case["stats"] else None]
    # the gradient of the forward definition, by differentiating it, a part of the rows at a time
    gamma, beta = gamma.requires_grad_(), beta.requires_grad_()
    dx = []
    for r in range(0, case["rows"], 4096):
        x = s["S"][r:r + 4096].double().requires_grad_()
        var, mean = torch.var_mean(x, 1, keepdim=True, correction=0)
        ((x - mean) / torch.sqrt(var + EPS) * gamma + beta).backward(s["dY"][r:r + 4096].double())
        dx.append(x.grad + (s["dS"][r:r + 4096].double() if case["residual"] else 0.0))
    return [torch.cat(dx), gamma.grad, beta.grad if case["bias"] else None]
