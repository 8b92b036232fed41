"""Attention of packed sequences by its formulas in 64 bits, with the errors that the kernels may have, element by element.

eps(t) / 2 is the relative rounding u(t) of a type, e = 2^-24.  A score is an fp32 sum of d products: (d + 2) e scale sum |q k|, 3 e of itself for its scaling,
and as an exponent its error is the exponential's relative one, with 4 e for the exponential itself.  Per query E is the largest of these.  Exponentials
are rounded to the type ahead of their products (u, nothing in fp32); a sum of m terms is off by (m + 2) e of the sum of magnitudes.  To first order:
  O    u |O| + (2 E + u + 2 (m + 2) e) sum p |v|
  lse  E + (m + 2) e + 4 e |lse| + 4 e
  ds   p ((E + 6 e |lse|) (|dp| + |D|) + (d + 4) e (sum |dO v| + sum |dO O|)),  rounded: + u |ds|;  p likewise
  dQ   u |dQ| + scale (sum err(ds) |k| + (m + 4) e sum |ds k|),  dK and dV the same over the queries of all heads
Second-order terms: 1 % on top."""
import math

import torch

import gpu_util as G

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E24 = 2.0 ** -24


def rounding(t):
    return torch.finfo(t).eps / 2


def offsets(lens, gap=0):
    at, out = 0, []
    for n in lens:
        out.append(at)
        at += n
    return torch.tensor(out + [at], dtype=torch.int32, device=G.DEV)


def tensors(rows, counts, d, t, layout, seed, scale=1.0):
    """Random tensors [rows, n, d]: apart, beside each other in one, or with a head's rows together."""
    g = torch.Generator(device=G.DEV).manual_seed(seed)
    if layout == "fused":
        out = list(torch.empty(rows, sum(counts) + 1, d, dtype=t, device=G.DEV)[:, 1:].split(counts, 1))
    elif layout == "heads":
        out = [torch.empty(n, rows, d, dtype=t, device=G.DEV).transpose(0, 1) for n in counts]
    else:
        out = [torch.empty(rows, n, d, dtype=t, device=G.DEV) for n in counts]
    for x in out:
        x.copy_(scale * torch.randn(rows, x.shape[1], d, generator=g, device=G.DEV) + 0.2 * scale * torch.randn(d, generator=g, device=G.DEV))
    return out


def _head(Q, K, V, h, group, q, k, scale, causal):
    a, b, v = Q[q, h].double(), K[k, h // group].double(), V[k, h // group].double()
    n, m = a.shape[0], b.shape[0]
    s = scale * (a @ b.T)
    seen = torch.ones(n, m, dtype=torch.bool, device=G.DEV)
    if causal:
        seen = seen.tril(m - n)
    lse = torch.full((n,), -math.inf, dtype=torch.float64, device=G.DEV)
    if m:
        lse = torch.logsumexp(s.masked_fill(~seen, -math.inf), 1)
    p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[:, None]), 0.0)
    e = (a.shape[1] + 2) * E24 * scale * (a.abs() @ b.abs().T) + 3 * E24 * s.abs() + 4 * E24
    E = torch.where(seen, e, 0.0).amax(1) if m else torch.zeros_like(lse)
    return a, b, v, p, lse, E


def forward(Q, K, V, parts, scale, causal):
    """parts: (first query, queries, first key, keys).  O and lse of the sequences' rows (NaN elsewhere), and their bounds."""
    t, group = Q.dtype, Q.shape[1] // K.shape[1]
    O, bO = (torch.full(Q.shape, math.nan, dtype=torch.float64, device=G.DEV) for _ in range(2))
    lse, bl = (torch.full((Q.shape[1], Q.shape[0]), math.nan, dtype=torch.float64, device=G.DEV) for _ in range(2))
    for q0, n, k0, m in parts:
        for h in range(Q.shape[1]):
            q, k = slice(q0, q0 + n), slice(k0, k0 + m)
            _, _, v, p, l, E = _head(Q, K, V, h, group, q, k, scale, causal)
            O[q, h], lse[h, q] = p @ v, l
            rel = 2 * E + (rounding(t) if t != torch.float32 else 0.0) + 2 * (m + 2) * E24
            bO[q, h] = 1.01 * (rounding(t) * O[q, h].abs() + rel[:, None] * (p @ v.abs())) + 1e-30
            bl[h, q] = 1.01 * (E + (m + 2) * E24 + 4 * E24 * torch.where(torch.isinf(l), 0.0, l).abs() + 4 * E24)
    return O, bO, lse, bl


def backward(dO, Q, K, V, O, lse, parts, scale, causal):
    """The gradients for an O and lse in hand, and their bounds: [(dQ, bound), (dK, bound), (dV, bound)]."""
    t, group, d = Q.dtype, Q.shape[1] // K.shape[1], Q.shape[2]
    u = rounding(t) if t != torch.float32 else 0.0
    out = [[torch.full(x.shape, math.nan, dtype=torch.float64, device=G.DEV) for _ in range(2)] for x in (Q, K, V)]
    for q0, n, k0, m in parts:
        q, k = slice(q0, q0 + n), slice(k0, k0 + m)
        for x in out[1] + out[2]:
            x[k] = 0.0
        for h in range(Q.shape[1]):
            kv = h // group
            a, b, v, p, _, E = _head(Q, K, V, h, group, q, k, scale, causal)
            do, o, l = dO[q, h].double(), O[q, h].double(), lse[h, q].double()
            l = torch.where(torch.isinf(l), 0.0, l)
            p = torch.where(p > 0.0, torch.exp(scale * (a @ b.T) - l[:, None]), 0.0)
            dp, D = do @ v.T, (do * o).sum(1, keepdim=True)
            ds = p * (dp - D)
            ep = (E + 6 * E24 * l.abs())[:, None]
            eds = p * (ep * (dp.abs() + D.abs()) + (d + 4) * E24 * (do.abs() @ v.abs().T + (do * o).abs().sum(1, keepdim=True))) + u * ds.abs()
            out[0][0][q, h] = scale * ds @ b
            out[0][1][q, h] = scale * (eds + (m + 4) * E24 * ds.abs()) @ b.abs()
            out[1][0][k, kv] += scale * ds.T @ a
            out[1][1][k, kv] += scale * (eds + (n * group + 4) * E24 * ds.abs()).T @ a.abs()
            out[2][0][k, kv] += p.T @ do
            out[2][1][k, kv] += (p * (ep + u + (n * group + 4) * E24)).T @ do.abs()
    for x, bound in out:
        bound.copy_(1.01 * (bound + rounding(t) * x.abs()) + 1e-30)
    return out


def near(got, want, bound):
    """Whether every element that has a value (rows of a sequence) is as near as it may be; infinities equal."""
    has = ~torch.isnan(want)
    same = (got.double() == want) & has
    return bool((same | ~has | ((got.double() - want).abs() <= bound)).all())
