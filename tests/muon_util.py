"""The experts' update in 64 bits, and a check of its results element by element, row by row and column by column.

What is allowed.  W1 = (1 - lr wd) W0 - lr scale X: half a step of the weights' type at |W1|, three fp32 roundings (the factor's last, the product with
the weight, the sum) at the sizes of the terms, and lr scale times the error of X.  That error, in units of the root mean square of X's elements, comes from
keeping the operands in 11 bits (bf16 weights) or 22 (fp32).  Measured on the CPU with every operand rounded as the kernels keep it, sums in 64 bits, gradients of
`gradient`, 17 sizes from 1 x 1 to 768 x 1500, largest: norm 9.6e-3 | 2.5e-6, element 3.4e-2 | 1.0e-5, row or column 2.1e-2 | 4.8e-6.  Twice that
is allowed in 11 bits; in 22, where fp32 sums, which those figures are without, leave four to five times as much, ten times."""
import math

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEF = (3.4445, -4.7750, 2.0315)
#            norm, element, row or column
FACTOR = {"bf16": (2e-2, 7e-2, 4.2e-2), "f32": (2.5e-5, 1e-4, 5e-5)}


def gradient(g, n, r, c, device):
    """A quarter of the rank with a falling spectrum, and noise below it."""
    k = max(1, min(r, c) // 4)
    left, right = torch.randn(n, r, k, generator=g, device=device), torch.randn(n, k, c, generator=g, device=device)
    left *= 1.0 / torch.sqrt(torch.arange(1, k + 1, device=device))
    return left @ right + 0.2 * torch.randn(n, r, c, generator=g, device=device)


def orthogonalised(u, steps=5, eps=1e-7, coef=COEF):
    a, b, c = coef
    u = u.double()
    x = u / (u.flatten(1).norm(dim=1)[:, None, None] + eps)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.mT.contiguous()
    for _ in range(steps):
        A = x @ x.mT.contiguous()
        x = a * x + (b * A + c * A @ A) @ x
    return x.mT.contiguous() if tall else x


def direction(G0, M0, mu=0.95, nesterov=True):
    m = mu * M0.double() + G0.double()
    return m, (G0.double() + mu * m if nesterov else m)


def weights_like(x, g, dtype, *, lr, scale):
    """Weights of the size of the update, so that it and the decay are far above what the type rounds away."""
    rms = lr * scale * float(x.square().mean().sqrt())
    return (torch.randn(x.shape, generator=g, device=x.device) * rms).to(TYPES[dtype])


def check(dtype, x, W0, W1, *, lr, wd, scale, factor=None):
    """x: the factor in 64 bits; W1: the weights after the step."""
    norm, element, line = factor or FACTOR[dtype]
    w = (1.0 - lr * wd) * W0.double() - lr * scale * x
    off = (W1.double() - w).abs()
    rounding = torch.finfo(W1.dtype).eps / 2 * w.abs() + 2.0 ** -24 * (2 * W0.double().abs() + 2 * lr * scale * x.abs())
    one = lr * scale * x.square().mean((1, 2), keepdim=True).sqrt()                    # per matrix
    bad = off - (element * one + rounding)
    assert (bad <= 0).all(), ("element", (bad > 0).nonzero()[0].tolist(), float(bad.max()))
    for dim in (1, 2):
        n = math.sqrt(x.shape[dim])
        assert (off.norm(dim=dim) <= line * one.squeeze(2) * n + rounding.norm(dim=dim)).all(), ("column", "row")[dim - 1]
    n = math.sqrt(x.shape[1] * x.shape[2])
    assert (off.flatten(1).norm(dim=1) <= norm * one.flatten() * n + rounding.flatten(1).norm(dim=1)).all(), "norm"
