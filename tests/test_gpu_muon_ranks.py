"""Gradients of low rank, as an expert has that received few rows.  What a rounding leaves outside the gradient's range grows by a = 3.4445 in each of five
steps, 485 times: with every operand rounded as the kernels keep it and sums in 64 bits (CPU, 64 x 256 to 1024 x 4096, ranks 1 to 256) the factor is off
by 0.16 / sqrt(rank) of its norm at most in 11 bits, 3.4e-5 / sqrt(rank) in 22, one element by 3.7 / sqrt(rank) and 8.0e-4 / sqrt(rank) root mean squares.
Twice that is allowed in 11 bits, ten times in 22, which leaves room for the fp32 sums (fp32 throughout: 1.4e-4 at rank one of 256 x 1024)."""
import math

import pytest
import torch

import gpu_util as G
import muon_util as U
from paper_2411_10003_amd import binding

pytestmark = pytest.mark.gpu
RATES = dict(lr=0.5, wd=0.5, scale=2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,rank", [(r, c, k) for r, c in ((64, 256), (256, 1024), (512, 512), (1024, 333), (1024, 4096)) for k in (1, 2, 4, 16, 64)
                                            if k <= min(r, c) // 2])
def test_rank(rows, cols, rank, dtype):
    g = torch.Generator(device=G.DEV).manual_seed(rows + cols + rank)
    randn = lambda *s: torch.randn(*s, generator=g, device=G.DEV)  # noqa: E731
    # products in 64 bits: rounded once, what lies outside the range is 2^-25 of it, a thousandth of what is allowed in 22 bits once it has grown
    grads = [(randn(2, rows, rank).double() @ randn(2, rank, cols).double()).float()]
    x = U.orthogonalised(grads[0])
    w0 = U.weights_like(x, g, dtype, lr=RATES["lr"], scale=RATES["scale"])
    weights, momenta = [w0.clone()], [torch.zeros_like(grads[0])]
    mu = binding.Muon(count=2, rows=rows, cols=cols, dtype=dtype, momentum=0.0, nesterov=False, device=G.DEV)
    mu.step(grads, momenta, weights, lr=RATES["lr"], weight_decay=RATES["wd"], scale=RATES["scale"])
    norm, element = (0.32, 7.4) if dtype == "bf16" else (3.4e-4, 8e-3)
    k = math.sqrt(rank)
    U.check(dtype, x, w0, weights[0], **RATES, factor=(norm / k, element / k, element / k))
