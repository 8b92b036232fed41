"""The weights of an update element by element, with rates at which update and decay are far above the rounding of the weights: every way a result
leaves its tile (whole and partial columns, both orientations, cut tiles, the block's patch, whole matrices in a block)."""
import pytest
import torch

import gpu_util as G
import muon_util as U
from paper_2411_10003_amd import binding

pytestmark = pytest.mark.gpu
RATES = dict(lr=0.5, wd=0.5, scale=2.0)
CASES = [(64, 64, 1, (False,)), (64, 256, 3, (False, True, False)), (100, 70, 3, (False, True)), (65, 129, 2, (True, False)), (63, 1000, 2, (False, True)), (8, 8, 3, (True,)),
         (3, 5, 3, (False, True)), (1, 1, 2, (False,)), (1, 300, 2, (False, True)), (128, 128, 2, (True,)), (128, 257, 2, (True, False)), (192, 320, 3, (False, True, False)),
         (320, 576, 3, (False, True)), (333, 517, 1, (False,)), (517, 333, 3, (False, True, False)), (768, 2304, 1, (True,)), (1537, 640, 3, (False, True, False)),
         (1024, 1088, 20, (False,)), (1100, 2112, 9, (False, True)), (576, 4032, 3, (False, True)), (640, 704, 40, (False,)), (641, 703, 20, (False, True)),
         (1100, 1500, 10, (True,)), (320, 3840, 2, (True,))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,count,transposed", CASES)
def test_weights(rows, cols, count, transposed, dtype):
    g = torch.Generator(device=G.DEV).manual_seed(rows + 3 * cols)
    shapes = [(count, cols, rows) if t else (count, rows, cols) for t in transposed]
    grads, momenta = [U.gradient(g, *s, G.DEV) for s in shapes], [3.0 * U.gradient(g, *s, G.DEV) for s in shapes]
    factors = [U.orthogonalised(U.direction(a, b)[1]) for a, b in zip(grads, momenta)]
    weights = [U.weights_like(x, g, dtype, lr=RATES["lr"], scale=RATES["scale"]) for x in factors]
    W0 = [w.clone() for w in weights]
    copies = [torch.zeros_like(w, dtype=torch.bfloat16) for w in weights] if dtype == "f32" else None
    mu = binding.Muon(count=count, rows=rows, cols=cols, dtype=dtype, transposed=transposed, device=G.DEV)
    mu.step(grads, momenta, weights, lr=RATES["lr"], weight_decay=RATES["wd"], scale=RATES["scale"], copies=copies)
    for x, w0, w1 in zip(factors, W0, weights):
        U.check(dtype, x, w0, w1, **RATES)
    if copies:
        assert all(torch.equal(c, w.to(torch.bfloat16)) for c, w in zip(copies, weights))


@pytest.mark.parametrize("dtype,transposed", [("f32", (False,)), ("f32", (True,)), ("bf16", (True,))])
def test_large_experts(dtype, transposed):
    """The largest configuration's sides, fp32 master weights with their bf16 copies among them.  Measured as in muon_util, at 2048 x 8192 and 4096 x 14336 an
    element of the factor is off by 5.0e-2 root mean squares at most in 11 bits: twice that."""
    rows, cols = 4096, 14336
    g = torch.Generator(device=G.DEV).manual_seed(5)
    shape = (1, cols, rows) if transposed[0] else (1, rows, cols)
    grads, momenta = [U.gradient(g, *shape, G.DEV)], [3.0 * U.gradient(g, *shape, G.DEV)]
    x = U.orthogonalised(U.direction(grads[0], momenta[0])[1])
    w0 = U.weights_like(x, g, dtype, lr=RATES["lr"], scale=RATES["scale"])
    weights, copies = [w0.clone()], [torch.zeros_like(w0, dtype=torch.bfloat16)] if dtype == "f32" else None
    mu = binding.Muon(count=1, rows=rows, cols=cols, dtype=dtype, transposed=transposed, device=G.DEV)
    mu.step(grads, momenta, weights, lr=RATES["lr"], weight_decay=RATES["wd"], scale=RATES["scale"], copies=copies)
    norm, element, line = U.FACTOR[dtype]
    U.check(dtype, x, w0, weights[0], **RATES, factor=(norm, 0.1 if dtype == "bf16" else element, line))
    if copies:
        assert torch.equal(copies[0], weights[0].to(torch.bfloat16))
