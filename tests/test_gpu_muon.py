"""The experts' update against the formulas in 64 bits: sides around the tiles (64, 128, 256) and off them, tall and wide, one and many matrices, both
types, tensors of both orientations in one call.

Tolerances.  W is compared through its update D = (1 - lr wd) W0 - W1, which is lr scale X: X is within TOL[dtype] of its norm (measured against 64 bits
on the CPU with every operand rounded as the kernels keep it: 11 bits 1.5e-3 for dense spectra, 4e-3 for the gradients used here, 2e-2
at a falling spectrum of an eighth of the rank; 22 bits 5e-6 at most.  Twice the largest is allowed), beside the rounding of W1.  Momentum: two fp32 roundings."""
import math

import pytest
import torch

import gpu_util as G
from paper_2411_10003_amd import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"bf16": 4e-2, "f32": 1e-5}
COEF = (3.4445, -4.7750, 2.0315)


def _gradient(g, n, r, c):
    k = max(1, min(r, c) // 4)
    left, right = torch.randn(n, r, k, generator=g, device=G.DEV), torch.randn(n, k, c, generator=g, device=G.DEV)
    left *= 1.0 / torch.sqrt(torch.arange(1, k + 1, device=G.DEV))
    return left @ right + 0.2 * torch.randn(n, r, c, generator=g, device=G.DEV)


def _orthogonalised(u, steps=5, eps=1e-7, coef=COEF):
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


def _want(G0, M0, W0, *, mu=0.95, nesterov=True, steps=5, lr, wd, scale, coef=COEF):
    m = mu * M0.double() + G0.double()
    u = G0.double() + mu * m if nesterov else m
    x = lr * scale * _orthogonalised(u, steps, coef=coef)
    return m, (1.0 - lr * wd) * W0.double() - x, x


def _check(dtype, G0, M0, W0, M1, W1, tol=None, **kw):
    m, w, x = _want(G0, M0, W0, **kw)
    size = 0.95 * M0.double().abs() + G0.double().abs()
    assert ((M1.double() - m).abs() <= 2 * 2.0 ** -24 * size).all()
    half = torch.finfo(TYPES[dtype]).eps / 2
    # per matrix: the factor's error, beside the rounding of the result (fp32: and of the product with the weight)
    off = (W1.double() - w).flatten(1).norm(dim=1)
    allowed = (tol or TOL[dtype]) * x.flatten(1).norm(dim=1) + (half + 2 * 2.0 ** -24) * 1.01 * (w.abs() + W0.double().abs() * 0).flatten(1).norm(dim=1) \
        + (2.0 ** -24) * W0.double().flatten(1).norm(dim=1)
    assert (off <= allowed).all(), (off / allowed).max()


def _case(rows, cols, count, dtype, transposed, seed=0):
    g = torch.Generator(device=G.DEV).manual_seed(7 * rows + cols + seed)
    shapes = [(count, cols, rows) if t else (count, rows, cols) for t in transposed]
    grads, momenta = [_gradient(g, *s) for s in shapes], [3.0 * _gradient(g, *s) for s in shapes]
    weights = [(torch.randn(*s, generator=g, device=G.DEV) / 16).to(TYPES[dtype]) for s in shapes]
    return grads, momenta, weights


SIZES = [(64, 64), (64, 256), (256, 64), (128, 128), (192, 320), (256, 256), (320, 576), (100, 70), (70, 100), (65, 129), (129, 65), (333, 517), (517, 333), (63, 1000),
         (1000, 63), (8, 8), (3, 5), (1, 1), (1, 300), (300, 1), (2, 1031), (1024, 1024), (768, 2304), (1537, 640)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_one_step(rows, cols, dtype):
    for count, transposed, nesterov in ((1, (False,), True), (3, (False, True, False), False)):
        grads, momenta, weights = _case(rows, cols, count, dtype, transposed)
        M0, W0 = [m.clone() for m in momenta], [w.clone() for w in weights]
        mu = binding.Muon(count=count, rows=rows, cols=cols, dtype=dtype, transposed=transposed, nesterov=nesterov, device=G.DEV)
        mu.ws.fill_(0xff)                                  # NaN everywhere: nothing is read that was not written
        lr, wd, scale = 0.02, 0.1, math.sqrt(max(rows, cols)) * 0.2
        version = torch.arange(count, dtype=torch.int32, device=G.DEV) if count > 1 else None
        copies = [torch.zeros_like(w, dtype=torch.bfloat16) for w in weights] if dtype == "f32" else None
        mu.step(grads, momenta, weights, lr=lr, weight_decay=wd, scale=scale, version=version, copies=copies)
        for i in range(len(transposed)):
            _check(dtype, grads[i], M0[i], W0[i], momenta[i], weights[i], nesterov=nesterov, lr=lr, wd=wd, scale=scale)
            if copies:
                assert torch.equal(copies[i], weights[i].to(torch.bfloat16))
        if version is not None:
            assert version.tolist() == list(range(1, count + 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
def test_number_of_steps(steps, dtype):
    rows, cols = 200, 456
    grads, momenta, weights = _case(rows, cols, 2, dtype, (False, True), seed=steps)
    M0, W0 = [m.clone() for m in momenta], [w.clone() for w in weights]
    mu = binding.Muon(count=2, rows=rows, cols=cols, dtype=dtype, transposed=(False, True), steps=steps, device=G.DEV)
    mu.step(grads, momenta, weights, lr=0.1, scale=2.0)
    for i in range(2):
        _check(dtype, grads[i], M0[i], W0[i], momenta[i], weights[i], steps=steps, lr=0.1, wd=0.0, scale=2.0)


@pytest.mark.parametrize("rows,cols,count,transposed,dtype", [
    (1024, 1088, 20, (False,), "bf16"),                    # squares in 256 x 256 tiles, with tiles left over after a full round
    (1100, 2112, 9, (False, True), "bf16"),                # the same, sides off the tiles, both orientations
    (1100, 1500, 10, (True,), "f32"),                      # in two numbers
    (576, 4032, 3, (False, True), "bf16"),                 # few tiles, a long contraction in parts
    (320, 3840, 2, (True,), "f32"),                        # parts that begin in the middle of a segment
    (640, 704, 40, (False,), "bf16"),                      # 128 x 128 tiles, two to a CU
    (640, 704, 20, (False, True), "f32"),
    (2048, 2560, 4, (False,), "bf16"),
    (128, 256, 300, (False,), "bf16"),                     # more small matrices than the chip has places
    (64, 448, 3, (True,), "f32"), (64, 512, 3, (False,), "bf16"), (64, 449, 3, (False,), "f32"), (64, 513, 3, (True,), "bf16"), (65, 256, 2, (False,), "bf16"),
    (128, 257, 2, (True,), "bf16"),                        # what a block takes whole, and one more
    (512, 65536, 1, (False,), "bf16"), (1, 65536, 2, (True,), "f32"), (2, 40000, 1, (False,), "bf16"),
])
def test_layouts(rows, cols, count, transposed, dtype):
    """The ways a product is laid out: every tile size, tiles cut along the contraction, whole matrices in a block; sums of a step that do not depend
    on which part of a tile is done last."""
    grads, momenta, weights = _case(rows, cols, count, dtype, transposed)
    M0, W0 = [m.clone() for m in momenta], [w.clone() for w in weights]
    mu = binding.Muon(count=count, rows=rows, cols=cols, dtype=dtype, transposed=transposed, device=G.DEV)
    mu.ws.fill_(0xff)
    lr, wd, scale = 0.02, 0.1, math.sqrt(max(rows, cols)) * 0.2
    mu.step(grads, momenta, weights, lr=lr, weight_decay=wd, scale=scale)
    for i in range(len(transposed)):
        _check(dtype, grads[i], M0[i], W0[i], momenta[i], weights[i], lr=lr, wd=wd, scale=scale)
    for _ in range(2):
        m, w = [x.clone() for x in M0], [x.clone() for x in W0]
        mu.step(grads, m, w, lr=lr, weight_decay=wd, scale=scale)
        assert all(torch.equal(x, y) for x, y in zip(m + w, momenta + weights))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matrices_do_not_meet(dtype):
    """A batch gives each matrix what it gets alone, in the same layout of tiles or another: within the tolerance of the type, and none is left out."""
    rows, cols, count = 200, 712, 23
    grads, momenta, weights = _case(rows, cols, count, dtype, (False, True))
    M0, W0 = [m.clone() for m in momenta], [w.clone() for w in weights]
    mu = binding.Muon(count=count, rows=rows, cols=cols, dtype=dtype, transposed=(False, True), device=G.DEV)
    mu.step(grads, momenta, weights, lr=0.1, scale=2.0)
    alone = binding.Muon(count=1, rows=rows, cols=cols, dtype=dtype, transposed=(False,), device=G.DEV)
    for i in (0, 11, 22):
        m, w = [M0[0][i].clone()], [W0[0][i].clone()]
        alone.step([grads[0][i]], m, w, lr=0.1, scale=2.0)
        assert torch.equal(m[0], momenta[0][i])
        d = (w[0].double() - weights[0][i].double()).norm() / (W0[0][i].double() - weights[0][i].double()).norm()
        # two results of the same inputs: twice the tolerance, and twice the rounding of the weights against the size of the update
        assert d <= 2 * TOL[dtype] + 2 * torch.finfo(TYPES[dtype]).eps * float(W0[0][i].double().norm() / (W0[0][i].double() - weights[0][i].double()).norm())


def test_other_coefficients():
    """A cubic that converges (c = 0), and the momentum off."""
    coef = (1.5, -0.5, 0.0)
    grads, momenta, weights = _case(96, 160, 2, "f32", (False,), seed=9)
    M0, W0 = [m.clone() for m in momenta], [w.clone() for w in weights]
    mu = binding.Muon(count=2, rows=96, cols=160, dtype="f32", momentum=0.0, nesterov=False, steps=5, coefficients=coef, device=G.DEV)
    mu.step(grads, momenta, weights, lr=0.1)
    m, w, x = _want(grads[0], M0[0], W0[0], mu=0.0, nesterov=False, lr=0.1, wd=0.0, scale=1.0, coef=coef)
    assert torch.equal(momenta[0], grads[0])
    assert float((weights[0].double() - w).norm()) <= 1e-5 * float(x.norm()) + 2.0 ** -23 * float(W0[0].norm())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_out_of_the_ordinary(dtype):
    """No gradient at all, one element, rank one, tiny and huge ones (their squares leave fp32); a NaN or an infinity stays in its own matrix."""
    rows, cols = 130, 200
    g = torch.Generator(device=G.DEV).manual_seed(3)
    grads = [torch.zeros(8, rows, cols, device=G.DEV)]
    grads[0][1, 77, 99] = 2.0
    grads[0][2] = torch.randn(rows, 1, generator=g, device=G.DEV) @ torch.randn(1, cols, generator=g, device=G.DEV)
    for i in range(3, 8):
        grads[0][i] = _gradient(g, 1, rows, cols)[0]
    grads[0][3] *= 1e-30
    grads[0][4] *= 1e30
    grads[0][5, 3, 4] = math.nan
    grads[0][6, 100, 0] = math.inf
    momenta = [torch.zeros_like(grads[0])]
    W0 = (torch.randn(8, rows, cols, generator=g, device=G.DEV) / 16).to(TYPES[dtype])
    weights = [W0.clone()]
    mu = binding.Muon(count=8, rows=rows, cols=cols, dtype=dtype, device=G.DEV)
    mu.step(grads, momenta, weights, lr=0.1, scale=2.0)
    fine = [1, 2, 4, 7]
    # rank one: what is left of the roundings in the other directions grows by 3.4445 a step, 2^-12 of the norm spread over them: 0.15 of the factor
    # in 11 bits, 3e-5 in 22, of a factor whose norm is one
    tol = {"bf16": [0.05, 0.4, 4e-2, 4e-2], "f32": [1e-5, 1e-4, 1e-5, 1e-5]}[dtype]
    for i, t in zip(fine, tol):
        _check(dtype, grads[0][i:i + 1], torch.zeros_like(grads[0][i:i + 1]), W0[i:i + 1], momenta[0][i:i + 1], weights[0][i:i + 1], tol=t, lr=0.1, wd=0.0, scale=2.0)
    # nothing, and so little that the damping of the norm is what it is divided by
    assert torch.equal(weights[0][0], W0[0]) and torch.equal(weights[0][3], W0[3])
    assert torch.isnan(weights[0][5]).all() and torch.isnan(weights[0][6]).all()


def test_repeats_and_streams():
    """The same bits every time, on another stream too; a workspace that other sizes have used."""
    grads, momenta, weights = _case(500, 333, 2, "bf16", (False, True))
    out = []
    mu = binding.Muon(count=2, rows=500, cols=333, dtype="bf16", transposed=(False, True), device=G.DEV)
    side = torch.cuda.Stream()
    for k in range(3):
        m, w = [x.clone() for x in momenta], [x.clone() for x in weights]
        mu.ws.random_(0, 255)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side if k == 2 else torch.cuda.current_stream()):
            mu.step(grads, m, w, lr=0.02, scale=3.0)
        torch.cuda.synchronize()
        out.append((m, w))
    for m, w in out[1:]:
        assert all(torch.equal(x, y) for x, y in zip(m + w, out[0][0] + out[0][1]))


def test_captured():
    """A step in a graph, replayed among eager work: each replay what an eager step gives."""
    grads, momenta, weights = _case(320, 200, 2, "bf16", (False, True))
    mu = binding.Muon(count=2, rows=320, cols=200, dtype="bf16", transposed=(False, True), device=G.DEV)
    version = torch.zeros(2, dtype=torch.int32, device=G.DEV)
    m, w = [x.clone() for x in momenta], [x.clone() for x in weights]
    mu.step(grads, m, w, lr=0.02, scale=3.0, version=version)              # kernels set up before the capture
    for x, y in zip(m + w, momenta + weights):
        x.copy_(y)
    version.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mu.step(grads, m, w, lr=0.02, scale=3.0, version=version)
    em, ew = [x.clone() for x in momenta], [x.clone() for x in weights]
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in m + w]
        mu.step(grads, em, ew, lr=0.02, scale=3.0)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, em + ew)), k
        assert version.tolist() == [k + 1, k + 1]


def test_no_alignment():
    """Tensors that begin at any element."""
    rows, cols = 65, 131
    grads, momenta, weights = _case(rows, cols, 1, "bf16", (False,))
    off = lambda t: torch.cat([t.new_zeros(3), t.flatten()])[3:].view(t.shape)  # noqa: E731
    g2, m2, w2 = off(grads[0]), off(momenta[0]), off(weights[0])
    assert w2.data_ptr() % 4 != 0 and g2.data_ptr() % 16 != 0
    mu = binding.Muon(count=1, rows=rows, cols=cols, dtype="bf16", device=G.DEV)
    mu.step(grads, momenta, weights, lr=0.02, scale=3.0)
    mu.step([g2], [m2], [w2], lr=0.02, scale=3.0)
    assert torch.equal(m2, momenta[0]) and torch.equal(w2, weights[0])


def test_refusals_of_the_binding():
    grads, momenta, weights = _case(64, 128, 2, "bf16", (False, True))
    mu = binding.Muon(count=2, rows=64, cols=128, dtype="bf16", transposed=(False, True), device=G.DEV)
    with pytest.raises(ValueError):
        mu.step(grads[:1], momenta, weights, lr=0.1)
    with pytest.raises(ValueError):
        mu.step(grads, momenta, [w.float() for w in weights], lr=0.1)
    with pytest.raises(ValueError):
        mu.step([g[:1] for g in grads], momenta, weights, lr=0.1)
    with pytest.raises(ValueError):
        mu.step([g.mT for g in grads], momenta, weights, lr=0.1)
    with pytest.raises(binding.MoeError):
        mu.step(grads, momenta, weights, lr=math.nan)
    with pytest.raises(binding.MoeError):
        mu.step(grads, momenta, weights, lr=0.1, copies=[w.clone() for w in weights])
    with pytest.raises(ValueError):
        binding.Muon(count=1, rows=4, cols=4, dtype="bf16", transposed=(), device=G.DEV)
    with pytest.raises(binding.MoeError):
        binding.Muon(count=1, rows=0, cols=4, dtype="bf16", device=G.DEV)
