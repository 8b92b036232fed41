"""The layer norm with the residual sum, and its gradient, against the formulas in 64 bits: widths around the pieces, threads and
waves that share a row, odd widths (rows that begin at any element), one row and none, rows more than the blocks of a launch, and rows
with infinities, NaN, nothing but zeros, or a mean far above their spread.

Tolerances.  eps(t) / 2 is the relative rounding of a type.  Forward: the sum S is exact up to one rounding of its type.  mean and rstd are fp32
sums of d terms in chains of at most 4 pieces and trees above: 32 + 16 additions at most, 48 x 2^-24 of the sum of magnitudes, so 3e-6 of it.
Y: one rounding, and the fp32 error of (s - mean) rstd gamma + beta: the mean's (3e-6 of the row's mean magnitude, times rstd gamma) and rstd's
(half the relative error of the variance, 48 x 2^-24, and two more).  Backward: dX the same with two sums; dgamma, dbeta: chains over the rows of a
thread, at most 2048 here (the bound of a chain of n: n x 2^-24 of the sum of magnitudes)."""
import math

import pytest
import torch

import gpu_util as G
from paper_2411_10003_amd import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FP32 = 48 * 2.0 ** -24


def _half(t):
    return torch.finfo(t).eps / 2


def _inputs(rows, d, dtype, seed=0):
    g = torch.Generator(device=G.DEV).manual_seed(1000 * rows + d + seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=G.DEV)  # noqa: E731
    t = TYPES[dtype]
    return dict(X=(randn(rows, d) + 0.5 * randn(d)).to(t), R=(3.0 * randn(rows, d)).to(t), gamma=1.0 + 0.3 * randn(d), beta=0.5 * randn(d),
                dY=randn(rows, d).to(t), dS=randn(rows, d).to(t))


def _forward(S, gamma, beta, eps):
    s = S.double()
    mean = s.mean(1)
    var = ((s - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / torch.sqrt(var + eps)
    y = (s - mean[:, None]) * rstd[:, None] * gamma.double()
    return mean, rstd, y + beta.double() if beta is not None else y


def _forward_bounds(S, gamma, beta, mean, rstd, y):
    """Allowed errors of mean, rstd (relative) and Y (element by element)."""
    size = S.double().abs().mean(1)
    m = FP32 * size + 2.0 ** -24 * mean.abs()
    # the mean's error adds to the variance in second order; the centred values' rounding and the sum's in first
    r = 0.5 * (FP32 + 4 * 2.0 ** -24) + 3 * 2.0 ** -24 + (m * rstd) ** 2
    core = ((S.double() - mean[:, None]) * rstd[:, None] * gamma.double()).abs()
    e = m[:, None] * rstd[:, None] * gamma.double().abs() + core * (r[:, None] + 4 * 2.0 ** -24) + y.abs() * (2.0 ** -24 + _half(S.dtype))
    return m, r, e


def _backward(dY, S, gamma, mean, rstd, dS):
    y, s = dY.double(), S.double()
    xh = (s - mean.double()[:, None]) * rstd.double()[:, None]
    g = y * gamma.double()
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = rstd.double()[:, None] * (g - c1 - xh * c2)
    e = rstd.double()[:, None] * (g.abs() + FP32 * 0 + c1.abs() + (xh * c2).abs())             # sizes of the terms
    sums = rstd.double()[:, None] * (g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    e = 8 * 2.0 ** -24 * e + (FP32 + 4 * 2.0 ** -24) * sums
    if dS is not None:
        dx = dx + dS.double()
    e = e + dx.abs() * (2.0 ** -24 + _half(S.dtype))
    return dx, e, (y * xh).sum(0), (y * xh).abs().sum(0), y.sum(0), y.abs().sum(0)


WIDTHS = [1, 3, 7, 8, 9, 64, 100, 127, 128, 129, 255, 256, 512, 513, 1021, 1024, 1025, 2048, 2056, 4095, 4096, 4104, 8192, 8200, 16383, 16384]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward_and_backward_by_width(d, dtype):
    for rows in (1, 2, 5, 33, 1030):
        i = _inputs(rows, d, dtype)
        n = binding.Norm(d=d, dtype=dtype, eps=1e-5, device=G.DEV)
        for residual in (False, True):
            beta = i["beta"] if residual else None
            R = i["R"] if residual else None
            S = torch.empty_like(i["X"]) if residual else None
            Y, mean, rstd = torch.full_like(i["X"], 7.0), torch.empty(rows, device=G.DEV), torch.empty(rows, device=G.DEV)
            n.fwd(i["X"], i["gamma"], beta, Y, residual=R, total=S, mean=mean, rstd=rstd)
            if residual:
                assert torch.equal(S, (i["X"].float() + R.float()).to(S.dtype)), (rows, "S")
            else:
                S = i["X"]
            wm, wr, wy = _forward(S, i["gamma"], beta, 1e-5)
            em, er, ey = _forward_bounds(S, i["gamma"], beta, wm, wr, wy)
            assert ((mean.double() - wm).abs() <= em).all(), (rows, "mean")
            assert ((rstd.double() / wr - 1).abs() <= er).all(), (rows, "rstd")
            assert ((Y.double() - wy).abs() <= ey).all(), (rows, "Y")
            Y2 = torch.empty_like(Y)
            n.fwd(i["X"], i["gamma"], beta, Y2, residual=R, total=torch.empty_like(S) if residual else None)       # nothing kept: the same Y
            assert torch.equal(Y, Y2)
            dX, dg, db = torch.empty_like(S), torch.full((d,), 7.0, device=G.DEV), torch.full((d,), 7.0, device=G.DEV) if residual else None
            dS = i["dS"] if residual else None
            n.bwd(i["dY"], S, i["gamma"], mean, rstd, dX, dg, db, residual_grad=dS)
            wx, ex, wg, sg, wb, sb = _backward(i["dY"], S, i["gamma"], mean, rstd, dS)
            assert ((dX.double() - wx).abs() <= ex).all(), (rows, "dX")
            assert ((dg.double() - wg).abs() <= (rows + 8) * 2.0 ** -24 * sg).all(), (rows, "dgamma")
            if residual:
                assert ((db.double() - wb).abs() <= (rows + 4) * 2.0 ** -24 * sb).all(), (rows, "dbeta")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [5, 15, 17, 130, 260, 300, 515, 770, 1283, 1540, 1795, 2055, 2570, 2571, 3079, 3585, 4099, 5001, 6145, 6986, 8195, 12281, 12290])
def test_short_last_pieces(d, dtype):
    """Widths that leave a short piece at every place it can have among a row's threads and pieces."""
    for rows in (1, 3, 70):
        i = _inputs(rows, d, dtype, seed=1)
        n = binding.Norm(d=d, dtype=dtype, eps=1e-5, device=G.DEV)
        # rows end to end with guards around them: nothing outside is read into the result or written
        guard = lambda: torch.full((rows * d + 64,), 7.0, dtype=TYPES[dtype], device=G.DEV)  # noqa: E731
        inside = lambda t: t[32:32 + rows * d].view(rows, d)  # noqa: E731
        bS, bY, bX = guard(), guard(), guard()
        S, Y, dX = inside(bS), inside(bY), inside(bX)
        mean, rstd = torch.empty(rows, device=G.DEV), torch.empty(rows, device=G.DEV)
        n.fwd(i["X"], i["gamma"], i["beta"], Y, residual=i["R"], total=S, mean=mean, rstd=rstd)
        assert torch.equal(S, (i["X"].float() + i["R"].float()).to(S.dtype))
        wm, wr, wy = _forward(S, i["gamma"], i["beta"], 1e-5)
        em, er, ey = _forward_bounds(S, i["gamma"], i["beta"], wm, wr, wy)
        assert ((mean.double() - wm).abs() <= em).all() and ((rstd.double() / wr - 1).abs() <= er).all() and ((Y.double() - wy).abs() <= ey).all()
        dg, db = torch.full((d + 8,), 7.0, device=G.DEV), torch.full((d + 8,), 7.0, device=G.DEV)
        n.bwd(i["dY"], S, i["gamma"], mean, rstd, dX, dg[:d], db[:d], residual_grad=i["dS"])
        wx, ex, wg, sg, wb, sb = _backward(i["dY"], S, i["gamma"], mean, rstd, i["dS"])
        assert ((dX.double() - wx).abs() <= ex).all()
        assert ((dg[:d].double() - wg).abs() <= (rows + 8) * 2.0 ** -24 * sg).all() and ((db[:d].double() - wb).abs() <= (rows + 4) * 2.0 ** -24 * sb).all()
        for t in (bS, bY, bX):
            assert (t[:32] == 7.0).all() and (t[32 + rows * d:] == 7.0).all()
        assert (dg[d:] == 7.0).all() and (db[d:] == 7.0).all()


@pytest.mark.parametrize("rows,d,dtype", [(100000, 64, "bf16"), (70001, 24, "f32"), (9000, 1000, "bf16"), (5000, 4096, "bf16"), (3001, 6001, "f32")])
def test_many_rows(rows, d, dtype):
    """More rows than a launch of the gradient has places for: every block walks several."""
    i = _inputs(rows, d, dtype)
    n = binding.Norm(d=d, dtype=dtype, device=G.DEV)
    Y, mean, rstd = torch.empty_like(i["X"]), torch.empty(rows, device=G.DEV), torch.empty(rows, device=G.DEV)
    S = torch.empty_like(Y)
    n.fwd(i["X"], i["gamma"], i["beta"], Y, residual=i["R"], total=S, mean=mean, rstd=rstd)
    wm, wr, wy = _forward(S, i["gamma"], i["beta"], 1e-5)
    em, er, ey = _forward_bounds(S, i["gamma"], i["beta"], wm, wr, wy)
    assert ((mean.double() - wm).abs() <= em).all() and ((rstd.double() / wr - 1).abs() <= er).all() and ((Y.double() - wy).abs() <= ey).all()
    out = []
    for _ in range(2):
        dX, dg, db = torch.empty_like(S), torch.empty(d, device=G.DEV), torch.empty(d, device=G.DEV)
        n.bwd(i["dY"], S, i["gamma"], mean, rstd, dX, dg, db, residual_grad=i["dS"])
        out.append((dX, dg, db))
    assert all(torch.equal(a, b) for a, b in zip(*out))                    # the same bits every time
    wx, ex, wg, sg, wb, sb = _backward(i["dY"], S, i["gamma"], mean, rstd, i["dS"])
    chain = 2048 * 2.0 ** -24
    assert ((dX.double() - wx).abs() <= ex).all()
    assert ((dg.double() - wg).abs() <= chain * sg).all() and ((db.double() - wb).abs() <= chain * sb).all()


def test_gradient_against_differences():
    """The backward call against central differences of the forward one, all in fp32: <dY, Y(X + h V)> for directions V, and the parameters'."""
    rows, d, h = 6, 96, 2.0 ** -6
    i = _inputs(rows, d, "f32")
    n = binding.Norm(d=d, dtype="f32", device=G.DEV)
    mean, rstd = torch.empty(rows, device=G.DEV), torch.empty(rows, device=G.DEV)

    def value(X, gamma, beta):
        Y = torch.empty_like(X)
        n.fwd(X, gamma, beta, Y, mean=mean, rstd=rstd)
        return float((Y.double() * i["dY"].double()).sum())

    g = torch.Generator(device=G.DEV).manual_seed(5)
    V, w = torch.randn(rows, d, generator=g, device=G.DEV), torch.randn(d, generator=g, device=G.DEV)
    numbers = [(value(i["X"] + h * V, i["gamma"], i["beta"]) - value(i["X"] - h * V, i["gamma"], i["beta"])) / (2 * h),
               (value(i["X"], i["gamma"] + h * w, i["beta"]) - value(i["X"], i["gamma"] - h * w, i["beta"])) / (2 * h),
               (value(i["X"], i["gamma"], i["beta"] + h * w) - value(i["X"], i["gamma"], i["beta"] - h * w)) / (2 * h)]
    value(i["X"], i["gamma"], i["beta"])
    dX, dg, db = torch.empty_like(i["X"]), torch.empty(d, device=G.DEV), torch.empty(d, device=G.DEV)
    n.bwd(i["dY"], i["X"], i["gamma"], mean, rstd, dX, dg, db)
    got = [float((dX.double() * V.double()).sum()), float((dg.double() * w.double()).sum()), float((db.double() * w.double()).sum())]
    # second-order term of the difference: h^2 / 6 of the third derivative, of the order of the terms' sum; 5e-4 of rows d terms of order one
    size = math.sqrt(rows * d)
    for a, b in zip(numbers, got):
        assert abs(a - b) <= 5e-4 * size * 3, (a, b)


def test_in_place_and_streams():
    """S over X or over R, Y over X, dX over dY or dS; and a call on another stream than the default."""
    rows, d = 300, 1021
    i = _inputs(rows, d, "bf16")
    n = binding.Norm(d=d, dtype="bf16", device=G.DEV)
    new = lambda: torch.empty(rows, d, dtype=torch.bfloat16, device=G.DEV)  # noqa: E731
    S, Y, mean, rstd = new(), new(), torch.empty(rows, device=G.DEV), torch.empty(rows, device=G.DEV)
    n.fwd(i["X"], i["gamma"], i["beta"], Y, residual=i["R"], total=S, mean=mean, rstd=rstd)
    for which in ("X", "R"):
        a, y = {k: i[k].clone() for k in ("X", "R")}, new()
        n.fwd(a["X"], i["gamma"], i["beta"], y, residual=a["R"], total=a[which])
        assert torch.equal(a[which], S) and torch.equal(y, Y)
    x = S.clone()
    n.fwd(x, i["gamma"], i["beta"], x)
    assert torch.equal(x, Y)
    dX, dg = new(), torch.empty(d, device=G.DEV)
    n.bwd(i["dY"], S, i["gamma"], mean, rstd, dX, dg, residual_grad=i["dS"])
    for which in ("dY", "dS"):
        a = {k: i[k].clone() for k in ("dY", "dS")}
        n.bwd(a["dY"], S, i["gamma"], mean, rstd, a[which], dg, residual_grad=a["dS"])
        assert torch.equal(a[which], dX)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = new()
    with torch.cuda.stream(side):
        n.fwd(i["X"], i["gamma"], i["beta"], y, residual=i["R"], total=new())
    side.synchronize()
    assert torch.equal(y, Y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [60, 1021, 4096])
def test_rows_out_of_the_ordinary(d, dtype):
    """A row of zeros, one of equal values, one far from zero, tiny and huge ones; rows with an infinity or a NaN stay alone in theirs."""
    t = TYPES[dtype]
    g = torch.Generator(device=G.DEV).manual_seed(d)
    X = torch.randn(9, d, generator=g, device=G.DEV)
    X[1] = 0.0
    X[2] = 3.0
    X[3] = 1000.0 + 8.0 * X[3]
    X[4] *= 1e-18
    X[5] *= 1e15
    X[6, d // 2] = math.inf
    X[7, d - 1] = math.nan
    X = X.to(t)
    gamma, beta = 1.0 + 0.3 * torch.randn(d, generator=g, device=G.DEV), 0.5 * torch.randn(d, generator=g, device=G.DEV)
    n = binding.Norm(d=d, dtype=dtype, device=G.DEV)
    Y, mean, rstd = torch.empty_like(X), torch.empty(9, device=G.DEV), torch.empty(9, device=G.DEV)
    n.fwd(X, gamma, beta, Y, mean=mean, rstd=rstd)
    fine = [0, 1, 2, 3, 4, 5, 8]
    wm, wr, wy = _forward(X, gamma, beta, 1e-5)
    em, er, ey = _forward_bounds(X, gamma, beta, wm, wr, wy)
    assert ((mean.double() - wm).abs() <= em)[fine].all() and ((rstd.double() / wr - 1).abs() <= er)[fine].all()
    assert ((Y.double() - wy).abs() <= ey)[fine].all()
    assert torch.equal(Y[1], beta.to(t))
    assert torch.isnan(Y[6]).all() and torch.isnan(Y[7]).all()
    # the gradient: nothing of rows 6 and 7 in the others
    dY = torch.randn(9, d, generator=g, device=G.DEV).to(t)
    dX, dg, db = torch.empty_like(X), torch.empty(d, device=G.DEV), torch.empty(d, device=G.DEV)
    n.bwd(dY, X, gamma, mean, rstd, dX, dg, db)
    wx, ex = _backward(dY, X, gamma, mean, rstd, None)[:2]
    assert ((dX.double() - wx).abs() <= ex)[fine].all()
    assert torch.isnan(dX[6]).all() and torch.isnan(dX[7]).all()
    assert torch.isfinite(db).all()


def test_no_rows():
    d = 128
    n = binding.Norm(d=d, dtype="bf16", device=G.DEV)
    none = torch.empty(0, d, dtype=torch.bfloat16, device=G.DEV)
    stats = torch.empty(0, device=G.DEV)
    gamma = torch.ones(d, device=G.DEV)
    n.fwd(none, gamma, None, none, mean=stats, rstd=stats)
    dg, db = torch.full((d,), 7.0, device=G.DEV), torch.full((d,), 7.0, device=G.DEV)
    n.bwd(none, none, gamma, stats, stats, none, dg, db)
    assert not dg.any() and not db.any()


@pytest.mark.parametrize("rows,d", [(700, 256), (9, 1021)])
def test_captured(rows, d):
    """Forward and backward in one graph, replayed on new inputs among eager calls: each replay what the eager calls give."""
    i = _inputs(rows, d, "bf16")
    n = binding.Norm(d=d, dtype="bf16", device=G.DEV)
    new = lambda: torch.empty(rows, d, dtype=torch.bfloat16, device=G.DEV)  # noqa: E731
    outs = [dict(S=new(), Y=new(), dX=new(), mean=torch.empty(rows, device=G.DEV), rstd=torch.empty(rows, device=G.DEV), dg=torch.empty(d, device=G.DEV),
                 db=torch.empty(d, device=G.DEV)) for _ in range(2)]

    def both(o):
        n.fwd(i["X"], i["gamma"], i["beta"], o["Y"], residual=i["R"], total=o["S"], mean=o["mean"], rstd=o["rstd"])
        n.bwd(i["dY"], o["S"], i["gamma"], o["mean"], o["rstd"], o["dX"], o["dg"], o["db"], residual_grad=i["dS"])

    both(outs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(outs[0])
    for k in range(4):
        for name, t in _inputs(rows, d, "bf16", seed=k + 1).items():
            i[name].copy_(t)
        graph.replay()
        both(outs[1])
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0][m], outs[1][m]) for m in outs[0]), k


def test_offsets_past_32_bits():
    """More than 2^32 bytes of rows: the last ones against the formulas."""
    d, rows = 4096, 540000
    X = torch.empty(rows, d, dtype=torch.bfloat16, device=G.DEV)
    X.view(torch.int16).random_(0x3c00, 0x4000)                            # positive numbers below two
    X[::2] *= -1
    n = binding.Norm(d=d, dtype="bf16", device=G.DEV)
    gamma, beta = torch.linspace(0.5, 1.5, d, device=G.DEV), torch.linspace(-1, 1, d, device=G.DEV)
    mean, rstd = torch.empty(rows, device=G.DEV), torch.empty(rows, device=G.DEV)
    last = X[-3:].clone()
    dX, dg = torch.empty_like(X), torch.empty(d, device=G.DEV)
    Y = torch.empty_like(X)
    n.fwd(X, gamma, beta, Y, mean=mean, rstd=rstd)
    wm, wr, wy = _forward(last, gamma, beta, 1e-5)
    assert ((Y[-3:].double() - wy).abs() <= _forward_bounds(last, gamma, beta, wm, wr, wy)[2]).all()
    n.bwd(Y, X, gamma, mean, rstd, dX, dg)
    wx, ex = _backward(Y[-3:], last, gamma, mean[-3:], rstd[-3:], None)[:2]
    assert ((dX[-3:].double() - wx).abs() <= ex).all()


def test_refusals_of_the_binding():
    n = binding.Norm(d=64, dtype="bf16", device=G.DEV)
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device=G.DEV)
    gamma, stats = torch.ones(64, device=G.DEV), torch.empty(4, device=G.DEV)
    with pytest.raises(ValueError):
        n.fwd(x[:, :63].contiguous(), gamma, None, x)                      # no whole rows
    with pytest.raises(ValueError):
        n.fwd(x.float(), gamma, None, x)
    with pytest.raises(ValueError):
        n.fwd(x.t().contiguous().t(), gamma, None, x)                      # rows that are not contiguous
    with pytest.raises(ValueError):
        n.fwd(x, gamma[:32], None, x)
    with pytest.raises(ValueError):
        n.fwd(x, gamma, None, x[:2])
    with pytest.raises(binding.MoeError):
        n.fwd(x, gamma, None, x, residual=x)                               # a residual without a place for the sum
    with pytest.raises(binding.MoeError):
        n.fwd(x, gamma, None, x, mean=stats)
    with pytest.raises(binding.MoeError):
        n.bwd(x, x, gamma, stats, stats, x, None)
