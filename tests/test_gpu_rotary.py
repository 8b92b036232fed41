"""Norm and rotation of heads, their way into a cache, and their gradient, against the formulas in 64 bits.

Tolerances, e = 2^-24, u = eps(t) / 2 of the type.  Angles are 64-bit products reduced to a turn: rounded to fp32 in units of half a turn, 2^-25 of them at most, pi 2^-25
of a radian, and cosine and sine 4 e off at most for that and for the functions (of two units in the last place).  A rotated element is two products and a sum:
(4 + 3) e amplitude (|a| + |b|).  The norm: a sum of d squares in chains of 16 and a tree, 24 e of it, half that in rstd, and 4 more roundings: 16 e of an element.
Gradients of the norm: sums of d terms with 24 e + 8 e of the sum of magnitudes; dgamma: chains over a thread's heads, at most n of them: (n + 40) e of the sum of magnitudes."""
import math

import pytest
import torch

import attn_util as A
import gpu_util as G
from paper_2411_10003_amd import binding

pytestmark = pytest.mark.gpu
E = A.E24


def _turn(x, positions, f, rot, interleaved, amplitude, sign=1.0):
    """Rotated heads and the sum |a| + |b| of each element's pair (zero where nothing turns)."""
    t = positions.double()[:, None, None] * f
    c, s = torch.cos(t) * amplitude, sign * torch.sin(t) * amplitude
    y, size = x.clone(), torch.zeros_like(x)
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = abs(amplitude) * (x[..., i].abs() + x[..., j].abs())
    return y, size


def _forward(x, gamma, positions, f, rot, interleaved, amplitude, eps):
    v = x.double()
    if gamma is not None:
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * gamma.double()
    y, size = _turn(v, positions, f, rot, interleaved, amplitude)
    u = A.rounding(x.dtype)
    return y, (7 + 16) * E * size + 16 * E * v.abs() * (size == 0) * (gamma is not None) + u * y.abs() + 1e-37


def _backward(dy, x, gamma, positions, f, rot, interleaved, amplitude, eps):
    g, size = _turn(dy.double(), positions, f, rot, interleaved, amplitude, -1.0)
    eg = 7 * E * size
    u = A.rounding(dy.dtype)
    if gamma is None:
        return g, eg + u * g.abs() + 1e-37, None, None
    x = x.double()
    rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xh, w = x * rstd, gamma.double()
    mid = (g * w * xh).mean(-1, keepdim=True)
    dx = rstd * (g * w - xh * mid)
    sizes = (g * w * xh).abs().mean(-1, keepdim=True)
    bound = rstd * (eg * w.abs() + 20 * E * (g * w).abs() + xh.abs() * ((eg * w * xh).abs().mean(-1, keepdim=True) + 48 * E * sizes)) + u * dx.abs()
    n = g.shape[0] * g.shape[1]
    return dx, 1.01 * bound + 1e-37, (g * xh).sum((0, 1)), (((n + 40) * E * (g * xh).abs()) + eg * xh.abs()).sum((0, 1)) + 1e-37


def _inputs(rows, heads, kv, d, dtype, seed, layout="fused"):
    g = torch.Generator(device=G.DEV).manual_seed(seed)
    t = A.TYPES[dtype]
    Q, K, V = A.tensors(rows, (heads, kv, kv), d, t, layout, seed)
    gammas = [1.0 + 0.3 * torch.randn(d, generator=g, device=G.DEV) for _ in range(2)]
    dQo, dKo = A.tensors(rows, (heads, kv), d, t, "apart", seed + 1)
    positions = torch.randint(0, 5000, (rows,), generator=g, device=G.DEV, dtype=torch.int32)
    return Q, K, V, gammas, dQo, dKo, positions


def _check(rows, heads, kv, d, dtype, *, rot, interleaved, norm, amplitude=1.0, positions=None, layout="fused", seed=0):
    Q, K, V, gammas, dQo, dKo, pos = _inputs(rows, heads, kv, d, dtype, 100 * rows + d + seed, layout)
    pos = pos if positions is None else positions
    f = binding.rotary_frequencies(rot, device=G.DEV)
    gq, gk = gammas if norm else (None, None)
    r = binding.Rotary(heads=heads, kv_heads=kv, d=d, dtype=dtype, rot=rot, interleaved=interleaved, norm=norm, amplitude=amplitude, device=G.DEV)
    Qo, Ko = (torch.full(x.shape, 7.0, dtype=x.dtype, device=G.DEV) for x in (Q, K))
    r.fwd(Q, K, pos, f, Qo, Ko, gamma_q=gq, gamma_k=gk)
    what = (f, rot, interleaved, amplitude, 1e-6)
    for name, got, x, gamma in (("Q", Qo, Q, gq), ("K", Ko, K, gk)):
        want, bound = _forward(x, gamma, pos, *what)
        assert A.near(got, want, bound), (name, float(((got.double() - want).abs() / bound).max()))
    dQ, dK = (torch.full(x.shape, 7.0, dtype=x.dtype, device=G.DEV) for x in (Q, K))
    dgq, dgk = (torch.full((d,), 7.0, device=G.DEV) for _ in range(2)) if norm else (None, None)
    more = dict(Q=Q, K=K, gamma_q=gq, gamma_k=gk, dgamma_q=dgq, dgamma_k=dgk) if norm else {}
    r.bwd(dQo, dKo, pos, f, dQ, dK, **more)
    for name, got, dy, x, gamma, dg in (("dQ", dQ, dQo, Q, gq, dgq), ("dK", dK, dKo, K, gk, dgk)):
        want, bound, wg, bg = _backward(dy, x, gamma, pos, *what)
        assert A.near(got, want, bound), (name, float(((got.double() - want).abs() / bound).max()))
        if norm:
            assert A.near(dg, wg, bg), (name, "gamma", float(((dg.double() - wg).abs() / bg).max()))
    if norm:
        again = [torch.empty_like(t) for t in (dQ, dK, dgq, dgk)]
        r.bwd(dQo, dKo, pos, f, again[0], again[1], Q=Q, K=K, gamma_q=gq, gamma_k=gk, dgamma_q=again[2], dgamma_k=again[3])
        assert all(torch.equal(a, b) for a, b in zip(again, (dQ, dK, dgq, dgk)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(8, 8), (8, 2), (16, 16), (24, 24), (32, 32), (32, 16), (40, 20), (48, 6), (64, 64), (72, 72), (80, 40), (80, 80), (96, 32), (120, 118), (128, 128),
                                   (128, 64), (128, 0), (136, 136), (192, 64), (256, 256), (256, 30)])
def test_widths_and_parts(d, rot, interleaved, dtype):
    for rows in (1, 7, 70):
        for norm in (False, True):
            _check(rows, 5, 2, d, dtype, rot=rot, interleaved=interleaved, norm=norm)


@pytest.mark.parametrize("rows,heads,kv,d", [(2100, 3, 1, 64), (1100, 32, 8, 128), (9001, 2, 2, 40), (5000, 40, 1, 32), (40000, 8, 2, 128)])
def test_many_rows(rows, heads, kv, d):
    """More rows than blocks; the last size goes past the caches."""
    _check(rows, heads, kv, d, "bf16", rot=d, interleaved=False, norm=True, layout="apart")
    _check(rows, heads, kv, d, "bf16", rot=d // 8 * 4, interleaved=True, norm=False, layout="heads", amplitude=1.2)


@pytest.mark.parametrize("rows,heads,kv,d", [(2000, 1, 1000, 8), (1500, 700, 1, 8), (900, 1, 1, 128)])
def test_partial_sums_stay_in_the_workspace(rows, heads, kv, d):
    """However the heads are shared out between queries and keys: more blocks than partial sums of either, and what lies behind the workspace stays."""
    Q, K, V, gammas, dQo, dKo, pos = _inputs(rows, heads, kv, d, "bf16", 5, "apart")
    f = binding.rotary_frequencies(d, device=G.DEV)
    r = binding.Rotary(heads=heads, kv_heads=kv, d=d, dtype="bf16", norm=True, device=G.DEV, alloc_workspace=False)
    room = torch.full((r.workspace_bytes + 4096,), 0x5a, dtype=torch.uint8, device=G.DEV)
    r.ws = room[:r.workspace_bytes]
    dQ, dK, dgq, dgk = torch.empty_like(Q), torch.empty_like(K), *(torch.empty(d, device=G.DEV) for _ in range(2))
    r.bwd(dQo, dKo, pos, f, dQ, dK, Q=Q, K=K, gamma_q=gammas[0], gamma_k=gammas[1], dgamma_q=dgq, dgamma_k=dgk)
    assert bool((room[r.workspace_bytes:] == 0x5a).all())
    for got, dy, x, gamma, dg in ((dQ, dQo, Q, gammas[0], dgq), (dK, dKo, K, gammas[1], dgk)):
        want, bound, wg, bg = _backward(dy, x, gamma, pos, f, d, False, 1.0, 1e-6)
        assert A.near(got, want, bound) and A.near(dg, wg, bg)


def test_more_rows_than_a_launch_takes():
    """2^24 + 5 rows of 256 elements, in place; looked at: the ends and where one launch gives way to the next."""
    rows, d = 2 ** 24 + 5, 256
    x = torch.ones(rows, 2, d, dtype=torch.bfloat16, device=G.DEV)
    look = torch.tensor([0, 1, 2 ** 24 - 5, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 3, rows - 1], device=G.DEV)
    x[look] = torch.randn(len(look), 2, d, generator=torch.Generator(device=G.DEV).manual_seed(3), device=G.DEV).to(torch.bfloat16)
    before = x[look].clone()
    f, pos = binding.rotary_frequencies(d, device=G.DEV), torch.arange(rows, dtype=torch.int32, device=G.DEV)
    r = binding.Rotary(heads=1, kv_heads=1, d=d, dtype="bf16", device=G.DEV)
    r.fwd(x[:, :1], x[:, 1:], pos, f, x[:, :1], x[:, 1:])
    want, bound = _forward(before, None, pos[look], f, d, False, 1.0, 1e-6)
    assert A.near(x[look], want, bound)
    before = x[look].clone()
    r.bwd(x[:, :1], x[:, 1:], pos, f, x[:, :1], x[:, 1:])
    want, bound, _, _ = _backward(before, None, None, pos[look], f, d, False, 1.0, 1e-6)
    assert A.near(x[look], want, bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions(dtype):
    """Angles of positions up to 2^31: their products with the frequencies are far past what 32 bits tell apart."""
    positions = torch.tensor([0, 1, 4095, 131071, 10 ** 6, 10 ** 9, 2 ** 31 - 1, -5], dtype=torch.int32, device=G.DEV)
    _check(8, 4, 4, 64, dtype, rot=64, interleaved=False, norm=False, positions=positions)


def test_frequencies():
    f = binding.rotary_frequencies(64, device=G.DEV).cpu()
    assert f.dtype == torch.float64 and f.shape == (32,) and f[0] == 1.0 and abs(float(f[1]) - 10000.0 ** (-1 / 32)) < 1e-15
    assert torch.equal(binding.rotary_frequencies(64, factor=4.0, device=G.DEV).cpu(), f / 4.0)
    by_parts = binding.rotary_frequencies(64, factor=4.0, trained=4096, device=G.DEV).cpu()
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(by_parts[turns >= 32.0], f[turns >= 32.0]) and torch.equal(by_parts[turns <= 1.0], f[turns <= 1.0] / 4.0)
    between = (turns > 1.0) & (turns < 32.0)
    assert ((by_parts < f) & (by_parts > f / 4.0))[between].all()
    for bad in (dict(rot=3), dict(rot=-2), dict(rot=4, factor=0.0), dict(rot=4, base=-1.0), dict(rot=4, trained=100, fast=1.0, slow=1.0)):
        with pytest.raises(ValueError):
            binding.rotary_frequencies(**bad, device=G.DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 33, 1500])
def test_into_a_cache(rows, dtype):
    """Keys and values to rows of a cache, whatever the order; those with no place nowhere; the other rows of the cache as they were."""
    heads, kv, d, places = 6, 2, 96, 4000
    Q, K, V, (gq, gk), _, _, pos = _inputs(rows, heads, kv, d, dtype, 3)
    g = torch.Generator(device=G.DEV).manual_seed(1)
    slots = torch.randperm(places, generator=g, device=G.DEV)[:rows].to(torch.int32)
    if rows > 1:
        slots[0], slots[rows // 2], slots[rows - 1] = -1, places, 2 ** 31 - 1
    r = binding.Rotary(heads=heads, kv_heads=kv, d=d, dtype=dtype, norm=True, device=G.DEV)
    f = binding.rotary_frequencies(d, device=G.DEV)
    Qo, Qw, Kw, Vw = torch.empty_like(Q), torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    Kc, Vc = (torch.full((kv, places, d), 7.0, dtype=Q.dtype, device=G.DEV).transpose(0, 1) for _ in range(2))
    r.fwd(Q, K, pos, f, Qo, Kc, gamma_q=gq, gamma_k=gk, V=V, Vo=Vc, slots=slots)
    r.fwd(Q, K, pos, f, Qw, Kw, gamma_q=gq, gamma_k=gk, V=V, Vo=Vw)
    assert torch.equal(Qo, Qw) and torch.equal(Vw, V)
    kept = (slots >= 0) & (slots < places)
    wantK, wantV = torch.full_like(Kc, 7.0), torch.full_like(Vc, 7.0)
    wantK[slots[kept].long()], wantV[slots[kept].long()] = Kw[kept], V[kept]
    assert torch.equal(Kc, wantK) and torch.equal(Vc, wantV)


@pytest.mark.parametrize("rot,interleaved", [(64, False), (40, False), (64, True)])
def test_in_place_and_streams(rot, interleaved):
    rows, heads, kv, d = 700, 4, 2, 64
    Q, K, V, (gq, gk), dQo, dKo, pos = _inputs(rows, heads, kv, d, "bf16", 5)
    r = binding.Rotary(heads=heads, kv_heads=kv, d=d, dtype="bf16", rot=rot, interleaved=interleaved, norm=True, device=G.DEV)
    f = binding.rotary_frequencies(rot, device=G.DEV)
    Qo, Ko, dQ, dK = (torch.empty(x.shape, dtype=x.dtype, device=G.DEV) for x in (Q, K, Q, K))
    dg = [torch.empty(d, device=G.DEV) for _ in range(4)]
    r.fwd(Q, K, pos, f, Qo, Ko, gamma_q=gq, gamma_k=gk)
    r.bwd(dQo, dKo, pos, f, dQ, dK, Q=Q, K=K, gamma_q=gq, gamma_k=gk, dgamma_q=dg[0], dgamma_k=dg[1])
    q, k = Q.clone(), K.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.fwd(q, k, pos, f, q, k, gamma_q=gq, gamma_k=gk)
    side.synchronize()
    assert torch.equal(q, Qo) and torch.equal(k, Ko)
    a, b = dQo.clone(), dKo.clone()
    r.bwd(a, b, pos, f, a, b, Q=Q, K=K, gamma_q=gq, gamma_k=gk, dgamma_q=dg[2], dgamma_k=dg[3])
    assert torch.equal(a, dQ) and torch.equal(b, dK) and torch.equal(dg[0], dg[2]) and torch.equal(dg[1], dg[3])
    q, k = Q.clone(), K.clone()
    r.bwd(dQo, dKo, pos, f, q, k, Q=q, K=k, gamma_q=gq, gamma_k=gk, dgamma_q=dg[2], dgamma_k=dg[3])
    assert torch.equal(q, dQ) and torch.equal(k, dK)


def test_gradient_against_differences():
    """The backward call against central differences of the forward one in fp32, along directions of Q, K and both gammas."""
    rows, heads, kv, d, h = 9, 3, 2, 48, 2.0 ** -6
    Q, K, _, (gq, gk), dQo, dKo, pos = _inputs(rows, heads, kv, d, "f32", 6, "apart")
    r = binding.Rotary(heads=heads, kv_heads=kv, d=d, dtype="f32", rot=32, norm=True, amplitude=1.3, device=G.DEV)
    f = binding.rotary_frequencies(32, device=G.DEV)

    def value(Q, K, gq, gk):
        Qo, Ko = torch.empty_like(Q), torch.empty_like(K)
        r.fwd(Q, K, pos, f, Qo, Ko, gamma_q=gq, gamma_k=gk)
        return float((Qo.double() * dQo.double()).sum() + (Ko.double() * dKo.double()).sum())

    at = [Q, K, gq, gk]
    out = [torch.empty_like(x) for x in at]
    r.bwd(dQo, dKo, pos, f, out[0], out[1], Q=Q, K=K, gamma_q=gq, gamma_k=gk, dgamma_q=out[2], dgamma_k=out[3])
    gen = torch.Generator(device=G.DEV).manual_seed(7)
    for i in range(4):
        U = torch.randn(at[i].shape, generator=gen, device=G.DEV)
        step = lambda s: value(*(x + s * h * U if j == i else x for j, x in enumerate(at)))  # noqa: E731
        difference, got = (step(1.0) - step(-1.0)) / (2 * h), float((out[i].double() * U.double()).sum())
        # The forward call is linear in the gammas.  In a head x along U it is a unit vector (cos t, sin t) in the plane of the two, t = atan(b s / (1 + a s)) with
        # (a, b) = U / |x| along and across x, r its length: with the derivatives t1 = b, t2 = -2 a b, t3 = 6 a^2 b - 2 b^3 of t its third one is i t3 - 3 t1 t2 - i t1^3 in
        # that plane, at most 6 a^2 b + 3 b^3 + 6 a b^2 <= 6 r^3.  So the difference is off by h^2 / 6 of 6 r^3 |dy| |y|, y's length being sqrt(d) max gamma amplitude at
        # most, 10 % for the terms after it, and by the values' own errors, 24 e of the sizes they are summed from, over h.
        size = math.sqrt(d) * 1.3 * float(torch.maximum(gq.abs().max(), gk.abs().max()))
        lengths = [g.norm(dim=-1).double() for g in (dQo, dKo)]
        off = 24 * E / h * size * float(sum(v.sum() for v in lengths))
        if i < 2:
            off += 1.1 * h * h * size * float((lengths[i] * (U.norm(dim=-1) / at[i].norm(dim=-1)).double() ** 3).sum())
        assert abs(got - difference) <= off, (i, got, difference, off)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_out_of_the_ordinary(dtype):
    """Heads of zeros, tiny and huge ones; an infinity or a NaN stays in its head."""
    rows, d = 6, 64
    Q, K, _, (gq, gk), dQo, dKo, pos = _inputs(rows, 2, 2, d, dtype, 8, "apart")
    Q[0] = 0.0
    Q[1] *= 1e-15
    Q[2] *= 1e12
    clean = [x.clone() for x in (Q, K, dQo, dKo)]
    r = binding.Rotary(heads=2, kv_heads=2, d=d, dtype=dtype, norm=True, device=G.DEV)
    f = binding.rotary_frequencies(d, device=G.DEV)

    def both(Q, K, dQo, dKo):
        out = [torch.empty_like(x) for x in (Q, K, Q, K)]
        dg = [torch.empty(d, device=G.DEV) for _ in range(2)]
        r.fwd(Q, K, pos, f, out[0], out[1], gamma_q=gq, gamma_k=gk)
        r.bwd(dQo, dKo, pos, f, out[2], out[3], Q=Q, K=K, gamma_q=gq, gamma_k=gk, dgamma_q=dg[0], dgamma_k=dg[1])
        return out

    want = both(*clean)
    y, bound = _forward(clean[0], gq, pos, f, d, False, 1.0, 1e-6)
    assert A.near(want[0], y, bound)
    Q[4, 1, 3] = math.nan
    K[5, 0, 63] = math.inf
    dQo[3, 0, 7] = math.nan
    got = both(Q, K, dQo, dKo)
    for i, heads in enumerate(({(4, 1)}, {(5, 0)}, {(4, 1), (3, 0)}, {(5, 0)})):
        for t in range(rows):
            for h in range(2):
                if (t, h) in heads:
                    assert torch.isnan(got[i][t, h]).any() or i == 1
                else:
                    assert torch.equal(got[i][t, h], want[i][t, h]), (i, t, h)


def test_captured():
    """Forward and backward in a graph, replayed on new inputs among eager calls."""
    rows, heads, kv, d = 3000, 4, 2, 64
    Q, K, V, (gq, gk), dQo, dKo, pos = _inputs(rows, heads, kv, d, "bf16", 9)
    rs = [binding.Rotary(heads=heads, kv_heads=kv, d=d, dtype="bf16", norm=True, device=G.DEV) for _ in range(2)]
    f = binding.rotary_frequencies(d, device=G.DEV)
    outs = [[torch.empty(x.shape, dtype=x.dtype, device=G.DEV) for x in (Q, K, Q, K, gq, gk)] for _ in range(2)]

    def both(r, o):
        r.fwd(Q, K, pos, f, o[0], o[1], gamma_q=gq, gamma_k=gk)
        r.bwd(dQo, dKo, pos, f, o[2], o[3], Q=Q, K=K, gamma_q=gq, gamma_k=gk, dgamma_q=o[4], dgamma_k=o[5])

    both(rs[0], outs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(rs[0], outs[0])
    for k in range(4):
        new = _inputs(rows, heads, kv, d, "bf16", 30 + k)
        for x, y in zip((Q, K, dQo, pos), (new[0], new[1], new[4], new[6])):
            x.copy_(y)
        graph.replay()
        both(rs[1], outs[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs)), k


def test_no_rows():
    d = 64
    r = binding.Rotary(heads=2, kv_heads=1, d=d, dtype="bf16", norm=True, device=G.DEV)
    q, k = torch.empty(0, 2, d, dtype=torch.bfloat16, device=G.DEV), torch.empty(0, 1, d, dtype=torch.bfloat16, device=G.DEV)
    pos, f, gamma = torch.empty(0, dtype=torch.int32, device=G.DEV), binding.rotary_frequencies(d, device=G.DEV), torch.ones(d, device=G.DEV)
    dg = [torch.full((d,), 7.0, device=G.DEV) for _ in range(2)]
    r.fwd(q, k, pos, f, q, k, gamma_q=gamma, gamma_k=gamma)
    r.bwd(q, k, pos, f, q, k, Q=q, K=k, gamma_q=gamma, gamma_k=gamma, dgamma_q=dg[0], dgamma_k=dg[1])
    assert not dg[0].any() and not dg[1].any()


def test_refusals_of_the_binding():
    d = 64
    r = binding.Rotary(heads=2, kv_heads=1, d=d, dtype="bf16", norm=True, device=G.DEV)
    q, k = torch.zeros(4, 2, d, dtype=torch.bfloat16, device=G.DEV), torch.zeros(4, 1, d, dtype=torch.bfloat16, device=G.DEV)
    pos, f, gamma = torch.zeros(4, dtype=torch.int32, device=G.DEV), binding.rotary_frequencies(d, device=G.DEV), torch.ones(d, device=G.DEV)
    r.fwd(q, k, pos, f, q, k, gamma_q=gamma, gamma_k=gamma)
    for a in ((q[:3], k, pos, f, q, k), (q, k, pos[:3], f, q, k), (q, k, pos, f.float(), q, k), (q, k, pos, f[:16], q, k), (q, k, pos, f, q.float(), k), (q, k, pos.long(), f, q, k),
              (q[..., :32], k, pos, f, q, k), (q, k, pos, f, q, q)):
        with pytest.raises(ValueError):
            r.fwd(*a, gamma_q=gamma, gamma_k=gamma)
    with pytest.raises(binding.MoeError):
        r.fwd(q, k, pos, f, q, k)                          # a norm without parameters
    with pytest.raises(binding.MoeError):
        r.fwd(q, k, pos, f, q, k, gamma_q=gamma, gamma_k=gamma, V=k)
    with pytest.raises(binding.MoeError):
        r.bwd(q, k, pos, f, q, k, gamma_q=gamma, gamma_k=gamma, dgamma_q=gamma.clone(), dgamma_k=gamma.clone())
    with pytest.raises(binding.MoeError):
        r.fwd(q, k, pos, f, q[:1].expand(4, 2, d), k, gamma_q=gamma, gamma_k=gamma)
