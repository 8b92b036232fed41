"""Gradient of the attention against the formulas in 64 bits (attn_util: values and bounds), against differences of the forward call, and what the forward
call's tests look at: widths, groups, lengths, keys more and fewer than queries, layouts, rows of no sequence, values that nothing may see, graphs."""
import math

import pytest
import torch

import attn_util as A
import gpu_util as G
from paper_2411_10003_amd import binding
from test_gpu_attention import MANY, _parts, _said, _where

pytestmark = pytest.mark.gpu


def _given(Q, K, V, parts, causal, seed):
    """An upstream gradient, and O and lse as 64 bits rounded to their types have them."""
    d = Q.shape[2]
    dO, = A.tensors(Q.shape[0], (Q.shape[1],), d, Q.dtype, "apart", seed)
    O, _, lse, _ = A.forward(Q, K, V, parts, d ** -0.5, causal)
    return dO, O.nan_to_num().to(Q.dtype), lse.nan_to_num(nan=0.0, neginf=-math.inf).float()


def _grads(at, dO, Q, K, V, O, lse, off, where, layout="apart"):
    make = lambda x: torch.full((x.shape[1], x.shape[0], x.shape[2]), 7.0, dtype=x.dtype, device=G.DEV).transpose(0, 1) if layout == "heads" else torch.full_like(x, 7.0, memory_format=torch.contiguous_format)  # noqa: E731
    out = make(Q), make(K), make(V)
    at.bwd(dO, Q, K, V, O, lse, off, *out, k_begin=where and where[0], k_end=where and where[1])
    return out


def _check(Q, K, V, lens, dtype, *, causal=True, keys=None, layout="apart", begin=None):
    parts = _parts(lens, keys, begin)
    heads, kv, d = Q.shape[1], K.shape[1], Q.shape[2]
    at = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype=dtype, rows=Q.shape[0], k_rows=K.shape[0], seqs=len(lens), causal=causal, device=G.DEV)
    where = None
    if keys is not None:
        where = tuple(torch.tensor(v, dtype=torch.int32, device=G.DEV) for v in ([p[2] for p in parts], [p[2] + p[3] for p in parts]))
    dO, O, lse = _given(Q, K, V, parts, causal, sum(lens))
    got = _grads(at, dO, Q, K, V, O, lse, A.offsets(lens), where, layout)
    want = A.backward(dO, Q, K, V, O, lse, parts, d ** -0.5, causal)
    for name, g, (w, b) in zip(("dQ", "dK", "dV"), got, want):
        assert A.near(g, w, b), (name, float(((g.double() - w).abs() / b).nan_to_num().max()))
        left = torch.isnan(w)
        assert (g[left] == 7.0).all(), name
    again = _grads(at, dO, Q, K, V, O, lse, A.offsets(lens), where, layout)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    return got, want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 24, 32, 40, 64, 72, 80, 96, 120, 128])
def test_widths(d, dtype):
    lens = [1, 37, 64, 65, 0, 130, 300]
    Q, K, V = A.tensors(sum(lens), (4, 2, 2), d, A.TYPES[dtype], "fused", d)
    _check(Q, K, V, lens, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (6, 2), (5, 1), (16, 8)])
def test_groups_of_heads(heads, kv, dtype):
    """The gradient of a key that several heads share is the sum over them."""
    lens = [5, 257, 33, 512]
    Q, K, V = A.tensors(sum(lens), (heads, kv, kv), 64, A.TYPES[dtype], "apart", heads * 10 + kv)
    _check(Q, K, V, lens, dtype, layout="heads")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,d,layout", [(18, 18, 128, "fused"), (36, 18, 64, "heads"), (20, 20, 72, "apart"), (40, 20, 32, "fused"), (24, 24, 8, "heads"), (36, 2, 128, "apart")])
def test_many_blocks(heads, kv, d, layout, causal, dtype):
    """The kernels of large calls; with two kv heads the first of them and that of few keys."""
    Q, K, V = A.tensors(sum(MANY), (heads, kv, kv), d, A.TYPES[dtype], layout, heads + d)
    _check(Q, K, V, MANY, dtype, causal=causal, layout="heads" if layout == "heads" else "apart")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_many_blocks_more_and_fewer_keys(causal, dtype):
    keys = [500, 70, 64, 0, 64, 512, 300, 65, 1000]
    Q, = A.tensors(sum(MANY), (20,), 64, A.TYPES[dtype], "apart", 3)
    K, V = A.tensors(sum(keys), (20, 20), 64, A.TYPES[dtype], "fused", 4)
    _check(Q, K, V, MANY, dtype, causal=causal, keys=keys)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [[1], [2, 1], [127], [128], [129], [256, 257], [31, 32, 33], [63, 64, 65, 66], [0, 0, 129, 0], [1] * 70 + [200], [1500, 3]])
def test_lengths(lens, causal):
    Q, K, V = A.tensors(sum(lens), (4, 2, 2), 128, torch.bfloat16, "heads", len(lens))
    _check(Q, K, V, lens, "bf16", causal=causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,keys", [([300, 200, 1], [500, 100, 40]), ([300, 65], [0, 64]), ([260, 0], [3, 200]), ([100, 400], [1000, 463]), ([3, 500], [500, 3])])
def test_more_and_fewer_keys_than_queries(lens, keys, causal, dtype):
    """Queries that see nothing have no gradient, nor have keys that no query sees."""
    Q, = A.tensors(sum(lens), (6,), 64, A.TYPES[dtype], "apart", 3)
    K, V = A.tensors(sum(keys), (2, 2), 64, A.TYPES[dtype], "fused", 4)
    (dQ, dK, dV), _ = _check(Q, K, V, lens, dtype, causal=causal, keys=keys)
    for (q, n, k, m) in _parts(lens, keys):
        nothing = n if m == 0 else max(0, n - m) if causal else 0
        assert not dQ[q:q + nothing].any()
        if n == 0:
            assert not dK[k:k + m].any() and not dV[k:k + m].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_no_sequence_and_gaps(dtype):
    """Keys in places of their own; rows outside every sequence, NaN among them, are neither looked at nor written."""
    t, lens, keys, begin = A.TYPES[dtype], [70, 300], [90, 310], [7, 150]
    Q, = A.tensors(370, (4,), 80, t, "apart", 3)
    K, V = A.tensors(500, (2, 2), 80, t, "apart", 4)
    inside = torch.zeros(500, dtype=torch.bool, device=G.DEV)
    for b, m in zip(begin, keys):
        inside[b:b + m] = True
    K[~inside], V[~inside] = math.nan, math.inf
    _check(Q, K, V, lens, dtype, keys=keys, begin=begin)


def test_gradient_against_differences():
    """<dO, O> along directions of Q, K and V: central differences of the forward call against the backward call's gradients, both in fp32.  The difference's
    own truncation, which the 64-bit formulas give (the step against a 64th of it, whose truncation is 4096 times smaller), is taken off; what is left is off by the forward call's
    bounds over the step, which is a long one for that reason; the gradients by theirs, and by what the bounds of O leave in D: scale p |<U, k>| of it in dQ, scale p |<q, U>| in dK."""
    lens, heads, kv, d, h = [40, 90], 4, 2, 32, 2.0 ** -2
    scale = d ** -0.5
    Q, K, V = A.tensors(130, (heads, kv, kv), d, torch.float32, "apart", 5)
    dO, = A.tensors(130, (heads,), d, torch.float32, "apart", 6)
    U = A.tensors(130, (heads, kv, kv), d, torch.float32, "apart", 7)
    off, parts = A.offsets(lens), _parts(lens)
    at = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype="f32", rows=130, seqs=2, device=G.DEV)

    def value(*x):
        O = torch.empty(130, heads, d, device=G.DEV)
        at.fwd(*x, O, off)
        return float((O.double() * dO.double()).sum())

    def exact(*x):
        return float((A.forward(*x, parts, scale, True)[0] * dO.double()).sum())

    O, lse = torch.empty_like(Q), torch.empty(heads, 130, device=G.DEV)
    at.fwd(Q, K, V, O, off, lse=lse)
    grads = _grads(at, dO, Q, K, V, O, lse, off, None)
    bounds = A.backward(dO, Q, K, V, O, lse, parts, scale, True)
    bO = A.forward(Q, K, V, parts, scale, True)[1]
    inside = (bO * dO.double().abs()).sum(2)                # of <dO, O> of every row and head
    for i in range(3):
        def difference(f, step):
            # the ends as fp32 has them, and the distance between them
            a, b = ([(x.double() + s * step * U[i].double()).to(x.dtype if f is value else torch.float64) if j == i else x if f is value else x.double()
                     for j, x in enumerate((Q, K, V))] for s in (1.0, -1.0))
            return (f(*a) - f(*b)) / (2 * step)
        got = float((grads[i].double() * U[i].double()).sum())
        truncation = difference(exact, h) - difference(exact, h / 64)
        # the ends are rounded to fp32: a unit of 2^-24 of each element moves the value by the gradient
        ends = 2.0 ** -24 * float((grads[i].double().abs() * (Q, K, V)[i].double().abs()).sum()) / h
        left = 0.0
        if i < 2:
            reach = float(torch.maximum((U[0].double().norm(dim=2).max() * K.double().norm(dim=2).max()), (U[1].double().norm(dim=2).max() * Q.double().norm(dim=2).max())))
            left = scale * reach * float(inside.sum())
        want = difference(value, h) - truncation
        allowed = abs(truncation) / 4000 + ends + float(inside.sum()) / h + float((bounds[i][1] * U[i].double().abs()).sum()) + left
        assert abs(got - want) <= allowed, (i, got, want, allowed)
        assert allowed < 0.5 * abs(got), (i, got, allowed)  # a factor of two or a sign would show


@pytest.mark.parametrize("heads,kv", [(4, 2), (120, 60)])
def test_values_out_of_the_ordinary(heads, kv):
    """Scores far apart; a NaN of one sequence stays in it."""
    lens, d = [200, 150, 170], 64
    Q, K, V = A.tensors(520, (heads, kv, kv), d, torch.bfloat16, "apart", 8)
    Q[3] *= 40.0
    Q[4] = 0.0
    _check(Q, K, V, lens, "bf16")
    at = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype="bf16", rows=520, seqs=3, device=G.DEV)
    dO, O, lse = _given(Q, K, V, _parts(lens), True, 1)
    off = A.offsets(lens)
    want = _grads(at, dO, Q, K, V, O, lse, off, None)
    for x in (Q, K, V, dO, O):
        x[200:350] = math.nan
    got = _grads(at, dO, Q, K, V, O, lse, off, None)
    for a, b in zip(got, want):
        assert torch.equal(a[:200], b[:200]) and torch.equal(a[350:], b[350:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,d", [(2, 64), (2, 128), (112, 64), (112, 128)])
def test_reach_of_a_value_that_is_no_number(heads, d, dtype):
    """A NaN in a row of one input: where the formulas have it, and in rows that causality hides from it no further away than the header says; the others keep their bits."""
    reach, n, m, t = _said(r"hides from it by up to (\d+) positions"), 600, 601, A.TYPES[dtype]
    Q, = A.tensors(n, (heads,), d, t, "apart", 51)
    K, V = A.tensors(m, (heads, heads), d, t, "apart", 52)
    parts, where = _parts([n], [m]), _where([m])
    dO, O, lse = _given(Q, K, V, parts, True, 53)
    at = binding.Attention(heads=heads, kv_heads=heads, d=d, dtype=dtype, rows=n, k_rows=m, seqs=1, device=G.DEV)
    clean = _grads(at, dO, Q, K, V, O, lse, A.offsets([n]), where)
    queries, keys = torch.arange(n, device=G.DEV) + m - n, torch.arange(m, device=G.DEV)           # a query stands where the last key that it sees does
    furthest = 0
    for which in range(5):
        for row in (0, 31, 32, 127, 224, 255, 256, 480, 511, 599):
            given = [dO, Q, K, V, O]
            given[which] = given[which].clone()
            given[which][row] = math.nan
            got = _grads(at, *given, lse, A.offsets([n]), where)
            changed = [~(a == b).flatten(1).all(1) for a, b in zip(got, clean)]
            if which in (2, 3):                            # a key: queries before it do not see it; other keys do not know of it
                away = row - queries[changed[0]]
                assert all(c.sum() <= 1 for c in changed[1:])
            else:                                          # a query: keys behind it are hidden from it; other queries do not know of it
                away = torch.cat([keys[c] - queries[row] for c in changed[1:]])
                assert changed[0].sum() <= 1
            if away.numel():
                furthest = max(furthest, int(away.max()))
    assert furthest <= reach
    if heads > 100 and dtype == "bf16":
        assert furthest == reach                           # blocks of 256 keys, tiles of 32 queries


@pytest.mark.parametrize("heads,kv", [(4, 2), (96, 48)])
def test_captured(heads, kv):
    """Forward and backward in one graph, replayed on new inputs among eager calls; the graph's calls have a workspace of their own."""
    lens, d, rows = [300, 1, 0, 211], 128, 512
    off = A.offsets(lens)
    make = lambda: binding.Attention(heads=heads, kv_heads=kv, d=d, dtype="bf16", rows=rows, seqs=4, device=G.DEV)  # noqa: E731
    ats = [make(), make()]
    Q, K, V = A.tensors(rows, (heads, kv, kv), d, torch.bfloat16, "fused", 1)
    dO, = A.tensors(rows, (heads,), d, torch.bfloat16, "apart", 2)
    outs = [dict(O=torch.empty_like(dO), lse=torch.empty(heads, rows, device=G.DEV), dQ=torch.empty_like(dO), dK=torch.empty(rows, kv, d, dtype=torch.bfloat16, device=G.DEV),
                 dV=torch.empty(rows, kv, d, dtype=torch.bfloat16, device=G.DEV)) for _ in range(2)]

    def both(at, o):
        at.fwd(Q, K, V, o["O"], off, lse=o["lse"])
        at.bwd(dO, Q, K, V, o["O"], o["lse"], off, o["dQ"], o["dK"], o["dV"])

    both(ats[0], outs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(ats[0], outs[0])
    for k in range(4):
        for x, y in zip((Q, K, V), A.tensors(rows, (heads, kv, kv), d, torch.bfloat16, "apart", 20 + k)):
            x.copy_(y)
        graph.replay()
        both(ats[1], outs[1])
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0][n], outs[1][n]) for n in outs[0]), k


def test_nothing_to_do():
    at = binding.Attention(heads=2, kv_heads=1, d=64, dtype="bf16", rows=0, k_rows=16, seqs=1, device=G.DEV)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=G.DEV)
    K, stats = torch.zeros(16, 1, 64, dtype=torch.bfloat16, device=G.DEV), torch.empty(2, 0, device=G.DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=G.DEV)  # noqa: E731
    dK, dV = torch.full_like(K, 7.0), torch.full_like(K, 7.0)
    at.bwd(none, none, K, K, none, stats, i32(0, 0), none, dK, dV, k_begin=i32(3), k_end=i32(9))
    for x in (dK, dV):                                     # keys that nothing looks at
        assert not x[3:9].any() and (x[:3] == 7.0).all() and (x[9:] == 7.0).all()
    at.ws = None
    with pytest.raises(ValueError):
        at.bwd(none, none, K, K, none, stats, i32(0, 0), none, dK, dV, k_begin=i32(3), k_end=i32(9))


@pytest.mark.parametrize("dtype,heads,d", [("bf16", 36, 128), ("bf16", 48, 64), ("bf16", 2, 128), ("f32", 60, 64), ("f32", 2, 128)])
def test_rows_past_32_bits(dtype, heads, d):
    """Rows as far apart as they may lie, 4 MB of bf16 or 8 MB of fp32: the last of them more than 2^32 bytes in; blocks of every kernel."""
    n, row = 1200, 2 ** 21 - 8
    whole = torch.empty(n * row, dtype=A.TYPES[dtype], device=G.DEV)
    Q, K, V = (whole.as_strided((n, heads, d), (row, d, 1), i * heads * d) for i in range(3))
    for x, y in zip((Q, K, V), A.tensors(n, (heads,) * 3, d, A.TYPES[dtype], "apart", 3)):
        x.copy_(y)
    _check(Q, K, V, [700, 500], dtype)


@pytest.mark.parametrize("lens,heads", [([300, 0, 77], 4), ([900, 1500], 24)])
def test_two_streams(lens, heads):
    """Two objects beside each other, each on a stream of its own, several times: the bits of the calls alone."""
    calls = []
    for seed in (1, 2):
        Q, K, V = A.tensors(sum(lens), (heads, heads, heads), 128, torch.bfloat16, "fused", seed)
        dO, O, lse = _given(Q, K, V, _parts(lens), True, seed)
        at = binding.Attention(heads=heads, kv_heads=heads, d=128, dtype="bf16", rows=sum(lens), seqs=len(lens), device=G.DEV)
        args = (at, dO, Q, K, V, O, lse, A.offsets(lens), None)
        calls.append((args, _grads(*args), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for args, _, stream in calls:
            with torch.cuda.stream(stream):
                got.append(_grads(*args))
        torch.cuda.synchronize()
        for (_, want, _), new in zip(calls, got):
            assert all(torch.equal(a, b) for a, b in zip(want, new))
