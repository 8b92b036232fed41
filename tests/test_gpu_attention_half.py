"""Norm, rotation and attention together, as a block uses them: the example's attention half against 64-bit autograd; an answer's tokens, one at a time through
rotation, cache and attention, against the whole sequence at once; both halves of the example's block in a captured step."""
import math
import os
import sys

import pytest
import torch

import attn_util as A
import gpu_util as G
from paper_2411_10003_amd import binding

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _turned(x, positions, f):
    t = positions.double()[:, None, None] * f
    a, b = x.chunk(2, -1)
    return torch.cat((a * torch.cos(t) - b * torch.sin(t), b * torch.cos(t) + a * torch.sin(t)), -1)


@pytest.mark.parametrize("T,d,heads,kv", [(200, 128, 4, 2), (333, 192, 8, 8), (257, 256, 2, 1)])
def test_gradients_of_the_half(T, d, heads, kv):
    """bf16 tensors pass through a dozen roundings on the way (2^-9 relative rms each, and two for each projection): 1.5e-2 of a whole tensor's norm, as for the block's
    other half."""
    from block_train_step import AttentionHalf, packed
    half = AttentionHalf(T=T, d=d, heads=heads, kv_heads=kv, seqs=4, seed=5)
    g = torch.Generator(device=G.DEV).manual_seed(T)
    randn = lambda *s: torch.randn(*s, generator=g, device=G.DEV)  # noqa: E731
    for p in (half.gamma, half.beta, half.gamma_q, half.gamma_k):
        p += 0.2 * randn(p.shape[0])
    S, dX, dS = (randn(T, d).to(torch.bfloat16) for _ in range(3))
    offsets, positions = packed(T, 4, g)
    out = half.forward(S, offsets, positions)
    back = half.backward(dX, dS)
    leaf = lambda t: t.double().clone().requires_grad_()  # noqa: E731
    names = ("gamma", "beta", "gamma_q", "gamma_k", "Wqkv", "Wo")
    s, p = leaf(S), {n: leaf(getattr(half, n)) for n in names}
    m = s.mean(1, keepdim=True)
    y = (s - m) / torch.sqrt(((s - m) ** 2).mean(1, keepdim=True) + 1e-5) * p["gamma"] + p["beta"]
    q, k, v = (y @ p["Wqkv"]).view(T, -1, d // heads).split((heads, kv, kv), 1)
    rms = lambda x, w: x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w  # noqa: E731
    q, k = _turned(rms(q, p["gamma_q"]), positions, half.frequencies), _turned(rms(k, p["gamma_k"]), positions, half.frequencies)
    rows = []
    for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist()):
        hidden = torch.ones(b - a, b - a, dtype=torch.bool, device=G.DEV).triu(1)
        o = [torch.softmax((q[a:b, i] @ k[a:b, i * kv // heads].T / math.sqrt(d // heads)).masked_fill(hidden, -math.inf), 1) @ v[a:b, i * kv // heads] for i in range(heads)]
        rows.append(torch.cat(o, 1))
    x = torch.cat(rows) @ p["Wo"]
    ((x * dX.double()).sum() + (s * dS.double()).sum()).backward()
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(out, x.detach()) <= 1.5e-2
    assert rel(back, s.grad) <= 1.5e-2
    for n in names:
        assert rel(getattr(half, "d" + n), p[n].grad) <= 1.5e-2, (n, rel(getattr(half, "d" + n), p[n].grad))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_by_token(dtype):
    """Three answers and an empty place in the batch, a token each a step: rotated into their places of a cache, then attended to.  Every row has to be within its bound of
    the formulas over the keys and values that the cache holds, and those have to be the bits of one rotation of the whole sequence."""
    heads, kv, d, room, lens = 4, 2, 64, 50, [37, 12, 50]
    t = A.TYPES[dtype]
    Q, K, V = A.tensors(4 * room, (heads, kv, kv), d, t, "fused", 8)       # answer s: rows s * room on
    f = binding.rotary_frequencies(d, device=G.DEV)
    gammas = [1.0 + 0.3 * torch.randn(d, generator=torch.Generator(device=G.DEV).manual_seed(i), device=G.DEV) for i in range(2)]
    rotary = binding.Rotary(heads=heads, kv_heads=kv, d=d, dtype=dtype, norm=True, device=G.DEV)
    attention = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype=dtype, rows=4, k_rows=4 * room, seqs=4, device=G.DEV)
    Kc, Vc = (torch.full((4 * room, kv, d), math.nan, dtype=t, device=G.DEV) for _ in range(2))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=G.DEV)  # noqa: E731
    offsets, begin = i32([0, 1, 2, 3, 4]), i32([0, room, 2 * room, 3 * room])
    q = torch.empty(4, heads, d, dtype=t, device=G.DEV)
    where = torch.arange(room, dtype=torch.int32, device=G.DEV).repeat(4)
    Qall, Kall = torch.empty(4 * room, heads, d, dtype=t, device=G.DEV), torch.empty(4 * room, kv, d, dtype=t, device=G.DEV)
    rotary.fwd(Q, K, where, f, Qall, Kall, gamma_q=gammas[0], gamma_k=gammas[1])
    for step in range(room):
        rows = [s * room + step for s in range(4)]
        alive = [s < 3 and step < lens[s] for s in range(4)]
        slots = i32([r if a else -1 for r, a in zip(rows, alive)])
        rotary.fwd(Q[rows], K[rows], i32([step] * 4), f, q, Kc, gamma_q=gammas[0], gamma_k=gammas[1], V=V[rows], Vo=Vc, slots=slots)
        end = begin + i32([step + 1 if a else 0 for a in alive])
        O = torch.full((4, heads, d), 7.0, dtype=t, device=G.DEV)
        attention.fwd(q, Kc, Vc, O, offsets, k_begin=begin, k_end=end)
        parts = [(s, 1, s * room, step + 1 if alive[s] else 0) for s in range(4)]
        want, bound, _, _ = A.forward(q, Kc, Vc, parts, d ** -0.5, True)
        assert A.near(O, want, bound), step
        assert torch.equal(q[:3], Qall[rows[:3]])
    for s in range(3):
        mine = slice(s * room, s * room + lens[s])
        assert torch.equal(Kc[mine], Kall[mine]) and torch.equal(Vc[mine], V[mine])
        assert bool(torch.isnan(Kc[mine.stop:(s + 1) * room]).all())
    assert bool(torch.isnan(Kc[3 * room:]).all() & torch.isnan(Vc[3 * room:]).all())


def test_both_halves_run():
    from block_train_step import train_both_halves
    losses, block, half = train_both_halves(3, 512, 128, 192, 4, 4, 2)
    assert all(math.isfinite(v) for v in losses) and block.version.tolist() == [3] * 4
    for n in ("Wqkv", "Wo", "gamma", "gamma_q", "gamma_k"):
        assert bool(torch.isfinite(getattr(half, n)).all()) and float(getattr(half, "d" + n).float().abs().max()) > 0.0, n


def test_a_captured_step():
    """Forward and gradients of the half in one graph, replayed over new rows and other sequences between eager steps of another object: the eager bits each time."""
    from block_train_step import AttentionHalf, packed
    T, d = 300, 128
    one, other = (AttentionHalf(T=T, d=d, heads=4, kv_heads=2, seqs=4, seed=2) for _ in range(2))
    g = torch.Generator(device=G.DEV).manual_seed(1)
    S, dX, dS = (torch.empty(T, d, dtype=torch.bfloat16, device=G.DEV) for _ in range(3))
    offsets, positions = packed(T, 4, g)

    def fill():
        for x in (S, dX, dS):
            x.copy_(torch.randn(T, d, generator=g, device=G.DEV))
        for to, new in zip((offsets, positions), packed(T, 4, g)):
            to.copy_(new)

    def step(half):
        return half.forward(S, offsets, positions), half.backward(dX, dS)

    fill()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(one)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, back = step(one)
    for _ in range(4):
        fill()
        graph.replay()
        want_out, want_back = step(other)
        torch.cuda.synchronize()
        assert torch.equal(out, want_out) and torch.equal(back, want_back)
        for n in ("dWqkv", "dWo", "dgamma", "dgamma_q", "dgamma_k"):
            assert torch.equal(getattr(one, n), getattr(other, n)), n
