"""The example of a block's training step: its gradients against 64-bit autograd through the same routing, and that it learns."""
import os
import sys

import pytest
import torch

import gpu_util as G

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_gradients_of_the_block():
    """bf16 tensors pass through a dozen roundings of 2^-9 relative rms each on the way: 1.5e-2 of a whole tensor's norm (the layer's own tests hold
    each of its tensors to 1e-2)."""
    from block_train_step import Block
    T, d, h, E, k = 256, 128, 192, 4, 2
    blk = Block(T=T, d=d, h=h, E=E, k=k, seed=3)
    g = torch.Generator(device=G.DEV).manual_seed(9)
    randn = lambda *s: torch.randn(*s, generator=g, device=G.DEV)  # noqa: E731
    for p in (*blk.gamma, *blk.beta):
        p += 0.2 * randn(d)
    X, R, dOut = randn(T, d).to(torch.bfloat16), randn(T, d).to(torch.bfloat16), randn(T, d).to(torch.bfloat16)
    out = blk.forward(X, R).clone()
    dX = blk.backward(dOut).clone()
    idx = blk.b.idx.long()
    # the same computation in 64 bits, on the routing that the gate chose
    leaf = lambda t: t.double().clone().requires_grad_()  # noqa: E731
    x, r, W1, W2, W3, Wg, bg = leaf(X), leaf(R), *(leaf(p) for p in blk.pools), leaf(blk.Wg), leaf(blk.bg)
    gam, bet = [leaf(p) for p in blk.gamma], [leaf(p) for p in blk.beta]

    def norm(s, i):
        m = s.mean(1, keepdim=True)
        return (s - m) / torch.sqrt(((s - m) ** 2).mean(1, keepdim=True) + 1e-5) * gam[i] + bet[i]

    s = x + r
    y = norm(s, 0)
    p = torch.softmax(y @ Wg + bg, 1).gather(1, idx)
    w = p / p.sum(1, keepdim=True)
    o = torch.zeros_like(y)
    for e in range(E):
        ye = (torch.nn.functional.silu(y @ W1[e]) * (y @ W3[e])) @ W2[e]
        o = o + (w * (idx == e)).sum(1, keepdim=True) * ye
    z = norm(o + s, 1)
    z.backward(dOut.double())
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(out, z.detach()) <= 1.5e-2
    got = dict(dX=dX, dW1=blk.b.dW1, dW2=blk.b.dW2, dW3=blk.b.dW3, dWg=blk.dWg, dbg=blk.dbg, dgamma0=blk.dgamma[0], dgamma1=blk.dgamma[1], dbeta0=blk.dbeta[0], dbeta1=blk.dbeta[1])
    want = dict(dX=x.grad, dW1=W1.grad, dW2=W2.grad, dW3=W3.grad, dWg=Wg.grad, dbg=bg.grad, dgamma0=gam[0].grad, dgamma1=gam[1].grad, dbeta0=bet[0].grad, dbeta1=bet[1].grad)
    assert torch.allclose(x.grad, r.grad)
    for n in got:
        assert rel(got[n], want[n]) <= 1.5e-2, (n, rel(got[n], want[n]))


def test_it_learns():
    from block_train_step import train
    losses, blk = train(12, 1024, 128, 256, 4)
    assert losses[-1] < 0.7 * losses[0], losses
    # every expert was updated in every step, and the slots hold what the pools held before the last update
    assert blk.version.tolist() == [12] * 4 and blk.slot_version.tolist() == [11] * 4
    assert all(torch.equal(c, m.to(torch.bfloat16)) for c, m in zip(blk.pools, blk.masters))
