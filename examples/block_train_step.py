"""A pre-norm MoE block trained on one GPU: the norm ahead of the gate, the layer, the norm after it, all gradients, the update of the experts
by Muon and the transfer of the updated ones into the slots the layer reads.

    python examples/block_train_step.py [--steps 20] [--tokens 2048] [--width 256] [--hidden 512] [--experts 8]

The block learns to give a fixed map of its input (synthetic).  All experts are this GPU's own (one destination), so nothing has to arrive from
elsewhere.  fp32 master weights live in pools of all experts beside the bf16 copies that moe_trans takes them from.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2411_10003_amd import binding  # noqa: E402

DEV = "cuda:0"


class Block:
    def __init__(self, *, T, d, h, E, k=2, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.T, self.d, self.h, self.E = T, d, h, E
        self.hd = binding.Handle(T=T, d=d, h=h, E=E, k=k, P=1, self_dest=0, G=E, dtype="bf16", act="swiglu", renorm=1, device=DEV)
        self.hd.set_act_saved(True)                                        # the workspace stays with the layer from forward to backward
        self.b = binding.LayerBuffers(self.hd, backward=True)
        self.norm = binding.Norm(d=d, dtype="bf16", device=DEV)
        # W1, W3 [E,d,h] and W2 [E,h,d]: one update for the three
        self.shapes = [(E, d, h), (E, h, d), (E, d, h)]
        self.masters = [randn(*s) / math.sqrt(s[1]) for s in self.shapes]
        self.pools = [w.to(torch.bfloat16) for w in self.masters]
        self.momenta = [torch.zeros(*s, device=DEV) for s in self.shapes]
        self.muon = binding.Muon(count=E, rows=d, cols=h, dtype="f32", transposed=(False, True, False), device=DEV)
        self.version = torch.zeros(E, dtype=torch.int32, device=DEV)
        # the slots the layer reads; the plan: every expert is computed here
        self.groups = [torch.zeros_like(p) for p in self.pools]
        self.dest = torch.zeros(E, dtype=torch.int32, device=DEV)
        self.slot_expert = torch.full((E,), -1, dtype=torch.int32, device=DEV)
        self.slot_version = torch.full((E,), -1, dtype=torch.int32, device=DEV)
        self.Wg, self.bg = randn(d, E) / math.sqrt(d), torch.zeros(E, device=DEV)
        self.gamma, self.beta = [torch.ones(d, device=DEV) for _ in range(2)], [torch.zeros(d, device=DEV) for _ in range(2)]
        rows = lambda: torch.empty(T, d, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        stat = lambda: torch.empty(T, device=DEV)  # noqa: E731
        self.S, self.Y, self.stats = [rows(), rows()], [rows(), rows()], [(stat(), stat()), (stat(), stat())]
        self.dY, self.dS, self.dX = rows(), rows(), rows()
        self.dgamma, self.dbeta = [torch.empty(d, device=DEV) for _ in range(2)], [torch.empty(d, device=DEV) for _ in range(2)]
        self.dWg, self.dbg = torch.empty(d, E, device=DEV), torch.empty(E, device=DEV)

    def forward(self, X, R):
        """X: what the half of the block before this one gives, R: the residual stream."""
        hd, b = self.hd, self.b
        hd.trans(self.dest, self.slot_expert, self.pools, self.groups, self.version, self.slot_version)
        self.norm.fwd(X, self.gamma[0], self.beta[0], self.Y[0], residual=R, total=self.S[0], mean=self.stats[0][0], rstd=self.stats[0][1])
        binding.layer_forward(hd, b, self.Y[0], self.Wg, self.bg, self.dest, *self.groups)
        self.norm.fwd(b.out, self.gamma[1], self.beta[1], self.Y[1], residual=self.S[0], total=self.S[1], mean=self.stats[1][0], rstd=self.stats[1][1])
        return self.Y[1]

    def backward(self, dOut):
        """dOut: gradient of what forward() returned.  Leaves the gradients of X and of R (the same) in dX."""
        hd, b = self.hd, self.b
        self.norm.bwd(dOut, self.S[1], self.gamma[1], *self.stats[1], self.dS, self.dgamma[1], self.dbeta[1])
        hd.combine_bwd(self.dS, b.Yp, b.layout.pos, b.w, b.dYp, b.dw)
        hd.expert_ffn_bwd(b.dYp, b.Xp, b.Z, b.U, b.layout, *self.groups, b.dXp, b.dW1, b.dW2, b.dW3)
        hd.gate_bwd(b.dw, b.logits, b.idx, b.dlogits)
        hd.gate_bwd_params(self.Y[0], b.dlogits, self.dWg, self.dbg)
        hd.input_grad(b.dXp, b.layout.pos, b.dlogits, self.Wg, self.dY)
        self.norm.bwd(self.dY, self.S[0], self.gamma[0], *self.stats[0], self.dX, self.dgamma[0], self.dbeta[0], residual_grad=self.dS)
        return self.dX

    def update(self, lr, lr_vectors):
        b = self.b
        self.muon.step([b.dW1, b.dW2, b.dW3], self.momenta, self.masters, lr=lr, weight_decay=0.01, scale=0.2 * math.sqrt(max(self.d, self.h)),
                       copies=self.pools, version=self.version)
        for p, g in ((self.Wg, self.dWg), (self.bg, self.dbg), *zip(self.gamma, self.dgamma), *zip(self.beta, self.dbeta)):
            p.sub_(lr_vectors * g)


def train(steps, T, d, h, E, seed=0, lr=0.02, lr_vectors=0.05):
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    block = Block(T=T, d=d, h=h, E=E, seed=seed)
    target_map = torch.randn(d, d, generator=g, device=DEV) / math.sqrt(d)
    losses = []
    for _ in range(steps):
        X = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
        R = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
        want = torch.tanh((X.float() + R.float()) @ target_map)
        diff = block.forward(X, R).float() - want
        losses.append(float(diff.square().mean()))
        block.backward((diff * (2.0 / T)).to(torch.bfloat16))
        block.update(lr, lr_vectors)
    return losses, block


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--experts", type=int, default=8)
    a = ap.parse_args()
    for i, loss in enumerate(train(a.steps, a.tokens, a.width, a.hidden, a.experts)[0]):
        print(f"step {i}: loss {loss:.4f}", flush=True)
