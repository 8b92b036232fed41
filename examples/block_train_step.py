"""A pre-norm MoE block trained on one GPU: the norm ahead of the gate, the layer, the norm after it, all gradients, the update of the experts
by Muon and the transfer of the updated ones into the slots the layer reads.  With --heads the half before it too: norm, projection, rotation of queries and
keys with a norm of their heads, attention over packed sequences of random lengths, projection.

    python examples/block_train_step.py [--steps 20] [--tokens 2048] [--width 256] [--hidden 512] [--experts 8] [--heads 4 --kv-heads 2]

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


class AttentionHalf:
    """S -> the attention's output over packed sequences; d / heads columns a head.  The projections are library products."""

    def __init__(self, *, T, d, heads, kv_heads, seqs, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        bf16 = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        w, n = d // heads, heads + 2 * kv_heads
        self.parts = (heads, kv_heads, kv_heads)
        self.norm = binding.Norm(d=d, dtype="bf16", device=DEV)
        self.rotary = binding.Rotary(heads=heads, kv_heads=kv_heads, d=w, dtype="bf16", norm=True, device=DEV)
        self.attention = binding.Attention(heads=heads, kv_heads=kv_heads, d=w, dtype="bf16", rows=T, seqs=seqs, device=DEV)
        self.frequencies = binding.rotary_frequencies(w, device=DEV)
        self.gamma, self.beta = torch.ones(d, device=DEV), torch.zeros(d, device=DEV)
        self.gamma_q, self.gamma_k = torch.ones(w, device=DEV), torch.ones(w, device=DEV)
        self.Wqkv, self.Wo = (randn(d, n * w) / math.sqrt(d)).to(torch.bfloat16), (randn(heads * w, d) / math.sqrt(heads * w)).to(torch.bfloat16)
        self.Y, self.mean, self.rstd = bf16(T, d), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        self.QKV, self.Q, self.K = bf16(T, n, w), bf16(T, heads, w), bf16(T, kv_heads, w)
        self.O, self.lse = torch.zeros(T, heads, w, dtype=torch.bfloat16, device=DEV), torch.empty(heads * T, device=DEV)
        self.dQKV, self.dS = torch.zeros_like(self.QKV), bf16(T, d)
        self.dgamma, self.dbeta = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        self.dgamma_q, self.dgamma_k = torch.empty(w, device=DEV), torch.empty(w, device=DEV)

    def forward(self, S, offsets, positions):
        """offsets: where each sequence begins and the last one ends (all rows); positions: of each row in its sequence."""
        T = S.shape[0]
        self.S, self.offsets, self.positions = S, offsets, positions
        self.norm.fwd(S, self.gamma, self.beta, self.Y, mean=self.mean, rstd=self.rstd)
        torch.mm(self.Y, self.Wqkv, out=self.QKV.view(T, -1))
        q, k, v = self.QKV.split(self.parts, 1)
        self.rotary.fwd(q, k, positions, self.frequencies, self.Q, self.K, gamma_q=self.gamma_q, gamma_k=self.gamma_k)
        self.attention.fwd(self.Q, self.K, v, self.O, offsets, lse=self.lse)
        return self.O.view(T, -1) @ self.Wo

    def backward(self, dX, dS):
        """dX: gradient of what forward() returned; dS: of S by the other ways it goes.  Returns the gradient of S."""
        T = dX.shape[0]
        q, k, v = self.QKV.split(self.parts, 1)
        dq, dk, dv = self.dQKV.split(self.parts, 1)
        self.dWo = self.O.view(T, -1).T.contiguous() @ dX
        dO = (dX @ self.Wo.T).view_as(self.O)
        self.attention.bwd(dO, self.Q, self.K, v, self.O, self.lse, self.offsets, dq, dk, dv)
        self.rotary.bwd(dq, dk, self.positions, self.frequencies, dq, dk, Q=q, K=k, gamma_q=self.gamma_q, gamma_k=self.gamma_k, dgamma_q=self.dgamma_q,
                        dgamma_k=self.dgamma_k)
        self.dWqkv = self.Y.T.contiguous() @ self.dQKV.view(T, -1)
        self.norm.bwd(self.dQKV.view(T, -1) @ self.Wqkv.T, self.S, self.gamma, self.mean, self.rstd, self.dS, self.dgamma, self.dbeta, residual_grad=dS)
        return self.dS

    def update(self, lr):
        for p, g in ((self.Wqkv, self.dWqkv), (self.Wo, self.dWo), (self.gamma, self.dgamma), (self.beta, self.dbeta), (self.gamma_q, self.dgamma_q),
                     (self.gamma_k, self.dgamma_k)):
            p.sub_((lr * g).to(p.dtype))


def packed(T, seqs, g):
    """T rows as `seqs` sequences of random lengths: offsets, and each row's position in its own."""
    cuts = torch.randint(0, T + 1, (seqs - 1,), generator=g, device=DEV).sort().values
    offsets = torch.cat((cuts.new_zeros(1), cuts, cuts.new_full((1,), T)))
    rows = torch.arange(T, device=DEV)
    return offsets.int(), (rows - offsets[torch.searchsorted(offsets, rows, right=True) - 1]).int()


def train_both_halves(steps, T, d, h, E, heads, kv_heads, seqs=4, seed=0, lr=0.02, lr_vectors=0.05):
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    block, half = Block(T=T, d=d, h=h, E=E, seed=seed), AttentionHalf(T=T, d=d, heads=heads, kv_heads=kv_heads, seqs=seqs, seed=seed)
    target_map = torch.randn(d, d, generator=g, device=DEV) / math.sqrt(d)
    losses = []
    for _ in range(steps):
        R = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
        diff = block.forward(half.forward(R, *packed(T, seqs, g)), R).float() - torch.tanh(R.float() @ target_map)
        losses.append(float(diff.square().mean()))
        dX = block.backward((diff * (2.0 / T)).to(torch.bfloat16))
        half.backward(dX, dX)
        block.update(lr, lr_vectors)
        half.update(lr_vectors)
    return losses, block, half


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
    ap.add_argument("--heads", type=int, default=0)
    ap.add_argument("--kv-heads", type=int, default=0)
    a = ap.parse_args()
    sizes = (a.steps, a.tokens, a.width, a.hidden, a.experts)
    losses = train_both_halves(*sizes, a.heads, a.kv_heads or a.heads)[0] if a.heads else train(*sizes)[0]
    for i, loss in enumerate(losses):
        print(f"step {i}: loss {loss:.4f}", flush=True)
