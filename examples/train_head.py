"""Trains a two-layer head, from the activations to the updated weights, with the
library's calls: a step is

    Z = X W1, A = gelu(Z)            shampoo_act_encode keeps X, Z and A in 8 bits
    logits = A W2                    shampoo_token_logprobs
    d logits                         shampoo_token_logprobs_grad (in place)
    G2 = A^T d logits                shampoo_act_weight_grad
    dA = d logits W2^T, dZ           shampoo_act_grad
    G1 = X^T dZ                      shampoo_act_weight_grad
    W1, W2                           shampoo_update_stats, _inv_root_batched, _precondition_graft

The three products with the weights are torch's.  Data are synthetic: classes
drawn from a fixed random linear map of the inputs, with a share of tokens that
carry no loss.

    python examples/train_head.py [--steps 30] [--tokens 4096] [--width 512] [--classes 1000]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2002_09018_amd import binding as B  # noqa: E402


class Head:
    """Weights, optimizer state and buffers of the head; step() runs one step."""

    def __init__(self, handle, dim, width, classes, tokens, device, eta0=0.02, refresh=5, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.h, self.eta0, self.refresh, self.t = handle, eta0, refresh, 0

        def weight(m, n):
            return torch.randn(m, n, generator=g, device=device) / m ** 0.5
        self.W = [weight(dim, width), weight(width, classes)]
        self.G = [torch.zeros_like(w) for w in self.W]
        blocks = []
        for w, grad in zip(self.W, self.G):
            m, n = w.shape
            eye = [torch.zeros(k, k, device=device) for k in (m, n, m, n)]
            blocks.append(B.Block(G=grad, W=w, D=torch.zeros_like(w), P=torch.zeros_like(w), L=eye[0], R=eye[1],
                                  Lr=eye[2], Rr=eye[3]))
        self.blocks = B.PackedBlocks(handle, blocks)
        stats = [s for b in blocks for s in (b.L, b.R)]
        roots = [s for b in blocks for s in (b.Lr, b.Rr)]
        self.jobs = B.PackedJobs(handle, stats, roots)
        self.params = B.shampoo_root_params_default(p=4, eps=1e-6, eps_relative=1)

        def byte_buffer(n):
            return torch.empty(n, device=device, dtype=torch.uint8) if n else None
        self.root_ws = byte_buffer(B.shampoo_inv_root_workspace_bytes([s.shape[0] for s in stats]))
        self.info = torch.zeros(8 * len(stats), device=device, dtype=torch.int32)
        self.keep = [byte_buffer(B.shampoo_act_checkpoint_bytes(tokens, n)) for n in (dim, width, width)]
        self.loss_ws = byte_buffer(B.shampoo_token_logprobs_workspace_bytes(tokens, classes))
        self.grad_ws = [byte_buffer(B.shampoo_act_weight_grad_workspace_bytes(tokens, *w.shape)) for w in self.W]
        self.logp, self.lse, self.entropy = (torch.zeros(tokens, device=device) for _ in range(3))

    def step(self, X, targets):
        """One step over X (tokens x dim, bf16) and targets (int32, -1: no
        loss); returns the mean loss before the update, on the device."""
        h, (kx, kz, ka) = self.h, self.keep
        w1, w2 = (w.bfloat16() for w in self.W)
        # forward: what the backward pass needs is kept in the checkpoints
        B.shampoo_act_encode(h, X, ckpt_x=kx)
        Z = X @ w1
        B.shampoo_act_encode(h, Z, ckpt_x=kz, act=B.ACT_GELU, Y=Z, ckpt_y=ka)  # Z is A from here on
        logits = Z @ w2
        B.shampoo_token_logprobs(h, logits, targets, self.logp, self.lse, entropy=self.entropy,
                                 workspace=self.loss_ws)
        count = (targets >= 0).sum().clamp(min=1)
        loss = -self.logp.sum() / count
        # backward
        g_logp = (-1.0 / count).expand(X.shape[0]).contiguous()
        B.shampoo_token_logprobs_grad(h, logits, targets, self.lse, logits, g_logp=g_logp)
        B.shampoo_act_weight_grad(h, ka, logits, self.G[1], workspace=self.grad_ws[1])
        dA = logits @ w2.t()
        B.shampoo_act_grad(h, kz, B.ACT_GELU, dA, dA)
        B.shampoo_act_weight_grad(h, kx, dA, self.G[0], workspace=self.grad_ws[0])
        # update
        B.shampoo_update_stats(h, self.blocks, 0.99)
        if self.t % self.refresh == 0:
            B.shampoo_inv_root_batched(h, self.jobs, None, self.params, self.root_ws, self.info)
        B.shampoo_precondition_graft(h, self.blocks, self.eta0)
        self.t += 1
        return loss


def data(tokens, dim, classes, device, seed):
    """Inputs and targets: the largest of `classes` fixed random projections, a
    tenth of the tokens without a target."""
    rule = torch.randn(dim, classes, generator=torch.Generator(device=device).manual_seed(99), device=device)
    g = torch.Generator(device=device).manual_seed(seed)
    X = torch.randn(tokens, dim, generator=g, device=device).bfloat16()
    t = (X.float() @ rule).argmax(1).to(torch.int32)
    t[torch.rand(tokens, generator=g, device=device) < 0.1] = -1
    return X, t


def main():
    p = argparse.ArgumentParser()
    for name, default in (("steps", 30), ("tokens", 4096), ("dim", 256), ("width", 512), ("classes", 1000)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    device = torch.device("cuda:0")
    handle = B.shampoo_create(0)
    head = Head(handle, a.dim, a.width, a.classes, a.tokens, device)
    batches = [data(a.tokens, a.dim, a.classes, device, s) for s in range(4)]
    held = sum(k.numel() for k in head.keep)
    full = 2 * a.tokens * (a.dim + 2 * a.width)
    print(f"activations kept: {held} bytes in 8 bits, {full} in bf16")
    for t in range(a.steps):
        loss = head.step(*batches[t % len(batches)])
        if t % 5 == 0 or t == a.steps - 1:
            print(f"step {t}: loss {float(loss):.4f}, entropy {float(head.entropy.mean()):.4f}", flush=True)
    B.shampoo_destroy(handle)


if __name__ == "__main__":
    main()
