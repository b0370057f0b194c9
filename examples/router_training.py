"""Training one MoE layer's router with the balance loss alone.

Each step projects the tokens (eqb_router_logits), routes them
(eqb_route_topk), takes the balance loss, the z-loss and their gradient per
microbatch (eqb_balance_loss, the gradient in bf16), takes that gradient back
to the router's weight and input (eqb_router_grad, accumulated over the
microbatches of the step), and updates the fp32 master weight and the bf16 copy
that the projection reads (EqbAdamW).

In a model the experts' path gives a gradient too, and dx is added to the gradient
of the layer's input.  The score gradients are dL/ds, s = sigmoid(z), and LEI
(lei_inject_grad) adds to dL/ds; the balance loss adds to dL/dz.  So they are taken
through the sigmoid, dL/dz = dL/ds s (1 - s), before they become grad_in: step()
does so with the grad_s that it is given.  main() trains on the loss alone, with
grad_in zero, and dx is only formed.

The tokens have a common component, as hidden states do, so a random router
sends most of them to a few experts; the loss spreads them.

    python examples/router_training.py [--steps N] [--state-bits 8|32]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_28053_gb300 as eqb  # noqa: E402


class RouterTrainer:
    """One router W_r [E, d] with its optimizer and the buffers of a step of
    `accumulate` passes over T tokens in M microbatches each."""

    def __init__(self, T, d, E, K, M, accumulate=2, alpha=0.02, zeta=1e-4, lr=2e-3, state_bits=32, seed=0, eta=0.0, c=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.d, self.E, self.K, self.M, self.accumulate = T, d, E, K, M, accumulate
        self.alpha, self.zeta, self.lr, self.eta, self.c = alpha, zeta, lr, eta, c
        self.master = torch.randn(E, d, generator=g, device="cuda") * d ** -0.5
        self.W_r = self.master.bfloat16()
        self.opt = eqb.EqbAdamW([self.master], state_bits=state_bits, copies=[self.W_r])
        self.bias = torch.zeros(E, device="cuda")
        self.offsets = torch.arange(M + 1, device="cuda") * T // M
        self.idx = torch.empty(T, K, dtype=torch.int32, device="cuda")
        self.z = torch.empty(T, E, dtype=torch.bfloat16, device="cuda")
        self.dz = torch.empty(T, E, dtype=torch.bfloat16, device="cuda")
        self.dx = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        self.dW = torch.empty(E, d, device="cuda")
        self.grad_in = torch.zeros(T, E, device="cuda")
        # the losses of the step's microbatches are averaged
        self.scale = torch.full((1,), 1.0 / (accumulate * M), device="cuda")
        self.tau = torch.empty(T, device="cuda")
        self.loads = torch.empty(M, E, dtype=torch.int32, device="cuda")
        self.counts = torch.empty(M, E, dtype=torch.int32, device="cuda")
        self.loss = torch.empty(M, 2, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws_loss = torch.empty(eqb.eqb_balance_loss_workspace_bytes(T, E, M), dtype=torch.uint8, device="cuda")
        self.ws_grad = torch.empty(eqb.eqb_router_grad_workspace_bytes(T, d, E), dtype=torch.uint8, device="cuda")
        self.steps = 0

    def step(self, batches, grad_s=None):
        """One optimizer step over `accumulate` batches x [T, d]; the mean
        balance loss and the last batch's [Global, Local] MaxVio, on the device.
        grad_s: the experts' path's dL/ds of every batch, fp32 [T, E], which LEI
        is added to (in place) with eta."""
        total = 0.0
        for i, x in enumerate(batches):
            eqb.eqb_router_logits(x, self.W_r, z=self.z, err_flag=self.err)
            self.loads.zero_()
            eqb.eqb_route_topk(self.z, self.bias, self.K, self.offsets, topk_idx=self.idx, tau=self.tau, loads=self.loads,
                               err_flag=self.err)
            if grad_s is not None:
                eqb.lei_inject_grad(grad_s[i], self.loads, self.offsets, self.K, self.eta, self.c)
                zf = self.z.float()
                torch.mul(grad_s[i], torch.sigmoid(zf) * torch.sigmoid(-zf), out=self.grad_in)  # dL/ds -> dL/dz
            eqb.eqb_balance_loss(self.z, self.idx, self.offsets, self.alpha, zeta=self.zeta, grad_in=self.grad_in,
                                 grad_out=self.dz, grad_scale=self.scale, counts=self.counts, loss=self.loss,
                                 workspace=self.ws_loss, err_flag=self.err)
            eqb.eqb_router_grad(self.dz, x, self.W_r, dx=self.dx, dW=self.dW, accumulate_dW=i > 0, workspace=self.ws_grad,
                                err_flag=self.err)
            total = total + self.loss[:, 0].mean()
        self.steps += 1
        self.opt.step([self.dW], lr=self.lr, step=self.steps, weight_decay=0.0, err_flag=self.err)
        return total / len(batches), eqb.eqb_maxvio(self.counts, self.offsets, self.K)


def tokens(T, d, seed):
    """x [T, d]: noise on a component that all tokens share."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    common = torch.randn(d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    return (torch.randn(T, d, generator=g, device="cuda") + 0.7 * common).bfloat16()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    ap.add_argument("--tokens", type=int, default=16384)
    a = ap.parse_args(argv)
    t = RouterTrainer(a.tokens, 1024, 64, 8, 4, state_bits=a.state_bits)
    for s in range(a.steps):
        loss, vio = t.step([tokens(t.T, t.d, 100 + 2 * s + i) for i in range(t.accumulate)])
        if s % 10 == 0 or s == a.steps - 1:
            print(f"step {s:4d}  balance loss {loss.item():.6f}  MaxVio global {vio[0].item():.3f} local {vio[1].item():.3f}")
    if t.err.item():
        raise eqb.EqbError(t.err.item(), "router training")


if __name__ == "__main__":
    main()
