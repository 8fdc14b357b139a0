"""Trains the routing part of one block on synthetic data: the layer norm in front of it, the gate matrix and the gate bias.

The experts are frozen.  A hidden router of the same form (its own norm and gate) says which experts make the target of a token;
the step learns to find them:

  norm -> gate -> dispatch -> experts -> combine          scmoe_layer_norm, _gate_topk, _dispatch, _expert_ffn, _combine
  mean squared error and balance loss                     scmoe_balance_loss
  combine -> experts -> gate, dispatch -> norm, backwards scmoe_combine_backward, _gate_backward, _layer_norm_backward

The gradient through the frozen experts is the only step in torch (the library has the forward pass of the experts alone).
`python -m paper_2404_05019_amd.train_routing --steps 200` prints the losses and how often router and hidden router agree.
"""
import argparse

import torch

from . import binding as B

DEV = "cuda:0"
EPS = 1e-5


class RoutingBlock:
    """Norm, gate and frozen experts of one block, with the buffers of a step of T tokens."""

    def __init__(self, T, d, F, E, k, capacity_factor=2.0, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        normal = lambda *s, scale=1.0: torch.randn(s, generator=g, device=DEV) * scale  # noqa: E731
        self.T, self.d, self.F, self.E, self.k, self.dtype = T, d, F, E, k, dtype
        # one expert's weight is its probability: as a softmax over the chosen one alone it would be 1, and the gate would not learn
        self.normalize = int(k > 1)
        self.capacity = B.scmoe_capacity(T, E, k, capacity_factor)
        self.W1, self.W2 = normal(E, F, d, scale=d ** -0.5).to(dtype), normal(E, d, F, scale=F ** -0.5).to(dtype)
        self.gamma, self.beta = torch.ones(d, device=DEV), torch.zeros(d, device=DEV)
        self.W_g, self.bias = normal(d, E, scale=0.02), torch.zeros(E, device=DEV)
        rows = min(T * k, E * self.capacity)
        acts = lambda n, w=d: torch.empty(n, w, dtype=dtype, device=DEV)  # noqa: E731
        f32 = lambda *s: torch.empty(s, device=DEV)  # noqa: E731
        i32 = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)  # noqa: E731
        self.h, self.y, self.dh, self.dx = acts(T), acts(T), acts(T), acts(T)
        self.x_perm, self.y_perm, self.dx_perm, self.dy_perm, self.hidden = acts(rows), acts(rows), acts(rows), acts(rows), acts(rows, F)
        self.mean, self.rstd, self.gate_w, self.probs, self.dgate_w = f32(T), f32(T), f32(T, k), f32(T, E), f32(T, k)
        self.idx, self.dst_row, self.src_token = i32(T, k), i32(T, k), i32(rows)
        self.counts, self.offsets, self.load = i32(E), i32(E + 1), i32(E)
        self.mean_prob, self.slope, self.balance = f32(E), f32(E), f32(1)
        self.grads = [f32(d), f32(d), f32(d, E), f32(E)]          # gamma, beta, W_g, bias
        need = max(B.scmoe_layer_norm_backward_workspace_bytes(T, d), B.scmoe_gate_backward_workspace_bytes(T, d, E),
                   B.scmoe_balance_loss_workspace_bytes(T, E), B.scmoe_dispatch_workspace_bytes(T, E, k),
                   B.scmoe_expert_ffn_workspace_bytes(B.dtype_code(self.h), d, F))
        self.scratch = torch.empty(need, dtype=torch.uint8, device=DEV)   # one for all: the calls follow each other on one stream

    def parameters(self):
        return [self.gamma, self.beta, self.W_g, self.bias]

    def forward(self, x):
        """The block's output for x [T, d]; what the backward pass needs stays in the buffers."""
        self.loss_slope = None                                    # (of this pass: there is none until the loss was asked for)
        B.scmoe_layer_norm(x, self.gamma, self.beta, EPS, self.h, mean=self.mean, rstd=self.rstd)
        B.scmoe_gate_topk(self.h, self.W_g, self.bias, self.k, self.idx, self.gate_w, self.probs, normalize=self.normalize)
        B.scmoe_dispatch(self.h, self.idx, self.E, self.k, self.capacity, self.counts, self.offsets, self.dst_row, self.src_token, self.x_perm,
                         self.scratch)
        B.scmoe_expert_ffn(self.x_perm, self.offsets, self.x_perm.shape[0], self.W1, None, self.W2, None, self.hidden, self.y_perm,
                           workspace=self.scratch)
        B.scmoe_combine(self.y_perm, self.dst_row, self.gate_w, self.k, None, None, None, self.y)
        return self.y

    def balance_loss(self, coef, mask=None):
        """The loss, on the device; its slope in the probabilities stays for the backward pass."""
        B.scmoe_balance_loss(self.probs, self.idx, self.k, coef, self.load, self.mean_prob, self.slope, self.balance, self.scratch, mask=mask)
        self.loss_slope = self.slope
        return self.balance

    def _experts_backward(self):
        """Gradient of the packed rows through the frozen experts."""
        ends = self.offsets.tolist()
        for e in range(self.E):
            at = slice(ends[e], ends[e + 1])
            if ends[e + 1] > ends[e]:
                x = self.x_perm[at].float().requires_grad_(True)
                y = torch.nn.functional.gelu(x @ self.W1[e].float().t()) @ self.W2[e].float().t()
                self.dx_perm[at] = torch.autograd.grad(y, x, self.dy_perm[at].float())[0].to(self.dtype)

    def backward(self, x, dy, mask=None):
        """Gradients of the parameters (in `grads`) and of x from the gradient dy of the output, with the balance loss's if it was asked for
        since the forward pass."""
        B.scmoe_combine_backward(dy, self.y_perm, self.dst_row, self.gate_w, self.k, dy_perm=self.dy_perm, dgate_w=self.dgate_w)
        self._experts_backward()
        B.scmoe_gate_backward(self.h, self.W_g, self.probs, self.idx, self.gate_w, self.dgate_w, self.dh, self.grads[2], self.grads[3],
                              self.scratch, k=self.k, normalize=self.normalize, slope=self.loss_slope, mask=mask, dx_perm=self.dx_perm, dst_row=self.dst_row)
        B.scmoe_layer_norm_backward(self.dh, x, self.gamma, self.mean, self.rstd, self.dx, self.grads[0], self.grads[1], self.scratch)
        return self.dx


def train(steps=200, T=2048, d=256, F=512, E=8, k=2, lr=3e-3, coef=0.01, dtype=torch.bfloat16, seed=0, report=None):
    """The mean squared errors of the steps, and the share of chosen experts that are the hidden router's, first and last."""
    block = RoutingBlock(T, d, F, E, k, dtype=dtype, seed=seed)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    hidden = RoutingBlock(T, d, F, E, k, dtype=dtype, seed=seed)          # the same experts
    hidden.W_g.copy_(torch.randn(d, E, generator=g, device=DEV) * d ** -0.5)
    hidden.gamma.copy_(1.0 + 0.3 * torch.randn(d, generator=g, device=DEV))
    optimizer = torch.optim.Adam(block.parameters(), lr=lr)
    errors, agree = [], []
    for step in range(steps):
        x = torch.randn(T, d, generator=g, device=DEV).to(dtype)
        target = hidden.forward(x).float()
        out = block.forward(x).float() - target
        balance = block.balance_loss(coef)
        dy = (out * (2.0 / out.numel())).to(dtype)
        block.backward(x, dy)
        for p, grad in zip(block.parameters(), block.grads):
            p.grad = grad
        optimizer.step()
        errors.append(out.square().mean())
        agree.append((block.idx[:, :, None] == hidden.idx[:, None, :]).any(2).float().mean())
        if report and (step % 20 == 0 or step == steps - 1):
            report("step %4d  error %.5f  balance loss %.5f  chosen alike %.3f  most loaded expert %.2f of an even share"
                   % (step, errors[-1], balance, agree[-1], block.load.max().item() * E / (k * T)))
    return [float(e) for e in errors], float(agree[0]), float(agree[-1])


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--f32", action="store_true")
    a = ap.parse_args()
    train(a.steps, a.tokens, a.width, 2 * a.width, a.experts, dtype=torch.float32 if a.f32 else torch.bfloat16, report=lambda s: print(s, flush=True))


if __name__ == "__main__":
    main()
