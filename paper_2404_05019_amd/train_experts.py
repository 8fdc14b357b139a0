"""Trains one whole block on synthetic data: norm, gate and gated experts, the experts' activations kept in 8 bits if wanted.

  norm -> gate -> dispatch -> gated experts -> combine     scmoe_layer_norm, _gate_topk, _dispatch, _gated_ffn, _combine
  backwards, all of it in the library                      scmoe_combine_backward, _gated_ffn_backward, _gate_backward, _layer_norm_backward

A hidden block of the same form makes the targets.  With keep="8bit" what stays of a step for its backward pass is the experts' input rows
(scmoe_checkpoint_pack) and their pre-activations (written so by scmoe_gated_ffn) at a little over a byte a value.
`python -m paper_2404_05019_amd.train_experts --steps 200 --keep 8bit` prints the losses and the bytes that are kept.
"""
import argparse

import torch

from . import binding as B
from .train_routing import DEV, EPS, RoutingBlock


class GatedBlock(RoutingBlock):
    """Norm, gate and gated experts of one block.  act: B.SILU, B.GELU_ERF or B.GELU_TANH; keep: "full" or "8bit"."""

    def __init__(self, T, d, F, E, k, capacity_factor=2.0, dtype=torch.bfloat16, seed=0, act=B.SILU, keep="full"):
        super().__init__(T, d, F, E, k, capacity_factor, dtype, seed)
        g = torch.Generator(device=DEV)
        g.manual_seed(seed + 1000)
        self.act, self.keep = act, keep
        self.W1 = (torch.randn(E, 2 * F, d, generator=g, device=DEV) * d ** -0.5).to(dtype)
        rows = self.x_perm.shape[0]
        eight = lambda n, w: torch.empty(n, B.scmoe_checkpoint_ld(w), dtype=torch.uint8, device=DEV)  # noqa: E731
        if keep == "8bit":
            self.pre, self.x_kept = eight(2 * rows, F), eight(rows, d)
        else:
            self.pre, self.x_kept = torch.empty(rows, 2 * F, dtype=dtype, device=DEV), self.x_perm
        self.expert_grads = [torch.empty_like(self.W1), torch.empty_like(self.W2)]
        code = B.dtype_code(self.x_perm)
        need = max(self.scratch.numel(), B.scmoe_gated_ffn_workspace_bytes(code, d, F), B.scmoe_gated_ffn_backward_workspace_bytes(code, rows, E, d, F))
        self.scratch = torch.empty(need, dtype=torch.uint8, device=DEV)

    def kept_bytes(self):
        """What stays of the experts' activations from the forward pass to the backward pass."""
        return self.pre.nbytes + self.x_kept.nbytes

    def forward(self, x):
        self.loss_slope = None
        B.scmoe_layer_norm(x, self.gamma, self.beta, EPS, self.h, mean=self.mean, rstd=self.rstd)
        B.scmoe_gate_topk(self.h, self.W_g, self.bias, self.k, self.idx, self.gate_w, self.probs, normalize=self.normalize)
        B.scmoe_dispatch(self.h, self.idx, self.E, self.k, self.capacity, self.counts, self.offsets, self.dst_row, self.src_token, self.x_perm,
                         self.scratch)
        B.scmoe_gated_ffn(self.x_perm, self.offsets, self.x_perm.shape[0], self.W1, self.W2, self.hidden, self.y_perm, self.act, pre=self.pre,
                          workspace=self.scratch)
        if self.keep == "8bit":
            B.scmoe_checkpoint_pack(self.x_perm, self.x_kept, n_rows=self.offsets[-1:])
        B.scmoe_combine(self.y_perm, self.dst_row, self.gate_w, self.k, None, None, None, self.y)
        return self.y

    def _experts_backward(self):
        """Gradients of the packed rows (dx_perm) and of the experts' weights (expert_grads)."""
        B.scmoe_gated_ffn_backward(self.dy_perm, self.x_kept, self.pre, self.offsets, self.dy_perm.shape[0], self.W1, self.W2, self.act,
                                   self.dx_perm, *self.expert_grads, workspace=self.scratch)


def train(steps=200, T=2048, d=256, F=512, E=8, k=2, lr=2e-3, coef=0.01, dtype=torch.bfloat16, seed=0, act=B.SILU, keep="8bit", report=None):
    """The mean squared errors of the steps.  The optimizer holds the experts' weights in 32 bits."""
    block = GatedBlock(T, d, F, E, k, dtype=dtype, seed=seed, act=act, keep=keep)
    hidden = GatedBlock(T, d, F, E, k, dtype=dtype, seed=seed + 7, act=act)
    hidden.W_g.copy_(block.W_g)                                   # the same router: the experts are what is learnt
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    experts = [block.W1.float(), block.W2.float()]
    optimizer = torch.optim.Adam(block.parameters() + experts, lr=lr)
    errors = []
    for step in range(steps):
        x = torch.randn(T, d, generator=g, device=DEV).to(dtype)
        target = hidden.forward(x).float()
        out = block.forward(x).float() - target
        block.balance_loss(coef)
        block.backward(x, (out * (2.0 / out.numel())).to(dtype))
        for p, grad in zip(block.parameters() + experts, block.grads + block.expert_grads):
            p.grad = grad.float()
        optimizer.step()
        block.W1.copy_(experts[0])
        block.W2.copy_(experts[1])
        errors.append(out.square().mean())
        if report and (step % 20 == 0 or step == steps - 1):
            report("step %4d  error %.5f  kept for the backward pass %.1f MB" % (step, errors[-1], block.kept_bytes() / 2 ** 20))
    return [float(e) for e in errors]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--keep", choices=("full", "8bit"), default="8bit")
    ap.add_argument("--f32", action="store_true")
    a = ap.parse_args()
    train(a.steps, a.tokens, a.width, 2 * a.width, a.experts, dtype=torch.float32 if a.f32 else torch.bfloat16, keep=a.keep, report=lambda s: print(s, flush=True))


if __name__ == "__main__":
    main()
