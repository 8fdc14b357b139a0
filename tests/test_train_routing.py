"""The example that trains a block's routing: its gradients against those of the same block in 64 bits, differentiated by torch."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2404_05019_amd.train_routing import EPS, RoutingBlock
    from gpu_util import DEV

COEF = 0.3


def inputs(block, seed=3):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return [torch.randn(block.T, block.d, generator=g, device=DEV).to(block.dtype) for _ in range(2)]


def exact(block, x, dy, coef):
    """Output and gradients of gamma, beta, W_g and bias for the choices and the kept items of the block's last forward pass: one
    expert a token is weighted by its probability, several by a softmax over their logits."""
    leaves = [p.detach().double().requires_grad_(True) for p in block.parameters()]
    gamma, beta, W_g, bias = leaves
    h = torch.nn.functional.layer_norm(x.double(), (block.d,), gamma, beta, EPS)
    logits = h @ W_g + bias
    probs, at = torch.softmax(logits, 1), block.idx.long()
    weight = probs.gather(1, at) if block.k == 1 else torch.softmax(logits.gather(1, at), 1)
    weight = weight * (block.dst_row >= 0)
    y = torch.zeros_like(h)
    for e in range(block.E):
        out = torch.nn.functional.gelu(h @ block.W1[e].double().t()) @ block.W2[e].double().t()
        y = y + (weight * (at == e)).sum(1, keepdim=True) * out
    share = torch.bincount(at.reshape(-1), minlength=block.E).double() / at.numel()
    value = (y * dy.double()).sum() + coef * block.E * (share * probs.mean(0)).sum()
    return y.detach(), torch.autograd.grad(value, leaves)


def close(got, want):
    """fp32: a few hundred roundings of 2^-24 each on the way through two expert products and sums over 256 tokens, 3e-5 of the largest
    value; 1e-3 of it is asked."""
    assert float((got.double() - want).abs().max()) <= 1e-3 * float(want.abs().max())


@pytest.mark.parametrize("k", [1, 2, 3])
def test_gradients_of_the_block(k):
    block = RoutingBlock(256, 64, 128, 4, k, dtype=torch.float32)
    x, dy = inputs(block)
    y = block.forward(x)
    block.balance_loss(COEF)
    block.backward(x, dy)
    wy, grads = exact(block, x, dy, COEF)
    close(y, wy)
    for got, want in zip(block.grads, grads):
        close(got, want)


def test_a_pass_without_the_balance_loss():
    """Nothing of what the memory held before, nor of an earlier pass's loss, is in the gradients."""
    held = [torch.full((n,), float("nan"), device=DEV) for n in (4, 64, 256, 1 << 20) for _ in range(8)]
    torch.cuda.synchronize()
    del held
    block = RoutingBlock(256, 64, 128, 4, 2, dtype=torch.float32)
    x, dy = inputs(block)
    for _ in range(2):
        y = block.forward(x)
        block.backward(x, dy)
        wy, grads = exact(block, x, dy, 0.0)
        close(y, wy)
        for got, want in zip(block.grads, grads):
            close(got, want)
        block.balance_loss(1000.0)                # (of this pass; the next one does not ask for it)
