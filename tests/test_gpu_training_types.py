"""The differentiable functions and the modules as a training program meets them: other
types than the parameters', other layouts, no gradients, no windows."""
import pytest
import torch

from paper_2506_08520_amd import binding as B
from paper_2506_08520_amd import training as T

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def randn(*shape, dtype=torch.float32, seed=0):
    g = torch.Generator().manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def make_block(dtype=torch.float32, p=0.1):
    torch.manual_seed(3)
    return T.DifferentialTransformerBlock(60, 3, 8, 4, p=p, dtype=dtype)


def test_block_converted_after_its_construction():
    """lam is formed in fp32 whatever type the parameters were moved to."""
    block = make_block().to(BF)
    assert block.attn.lam.dtype == BF
    a1, b1, a2, b2 = block.attn.lam.detach().double()
    want = torch.exp((a1 * b1).sum(-1)) - torch.exp((a2 * b2).sum(-1)) + block.attn.lam_init
    lam = block.attn.weights()
    # two exponentials of sums of 10 products, and their difference: 16 fp32 roundings of
    # terms below 4
    assert lam.dtype == torch.float32 and (lam - want).abs().max() <= 16 * 4 * 2.0 ** -24
    x = randn(1, 16, 16, 60, dtype=BF).requires_grad_()
    y = block(x, seed=5)
    y.backward(randn(1, 16, 16, 60, dtype=BF, seed=1))
    assert y.dtype == BF and torch.isfinite(y).all()
    for name, t in [("x", x), *block.named_parameters()]:
        assert t.grad is not None and t.grad.dtype == BF and torch.isfinite(t.grad).all(), name


def test_attention_takes_lam_in_any_type():
    q, k, v = (randn(2, h, 20, w, dtype=BF, seed=h) for h, w in ((4, 16), (4, 16), (2, 32)))
    do = randn(2, 2, 20, 32, dtype=BF, seed=9)
    lam = torch.tensor([0.3, 0.7], device="cuda").to(BF)
    outs = []
    for t in (lam, lam.float()):
        t = t.clone().requires_grad_()
        o = T.differential_attention(q, k, v, t)
        o.backward(do)
        outs.append((o, t.grad))
    assert torch.equal(outs[0][0], outs[1][0])
    assert outs[0][1].dtype == BF and torch.equal(outs[0][1], outs[1][1].to(BF))
