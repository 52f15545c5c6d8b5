"""The residual block of examples/ against autograd in 64 bits.

The block's gradients come from 8-bit checkpoints, whose values are off by at most
1/508 of a channel's range, about 7 standard deviations at these sizes: 0.8% of the
spread in the mean square.  That enters each norm's gradient and the weight gradients'
inputs once each: bounds of 5% of the gradients' norm, and of F(2x2,3x3)'s 1e-4 for the
forward pass, which the checkpoints do not touch."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "residual_block.py")


def _example():
    spec = importlib.util.spec_from_file_location("residual_block", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _reference(block, x, dy):
    """(y, dx, parameter gradients) on the CPU in 64 bits, in block.parameters()' order."""
    F = torch.nn.functional
    leaves = [v.detach().cpu().double().requires_grad_() for v, _ in block.parameters()]
    g1, g2, gamma1, beta1, gamma2, beta2 = leaves
    xr = x.cpu().double().requires_grad_()
    h = xr.permute(0, 3, 1, 2)
    G = block.norms[0].G
    a = F.conv2d(F.silu(F.group_norm(h, G, gamma1, beta1, 1e-5)), g1, padding=1)
    y = h + F.conv2d(F.silu(F.group_norm(a, G, gamma2, beta2, 1e-5)), g2, padding=1)
    y = y.permute(0, 2, 3, 1)
    (y * dy.cpu().double()).sum().backward()
    return y.detach(), xr.grad, [v.grad for v in leaves]


@pytest.mark.parametrize("N,C,side,G", [(2, 32, 14, 8), (3, 20, 9, 4), (1, 48, 57, 16)])
def test_gradients(N, C, side, G):
    ex = _example()
    block = ex.Block(N, C, side, side, G, seed=3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    for n in block.norms:
        n.gamma.add_(0.2 * torch.randn(C, generator=gen, device="cuda"))
        n.beta.add_(0.3 * torch.randn(C, generator=gen, device="cuda"))
    x = torch.randn((N, side, side, C), generator=gen, device="cuda")
    dy = torch.randn((N, side, side, C), generator=gen, device="cuda")
    y = block.forward(x).clone()
    dx = block.backward(dy).clone()
    ry, rdx, rgrads = _reference(block, x, dy)
    assert float((y.cpu().double() - ry).norm() / ry.norm()) < 1e-4
    assert float((dx.cpu().double() - rdx).norm() / rdx.norm()) < 0.05
    for (_, grad), ref in zip(block.parameters(), rgrads):
        assert float((grad.cpu().double() - ref).norm() / ref.norm()) < 0.05


def test_training_lowers_the_error():
    losses = _example().train(steps=12, N=2, C=32, side=14, G=8)
    assert losses[-1] < 0.7 * losses[0] and all(b < a for a, b in zip(losses, losses[1:]))
