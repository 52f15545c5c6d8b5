"""A residual block trained through the library, channel-last: two group norms with
SiLU, each before a 3x3 layer, and the sum with the block's input.

    y = x + conv(silu(norm(conv(silu(norm(x)), g1))), g2)

The forward pass keeps an 8-bit checkpoint of each norm's input and its statistics,
a quarter of what fp32 activations take; the backward pass forms the norms' gradients
and both weight gradients from them, and each layer's input gradient with the forward
layer on flipped filters.

    python examples/residual_block.py [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1903_01521_amd import binding as B  # noqa: E402

EPS = 1e-5
SILU = B.WINO_FLAG_SILU
ACT8 = B.WINO_FLAG_ACT8


class Layer:
    """A 3x3 layer [N][H][W][C] -> [N][H][W][K] of F(2x2,3x3), and its gradients."""

    def __init__(self, N, C, H, W, K):
        self.shape = N, C, H, W, K
        self.U = torch.empty(B.wino_filter_bytes(C, K, 2) // 4, device="cuda")
        self.Ub = torch.empty(B.wino_filter_bytes(K, C, 2) // 4, device="cuda")
        self.sizes = (B.wino_workspace_bytes_nhwc(N, C, H, W, K, 1, 2), B.wino_workspace_bytes_nhwc(N, K, H, W, C, 1, 2),
                      B.wino_conv2d_wgrad_workspace_bytes(N, C, H, W, K, 1, ACT8 | SILU))
        self.space = torch.empty(max(self.sizes) // 4 + 4, device="cuda")

    def forward(self, a, g, y):
        N, C, H, W, K = self.shape
        B.check(B.wino_filter_transform(g, self.U, C, K, 2), "filters")
        B.check(B.wino_conv2d_nhwc(a, self.U, y, N, C, H, W, K, 1, 2, 0, self.space, self.sizes[0]), "layer")

    def input_gradient(self, dy, g, da):
        N, C, H, W, K = self.shape
        flipped = g.flip(2, 3).transpose(0, 1).contiguous()
        B.check(B.wino_filter_transform(flipped, self.Ub, K, C, 2), "flipped filters")
        B.check(B.wino_conv2d_nhwc(dy, self.Ub, da, N, K, H, W, C, 1, 2, 0, self.space, self.sizes[1]), "input gradient")

    def weight_gradient(self, ckpt, norm, dy, dg):
        """dg of the layer whose input was norm's output, from the checkpoint of norm's input."""
        N, C, H, W, K = self.shape
        B.check(B.wino_conv2d_wgrad_nhwc(ckpt, dy, dg, norm.stats, norm.gamma, norm.beta, norm.G, N, C, H, W, K, 1,
                                         ACT8 | SILU, self.space, self.sizes[2]), "weight gradient")


class Norm:
    """Group norm with SiLU on [N][H][W][C]; keeps statistics and a checkpoint of its input."""

    def __init__(self, N, C, H, W, G):
        self.shape, self.G = (N, C, H, W, G), G
        self.gamma, self.beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
        self.dgamma, self.dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        self.stats = torch.empty((N, G, 2), device="cuda")
        self.ckpt = torch.empty(B.wino_act8_bytes(N, C, H, W), dtype=torch.int8, device="cuda")
        self.sizes = (B.wino_group_norm_workspace_bytes(N, C, H, W, G, SILU),
                      B.wino_group_norm_backward_workspace_bytes(N, C, H, W, G, SILU | ACT8))
        self.space = torch.empty(max(self.sizes) // 4 + 4, device="cuda")

    def forward(self, x, y):
        B.check(B.wino_group_norm_nhwc(x, self.gamma, self.beta, y, self.stats, self.ckpt, *self.shape, EPS, SILU,
                                       self.space, self.sizes[0]), "norm")

    def backward(self, dy, dx):
        B.check(B.wino_group_norm_backward_nhwc(dy, self.ckpt, self.stats, self.gamma, self.beta, dx, self.dgamma,
                                                self.dbeta, *self.shape, SILU | ACT8, self.space, self.sizes[1]),
                "norm's gradient")


class Block:
    def __init__(self, N, C, H, W, G, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.norms = [Norm(N, C, H, W, G) for _ in range(2)]
        self.layers = [Layer(N, C, H, W, C) for _ in range(2)]
        self.filters = [torch.randn((C, C, 3, 3), generator=gen, device="cuda") * (2.0 / (9 * C)) ** 0.5
                        for _ in range(2)]
        self.dfilters = [torch.empty_like(g) for g in self.filters]
        shape = (N, H, W, C)
        self.a, self.h, self.y, self.da, self.dh, self.dx = (torch.empty(shape, device="cuda") for _ in range(6))

    def forward(self, x):
        """y, kept in the block; of the activations only the checkpoints are needed later."""
        self.norms[0].forward(x, self.a)
        self.layers[0].forward(self.a, self.filters[0], self.h)
        self.norms[1].forward(self.h, self.a)
        self.layers[1].forward(self.a, self.filters[1], self.y)
        return self.y.add_(x)

    def backward(self, dy):
        """dx; the parameters' gradients go to dfilters and the norms' dgamma and dbeta."""
        self.layers[1].weight_gradient(self.norms[1].ckpt, self.norms[1], dy, self.dfilters[1])
        self.layers[1].input_gradient(dy, self.filters[1], self.da)
        self.norms[1].backward(self.da, self.dh)
        self.layers[0].weight_gradient(self.norms[0].ckpt, self.norms[0], self.dh, self.dfilters[0])
        self.layers[0].input_gradient(self.dh, self.filters[0], self.da)
        self.norms[0].backward(self.da, self.dx)
        return self.dx.add_(dy)

    def parameters(self):
        """(value, gradient) pairs."""
        pairs = list(zip(self.filters, self.dfilters))
        for n in self.norms:
            pairs += [(n.gamma, n.dgamma), (n.beta, n.dbeta)]
        return pairs


def train(steps=20, N=8, C=128, side=28, G=32, rate=0.05, seed=0):
    """Mean squared errors of `steps` steps towards a fixed random target block's output."""
    block, target = Block(N, C, side, side, G, seed), Block(N, C, side, side, G, seed + 1)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 2)
    x = torch.randn((N, side, side, C), generator=gen, device="cuda")
    want = target.forward(x).clone()
    losses = []
    for _ in range(steps):
        off = block.forward(x) - want
        losses.append(float(off.square().mean()))
        block.backward(off * (2.0 / off[0].numel()))
        for value, grad in block.parameters():
            value.sub_(grad, alpha=rate)
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=20)
    for i, loss in enumerate(train(parser.parse_args().steps)):
        print(f"step {i}: mean squared error {loss:.6f}", flush=True)
