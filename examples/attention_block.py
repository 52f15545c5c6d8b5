"""A block that attends to an encoder's states, trained through the library, channel-last:
the pixels' queries and the states' keys normalised and turned by their positions, cross
attention under the states' lengths, and a gated layer, each added to the block's input.

    h = x + attention(norm(x Wq), norm(e Wk), e Wv) Wo,   y = h + gated(h) Wd

Keys and values are views of one projection, and their gradients of one tensor, so the
projection's own backward pass takes it as it is.  The projections are matrix products of
the program's own.

    python examples/attention_block.py [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1903_01521_amd import binding as B  # noqa: E402

EPS = 1e-6
IO = {torch.float32: 0, torch.float16: B.WINO_IO_F16, torch.bfloat16: B.WINO_IO_BF16}


def table(rows, R):
    """(cos, sin) of each position and pair of channels, angles in 64 bits."""
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    return torch.stack((torch.cos(angle), torch.sin(angle)), -1).float().cuda()


class Block:
    """x [N][H][W][C], e [N][Lk][E] with klen [N] states of each image; heads of D channels."""

    def __init__(self, N, H, W, C, Lk, E, Hq, Hk, D, K, dtype=torch.float32, seed=0):
        self.shape = N, H, W, C, Lk, E, Hq, Hk, D, K
        L = self.L = H * W
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen, device="cuda") / shape[-1] ** 0.5).to(dtype)
        self.wq, self.wkv, self.wo = weight(Hq * D, C), weight(2 * Hk * D, E), weight(C, Hq * D)
        self.wgu, self.wd = weight(2, K, C), weight(C, K)
        self.gq, self.gk = torch.ones(D, device="cuda"), torch.ones(D, device="cuda")
        self.bias = torch.zeros((2, K), device="cuda")
        self.rot = table(max(L, Lk), D // 2 // 2 * 2)
        self.flags, self.act = IO[dtype], IO[dtype] | B.WINO_FLAG_SILU
        self.attn_size = N, L, Lk, Hq, Hk, D

        def empty(*shape):
            return torch.empty(shape, dtype=dtype, device="cuda")
        self.qn, self.kn, self.a = empty(N, L, Hq, D), empty(N, Lk, Hk, D), empty(N, L, Hq, D)
        self.dqn, self.dkn, self.dq = empty(N, L, Hq, D), empty(N, Lk, Hk, D), empty(N, L, Hq, D)
        self.dkv, self.u = empty(N, Lk, 2, Hk, D), empty(N, H, W, K)
        self.dh, self.dwgu, self.dbias = empty(N, H, W, C), empty(2, K, C), torch.empty_like(self.bias)
        self.dgq, self.dgk = torch.empty_like(self.gq), torch.empty_like(self.gk)
        self.lse = torch.empty((N, Hq, L), device="cuda")
        gated = N, C, H, W, K, self.act
        self.sizes = (B.wino_cross_attention_workspace_bytes(*self.attn_size, self.flags),
                      B.wino_gated_layer_workspace_bytes(*gated),
                      B.wino_gated_layer_backward_workspace_bytes(*gated),
                      B.wino_cross_attention_backward_workspace_bytes(*self.attn_size, self.flags),
                      B.wino_qk_norm_backward_workspace_bytes(*self.attn_size, self.flags))
        self.space = torch.empty(max(self.sizes) // 4 + 4, device="cuda")     # one call's at a time

    def _norm_sizes(self):
        N, H, W, C, Lk, E, Hq, Hk, D, K = self.shape
        return (*self.attn_size, 2 * self.rot.shape[1], self.rot.shape[0], Hq * D, 2 * Hk * D, EPS, self.flags)

    def _attn_sizes(self):
        N, H, W, C, Lk, E, Hq, Hk, D, K = self.shape
        return (*self.attn_size, Hq * D, Hk * D, 2 * Hk * D, D ** -0.5, self.flags)

    def forward(self, x, e, klen):
        N, H, W, C, Lk, E, Hq, Hk, D, K = self.shape
        self.x, self.e, self.klen = x, e, klen
        self.q = (x.view(-1, C) @ self.wq.t()).view(N, self.L, Hq, D)
        self.kv = (e.view(-1, E) @ self.wkv.t()).view(N, Lk, 2, Hk, D)
        B.check(B.wino_qk_norm_nhwc(self.q, self.kv[:, :, 0], self.gq, self.gk, self.rot, None, None, self.qn, self.kn,
                                    *self._norm_sizes()), "norm")
        B.check(B.wino_cross_attention_nhwc(self.qn, self.kn, self.kv[:, :, 1], klen, None, self.a, self.lse,
                                            *self._attn_sizes(), self.space, self.sizes[0]), "attention")
        self.h = torch.addmm(x.view(-1, C), self.a.view(-1, Hq * D), self.wo.t()).view(N, H, W, C)
        B.check(B.wino_gated_layer_nhwc(self.h, self.wgu, self.bias, self.u, N, C, H, W, K, self.act, self.space,
                                        self.sizes[1]), "gated layer")
        return torch.addmm(self.h.view(-1, C), self.u.view(-1, K), self.wd.t()).view(N, H, W, C)

    def backward(self, dy):
        """dx, de; the parameters' gradients are kept in the block."""
        N, H, W, C, Lk, E, Hq, Hk, D, K = self.shape
        dy2 = dy.view(-1, C)
        self.dwd = dy2.t() @ self.u.view(-1, K)
        du = (dy2 @ self.wd).view(N, H, W, K)
        B.check(B.wino_gated_layer_backward_nhwc(du, self.h, self.wgu, self.bias, self.dh, self.dwgu, self.dbias, N, C, H,
                                                 W, K, self.act, self.space, self.sizes[2]), "gated layer's gradient")
        dh = self.dh.add_(dy).view(-1, C)
        self.dwo = dh.t() @ self.a.view(-1, Hq * D)
        da = (dh @ self.wo).view(N, self.L, Hq, D)
        B.check(B.wino_cross_attention_backward_nhwc(da, self.qn, self.kn, self.kv[:, :, 1], self.a, self.lse, self.klen,
                                                     None, self.dqn, self.dkn, self.dkv[:, :, 1], *self._attn_sizes(),
                                                     self.space, self.sizes[3]), "attention's gradient")
        B.check(B.wino_qk_norm_backward_nhwc(self.dqn, self.dkn, self.q, self.kv[:, :, 0], self.gq, self.gk, self.rot,
                                             None, None, self.dq, self.dkv[:, :, 0], self.dgq, self.dgk,
                                             *self._norm_sizes(), self.space, self.sizes[4]), "norm's gradient")
        dq, dkv = self.dq.view(-1, Hq * D), self.dkv.view(-1, 2 * Hk * D)
        self.dwq, self.dwkv = dq.t() @ self.x.view(-1, C), dkv.t() @ self.e.view(-1, E)
        return torch.addmm(dh, dq, self.wq).view(N, H, W, C), (dkv @ self.wkv).view(N, Lk, E)

    def parameters(self):
        """(value, gradient) pairs, after backward()."""
        return [(self.wq, self.dwq), (self.wkv, self.dwkv), (self.wo, self.dwo), (self.wgu, self.dwgu), (self.wd, self.dwd),
                (self.gq, self.dgq), (self.gk, self.dgk), (self.bias, self.dbias)]


def train(steps=20, N=4, side=28, C=128, Lk=77, E=96, Hq=8, Hk=4, D=32, K=256, rate=0.02, seed=0):
    """Mean squared errors of `steps` steps towards a fixed random target block's output."""
    size = N, side, side, C, Lk, E, Hq, Hk, D, K
    block, target = Block(*size, seed=seed), Block(*size, seed=seed + 1)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 2)
    x = torch.randn((N, side, side, C), generator=gen, device="cuda")
    e = torch.randn((N, Lk, E), generator=gen, device="cuda")
    klen = torch.randint(1, Lk + 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
    want = target.forward(x, e, klen)
    losses = []
    for _ in range(steps):
        off = block.forward(x, e, klen) - want
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
