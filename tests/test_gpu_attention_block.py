"""The attention block of examples/, forward and backward, against autograd in 64 bits, on
the weights and inputs as they are rounded.

fp32: sums of at most 300 products (300 * 2^-24) and operands split to 2^-20 in eight
products in turn: 1e-4 of the norm.  bf16: some twelve tensors on the way are rounded to
2^-9 of a value each, 2^-8 at worst, P and dS among them: 12 * 2^-8 = 4.7%, held to 5%."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")


def _example():
    spec = importlib.util.spec_from_file_location("attention_block", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _turned(x, rot):
    """The first R channels of x [N][L][heads][D] turned, token t by row t."""
    half = rot.shape[1]
    c, s = rot[:x.shape[1], None, :, 0], rot[:x.shape[1], None, :, 1]
    a, b = x[..., :half], x[..., half:2 * half]
    return torch.cat((a * c - b * s, b * c + a * s, x[..., 2 * half:]), -1)


def _reference(block, x, e, klen, dy):
    """y, dx, de and the gradients in block.parameters()' order, on the CPU in 64 bits."""
    N, H, W, C, Lk, E, Hq, Hk, D, K = block.shape
    leaves = [v.detach().cpu().double().requires_grad_() for v, _ in block.parameters()]
    wq, wkv, wo, wgu, wd, gq, gk, bias = leaves
    xr, er = x.cpu().double().requires_grad_(), e.cpu().double().requires_grad_()
    rot = block.rot.cpu().double()

    def norm(t, g):
        return _turned(t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6) * g, rot)
    x2 = xr.view(-1, C)
    q = norm((x2 @ wq.t()).view(N, H * W, Hq, D), gq)
    kv = (er.view(-1, E) @ wkv.t()).view(N, Lk, 2, Hk, D)
    k, v = (t.repeat_interleave(Hq // Hk, 2).permute(0, 2, 1, 3) for t in (norm(kv[:, :, 0], gk), kv[:, :, 1]))
    s = (q.permute(0, 2, 1, 3) @ k.transpose(2, 3)) * D ** -0.5
    kept = (torch.arange(Lk) < klen.cpu()[:, None])[:, None, None]
    p = torch.softmax(s.masked_fill(~kept, -1e300), -1) * kept
    a = (p @ v).permute(0, 2, 1, 3).reshape(-1, Hq * D)
    h = x2 + a @ wo.t()
    u = torch.nn.functional.silu(h @ wgu[0].t() + bias[0]) * (h @ wgu[1].t() + bias[1])
    y = (h + u @ wd.t()).view(N, H, W, C)
    (y * dy.cpu().double()).sum().backward()
    return [y.detach(), xr.grad, er.grad] + [v.grad for v in leaves]


@pytest.mark.parametrize("dtype,bound", [(torch.float32, 1e-4), (torch.bfloat16, 0.05)])
@pytest.mark.parametrize("size", [(2, 9, 11, 48, 37, 40, 4, 2, 32, 72), (3, 14, 14, 64, 130, 24, 2, 2, 40, 96),
                                  (2, 1, 1, 32, 300, 16, 8, 1, 64, 40)])
def test_forward_and_gradients(size, dtype, bound):
    block = _example().Block(*size, dtype=dtype, seed=5)
    N, H, W, C, Lk, E = size[:6]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    for g in (block.gq, block.gk):
        g.add_(0.2 * randn(*g.shape))
    block.bias.add_(0.3 * randn(*block.bias.shape))
    x, e, dy = randn(N, H, W, C).to(dtype), randn(N, Lk, E).to(dtype), randn(N, H, W, C).to(dtype)
    klen = torch.tensor([Lk, 0, Lk // 2][:N], dtype=torch.int32, device="cuda")     # an image without states
    y = block.forward(x, e, klen)
    dx, de = block.backward(dy)
    got = [y, dx, de] + [g for _, g in block.parameters()]
    for name, g, r in zip("y dx de wq wkv wo wgu wd gq gk bias".split(), got, _reference(block, x, e, klen, dy)):
        assert float((g.cpu().double() - r).norm()) <= bound * float(r.norm()), name
    assert bool((de[1] == 0).all())


def test_training_runs():
    losses = _example().train(steps=3, N=2, side=7, C=32, Lk=20, E=16, Hq=2, Hk=1, D=16, K=48)
    assert all(x == x and x < float("inf") for x in losses)
