"""The gated layer on tiles of every shape, whole and in parts, straight to LDS and not: whole numbers
small enough that every sum is exact, so that a result differs only where a value was taken
from elsewhere; SiLU on real values within its bounds; the limits of 32-bit offsets."""
import math

import pytest
import torch

from block_helpers import ACT, DEV, DTYPE, IO, B, gated, gated_back
from gated_sizes import ODD, SIZES, WIDE, plan
from test_gpu_gated_layer import check, check_back, make

pytestmark = pytest.mark.gpu


def numbers(gen, nonzero, *shape):
    """-1, 0 and 1."""
    r = torch.rand(shape, generator=gen, device=DEV)
    return (r < nonzero / 2).float() - (r > 1 - nonzero / 2).float()


def exact(M, C, K, dtype, act, offset=0, bias=True, seed=95):
    """Inputs in whole numbers, and y, dx, dw, dbias of them: |zg| and |zu| are below 32, so that dz
    has no more than bfloat16's eight bits, and sums stay below 2^24, in fp32 products too."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    x, w, dy = numbers(gen, min(1.0, 16 / C), M, C), numbers(gen, 0.5, 2, K, C), numbers(gen, 0.5, M, K)
    b = torch.randint(-2, 3, (2, K), generator=gen, device=DEV).float() if bias else torch.zeros((2, K), device=DEV)
    zg, zu = x @ w[0].t() + b[0], x @ w[1].t() + b[1]
    v, d = (zg.clamp(min=0), (zg > 0).float()) if act == "relu" else (zg, torch.ones_like(zg))
    dz = dy * zu * d, dy * v
    assert max(float(t.abs().max()) for t in dz) <= 256
    want = (v * zu, dz[0] @ w[0] + dz[1] @ w[1], torch.stack([t.t() @ x for t in dz]), torch.stack([t.sum(0) for t in dz]))
    assert max(float(t.abs().max()) for t in want) < 2 ** 24

    bounds = []

    def put(a):
        return torch.empty(a.numel() + offset, dtype=DTYPE[dtype], device=DEV)[offset:].view(a.shape).copy_(a)

    def empty(*shape, t=DTYPE[dtype], offset=offset):
        n = math.prod(shape)
        buf = torch.full((n + offset + 64,), 7.0, dtype=t, device=DEV)
        buf[offset:offset + n] = float("nan")
        bounds.append((buf[:offset], buf[offset + n:]))
        return buf[offset:offset + n].view(shape)
    flags = IO[dtype] | ACT[act]
    xt, wt, dyt, bt = put(x), put(w), put(dy), b if bias else None
    y, dx, dw, db = empty(M, K), empty(M, C), empty(2, K, C), empty(2, K, t=torch.float32, offset=0)
    size = (1, C, 1, M, K, flags)
    B.check(B.wino_gated_layer_nhwc(xt, wt, bt, y, *size))
    need = B.wino_gated_layer_backward_workspace_bytes(*size)
    ws = torch.full((need // 4 + 64,), float("nan"), device=DEV)
    B.check(B.wino_gated_layer_backward_nhwc(dyt, xt, wt, bt, dx, dw, db, *size, ws, need))
    assert bool(torch.isnan(ws[(need + 3) // 4:]).all())
    assert all(bool((b == 7).all()) for pair in bounds for b in pair)
    for name, got, ref in zip(("y", "dx", "dw", "dbias"), (y, dx, dw, db), want):
        # rounded once, from an exact sum
        bad = got != ref.to(got.dtype)
        assert not bool(bad.any()), f"{name}: {int(bad.sum())} of {bad.numel()} differ, first at {bad.nonzero()[0].tolist()}"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES + ODD)
def test_every_tile(size, dtype):
    exact(*size, dtype, "none")
    exact(*size, dtype, "relu", bias=False, seed=96)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [SIZES[0], SIZES[2], (16641, 56, 520), SIZES[12]])
def test_whole_words_at_any_address(size, dtype):
    exact(*size, dtype, "relu", offset=1)


# first products of one to three steps, whose last two bring dy; tokens that end in each wave's blocks
@pytest.mark.parametrize("tokens", [16641, 16640 - 31, 16640 - 32, 16640 - 33, 16640 - 63, 16640 - 97, 16640 - 128, 16640 - 255])
def test_tokens_at_the_edges_of_wide_tiles(tokens):
    for C, K in ((24, 1000), (64, 1032), (96, 984)):
        assert plan((tokens, C, K), IO["bf16"])[0][0] == WIDE
        exact(tokens, C, K, "bf16", "none")


# wide and square first products, dx and dw of several shapes, on real values
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,C,H,W,K,offset", [(1, 24, 130, 128, 1000, 0), (1, 40, 129, 129, 1000, 0), (1, 72, 127, 131, 1000, 0),
                                              (1, 71, 129, 130, 999, 0), (1, 72, 129, 129, 600, 1)])
def test_silu_on_large_tiles(N, C, H, W, K, offset, dtype):
    x, w, b, dy = make(N, C, H, W, K, dtype, 97)
    check(x, w, b, dtype, "silu", offset=offset)
    check_back(dy, x, w, b, dtype, "silu", offset=offset)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_tiles_repeat_themselves(dtype):
    x, w, b, dy = make(1, 72, 127, 131, 1000, dtype, 98)
    first = [gated(x, w, b, dtype, "silu")] + gated_back(dy, x, w, b, dtype, "silu")
    for _ in range(3):
        again = [gated(x, w, b, dtype, "silu")] + gated_back(dy, x, w, b, dtype, "silu")
        assert all(torch.equal(p, q) for p, q in zip(first, again))


# on both sides of the limits of tiles that go straight to LDS: 2^20 channels, 2^19 units, 2^27 weights
@pytest.mark.parametrize("M,C,K,dtype", [(260, 1 << 20, 8, "bf16"), (40, (1 << 20) + 8, 8, "bf16"), (130, 1 << 20, 8, "f32"),
                                         (260, 8, 1 << 19, "bf16"), (40, 8, (1 << 19) + 8, "bf16"), (130, 8, 1 << 19, "f32"),
                                         (40, 1 << 14, 8184, "bf16"), (40, 1 << 14, 8192, "bf16")])
def test_the_limits_of_offsets(M, C, K, dtype):
    exact(M, C, K, dtype, "none")
