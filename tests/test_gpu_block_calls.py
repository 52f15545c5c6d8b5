"""How the attention half's calls are used: on other streams, captured and replayed, two
graphs with one workspace, and 60 seeded random calls against 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

import test_gpu_cross_attention as attention
import test_gpu_gated_layer as gated_layer
import test_gpu_qk_norm as qk_norm
from block_helpers import B, DEV, IO, dev, ints, space

pytestmark = pytest.mark.gpu


class Step:
    """Norm, attention and gated layer of one size, forward and backward, on one workspace."""

    def __init__(self, size, dtype, ws=None, mask=False):
        N, L, Lk, Hq, Hk, D, K = self.size = size
        C = self.C = Hq * D
        rng = np.random.default_rng(81)
        self.x, self.kv, self.dy = (dev(rng.standard_normal(s), dtype) for s in ((N, L, Hq, D), (N, Lk, 2, Hk, D), (N, 1, L, K)))
        self.w = dev(rng.standard_normal((2, K, C)) / C ** 0.5, dtype)
        self.g, self.b = dev(1 + 0.1 * rng.standard_normal(D)), dev(rng.standard_normal((2, K)))
        a = rng.uniform(-3, 3, (max(L, Lk), D // 2))
        self.rot = dev(np.stack((np.cos(a), np.sin(a)), -1))
        self.klen = ints(rng.integers(0, Lk + 1, N))
        self.mask = torch.from_numpy(rng.integers(0, 2, (N, Lk)).astype(np.uint8)).to(DEV) if mask else None
        t = self.x.dtype

        def out(*shape, dtype=t):
            return torch.zeros(shape, dtype=dtype, device=DEV)
        f = torch.float32
        self.outs = (out(N, L, Hq, D), out(N, Lk, Hk, D), out(N, L, Hq, D), out(N, Hq, L, dtype=f), out(N, 1, L, K),
                     out(N, 1, L, C), out(2, K, C), out(2, K, dtype=f), out(N, L, Hq, D), out(N, Lk, Hk, D),
                     out(N, Lk, 2, Hk, D), out(N, L, Hq, D), out(D, dtype=f), out(D, dtype=f))
        self.f = IO[dtype]
        self.asize, self.gsize = (N, L, Lk, Hq, Hk, D), (N, C, 1, L, K)
        self.need = max(B.wino_cross_attention_workspace_bytes(*self.asize, self.f),
                        B.wino_cross_attention_backward_workspace_bytes(*self.asize, self.f),
                        B.wino_qk_norm_backward_workspace_bytes(*self.asize, self.f),
                        B.wino_gated_layer_workspace_bytes(*self.gsize, self.f),
                        B.wino_gated_layer_backward_workspace_bytes(*self.gsize, self.f))
        self.ws = space(self.need) if ws is None else ws

    def __call__(self):
        N, L, Lk, Hq, Hk, D, K = self.size
        yq, yk, a, lse, u, dh, dw, db, dqn, dkn, dkv, dq, dgq, dgk = self.outs
        C, k, v, ws = self.C, self.kv[:, :, 0], self.kv[:, :, 1], (self.ws, self.need)
        norm = (*self.asize, D // 2 * 2, self.rot.shape[0], C, 2 * Hk * D, 1e-6, self.f)
        attn = (*self.asize, C, Hk * D, 2 * Hk * D, D ** -0.5, self.f, *ws)
        given = (self.x, k, self.g, self.g, self.rot, None, None)
        B.check(B.wino_qk_norm_nhwc(*given, yq, yk, *norm))
        B.check(B.wino_cross_attention_nhwc(yq, yk, v, self.klen, self.mask, a, lse, *attn))
        gated = (*self.gsize, self.f | B.WINO_FLAG_SILU, *ws)
        h = a.view(N, 1, L, C)
        B.check(B.wino_gated_layer_nhwc(h, self.w, self.b, u, *gated))
        B.check(B.wino_gated_layer_backward_nhwc(self.dy, h, self.w, self.b, dh, dw, db, *gated))
        B.check(B.wino_cross_attention_backward_nhwc(dh.view(N, L, Hq, D), yq, yk, v, a, lse, self.klen, self.mask, dqn, dkn,
                                                     dkv[:, :, 1], *attn))
        B.check(B.wino_qk_norm_backward_nhwc(dqn, dkn, *given, dq, dkv[:, :, 0], dgq, dgk, *norm, *ws))

    def clear(self):
        for o in self.outs:
            o.zero_()

    def results(self):
        torch.cuda.synchronize()
        return [o.clone() for o in self.outs]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


# parts of keys and of rows that are joined, and none; one token; a masked batch
STEPS = [((1, 40, 700, 2, 1, 64, 96), False), ((2, 1, 900, 4, 2, 64, 48), True), ((3, 300, 77, 4, 4, 40, 64), True),
         ((2, 257, 130, 2, 2, 128, 80), False)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size,mask", STEPS)
def test_another_stream_and_a_graph(size, mask, dtype):
    step = Step(size, dtype, mask=mask)
    step()
    first = step.results()
    assert bool(torch.isnan(step.ws[(step.need + 3) // 4:]).all())
    assert all(bool(torch.isfinite(o.float()).all()) for o in first[4:])
    side = torch.cuda.Stream()
    step.clear()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    assert same(first, step.results())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        step.x.mul_(1.0 + 0.25 * i)
        step.klen.copy_(step.klen.flip(0))
        step.clear()
        step.ws.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        got = step.results()
        step.clear()
        step()
        assert same(got, step.results())


def test_two_graphs_with_one_workspace():
    """Replayed in turn on one stream, each leaves what it leaves alone."""
    steps = [Step(s, "bf16", mask=m) for s, m in STEPS[:3]]
    ws = max((s.ws for s in steps), key=lambda w: w.numel())
    graphs = []
    for s in steps:
        s.ws = ws
        s()
        s.alone = s.results()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s()
        graphs.append(graph)
    for _ in range(3):
        for s in steps:
            s.clear()
        for graph in graphs:
            graph.replay()
        for s in steps:
            assert same(s.alone, s.results())


def test_two_streams_at_once():
    """Calls that overlap in time, each with a workspace of its own."""
    steps = [Step(s, "bf16", mask=m) for s, m in STEPS[:2]]
    for s in steps:
        s()
        s.alone = s.results()
        s.clear()
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s()
    assert all(same(s.alone, s.results()) for s in steps)


# ---------------------------------------------------------------- random calls

def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(seed):
    rng = random.Random(1000 + seed)
    Hk = rng.choice([1, 2, 3])
    N, Hq, D = rng.choice([1, 2, 3]), Hk * rng.choice([1, 2, 3, 4]), rng.choice([8, 16, 20, 24, 33, 40, 64, 64, 80, 96, 112, 128])
    Lq, Lk = rng.choice([1, _log(rng, 2, 400)]), _log(rng, 1, 700)
    while N * Hq * Lq * Lk > 400000:
        Lq, Lk = (Lq + 1) // 2, (Lk + 1) // 2
    return rng, rng.choice(["f32", "f16", "bf16"]), (N, Lq, Lk, Hq, Hk, D)


@pytest.mark.parametrize("seed", range(24))
def test_random_attention(seed):
    rng, dtype, size = _draw(seed)
    N, Lq, Lk, Hq, Hk, D = size
    q, k, v, r = attention.make(*size, dtype, 900 + seed)
    dy = attention.rounded(r.standard_normal(q.shape), dtype).astype(np.float64)
    kw = {"klen": r.integers(0, Lk + 1, N) if rng.random() < 0.5 else None,
          "mask": r.integers(0, 3, (N, Lk)) if rng.random() < 0.5 else None,
          "ld": rng.choice([(None,) * 3, (Hq * D + 8, 2 * Hk * D, 2 * Hk * D), (None, Hk * D + 1, None)]),
          "offset": rng.choice([0, 0, 1])}
    attention.check(q, k, v, dtype, **kw)
    attention.check_back(dy, q, k, v, dtype, **kw)


@pytest.mark.parametrize("seed", range(18))
def test_random_norms(seed):
    rng, dtype, (N, Lq, Lk, Hq, Hk, D) = _draw(100 + seed)
    R = rng.choice([0, D // 2 * 2, D // 2 // 2 * 2])
    size, pairs = (N, Lq, Lk, Hq, Hk, D, R), rng.random() < 0.5
    d = qk_norm.make(size, dtype, 950 + seed, rng.choice([0, 700]) if R else 0)
    gap, offset = rng.choice([0, 3, 8]), rng.choice([0, 0, 1])
    qk_norm.check_forward(d, size, dtype, qk_norm.call(d, size, dtype, pairs, gap, offset), pairs)
    qk_norm.check_backward(d, size, dtype, qk_norm.call(d, size, dtype, pairs, gap, offset, back=True), pairs)


@pytest.mark.parametrize("seed", range(18))
def test_random_gated_layers(seed):
    rng = random.Random(2000 + seed)
    C, K = _log(rng, 1, 300), _log(rng, 1, 300)
    if rng.random() < 0.6:
        C, K = (C + 15) // 16 * 16, (K + 15) // 16 * 16
    dtype, act = rng.choice(["f32", "f16", "bf16"]), rng.choice(["none", "silu", "silu"])
    x, w, b, dy = gated_layer.make(rng.choice([1, 2]), C, rng.choice([1, _log(rng, 1, 25)]), _log(rng, 1, 25), K, dtype,
                                   980 + seed, rng.random() < 0.5)
    offset = rng.choice([0, 0, 1])
    gated_layer.check(x, w, b, dtype, act, offset=offset)
    gated_layer.check_back(dy, x, w, b, dtype, act, offset=offset)
