"""Calls of the training entry points on numpy inputs, and the error bounds that
their tests share."""
import numpy as np
import torch

from paper_1903_01521_amd import binding as B

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
IO = {"f32": 0, "f16": B.WINO_IO_F16, "bf16": B.WINO_IO_BF16}
ACT = {"none": 0, "relu": B.WINO_FLAG_RELU, "silu": B.WINO_FLAG_SILU}
U32 = 2.0 ** -24                                        # fp32's unit roundoff
HALF_ULP = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # of a stored result, relative
# fp32 sums here add at most about 64 values a thread, 32 partial rows twice and
# the parts in turn: 256 roundings bound all of them.
SUM = 256 * U32


def dev(a, dtype="f32", offset=0):
    """A contiguous device tensor of a's values, `offset` elements past an aligned address."""
    a = np.ascontiguousarray(a, dtype=np.float32)
    t = torch.empty(a.size + offset, dtype=DTYPE[dtype], device=DEV)[offset:].view(a.shape)
    t.copy_(torch.from_numpy(a))
    return t


def like(t, fill=float("nan")):
    return torch.full(t.shape, fill, dtype=t.dtype, device=DEV)


def host(t):
    torch.cuda.synchronize()
    return t.detach().cpu().float().numpy().astype(np.float64)


def rounded(a, dtype):
    """a as stored in dtype, in float32."""
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DTYPE[dtype]).float().numpy()


def space(nbytes):
    """A workspace of that size with a guard of 64 bytes after it, filled with NaN."""
    assert nbytes != 2**64 - 1
    return torch.full(((nbytes + 64 + 3) // 4,), float("nan"), dtype=torch.float32, device=DEV)


def group_norm(x, gamma, beta, G, eps, dtype="f32", act="none", stats=True, ckpt=False, offset=0, y=None):
    """(y, stats, ckpt) device tensors through wino_group_norm_nhwc."""
    N, H, W, C = x.shape
    xt = x if isinstance(x, torch.Tensor) else dev(x, dtype, offset)
    y = dev(np.full(x.shape, np.nan), dtype, offset) if y is None else y
    st = torch.full((N, G, 2), float("nan"), device=DEV) if stats else None
    q = torch.full((B.wino_act8_bytes(N, C, H, W),), 85, dtype=torch.int8, device=DEV) if ckpt else None
    flags = IO[dtype] | ACT[act]
    wsb = B.wino_group_norm_workspace_bytes(N, C, H, W, G, flags)
    ws = space(wsb)
    g, b = (None if v is None else dev(v) for v in (gamma, beta))
    B.check(B.wino_group_norm_nhwc(xt, g, b, y, st, q, N, C, H, W, G, eps, flags, ws, wsb))
    return y, st, q


def backward(dy, x, stats, gamma, beta, dtype="f32", act="none", ckpt=False, offset=0):
    """(dx, dgamma, dbeta); x a numpy array, or a checkpoint's tensor."""
    N, H, W, C = dy.shape
    G = stats.shape[1]
    dyt = dev(dy, dtype, offset)
    xt = x if ckpt else dev(x, dtype, offset)
    dx = dev(np.full(dy.shape, np.nan), dtype, offset)
    dgamma, dbeta = torch.full((C,), float("nan"), device=DEV), torch.full((C,), float("nan"), device=DEV)
    flags = IO[dtype] | ACT[act] | (B.WINO_FLAG_ACT8 if ckpt else 0)
    wsb = B.wino_group_norm_backward_workspace_bytes(N, C, H, W, G, flags)
    g, b = (None if v is None else dev(v) for v in (gamma, beta))
    B.check(B.wino_group_norm_backward_nhwc(dyt, xt, dev(stats), g, b, dx, dgamma, dbeta, N, C, H, W, G, flags,
                                            space(wsb), wsb))
    return dx, dgamma, dbeta


def split_ckpt(q, N, H, W, C):
    """(codes, centre, step) numpy of a checkpoint's tensor."""
    X = N * H * W * C
    raw = q.cpu().numpy()
    rows = raw[(X + 15) // 16 * 16:].view(np.float32).reshape(N, C, 2)
    return raw[:X].reshape(N, H, W, C), rows[..., 0], rows[..., 1]


def make_ckpt(codes, centre, step):
    X = codes.size
    raw = np.zeros((X + 15) // 16 * 16 + centre.size * 8, np.int8)
    raw[:X] = codes.reshape(-1)
    raw[(X + 15) // 16 * 16:] = np.stack((centre, step), -1).astype(np.float32).reshape(-1).view(np.int8)
    return torch.from_numpy(raw).to(DEV)
