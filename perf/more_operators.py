"""What the attention half of an image model's block does around the library's
channel-last tensors: queries and keys normalised and rotated, attention of the pixels
to an encoder's states, and the gated layer after it, each with its backward pass.

In a block that is conditioned on an encoder's output, pixels [N][H][W][C] are the
queries' tokens and the encoder's states, of another and ragged length, the keys'.

    norm    each head of queries and keys over its root mean square, scaled by a learned
            vector, the first R channels rotated by the token's position
    nback   dq, dk and the gradients of both vectors
    attn    y = softmax(scale q k^T) v over the keys that an image's length and mask leave,
            query heads sharing key heads in groups; an image without keys gives zeros
    aback   dq, dk, dv from dy and what the forward pass left (y and the rows' log sums)
    gated   y = act(x w0^T + b0) * (x w1^T + b1), both 1x1 layers of a channel-last tensor
    gback   dx, dw, db from dy and x

Sizes: the images are those of the library's own layers (7x7 to 112x112, 64 to 512
channels), the encoder's states generic, one token to some thousand.
"""
import math

import torch

own = False

EPS = 1e-6
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _norm(name, op, dtype, N, Lq, Lk, Hq, Hk, D, R, T=0, pairs=False):
    """T: rows of the table, where tokens are at positions of their own (0: token i is at i)."""
    return {"name": name, "op": op, "dtype": dtype, "N": N, "Lq": Lq, "Lk": Lk, "Hq": Hq, "Hk": Hk, "D": D, "R": R,
            "T": T, "pairs": pairs}


def _attn(name, op, dtype, N, Lq, Lk, Hq, Hk, D, ragged=False, mask=False, lse=False):
    return {"name": name, "op": op, "dtype": dtype, "N": N, "Lq": Lq, "Lk": Lk, "Hq": Hq, "Hk": Hk, "D": D,
            "ragged": ragged, "mask": mask, "lse": lse}


def _gated(name, op, dtype, N, C, H, W, K, act="silu", bias=False):
    return {"name": name, "op": op, "dtype": dtype, "N": N, "C": C, "H": H, "W": W, "K": K, "act": act, "bias": bias}


def listed():
    return [
        # serving, one token a sequence, far along: the smallest call, latency alone
        _norm("norm_token_n8_bf16", "norm", "bf16", 8, 1, 1, 8, 2, 64, 64, T=32768),
        # batch inference at the headline layer's size, 256 channels in four heads
        _norm("norm_n64_56x56_bf16", "norm", "bf16", 64, 3136, 3136, 4, 4, 64, 64),
        # training at the same image, shared key heads, half of each head rotated
        _norm("nback_n32_56x56", "nback", "f32", 32, 3136, 1500, 4, 2, 64, 32),
        # serving, one token a sequence, over long states of ragged length, shared heads
        _attn("attn_token_n32_l4096_bf16", "attn", "bf16", 32, 1, 4096, 32, 8, 128, ragged=True),
        # a stage's small batch attending to a short text, its padding masked; heads of 40
        _attn("attn_n8_28x28_l77_f16", "attn", "f16", 8, 784, 77, 8, 8, 40, mask=True),
        # the headline image against long states, training's forward
        _attn("attn_n16_56x56_l2048_bf16", "attn", "bf16", 16, 3136, 2048, 8, 8, 64, ragged=True, lse=True),
        # fine-tuning the small batch in fp32
        _attn("aback_n4_28x28_l300", "aback", "f32", 4, 784, 300, 4, 4, 64, mask=True),
        # the headline image's backward, shared key heads, ragged lengths
        _attn("aback_n16_56x56_l1024_bf16", "aback", "bf16", 16, 3136, 1024, 8, 4, 64, ragged=True),
        # serving, one token: the weights' bytes are all there is
        _gated("gated_token_bf16", "gated", "bf16", 1, 512, 1, 1, 2048),
        # a deep layer's batch inference
        _gated("gated_n32_14x14_c512_bf16", "gated", "bf16", 32, 512, 14, 14, 2048),
        # fine-tuning the stage's small batch in fp32
        _gated("gback_n8_28x28_c128", "gback", "f32", 8, 128, 28, 28, 512, bias=True),
        # the headline image's backward
        _gated("gback_n64_56x56_c256_bf16", "gback", "bf16", 64, 256, 56, 56, 1024),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more call of these ranges: odd lengths and widths, one token to many, every
    type, heads of 8 to 128 channels, no group shared or all."""
    every = listed()
    while True:
        op, dtype = rng.choice(["norm", "nback", "attn", "aback", "gated", "gback"]), rng.choice(["f32", "f16", "bf16", "bf16"])
        N = _log_int(rng, 1, 64)
        if op in ("gated", "gback"):
            H = 1 if rng.random() < 0.25 else _log_int(rng, 2, 112)
            C, K = _log_int(rng, 16, 1024), _log_int(rng, 32, 4096)
            if rng.random() < 0.7:              # channel counts are mostly multiples of 16
                C, K = (C + 15) // 16 * 16, (K + 15) // 16 * 16
            c = _gated("", op, dtype, N, C, H, H if rng.random() < 0.7 else _log_int(rng, 1, 112), K,
                       rng.choice(["none", "relu", "silu", "silu"]), rng.random() < 0.5)
            if op == "gback" and dtype == "f32" and c["act"] == "relu":
                c["act"] = "silu"               # a sum of 32 bits may fall on either side of relu's jump
        else:
            Hk = rng.choice([1, 2, 3, 4, 8])
            Hq, D = Hk * rng.choice([1, 1, 2, 4, 8]), rng.choice([8, 20, 32, 40, 64, 64, 64, 80, 96, 128, 128])
            Lq = 1 if rng.random() < 0.25 else _log_int(rng, 2, 12544)
            Lk = 1 if op == "norm" and Lq == 1 else _log_int(rng, 1, 8192)
            if op in ("norm", "nback"):
                c = _norm("", op, dtype, N, Lq, Lk, Hq, Hk, D, rng.choice([0, D, D, D // 2 // 2 * 2]),
                          rng.choice([0, _log_int(rng, 1024, 131072)]), rng.random() < 0.3)
            else:
                c = _attn("", op, dtype, N, Lq, Lk, Hq, Hk, D, rng.random() < 0.5, rng.random() < 0.3,
                          rng.random() < 0.5 and op == "attn")
        del c["name"]
        w, same = work(c), [work(e) for e in every if e["op"] == op]
        scores = lambda e: e["N"] * e["Lq"] * e["Lk"] * e["Hq"] if op in ("attn", "aback") else 0  # noqa: E731
        if (w["bytes"] <= max(e["bytes"] for e in same) and w["flops"] <= max(e["flops"] for e in same) and
                scores(c) <= max(scores(e) for e in every if e["op"] == op)):
            return c


def _lens(case):
    """The images' lengths, before they are shuffled: from no key to all of them."""
    N, Lk = case["N"], case["Lk"]
    if not case["ragged"]:
        return [Lk] * N
    return [Lk] if N == 1 else [(i * Lk + (N - 1) // 2) // (N - 1) for i in range(N)]


def work(case):
    """Every input read once and every output written once.  2 flops a product: of scores
    and values (4 D for each query head's pair of tokens; backward scores again, dP, dv, dk
    and dq), of the two layers (backward once more, then dx and dw); some 10 a value of the norm."""
    op, s = case["op"], 4 if case["dtype"] == "f32" else 2
    N = case["N"]
    if op in ("gated", "gback"):
        M, C, K = N * case["H"] * case["W"], case["C"], case["K"]
        move, flops = s * (M * C + 2 * K * C + M * K), 4 * M * C * K
        return {"bytes": move, "flops": flops} if op == "gated" else {"bytes": move + s * (M * C + 2 * K * C),
                                                                      "flops": 3 * flops}
    Lq, Lk, Hq, Hk, D = case["Lq"], case["Lk"], case["Hq"], case["Hk"], case["D"]
    Q = N * Lq * Hq * D
    if op in ("norm", "nback"):
        X = Q + N * Lk * Hk * D
        table = 4 * case["R"] * (min(case["T"], N * (Lq + Lk)) if case["T"] else max(Lq, Lk))
        return {"bytes": (2 if op == "norm" else 3) * s * X + table, "flops": (10 if op == "norm" else 20) * X}
    keys = sum(_lens(case))
    KV = 2 * keys * Hk * D
    bits = N * Lk if case["mask"] else 0
    rows = 4 * N * Lq * Hq if case["lse"] or op == "aback" else 0
    if op == "attn":
        return {"bytes": s * (2 * Q + KV) + bits + rows, "flops": 4 * Lq * keys * Hq * D}
    # the gradients of all keys are written, of those past the lengths as zeros
    return {"bytes": s * (4 * Q + KV + 2 * N * Lk * Hk * D) + bits + rows, "flops": 10 * Lq * keys * Hq * D}


# ---------------------------------------------------------------- inputs

def _inputs(case, seed):
    """Projections of unit scale whose channels differ in mean and spread, as norm inputs;
    queries and keys that score with a deviation of two; gradients of unit scale; weights
    that keep the scale.  Keys and values, and the norm's queries and keys where there are as
    many of both, come of one projection and lie in one tensor."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, t, N = case["op"], DTYPE[case["dtype"]], case["N"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    if op in ("gated", "gback"):
        C, H, W, K = case["C"], case["H"], case["W"], case["K"]
        d = {"x": randn(N, H, W, C).to(t), "w": randn(2, K, C).div_(math.sqrt(C)).to(t),
             "bias": 0.3 * randn(2, K) if case["bias"] else None}
        if op == "gback":
            d["dy"] = randn(N, H, W, K).to(t)
        return d
    Lq, Lk, Hq, Hk, D = case["Lq"], case["Lk"], case["Hq"], case["Hk"], case["D"]
    if op in ("norm", "nback"):
        def spread(*shape):
            return randn(*shape).mul_(torch.exp(0.3 * randn(shape[-1]))).add_(0.3 * randn(shape[-1])).to(t)
        if Lq == Lk:
            qk = spread(N, Lq, Hq + Hk, D)
            d = {"qk": qk, "q": qk[:, :, :Hq], "k": qk[:, :, Hq:]}
        else:
            d = {"q": spread(N, Lq, Hq, D), "k": spread(N, Lk, Hk, D)}
        d["gq"], d["gk"] = 1.0 + 0.2 * randn(D), 1.0 + 0.2 * randn(D)
        R, T = case["R"], case["T"]
        rows = T or max(Lq, Lk)
        # angles in 64 bits: far positions are whole turns past what 32 hold
        angle = (torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] *
                 10000.0 ** (-torch.arange(R // 2, device="cuda", dtype=torch.float64) * 2 / max(R, 1)))
        d["rot"] = torch.stack((torch.cos(angle), torch.sin(angle)), -1).float() if R else None
        d["qpos"] = d["kpos"] = None
        if T and R:
            d["qpos"] = torch.randint(0, T, (N, Lq), generator=gen, device="cuda", dtype=torch.int32)
            d["kpos"] = torch.randint(0, T, (N, Lk), generator=gen, device="cuda", dtype=torch.int32)
        if op == "nback":
            d["dyq"], d["dyk"] = randn(N, Lq, Hq, D).to(t), randn(N, Lk, Hk, D).to(t)
        return d
    d = {"q": randn(N, Lq, Hq, D).mul_(2.0).to(t)}
    d["kv"] = randn(N, Lk, 2, Hk, D).add_(0.3 * randn(2, Hk, D)).to(t)
    d["k"], d["v"] = d["kv"][:, :, 0], d["kv"][:, :, 1]
    d["klen"] = d["mask"] = None
    if case["ragged"]:
        lens = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
        d["klen"] = lens[torch.randperm(N, generator=gen, device="cuda")]
    if case["mask"]:
        d["mask"] = (torch.rand((N, Lk), generator=gen, device="cuda") < 0.8).to(torch.uint8)
    if op == "aback":
        d["dy"] = randn(N, Lq, Hq, D).to(t)
        y, d["lse"] = _attend(d, case)          # what the forward pass left
        d["y"] = y.to(t)
    return d


def prepare(case, seed):
    state = {"case": dict(case), **_inputs(case, seed)}
    if own:
        state.update(_plan(case, state))
    return state


# ---------------------------------------------------------------- the framework's calls

def _plan(case, d):
    """Output buffers and workspace, kept from call to call, and the flags."""
    from paper_1903_01521_amd import binding as B
    op, N = case["op"], case["N"]
    flags = {"f32": 0, "f16": B.WINO_IO_F16, "bf16": B.WINO_IO_BF16}[case["dtype"]]
    out, ws = {}, 0
    if op in ("gated", "gback"):
        C, H, W, K = case["C"], case["H"], case["W"], case["K"]
        flags |= {"none": 0, "relu": B.WINO_FLAG_RELU, "silu": B.WINO_FLAG_SILU}[case["act"]]
        if op == "gated":
            out["y"] = torch.empty((N, H, W, K), dtype=d["x"].dtype, device="cuda")
            ws = B.wino_gated_layer_workspace_bytes(N, C, H, W, K, flags)
        else:
            out["dx"], out["dw"] = torch.empty_like(d["x"]), torch.empty_like(d["w"])
            out["dbias"] = torch.empty_like(d["bias"]) if case["bias"] else None
            ws = B.wino_gated_layer_backward_workspace_bytes(N, C, H, W, K, flags)
    elif op in ("norm", "nback"):
        flags |= B.WINO_FLAG_PAIRS if case["pairs"] else 0
        if op == "norm":
            out["yq"], out["yk"] = (torch.empty(d[x].shape, dtype=d[x].dtype, device="cuda") for x in "qk")
        else:
            if "qk" in d:
                out["dqk"] = torch.empty_like(d["qk"])
                out["dq"], out["dk"] = out["dqk"][:, :, :case["Hq"]], out["dqk"][:, :, case["Hq"]:]
            else:
                out["dq"], out["dk"] = torch.empty_like(d["q"]), torch.empty_like(d["k"])
            out["dgq"], out["dgk"] = torch.empty_like(d["gq"]), torch.empty_like(d["gk"])
            ws = B.wino_qk_norm_backward_workspace_bytes(N, case["Lq"], case["Lk"], case["Hq"], case["Hk"], case["D"],
                                                         flags)
    else:
        size = (N, case["Lq"], case["Lk"], case["Hq"], case["Hk"], case["D"], flags)
        if op == "attn":
            out["y"] = torch.empty_like(d["q"])
            out["lse"] = torch.empty((N, case["Hq"], case["Lq"]), device="cuda") if case["lse"] else None
            ws = B.wino_cross_attention_workspace_bytes(*size)
        else:
            out["dq"], out["dkv"] = torch.empty_like(d["q"]), torch.empty_like(d["kv"])
            out["dk"], out["dv"] = out["dkv"][:, :, 0], out["dkv"][:, :, 1]
            ws = B.wino_cross_attention_backward_workspace_bytes(*size)
    assert 0 <= ws < 1 << 40
    plan = {"out": out, "flags": flags, "space": torch.empty(ws, dtype=torch.int8, device="cuda") if ws else None,
            "bytes": ws}
    if op == "aback":
        plan["y"] = d["y"].contiguous()         # as the forward call wrote it
    return plan


def _call(s):
    from paper_1903_01521_amd import binding as B
    c, out, flags, ws, wsb = s["case"], s["out"], s["flags"], s["space"], s["bytes"]
    op, N = c["op"], c["N"]
    if op in ("gated", "gback"):
        size = (N, c["C"], c["H"], c["W"], c["K"], flags, ws, wsb)
        if op == "gated":
            B.check(B.wino_gated_layer_nhwc(s["x"], s["w"], s["bias"], out["y"], *size), "gated")
            return {"y": out["y"]}
        B.check(B.wino_gated_layer_backward_nhwc(s["dy"], s["x"], s["w"], s["bias"], out["dx"], out["dw"],
                                                 out["dbias"], *size), "gback")
        return {"dx": out["dx"], "dw": out["dw"], "db": out["dbias"]}
    Lq, Lk, Hq, Hk, D = c["Lq"], c["Lk"], c["Hq"], c["Hk"], c["D"]
    if op in ("norm", "nback"):
        T = 0 if s["rot"] is None else s["rot"].shape[0]
        ldq, ldk = ((Hq + Hk) * D,) * 2 if "qk" in s else (Hq * D, Hk * D)
        size = (N, Lq, Lk, Hq, Hk, D, c["R"], T, ldq, ldk, EPS, flags)
        given = (s["q"], s["k"], s["gq"], s["gk"], s["rot"], s["qpos"], s["kpos"])
        if op == "norm":
            B.check(B.wino_qk_norm_nhwc(*given, out["yq"], out["yk"], *size), "norm")
            return {"q": out["yq"], "k": out["yk"]}
        B.check(B.wino_qk_norm_backward_nhwc(s["dyq"], s["dyk"], *given, out["dq"], out["dk"], out["dgq"], out["dgk"],
                                             *size, ws, wsb), "nback")
        return {"dq": out["dq"], "dk": out["dk"], "dgq": out["dgq"], "dgk": out["dgk"]}
    size = (N, Lq, Lk, Hq, Hk, D, Hq * D, 2 * Hk * D, 2 * Hk * D, D ** -0.5, flags, ws, wsb)
    if op == "attn":
        B.check(B.wino_cross_attention_nhwc(s["q"], s["k"], s["v"], s["klen"], s["mask"], out["y"], out["lse"], *size),
                "attn")
        return {"y": out["y"], "lse": out["lse"]}
    B.check(B.wino_cross_attention_backward_nhwc(s["dy"], s["q"], s["k"], s["v"], s["y"], s["lse"], s["klen"],
                                                 s["mask"], out["dq"], out["dk"], out["dv"], *size), "aback")
    return {"dq": out["dq"], "dkv": out["dkv"]}


# ---------------------------------------------------------------- the plain forms

def _turned(x, c, s, case, back=False):
    """The first R channels of x [N][L][heads][D] rotated by c, s [.][L][1][R/2], or back."""
    R = case["R"]
    if R == 0:
        return x
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if case["pairs"] else (x[..., :R // 2], x[..., R // 2:R])
    if back:
        s = -s
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack((a, b), -1).flatten(-2) if case["pairs"] else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., R:]), -1)


def _angles(s, pos, L):
    if s["rot"] is None:
        return None, None
    rows = s["rot"][None, :L] if s[pos] is None else s["rot"][s[pos].long()]
    return rows[:, :, None, :, 0], rows[:, :, None, :, 1]


def _normed(s, c, name):
    """x over its heads' root mean square, and that factor."""
    x = s[name].float()
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _norm_back(s, c, name):
    n, r = _normed(s, c, name)
    cos, sin = _angles(s, name + "pos", n.shape[1])
    dz = _turned(s["dy" + name].float(), cos, sin, c, back=True)
    dg = (dz * n).sum((0, 1, 2))
    dn = dz * s["g" + name]
    return (r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(s[name].dtype), dg


def _grouped(x, Hk):
    """[N][L][Hq][D] to [N][Hk][Hq/Hk * L][D], in 32 bits: the rows that share a key head."""
    N, L, Hq, D = x.shape
    return x.float().view(N, L, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(N, Hk, Hq // Hk * L, D)


def _ungrouped(x, L):
    N, Hk, rows, D = x.shape
    return x.view(N, Hk, rows // L, L, D).permute(0, 3, 1, 2, 4).reshape(N, L, Hk * (rows // L), D)


def _scores(d, c):
    """exp(scores - their rows' largest), that largest, and the scaled queries, keys and
    values, by key head; 0 for a key that is left out."""
    Hk, Lk = c["Hk"], c["Lk"]
    q = _grouped(d["q"], Hk) * c["D"] ** -0.5
    k, v = d["k"].float().transpose(1, 2).contiguous(), d["v"].float().transpose(1, 2).contiguous()
    p = q @ k.transpose(2, 3).contiguous()
    kept = torch.ones((c["N"], Lk), dtype=torch.bool, device=p.device)
    if d["klen"] is not None:
        kept &= torch.arange(Lk, device=p.device) < d["klen"][:, None]
    if d["mask"] is not None:
        kept &= d["mask"] != 0
    p.masked_fill_(~kept[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    return p.sub_(top).exp_(), top, q, k, v


def _attend(d, c):
    """y in 32 bits and the log of the rows' sums [N][Hq][Lq], -inf where no key is left."""
    p, top, _, _, v = _scores(d, c)
    total = p.sum(-1, keepdim=True)
    y = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return _ungrouped(y, c["Lq"]), (top + torch.log(total)).view(c["N"], c["Hq"], c["Lq"])


def _attend_back(d, c):
    p, _, q, k, v = _scores(d, c)
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    dy = _grouped(d["dy"], c["Hk"])
    dv = p.transpose(2, 3).contiguous() @ dy
    ds = dy @ v.transpose(2, 3).contiguous()
    ds = ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p)
    dq = (ds @ k) * c["D"] ** -0.5
    dk = ds.transpose(2, 3).contiguous() @ q
    t = d["q"].dtype
    return {"dq": _ungrouped(dq, c["Lq"]).to(t), "dkv": torch.stack((dk, dv), 1).permute(0, 3, 1, 2, 4).contiguous().to(t)}


def _act(z, act):
    return z if act == "none" else z.clamp_min(0.0) if act == "relu" else z / (1.0 + torch.exp(-z))


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op in ("norm", "nback"):
        if op == "nback":
            (dq, dgq), (dk, dgk) = _norm_back(s, c, "q"), _norm_back(s, c, "k")
            return {"dq": dq, "dk": dk, "dgq": dgq, "dgk": dgk}
        t = s["q"].dtype
        return {x: _turned(_normed(s, c, x)[0] * s["g" + x], *_angles(s, x + "pos", c["L" + x]), c).to(t) for x in "qk"}
    if op == "attn":
        y, lse = _attend(s, c)
        return {"y": y.to(s["q"].dtype), "lse": lse if c["lse"] else None}
    if op == "aback":
        return _attend_back(s, c)
    N, C, H, W, K, t = c["N"], c["C"], c["H"], c["W"], c["K"], s["x"].dtype
    x, w = s["x"].float().view(-1, C), s["w"].float()
    zg, zu = x @ w[0].t(), x @ w[1].t()
    if s["bias"] is not None:
        zg, zu = zg + s["bias"][0], zu + s["bias"][1]
    if op == "gated":
        return {"y": (_act(zg, c["act"]) * zu).view(N, H, W, K).to(t)}
    dy = s["dy"].float().view(-1, K)
    if c["act"] == "none":
        slope = torch.ones_like(zg)
    elif c["act"] == "relu":
        slope = (zg > 0).float()
    else:
        sig = 1.0 / (1.0 + torch.exp(-zg))
        slope = sig * (1.0 + zg * (1.0 - sig))
    dzg, dzu = dy * zu * slope, dy * _act(zg, c["act"])
    db = None if s["bias"] is None else torch.stack((dzg.sum(0), dzu.sum(0)))
    return {"dx": (dzg @ w[0] + dzu @ w[1]).view(N, H, W, C).to(t), "dw": torch.stack((dzg.t() @ x, dzu.t() @ x)).to(t),
            "db": db}


def run(state):
    return _call(state) if own else _plain(state)


# ---------------------------------------------------------------- in 64 bits

def _leaf(x):
    return x.double().clone().requires_grad_()


def _norm64(x, g, rot, pos, pairs, R):
    """The rotation as a product of complex numbers."""
    z = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * g
    if R == 0:
        return z
    turn = torch.view_as_complex(rot.double())
    turn = (turn[:x.shape[1]].unsqueeze(0) if pos is None else turn[pos.long()]).unsqueeze(2)
    head = z[..., :R].unflatten(-1, (R // 2, 2) if pairs else (2, R // 2))
    if not pairs:
        head = head.transpose(-1, -2)
    head = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
    if not pairs:
        head = head.transpose(-1, -2)
    return torch.cat((head.reshape(*z.shape[:-1], R), z[..., R:]), -1)


def _image64(q, k, v, scale):
    """One image's rows: q [rows][Hq][D], k and v [keys][Hk][D] of the keys that are left."""
    rep = q.shape[1] // k.shape[1]
    q, k, v = q.transpose(0, 1), k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
    s = torch.bmm(q, k.permute(1, 2, 0).contiguous()) * scale
    return torch.bmm(torch.softmax(s, -1), v.transpose(0, 1).contiguous()).transpose(0, 1), torch.logsumexp(s, -1)


def exact(case, seed):
    d = _inputs(case, seed)
    op, N = case["op"], case["N"]
    if op in ("norm", "nback"):
        out = {}
        for x in "qk":
            v, g = _leaf(d[x]), _leaf(d["g" + x])
            with torch.set_grad_enabled(op == "nback"):
                y = _norm64(v, g, d["rot"], d[x + "pos"], case["pairs"], case["R"])
            if op == "norm":
                out[x] = y
            else:
                out["d" + x], out["dg" + x] = torch.autograd.grad(y, (v, g), d["dy" + x].double())
        return out
    if op in ("attn", "aback"):
        Lq, Hq, Lk, scale = case["Lq"], case["Hq"], case["Lk"], case["D"] ** -0.5
        q = d["q"].double()
        y, lse = torch.zeros_like(q), torch.full((N, Hq, Lq), -math.inf, dtype=torch.float64, device=q.device)
        dq, dkv = torch.zeros_like(q), torch.zeros(d["kv"].shape, dtype=torch.float64, device=q.device)
        step = max(1, (1 << 28) // (Hq * Lk))       # rows at a time: 2 GB of scores
        for i in range(N):
            keep = torch.ones(Lk, dtype=torch.bool, device=q.device) if d["mask"] is None else d["mask"][i] != 0
            if d["klen"] is not None:
                keep[int(d["klen"][i]):] = False
            at = keep.nonzero()[:, 0]
            if at.numel() == 0:
                continue
            k, v = d["k"][i, at].double(), d["v"][i, at].double()
            for a in range(0, Lq, step):
                b = min(Lq, a + step)
                if op == "attn":
                    y[i, a:b], lse[i, :, a:b] = _image64(q[i, a:b], k, v, scale)
                else:
                    lq, lk, lv = _leaf(q[i, a:b]), _leaf(k), _leaf(v)
                    o, _ = _image64(lq, lk, lv, scale)
                    dq[i, a:b], gk, gv = torch.autograd.grad(o, (lq, lk, lv), d["dy"][i, a:b].double())
                    dkv[i, at] += torch.stack((gk, gv), 1)
        return {"y": y, "lse": lse if case["lse"] else None} if op == "attn" else {"dq": dq, "dkv": dkv}
    x, w = _leaf(d["x"]), _leaf(d["w"])
    b = None if d["bias"] is None else _leaf(d["bias"])
    with torch.set_grad_enabled(op == "gback"):
        z = [torch.nn.functional.linear(x, w[i], None if b is None else b[i]) for i in (0, 1)]
        gate = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu}[case["act"]](z[0])
        y = gate * z[1]
    if op == "gated":
        return {"y": y}
    dx, dw, *db = torch.autograd.grad(y, (x, w) if b is None else (x, w, b), d["dy"].double())
    return {"dx": dx, "dw": dw, "db": db[0] if db else None}
