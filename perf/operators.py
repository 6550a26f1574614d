"""Layer norm and 8-bit activation checkpoints around the sparse linear layer, as cases that can be timed and compared.

Four kinds of pass:

* ``ln_fwd``  layer norm forward, with the residual addition in front of it and the checkpoints that a training step keeps;
* ``ln_bwd``  its backward pass: input gradient (with the gradient that comes down the residual stream), gamma's and beta's;
* ``ckpt``    a matrix of activations into 8 bits and back;
* ``dw``      the weight gradient of a linear layer from its input's checkpoint, with the adapters' when there are any.

A checkpoint holds 32 consecutive values of a row as 8-bit integers times one power of two: value = code * 2^k, with k the
smallest integer for which the block's largest magnitude is at most 127.5 * 2^k, in [-126, 121]; codes are rounded half to even
and held in [-127, 127].  A block with an infinity or a NaN has exponent byte 255 and reads back as NaN.  One buffer of bytes: all
codes, row by row, then one byte k + 127 per block.  Outputs are the values that the codes stand for.
"""
import math

import torch

own = False            # True: the calls of the framework's binding; False: the same in elementary torch operations
B = None

EPS = 1e-5
BLOCK = 32


def listed():
    return [
        # decoding one sequence of a 7B-wide model: one row, bound by latency and by the cost of a call
        {"name": "ln_fwd_decode", "kind": "ln_fwd", "b": 1, "d": 4096, "x": "bf16", "p": "bf16", "residual": True, "train": False, "ckpt": "none"},
        # GPT-2-small's pretraining batch, pre-LN block: sub-layer output added, both checkpoints kept
        {"name": "ln_fwd_gpt2", "kind": "ln_fwd", "b": 8192, "d": 768, "x": "bf16", "p": "bf16", "residual": True, "train": True, "ckpt": "both"},
        # a 7B-wide block whose residual stream and parameters are held in fp32; the linears' input is checkpointed
        {"name": "ln_fwd_7b_f32", "kind": "ln_fwd", "b": 16384, "d": 4096, "x": "f32", "p": "f32", "residual": True, "train": True, "ckpt": "y"},
        # a ragged batch at 13B width, first layer norm of a stack: no residual, nothing in 8 bits
        {"name": "ln_fwd_13b_ragged", "kind": "ln_fwd", "b": 2039, "d": 5120, "x": "bf16", "p": "f32", "residual": False, "train": True, "ckpt": "none"},
        # one small layer at a small batch: two short launches
        {"name": "ln_bwd_512", "kind": "ln_bwd", "b": 256, "d": 512, "x": "bf16", "dx": "bf16", "p": "bf16", "dh": False},
        # GPT-2-small's batch, everything kept in 8 bits
        {"name": "ln_bwd_gpt2_q8", "kind": "ln_bwd", "b": 8192, "d": 768, "x": "q8", "dx": "bf16", "p": "f32", "dh": True},
        # a 7B-wide block in bf16
        {"name": "ln_bwd_7b", "kind": "ln_bwd", "b": 16384, "d": 4096, "x": "bf16", "dx": "bf16", "p": "bf16", "dh": True},
        # the projections' input of a small model, ragged batch
        {"name": "ckpt_ragged", "kind": "ckpt", "b": 1000, "d": 2304, "x": "bf16"},
        # the down projection's input of a 7B model at its pretraining batch
        {"name": "ckpt_7b_down", "kind": "ckpt", "b": 16384, "d": 11008, "x": "bf16"},
        # one small layer at a small batch
        {"name": "dw_512", "kind": "dw", "b": 256, "d_in": 512, "d_out": 512, "r": 0},
        # a square attention projection of a 7B model in the adapter phase
        {"name": "dw_7b_q_r64", "kind": "dw", "b": 16384, "d_in": 4096, "d_out": 4096, "r": 64},
        # the down projection of the same model before the adapters come in: the widest checkpoint
        {"name": "dw_7b_down", "kind": "dw", "b": 16384, "d_in": 11008, "d_out": 4096, "r": 0},
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _multiple(rng, step, lo, hi):
    return step * max(1, round(_log_uniform(rng, lo, hi) / step))


def draw(rng):
    kind = rng.choices(["ln_fwd", "ln_bwd", "ckpt", "dw"], [4, 4, 2, 4])[0]
    types = ["bf16", "bf16", "f32"]
    if kind == "dw":
        d_in, d_out = _multiple(rng, 128, 512, 13824), _multiple(rng, 128, 512, 13824)
        b = max(1, min(round(_log_uniform(rng, 64, 16384)), int(16384 * 4096 * 11008 // (d_in * d_out))))
        return {"kind": kind, "b": b, "d_in": d_in, "d_out": d_out, "r": rng.choice([0, 0, 0, 16, 64, 128, 256])}
    if kind == "ckpt":
        d = _multiple(rng, 32, 128, 13824)
        return {"kind": kind, "b": round(_log_uniform(rng, 1, 16384 * 11008 / max(d, 11008))), "d": d, "x": rng.choice(types)}
    # widths of 8 where nothing is in 8 bits, else whole blocks
    ckpt = rng.choice(["none", "h", "y", "both"])
    x = rng.choice(types) if kind == "ln_fwd" else rng.choice(["bf16", "f32", "q8", "q8"])
    d = _multiple(rng, 8 if (ckpt == "none" if kind == "ln_fwd" else x != "q8") else 32, 64, 8192)
    b = round(_log_uniform(rng, 1, min(32768, 16384 * 4096 / d)))
    case = {"kind": kind, "b": b, "d": d, "x": x, "p": rng.choice(types)}
    if kind == "ln_fwd":
        return {**case, "residual": rng.random() < 0.6, "train": ckpt != "none" or rng.random() < 0.5, "ckpt": ckpt}
    return {**case, "dx": "bf16" if x == "bf16" else "f32" if x == "f32" else rng.choice(types), "dh": rng.random() < 0.6}


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _stream(gen, b, d):
    """Activations as a residual stream has them: channels of unlike size, a few of them far larger, a small offset, rows of unlike scale."""
    new = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    channel = torch.exp(0.3 * new(d))
    channel[torch.randint(0, d, (max(1, d // 256),), device="cuda", generator=gen)] *= 12.0
    return (new(b, d) * channel + (0.25 + 0.1 * new(d))) * torch.exp(0.3 * new(b, 1))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *shape, sigma=1.0: torch.randn(shape, device="cuda", generator=gen, dtype=torch.bfloat16).mul_(sigma)
    empty = lambda *shape, t=torch.bfloat16: torch.empty(shape, device="cuda", dtype=t)
    ckpt = lambda b, d: empty(b * d + b * d // BLOCK, t=torch.uint8)
    kind, s, b = case["kind"], dict(case), case["b"]
    if kind == "dw":
        d_in, d_out, r = case["d_in"], case["d_out"], case["r"]
        X = _stream(gen, b, d_in).bfloat16()
        s["Xc"], s["dY"] = _encode(X), new(b, d_out)
        # the first pruning pass: the two largest of every four consecutive weights of a row
        kept = new(d_out, d_in // 4, 4).float().abs().topk(2, dim=-1).indices
        bits = torch.zeros(d_out, d_in // 4, 4, dtype=torch.int32, device="cuda").scatter_(2, kept, 1).view(d_out, d_in // 8, 8)
        s["mask"] = (bits << torch.arange(8, device="cuda", dtype=torch.int32)).sum(-1).to(torch.uint8)
        s["dWc"] = empty(d_out, d_in // 2)
        if r:
            s["T"], s["dT"], s["dL"], s["dR"] = new(b, r, sigma=0.3), new(b, r, sigma=0.3), empty(d_in, r), empty(r, d_out)
        return s
    d = case["d"]
    if kind == "ckpt":
        s["X"], s["Xc"] = _stream(gen, b, d).to(_TYPES[case["x"]]), ckpt(b, d)
        s["out"] = empty(b, d)
        return s
    p = _TYPES[case["p"]]
    s["gamma"], s["beta"] = (1.0 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(p), (0.1 * torch.randn(d, device="cuda", generator=gen)).to(p)
    if kind == "ln_fwd":
        x = _TYPES[case["x"]]
        s["X"] = _stream(gen, b, d).to(x)
        s["Y"] = empty(b, d)
        s["R"], s["H"] = (new(b, d, sigma=0.5), empty(b, d, t=x)) if case["residual"] else (None, None)
        s["mean"], s["rstd"] = (empty(b, t=torch.float32), empty(b, t=torch.float32)) if case["train"] else (None, None)
        s["Hc"], s["Hv"] = (ckpt(b, d), empty(b, d)) if case["ckpt"] in ("h", "both") else (None, None)
        s["Yc"], s["Yv"] = (ckpt(b, d), empty(b, d)) if case["ckpt"] in ("y", "both") else (None, None)
        return s
    # what the forward pass has left: the stream (or its checkpoint) and the statistics of the stream itself
    X = _stream(gen, b, d).to(torch.float32 if case["x"] == "f32" else torch.bfloat16)
    X64 = X.double()
    s["mean"] = X64.mean(-1).float()
    s["rstd"] = (X64.var(-1, unbiased=False) + EPS).rsqrt().float()
    s["X"] = _encode(X) if case["x"] == "q8" else X
    dx = _TYPES[case["dx"]]
    s["dY"], s["dX"] = new(b, d, sigma=0.02), empty(b, d, t=dx)
    s["dH"] = new(b, d, sigma=0.02).to(dx) if case["dh"] else None
    s["dgamma"], s["dbeta"] = empty(d, t=p), empty(d, t=p)
    return s


# ------------------------------------------------------------------ the plain forms
def _power(k):
    """2^k as fp32, k whole and in [-126, 127]."""
    return ((k + 127) << 23).view(torch.float32)


def _encode(x):
    rows, cols = x.shape
    blocks = x.float().reshape(rows, cols // BLOCK, BLOCK)
    a = blocks.abs().amax(-1)
    fine = torch.isfinite(a)
    a = torch.where(fine, a, torch.zeros_like(a))
    k = (a.view(torch.int32) >> 23) - 127 - 6
    k = (k + (a * _power(-k.clamp(-126, 121)) > 127.5)).clamp(-126, 121)
    codes = torch.round(torch.where(fine[..., None], blocks, torch.zeros_like(blocks)) * _power(-k)[..., None]).clamp(-127, 127).to(torch.int8)
    exponents = torch.where(fine, k + 127, torch.full_like(k, 255)).to(torch.uint8)
    return torch.cat([codes.reshape(-1).view(torch.uint8), exponents.reshape(-1)])


def _decode(c, rows, cols):
    codes = c[:rows * cols].view(torch.int8).reshape(rows, cols // BLOCK, BLOCK).float()
    e = c[rows * cols:].reshape(rows, cols // BLOCK, 1).int()
    return (codes * (e << 23).view(torch.float32)).reshape(rows, cols)


def _plain_ln_fwd(s):
    H = None
    h = s["X"].float()
    if s["R"] is not None:
        H = (h + s["R"].float()).to(s["X"].dtype)
        h = H.float()
    mean = h.mean(-1, keepdim=True)
    c = h - mean
    rstd = ((c * c).mean(-1, keepdim=True) + EPS).rsqrt()
    Y = (c * rstd * s["gamma"].float() + s["beta"].float()).bfloat16()
    out = {"Y": Y}
    if H is not None:
        out["H"] = H
    if s["train"]:
        out["mean"], out["rstd"] = mean[:, 0], rstd[:, 0]
    if s["Hc"] is not None:
        out["Hv"] = _decode(_encode(h), s["b"], s["d"]).bfloat16()
    if s["Yc"] is not None:
        out["Yv"] = _decode(_encode(Y), s["b"], s["d"]).bfloat16()
    return out


def _plain_ln_bwd(s):
    x = _decode(s["X"], s["b"], s["d"]) if s["x"] == "q8" else s["X"].float()
    rstd = s["rstd"][:, None]
    x = (x - s["mean"][:, None]) * rstd
    dY = s["dY"].float()
    g = dY * s["gamma"].float()
    dX = rstd * (g - g.mean(-1, keepdim=True) - x * (g * x).mean(-1, keepdim=True))
    if s["dH"] is not None:
        dX = dX + s["dH"].float()
    return {"dX": dX.to(s["dX"].dtype), "dgamma": (dY * x).sum(0).to(s["dgamma"].dtype), "dbeta": dY.sum(0).to(s["dbeta"].dtype)}


def _kept_columns(mask, d_in):
    """Column numbers of the two kept entries of every group of four, ascending, [d_out x d_in/2]."""
    bits = (mask[:, :, None].int() >> torch.arange(8, device=mask.device, dtype=torch.int32)) & 1
    groups = bits.reshape(mask.shape[0], d_in // 4, 4)
    places = torch.sort(groups, dim=-1, descending=True, stable=True).indices[..., :2]
    return (places + 4 * torch.arange(d_in // 4, device=mask.device)[:, None]).reshape(mask.shape[0], d_in // 2)


def _plain_dw(s):
    X, dY = _decode(s["Xc"], s["b"], s["d_in"]), s["dY"].float()
    out = {"dWc": (dY.t() @ X).gather(1, _kept_columns(s["mask"], s["d_in"])).bfloat16()}
    if s["r"]:
        out["dL"], out["dR"] = (X.t() @ s["dT"].float()).bfloat16(), (s["T"].float().t() @ dY).bfloat16()
    return out


# ------------------------------------------------------------------ the framework's calls
def _own_ln_fwd(s):
    B.slope_layer_norm_fwd(s["X"], s["gamma"], s["beta"], EPS, s["Y"], mean=s["mean"], rstd=s["rstd"], residual=s["R"], H=s["H"], H_ckpt=s["Hc"],
                           Y_ckpt=s["Yc"])
    out = {"Y": s["Y"]}
    if s["H"] is not None:
        out["H"] = s["H"]
    if s["train"]:
        out["mean"], out["rstd"] = s["mean"], s["rstd"]
    if s["Hc"] is not None:
        B.slope_checkpoint_load(s["Hc"], s["Hv"])
        out["Hv"] = s["Hv"]
    if s["Yc"] is not None:
        B.slope_checkpoint_load(s["Yc"], s["Yv"])
        out["Yv"] = s["Yv"]
    return out


def _workspace(s, nbytes):
    """Scratch that a program allocates once and keeps."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_ln_bwd(s):
    ws = s.get("workspace")
    if ws is None:
        ws = _workspace(s, B.slope_layer_norm_bwd_workspace_bytes(s["b"], s["d"]))
    B.slope_layer_norm_bwd(s["dY"], s["X"], s["mean"], s["rstd"], s["gamma"], s["dX"], s["dgamma"], s["dbeta"], ws, dH=s["dH"])
    return {"dX": s["dX"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _own_dw(s):
    ws = s.get("workspace")
    if ws is None:
        ws = _workspace(s, B.slope_bwd_dw_q8_workspace_bytes(s["b"], s["d_out"], s["d_in"], s["r"]))
    if not s["r"]:
        B.slope_linear_bwd_dw_masked_q8(s["dY"], s["Xc"], s["mask"], s["dWc"], ws)
        return {"dWc": s["dWc"]}
    B.slope_linear_bwd_dw_adapter_q8(s["dY"], s["Xc"], s["T"], s["dT"], s["mask"], s["dWc"], s["dL"], s["dR"], ws)
    return {"dWc": s["dWc"], "dL": s["dL"], "dR": s["dR"]}


def run(s):
    kind = s["kind"]
    if own:
        global B
        if B is None:
            from paper_2608_24070_b200 import binding as B
        if kind == "ln_fwd":
            return _own_ln_fwd(s)
        if kind == "ln_bwd":
            return _own_ln_bwd(s)
        if kind == "dw":
            return _own_dw(s)
        B.slope_checkpoint_store(s["X"], s["Xc"])
        B.slope_checkpoint_load(s["Xc"], s["out"])
        return s["out"]
    if kind == "ln_fwd":
        return _plain_ln_fwd(s)
    if kind == "ln_bwd":
        return _plain_ln_bwd(s)
    if kind == "dw":
        return _plain_dw(s)
    return _decode(_encode(s["X"]), s["b"], s["d"]).bfloat16()


def work(case):
    size, b = {"bf16": 2, "f32": 4, "q8": 1 + 1 / BLOCK}, case["b"]
    if case["kind"] == "dw":
        d_in, d_out, r = case["d_in"], case["d_out"], case["r"]
        read = size["q8"] * b * d_in + 2 * b * d_out + d_out * d_in / 8 + 2 * 2 * b * r
        return {"bytes": read + d_out * d_in + 2 * r * (d_in + d_out), "flops": 2.0 * b * (d_in * d_out + r * (d_in + d_out))}
    n, d = b * case["d"], case["d"]
    back = n * (2 * size["q8"] + 2)                      # a checkpoint written, read, and its values written
    if case["kind"] == "ckpt":
        return {"bytes": n * size[case["x"]] + back, "flops": 0}
    if case["kind"] == "ln_fwd":
        total = n * (size[case["x"]] + 2) + 2 * d * size[case["p"]] + (8 * b if case["train"] else 0)
        if case["residual"]:
            total += n * (2 + size[case["x"]])
        total += {"none": 0, "h": 1, "y": 1, "both": 2}[case["ckpt"]] * back
        return {"bytes": total, "flops": 8.0 * n}
    total = n * (2 + size[case["x"]] + size[case["dx"]]) + 8 * b + 3 * d * size[case["p"]]
    return {"bytes": total + (n * size[case["dx"]] if case["dh"] else 0), "flops": 14.0 * n}


# ------------------------------------------------------------------ the definitions in 64 bits
def _binary_unit(k):
    """2^k in fp64 for whole k, from its bits: a power that is off by one in the last place turns ties the other way."""
    return (k.to(torch.int64) + 1023).bitwise_left_shift(52).view(torch.float64)


def _exact_checkpoint(v):
    """What a checkpoint of the fp64 matrix v reads back as, from the definition of the format."""
    blocks = v.unflatten(1, (-1, BLOCK))
    largest = blocks.abs().max(dim=-1, keepdim=True).values
    m, e = torch.frexp(largest.nan_to_num(0.0, 0.0) / 127.5)             # largest / 127.5 = m 2^e, 1/2 <= m < 1
    # the smallest k with largest <= 127.5 2^k: e, or e - 1 where m is 1/2 itself
    unit = _binary_unit(torch.where(m == 0.5, e - 1, e).where(largest > 0, torch.full_like(e, -126)).clamp(-126, 121))
    got = torch.clamp(torch.round(blocks / unit), -127.0, 127.0) * unit
    return torch.where(torch.isfinite(largest), got, torch.full_like(got, math.nan)).flatten(1)


def _exact_stored(c, rows, cols):
    """The values that a checkpoint in memory stands for, in fp64."""
    code = c.narrow(0, 0, rows * cols).view(torch.int8).double()
    k = c.narrow(0, rows * cols, rows * cols // BLOCK).double() - 127.0
    return (code.view(-1, BLOCK) * torch.where(k > 127, math.nan, _binary_unit(k)).unsqueeze(1)).view(rows, cols)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "ckpt":
        return _exact_checkpoint(s["X"].double())
    if kind == "dw":
        X, dY = _exact_stored(s["Xc"], s["b"], s["d_in"]), s["dY"].double()
        kept = torch.stack([(s["mask"] >> j) & 1 for j in range(8)], dim=2).reshape(s["d_out"], s["d_in"]).bool()
        out = {"dWc": torch.mm(dY.T, X)[kept].view(s["d_out"], -1)}
        if s["r"]:
            out["dL"], out["dR"] = torch.mm(X.T, s["dT"].double()), torch.mm(s["T"].double().T, dY)
        return out
    gamma = s["gamma"].double()
    if kind == "ln_fwd":
        h = s["X"].double()
        out = {}
        if s["R"] is not None:
            # the stream that the layer norm sees is the one that is stored
            h = (h + s["R"].double()).to(s["X"].dtype).double()
            out["H"] = h
        var, mean = torch.var_mean(h, dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        out["Y"] = torch.addcmul(s["beta"].double(), (h - mean.unsqueeze(1)) * rstd.unsqueeze(1), gamma)
        if s["train"]:
            out["mean"], out["rstd"] = mean, rstd
        if s["Hc"] is not None:
            out["Hv"] = _exact_checkpoint(h)
        if s["Yc"] is not None:
            out["Yv"] = _exact_checkpoint(out["Y"].to(torch.bfloat16).double())
        return out
    h = _exact_stored(s["X"], s["b"], s["d"]) if case["x"] == "q8" else s["X"].double()
    mean, rstd, dY = s["mean"].double().unsqueeze(1), s["rstd"].double().unsqueeze(1), s["dY"].double()
    xhat = (h - mean) * rstd
    dxhat = dY * gamma
    d = case["d"]
    dX = (dxhat * d - dxhat.sum(1, keepdim=True) - xhat * (dxhat * xhat).sum(1, keepdim=True)) * rstd / d
    if s["dH"] is not None:
        dX = dX + s["dH"].double()
    return {"dX": dX, "dgamma": torch.einsum("bd,bd->d", dY, xhat), "dbeta": torch.einsum("bd->d", dY)}
