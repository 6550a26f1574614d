"""Rotary positions and softmax attention between the linear layers of a block, as cases that can be timed and compared.

Three kinds of pass, on matrices [tokens x heads * head_dim] as the linear layers write and read them:

* ``rotary``    queries and keys turned by their positions, or the gradients turned back: pairs of a head half a rotated part apart or
                next to each other, all of the head or its first columns, positions anywhere in 31 bits, frequencies as the caller has them;
* ``attn_fwd``  O = softmax(scale Q K^T) V per sequence and head, and the logarithm of every row's sum;
* ``attn_bwd``  dQ, dK and dV from dO, Q, K, V, O and those logarithms: the probabilities are formed once more.

Sequences lie behind one another: all of one length, of several lengths with their starts given, or each at the front of a place of its own
(a padded batch).  A token sees its sequence, with ``causal`` up to itself, with a window at most that many of them.  Query heads share
key and value heads evenly.  Rows of no sequence are neither read for others nor written.
"""
import math
import random

import torch

own = False            # True: the calls of the framework's binding; False: the same in elementary torch operations
B = None


def listed():
    rot = lambda **k: {"kind": "rotary", "layout": "half", "type": "bf16", "back": False, "base": 10000.0, "stretch": 1.0, "offset": 0, **k}
    att = lambda **k: {"causal": True, "window": 0, "batch": "equal", **k}
    return [
        # decoding one sequence of a 7B-wide model: one token far from the start, bound by the cost of a call
        rot(name="rotary_decode", b=1, heads=32, kv=32, hd=128, rot=128, offset=3900),
        # a small model that rotates a quarter of 80 columns, neighbours paired, ragged batch
        rot(name="rotary_partial", b=2039, heads=32, kv=32, hd=80, rot=20, layout="pairs"),
        # gradients of a 7B-wide block at its pretraining batch, on their way back to the projections
        rot(name="rotary_7b_back", b=16384, heads=32, kv=32, hd=128, rot=128, back=True),
        # shared key heads, an fp32 stream, a context stretched to eight times what the model was trained on
        rot(name="rotary_long", b=8191, heads=32, kv=8, hd=128, rot=128, type="f32", base=500000.0, stretch=8.0, offset=100000),
        # one short prompt of a GPT-2-small-wide model
        att(name="fwd_short", kind="attn_fwd", seqs=1, len=128, heads=12, kv=12, hd=64),
        # that model's pretraining batch
        att(name="fwd_gpt2", kind="attn_fwd", seqs=8, len=1024, heads=12, kv=12, hd=64),
        # BERT-Large's width: every token sees its whole sequence, padded batch
        att(name="fwd_padded", kind="attn_fwd", seqs=32, len=512, heads=16, kv=16, hd=64, causal=False, batch="padded"),
        # a LLaMA-13B block's batch
        att(name="fwd_13b", kind="attn_fwd", seqs=4, len=2048, heads=40, kv=40, hd=128),
        # the backward pass of the short prompt
        att(name="bwd_short", kind="attn_bwd", seqs=1, len=128, heads=12, kv=12, hd=64),
        # of GPT-2-small's batch
        att(name="bwd_gpt2", kind="attn_bwd", seqs=8, len=1024, heads=12, kv=12, hd=64),
        # of documents packed behind one another, shared key heads and a window, as a 7B model of that kind trains
        att(name="bwd_packed", kind="attn_bwd", seqs=5, len=6000, heads=32, kv=8, hd=128, batch="packed", window=4096),
        # of one long document
        att(name="bwd_long", kind="attn_bwd", seqs=1, len=16384, heads=32, kv=8, hd=128),
    ]


_MOST = 32 * 128 * 16384 * 16384 / 2      # pairs x heads x columns of the largest listed case


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choices(["rotary", "attn_fwd", "attn_bwd"], [3, 4, 4])[0]
    hd = rng.choice([32, 64, 64, 64, 80, 96, 112, 128, 128, 128])
    heads = rng.choice([1, 4, 8, 12, 16, 25, 32, 40])
    kv = heads // rng.choice([g for g in (1, 1, 1, 2, 4, 8, heads) if heads % g == 0])
    if kind == "rotary":
        b = round(_log_uniform(rng, 1, 16384 * 4096 / max(4096, heads * hd)))
        return {"kind": kind, "b": b, "heads": heads, "kv": kv, "hd": hd, "rot": rng.choice([hd, hd, hd, hd // 2, hd // 4]),
                "layout": rng.choice(["half", "pairs"]), "type": rng.choice(["bf16", "bf16", "f32"]), "back": rng.random() < 0.4,
                "base": rng.choice([10000.0, 500000.0]), "stretch": rng.choice([1.0, 1.0, 4.0, 8.0]), "offset": rng.choice([0, 0, 4000, 1000000])}
    batch = rng.choice(["equal", "equal", "padded", "packed"])
    seqs = round(_log_uniform(rng, 1, 32))
    longest = min(16384 / seqs, math.sqrt(2 * _MOST / (heads * hd * seqs)))
    # (a token that sees itself alone has gradients of exactly zero for its query and key: nothing that could be compared relative to its size)
    least = 1 if kind == "attn_fwd" else 8
    length = max(least, round(_log_uniform(rng, least, longest)))
    causal = rng.random() < 0.7
    window = round(_log_uniform(rng, least, 2 * length)) if causal and rng.random() < 0.3 else 0
    return {"kind": kind, "seqs": seqs, "len": length, "heads": heads, "kv": kv, "hd": hd, "causal": causal, "window": window, "batch": batch}


def _sequences(case):
    """[(first row, length)] and the number of rows."""
    n, most = case["seqs"], case["len"]
    if case["batch"] == "equal":
        return [(i * most, most) for i in range(n)], n * most
    rng = random.Random(n * 1000003 + most)
    lengths = [rng.randint(max(1, most // 8), most) for _ in range(n)]
    if case["batch"] == "padded":
        return [(i * most, length) for i, length in enumerate(lengths)], n * most
    firsts = [sum(lengths[:i]) for i in range(n)]
    return list(zip(firsts, lengths)), sum(lengths) + 5          # five rows behind the last sequence


def _pairs(case):
    """Query and key pairs that meet, per head."""
    total = 0
    for _, n in _sequences(case)[0]:
        if not case["causal"]:
            total += n * n
        else:
            w = min(case["window"] or n, n)
            total += w * (w + 1) // 2 + (n - w) * w
    return total


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _frequencies(case):
    """Radians a position, fp64: base^(-2 i / rot); of a stretched context the slow ones are divided by the stretch, with a ramp between
    those that turn 32 times and once within 8192 positions."""
    n = case["rot"] // 2
    f = torch.tensor([case["base"] ** (-i / n) for i in range(n)], dtype=torch.float64)
    turns = 8192.0 * f / (2.0 * math.pi)
    keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / case["stretch"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    s = dict(case)
    heads, kv, hd = case["heads"], case["kv"], case["hd"]

    def projected(b, n, t=torch.bfloat16, sigma=1.0):
        """What a projection writes: columns of unlike size, heads of unlike size."""
        x = new(b, n, hd) * torch.exp(0.3 * new(hd)) * (torch.exp(0.2 * new(n, 1)) * sigma)
        return x.reshape(b, n * hd).to(t)

    if case["kind"] == "rotary":
        b, t = case["b"], _TYPES[case["type"]]
        sigma = 0.02 if case["back"] else 1.0
        s["Q"], s["K"] = projected(b, heads, t, sigma), projected(b, kv, t, sigma)
        s["Qr"], s["Kr"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
        s["frequencies"] = _frequencies(case).cuda()
        s["factor"] = 1.0 if case["stretch"] == 1.0 else 0.1 * math.log(case["stretch"]) + 1.0
        # documents of a packed batch, each from its own start
        period = max(1, min(b, 4096))
        s["positions"] = (torch.arange(b, device="cuda") % period + (case["offset"] + seed % 97)).int()
        return s
    sequences, b = _sequences(case)
    s["sequences"], s["scale"] = sequences, 1.0 / math.sqrt(hd)
    s["Q"], s["K"], s["V"] = projected(b, heads), projected(b, kv), projected(b, kv)
    s["starts"] = s["lengths"] = None
    if case["batch"] == "packed":
        s["starts"] = torch.tensor([first for first, _ in sequences] + [sequences[-1][0] + sequences[-1][1]], dtype=torch.int32).cuda()
    if case["batch"] == "padded":
        s["lengths"] = torch.tensor([n for _, n in sequences], dtype=torch.int32).cuda()
    empty = lambda t: torch.zeros_like(t)                 # (rows of no sequence stay as they are)
    s["O"], s["lse"] = empty(s["Q"]), torch.zeros(heads, b, device="cuda")
    if case["kind"] == "attn_bwd":
        out = _plain_fwd(s)
        s["O"], s["lse"] = out["O"], out["lse"]
        s["dO"] = projected(b, heads, sigma=0.02)
        s["dQ"], s["dK"], s["dV"] = empty(s["Q"]), empty(s["K"]), empty(s["V"])
    return s


# ------------------------------------------------------------------ the plain forms
def _plain_rotary(s):
    angle = s["positions"].double()[:, None] * s["frequencies"]
    cos, sin = (angle.cos() * s["factor"]).float()[:, None], (angle.sin() * s["factor"]).float()[:, None]
    if s["back"]:
        sin = -sin
    rot, out = s["rot"], {}
    for name in ("Q", "K"):
        x = s[name].float().reshape(s["b"], -1, s["hd"])
        y = x.clone()
        if s["layout"] == "half":
            u, v = x[..., :rot // 2], x[..., rot // 2:rot]
            y[..., :rot // 2], y[..., rot // 2:rot] = u * cos - v * sin, v * cos + u * sin
        else:
            u, v = x[..., 0:rot:2], x[..., 1:rot:2]
            y[..., 0:rot:2], y[..., 1:rot:2] = u * cos - v * sin, v * cos + u * sin
        out[name] = y.reshape(s["b"], -1).to(s[name].dtype)
    return out


def _visible(s, n):
    """[n x n] truth values, or None where everything is seen."""
    if not s["causal"]:
        return None
    i = torch.arange(n, device="cuda")
    seen = i[:, None] >= i[None, :]
    return seen & (i[:, None] - i[None, :] < s["window"]) if s["window"] else seen


def _pieces(s):
    """(rows, key heads, mask) of what fits in memory at a time."""
    group = s["heads"] // s["kv"]
    for first, n in s["sequences"]:
        mask = _visible(s, n)
        step = max(1, int(2 ** 29 // (group * n * n)))
        for h in range(0, s["kv"], step):
            yield slice(first, first + n), slice(h, min(h + step, s["kv"])), mask


def _queries(s, x, rows, heads):
    """[key heads x queries that share one x rows x columns], fp32."""
    n = rows.stop - rows.start
    return x[rows].reshape(n, s["kv"], -1, s["hd"])[:, heads].permute(1, 2, 0, 3).float()


def _keys(s, x, rows, heads):
    n = rows.stop - rows.start
    return x[rows].reshape(n, s["kv"], s["hd"])[:, heads].permute(1, 0, 2)[:, None].float()


def _put(s, out, rows, heads, value):
    n = rows.stop - rows.start
    out[rows].view(n, s["kv"], -1, s["hd"])[:, heads] = value.permute(2, 0, 1, 3).to(out.dtype)


def _plain_fwd(s):
    O, lse = torch.zeros_like(s["Q"]), torch.zeros_like(s["lse"])
    for rows, heads, mask in _pieces(s):
        S = _queries(s, s["Q"], rows, heads) @ (_keys(s, s["K"], rows, heads).transpose(-1, -2) * s["scale"])
        if mask is not None:
            S.masked_fill_(~mask, -math.inf)
        m = S.amax(-1, keepdim=True)
        P = S.sub_(m).exp_()
        total = P.sum(-1, keepdim=True)
        _put(s, O, rows, heads, (P @ _keys(s, s["V"], rows, heads)) / total)
        lse.view(s["kv"], -1, lse.shape[-1])[heads, :, rows] = (m + total.log())[..., 0]
    return {"O": O, "lse": lse}


def _plain_bwd(s):
    dQ, dK, dV = torch.zeros_like(s["Q"]), torch.zeros_like(s["K"]), torch.zeros_like(s["V"])
    for rows, heads, mask in _pieces(s):
        Q, dO = _queries(s, s["Q"], rows, heads), _queries(s, s["dO"], rows, heads)
        K = _keys(s, s["K"], rows, heads)
        P = Q @ (K.transpose(-1, -2) * s["scale"])
        P.sub_(s["lse"].view(s["kv"], -1, s["lse"].shape[-1])[heads, :, rows, None])
        if mask is not None:
            P.masked_fill_(~mask, -math.inf)
        P.exp_()
        _put(s, dV, rows, heads, (P.transpose(-1, -2) @ dO).sum(1, keepdim=True))
        D = (dO * _queries(s, s["O"], rows, heads)).sum(-1, keepdim=True)
        dS = (dO @ _keys(s, s["V"], rows, heads).transpose(-1, -2)).sub_(D).mul_(P).mul_(s["scale"])
        _put(s, dQ, rows, heads, dS @ K)
        _put(s, dK, rows, heads, (dS.transpose(-1, -2) @ Q).sum(1, keepdim=True))
    return {"dQ": dQ, "dK": dK, "dV": dV}


# ------------------------------------------------------------------ the framework's calls
def _batch(s):
    return {"sequences": s["seqs"], "starts": s["starts"], "lengths": s["lengths"], "causal": s["causal"], "window": s["window"], "scale": s["scale"]}


def _own_rotary(s):
    B.slope_rotary(s["Q"], s["K"], s["positions"], s["frequencies"], s["hd"], s["Qr"], s["Kr"], factor=s["factor"],
                   interleaved=s["layout"] == "pairs", backward=s["back"])
    return {"Q": s["Qr"], "K": s["Kr"]}


def _own_fwd(s):
    B.slope_attention_fwd(s["Q"], s["K"], s["V"], s["hd"], s["O"], s["lse"], **_batch(s))
    return {"O": s["O"], "lse": s["lse"]}


def _own_bwd(s):
    ws = s.get("workspace")
    if ws is None:                                        # scratch that a program allocates once and keeps
        n = B.slope_attention_bwd_workspace_bytes(s["Q"].shape[0], s["heads"], s["kv"], s["hd"])
        ws = s["workspace"] = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    B.slope_attention_bwd(s["dO"], s["Q"], s["K"], s["V"], s["O"], s["lse"], s["hd"], s["dQ"], s["dK"], s["dV"], ws, **_batch(s))
    return {"dQ": s["dQ"], "dK": s["dK"], "dV": s["dV"]}


def run(s):
    kind = s["kind"]
    if own:
        global B
        if B is None:
            from paper_2608_24070_b200 import binding as B
        return {"rotary": _own_rotary, "attn_fwd": _own_fwd, "attn_bwd": _own_bwd}[kind](s)
    return {"rotary": _plain_rotary, "attn_fwd": _plain_fwd, "attn_bwd": _plain_bwd}[kind](s)


def work(case):
    heads, kv, hd = case["heads"], case["kv"], case["hd"]
    if case["kind"] == "rotary":
        n = case["b"] * (heads + kv)
        return {"bytes": 2 * n * hd * (2 if case["type"] == "bf16" else 4) + 4 * case["b"] + 4 * case["rot"], "flops": 3.0 * n * case["rot"]}
    rows = sum(n for _, n in _sequences(case)[0])
    products = 4.0 * _pairs(case) * heads * hd            # the two products of the forward pass
    if case["kind"] == "attn_fwd":
        return {"bytes": rows * (2 * 2 * heads * hd + 2 * 2 * kv * hd + 4 * heads), "flops": products}
    # Q, O, dO read and dQ written, K, V read and dK, dV written; five products
    return {"bytes": rows * (4 * 2 * heads * hd + 4 * 2 * kv * hd + 4 * heads), "flops": 2.5 * products}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_rotary(s):
    """Pairs as complex numbers, times factor e^(+-i angle)."""
    angle = torch.outer(s["positions"].double(), s["frequencies"])
    turn = torch.polar(torch.full_like(angle, float(s["factor"])), -angle if s["back"] else angle).unsqueeze(1)
    out = {}
    for name in ("Q", "K"):
        x = s[name].double().unflatten(1, (-1, s["hd"]))
        part, rest = x.split([s["rot"], s["hd"] - s["rot"]], dim=2)
        axis = 2 if s["layout"] == "half" else 3
        pair = part.unflatten(2, (2, -1) if axis == 2 else (-1, 2))
        z = torch.complex(*pair.unbind(axis)) * turn
        out[name] = torch.cat([torch.stack([z.real, z.imag], dim=axis).flatten(2), rest], dim=2).flatten(1)
    return out


def _exact_scores(s, first, n, h):
    """scale q.k of one query head's sequence, -inf where nothing is seen."""
    hd = s["hd"]
    rows = torch.arange(first, first + n, device="cuda")
    g = h // (s["heads"] // s["kv"])
    q, k = s["Q"][rows, h * hd:(h + 1) * hd].double(), s["K"][rows, g * hd:(g + 1) * hd].double()
    S = torch.einsum("id,jd->ij", q, k) * s["scale"]
    if s["causal"]:
        back = torch.arange(n, device="cuda").unsqueeze(1) - torch.arange(n, device="cuda")
        S[back < 0] = -math.inf
        if s["window"]:
            S[back >= s["window"]] = -math.inf
    return q, k, S, g


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(s)
    hd = case["hd"]
    zeros = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "attn_fwd":
        out = {"O": zeros(s["O"]), "lse": zeros(s["lse"])}
        for first, n in s["sequences"]:
            for h in range(case["heads"]):
                _, _, S, g = _exact_scores(s, first, n, h)
                out["lse"][h, first:first + n] = torch.logsumexp(S, dim=1)
                out["O"][first:first + n, h * hd:(h + 1) * hd] = torch.softmax(S, dim=1) @ s["V"][first:first + n, g * hd:(g + 1) * hd].double()
        return out
    out = {"dQ": zeros(s["dQ"]), "dK": zeros(s["dK"]), "dV": zeros(s["dV"])}
    for first, n in s["sequences"]:
        for h in range(case["heads"]):
            q, k, S, g = _exact_scores(s, first, n, h)
            at = lambda t, i: t[first:first + n, i * hd:(i + 1) * hd]
            dO = at(s["dO"], h).double()
            P = torch.exp(S - s["lse"][h, first:first + n].double().unsqueeze(1))
            del S
            D = torch.einsum("id,id->i", dO, at(s["O"], h).double())
            dS = (torch.einsum("id,jd->ij", dO, at(s["V"], g).double()) - D.unsqueeze(1)) * P
            at(out["dV"], g).addmm_(P.T, dO)
            at(out["dQ"], h).copy_(dS @ k * s["scale"])
            at(out["dK"], g).add_(dS.T @ q, alpha=s["scale"])
    return out
