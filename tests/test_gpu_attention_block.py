"""GPU: a decoder block's training step with positions and attention on the library's calls between the sparse linears, as torch autograd runs
it, against the same block in float64."""
import math

import numpy as np
import pytest
import torch

import attention_reference as ref
from paper_2608_24070_b200 import inputs as si
from test_gpu_block import compress_rows, rel

pytestmark = pytest.mark.gpu

TOL = 1.5e-2            # a path of bf16 roundings, as for the block with torch's attention (test_gpu_block)


@pytest.fixture(scope="module")
def H():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_24070_b200 import binding, block_harness, build

    build.build()
    binding.lib()
    return block_harness


def attend64(q, k, v, hd, sequences, positions, frequencies, causal=True, window=0, interleaved=False):
    """Rotation and attention in float64 under autograd."""
    if positions is not None:
        q, k = (ref.rotary(x, positions, frequencies, hd, interleaved=interleaved) for x in (q, k))
    out = torch.zeros_like(q)
    for first, n in sequences:
        cut = lambda x: x[first:first + n].reshape(n, -1, hd).permute(1, 0, 2)
        qh, kh, vh = cut(q), cut(k), cut(v)
        kh, vh = (x.repeat_interleave(qh.shape[0] // kh.shape[0], 0) for x in (kh, vh))
        S = (qh @ kh.transpose(1, 2) / math.sqrt(hd)).masked_fill(~ref.visible(n, causal, window, q.device), -math.inf)
        out = out.index_copy(0, torch.arange(first, first + n, device=q.device), (torch.softmax(S, -1) @ vh).permute(1, 0, 2).reshape(n, -1))
    return out


@pytest.mark.parametrize("r", [0, 64])
@pytest.mark.parametrize("heads,kv", [(4, 4), (8, 2)])
def test_block_step_matches_float64(H, oracle, r, heads, kv):
    from oracle import block as OB
    from paper_2608_24070_b200 import binding as B

    d, ffn, batch, seq = 512, 1408, 2, 160
    hd = d // heads
    shapes = {"q": (d, d), "k": (kv * hd, d), "v": (kv * hd, d), "o": (d, d), "gate": (ffn, d), "up": (ffn, d), "down": (d, ffn)}
    gpu, cpu = {}, {}
    for i, (name, (d_out, d_in)) in enumerate(shapes.items()):
        W = si.gaussian_bf16((d_out, d_in), 0.05, 7000 + 10 * i)
        L = si.gaussian_bf16((d_in, r), 0.02, 7003 + 10 * i) if r else None
        R = si.gaussian_bf16((r, d_out), 0.02, 7004 + 10 * i) if r else None
        cpu[name] = OB.make_layer(W, L, R)
        gpu[name] = H.SlopeLinear(B.bf16_from_bits(W), None if L is None else B.bf16_from_bits(L), None if R is None else B.bf16_from_bits(R))
    x, dout = si.gaussian_bf16((batch * seq, d), 1.0, 7101), si.gaussian_bf16((batch * seq, d), 1.0, 7102)
    frequencies = B.rotary_frequencies(hd)
    positions = torch.arange(seq, dtype=torch.int32).repeat(batch)
    # the oracle's block, its attention replaced
    plain = OB.causal_attention
    OB.causal_attention = lambda q, k, v, *_: attend64(q, k, v, hd, [(0, seq), (seq, seq)], positions, frequencies.cpu())
    try:
        out_o, dx_o, grads_o = OB.block_fwd_bwd(x, dout, cpu, batch, seq, heads)
    finally:
        OB.causal_attention = plain
    attention = H.Attention(heads, kv, frequencies)
    out_g, dx_g = H.block_step(B.bf16_from_bits(x), B.bf16_from_bits(dout), gpu, batch, seq, heads, attention=attention, positions=positions.cuda())
    assert B.slope_poll_status() == 0
    f = lambda t: t.float().cpu().numpy()
    errs = {"out": rel(f(out_g), out_o), "dx": rel(f(dx_g), dx_o)}
    for name in H.LAYER_NAMES:
        errs[f"dWc.{name}"] = rel(f(gpu[name].dWc), compress_rows(grads_o[name]["dW"], cpu[name].mask1.numpy().astype(bool)))
        if r:
            errs[f"dL.{name}"], errs[f"dR.{name}"] = rel(f(gpu[name].dL), grads_o[name]["dL"]), rel(f(gpu[name].dR), grads_o[name]["dR"])
    print({k: round(v, 5) for k, v in errs.items()})
    bad = {k: v for k, v in errs.items() if not v <= TOL}
    assert not bad, bad


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("batch", ["equal", "padded", "packed"])
def test_gradients_through_rotation_and_attention(H, interleaved, batch):
    """Against autograd in float64.  Roundings: turned queries and keys, P, dS, O, and each output once: six of 2^-8 / sqrt(3) at most."""
    hd, heads, kv, b = 64, 4, 2, 600
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    where = {"equal": dict(sequences=3), "padded": dict(sequences=3, lengths=on([200, 37, 0])), "packed": dict(starts=on([0, 129, 400, 590]))}[batch]
    sequences = {"equal": [(0, 200), (200, 200), (400, 200)], "padded": [(0, 200), (200, 37)], "packed": [(0, 129), (129, 271), (400, 190)]}[batch]
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda n: torch.randn(b, n * hd, device="cuda", generator=gen).bfloat16()
    q, k, v, g = new(heads), new(kv), new(kv), new(heads)
    positions = torch.arange(b, dtype=torch.int32, device="cuda")
    from paper_2608_24070_b200 import binding as B

    frequencies = B.rotary_frequencies(32)
    attention = H.Attention(heads, kv, frequencies, interleaved=interleaved, window=100)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    out = attention(*leaves, positions=positions, **where)
    out.backward(g)
    assert B.slope_poll_status() == 0
    exact = [t.double().requires_grad_(True) for t in (q, k, v)]
    want = attend64(*exact, hd, sequences, positions, frequencies, True, 100, interleaved)
    want.backward(g.double())
    inside = torch.zeros(b, dtype=torch.bool, device="cuda")
    for first, n in sequences:
        inside[first:first + n] = True
    for got, ref64 in ((out.detach(), want.detach()), *((a.grad, e.grad) for a, e in zip(leaves, exact))):
        assert not got[~inside].any()
        assert float((got.double() - ref64)[inside].norm() / ref64[inside].norm()) <= 6 * 2.0 ** -8 / math.sqrt(3)


def test_refusals_and_second_derivative(H):
    from paper_2608_24070_b200 import binding as B

    q = torch.randn(32, 128, device="cuda").bfloat16().requires_grad_(True)
    with pytest.raises(ValueError, match="belong together"):
        H.Attention(2)(q, q, q, positions=torch.arange(32, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="heads"):
        H.Attention(2, 1)(q, q, q)
    (g,) = torch.autograd.grad(H.Attention(2)(q, q, q).float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        g.float().sum().backward()
    ok = torch.empty(32, 128, device="cuda", dtype=torch.bfloat16)
    f = B.rotary_frequencies(64)
    pos = torch.arange(32, dtype=torch.int32, device="cuda")
    k = q.detach()
    for call in (lambda: B.slope_attention_fwd(k, k[:16], k[:16], 64, ok), lambda: B.slope_attention_fwd(k, k, k, 60, ok),
                 lambda: B.slope_attention_fwd(k, k, k, 64, ok, torch.empty(1, 32, device="cuda")),
                 lambda: B.slope_attention_fwd(k, k, k, 64, ok, starts=pos[:3], sequences=3), lambda: B.slope_rotary(k, None, pos[:5], f, 64, ok, None),
                 lambda: B.slope_rotary(k, k, pos, f, 64, ok, None)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.slope_attention_fwd(k.float(), k, k, 64, ok), lambda: B.slope_attention_fwd(k, k, k, 64, ok, starts=pos[:3].long()),
                 lambda: B.slope_rotary(k, None, pos, f.float(), 64, ok, None), lambda: B.slope_rotary(k.half(), None, pos, f, 64, ok.half(), None)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.slope_attention_fwd(k.T, k, k, 64, ok), lambda: B.slope_attention_fwd(k.cpu(), k, k, 64, ok)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: B.slope_attention_fwd(k, k, k, 64, ok, window=3, causal=False), lambda: B.slope_attention_fwd(k, k, k, 64, ok, sequences=5),
                 lambda: B.slope_attention_fwd(k, k, k, 64, ok, scale=0.0), lambda: B.slope_attention_fwd(k[:, 2:66], k[:, :64], k[:, :64], 64, ok[:, :64])):
        with pytest.raises(B.SlopeError):
            call()
    assert B.slope_poll_status() == 0


def test_a_step_in_a_graph(H):
    """Forward and backward of rotation and attention, captured and replayed on other inputs."""
    from paper_2608_24070_b200 import binding as B

    hd, heads, b = 64, 4, 256
    frequencies, positions = B.rotary_frequencies(hd), torch.arange(b, dtype=torch.int32, device="cuda") % 128
    attention = H.Attention(heads, None, frequencies)
    gen = torch.Generator(device="cuda").manual_seed(4)
    new = lambda: torch.randn(b, heads * hd, device="cuda", generator=gen).bfloat16()
    q, k, v, g = (new().requires_grad_(i < 3) for i in range(4))

    def step():
        out = attention(q, k, v, sequences=2, positions=positions)
        return (out, *torch.autograd.grad(out, (q, k, v), g))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    with torch.no_grad():
        for t in (q, k, v, g):
            t.copy_(new())
    graph.replay()
    want = step()
    for a, b_ in zip(kept, want):
        assert torch.equal(a, b_)
    assert B.slope_poll_status() == 0
