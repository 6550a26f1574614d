"""GPU: a decoder block's training step with layer norms in front of the sparse linears, against the float64 block oracle: everything in
bf16, and with the inputs of the linears and the stream kept in 8 bits for the backward pass.

Tolerance: 1.5e-2 for a path of bf16 roundings as in the block without layer norms (test_gpu_block).  Codes add an independent error to the weight gradients and
to dgamma: a code is off by at most half a unit of 2^k, 2^k / sqrt(12) in the mean square, and 2^k is at most 1 / 63.75 of a block's
largest magnitude, which for 32 Gaussian values is 2.1 sigma on average and seldom above 3: 0.95e-2 to 1.4e-2 sigma at the most, 0.8e-2 over
all positions of the largest magnitude between two powers of two.  Root of the sum of squares with 1.4e-2: 2.1e-2.
"""
import numpy as np
import pytest

from paper_2608_24070_b200 import inputs as si
from test_gpu_block import compress_rows, rel

pytestmark = pytest.mark.gpu

TOL = {False: 1.5e-2, True: 2.1e-2}


@pytest.fixture(scope="module")
def H():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_24070_b200 import binding, block_harness, build

    build.build()
    binding.lib()
    return block_harness


def model(H, r, checkpoint, oracle_block=None):
    import torch
    from paper_2608_24070_b200 import binding as B

    d, ffn = 512, 1408
    shapes = {"q": (d, d), "k": (d, d), "v": (d, d), "o": (d, d), "gate": (ffn, d), "up": (ffn, d), "down": (d, ffn)}
    gpu, cpu = {}, {}
    for i, (name, (d_out, d_in)) in enumerate(shapes.items()):
        W = si.gaussian_bf16((d_out, d_in), 0.02, 5000 + 10 * i)
        L = si.gaussian_bf16((d_in, r), 0.01, 5003 + 10 * i) if r else None
        R = si.gaussian_bf16((r, d_out), 0.01, 5004 + 10 * i) if r else None
        if oracle_block:
            cpu[name] = oracle_block.make_layer(W, L, R)
        gpu[name] = H.SlopeLinear(B.bf16_from_bits(W), None if L is None else B.bf16_from_bits(L), None if R is None else B.bf16_from_bits(R),
                                  checkpoint=checkpoint)
    gen = torch.Generator().manual_seed(7)
    params = [[(1 + 0.2 * torch.randn(d, generator=gen)).bfloat16(), (0.2 * torch.randn(d, generator=gen)).bfloat16()] for _ in range(2)]
    norms = {n: H.LayerNorm(g.cuda(), b.cuda(), checkpoint=checkpoint) for n, (g, b) in zip(("attention", "mlp"), params)}
    return gpu, norms, cpu, params


@pytest.mark.parametrize("r", [0, 64])
@pytest.mark.parametrize("checkpoint", [False, True])
def test_block_step_with_layer_norms_matches_the_oracle(H, oracle, r, checkpoint):
    import torch
    from oracle import block as OB
    from paper_2608_24070_b200 import binding as B

    d, batch, seq, heads = 512, 2, 128, 4
    gpu, norms, cpu, params = model(H, r, checkpoint, OB)
    exact = [tuple(p.double().requires_grad_(True) for p in pair) for pair in params]
    x, dout = si.gaussian_bf16((batch * seq, d), 1.0, 5101), si.gaussian_bf16((batch * seq, d), 1.0, 5102)
    out_o, dx_o, grads_o = OB.block_fwd_bwd(x, dout, cpu, batch, seq, heads, norms=exact)
    out_g, dx_g = H.block_step(B.bf16_from_bits(x), B.bf16_from_bits(dout), gpu, batch, seq, heads, norms=norms)
    assert B.slope_poll_status() == 0
    f = lambda t: t.float().cpu().numpy()
    errs = {"out": rel(f(out_g), out_o), "dx": rel(f(dx_g), dx_o)}
    for (name, norm), (g, b) in zip(norms.items(), exact):
        errs[f"dgamma.{name}"], errs[f"dbeta.{name}"] = rel(f(norm.dgamma), g.grad.numpy()), rel(f(norm.dbeta), b.grad.numpy())
    for name in H.LAYER_NAMES:
        errs[f"dWc.{name}"] = rel(f(gpu[name].dWc), compress_rows(grads_o[name]["dW"], cpu[name].mask1.numpy().astype(bool)))
        if r:
            errs[f"dL.{name}"], errs[f"dR.{name}"] = rel(f(gpu[name].dL), grads_o[name]["dL"]), rel(f(gpu[name].dR), grads_o[name]["dR"])
    print({k: round(v, 5) for k, v in errs.items()})
    bad = {k: v for k, v in errs.items() if not v <= TOL[checkpoint]}
    assert not bad, bad


def test_what_a_step_keeps(H):
    """With checkpoints the linears and layer norms keep no bf16 copy of their inputs: 33 bytes for 32 values, shared where the input is shared."""
    import torch
    from paper_2608_24070_b200 import binding as B

    d, ffn, tokens = 512, 1408, 256
    kept = {}
    for checkpoint in (False, True):
        gpu, norms, _, _ = model(H, 0, checkpoint)
        seen = {}

        def pack(t):
            seen[t.data_ptr()] = t.dtype, t.numel()
            return t

        x = B.bf16_from_bits(si.gaussian_bf16((tokens, d), 1.0, 5201)).requires_grad_(True)
        with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
            stream, n1, c = norms["attention"](x)
            q = gpu["q"](n1, c), gpu["k"](n1, c)
            h, n2, c2 = norms["mlp"](stream, gpu["o"](q[0] * q[1]))
            out = h + gpu["down"](gpu["gate"](n2, c2) * gpu["up"](n2, c2))
        out.sum().backward()
        kept[checkpoint] = sorted(n for t, n in seen.values() if t == torch.uint8)
    assert kept[False] == []
    # stream and output of either layer norm, inputs of o and down
    assert kept[True] == sorted([tokens * d * 33 // 32] * 5 + [tokens * ffn * 33 // 32])


def test_a_stream_in_fp32(H):
    """The stream may be fp32 between bf16 sub-layers; a layer norm whose output nobody uses passes the stream's gradient on."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(8)
    new = lambda *s: torch.randn(s, device="cuda", generator=gen)
    norm = H.LayerNorm(1 + 0.1 * new(768), 0.1 * new(768), checkpoint=True)
    x, r = new(65, 768).requires_grad_(True), new(65, 768).bfloat16().requires_grad_(True)
    h, y, _ = norm(x, r)
    weights = new(65, 768), new(65, 768).bfloat16()
    ((h * weights[0]).sum() + (y * weights[1]).float().sum()).backward()
    x64, r64 = x.detach().double().requires_grad_(True), r.detach().double().requires_grad_(True)
    h64 = x64 + r64
    g64, b64 = norm.gamma.double().requires_grad_(True), norm.beta.double().requires_grad_(True)
    y64 = torch.nn.functional.layer_norm(h64, (768,), g64, b64, norm.eps)
    ((h64 * weights[0].double()).sum() + (y64 * weights[1].double()).sum()).backward()
    off = lambda a, b: float((a.double() - b).norm() / b.norm())
    # dX is a sum of the stream's gradient and the layer norm's, which knows xhat to 1.4e-2 (its term with xhat is a 1/768 share)
    assert off(x.grad, x64.grad) <= 2e-3 and off(r.grad, r64.grad) <= 2.0 ** -8 + 2e-3
    assert off(norm.dgamma, g64.grad) <= 1.4e-2 and off(norm.dbeta, b64.grad) <= 1e-5
    x.grad = r.grad = None
    h, y, _ = norm(x, r)
    (h * weights[0]).sum().backward()
    assert torch.equal(x.grad, weights[0]) and not norm.dgamma.any()
