"""Pins of the float64 block oracle with layer norms (no GPU): the layer norm against torch's in float64, and the parameters' gradients of a
block against central differences of its loss."""
import numpy as np
import pytest
import torch

from paper_2608_24070_b200 import inputs as si


@pytest.fixture(scope="module")
def blk(oracle):
    from oracle import block
    return block


def test_layer_norm_is_torchs(blk):
    gen = torch.Generator().manual_seed(3)
    x, gamma, beta = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((7, 40), (40,), (40,)))
    np.testing.assert_allclose(blk.layer_norm(x * 3 + 1, gamma, beta, 1e-5), torch.nn.functional.layer_norm(x * 3 + 1, (40,), gamma, beta, 1e-5), rtol=1e-12, atol=1e-13)


def test_parameter_gradients_of_a_block_against_differences(blk):
    d, ffn, batch, seq, heads = 16, 32, 1, 4, 2
    shapes = {"q": (d, d), "k": (d, d), "v": (d, d), "o": (d, d), "gate": (ffn, d), "up": (ffn, d), "down": (d, ffn)}
    layers = {}
    for i, (name, (d_out, d_in)) in enumerate(shapes.items()):
        lay = blk.make_layer(si.gaussian_bf16((d_out, d_in), 0.3, 900 + i))
        lay.WRC = lay.WR.detach().clone()                                    # then the layer's backward is the derivative of its forward
        layers[name] = lay
    x, dout = si.gaussian_bf16((batch * seq, d), 1.0, 950), si.gaussian_bf16((batch * seq, d), 1.0, 951)
    gen = torch.Generator().manual_seed(4)
    norms = [tuple((torch.randn(d, generator=gen, dtype=torch.float64) * 0.3 + offset).requires_grad_(True) for offset in (1.0, 0.0)) for _ in range(2)]
    blk.block_fwd_bwd(x, dout, layers, batch, seq, heads, norms=norms)
    weight = torch.from_numpy(blk.bf16_to_f64(dout))

    def loss():
        with torch.no_grad():
            return float((blk.decoder_block(torch.from_numpy(blk.bf16_to_f64(x)), layers, batch, seq, heads, norms=norms) * weight).sum())

    for pair in norms:
        for p in pair:
            for i in (0, 7, 15):
                kept, step = p.data[i].item(), 1e-6
                p.data[i] = kept + step
                up = loss()
                p.data[i] = kept - step
                down = loss()
                p.data[i] = kept
                assert abs((up - down) / (2 * step) - p.grad[i].item()) <= 1e-6 * (1 + abs(p.grad[i].item()))
