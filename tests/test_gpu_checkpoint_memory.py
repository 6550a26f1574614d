"""GPU: what training steps with 8-bit checkpoints hold in memory, through the block harness: the saved tensors of either kind of layer, what is left
when a step is over, and the peak.
"""
import pytest

from paper_2608_24070_b200 import inputs as si
from test_gpu_norm_block import H, model  # noqa: F401  (H: the fixture)

pytestmark = pytest.mark.gpu

D, FFN = 512, 1408


def forward(gpu, norms, x):
    """A block whose glue saves nothing (sums in the places of the products), so that all that is kept is the layers'."""
    stream, n1, c = norms["attention"](x)
    q = gpu["q"](n1, c) + gpu["k"](n1, c) + gpu["v"](n1, c)
    h, n2, c2 = norms["mlp"](stream, gpu["o"](q))
    return h + gpu["down"](gpu["gate"](n2, c2) + gpu["up"](n2, c2))


@pytest.mark.parametrize("r", [0, 64])
def test_no_copy_in_bf16_is_saved(H, r):  # noqa: F811
    """Every tensor that the layers save, of whatever type: with checkpoints none of the inputs, the stream or the outputs themselves."""
    import torch
    from paper_2608_24070_b200 import binding as B

    tokens = 256
    saved = {}
    for checkpoint in (False, True):
        gpu, norms, _, _ = model(H, r, checkpoint)
        seen = {}

        def pack(t):
            seen[t.data_ptr()] = t.dtype, t.numel()
            return t

        x = B.bf16_from_bits(si.gaussian_bf16((tokens, D), 1.0, 5301)).requires_grad_(True)
        with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
            out = forward(gpu, norms, x)
        out.sum().backward()
        saved[checkpoint] = sorted((str(t), n) for t, n in seen.values())
    statistics = [("torch.float32", tokens)] * 4
    kept = [("torch.bfloat16", tokens * r)] * 7 if r else []               # the adapters' T
    full = [("torch.bfloat16", tokens * D)] * 5 + [("torch.bfloat16", tokens * FFN)]
    codes = [("torch.uint8", tokens * D * 33 // 32)] * 5 + [("torch.uint8", tokens * FFN * 33 // 32)]
    assert saved[False] == sorted(statistics + kept + full)
    assert saved[True] == sorted(statistics + kept + codes)


def requested(which):
    """Bytes that were asked for.  (What the allocator counts as allocated depends on what ran before: a block of which less than 1 MB would be left is not split.)"""
    import torch

    return torch.cuda.memory_stats()[f"requested_bytes.all.{which}"]


def held(H, r, checkpoint, blocks=4, tokens=4096):  # noqa: F811
    """Bytes beyond the model's own: behind the second step's forward pass, when that step is over, and at its peak."""
    import torch
    from paper_2608_24070_b200 import binding as B

    layers = [model(H, r, checkpoint)[:2] for _ in range(blocks)]
    x = B.bf16_from_bits(si.gaussian_bf16((tokens, D), 1.0, 5302))
    torch.cuda.synchronize()
    start = requested("current")
    for _ in range(2):
        torch.cuda.reset_peak_memory_stats()
        out = x.detach().requires_grad_(True)
        for gpu, norms in layers:
            out = forward(gpu, norms, out)
        behind_forward = requested("current") - start
        out.sum().backward()
        del out
    return behind_forward, requested("current") - start, requested("peak") - start


@pytest.mark.parametrize("r", [0, 64])
def test_steps_with_checkpoints_hold_less(H, r):  # noqa: F811
    """A block saves five matrices of [tokens x d] and one of [tokens x ffn], 31 / 64 of which checkpoints spare (the first block's stream is the
    caller's input, which stays, so that its codes come on top: with what the caller holds of the last output the difference is exact); the backward
    pass adds one decoded matrix at a time, and the other workspaces are below 16 MB."""
    blocks, tokens = 4, 4096
    off, on = held(H, r, False, blocks, tokens), held(H, r, True, blocks, tokens)
    print("bytes behind the forward pass, behind the step, at the peak:", off, on)
    spared = blocks * 31 * 2 * tokens * (5 * D + FFN) // 64 - 2 * tokens * D
    assert on[0] == off[0] - spared if r == 0 else on[0] <= off[0] - spared
    assert on[1] == 0
    assert on[2] <= off[2] - spared + 2 * tokens * FFN + (1 << 24)


def test_a_workspace_for_the_largest_batch_is_not_taken_twice(H):  # noqa: F811
    """`max_tokens` is for the calls on bf16; a layer with checkpoints does not use that workspace."""
    import torch

    W, L, R = (torch.randn(s, device="cuda").bfloat16() for s in ((512, 512), (512, 64), (64, 512)))
    assert H.SlopeLinear(W, L, R, max_tokens=4096, checkpoint=True).workspace is None
    assert H.SlopeLinear(W, L, R, max_tokens=4096).workspace is not None


def test_layers_with_checkpoints_in_graphs_on_two_streams(H):  # noqa: F811
    """One layer and one layer norm captured twice with other inputs; the replays run side by side and have the bits of eager steps."""
    import torch
    from paper_2608_24070_b200 import binding as B

    gpu, norms, _, _ = model(H, 64, True)
    layer, norm = gpu["q"], norms["attention"]
    xs = [B.bf16_from_bits(si.gaussian_bf16((2048, D), 1.0, 5310 + k)) for k in range(2)]

    def step(x):
        x = x.detach().requires_grad_(True)
        _, y, c = norm(x)
        layer(y, c).sum().backward()
        return x.grad

    want = [step(x).clone() for x in xs]
    grads, graphs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(2):
        streams[k].wait_stream(torch.cuda.current_stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k], stream=streams[k]):
            grads.append(step(xs[k]))
    torch.cuda.synchronize()
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                graphs[k].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(grads[k], want[k]) for k in range(2))
    assert B.slope_poll_status() == 0
