"""GPU: positions, starts, lengths, frequencies and lse may be parts of longer vectors, from any element on."""
import pytest

from test_gpu_attention import B, run, tensors  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu


def part_of_longer(t, at, pad):
    """The values of `t` behind `at` others."""
    import torch

    flat = torch.cat([torch.full((at,), pad, dtype=t.dtype, device=t.device), t.reshape(-1), torch.full((5,), pad, dtype=t.dtype, device=t.device)])
    return flat[at:at + t.numel()].reshape(t.shape)


@pytest.mark.parametrize("at", [1, 2, 3, 4])
def test_rotation(B, at):  # noqa: F811
    import torch

    Q, K, _, _ = tensors(9, 4, 2, 64, 61)
    positions, f = torch.arange(40, 49, dtype=torch.int32, device="cuda"), B.rotary_frequencies(64)
    want = [torch.empty_like(Q), torch.empty_like(K)]
    B.slope_rotary(Q, K, positions, f, 64, *want)
    got = [torch.empty_like(Q), torch.empty_like(K)]
    B.slope_rotary(Q, K, part_of_longer(positions, at, 7), part_of_longer(f, at, 0.5), 64, *got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_decoding_loop(B):  # noqa: F811
    """One token after the other, its position a part of all of them; in a graph, too."""
    import torch

    n, hd = 11, 64
    Q, K, _, _ = tensors(n, 4, 2, hd, 62)
    positions, f = torch.arange(n, dtype=torch.int32, device="cuda") + 1000, B.rotary_frequencies(hd)
    want, got = ([torch.empty_like(Q), torch.empty_like(K)] for _ in range(2))
    B.slope_rotary(Q, K, positions, f, hd, *want)
    for t in range(n):
        row = slice(t, t + 1)
        B.slope_rotary(Q[row], K[row], positions[row], f, hd, got[0][row], got[1][row])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(Q)
    with torch.cuda.graph(graph):
        B.slope_rotary(Q[:8], None, positions[3:11], f, hd, out[:8], None)
    positions += 5
    graph.replay()
    want8 = torch.empty_like(Q)
    B.slope_rotary(Q[:8], None, positions[3:11].clone(), f, hd, want8[:8], None)
    assert torch.equal(out[:8], want8[:8])
    assert B.slope_poll_status() == 0


@pytest.mark.parametrize("at", [1, 2, 3])
def test_attention(B, at):  # noqa: F811
    import torch

    on = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    Q, K, V, dO = tensors(300, 2, 1, 64, 63)
    starts, lengths = on(0, 100, 290), on(70, 190)
    want = run(B, Q, K, V, dO, 64, starts=starts, lengths=lengths)
    lse = part_of_longer(want["lse"], at, 3.0)
    batch = {"starts": part_of_longer(starts, at, -9), "lengths": part_of_longer(lengths, at, 999)}
    O, grads = torch.full_like(Q, 7.0), [torch.full_like(x, 7.0) for x in (Q, K, V)]
    B.slope_attention_fwd(Q, K, V, 64, O, **batch)
    ws = torch.empty(B.slope_attention_bwd_workspace_bytes(300, 2, 1, 64), dtype=torch.uint8, device="cuda")
    B.slope_attention_bwd(dO, Q, K, V, O, lse, 64, *grads, ws, **batch)
    assert B.slope_poll_status() == 0
    for x, name in zip((O, *grads), ("O", "dQ", "dK", "dV")):
        assert torch.equal(x, want[name]), name


def test_what_stays_refused(B):  # noqa: F811
    """Matrices, the workspace, and an lse that is written: their 16 bytes are needed or cannot be had by a copy."""
    import torch

    Q, K, V, dO = tensors(40, 2, 1, 64, 64)
    lse = torch.empty(2 * 40 + 1, device="cuda")[1:].view(2, 40)
    with pytest.raises(B.SlopeError, match="ALIGNMENT"):
        B.slope_attention_fwd(Q, K, V, 64, torch.empty_like(Q), lse)
    with pytest.raises(B.SlopeError, match="ALIGNMENT"):
        B.slope_attention_fwd(torch.empty(40 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(40, 128), K, V, 64, torch.empty_like(Q))
    ws = torch.empty(B.slope_attention_bwd_workspace_bytes(40, 2, 1, 64) + 4, dtype=torch.uint8, device="cuda")[4:]
    with pytest.raises(B.SlopeError, match="ALIGNMENT"):
        B.slope_attention_bwd(dO, Q, K, V, Q, torch.empty(2, 40, device="cuda"), 64, Q, K, V, ws)
