"""GPU: which of the forward pass's kernels takes a batch."""
import pytest

import attention_reference as ref
from test_gpu_attention import B, tensors  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu


def kernel_of(call):
    """The template arguments of the attention kernel that a call launches."""
    import torch
    from torch.profiler import ProfilerActivity, profile

    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    found = [e.name.split("attention_fwd_kernel")[1].split("(")[0] for e in p.events() if "attention_fwd_kernel" in e.name]
    if not found:
        pytest.skip("the profiler does not show kernels here")
    assert len(found) == 1
    return found[0]


@pytest.mark.parametrize("hd,sequences,n,heads", [(64, 4, 4096, 16), (64, 8, 3000, 16), (128, 16, 1024, 8), (128, 32, 700, 8)])
def test_a_window_as_long_as_the_sequences_is_none(B, hd, sequences, n, heads):  # noqa: F811
    import torch

    Q, K, V, _ = tensors(sequences * n, heads, heads, hd, 51)
    O, P = torch.empty_like(Q), torch.empty_like(Q)
    plain = kernel_of(lambda: B.slope_attention_fwd(Q, K, V, hd, O, sequences=sequences))
    for window in (n, n + 1, 2 * n):
        assert kernel_of(lambda: B.slope_attention_fwd(Q, K, V, hd, P, sequences=sequences, window=window)) == plain
        assert torch.equal(O, P)
    assert B.slope_poll_status() == 0


@pytest.mark.parametrize("hd,sequences,n,heads,window", [(64, 2, 5200, 8, 4100), (64, 3, 6000, 8, 3001), (128, 3, 2000, 10, 999)])
def test_windows_in_blocks_of_two_tiles(B, hd, sequences, n, heads, window):  # noqa: F811
    """The second tile's first keys may lie behind the first one's."""
    import torch

    Q, K, V, _ = tensors(sequences * n, heads, heads // 2, hd, 52)
    O, lse = torch.full_like(Q, 7.0), torch.full((heads, sequences * n), 7.0, device="cuda")
    call = lambda: B.slope_attention_fwd(Q, K, V, hd, O, lse, sequences=sequences, window=window)
    name = kernel_of(call)
    assert name.replace(" ", "") == f"<{hd},2>"
    assert B.slope_poll_status() == 0
    want = ref.attention(Q, K, V, hd, [(i * n, n) for i in range(sequences)], True, window)
    ref.check(O, want["O"], "O")
    ref.check(lse, want["lse"], "lse")
