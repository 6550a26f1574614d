"""GPU: matrices of more than 2^31 values.  What stands at their ends comes out as it does alone."""
import pytest

from test_gpu_attention import B, run, tensors  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu


def test_the_last_rows(B):  # noqa: F811
    import torch

    hd, heads, kv, n = 64, 32, 4, 300
    b = 2 ** 31 // (heads * hd) + 1000
    near = tensors(n, heads, kv, hd, 71)
    Q, K, V, dO = (torch.zeros(b, x.shape[1], dtype=torch.bfloat16, device="cuda") for x in near)
    for far, x in zip((Q, K, V, dO), near):
        far[:200], far[-n:] = x[:200], x
    on = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    got = run(B, Q, K, V, dO, hd, starts=on(0, b - n, b), lengths=on(200, n))
    last, first = run(B, *near, hd), run(B, *(x[:200].contiguous() for x in near), hd)
    for name in got:
        rows = lambda a, z: got[name][:, a:z] if name == "lse" else got[name][a:z]
        assert torch.equal(rows(b - n, b), last[name]) and torch.equal(rows(0, 200), first[name]), name
        assert (rows(200, 1000) == 7).all() and (rows(b - n - 1000, b - n) == 7).all(), name
    del got
    positions, f = torch.arange(b, dtype=torch.int32, device="cuda"), B.rotary_frequencies(hd)
    q, k = near[0].clone(), near[1].clone()
    B.slope_rotary(q, k, positions[-n:].clone(), f, hd, q, k)
    B.slope_rotary(Q, K, positions, f, hd, Q, K)
    assert torch.equal(Q[-n:], q) and torch.equal(K[-n:], k)
    assert B.slope_poll_status() == 0
