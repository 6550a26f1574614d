"""GPU: the bits of a row of O and lse depend on its own query and on the keys and values that it sees, on nothing else."""
import pytest

from test_gpu_attention import B, run, tensors  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu


def forward(B, Q, K, V, hd, **batch):  # noqa: F811
    import torch

    O, lse = torch.full_like(Q, 7.0), torch.full((Q.shape[1] // hd, Q.shape[0]), 7.0, device="cuda")
    B.slope_attention_fwd(Q, K, V, hd, O, lse, **batch)
    assert B.slope_poll_status() == 0
    return O, lse


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("value", [1e3, 3.0, -40.0])
def test_finite_rows_of_no_sequence(B, value, causal):  # noqa: F811
    """Padding of large finite values: its scores rise by far more than a power of two of 16 from one tile of keys to the next."""
    import torch

    part, lengths = 700, [690, 413, 128, 5, 270]
    inside = torch.zeros(part * len(lengths), dtype=torch.bool, device="cuda")
    for i, n in enumerate(lengths):
        inside[part * i:part * i + n] = True
    batch = {"sequences": len(lengths), "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "causal": causal}
    for hd in (64, 128, 80):
        clean = tensors(part * len(lengths), 4, 2, hd, 41)
        dirty = [x.masked_fill(~inside[:, None], value) for x in clean]
        a, b = run(B, *clean, hd, **batch), run(B, *dirty, hd, **batch)
        for name in a:
            assert torch.equal(a[name], b[name]), (name, hd)


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 300), (False, 0)])
@pytest.mark.parametrize("n,heads", [(700, 4), (2600, 40)])
def test_other_queries(B, n, heads, causal, window):  # noqa: F811
    """Every third query forty times as large: the others' rows stay as they are, with one tile of queries a block and with two."""
    import torch

    keep = torch.arange(n, device="cuda") % 3 != 0
    for hd in (64, 128):
        Q, K, V, _ = tensors(n, heads, heads // 4, hd, 42)
        a = forward(B, Q, K, V, hd, causal=causal, window=window)
        b = forward(B, torch.where(keep[:, None], Q, Q * 40), K, V, hd, causal=causal, window=window)
        assert torch.equal(a[0][keep], b[0][keep]) and torch.equal(a[1][:, keep], b[1][:, keep]), hd


def test_later_tokens(B):  # noqa: F811
    """Through a causal mask: whatever tokens follow, and however many."""
    import torch

    for hd in (64, 128):
        x = tensors(900, 4, 2, hd, 43)[:3]
        a = forward(B, *x, hd)
        for n in (333, 500):
            changed = [torch.cat([t[:n], t[n:] * 30]) for t in x]
            b, c = forward(B, *changed, hd), forward(B, *(t[:n].contiguous() for t in x), hd)
            for other in (b, c):
                assert torch.equal(a[0][:n], other[0][:n]) and torch.equal(a[1][:, :n], other[1][:, :n]), (hd, n)


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1300), (False, 0)])
def test_the_batch_around(B, causal, window):  # noqa: F811
    """A sequence's head alone, in blocks of one tile of queries, and among others, in blocks of two where these fill the device."""
    import torch

    n, heads = 2600, 20
    for hd in (64, 128):
        Q, K, V, _ = tensors(3 * n, heads, heads, hd, 44)
        O, lse = forward(B, Q, K, V, hd, sequences=3, causal=causal, window=window)
        for i, h in ((0, 0), (1, 7), (2, 19)):
            rows, cols = slice(i * n, i * n + n), slice(h * hd, h * hd + hd)
            alone = forward(B, *(t[rows, cols].contiguous() for t in (Q, K, V)), hd, causal=causal, window=window)
            assert torch.equal(O[rows, cols], alone[0]) and torch.equal(lse[h:h + 1, rows], alone[1]), (hd, i, h)
