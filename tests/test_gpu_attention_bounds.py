"""GPU: starts and lengths that no batch has are held to the rows that there are."""
import pytest

from test_gpu_attention import B, compare, run, tensors  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu

LEAST, MOST = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("starts,lengths,held", [
    ([100, LEAST], None, []),                                          # an end before 0, further below its start than 32 bits count
    ([300, LEAST + 50, 200], None, [(0, 200)]),                        # ... and as the start of the next
    ([LEAST, MOST], None, [(0, 300)]),
    ([LEAST, 40, MOST], [MOST, LEAST], [(0, 40)]),
    ([299, LEAST + 299, 130], [7, 129], [(0, 129)]),
    ([MOST, LEAST, LEAST, MOST], [5, 5, 5], [(0, 5)]),
])
def test_starts_and_lengths_outside_the_batch(B, starts, lengths, held, causal):  # noqa: F811
    import torch

    on = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")
    for hd in (64, 128):
        Q, K, V, dO = tensors(300, 2, 1, hd, 31)
        got = run(B, Q, K, V, dO, hd, starts=on(starts), lengths=on(lengths), causal=causal)
        if held:
            compare(got, Q, K, V, dO, hd, held, causal)
        else:
            assert all((x == 7).all() for x in got.values())
