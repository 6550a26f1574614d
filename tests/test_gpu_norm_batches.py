"""Layer norms of many short rows, of which several travel together: one row more or less than where the number changes, against 64 bits, and a row's bits whatever
number it is (tolerances: test_gpu_norm)."""
import pytest

from test_gpu_norm import B, case, check_forward, forward  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu

# 12 rows of a block at a time, 296 blocks: two, four and eight rows together from 4, 8 and 16 times as many on
EDGES = [(14207, 512), (14208, 512), (14209, 512), (14207, 256), (28415, 256), (28417, 256), (28416, 96), (56831, 96), (56833, 96), (60011, 64)]


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("b,d", EDGES)
def test_forward_where_the_number_changes(B, b, d, x):  # noqa: F811
    c = case(b, d, x, "f32", b + d, residual=b % 2 == 1)
    check_forward(B, c, forward(B, c, 1e-5, ckpt=b == 60011), 1e-5, x)
    assert B.slope_poll_status() == 0


@pytest.mark.parametrize("d", [64, 256, 512])
def test_a_row_does_not_depend_on_the_number(B, d):  # noqa: F811
    import torch

    c = case(60011, d, "bf16", "bf16", d, residual=True)
    want = forward(B, c, 1e-5)
    for first, rows in ((0, 7), (4000, 14207), (1, 30000)):
        part = dict(c, X=c["X"][first:first + rows].contiguous(), residual=c["residual"][first:first + rows].contiguous())
        got = forward(B, part, 1e-5)
        assert all(torch.equal(got[k], want[k][first:first + rows]) for k in ("Y", "H", "mean", "rstd"))
