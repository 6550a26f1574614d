"""GPU: the C ABI counts rows in int; the binding refuses a matrix with more of them instead of handing on the rest of a division by 2^32."""
import pytest

from test_gpu_norm import B  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def test_more_rows_than_an_int_counts(B):  # noqa: F811
    import torch

    X = torch.empty((1 << 31) + 8, 1, dtype=torch.bfloat16, device="cuda")
    c = torch.empty(16, dtype=torch.uint8, device="cuda")
    launches = B.slope_launch_count()
    for call in (lambda: B.slope_layer_norm_fwd(X, None, None, 1e-5, X), lambda: B.slope_checkpoint_load(B.alloc_checkpoint(1, 32), X),
                 lambda: B.slope_linear_fwd(X, c, c, 16, X), lambda: B.slope_dense_linear_fwd(X, X, X)):
        with pytest.raises((OverflowError, ValueError)):
            call()
    assert B.slope_launch_count() == launches
