"""Layer norm: every plan of the forward and backward pass with enough rows that a group's ring is filled again and again, and with one checkpoint, the other or both.
Element by element against 64 bits, checkpoints bit for bit (tolerances: test_gpu_norm)."""
import numpy as np
import pytest

import norm_reference as ref
from test_gpu_norm import B, backward, case, check_backward, check_forward, f64, forward  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu

# At least three rows, or batches of short ones, for every group of warps and a ring of one or two stages: two to six groups in each of two blocks per SM up to
# 5120 wide (4064 with checkpoints), one to four in one block beyond.
FORWARD = [(6000, 1536), (4000, 2304), (3000, 4064), (3000, 4096), (2000, 5120), (2000, 5152), (2000, 5376), (2000, 6144), (1500, 6176), (1200, 8192), (1200, 8224),
           (1200, 9216), (700, 9248), (700, 13824), (500, 16384)]


@pytest.mark.parametrize("ckpt", ["none", "h", "y", "both"])
@pytest.mark.parametrize("b,d", FORWARD)
def test_forward_of_many_rows(B, b, d, ckpt):  # noqa: F811
    import torch

    turn = FORWARD.index((b, d)) + ["none", "h", "y", "both"].index(ckpt)
    x, residual = ("bf16", "f32")[turn % 2], turn % 4 < 2
    c = case(b, d, x, ("f32", "bf16")[turn // 2 % 2], b + d, residual)
    X = c["X"]
    new = lambda t: torch.full((b + 1, d), 7.0, dtype=t, device="cuda")
    out = {"Y": new(torch.bfloat16)[:b], "mean": torch.empty(b, device="cuda"), "rstd": torch.empty(b, device="cuda")}
    if residual:
        out["H"] = new(X.dtype)[:b]
    kept = {k: torch.full_like(B.alloc_checkpoint(b, d), 0xA5) for k, on in (("Hc", "h"), ("Yc", "y")) if ckpt in (on, "both")}
    B.slope_layer_norm_fwd(X, c["gamma"], c["beta"], 1e-5, out["Y"], out["mean"], out["rstd"], c["residual"], out.get("H"), kept.get("Hc"), kept.get("Yc"))
    h, *_ = check_forward(B, c, out, 1e-5, x)
    for name, of in (("Hc", h), ("Yc", f64(out["Y"]))):
        if name in kept:
            assert np.array_equal(kept[name].cpu().numpy(), ref.buffer(*ref.encode(of)))
    assert B.slope_poll_status() == 0


@pytest.mark.parametrize("b,d", [(1111, 256), (14000, 512), (20011, 64), (30011, 32), (60011, 32), (9999, 512), (5000, 992)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_checkpoints_of_short_rows(B, b, d, x):  # noqa: F811
    """Written by the layer norm itself, several rows together."""
    c = case(b, d, x, "bf16", b, residual=d == 512)
    check_forward(B, c, forward(B, c, 1e-5, ckpt=True), 1e-5, x)


@pytest.mark.parametrize("x,dx,p,dh", [("bf16", "bf16", "f32", True), ("f32", "f32", "bf16", True), ("q8", "bf16", "bf16", True), ("q8", "f32", "f32", False),
                                       ("bf16", "bf16", "bf16", False)])
@pytest.mark.parametrize("b,d", [(28000, 256), (9000, 768), (9000, 1024), (6000, 1536), (4000, 2304), (2000, 4096), (1500, 5120), (1500, 5376), (1500, 6144), (1000, 8192),
                                 (700, 9216), (700, 12288), (500, 16384)])
def test_backward_of_many_rows(B, b, d, x, dx, p, dh):  # noqa: F811
    kind = "bf16" if x == "q8" else x
    c = case(b, d, kind, p, b + 3 * d)
    out = forward(B, c, 1e-5, ckpt=x == "q8")
    h = ref.decode(*ref.split(out["Hc"].cpu().numpy(), b, d)) if x == "q8" else f64(c["X"])
    got = backward(B, c, out, out["Hc"] if x == "q8" else c["X"], dx, p, dh)
    check_backward(c, out, h, got, dx, p, dh)
    assert B.slope_poll_status() == 0
