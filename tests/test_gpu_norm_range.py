"""Layer norms of rows whose sums, or whose squared differences, leave the range of fp32 while the rows themselves are in it.

Tolerances are those of test_gpu_norm (roundings of 2^-24 of the terms; bf16 2^-8), and half a unit of the smallest numbers, 2^-150 in fp32, where a
reciprocal of 2^126 or more is held.
"""
import numpy as np
import pytest

import norm_reference as ref
from test_gpu_norm import ADDS, B, HALF, U, backward, case, f64, forward, within  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu

# (scale, offset): squares beyond fp32 at some of the widths; at all; sums beyond it too; the largest
ROWS = [(1e17, 0.0), (1e18, -3e18), (1e20, 0.0), (1e30, 1e30), (3e33, 2e34), (1e36, 1e37), (2e37, 0.0), (1e37, -1.2e38)]


def wide(b, d, x, p, seed, residual):
    import torch

    c = case(b, d, x, p, seed, residual)
    gen = torch.Generator().manual_seed(seed + 1)
    for i, (scale, offset) in enumerate(ROWS):
        if 2 * i + 1 < b:                           # every other row is an ordinary one
            row = (torch.randn(d, generator=gen, dtype=torch.float64).clamp(-4, 4) * scale + offset)
            c["X"][2 * i + 1] = row.to(c["X"].dtype).cuda()
    return c


@pytest.mark.parametrize("x,p", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("b,d,residual,ckpt", [(17, 64, False, True), (17, 264, True, False), (17, 768, True, True), (18, 1000, False, False), (17, 4096, True, False),
                                               (17, 4096, False, True), (17, 8192, False, False), (17, 11008, True, True), (17, 16384, False, False)])
def test_forward_of_rows_whose_sums_leave_fp32(B, b, d, residual, ckpt, x, p):  # noqa: F811
    c = wide(b, d, x, p, b + d, residual)
    out = forward(B, c, 1e-5, ckpt=ckpt)
    h = f64(out["H"]) if residual else f64(c["X"])
    assert np.isfinite(h).all()
    y, mean, rstd, xhat = ref.layer_norm(h, f64(c["gamma"]), f64(c["beta"]), np.float64(np.float32(1e-5)))
    e_mean = U * ADDS * np.abs(h).mean(-1)
    lean = e_mean * rstd
    e_rstd = rstd * (U * (ADDS + 8) / 2 + 2 * U + lean * lean) + 2.0 ** -150
    within(f64(out["mean"]), mean, e_mean + U * np.abs(mean), "mean")
    within(f64(out["rstd"]), rstd, e_rstd, "rstd")
    gamma, beta = f64(c["gamma"]), f64(c["beta"])
    e_y = np.abs(gamma) * (lean[:, None] + np.abs(xhat) * (e_rstd / rstd + 3 * U)[:, None]) + 2 * U * (np.abs(gamma * xhat) + np.abs(beta))
    within(f64(out["Y"]), y, e_y * (1 + HALF["bf16"]) + HALF["bf16"] * np.abs(y), "Y")
    if ckpt:
        assert np.array_equal(out["Hc"].cpu().numpy(), ref.buffer(*ref.encode(h)))
        assert np.array_equal(out["Yc"].cpu().numpy(), ref.buffer(*ref.encode(f64(out["Y"]))))
    assert B.slope_poll_status() == 0


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 1024, 4096, 8192])
def test_large_values_of_both_signs(B, d, x):  # noqa: F811
    """Partial sums that are infinite with either sign, while mean and differences are fp32's."""
    import torch

    c = case(5, d, x, "f32", d)
    sign = torch.ones(d)
    sign[d // 2:] = -1.0
    c["X"][1] = (3e38 * sign).to(c["X"].dtype).cuda()
    c["X"][3] = (3e38 * sign.view(2, -1).t().reshape(-1)).to(c["X"].dtype).cuda()
    out = forward(B, c, 1e-5)
    h = f64(c["X"])
    y, mean, rstd, _ = ref.layer_norm(h, f64(c["gamma"]), f64(c["beta"]), 1e-5)
    for row in (1, 3):
        # equal magnitudes: the mean is 0 but for roundings of partial sums, xhat is +-1 within a few of them
        assert abs(f64(out["mean"])[row]) <= U * ADDS * 3.1e38
        within(f64(out["rstd"])[row:row + 1], rstd[row:row + 1], rstd[row:row + 1] * ADDS * U + 2.0 ** -150, "rstd")
        bound = HALF["bf16"] * np.abs(y[row]) + (1 + HALF["bf16"]) * np.abs(f64(c["gamma"])) * (2 * ADDS * U + 2.0 ** -150 / rstd[row]) + 2 * U
        within(f64(out["Y"])[row], y[row], bound, "Y")


@pytest.mark.parametrize("x,dx", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("b,d", [(17, 264), (17, 768), (17, 4096), (17, 11008)])
def test_backward_of_such_rows(B, b, d, x, dx):  # noqa: F811
    """From the forward's own statistics.  What is below 2^-126 has an absolute error of half a unit: 2^-150 in fp32, and 2^-134 more in bf16."""
    c = wide(b, d, x, "f32", b + d, False)
    out = forward(B, c, 1e-5)
    h, mean, rstd = f64(c["X"]), f64(out["mean"]), f64(out["rstd"])
    got = backward(B, c, out, c["X"], dx, "f32", dh=False)
    dy, gamma = f64(c["dY"]), f64(c["gamma"])
    want, dgamma, dbeta, terms = ref.layer_norm_grads(dy, h, mean, rstd, gamma)
    within(f64(got["dX"]), want, HALF[dx] * np.abs(want) + (ADDS + 12) * U * terms + (2.0 ** -134 if dx == "bf16" else 0.0) + 2.0 ** -150, "dX")
    xhat = np.abs((h - mean[:, None]) * rstd[:, None])
    within(f64(got["dgamma"]), dgamma, U * np.abs(dgamma) + (b + 68) * U * (np.abs(dy) * xhat).sum(0), "dgamma")
    within(f64(got["dbeta"]), dbeta, U * np.abs(dbeta) + (b + 68) * U * np.abs(dy).sum(0), "dbeta")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 768, 4096, 9216])
def test_rows_that_are_not_numbers_are_so_throughout(B, d, x):  # noqa: F811
    """An infinity or a NaN in a row, and values whose difference from the mean is none of fp32's: rstd and Y are NaN throughout, other rows as they were."""
    import torch

    c = case(9, d, x, "f32", d)
    clean = forward(B, c, 1e-5, ckpt=True)
    top = torch.finfo(c["X"].dtype).max
    c["X"][1, 5], c["X"][3, d - 1], c["X"][5, 7] = float("inf"), float("nan"), -float("inf")
    c["X"][7] = -top
    c["X"][7, 3] = top                              # off the mean by nearly twice the largest number
    out = forward(B, c, 1e-5, ckpt=True)
    for row in range(9):
        if row % 2:
            assert torch.isnan(out["Y"][row]).all() and torch.isnan(out["rstd"][row]), row
        else:
            assert all(torch.equal(out[k][row], clean[k][row]) for k in ("Y", "mean", "rstd"))
    assert not torch.isfinite(out["mean"][[1, 3, 5]]).any()


@pytest.mark.parametrize("d", [64, 4096])
def test_an_eps_that_outweighs_the_variance(B, d):  # noqa: F811
    """eps next to the largest number: 1 / sqrt(v + eps) as it is, not zero."""
    c = wide(17, d, "f32", "f32", 3, False)
    eps = np.float64(np.finfo(np.float32).max)
    out = forward(B, c, float(eps))
    _, mean, rstd, _ = ref.layer_norm(f64(c["X"]), 1.0, 0.0, eps)
    within(f64(out["rstd"]), rstd, rstd * (U * (ADDS + 8) / 2 + 4 * U + (U * ADDS * np.abs(f64(c["X"])).mean(-1) * rstd) ** 2) + 2.0 ** -150, "rstd")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", [256, 4096])
def test_such_rows_wherever_the_sum_stands(B, d, x):  # noqa: F811
    """The sum kept apart, over X, over the residual (bf16), or not at all; and in a graph that is replayed on other rows."""
    import torch

    c = wide(17, d, x, "f32", d, True)
    want = forward(B, c, 1e-5)
    lean = forward(B, c, 1e-5, stats=False, keep_h=False)
    assert torch.equal(lean["Y"], want["Y"])
    for place in ("X", "residual") if x == "bf16" else ("X",):
        X, R, Y = c["X"].clone(), c["residual"].clone(), torch.empty_like(want["Y"])
        H = X if place == "X" else R
        B.slope_layer_norm_fwd(X, c["gamma"], c["beta"], 1e-5, Y, residual=R, H=H)
        assert torch.equal(H, want["H"]) and torch.equal(Y, want["Y"])
    e = case(17, d, x, "f32", d + 1, True)
    plain = forward(B, e, 1e-5)
    X, R, Y, graph = e["X"].clone(), e["residual"].clone(), torch.empty_like(want["Y"]), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.slope_layer_norm_fwd(X, c["gamma"], c["beta"], 1e-5, Y, residual=R)
    graph.replay()
    ordinary = Y.clone()
    X.copy_(c["X"])
    R.copy_(c["residual"])
    graph.replay()
    assert torch.equal(Y, want["Y"])
    X.copy_(e["X"])
    R.copy_(e["residual"])
    graph.replay()
    assert torch.equal(Y, ordinary)
    B.slope_layer_norm_fwd(e["X"], e["gamma"], e["beta"], 1e-5, Y, residual=e["residual"])
    assert torch.equal(Y, plain["Y"])


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", [256, 768, 1000, 4096, 8192, 16384])
def test_rows_next_to_the_range_do_not_depend_on_others(B, d, x):  # noqa: F811
    """Rows whose squares add up to nearly 2^128, or whose magnitudes do, alone and among rows beyond: the same bits."""
    import torch

    b = 600
    gen = torch.Generator().manual_seed(d)
    rows = torch.randn(6, d, generator=gen, dtype=torch.float64).clamp(-4, 4)
    near = [rows[k] * (2.0 ** 64 * f / float(rows[k].norm())) for k, f in enumerate((0.99, 0.7, 0.5, 0.36))]
    near += [rows[4] * (2.0 ** 128 * 0.9 / d / 4) + 2.0 ** 128 * 0.7 / d, rows[5]]          # its sum is in range, its squares are not
    c = case(b, d, x, "f32", d)
    for i in range(b):
        c["X"][i] = near[i % 6].to(c["X"].dtype).cuda()
    alone = forward(B, c, 1e-5)
    mixed = dict(c, X=c["X"].clone())
    beyond = torch.arange(b, device="cuda") % 7 == 3
    mixed["X"][beyond] = (torch.randn(d, generator=gen, dtype=torch.float64).clamp(-4, 4) * 1e30).to(c["X"].dtype).cuda()
    out = forward(B, mixed, 1e-5)
    for k in ("Y", "mean", "rstd"):
        assert torch.equal(out[k][~beyond], alone[k][~beyond]), k
        for first in range(6):                       # equal rows of one call, wherever they stand
            assert (alone[k][first::6] == alone[k][first]).all(), k
    assert torch.isfinite(out["Y"]).all() and (out["rstd"] > 0).all()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 768, 5120])
def test_one_large_value_in_an_ordinary_row(B, d, x):  # noqa: F811
    """A single value next to the type's largest number: its square leaves fp32, the row's other values stand at next to nothing beside it."""
    import torch

    c = case(9, d, x, "f32", d, residual=True)
    c["X"][6, 33] = -0.99 * torch.finfo(c["X"].dtype).max
    out = forward(B, c, 1e-5, ckpt=True)
    h = f64(out["H"])
    y, mean, rstd, xhat = ref.layer_norm(h, f64(c["gamma"]), f64(c["beta"]), 1e-5)
    e_mean = U * ADDS * np.abs(h).mean(-1)
    lean = e_mean * rstd
    e_rstd = rstd * (U * (ADDS + 8) / 2 + 2 * U + lean * lean) + 2.0 ** -150
    within(f64(out["mean"]), mean, e_mean + U * np.abs(mean), "mean")
    within(f64(out["rstd"]), rstd, e_rstd, "rstd")
    gamma, beta = np.abs(f64(c["gamma"])), np.abs(f64(c["beta"]))
    e_y = gamma * (lean[:, None] + np.abs(xhat) * (e_rstd / rstd + 3 * U)[:, None]) + 2 * U * (gamma * np.abs(xhat) + beta)
    within(f64(out["Y"]), y, e_y * (1 + HALF["bf16"]) + HALF["bf16"] * np.abs(y), "Y")
    assert np.array_equal(out["Yc"].cpu().numpy(), ref.buffer(*ref.encode(f64(out["Y"]))))
