"""Layer norm, forward and backward, element by element against 64 bits.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value, one to fp32 by 2^-24.  An fp32 sum of a row passes at most 32 additions in a lane, 5 in
a warp and 31 over warps, so a mean is off by at most 2^-24 * 70 of the mean magnitude (ADDS below, with the two roundings of its terms);
relative to a row's own spread that is what `lean` counts.  rstd: half the relative error of the variance (a sum of ADDS roundings, and the square of the
mean's error beside it) and 2 ulp of rsqrt.  The rest of the arithmetic is 4 to 8 roundings of the terms it adds, which stand beside each check.
A column sum over b rows passes at most b + 64 additions.
"""
import numpy as np
import pytest

import norm_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
ADDS = 72


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_24070_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def types():
    import torch

    return {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.double().cpu().numpy()


def within(got, want, bound, what):
    off = np.abs(got - want) - bound
    worst = np.unravel_index(int(np.argmax(off)), off.shape)
    assert (off <= 0).all(), f"{what}: {np.count_nonzero(off > 0)} of {off.size}; worst at {worst}: {got[worst]!r} for {want[worst]!r} within {bound[worst]!r}"


def stream(gen, b, d, offset=0.3):
    import torch

    new = lambda *s: torch.randn(s, generator=gen)
    return (new(b, d) * torch.exp(0.5 * new(d)) + offset) * torch.exp(0.5 * new(b, 1))


def case(b, d, x, p, seed, residual=False, offset=0.3):
    import torch

    t, gen = types(), torch.Generator().manual_seed(seed)
    c = {"X": stream(gen, b, d, offset).to(t[x]).cuda(), "gamma": (1 + 0.3 * torch.randn(d, generator=gen)).to(t[p]).cuda(),
         "beta": (0.3 * torch.randn(d, generator=gen)).to(t[p]).cuda(), "residual": torch.randn(b, d, generator=gen).bfloat16().cuda() if residual else None}
    c["dY"], c["dH"] = torch.randn(b, d, generator=gen).bfloat16().cuda(), torch.randn(b, d, generator=gen)
    return c


def forward(B, c, eps, stats=True, keep_h=True, ckpt=False):
    import torch

    X = c["X"]
    b, d = X.shape
    out = {"Y": torch.full((b + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")}
    if stats:
        out["mean"], out["rstd"] = (torch.full((b,), float("nan"), device="cuda") for _ in range(2))
    if c["residual"] is not None and keep_h:
        out["H"] = torch.full_like(X, float("nan"))
    if ckpt:
        out["Hc"], out["Yc"] = (torch.full_like(B.alloc_checkpoint(b, d), 0xA5) for _ in range(2))
    B.slope_layer_norm_fwd(X, c["gamma"], c["beta"], eps, out["Y"][:b], out.get("mean"), out.get("rstd"), c["residual"], out.get("H"), out.get("Hc"), out.get("Yc"))
    assert (out["Y"][b] == 7.0).all()                                        # the row behind the last one is left as it was
    out["Y"] = out["Y"][:b]
    return out


def check_forward(B, c, out, eps, x):
    X = c["X"]
    b, d = X.shape
    h = f64(X)
    if c["residual"] is not None:
        total = (X.float() + c["residual"].float()).to(X.dtype)
        h = f64(total)
        if "H" in out:
            assert np.array_equal(f64(out["H"]), h)
    gamma = np.ones(d) if c["gamma"] is None else f64(c["gamma"])
    beta = np.zeros(d) if c["beta"] is None else f64(c["beta"])
    y, mean, rstd, xhat = ref.layer_norm(h, gamma, beta, np.float64(np.float32(eps)))
    e_mean = U * ADDS * np.abs(h).mean(-1)
    lean = e_mean * rstd
    e_rstd = rstd * (U * (ADDS + 8) / 2 + 2 * U + lean * lean)
    if "mean" in out:
        within(f64(out["mean"]), mean, e_mean + U * np.abs(mean), "mean")
        within(f64(out["rstd"]), rstd, e_rstd, "rstd")
    # xhat: the mean's error, rstd's, the subtraction and the product; then gamma, beta and the rounding to bf16
    e_x = lean[:, None] + np.abs(xhat) * (e_rstd / rstd + 3 * U)[:, None]
    e_y = np.abs(gamma) * e_x + 2 * U * (np.abs(gamma * xhat) + np.abs(beta))
    got = f64(out["Y"])
    within(got, y, e_y * (1 + HALF["bf16"]) + HALF["bf16"] * np.abs(y), "Y")
    if "Hc" in out:
        assert np.array_equal(out["Hc"].cpu().numpy(), ref.buffer(*ref.encode(h)))
        assert np.array_equal(out["Yc"].cpu().numpy(), ref.buffer(*ref.encode(got)))
    return h, mean, rstd, gamma


WIDTHS = [(1, 8), (5, 64), (37, 264), (1, 4096), (2, 16384), (3, 13824), (70, 768), (129, 1000), (33, 2304), (40, 5120), (9, 8200), (301, 512), (1111, 256)]


@pytest.mark.parametrize("x,p", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("b,d", WIDTHS)
def test_forward(B, b, d, x, p):
    residual = (b + d) % 2 == 1 or d == 768
    c = case(b, d, x, p, b + d, residual)
    out = forward(B, c, 1e-5, ckpt=d % 32 == 0)
    check_forward(B, c, out, 1e-5, x)
    assert B.slope_poll_status() == 0


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("b,d", [(3, 16384), (5, 9216), (4, 9224), (3, 11008), (3, 15360), (2, 15368), (5, 5632), (7, 6144), (6, 2312), (301, 4096), (150, 4608), (40, 8192), (20011, 64), (15001, 200), (30011, 8), (9999, 512)])
def test_forward_at_the_edges_of_its_plans(B, b, d, x):
    """The widest rows with all that a block has to hold, and rows so short and many that several travel together."""
    c = case(b, d, x, "f32", b + d, residual=True)
    check_forward(B, c, forward(B, c, 1e-5), 1e-5, x)


def test_forward_at_inference_is_the_same(B):
    """Without statistics, sum and checkpoints: the same Y, bit for bit."""
    import torch

    c = case(19, 2048, "bf16", "bf16", 8, residual=True)
    full, lean = forward(B, c, 1e-5, ckpt=True), forward(B, c, 1e-5, stats=False, keep_h=False)
    assert torch.equal(full["Y"], lean["Y"])


@pytest.mark.parametrize("gamma,beta", [(False, False), (True, False), (False, True)])
def test_without_gain_or_offset(B, gamma, beta):
    c = case(17, 1152, "f32", "f32", 9)
    c["gamma"], c["beta"] = c["gamma"] if gamma else None, c["beta"] if beta else None
    check_forward(B, c, forward(B, c, 1e-6), 1e-6, "f32")


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_rows_that_hardly_spread(B, x):
    """Means far above the spread, constant rows, rows of zeros: the variance is that of the differences."""
    import torch

    c = case(12, 1024, x, "f32", 10, offset=300.0)
    c["X"][3], c["X"][4], c["X"][5] = 5.0, 0.0, -1e-20
    out = forward(B, c, 1e-5)
    check_forward(B, c, out, 1e-5, x)
    assert torch.equal(out["Y"][4], c["beta"].bfloat16())


def test_rows_with_infinities_and_nan_stay_among_themselves(B):
    import torch

    c = case(9, 768, "bf16", "bf16", 11, residual=True)
    clean = forward(B, c, 1e-5, ckpt=True)
    c["X"][2, 5], c["residual"][4, 700], c["X"][6, 33] = float("inf"), float("nan"), -torch.finfo(torch.bfloat16).max
    out = forward(B, c, 1e-5, ckpt=True)
    for row in range(9):
        if row in (2, 4):
            assert torch.isnan(out["Y"][row]).all() and torch.isnan(out["rstd"][row])
        elif row != 6:
            assert torch.equal(out["Y"][row], clean["Y"][row])
    back = torch.empty_like(out["Y"])
    B.slope_checkpoint_load(out["Hc"], back)
    assert torch.isnan(back[2, :32]).all() and torch.isfinite(back[2, 32:]).all() and torch.isnan(back[4, 672:704]).all()


def backward(B, c, out, h, dx, p, dh=True, params=True):
    import torch

    b, d = c["dY"].shape
    t = types()
    got = {"dX": torch.full((b + 1, d), 7.0, dtype=t[dx], device="cuda")}
    if params:
        got["dgamma"], got["dbeta"] = (torch.full((d,), float("nan"), dtype=t[p], device="cuda") for _ in range(2))
    ws = torch.full((max(16, B.slope_layer_norm_bwd_workspace_bytes(b, d)),), 0xFF, dtype=torch.uint8, device="cuda")
    B.slope_layer_norm_bwd(c["dY"], h, out["mean"], out["rstd"], c["gamma"], got["dX"][:b], got.get("dgamma"), got.get("dbeta"), ws,
                           c["dH"].to(t[dx]).cuda() if dh else None)
    assert (got["dX"][b] == 7.0).all()
    got["dX"] = got["dX"][:b]
    return got


def check_backward(c, out, h, got, dx, p, dh=True):
    b, d = c["dY"].shape
    mean, rstd, dy = f64(out["mean"]), f64(out["rstd"]), f64(c["dY"])
    gamma = np.ones(d) if c["gamma"] is None else f64(c["gamma"])
    side = f64(c["dH"].to(types()[dx])) if dh else None
    want, dgamma, dbeta, terms = ref.layer_norm_grads(dy, h, mean, rstd, gamma, side)
    within(f64(got["dX"]), want, HALF[dx] * np.abs(want) + (ADDS + 12) * U * terms, "dX")
    xhat = np.abs((h - mean[:, None]) * rstd[:, None])
    adds = b + 64 + 4
    if "dgamma" in got:
        within(f64(got["dgamma"]), dgamma, HALF[p] * np.abs(dgamma) + adds * U * (np.abs(dy) * xhat).sum(0), "dgamma")
        within(f64(got["dbeta"]), dbeta, HALF[p] * np.abs(dbeta) + adds * U * np.abs(dy).sum(0), "dbeta")


@pytest.mark.parametrize("x,dx,p", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("q8", "bf16", "f32"), ("q8", "f32", "bf16"), ("f32", "bf16", "bf16"),
                                    ("bf16", "f32", "f32")])
@pytest.mark.parametrize("b,d", WIDTHS)
def test_backward(B, b, d, x, dx, p):
    if x == "q8" and d % 32:
        pytest.skip("a checkpoint has whole blocks")
    kind = "bf16" if x == "q8" else x
    c = case(b, d, kind, p, 2 * b + d)
    out = forward(B, c, 1e-5, ckpt=x == "q8")
    h = ref.decode(*ref.split(out["Hc"].cpu().numpy(), b, d)) if x == "q8" else f64(c["X"])
    dh = (b + d) % 2 == 0
    got = backward(B, c, out, out["Hc"] if x == "q8" else c["X"], dx, p, dh)
    check_backward(c, out, h, got, dx, p, dh)
    assert B.slope_poll_status() == 0


@pytest.mark.parametrize("x", ["bf16", "f32", "q8"])
@pytest.mark.parametrize("b,d", [(20011, 64), (30011, 32), (9999, 512), (17, 768), (1025, 512), (330, 5376), (7, 6144), (301, 9216), (2, 12288), (150, 4608)])
def test_backward_at_the_edges_of_its_plans(B, b, d, x):
    kind = "bf16" if x == "q8" else x
    c = case(b, d, kind, "f32", b, offset=0.1)
    out = forward(B, c, 1e-5, ckpt=x == "q8")
    h = ref.decode(*ref.split(out["Hc"].cpu().numpy(), b, d)) if x == "q8" else f64(c["X"])
    got = backward(B, c, out, out["Hc"] if x == "q8" else c["X"], kind, "f32")
    check_backward(c, out, h, got, kind, "f32")


def test_gradients_against_differences(B):
    """dX, dgamma and dbeta against central differences of the forward's formula in 64 bits."""
    import torch

    c = case(3, 64, "f32", "f32", 21)
    out = forward(B, c, 1e-5)
    got = backward(B, c, out, c["X"], "f32", "f32", dh=False)
    h, gamma, beta, dy = f64(c["X"]), f64(c["gamma"]), f64(c["beta"]), f64(c["dY"])
    loss = lambda h, g, be: float((ref.layer_norm(h, g, be, 1e-5)[0] * dy).sum())
    step = 1e-5
    for name, args, k in (("dX", (h, gamma, beta), 0), ("dgamma", (h, gamma, beta), 1), ("dbeta", (h, gamma, beta), 2)):
        want = np.empty_like(args[k])
        for i in np.ndindex(want.shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[k][i] += step
            down[k][i] -= step
            want[i] = (loss(*up) - loss(*down)) / (2 * step)
        # differences: step^2 and the cancellation of the loss (1e-16 * |loss| / step) are below 1e-8; fp32 gives some 1e-6
        assert np.linalg.norm(f64(got[name]) - want) <= 1e-5 * np.linalg.norm(want), name


def test_each_parameter_gradient_alone(B):
    import torch

    c = case(600, 768, "bf16", "f32", 22)
    out = forward(B, c, 1e-5)
    both = backward(B, c, out, c["X"], "bf16", "f32")
    ws = torch.empty(B.slope_layer_norm_bwd_workspace_bytes(600, 768), dtype=torch.uint8, device="cuda")
    dX, one = torch.empty_like(both["dX"]), torch.empty_like(both["dgamma"])
    dH = c["dH"].bfloat16().cuda()
    B.slope_layer_norm_bwd(c["dY"], c["X"], out["mean"], out["rstd"], c["gamma"], dX, one, None, ws, dH)
    assert torch.equal(one, both["dgamma"]) and torch.equal(dX, both["dX"])
    B.slope_layer_norm_bwd(c["dY"], c["X"], out["mean"], out["rstd"], c["gamma"], dX, None, one, ws, dH)
    assert torch.equal(one, both["dbeta"]) and torch.equal(dX, both["dX"])
    dX.zero_()
    B.slope_layer_norm_bwd(c["dY"], c["X"], out["mean"], out["rstd"], c["gamma"], dX, dH=dH)      # neither: no workspace
    assert torch.equal(dX, both["dX"])


def test_outputs_in_the_place_of_inputs(B):
    """What the header allows: H over X or over the residual, dX over dY or over dH."""
    import torch

    c = case(150, 1280, "bf16", "bf16", 23, residual=True)
    want = forward(B, c, 1e-5)
    grads = backward(B, c, want, want["H"], "bf16", "bf16")
    for place in ("X", "residual"):
        X, R, Y = c["X"].clone(), c["residual"].clone(), torch.empty_like(c["X"])
        H = X if place == "X" else R
        B.slope_layer_norm_fwd(X, c["gamma"], c["beta"], 1e-5, Y, residual=R, H=H)
        assert torch.equal(H, want["H"]) and torch.equal(Y, want["Y"])
    ws = torch.empty(B.slope_layer_norm_bwd_workspace_bytes(150, 1280), dtype=torch.uint8, device="cuda")
    for place in ("dY", "dH"):
        dY, dH = c["dY"].clone(), c["dH"].bfloat16().cuda()
        dX, dgamma, dbeta = (dY if place == "dY" else dH), torch.empty_like(c["gamma"]), torch.empty_like(c["beta"])
        B.slope_layer_norm_bwd(dY, want["H"], want["mean"], want["rstd"], c["gamma"], dX, dgamma, dbeta, ws, dH)
        assert torch.equal(dX, grads["dX"]) and torch.equal(dgamma, grads["dgamma"]) and torch.equal(dbeta, grads["dbeta"])


@pytest.mark.parametrize("d", [768, 4096, 11008])
def test_equal_rows_of_a_call_have_equal_results(B, d):
    """Wherever in the batch they stand."""
    import torch

    b = 700
    c = case(b, d, "bf16", "bf16", 24, residual=True)
    for name in ("X", "residual", "dY"):
        c[name][1::2] = c[name][0]
    c["dH"][1::2] = c["dH"][0]
    out = forward(B, c, 1e-5)
    got = backward(B, c, out, out["H"], "bf16", "bf16")
    for t in (out["Y"], out["mean"], out["rstd"], got["dX"]):
        assert (t[1::2] == t[0]).all()


def test_on_another_stream_and_in_a_graph(B):
    """A forward and backward pass captured once and replayed on other inputs; two graphs with workspaces of their own."""
    import torch

    b, d = 900, 1536
    c, e = case(b, d, "bf16", "f32", 25, residual=True), case(b, d, "bf16", "f32", 26, residual=True)
    ws = [torch.empty(B.slope_layer_norm_bwd_workspace_bytes(b, d), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(c, o, ws):
        B.slope_layer_norm_fwd(c["X"], c["gamma"], c["beta"], 1e-5, o["Y"], o["mean"], o["rstd"], c["residual"], None, o["Hc"], o["Yc"])
        B.slope_layer_norm_bwd(c["dY"], o["Hc"], o["mean"], o["rstd"], c["gamma"], o["dX"], o["dgamma"], o["dbeta"], ws, c["residual"])

    def buffers():
        new = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")
        return {"Y": new(b, d, t=torch.bfloat16), "mean": new(b), "rstd": new(b), "Hc": B.alloc_checkpoint(b, d), "Yc": B.alloc_checkpoint(b, d),
                "dX": new(b, d, t=torch.bfloat16), "dgamma": new(d), "dbeta": new(d)}

    eager = [buffers(), buffers()]
    step(c, eager[0], ws[0])
    step(e, eager[1], ws[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = buffers()
    with torch.cuda.stream(side):
        step(c, got, ws[1])
    side.synchronize()
    assert all(torch.equal(got[k], eager[0][k]) for k in got)
    graphs, outs = [], []
    for k in range(2):
        outs.append(buffers())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            step((c, e)[k], outs[k], ws[k])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                graphs[k].replay()
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(outs[k][n], eager[k][n]) for n in outs[k])
    for n in ("X", "residual", "dY", "gamma", "beta"):
        c[n].copy_(e[n])
    graphs[0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0][n], eager[1][n]) for n in outs[0])


def test_rows_beyond_32_bits_of_values(B):
    """More than 2^31 values: the last rows equal the first ones."""
    import torch

    d = 16384
    b = (1 << 31) // d + 5
    c = case(8, d, "bf16", "bf16", 27)
    X = torch.zeros(b, d, dtype=torch.bfloat16, device="cuda")
    X[:8], X[-8:] = c["X"], c["X"]
    Y, mean, rstd = torch.empty_like(X), torch.empty(b, device="cuda"), torch.empty(b, device="cuda")
    B.slope_layer_norm_fwd(X, c["gamma"], c["beta"], 1e-5, Y, mean, rstd)
    small = forward(B, c, 1e-5)
    assert torch.equal(Y[:8], small["Y"]) and torch.equal(Y[-8:], small["Y"]) and torch.equal(rstd[-8:], small["rstd"])
    dY = Y.zero_()
    dY[:8], dY[-8:] = c["dY"], c["dY"]
    ws = torch.empty(B.slope_layer_norm_bwd_workspace_bytes(b, d), dtype=torch.uint8, device="cuda")
    dX, dgamma, dbeta = torch.empty_like(X), torch.empty(d, device="cuda").bfloat16(), torch.empty(d, device="cuda").bfloat16()
    B.slope_layer_norm_bwd(dY, X, mean, rstd, c["gamma"], dX, dgamma, dbeta, ws)
    want = backward(B, c, small, c["X"], "bf16", "bf16", dh=False)
    assert torch.equal(dX[:8], want["dX"]) and torch.equal(dX[-8:], want["dX"]) and not dX[8:-8].any()


def test_refusals_of_the_binding(B):
    import torch

    c = case(4, 64, "bf16", "bf16", 28)
    X, g, Y, s = c["X"], c["gamma"], torch.empty_like(c["X"]), torch.empty(4, device="cuda")
    launches = B.slope_launch_count()
    for call, error in [(lambda: B.slope_layer_norm_fwd(X, g.float(), c["beta"], 1e-5, Y), TypeError),
                        (lambda: B.slope_layer_norm_fwd(X, g[:32], None, 1e-5, Y), ValueError),
                        (lambda: B.slope_layer_norm_fwd(X, g, None, 1e-5, Y[:3]), ValueError),
                        (lambda: B.slope_layer_norm_fwd(X, g, None, 1e-5, Y.float()), TypeError),
                        (lambda: B.slope_layer_norm_fwd(X.half(), g, None, 1e-5, Y), TypeError),
                        (lambda: B.slope_layer_norm_fwd(X, g, None, 1e-5, Y, s[:3], s), ValueError),
                        (lambda: B.slope_layer_norm_fwd(X, g, None, 1e-5, Y, residual=X.float()), TypeError),
                        (lambda: B.slope_layer_norm_fwd(X, g, None, 1e-5, Y, H_ckpt=B.alloc_checkpoint(4, 32)), ValueError),
                        (lambda: B.slope_layer_norm_fwd(X, g, None, 1e-5, Y, s, None), B.SlopeError),
                        (lambda: B.slope_layer_norm_fwd(X, g, None, 1e-5, Y, H=Y), B.SlopeError),
                        (lambda: B.slope_layer_norm_fwd(X.t(), g, None, 1e-5, Y), AssertionError),
                        (lambda: B.slope_layer_norm_bwd(c["dY"], X, s, s, g, Y, g.float(), None), TypeError),
                        (lambda: B.slope_layer_norm_bwd(c["dY"], X[:2], s, s, g, Y), ValueError),
                        (lambda: B.slope_layer_norm_bwd(c["dY"], B.alloc_checkpoint(4, 32), s, s, g, Y), ValueError),
                        (lambda: B.slope_layer_norm_bwd(c["dY"], X, s, s, g, Y, dH=Y.float()), TypeError),
                        (lambda: B.slope_layer_norm_bwd(c["dY"], X, s.double(), s, g, Y), TypeError)]:
        with pytest.raises(error):
            call()
    many = torch.zeros(2048, 64, dtype=torch.bfloat16, device="cuda")
    stats = torch.zeros(2048, device="cuda")
    with pytest.raises(B.SlopeError):                                        # dgamma over many blocks needs its workspace
        B.slope_layer_norm_bwd(many, many, stats, stats, g, many.clone(), g.clone(), None)
    assert B.slope_launch_count() == launches
