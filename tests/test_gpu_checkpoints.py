"""8-bit checkpoints bit for bit against their definition, and the weight gradients that read them against 64 bits."""
import numpy as np
import pytest

import norm_reference as ref
from helpers import REL_TOL, parity_error

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_24070_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def values(shape, f32, seed):
    """Values of every size, and the ones at the format's borders."""
    import torch

    rng = np.random.Generator(np.random.PCG64(seed))
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-8, 9, (shape[0], 1))
    blocks = x.reshape(-1, 32)
    special = [np.zeros(32), np.full(32, 127.5), np.full(32, -127.5), np.linspace(-63.75, 63.75, 32), np.arange(32) - 15.5, np.full(32, 1e-40),
               np.full(32, 1.2e-38), np.r_[np.inf, np.ones(31)], np.r_[np.ones(31), -np.inf], np.r_[np.ones(15), np.nan, np.ones(16)],
               np.r_[3.38e38, np.ones(31)], np.r_[-3.3895e38, np.full(31, 1e36)], np.r_[1.0, np.full(31, 0.5 / 64)], np.r_[-0.0, np.zeros(31)]]
    for i, s in enumerate(special):
        if i * 3 < len(blocks):
            blocks[i * 3] = s
    t = torch.from_numpy(x.astype(np.float32))
    return t if f32 else t.bfloat16()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 96), (3, 128), (37, 800), (257, 2304), (64, 11008), (1025, 128)])
def test_store_and_load_bit_for_bit(B, rows, cols, f32):
    import torch

    x = values((rows, cols), f32, rows + cols)
    codes, exponents = ref.encode(x.double().numpy())
    want = ref.buffer(codes, exponents)
    room = torch.full((want.size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    ckpt = room[:want.size]
    B.slope_checkpoint_store(x.cuda(), ckpt)
    got = room.cpu().numpy()
    assert np.array_equal(got[:want.size], want)
    assert (got[want.size:] == 0xA5).all()                                  # nothing behind the buffer
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.full((rows + 1, cols), 7.0, dtype=dtype, device="cuda")
        B.slope_checkpoint_load(ckpt, out[:rows])
        back = out.double().cpu().numpy()
        assert np.array_equal(back[:rows], ref.decode(codes, exponents), equal_nan=True)
        assert (back[rows] == 7.0).all()
    assert B.slope_poll_status() == 0


def test_more_values_than_32_bits_count(B):
    """2^31 values and a few: the last rows are stored and read at offsets that do not fit an int."""
    import torch

    rows, cols = (1 << 31) // 8192 + 3, 8192
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(5, cols, device="cuda").bfloat16()
    x[-5:] = tail
    x[:5] = tail
    ckpt = B.alloc_checkpoint(rows, cols)
    B.slope_checkpoint_store(x, ckpt)
    x.fill_(1.0)
    B.slope_checkpoint_load(ckpt, x)
    codes, exponents = ref.encode(tail.double().cpu().numpy())
    want = torch.from_numpy(ref.decode(codes, exponents)).bfloat16().cuda()
    assert torch.equal(x[:5], want) and torch.equal(x[-5:], want) and not x[5:-5].any()


def test_refusals_of_the_binding(B):
    import torch

    x, c = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda"), B.alloc_checkpoint(4, 64)
    launches = B.slope_launch_count()
    for call, error in [(lambda: B.slope_checkpoint_store(x.half(), c), TypeError), (lambda: B.slope_checkpoint_store(x, c[:-1]), ValueError),
                        (lambda: B.slope_checkpoint_store(x, x), TypeError), (lambda: B.slope_checkpoint_load(c, x[:3]), ValueError),
                        (lambda: B.slope_checkpoint_store(x[0], c), ValueError),
                        (lambda: B.slope_checkpoint_store(x[:, :32], c), AssertionError)]:
        with pytest.raises(error):
            call()
    with pytest.raises(B.SlopeError):                                        # half a block
        B.slope_checkpoint_store(torch.zeros(2, 48, dtype=torch.bfloat16, device="cuda"), torch.zeros(99, dtype=torch.uint8, device="cuda"))
    dY, mask, dWc = (torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(128, 16, dtype=torch.uint8, device="cuda"),
                     torch.zeros(128, 64, dtype=torch.bfloat16, device="cuda"))
    xc, ws = B.alloc_checkpoint(4, 128), torch.zeros(B.slope_bwd_dw_q8_workspace_bytes(4, 128, 128), dtype=torch.uint8, device="cuda")
    for call, error in [(lambda: B.slope_linear_bwd_dw_masked_q8(dY, c, mask, dWc, ws), ValueError),
                        (lambda: B.slope_linear_bwd_dw_masked_q8(dY.float(), xc, mask, dWc, ws), TypeError),
                        (lambda: B.slope_linear_bwd_dw_masked_q8(dY, xc, mask, dWc[:64], ws), ValueError),
                        (lambda: B.slope_linear_bwd_dw_masked_q8(dY, xc, mask[:64], dWc, ws), ValueError),
                        (lambda: B.slope_dense_linear_bwd_dw_q8(dY, xc, dWc, ws), ValueError),
                        (lambda: B.slope_linear_bwd_dw_adapter_q8(dY, xc, dY[:, :16].contiguous(), dY[:3, :16].contiguous(), mask, dWc, dWc, dWc, ws), ValueError)]:
        with pytest.raises(error):
            call()
    assert B.slope_launch_count() == launches


def layer(B, b, d_out, d_in, r, seed):
    """Operands of a weight gradient on the GPU, and the decoded activations and mask in 64 bits on the CPU."""
    import torch

    gen = torch.Generator().manual_seed(seed)
    new = lambda *s: torch.randn(s, generator=gen)
    X = new(b, d_in) * torch.exp(new(d_in)) * torch.exp(0.5 * new(b, 1))
    codes, exponents = ref.encode(X.bfloat16().double().numpy())
    t = {"X": ref.decode(codes, exponents), "Xc": torch.from_numpy(ref.buffer(codes, exponents)).cuda(), "dY": new(b, d_out).bfloat16().cuda()}
    kept = new(d_out, d_in // 4, 4).topk(2, -1).indices
    t["keep"] = torch.zeros(d_out, d_in // 4, 4, dtype=torch.bool).scatter_(2, kept, True).reshape(d_out, d_in).numpy()
    t["mask"] = torch.from_numpy(np.packbits(t["keep"], axis=1, bitorder="little")).cuda()
    t["dWc"] = torch.full((d_out, d_in // 2), float("nan"), dtype=torch.bfloat16, device="cuda")
    t["ws"] = torch.full((max(16, B.slope_bwd_dw_q8_workspace_bytes(b, d_out, d_in, r)),), 0xFF, dtype=torch.uint8, device="cuda")
    if r:
        t["T"], t["dT"] = new(b, r).bfloat16().cuda(), new(b, r).bfloat16().cuda()
        t["dL"], t["dR"] = (torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda") for s in ((d_in, r), (r, d_out)))
    return t


def f64(t):
    return t.double().cpu().numpy()


SHAPES = [(1, 128, 128, 0), (1, 128, 256, 16), (63, 256, 128, 0), (64, 128, 384, 32), (65, 640, 384, 0), (300, 512, 512, 64), (257, 384, 1152, 256),
          (1000, 2304, 768, 0), (1000, 2304, 768, 16), (2100, 1024, 1408, 0), (777, 3200, 3328, 64), (640, 3328, 3200, 128), (513, 2560, 4096, 0),
          (5700, 1792, 2048, 0), (5700, 1792, 2560, 64)]


@pytest.mark.parametrize("b,d_out,d_in,r", SHAPES)
def test_weight_gradient_from_a_checkpoint(B, b, d_out, d_in, r):
    """Against the sums over the decoded matrix in 64 bits, element by element as for the bf16 operands (helpers.parity_error)."""
    t = layer(B, b, d_out, d_in, r, b + d_out)
    if r:
        B.slope_linear_bwd_dw_adapter_q8(t["dY"], t["Xc"], t["T"], t["dT"], t["mask"], t["dWc"], t["dL"], t["dR"], t["ws"])
    else:
        B.slope_linear_bwd_dw_masked_q8(t["dY"], t["Xc"], t["mask"], t["dWc"], t["ws"])
    assert B.slope_poll_status() == 0
    dY = f64(t["dY"])
    want = (dY.T @ t["X"])[t["keep"]].reshape(d_out, d_in // 2)
    assert parity_error(f64(t["dWc"]), want) <= REL_TOL
    if r:
        assert parity_error(f64(t["dL"]), t["X"].T @ f64(t["dT"])) <= REL_TOL
        assert parity_error(f64(t["dR"]), f64(t["T"]).T @ dY) <= REL_TOL


@pytest.mark.parametrize("b,d_out,d_in", [(1, 128, 128), (300, 512, 640), (1000, 2304, 768), (513, 2560, 4096), (5700, 1792, 2048)])
def test_dense_weight_gradient_from_a_checkpoint(B, b, d_out, d_in):
    import torch

    t = layer(B, b, d_out, d_in, 0, b)
    dW = torch.full((d_out, d_in), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.slope_dense_linear_bwd_dw_q8(t["dY"], t["Xc"], dW, t["ws"])
    assert B.slope_poll_status() == 0
    assert parity_error(f64(dW), f64(t["dY"]).T @ t["X"]) <= REL_TOL


@pytest.mark.parametrize("b,d_out,d_in,r", [(1, 128, 128, 0), (300, 512, 640, 16), (1000, 2304, 768, 0), (777, 3200, 3328, 64), (5700, 1792, 2048, 0)])
def test_the_bits_are_those_of_the_matrix_read_back(B, b, d_out, d_in, r):
    import torch

    t = layer(B, b, d_out, d_in, r, 5)
    X = torch.empty(b, d_in, dtype=torch.bfloat16, device="cuda")
    B.slope_checkpoint_load(t["Xc"], X)
    want = {k: torch.empty_like(t[k]) for k in ("dWc", "dL", "dR") if k in t}
    if r:
        ws = torch.empty(B.slope_bwd_dw_adapter_workspace_bytes(b, d_out, d_in, r), dtype=torch.uint8, device="cuda")
        B.slope_linear_bwd_dw_adapter(t["dY"], X, t["T"], t["dT"], t["mask"], want["dWc"], want["dL"], want["dR"], ws)
        B.slope_linear_bwd_dw_adapter_q8(t["dY"], t["Xc"], t["T"], t["dT"], t["mask"], t["dWc"], t["dL"], t["dR"], t["ws"])
    else:
        B.slope_linear_bwd_dw_masked(t["dY"], X, t["mask"], want["dWc"])
        B.slope_linear_bwd_dw_masked_q8(t["dY"], t["Xc"], t["mask"], t["dWc"], t["ws"])
        dense = [torch.empty(d_out, d_in, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        B.slope_dense_linear_bwd_dw(t["dY"], X, dense[0])
        B.slope_dense_linear_bwd_dw_q8(t["dY"], t["Xc"], dense[1], t["ws"])
        assert torch.equal(dense[0], dense[1])
    assert all(torch.equal(want[k], t[k]) for k in want)


@pytest.mark.parametrize("b,d_out,d_in", [(200, 256, 512), (700, 2560, 4096)])
def test_an_overflow_shows_in_the_gradient(B, b, d_out, d_in):
    """A block that held an infinity reads back as NaN: the columns of its 32 inputs are NaN in every row, no other is."""
    import torch

    t = layer(B, b, d_out, d_in, 0, 3)
    codes, exponents = ref.split(t["Xc"].cpu().numpy(), b, d_in)
    codes[b // 2, 64:96], exponents[b // 2, 2] = 0, 255
    t["Xc"] = torch.from_numpy(ref.buffer(codes, exponents)).cuda()
    dW = torch.zeros((d_out, d_in), dtype=torch.bfloat16, device="cuda")
    B.slope_dense_linear_bwd_dw_q8(t["dY"], t["Xc"], dW, t["ws"])
    assert torch.isnan(dW[:, 64:96]).all() and torch.isfinite(dW[:, :64]).all() and torch.isfinite(dW[:, 96:]).all()


@pytest.mark.parametrize("r", [0, 64])
def test_calls_are_deterministic_and_replay_in_a_graph(B, r):
    import torch

    b, d_out, d_in = 1500, 2560, 3200
    t, u = layer(B, b, d_out, d_in, r, 11), layer(B, b, d_out, d_in, r, 12)

    def call(t):
        if r:
            B.slope_linear_bwd_dw_adapter_q8(t["dY"], t["Xc"], t["T"], t["dT"], t["mask"], t["dWc"], t["dL"], t["dR"], t["ws"])
        else:
            B.slope_linear_bwd_dw_masked_q8(t["dY"], t["Xc"], t["mask"], t["dWc"], t["ws"])
        return {k: t[k] for k in ("dWc", "dL", "dR") if k in t}

    first = {k: v.clone() for k, v in call(t).items()}
    other = {k: v.clone() for k, v in call(u).items()}
    again = call(t)
    assert all(torch.equal(first[k], again[k]) for k in first)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(t)
    for k in first:
        t[k].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(first[k], t[k]) for k in first)
    for k in ("Xc", "dY", "mask", "T", "dT"):                                # other operands in the same buffers
        if k in t:
            t[k].copy_(u[k])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(other[k], t[k]) for k in other)
    assert B.slope_poll_status() == 0
