"""GPU: softmax attention, forward and backward, against its definition in 64 bits, element by element (bounds: attention_reference)."""
import pytest

import attention_reference as ref

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


def tensors(b, heads, kv, hd, seed=0, sigma=1.0):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda n: (torch.randn(b, n * hd, device="cuda", generator=gen) * sigma).bfloat16()
    return new(heads), new(kv), new(kv), new(heads)


def run(B, Q, K, V, dO, hd, **batch):
    """Outputs in matrices that held 7 before."""
    import torch

    O, dQ, dK, dV = (torch.full(x.shape, 7.0, dtype=torch.bfloat16, device="cuda") for x in (Q, Q, K, V))
    lse = torch.full((Q.shape[1] // hd, Q.shape[0]), 7.0, device="cuda")
    B.slope_attention_fwd(Q, K, V, hd, O, lse, **batch)
    ws = torch.empty(B.slope_attention_bwd_workspace_bytes(Q.shape[0], Q.shape[1] // hd, K.shape[1] // hd, hd), dtype=torch.uint8, device="cuda")
    B.slope_attention_bwd(dO, Q, K, V, O, lse, hd, dQ, dK, dV, ws, **batch)
    assert B.slope_poll_status() == 0
    return {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV}


def compare(got, Q, K, V, dO, hd, sequences, causal=True, window=0, scale=None):
    want = ref.attention(Q, K, V, hd, sequences, causal, window, scale)
    want |= ref.attention(Q, K, V, hd, sequences, causal, window, scale, dO, got["O"], got["lse"])
    for name, pair in want.items():
        ref.check(got[name], pair, name)
        outside = pair[0].isnan()
        assert (got[name][outside] == 7).all(), name             # rows of no sequence are as they were


LENGTHS = [1, 2, 16, 17, 100, 127, 128, 129, 255, 256, 257, 300, 384, 511, 520, 1000]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", LENGTHS)
def test_lengths(B, hd, causal, n):
    Q, K, V, dO = tensors(2 * n, 2, 2, hd, n)
    got = run(B, Q, K, V, dO, hd, sequences=2, causal=causal)
    compare(got, Q, K, V, dO, hd, [(0, n), (n, n)], causal)


@pytest.mark.parametrize("hd", [8, 16, 24, 32, 40, 72, 80, 96, 112, 120])
def test_head_widths(B, hd):
    Q, K, V, dO = tensors(333, 3, 3, hd, hd)
    compare(run(B, Q, K, V, dO, hd), Q, K, V, dO, hd, [(0, 333)])
    compare(run(B, Q, K, V, dO, hd, causal=False), Q, K, V, dO, hd, [(0, 333)], False)


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 2), (8, 1), (6, 2), (25, 5)])
def test_shared_key_heads(B, heads, kv):
    for hd in (64, 128):
        Q, K, V, dO = tensors(290, heads, kv, hd, heads)
        compare(run(B, Q, K, V, dO, hd), Q, K, V, dO, hd, [(0, 290)])


@pytest.mark.parametrize("window", [1, 2, 64, 127, 128, 129, 130, 255, 256, 257, 400, 699, 700, 5000, 2 ** 31 - 1])
def test_windows(B, window):
    for hd in (64, 128):
        Q, K, V, dO = tensors(700, 2, 1, hd, window % 1000)
        compare(run(B, Q, K, V, dO, hd, window=window), Q, K, V, dO, hd, [(0, 700)], True, window)


@pytest.mark.parametrize("causal", [True, False])
def test_packed_sequences(B, causal):
    """Sequences of length 0 among them, rows in front of the first and behind the last; more sequences than a warp looks through at once."""
    import torch

    starts = [3, 3, 140, 141, 141, 400, 656, 912] + [912 + 5 * i for i in range(1, 70)]
    b = starts[-1] + 9
    sequences = [(a, z - a) for a, z in zip(starts, starts[1:])]
    for hd in (64, 128):
        Q, K, V, dO = tensors(b, 2, 2, hd, 11)
        got = run(B, Q, K, V, dO, hd, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"), causal=causal)
        compare(got, Q, K, V, dO, hd, sequences, causal)


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 70), (False, 0)])
def test_padded_batches(B, causal, window):
    import torch

    lengths = [300, 0, 1, 299, 128, 256, 17]
    for hd in (64, 128):
        Q, K, V, dO = tensors(300 * len(lengths), 2, 2, hd, 12)
        got = run(B, Q, K, V, dO, hd, sequences=len(lengths), lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), causal=causal, window=window)
        compare(got, Q, K, V, dO, hd, [(300 * i, n) for i, n in enumerate(lengths)], causal, window)
    # starts and lengths together; lengths beyond their part and below zero
    starts, lengths = [0, 200, 500, 500], [150, 400, -3]
    Q, K, V, dO = tensors(510, 2, 2, 64, 13)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    got = run(B, Q, K, V, dO, 64, starts=on(starts), lengths=on(lengths), causal=causal, window=window)
    compare(got, Q, K, V, dO, 64, [(0, 150), (200, 300)], causal, window)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_of_no_sequence_reach_no_other(B, bad, causal):
    """Padding rows and other sequences may hold anything."""
    import torch

    part, lengths = 300, [290, 37, 128, 5]
    for hd in (64, 128, 80):
        clean = tensors(part * len(lengths), 2, 2, hd, 14)
        inside = torch.zeros(part * len(lengths), dtype=torch.bool, device="cuda")
        for i, n in enumerate(lengths):
            inside[part * i:part * i + n] = True
        dirty = [x.masked_fill(~inside[:, None], bad) for x in clean]
        batch = {"sequences": len(lengths), "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "causal": causal}
        a, b = run(B, *clean, hd, **batch), run(B, *dirty, hd, **batch)
        for name in a:
            assert torch.equal(a[name], b[name]), name
        # a sequence that is not finite leaves its neighbours as they are
        starts = torch.tensor([0, 100, 350, 600], dtype=torch.int32, device="cuda")
        x = [t[:600].clone() for t in clean]
        y = [t.clone() for t in x]
        for t in y:
            t[100:350] = bad
        a, b = run(B, *x, hd, starts=starts, causal=causal), run(B, *y, hd, starts=starts, causal=causal)
        keep = torch.cat([torch.arange(100), torch.arange(350, 600)]).cuda()
        for name in a:
            axis = 1 if name == "lse" else 0
            assert torch.equal(a[name].index_select(axis, keep), b[name].index_select(axis, keep)), name


def test_values_that_are_not_finite_show(B):
    import torch

    Q, K, V, dO = tensors(300, 1, 1, 64, 15)
    Q[40, 3] = float("nan")
    K[250, 5] = float("inf")
    got = run(B, Q, K, V, dO, 64)
    bad = got["O"].isnan().any(1)
    # a score of minus infinity is a probability of zero: the row has its value; one of plus infinity makes it NaN
    assert torch.equal(bad[250:], Q[250:, 5] > 0)
    assert bad[40] and not bad[:40].any() and not bad[41:128].any()
    V[10, 0] = float("inf")
    got = run(B, Q, K, V, dO, 64)
    assert not got["O"][10:, 0].isfinite().any()


@pytest.mark.parametrize("sigma", [1e-3, 8.0])
def test_flat_and_peaked_scores(B, sigma):
    """Nearly equal probabilities, and scores in the hundreds whose maximum keeps rising along the keys."""
    import torch

    for hd in (64, 128):
        Q, K, V, dO = tensors(640, 2, 2, hd, 16)
        rise = torch.linspace(0.2, 1.0, 640, device="cuda")[:, None]
        Q, K = (Q.float() * sigma ** 0.5).bfloat16(), (K.float() * rise * sigma ** 0.5).bfloat16()
        for causal in (True, False):
            compare(run(B, Q, K, V, dO, hd, causal=causal), Q, K, V, dO, hd, [(0, 640)], causal)


def test_scale(B):
    Q, K, V, dO = tensors(200, 2, 2, 64, 17)
    for scale in (1.0, 0.01):
        compare(run(B, Q, K, V, dO, 64, scale=scale), Q, K, V, dO, 64, [(0, 200)], True, 0, scale)


def test_columns_of_one_matrix(B):
    """Q, K and V side by side in the output of one projection, and the gradients in the same places; the rest is not touched."""
    import torch

    hd, heads, kv, b = 64, 4, 2, 300
    Q, K, V, dO = tensors(b, heads, kv, hd, 18)
    a = run(B, Q, K, V, dO, hd)
    wide = torch.full((b, (heads + 2 * kv) * hd + 24), 9.0, dtype=torch.bfloat16, device="cuda")
    cut = lambda m: (m[:, 8:8 + heads * hd], m[:, 8 + heads * hd:8 + (heads + kv) * hd], m[:, 8 + (heads + kv) * hd:8 + (heads + 2 * kv) * hd])
    for part, x in zip(cut(wide), (Q, K, V)):
        part.copy_(x)
    grads, O = torch.full_like(wide, 9.0), torch.full((b, heads * hd + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(heads, b, device="cuda")
    B.slope_attention_fwd(*cut(wide), hd, O[:, :heads * hd], lse)
    ws = torch.empty(B.slope_attention_bwd_workspace_bytes(b, heads, kv, hd), dtype=torch.uint8, device="cuda")
    gO = torch.full_like(O, 9.0)
    gO[:, :heads * hd] = dO
    B.slope_attention_bwd(gO[:, :heads * hd], *cut(wide), O[:, :heads * hd], lse, hd, *cut(grads), ws)
    assert B.slope_poll_status() == 0
    assert torch.equal(O[:, :heads * hd], a["O"]) and torch.equal(lse, a["lse"]) and (O[:, heads * hd:] == 9).all()
    for part, name in zip(cut(grads), ("dQ", "dK", "dV")):
        assert torch.equal(part, a[name]), name
    assert (grads[:, :8] == 9).all() and (grads[:, 8 + (heads + 2 * kv) * hd:] == 9).all()


def test_same_bits_again(B):
    import torch

    for hd, heads, kv in ((64, 12, 12), (128, 8, 2)):
        Q, K, V, dO = tensors(4 * 520, heads, kv, hd, 19)
        first = run(B, Q, K, V, dO, hd, sequences=4)
        for _ in range(5):
            again = run(B, Q, K, V, dO, hd, sequences=4)
            for name in first:
                assert torch.equal(first[name], again[name]), name
        # a sequence's results do not depend on where it stands
        one = run(B, *(x[1040:1560].contiguous() for x in (Q, K, V, dO)), hd)
        for name in first:
            got = first[name][:, 1040:1560] if name == "lse" else first[name][1040:1560]
            assert torch.equal(got, one[name]), name


def test_without_lse_and_on_another_stream_and_in_a_graph(B):
    import torch

    hd = 128
    Q, K, V, dO = tensors(2 * 400, 4, 2, hd, 20)
    want = run(B, Q, K, V, dO, hd, sequences=2)
    O = torch.zeros_like(Q)
    B.slope_attention_fwd(Q, K, V, hd, O, sequences=2)
    assert torch.equal(O, want["O"])
    lse, grads = torch.empty(4, 800, device="cuda"), [torch.zeros_like(x) for x in (Q, K, V)]
    ws = torch.empty(B.slope_attention_bwd_workspace_bytes(800, 4, 2, hd), dtype=torch.uint8, device="cuda")
    inputs = [torch.zeros_like(x) for x in (Q, K, V, dO)]
    side = torch.cuda.Stream()

    def step():
        B.slope_attention_fwd(*inputs[:3], hd, O, lse, sequences=2)
        B.slope_attention_bwd(inputs[3], *inputs[:3], O, lse, hd, *grads, ws, sequences=2)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t, x in zip(inputs, (Q, K, V, dO)):
            t.copy_(x)
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t, name in zip((O, lse, *grads), ("O", "lse", "dQ", "dK", "dV")):
        assert torch.equal(t, want[name]), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other = tensors(800, 4, 2, hd, 21)
    want = run(B, *other, hd, sequences=2)
    for t, x in zip(inputs, other):
        t.copy_(x)
    for _ in range(3):
        for t in (O, lse, *grads):
            t.zero_()
        graph.replay()
        for t, name in zip((O, lse, *grads), ("O", "lse", "dQ", "dK", "dV")):
            assert torch.equal(t, want[name]), name
    assert B.slope_poll_status() == 0


def test_a_gradient_against_differences(B):
    """d(sum O dO) along a direction, from the forward pass in 64 bits at both ends of a short step."""
    import torch

    hd, n = 64, 200
    Q, K, V, dO = tensors(n, 2, 1, hd, 22)
    got = run(B, Q, K, V, dO, hd)
    step = 2.0 ** -10
    for i, name in enumerate(("dQ", "dK", "dV")):
        d = torch.randn((Q, K, V)[i].shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(i))
        ends = []
        for sign in (1, -1):
            x = [t.double() for t in (Q, K, V)]
            x[i] = x[i] + sign * step * d
            ends.append(float((ref.attention(*x, hd, [(0, n)], True)["O"][0] * dO.double()).sum()))
        slope = (ends[0] - ends[1]) / (2 * step)
        along = got[name].double() * d
        # roundings are independent: their sum is that of the squares; six sigma of one rounding and of two operands'
        assert abs(float(along.sum()) - slope) <= 6 * 2.0 ** -8 * float(along.norm()) + 1e-4 * float(along.abs().sum()), name


def test_long_sequence(B):
    import torch

    hd, n = 128, 5000
    Q, K, V, dO = tensors(n, 2, 1, hd, 23)
    compare(run(B, Q, K, V, dO, hd), Q, K, V, dO, hd, [(0, n)])


@pytest.mark.parametrize("hd,heads,kv,lengths,causal,window", [
    (64, 8, 4, [5000, 300, 1000], False, 0), (64, 4, 2, [8000, 300, 4000], True, 0),
    (128, 12, 6, [1000, 1, 0, 900, 2040], False, 0), (128, 12, 6, [1000, 1, 2300, 900, 2040], True, 0), (128, 12, 6, [600] * 6, True, 520),
])
def test_blocks_of_two_tiles(B, hd, heads, kv, lengths, causal, window):
    """Many keys to a query and blocks enough for every SM: the forward pass takes 256 queries to a block."""
    import torch

    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    Q, K, V, dO = tensors(starts[-1], heads, kv, hd, 24)
    got = run(B, Q, K, V, dO, hd, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"), causal=causal, window=window)
    compare(got, Q, K, V, dO, hd, list(zip(starts, lengths)), causal, window)


@pytest.mark.parametrize("lengths", [[600, 0, 1, 599, 256, 257], [255, 129, 128, 127, 512, 513]])
def test_blocks_of_two_tiles_in_padded_batches(B, lengths):
    import torch

    hd, heads = 128, 9
    clean = tensors(1100 * len(lengths), heads, heads, hd, 25)
    inside = torch.zeros(1100 * len(lengths), dtype=torch.bool, device="cuda")
    for i, n in enumerate(lengths):
        inside[1100 * i:1100 * i + n] = True
    for causal in (True, False):
        batch = {"sequences": len(lengths), "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "causal": causal}
        for bad in (0.0, float("nan")):
            Q, K, V, dO = (x.masked_fill(~inside[:, None], bad) for x in clean)
            compare(run(B, Q, K, V, dO, hd, **batch), Q, K, V, dO, hd, [(1100 * i, n) for i, n in enumerate(lengths)], causal)


def test_nothing_to_do(B):
    """Sequences that are all empty: the call returns, and nothing is written."""
    import torch

    for hd in (64, 128):
        Q, K, V, dO = tensors(600, 2, 1, hd, 26)
        for batch in ({"sequences": 2, "lengths": torch.zeros(2, dtype=torch.int32, device="cuda")},
                      {"starts": torch.full((6,), 300, dtype=torch.int32, device="cuda")}):
            for name, x in run(B, Q, K, V, dO, hd, **batch).items():
                assert (x == 7).all(), name


@pytest.mark.parametrize("hd,heads,n", [(64, 16, 1024), (128, 40, 512)])
def test_more_blocks_than_fit_at_once(B, hd, heads, n):
    """Several times as many blocks as the device holds, on two streams at once: every sequence as if it were alone."""
    import torch

    x = tensors(4 * n, heads, heads // 4, hd, 27)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = run(B, *x, hd, sequences=4)
    with torch.cuda.stream(side):
        b = run(B, *x, hd, sequences=4)
    torch.cuda.synchronize()
    for name in a:
        assert torch.equal(a[name], b[name]), name
    Q, K, V, dO = (t[2 * n:3 * n] for t in x)
    got = {name: t[:, 2 * n:3 * n] if name == "lse" else t[2 * n:3 * n] for name, t in a.items()}
    compare(got, Q, K, V, dO, hd, [(0, n)])


@pytest.mark.parametrize("hd,n,causal", [(24, 333, True), (64, 384, False), (128, 200, True)])
def test_small_calls_many_times(B, hd, n, causal):
    """A few blocks whose first tiles are used up at once: no order of a block's warps may leave one of them waiting."""
    import torch

    Q, K, V, dO = tensors(n, 3, 3, hd, 28)
    want = run(B, Q, K, V, dO, hd, causal=causal)
    O, lse, grads = torch.empty_like(Q), torch.empty(3, n, device="cuda"), [torch.empty_like(x) for x in (Q, K, V)]
    ws = torch.empty(B.slope_attention_bwd_workspace_bytes(n, 3, 3, hd), dtype=torch.uint8, device="cuda")
    for _ in range(2000):
        B.slope_attention_fwd(Q, K, V, hd, O, lse, causal=causal)
        B.slope_attention_bwd(dO, Q, K, V, O, lse, hd, *grads, ws, causal=causal)
    assert B.slope_poll_status() == 0
    for name, x in zip(("O", "lse", "dQ", "dK", "dV"), (O, lse, *grads)):
        assert torch.equal(x, want[name]), name
