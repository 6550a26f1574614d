"""GPU: queries and keys turned by their positions, against the definition in 64 bits."""
import math

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


def matrices(b, heads, kv, hd, dtype, seed=0):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(seed)
    return tuple(torch.randn(b, n * hd, device="cuda", generator=gen).to(dtype) for n in (heads, kv))


def check(got, X, positions, frequencies, hd, factor, interleaved, backward):
    import torch

    want = ref.rotary(X, positions, frequencies, hd, factor, interleaved, backward)
    half = 2.0 ** -8 if X.dtype == torch.bfloat16 else 2.0 ** -24
    bound = ref.rotary_bound(X, want, hd, frequencies.numel(), factor, interleaved, half)
    off = (got.double() - want).abs()
    assert (off <= bound).all(), float((off / bound.clamp_min(1e-30)).max())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,rot", [(128, 128), (128, 64), (64, 16), (80, 20), (80, 80), (96, 24), (112, 28), (64, 10), (64, 2), (8, 6), (256, 256), (4096, 4096)])
def test_widths(B, dtype, interleaved, hd, rot):
    import torch

    b, heads, kv = 77, 5, 2
    Q, K = matrices(b, heads, kv, hd, getattr(torch, dtype), rot)
    positions = torch.randint(0, 5000, (b,), dtype=torch.int32, device="cuda")
    f = B.rotary_frequencies(rot)
    for backward in (False, True):
        Qr, Kr = torch.full_like(Q, 7.0), torch.full_like(K, 7.0)
        B.slope_rotary(Q, K, positions, f, hd, Qr, Kr, factor=1.25, interleaved=interleaved, backward=backward)
        assert B.slope_poll_status() == 0
        check(Qr, Q, positions, f, hd, 1.25, interleaved, backward)
        check(Kr, K, positions, f, hd, 1.25, interleaved, backward)
        q, k = Q.clone(), K.clone()
        B.slope_rotary(q, k, positions, f, hd, q, k, factor=1.25, interleaved=interleaved, backward=backward)
        assert torch.equal(q, Qr) and torch.equal(k, Kr)          # in place: the same bits
        alone = torch.full_like(Q, 7.0)
        B.slope_rotary(Q, None, positions, f, hd, alone, None, factor=1.25, interleaved=interleaved, backward=backward)
        assert torch.equal(alone, Qr)


@pytest.mark.parametrize("b", [1, 2, 3, 5, 64, 1000, 4099])
def test_tokens(B, b):
    import torch

    Q, K = matrices(b, 4, 1, 128, torch.bfloat16, b)
    positions = torch.arange(b, dtype=torch.int32, device="cuda") + 17
    f = B.rotary_frequencies(128, scaling="parts", stretch=4.0)
    Qr, Kr = torch.empty_like(Q), torch.empty_like(K)
    B.slope_rotary(Q, K, positions, f, 128, Qr, Kr)
    check(Qr, Q, positions, f, 128, 1.0, False, False)
    check(Kr, K, positions, f, 128, 1.0, False, False)


def test_far_positions(B):
    """Any 32-bit position: angles are reduced in fp64.  (Bound 2^-20 of a pair: 1e-7 of a turn is 6.3e-7 rad.)"""
    import torch

    far = [0, 1, -1, 10 ** 6, 10 ** 6 + 1, 123456789, 2 ** 31 - 1, -2 ** 31]
    positions = torch.tensor(far, dtype=torch.int32, device="cuda")
    Q, _ = matrices(len(far), 3, 1, 128, torch.float32, 3)
    f = B.rotary_frequencies(128, base=500000.0)
    Qr = torch.empty_like(Q)
    B.slope_rotary(Q, None, positions, f, 128, Qr, None)
    check(Qr, Q, positions, f, 128, 1.0, False, False)


def test_backward_is_the_transposed_map(B):
    """<R x, y> = <x, R^T y>, and there and back is the identity times factor^2."""
    import torch

    X, _ = matrices(50, 4, 1, 64, torch.float32, 4)
    Y, _ = matrices(50, 4, 1, 64, torch.float32, 5)
    positions = torch.arange(50, dtype=torch.int32, device="cuda") * 31
    for interleaved in (False, True):
        f = B.rotary_frequencies(32)
        RX, RtY, back = (torch.empty_like(X) for _ in range(3))
        B.slope_rotary(X, None, positions, f, 64, RX, None, factor=1.5, interleaved=interleaved)
        B.slope_rotary(Y, None, positions, f, 64, RtY, None, factor=1.5, interleaved=interleaved, backward=True)
        a, b = float((RX.double() * Y.double()).sum()), float((X.double() * RtY.double()).sum())
        # 12800 terms with independent relative errors of a few 2^-24, six sigma
        assert abs(a - b) <= 6 * 2.0 ** -21 * math.sqrt(float(((RX.double() * Y.double()) ** 2).sum()))
        B.slope_rotary(RX, None, positions, f, 64, back, None, factor=1.5, interleaved=interleaved, backward=True)
        want = X.double().reshape(50, 4, 64).clone()
        want[..., :32] *= 2.25
        assert (back.double() - want.reshape(50, 256)).abs().max() <= 2.0 ** -19 * float(want.abs().max())


def test_columns_of_a_wider_matrix_graph_and_stream(B):
    import torch

    b, hd, heads, kv = 130, 64, 3, 2
    Q, K = matrices(b, heads, kv, hd, torch.bfloat16, 6)
    positions = torch.arange(b, dtype=torch.int32, device="cuda")
    f = B.rotary_frequencies(hd)
    Qr, Kr = torch.empty_like(Q), torch.empty_like(K)
    B.slope_rotary(Q, K, positions, f, hd, Qr, Kr)
    wide = torch.full((b, (heads + kv) * hd + 16), 9.0, dtype=torch.bfloat16, device="cuda")
    q, k = wide[:, 8:8 + heads * hd], wide[:, 8 + heads * hd:8 + (heads + kv) * hd]
    q.copy_(Q)
    k.copy_(K)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.slope_rotary(q, k, positions, f, hd, q, k)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(q, Qr) and torch.equal(k, Kr) and (wide[:, :8] == 9).all() and (wide[:, -8:] == 9).all()
    graph, out, out_k = torch.cuda.CUDAGraph(), torch.zeros_like(Q), torch.zeros_like(K)
    with torch.cuda.graph(graph):
        B.slope_rotary(Q, K, positions, f, hd, out, out_k)
    positions += 5
    graph.replay()
    check(out, Q, positions, f, hd, 1.0, False, False)
    assert B.slope_poll_status() == 0


def test_frequencies(B):
    import torch

    f = B.rotary_frequencies(8, base=10000.0, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14)
