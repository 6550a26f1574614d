"""CPU-only checks of attention and of the rotation by positions: workspace sizes, every kind of refusal before any CUDA call, the
binding's checks, the frequencies, and the reference of the GPU tests against autograd and differences."""
import ctypes
import math

import pytest
import torch

import attention_reference as ref

BF16, F32, Q8 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2608_24070_b200 import binding, build

    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def a():
    """A 16-byte aligned host address: no call here gets as far as reading it."""
    buf = ctypes.create_string_buffer(64)
    yield (ctypes.addressof(buf) + 15) & ~15


def test_workspace(lib):
    size = lib.slope_attention_bwd_workspace_bytes
    assert size(1000, 12, 12, 64) >= 4 * 12 * 1000 and size(1 << 20, 128, 8, 128) >= 4 << 27
    assert size(0, 12, 12, 64) == 0 and size(16, 12, 5, 64) == 0 and size(16, 12, 12, 60) == 0 and size(16, 12, 12, 136) == 0


def test_attention_refusals(lib, a):
    shape = dict(b=256, heads=4, kv=2, hd=64, sequences=2, starts=None, lengths=None, causal=1, window=0, scale=0.125)

    def fwd(Q=a, K=a, V=a, O=a, lse=a, q_ld=256, k_ld=128, v_ld=128, o_ld=256, **change):
        s = {**shape, **change}
        return lib.slope_attention_fwd(Q, q_ld, K, k_ld, V, v_ld, s["b"], s["heads"], s["kv"], s["hd"], s["sequences"], s["starts"], s["lengths"],
                                       s["causal"], s["window"], s["scale"], O, o_ld, lse, None)

    def bwd(dO=a, Q=a, K=a, V=a, O=a, lse=a, dQ=a, dK=a, dV=a, ws=a, n=1 << 30, do_ld=256, q_ld=256, k_ld=128, v_ld=128, o_ld=256, dq_ld=256, dk_ld=128,
            dv_ld=128, **change):
        s = {**shape, **change}
        return lib.slope_attention_bwd(dO, do_ld, Q, q_ld, K, k_ld, V, v_ld, O, o_ld, lse, s["b"], s["heads"], s["kv"], s["hd"], s["sequences"],
                                       s["starts"], s["lengths"], s["causal"], s["window"], s["scale"], dQ, dq_ld, dK, dk_ld, dV, dv_ld, ws, n, None)

    for call in (fwd, bwd):
        for name in ("Q", "K", "V", "O"):
            assert call(**{name: None}) == 1 and call(**{name: a + 8}) == 3, name
        for scale in (0.0, -1.0, math.inf, math.nan, 3e38):              # (the last is finite, but not in powers of two)
            assert call(scale=scale) == 1
        assert call(window=-1) == 1 and call(window=5, causal=0) == 1
        assert call(b=0) == 2 and call(b=255) == 2 and call(b=(1 << 30) + 2) == 2 and call(sequences=0) == 2
        assert call(heads=0) == 2 and call(kv=0) == 2 and call(kv=3) == 2 and call(hd=0) == 2 and call(hd=60) == 2 and call(hd=136) == 2
        assert call(heads=1 << 28, kv=1 << 28, hd=64) == 2                                      # more columns than an int counts
        assert call(b=1 << 30, sequences=1, heads=1024, kv=1024, hd=8, **{n: 8192 for n in ("q_ld", "k_ld", "v_ld", "o_ld")}) == 2   # more tiles than a launch has
        for name, least in (("q_ld", 256), ("o_ld", 256), ("k_ld", 128), ("v_ld", 128)):
            assert call(**{name: least - 8}) == 2 and call(**{name: least + 4}) == 2, name
        assert call(starts=a + 4, sequences=3) == 3 and call(lengths=a + 4) == 3
    assert fwd(lse=a + 4) == 3
    for name in ("dO", "lse", "dQ", "dK", "dV", "ws"):
        assert bwd(**{name: None}) == 1 and bwd(**{name: a + 8}) == 3, name
    for name, least in (("do_ld", 256), ("dq_ld", 256), ("dk_ld", 128), ("dv_ld", 128)):
        assert bwd(**{name: least - 8}) == 2 and bwd(**{name: least + 4}) == 2, name
    assert bwd(n=lib.slope_attention_bwd_workspace_bytes(256, 4, 2, 64) - 1) == 1


def test_rotary_refusals(lib, a):
    def call(Q=a, K=a, Qr=a + 32, Kr=a + 32, q_ld=256, k_ld=128, qr_ld=256, kr_ld=128, type=BF16, b=8, heads=4, kv=2, hd=64, rot=32, pos=a, freq=a,
             factor=1.0):
        return lib.slope_rotary(Q, q_ld, K, k_ld, type, b, heads, kv, hd, rot, 0, 0, pos, freq, factor, Qr, qr_ld, Kr, kr_ld, None)

    for name in ("Q", "K", "Qr", "Kr", "pos", "freq"):
        assert call(**{name: None}) == 1, name
    assert call(type=Q8) == 1 and call(factor=math.inf) == 1 and call(factor=math.nan) == 1
    assert call(Qr=a) == 1 and call(Qr=a, Kr=a, qr_ld=264) == 1                                 # in place: both, at the same strides
    assert call(b=0) == 2 and call(heads=0) == 2 and call(kv=0) == 2 and call(hd=60) == 2 and call(hd=4) == 2 and call(hd=8192, q_ld=1 << 20) == 2
    assert call(rot=0) == 2 and call(rot=31) == 2 and call(rot=66) == 2
    for name, least in (("q_ld", 256), ("k_ld", 128), ("qr_ld", 256), ("kr_ld", 128)):
        assert call(**{name: least - 8}) == 2 and call(**{name: least + 4}) == 2, name
    for name in ("Q", "K", "Qr", "Kr", "pos", "freq"):
        assert call(**{name: a + 8}) == 3, name


def test_only_cuda_tensors_are_taken(lib):
    from paper_2608_24070_b200 import binding as B

    x, f = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(32, dtype=torch.float64)
    for call in (lambda: B.slope_attention_fwd(x, x, x, 64, x), lambda: B.slope_attention_bwd(x, x, x, x, x, x, 64, x, x, x, x),
                 lambda: B.slope_rotary(x, None, f, f, 64, x, None)):
        with pytest.raises(AssertionError, match="CUDA"):
            call()


def test_frequencies():
    from paper_2608_24070_b200 import binding as B

    make = lambda *a, **k: B.rotary_frequencies(*a, device="cpu", **k)
    plain = make(64)
    assert plain.dtype == torch.float64 and torch.allclose(plain, 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32), rtol=1e-13)
    assert torch.equal(make(64, scaling="linear", stretch=4.0), plain / 4)
    base = make(64, scaling="base", stretch=4.0)
    assert base[0] == 1.0 and math.isclose(float(base[-1] * 4), float(plain[-1]), rel_tol=1e-12)
    parts = make(64, scaling="parts", stretch=4.0, trained=2048)
    turns = 2048 * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and torch.allclose(parts[turns <= 1], plain[turns <= 1] / 4, rtol=1e-13)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (parts[between] < plain[between]).all() and (parts[between] > plain[between] / 4).all()
    for bad in (dict(rot_dim=63), dict(rot_dim=0), dict(rot_dim=8, base=0.0), dict(rot_dim=8, scaling="other"), dict(rot_dim=8, stretch=0.0),
                dict(rot_dim=2, scaling="base"), dict(rot_dim=8, scaling="parts", fast=1.0, slow=1.0)):
        with pytest.raises(ValueError):
            make(**bad)


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 5), (False, 0)])
def test_the_reference_against_autograd(causal, window):
    """Outputs and gradients of the 64-bit reference against torch's softmax under autograd, shared key heads and two sequences."""
    gen = torch.Generator().manual_seed(1)
    hd, heads, kv, sequences = 8, 4, 2, [(0, 13), (13, 9)]
    new = lambda n: torch.randn(24, n * hd, generator=gen, dtype=torch.float64)
    Q, K, V = (t.requires_grad_(True) for t in (new(heads), new(kv), new(kv)))
    dO, parts = new(heads), []
    for first, n in sequences:
        q, k, v = (t[first:first + n].reshape(n, -1, hd).permute(1, 0, 2) for t in (Q, K, V))
        k, v = (t.repeat_interleave(heads // kv, 0) for t in (k, v))
        S = (q @ k.transpose(1, 2) / math.sqrt(hd)).masked_fill(~ref.visible(n, causal, window, "cpu"), -math.inf)
        parts.append((torch.softmax(S, -1) @ v).permute(1, 0, 2).reshape(n, -1))
    O = torch.cat(parts + [torch.zeros(2, heads * hd, dtype=torch.float64)])
    (O * dO).sum().backward()
    got = ref.attention(Q.detach(), K.detach(), V.detach(), hd, sequences, causal, window)
    assert torch.allclose(got["O"][0][:22], O.detach()[:22], atol=1e-12) and got["O"][0][22:].isnan().all()
    back = ref.attention(Q.detach(), K.detach(), V.detach(), hd, sequences, causal, window, dO=dO, O=O.detach(), lse=got["lse"][0])
    for name, t in (("dQ", Q), ("dK", K), ("dV", V)):
        assert torch.allclose(back[name][0][:22], t.grad[:22], atol=1e-11), name
        assert (back[name][1][:22] >= 0).all()


def test_a_planted_mistake_is_outside_the_bounds():
    """A key left out, a head's gradient dropped from a shared sum, a pair turned the wrong way: each is far outside."""
    gen = torch.Generator().manual_seed(2)
    hd, n = 16, 40
    Q, K, V, dO = (torch.randn(n, c * hd, generator=gen, dtype=torch.float64) for c in (2, 1, 1, 2))
    right = ref.attention(Q, K, V, hd, [(0, n)], True)
    wrong = ref.attention(Q, K, V, hd, [(0, n)], True, window=n - 1)
    with pytest.raises(AssertionError):
        ref.check(wrong["O"][0], right["O"], "O")
    grads = ref.attention(Q, K, V, hd, [(0, n)], True, dO=dO, O=right["O"][0], lse=right["lse"][0])
    one = ref.attention(Q[:, :hd], K, V, hd, [(0, n)], True, dO=dO[:, :hd], O=right["O"][0][:, :hd], lse=right["lse"][0][:1])
    for name in ("dK", "dV"):
        with pytest.raises(AssertionError):
            ref.check(one[name][0], grads[name], name)
    positions, f = torch.arange(n), torch.ones(8, dtype=torch.float64) * 0.3
    want, other = (ref.rotary(Q, positions, f, hd, backward=back) for back in (False, True))
    assert ((other - want).abs() > ref.rotary_bound(Q, want, hd, 8, 1.0, False, 2.0 ** -8)).any()
