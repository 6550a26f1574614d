"""CPU-only checks of the layer norm, the 8-bit checkpoints and the weight gradients from them: sizes, every kind of refusal
before any CUDA call, and the format's definition."""
import ctypes

import numpy as np
import pytest

import norm_reference as ref

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


def test_sizes(lib):
    assert lib.slope_checkpoint_bytes(3, 96) == 3 * 96 + 9
    assert lib.slope_checkpoint_bytes(1 << 20, 16384) == (1 << 34) + (1 << 29)
    assert lib.slope_checkpoint_bytes(3, 100) == 0 and lib.slope_checkpoint_bytes(0, 96) == 0 and lib.slope_checkpoint_bytes(3, -32) == 0
    assert lib.slope_layer_norm_bwd_workspace_bytes(1, 512) == 0                   # one block: no sums to join
    assert lib.slope_layer_norm_bwd_workspace_bytes(16384, 4096) % (2 * 4 * 4096) == 0
    assert lib.slope_layer_norm_bwd_workspace_bytes(16384, 4096) > 0
    assert lib.slope_layer_norm_bwd_workspace_bytes(0, 512) == 0 and lib.slope_layer_norm_bwd_workspace_bytes(8, 1 << 20) == 0
    assert lib.slope_bwd_dw_q8_workspace_bytes(0, 128, 128, 0) == 0
    assert lib.slope_bwd_dw_q8_workspace_bytes(512, 4096, 4096, 64) >= lib.slope_bwd_dw_q8_workspace_bytes(512, 4096, 4096, 0)


def test_checkpoint_refusals(lib, a):
    assert lib.slope_checkpoint_store(None, BF16, 4, 64, a, None) == 1
    assert lib.slope_checkpoint_store(a, BF16, 4, 64, None, None) == 1
    assert lib.slope_checkpoint_store(a, Q8, 4, 64, a, None) == 1                  # not a plain type
    assert lib.slope_checkpoint_store(a, BF16, 4, 48, a, None) == 2                # half a block
    assert lib.slope_checkpoint_store(a, BF16, 0, 64, a, None) == 2
    assert lib.slope_checkpoint_store(a + 8, BF16, 4, 64, a, None) == 3
    assert lib.slope_checkpoint_load(a, 4, 64, a, 7, None) == 1
    assert lib.slope_checkpoint_load(a, 4, 33, a, F32, None) == 2
    assert lib.slope_checkpoint_load(a, 4, 64, a + 4, F32, None) == 3


def test_layer_norm_refusals(lib, a):
    def fwd(X=a, x_type=BF16, residual=None, gamma=a, beta=a, p_type=BF16, b=4, d=64, eps=1e-5, H=None, Y=a, mean=None, rstd=None, Hc=None, Yc=None):
        return lib.slope_layer_norm_fwd(X, x_type, residual, gamma, beta, p_type, b, d, eps, H, Y, mean, rstd, Hc, Yc, None)

    assert fwd(X=None) == 1 and fwd(Y=None) == 1 and fwd(x_type=Q8) == 1 and fwd(p_type=Q8) == 1
    assert fwd(eps=-1.0) == 1 and fwd(eps=float("nan")) == 1 and fwd(eps=float("inf")) == 1
    assert fwd(H=a) == 1                                                           # a sum without a residual
    assert fwd(mean=a) == 1 and fwd(rstd=a) == 1                                   # one statistic without the other
    assert fwd(b=0) == 2 and fwd(d=0) == 2 and fwd(d=12) == 2 and fwd(d=16392) == 2
    assert fwd(d=40, Hc=a) == 2 and fwd(d=40, Yc=a) == 2                           # a checkpoint has whole blocks
    for name in ("X", "residual", "gamma", "beta", "Y", "Hc", "Yc"):
        assert fwd(**{name: a + 2}) == 3, name
    assert fwd(residual=a, H=a + 2) == 3 and fwd(mean=a + 4, rstd=a) == 3 and fwd(mean=a, rstd=a + 4) == 3

    def bwd(dY=a, H=a, h_type=BF16, mean=a, rstd=a, gamma=a, p_type=BF16, dH=None, b=4, d=64, dX=a, dx_type=BF16, dgamma=a, dbeta=a, ws=a, n=1 << 30):
        return lib.slope_layer_norm_bwd(dY, H, h_type, mean, rstd, gamma, p_type, dH, b, d, dX, dx_type, dgamma, dbeta, ws, n, None)

    for name in ("dY", "H", "mean", "rstd", "dX"):
        assert bwd(**{name: None}) == 1, name
    assert bwd(h_type=3) == 1 and bwd(dx_type=Q8) == 1 and bwd(p_type=Q8) == 1
    assert bwd(b=0) == 2 and bwd(d=4) == 2 and bwd(d=16392) == 2 and bwd(h_type=Q8, d=72) == 2
    for name in ("dY", "H", "mean", "rstd", "gamma", "dH", "dX", "dgamma", "dbeta", "ws"):
        assert bwd(**{name: a + 8}) == 3, name
    need = lib.slope_layer_norm_bwd_workspace_bytes(4096, 64)
    assert need > 0 and bwd(b=4096, n=need - 1) == 1 and bwd(b=4096, ws=None) == 1


def test_weight_gradient_refusals(lib, a):
    big = 1 << 40
    assert lib.slope_linear_bwd_dw_masked_q8(a, None, 16, 128, 128, a, a, a, big, None) == 1
    assert lib.slope_linear_bwd_dw_masked_q8(a, a, 16, 128, 128, None, a, a, big, None) == 1
    assert lib.slope_linear_bwd_dw_masked_q8(a, a, 16, 128, 96, a, a, a, big, None) == 2
    assert lib.slope_linear_bwd_dw_masked_q8(a, a, 0, 128, 128, a, a, a, big, None) == 2
    assert lib.slope_linear_bwd_dw_masked_q8(a, a + 8, 16, 128, 128, a, a, a, big, None) == 3
    assert lib.slope_linear_bwd_dw_adapter_q8(a, a, a, a, 16, 128, 128, 0, a, a, a, a, a, big, None) == 2
    assert lib.slope_linear_bwd_dw_adapter_q8(a, a, a, a, 16, 128, 128, 24, a, a, a, a, a, big, None) == 2
    assert lib.slope_linear_bwd_dw_adapter_q8(a, a, a, None, 16, 128, 128, 16, a, a, a, a, a, big, None) == 1
    assert lib.slope_linear_bwd_dw_adapter_q8(a, a, a, a + 2, 16, 128, 128, 16, a, a, a, a, a, big, None) == 3
    assert lib.slope_dense_linear_bwd_dw_q8(a, a, 16, 128, 128, None, a, big, None) == 1
    assert lib.slope_dense_linear_bwd_dw_q8(a, a, 16, 100, 128, a, a, big, None) == 2
    assert lib.slope_dense_linear_bwd_dw_q8(a, a, 16, 128, 128, a + 4, a, big, None) == 3
    need = lib.slope_bwd_dw_q8_workspace_bytes(16, 128, 128, 16)
    assert need > 0 and lib.slope_linear_bwd_dw_adapter_q8(a, a, a, a, 16, 128, 128, 16, a, a, a, a, a, need - 1, None) == 1


def test_only_contiguous_cuda_tensors_are_taken(lib):
    import torch
    from paper_2608_24070_b200 import binding as B

    x, c = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4 * 66, dtype=torch.uint8)
    for call in (lambda: B.slope_checkpoint_store(x, c), lambda: B.slope_checkpoint_load(c, x), lambda: B.slope_layer_norm_fwd(x, None, None, 1e-5, x),
                 lambda: B.slope_layer_norm_bwd(x, x, x, x, None, x), lambda: B.slope_linear_bwd_dw_masked_q8(x, c, c, x),
                 lambda: B.slope_dense_linear_bwd_dw_q8(x, c, x)):
        with pytest.raises(AssertionError, match="contiguous CUDA tensors"):
            call()
    with pytest.raises(ValueError, match="multiple of 32"):
        B.alloc_checkpoint(4, 40, device="cpu")


def test_the_format_in_64_bits():
    """What the definition promises, on values that reach each of its borders."""
    rng = np.random.Generator(np.random.PCG64(5))
    x = rng.standard_normal((64, 96)).astype(np.float32).astype(np.float64) * 2.0 ** rng.integers(-140, 120, (64, 1))
    x[0, :32], x[0, 40], x[1, 3], x[2, :32] = 0.0, np.inf, np.nan, np.linspace(-127.5, 127.5, 32)
    codes, exponents = ref.encode(x)
    back = ref.decode(codes, exponents)
    assert np.isnan(back[0, 32:64]).all() and np.isnan(back[1, :32]).all() and np.isfinite(back[2:]).all() and not back[0, :32].any()
    assert exponents[0, 0] == 1 and exponents[0, 1] == 255 and exponents[2, 0] == 127 and codes[2, 0] == -127 and codes[2, 31] == 127
    unit = np.repeat(np.ldexp(1.0, exponents[2:].astype(int) - 127), 32, axis=1)
    assert (np.abs(back[2:] - x[2:]) <= unit / 2).all()
    # no smaller power of two would have held a block's largest magnitude
    largest = np.abs(x[2:].reshape(62, 3, 32)).max(-1)
    small = exponents[2:] > 1
    assert (largest[small] > 127.5 * np.ldexp(1.0, exponents[2:][small].astype(int) - 128)).all()
    assert np.array_equal(ref.encode(back[2:])[0], codes[2:])                      # values that are read back are stored as they are
    as_bf16 = (np.ascontiguousarray(back[2:], np.float32).view(np.uint32) & 0xFFFF) == 0
    assert as_bf16.all() and np.array_equal(back[2:].astype(np.float32).astype(np.float64), back[2:])
