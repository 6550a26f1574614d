"""8-bit checkpoints at the ends of their range: the largest numbers of fp32 and bf16, and blocks at the smallest unit, bit for bit and within the stated bounds."""
import numpy as np
import pytest

import norm_reference as ref
from test_gpu_norm import B  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def blocks():
    top, step = np.finfo(np.float32).max, 2.0 ** 121
    row = np.linspace(-1, 1, 32)
    return np.stack([np.full(32, top), np.full(32, -top), row * float(top), np.r_[top, row[1:]], np.r_[-top, row[1:] * 1e30],
                     np.full(32, 127.5 * step), np.full(32, np.nextafter(np.float32(127.5 * step), np.float32(np.inf))), np.full(32, 127.0 * step), row * 126.5 * step,
                     np.full(32, 63.75 * step), np.full(32, np.nextafter(np.float32(63.75 * step), np.float32(np.inf))),
                     row * 127.5 * 2.0 ** -126, row * 2.0 ** -126, np.full(32, 2.0 ** -127), np.full(32, 2.0 ** -149), row * 2.0 ** -140, np.zeros(32)])


@pytest.mark.parametrize("f32", [True, False])
def test_both_ends(B, f32):  # noqa: F811
    import torch

    x = torch.from_numpy(blocks().astype(np.float32))
    if not f32:
        x = x.bfloat16()
        x = torch.where(torch.isfinite(x), x, torch.full_like(x, torch.finfo(torch.bfloat16).max).copysign(x))
    x = x.repeat(9, 1).reshape(17, -1).contiguous()
    v = x.double().numpy()
    codes, exponents = ref.encode(v)
    ckpt, back = B.alloc_checkpoint(*x.shape), torch.empty(x.shape, device="cuda")
    B.slope_checkpoint_store(x.cuda(), ckpt)
    assert np.array_equal(ckpt.cpu().numpy(), ref.buffer(codes, exponents))
    B.slope_checkpoint_load(ckpt, back)
    got = back.double().cpu().numpy()
    assert np.isfinite(got).all()
    unit = np.repeat(np.ldexp(1.0, exponents.astype(np.int64) - 127), 32, axis=1)
    beyond = np.abs(v) > 127.5 * 2.0 ** 121
    assert beyond.any() == f32
    off = np.abs(got - v)
    assert (off <= np.where(beyond, 2.0 ** 121, unit / 2)).all() and (np.abs(got[beyond]) == 127 * 2.0 ** 121).all()
    largest = np.repeat(np.abs(v).reshape(17, -1, 32).max(-1), 32, axis=1)
    inner = (unit > 2.0 ** -126) & ~beyond
    assert (off[inner] <= largest[inner] / 127).all()
