"""GPU: a call may be the first CUDA call of its host thread."""
import threading

import pytest

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


def calls(B, b):
    """Calls of every kind, with their outputs."""
    import torch

    d_out, d_in, r = 512, 768, 64
    gen = torch.Generator(device="cuda").manual_seed(b)
    new = lambda *s: torch.randn(s, device="cuda", generator=gen).bfloat16()
    W, X, dY, L, R = new(d_out, d_in), new(b, d_in), new(b, d_out), new(d_in, r), new(r, d_out)
    vals, meta, mask = B.alloc_compressed(d_out, d_in)
    valsT, metaT, _ = B.alloc_compressed(d_in, d_out)
    B.slope_prune_24_double(W, vals, meta, mask, valsT, metaT, None)
    Y, dX, dWc, dW, T, ckpt = torch.empty_like(dY), torch.empty_like(X), torch.empty_like(vals), torch.empty_like(W), new(b, r), B.alloc_checkpoint(b, d_in)
    out, part = [torch.empty_like(vals), torch.empty_like(meta), torch.empty_like(mask)], torch.empty(b, r, device="cuda").bfloat16()
    ws = torch.empty(max(16, B.slope_bwd_dw_q8_workspace_bytes(b, d_out, d_in, r)), dtype=torch.uint8, device="cuda")
    B.slope_checkpoint_store(X, ckpt)
    return {"prune": (lambda: B.slope_prune_24(W, *out), out),
            "forward": (lambda: B.slope_linear_fwd(X, vals, meta, d_out, Y), [Y]),
            "forward with adapters": (lambda: B.slope_linear_fwd_adapter(X, vals, meta, d_out, L, R, part, Y), [Y, part]),
            "input gradient": (lambda: B.slope_linear_bwd_dx(dY, valsT, metaT, d_in, dX), [dX]),
            "weight gradient": (lambda: B.slope_linear_bwd_dw_masked(dY, X, mask, dWc), [dWc]),
            "weight gradient from a checkpoint": (lambda: B.slope_linear_bwd_dw_masked_q8(dY, ckpt, mask, dWc, ws), [dWc]),
            "adapter product": (lambda: B.slope_adapter_fwd_bwd(2, None, dY, None, R, b, d_out, d_in, r, dT=T), [T]),
            "dense forward": (lambda: B.slope_dense_linear_fwd(X, W, Y), [Y]),
            "dense weight gradient": (lambda: B.slope_dense_linear_bwd_dw(dY, X, dW), [dW]),
            "layer norm": (lambda: B.slope_layer_norm_fwd(X, None, None, 1e-5, dX), [dX])}


@pytest.mark.parametrize("b", [4, 600])
def test_first_cuda_call_of_a_host_thread(B, b):
    import torch

    for name, (call, outputs) in calls(B, b).items():
        call()
        want = [t.clone() for t in outputs]
        for t in outputs:
            t.zero_()
        torch.cuda.synchronize()
        failed = []

        def thread():
            try:
                call()
            except Exception as e:  # noqa: BLE001
                failed.append(e)

        t = threading.Thread(target=thread)
        t.start()
        t.join()
        torch.cuda.synchronize()
        assert not failed, (name, failed)
        assert all(torch.equal(a, b) for a, b in zip(want, outputs)), name
    assert B.slope_poll_status() == 0
