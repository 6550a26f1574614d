"""GPU: a kernel's attributes are set once per host thread and device, however many kernels the thread uses."""
from concurrent.futures import ThreadPoolExecutor

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


def calls(B):
    """A dense layer's forward pass, all 64 instances of the layer norm's and all 96 of its backward pass."""
    import torch

    new = lambda *s, t=torch.bfloat16: torch.ones(s, dtype=t, device="cuda")
    X, W, Y = new(256, 512), new(512, 512), new(256, 512)
    todo = [lambda: B.slope_dense_linear_fwd(X, W, Y)]
    types = torch.bfloat16, torch.float32
    stats = new(4, t=torch.float32), new(4, t=torch.float32)
    for d in (256, 224, 512, 480, 768, 736, 1024, 992):
        y, r, ckpt = new(4, d), new(4, d), B.alloc_checkpoint(4, d)
        B.slope_checkpoint_store(r, ckpt)
        for x in types:
            h = new(4, d, t=x)
            for residual in (None, r):
                for kept in (None, ckpt):
                    todo.append(lambda h=h, y=y, residual=residual, kept=kept: B.slope_layer_norm_fwd(h, None, None, 1e-5, y, residual=residual, Y_ckpt=kept))
            for dx in types:
                out, side = new(4, d, t=dx), new(4, d, t=dx)
                for dH in (None, side):
                    todo.append(lambda h=h, r=r, out=out, dH=dH: B.slope_layer_norm_bwd(r, h, *stats, None, out, dH=dH))
                    if x is torch.float32:
                        todo.append(lambda ckpt=ckpt, r=r, out=out, dH=dH: B.slope_layer_norm_bwd(r, ckpt, *stats, None, out, dH=dH))
    assert len(todo) == 1 + 64 + 96
    return todo


def test_attributes_are_set_once(B):
    import torch
    from torch.profiler import ProfilerActivity, profile

    todo, counts = calls(B), []

    def run():
        for call in todo:
            call()

    with ThreadPoolExecutor(max_workers=1) as pool:         # a host thread of its own, to which all kernels are new
        for _ in range(3):
            torch.cuda.synchronize()
            with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as prof:
                pool.submit(run).result()
                torch.cuda.synchronize()
            names = [e.name for e in prof.events()]
            counts.append((sum(n.startswith("cudaLaunch") for n in names), sum(n == "cudaFuncSetAttribute" for n in names)))
    print("launches seen, attributes set:", counts)
    if counts[0][1] == 0:
        pytest.skip("the profiler does not show cudaFuncSetAttribute here")
    assert counts[0][0] >= len(todo) and counts[1][1] == 0 and counts[2][1] == 0
