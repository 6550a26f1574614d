"""GPU: the harness's layers have first derivatives only, and say so when a second one is asked for."""
import pytest

from test_gpu_norm_block import H, model  # noqa: F401  (H: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["linear", "norm", "norm with residual"])
@pytest.mark.parametrize("checkpoint", [False, True])
def test_a_second_derivative_is_refused(H, kind, checkpoint):  # noqa: F811
    import torch

    gpu, norms, _, _ = model(H, 0, checkpoint)
    x = torch.randn(64, 512, device="cuda").bfloat16().requires_grad_(True)
    r = torch.randn(64, 512, device="cuda").bfloat16().requires_grad_(True)
    if kind == "linear":
        y = gpu["q"](x).float().pow(2)              # the gradient that comes back depends on x
    else:
        y = norms["attention"](x, r if "residual" in kind else None)[1].float()
        y = y * torch.randn_like(y)                 # (it does not: the layer norm's own derivative does)
    (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (g.float().pow(2).sum() + x.float().sum()).backward()


@pytest.mark.parametrize("kind", ["linear", "norm"])
def test_the_first_one_is_the_same_with_a_graph(H, kind):  # noqa: F811
    import torch

    gpu, norms, _, _ = model(H, 0, False)
    call = gpu["q"] if kind == "linear" else lambda x: norms["mlp"](x)[1]
    x = torch.randn(64, 512, device="cuda").bfloat16().requires_grad_(True)
    weights = torch.randn(64, 512, device="cuda")
    want = torch.autograd.grad((call(x) * weights).sum(), x)[0]
    got = torch.autograd.grad((call(x) * weights).sum(), x, create_graph=True)[0]
    assert torch.equal(want, got)


def test_a_stream_past_the_layer_norm_keeps_its_second_derivative(H):  # noqa: F811
    import torch

    norm = model(H, 0, False)[1]["mlp"]
    x = torch.randn(8, 512, device="cuda").requires_grad_(True)
    stream, _, _ = norm(x)
    (g,) = torch.autograd.grad((stream ** 3).sum(), x, create_graph=True)
    g.sum().backward()
    assert torch.equal(x.grad, 6 * x.detach())
