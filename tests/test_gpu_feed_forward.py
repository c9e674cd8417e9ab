"""The feed-forward example: it runs, and its gradients against automatic differentiation in 64 bits."""
import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")


@pytest.fixture(scope="module")
def example():
    from paper_2205_00119_amd.examples import feed_forward
    return feed_forward


@pytest.mark.parametrize("rows,h", [(96, 64), (300, 200), (17, 96), (520, 256)])
def test_gradients(example, rows, h):
    """The 16-bit intermediates are rounded to 8 bits, each within 2^-8 of itself (half of that on average and of random sign), half
    a dozen of them in a row; the checkpoint is off by at most 1/254 of a block's largest, some 1 % of a typical z, which changes
    slopes by less: a gradient is within 3 % in the 2-norm."""
    inner, drop, seed, offset = 4 * h, 0.25, 11, 5
    layer = example.FeedForward(rows, h, inner, drop)
    params = example.initial(layer, 4)
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    views = layer.views(params)
    for name in ("b1", "b2", "norm_bias"):
        views[name].normal_(0.0, 0.2, generator=gen)
    x, dy = (torch.randn(rows, h, generator=gen, device="cuda:0").to(torch.bfloat16) for _ in range(2))
    grads = torch.full((layer.numel,), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    y = layer.forward(params, x, seed, offset).clone()
    dx = layer.backward(params, grads, x, dy, seed, offset)

    w = {n: t.double().cpu().requires_grad_() for n, t in views.items()}
    x64 = x.double().cpu().requires_grad_()
    keep = torch.from_numpy(ref.kept(rows, h, drop, seed, offset))
    scale = 65536.0 / (65536 - ref.threshold(drop))
    g = torch.nn.functional.gelu(x64 @ w["W1"].t() + w["b1"])
    s = x64 + torch.where(keep, (g @ w["W2"].t() + w["b2"]) * scale, torch.zeros(()).double())
    want = torch.nn.functional.layer_norm(s, (h,), w["weight"], w["norm_bias"], example.EPS)
    want.backward(dy.double().cpu())
    off = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())                  # noqa: E731
    assert off(y, want.detach()) < 0.01
    assert off(dx, x64.grad) < 0.03
    for name, got in layer.views(grads).items():
        assert off(got, w[name].grad) < 0.03, name


def test_it_runs(example):
    assert example.main(["--rows", "256", "--hidden", "512", "--steps", "2"]) > 0
