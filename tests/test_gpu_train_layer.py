"""The training example: its gradients against automatic differentiation in 64 bits, and its loss over a few steps."""
import numpy as np
import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")


@pytest.fixture(scope="module")
def example():
    from paper_2205_00119_amd.examples import train_layer
    return train_layer


def test_gradients_of_a_step(example):
    """The 16-bit intermediates (u, gelu, the products, dlogits) are rounded to 8 bits, each within 2^-8 of itself (half of
    that on average and of random sign); a dozen of them in a row, so a gradient is within 3 % in the 2-norm."""
    rows, h, v, drop, seed, offset = 96, 64, 203, 0.25, 11, 5
    layer = example.Layer(rows, h, 4 * h, v, drop)
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    flat = torch.zeros(layer.numel, device="cuda:0")
    for name, view in layer.views(flat).items():
        view.normal_(1.0 if name == "weight" else 0.0, 0.1, generator=gen)
    params = flat.to(torch.bfloat16)
    grads = torch.full((layer.numel,), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    x = torch.randn(rows, h, generator=gen, device="cuda:0").to(torch.bfloat16)
    targets = torch.randint(0, v, (rows,), generator=gen, device="cuda:0")
    loss = layer.step(params, grads, x, targets, seed, offset)

    w = {n: t.double().cpu().requires_grad_() for n, t in layer.views(params).items()}
    x64 = x.double().cpu()
    keep = torch.from_numpy(ref.kept(rows, h, drop, seed, offset))
    scale = 65536.0 / (65536 - ref.threshold(drop))
    act = torch.nn.functional.gelu(x64 @ w["W1"] + w["b1"])
    s = x64 + torch.where(keep, (act @ w["W2"] + w["b2"]) * scale, torch.zeros(()).double())
    y = torch.nn.functional.layer_norm(s, (h,), w["weight"], w["norm_bias"], example.EPS)
    want = torch.nn.functional.cross_entropy(y @ w["E"], targets.cpu())
    want.backward()
    assert abs(float(loss) - float(want)) < 0.01 * float(want)
    for name, got in layer.views(grads).items():
        a, b = got.double().cpu(), w[name].grad
        assert float((a - b).norm() / b.norm()) < 0.03, name


def test_loss_falls(example):
    losses = example.main(["--steps", "12", "--rows", "256", "--hidden", "256", "--vocab", "300"])
    assert np.isfinite(losses).all()
    # it starts near log(vocab), what a uniform guess has, and the table is learnt from 2048 pairs a step
    assert abs(losses[0] - np.log(300)) < 1.0
    assert losses[-1] < 0.5 * losses[0]
