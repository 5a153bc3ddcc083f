"""trunk.layer_norm where there is nothing to do, or little."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("shape", [(0, 64), (3, 0, 1001), (0, 1)])
@pytest.mark.parametrize("weight", [False, True])
def test_gradients_of_an_empty_batch(shape, weight):
    from paper_1910_02120_b200 import trunk
    x = torch.randn(shape, device=DEV).requires_grad_()
    w = torch.ones(shape[-1], device=DEV).requires_grad_() if weight else None
    y = trunk.layer_norm(x, w)
    y.sum().backward()
    assert y.shape == shape and x.grad.shape == shape
    assert w is None or (w.grad.shape == w.shape and not w.grad.any())


@pytest.mark.parametrize("wanted", [(True, False, False), (False, True, False), (False, False, True), (False, True, True)])
def test_only_some_gradients(wanted):
    from paper_1910_02120_b200 import trunk
    gen = torch.Generator(device=DEV).manual_seed(1)
    args = [torch.randn(5, 40, generator=gen, device=DEV), torch.randn(40, generator=gen, device=DEV), torch.randn(40, generator=gen, device=DEV)]
    for t, want in zip(args, wanted):
        t.requires_grad_(want)
    trunk.layer_norm(*args).square().sum().backward()
    a64 = [t.detach().double().requires_grad_(want) for t, want in zip(args, wanted)]
    x, w, b = a64
    h = (x - x.mean(-1, keepdim=True)) / (x.var(-1, correction=0, keepdim=True) + 1e-5).sqrt()
    (h * w + b).square().sum().backward()
    for t, t64, want in zip(args, a64, wanted):
        assert (t.grad is not None) == want
        if want:                                            # 64 u of what is added up, in both passes and the square between them
            assert ((t.grad.double() - t64.grad).abs() <= 256 * 2.0 ** -24 * (t64.grad.abs() + t64.grad.abs().max())).all()
