"""The trunk_head command's optimizers: what their first step does to every tensor of every site, and that a run repeats itself."""
import pytest
import torch

pytestmark = pytest.mark.gpu

OPTIONS = [dict(optimizer="adamw"), dict(optimizer="adamw8"), dict(optimizer="adamw", clip=0.5), dict(optimizer="adamw8", clip=0.5)]


@pytest.fixture
def deterministic():
    was = torch.backends.cudnn.deterministic
    torch.backends.cudnn.deterministic = True
    yield
    torch.backends.cudnn.deterministic = was


@pytest.mark.parametrize("options", OPTIONS)
def test_the_first_step_of_every_site(monkeypatch, options):
    """From zero states the first step is -lr (decay p + g' / (|g'| + eps)), whatever the states' bits: they are rounded after it.
    The change is good to 16 u of its size and 3 u of the parameter's, and the clipping factor to 4 u."""
    from paper_1910_02120_b200 import api, trunk_head
    lr, eps, u, checked = 0.003, 1e-8, 2.0 ** -24, []
    step = api.AdamW.step

    def checking(opt, grads=None, **kw):
        before = [p.double() for p in opt.params]
        g = [t.double() for t in grads]
        norm = step(opt, grads, **kw)
        if opt.steps == 1:
            factor = 1.0
            if options.get("clip"):
                want = sum(float(t.square().sum()) for t in g) ** 0.5
                assert abs(float(norm) - want) <= 4 * u * want
                factor = min(1.0, options["clip"] / want)
            for p, q, t in zip(opt.params, before, g):
                decay = 0.01 if p.dim() > 1 else 0.0
                change = t * factor / ((t * factor).abs() + eps)
                tol = 3 * u * (q.abs() + p.double().abs()) + (16 + 8) * u * lr * change.abs() + 2.0 ** -149
                assert ((p.double() - (q * (1 - lr * decay) - lr * change)).abs() <= tol).all()
                checked.append(tuple(p.shape))
        return norm

    monkeypatch.setattr(api.AdamW, "step", checking)
    trunk_head.train(rounds=1, S=3, K=2, B=32, seed=2, norm=True, trunk_lr=lr, **options)
    # two convolution tensors, two of the linear layer, and the site's weight and bias of the norm
    assert len(checked) == 3 * 6 and checked.count((64,)) == 3 * 3


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("options", [dict(optimizer="sgd")] + OPTIONS)
def test_a_run_repeats_itself(deterministic, precision, options):
    """Same seeds, same bits, library convolutions aside, which are told to be deterministic."""
    from paper_1910_02120_b200 import trunk_head
    a, b = (trunk_head.train(rounds=2, S=2, K=3, B=32, precision=precision, seed=3, norm=True, trunk_lr=0.003, **options) for _ in range(2))
    assert a == b
