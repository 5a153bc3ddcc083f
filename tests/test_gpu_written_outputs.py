"""Tensors that a call without a context writes in place: a graph that saved the old values is told."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import api as a
    return a


def saved(t):
    """A loss whose backward pass needs t's present values."""
    w = torch.ones_like(t).requires_grad_()
    return (t * w).sum()


def test_layer_norms_outputs(api):
    x = torch.randn(6, 40, device=DEV)
    y, dx = torch.randn(6, 40, device=DEV), torch.randn(6, 40, device=DEV)
    loss = saved(y)
    out, mean, rstd = api.ist_layer_norm_forward(x, y=y)
    assert out is y
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    loss = saved(dx)
    api.ist_layer_norm_backward(y, x, None, mean, rstd, dx=dx)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    loss = saved(x)                                        # read, not written
    api.ist_layer_norm_backward(y, x, None, mean, rstd, dx=dx)
    loss.backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    before = y._version
    api.ist_layer_norm_forward(x, y=y, stream=side)
    side.synchronize()
    assert y._version == before + 1
    with torch.inference_mode():
        api.ist_layer_norm_forward(x, y=torch.empty(6, 40, device=DEV))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamws_states(api, bits):
    opt = api.AdamW([torch.ones(300, device=DEV)], state_bits=bits)
    loss = saved(opt.state["exp_avg"]) if bits == 32 else None
    versions = {k: v._version for k, v in opt.state.items()}
    opt.step([torch.ones(300, device=DEV)])
    assert all(opt.state[k]._version > v for k, v in versions.items())
    if bits == 32:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


def test_a_refused_call_writes_nothing(api):
    x, y = torch.randn(6, 40, device=DEV), torch.randn(6, 40, device=DEV)
    loss = saved(y)
    with pytest.raises(api.IstError):
        api.ist_layer_norm_forward(x, y=y, eps=-1.0)
    loss.backward()
