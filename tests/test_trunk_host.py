"""trunk.layer_norm's host side with a stand-in for the library call."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad


@pytest.fixture
def api(monkeypatch):
    from paper_1910_02120_b200 import build
    build.build()
    from paper_1910_02120_b200 import api as a
    monkeypatch.setattr(a, "ist_layer_norm_forward", lambda x, *args, **kw: (torch.zeros(x.shape), None, None))
    return a


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("grad", [False, True])
def test_forward_mode_is_refused(api, which, grad):
    """A result without a tangent would read as a derivative of zero."""
    from paper_1910_02120_b200 import trunk
    args = [torch.randn(4, 8), torch.ones(8), torch.zeros(8)]
    args[which].requires_grad_(grad)
    with forward_ad.dual_level():
        trunk.layer_norm(*(t.detach() for t in args))             # no tangent: nothing is lost
        args[which] = forward_ad.make_dual(args[which], torch.ones_like(args[which]))
        with pytest.raises(api.IstError, match="forward") as e:
            trunk.layer_norm(*args)
        assert e.value.status == api.IST_ERR_UNSUPPORTED
        with torch.no_grad(), pytest.raises(api.IstError, match="forward"):      # forward mode goes on under it
            trunk.layer_norm(*args)
        with forward_ad._set_fwd_grad_enabled(False):
            trunk.layer_norm(*(t.detach() for t in args))
