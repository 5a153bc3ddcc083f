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


@pytest.mark.parametrize("bad, word", [
    (dict(rows=0), "rows"), (dict(rows=65537), "rows"), (dict(cols=16384), "cols"), (dict(cols=65537), "cols"), (dict(x=None), "null"),
    (dict(out=None), "null"), (dict(dy=1 << 21), "statistics"), (dict(x=(1 << 20) + 2), "aligned"), (dict(limit=0), "limit_cycles"),
    (dict(limit=2_000_000_001), "limit_cycles"), (dict(limit=-5), "limit_cycles"),
])
def test_the_self_test_of_waits_refuses(api, bad, word):
    """Refused before anything is enqueued."""
    a = {**dict(x=1 << 20, dy=None, stats=None, rows=4, cols=20000, out=1 << 22, limit=1000), **bad}
    status = api.lib.ist_selftest_layer_norm_wait(a["x"], a["dy"], a["stats"], a["rows"], a["cols"], a["out"], a["limit"], None)
    assert status == api.IST_ERR_ARG
    assert word in api.lib.ist_last_error(None).decode()


@pytest.mark.parametrize("dx_stride", [0, 8])
def test_the_way_back_of_no_rows(api, dx_stride):
    """An empty dx has no address; nothing is enqueued."""
    back = api.lib.ist_layer_norm_backward
    assert back(None, 0, 8, None, 0, 8, 0, 8, 2, None, None, None, None, dx_stride, None, None, None, 0, None) == api.IST_OK
    assert back(1 << 20, 0, 8, 1 << 21, 0, 8, 4, 8, 2, None, 1 << 22, 1 << 23, None, dx_stride, None, None, None, 0, None) == api.IST_ERR_ARG
    assert "no output" in api.lib.ist_last_error(None).decode()
