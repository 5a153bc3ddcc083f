"""Rows that several blocks share: a wait for another block's sums that cannot end gives up after its limit, its rows come out as
NaN, the status says so once, and stream and device stay usable.  The failure is that blocks withhold their sums."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LIMIT = 2_000_000                                          # about a millisecond


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import api as a
    a.ist_layer_norm_status()
    return a


def withheld(api, x, dy, stats, out, stream=None):
    stream = torch.cuda.current_stream() if stream is None else stream
    status = api.lib.ist_selftest_layer_norm_wait(x.data_ptr(), None if dy is None else dy.data_ptr(), None if stats is None else stats.data_ptr(),
                                                  *x.shape, out.data_ptr(), LIMIT, stream.cuda_stream)
    assert status == api.IST_OK, api.lib.ist_last_error(None)


# rows of whole aligned pieces and others; clusters of two and of four blocks (forward), of four and of eight (backward); one row, and
# more rows than clusters fit the GPU
@pytest.mark.parametrize("rows, cols", [(1, 20000), (1, 65536), (3, 20001), (300, 33000), (300, 32767), (7, 65535)])
@pytest.mark.parametrize("backward", [False, True])
def test_a_wait_that_cannot_end(api, rows, cols, backward):
    gen = torch.Generator(device=DEV).manual_seed(cols)
    x, dy = (torch.randn(rows, cols, generator=gen, device=DEV) for _ in range(2))
    y, mean, rstd = api.ist_layer_norm_forward(x)
    dx = api.ist_layer_norm_backward(dy, x, None, mean, rstd)[0]
    api.ist_layer_norm_status()                            # healthy so far
    out = torch.zeros(rows, cols, device=DEV)
    withheld(api, x, dy if backward else None, torch.cat([mean, rstd]) if backward else None, out)
    with pytest.raises(api.IstError, match="gave up") as e:
        api.ist_layer_norm_status()
    assert e.value.status == api.IST_ERR_DEVICE_TIMEOUT
    api.ist_layer_norm_status()                            # told once
    assert bool(out.isnan().all())
    y2, mean2, rstd2 = api.ist_layer_norm_forward(x)
    assert torch.equal(y2, y) and torch.equal(mean2, mean) and torch.equal(rstd2, rstd)
    assert torch.equal(api.ist_layer_norm_backward(dy, x, None, mean, rstd)[0], dx)
    api.ist_layer_norm_status()


def test_the_status_on_a_stream(api):
    side = torch.cuda.Stream()
    x, out = torch.randn(2, 20000, device=DEV), torch.zeros(2, 20000, device=DEV)
    torch.cuda.synchronize()
    withheld(api, x, None, None, out, side)
    with pytest.raises(api.IstError, match="gave up"):
        api.ist_layer_norm_status(side)
    api.ist_layer_norm_status()
