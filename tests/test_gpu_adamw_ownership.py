"""What api.AdamW owns and borrows: on which stream its states are made, and where its tensors lie when a step runs."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import api as a
    return a


@pytest.mark.parametrize("bits", [32, 8])
def test_states_are_made_on_the_stream_of_the_steps(api, bits):
    """Work that is queued on the stream of the construction holds nothing up, and no write of it comes after a step's."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    g = torch.randn(300001, generator=gen, device=DEV)
    want_p = torch.ones(300001, device=DEV)
    want = api.AdamW([want_p], state_bits=bits, max_norm=1.0, seed=3)
    want_norm, want_values = want.step([g]), want.state_values()        # a kernel's first call loads it, which waits for the device
    p, side = torch.ones(300001, device=DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(300_000_000)                        # a seventh of a second on the current stream
    opt = api.AdamW([p], state_bits=bits, max_norm=1.0, seed=3, stream=side)
    norm = opt.step([g])
    values = opt.state_values()
    side.synchronize()
    assert not torch.cuda.current_stream().query()        # it still sleeps
    torch.cuda.synchronize()
    assert torch.equal(p, want_p) and torch.equal(norm, want_norm)
    assert all(torch.equal(opt.state[k], want.state[k]) for k in want.state)
    assert all(torch.equal(a, b) for a, b in zip(values, want_values))
