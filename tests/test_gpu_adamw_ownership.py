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


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_follows_tensors_whose_storage_changed(api, bits):
    """Parameters taken to the host and back, a copy and a state given other storage: the steps go on as if nothing had moved."""
    runs = []
    for moves in (False, True):
        gen = torch.Generator(device=DEV).manual_seed(2)
        layer = torch.nn.Linear(300, 77).to(DEV)
        with torch.no_grad():
            for p in layer.parameters():
                p.copy_(torch.randn(p.shape, generator=gen, device=DEV))
        params = list(layer.parameters())
        copies = [torch.zeros(p.shape, dtype=torch.bfloat16, device=DEV) for p in params]
        opt = api.AdamW(params, copies=copies, state_bits=bits, max_norm=1.0, seed=5)
        keep = []
        for t in range(4):
            if moves and t:
                keep += [p.data for p in params] + list(opt.state.values()) + [c.data for c in copies]    # no address comes back
                layer.cpu()
                layer.cuda()
                copies[t % 2].data = copies[t % 2].data.clone()
                opt.state["exp_avg"] = opt.state["exp_avg"].clone()
                stale = [k.clone() for k in keep]
            opt.step([torch.randn(p.shape, generator=gen, device=DEV) for p in params])
            if moves and t:
                now = {x.data_ptr() for x in opt._tensors()}
                assert all(torch.equal(a, b) for a, b in zip(keep, stale) if a.data_ptr() not in now)
        runs.append([p.data for p in params] + copies + list(opt.state_values()))
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_a_captured_step_finds_what_was_moved_before_the_capture(api):
    p = torch.nn.Parameter(torch.ones(5000, device=DEV))
    g = torch.ones(5000, device=DEV)
    opt = api.AdamW([p], lr=0.1, weight_decay=0.0)
    opt.step([g])
    first = p.data
    p.data = p.data.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([g])
    graph.replay()
    torch.cuda.synchronize()
    assert ((first - 0.9).abs() < 1e-5).all() and ((p.data - 0.8).abs() < 1e-5).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_a_gradient_may_be_its_own_parameter_and_gradients_may_be_one(api, bits, offset):
    gen = torch.Generator(device=DEV).manual_seed(4)
    start = torch.randn(3000001 + offset, generator=gen, device=DEV)[offset:]
    runs = []
    for own in (True, False):
        p, q, r = start.clone() if not offset else torch.cat([start[:1], start])[1:], torch.ones(500, device=DEV), torch.ones(500, device=DEV)
        shared = torch.full((500,), 0.5, device=DEV)
        opt = api.AdamW([p, q, r], state_bits=bits, max_norm=10.0, seed=1)
        for _ in range(3):
            opt.step([p if own else p.clone(), shared, shared if own else shared.clone()])
        runs.append([p, q, r, *opt.state.values()])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
