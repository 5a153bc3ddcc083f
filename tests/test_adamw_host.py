"""api.AdamW's host side with a stand-in for the library call: the table that a step hands over has the addresses that its
tensors have then."""
import ctypes

import numpy as np
import pytest
import torch


@pytest.fixture
def api(monkeypatch):
    from paper_1910_02120_b200 import build
    build.build()
    from paper_1910_02120_b200 import api as a
    monkeypatch.setattr(a, "_cuda_device", lambda t, name: t.device)
    a.calls = []

    def call(index, function, table_at, count, args, workspace_at, workspace_bytes):
        rows = np.frombuffer(ctypes.string_at(table_at, count * a.ADAMW_TENSOR.itemsize), a.ADAMW_TENSOR).copy()
        a.calls.append((rows, args.step_dev, args.lr_dev))

    monkeypatch.setattr(a, "_call", call)
    yield a
    del a.calls


def check_table(api, opt, bits):
    rows, step_dev, lr_dev = api.calls[-1]
    assert [int(r) for r in rows["param"]] == [p.data_ptr() for p in opt.params]
    assert [int(r) for r in rows["param_bf16"]] == [c.data_ptr() for c in opt.copies]
    assert list(rows["n"]) == opt.sizes
    for name in opt.state:
        per = api.IST_ADAMW_BLOCK if name.endswith("base") else 1
        assert [int(r) for r in rows[name]] == [opt.state[name][o // per:].data_ptr() for o in opt.offsets], name
    assert step_dev == opt.step_dev.data_ptr() and lr_dev == opt.lr_dev.data_ptr()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_finds_tensors_whose_storage_changed(api, bits):
    params, copies = [torch.ones(300), torch.ones(20, 7)], [torch.ones(300).bfloat16(), torch.ones(20, 7).bfloat16()]
    opt = api.AdamW(params, copies=copies, state_bits=bits, step_dev=torch.zeros(1, dtype=torch.int64), lr_dev=torch.zeros(1))
    grads = [torch.ones(300), torch.ones(20, 7)]
    keep = []                                             # so that no address comes back
    for change in (lambda: None, lambda: setattr(params[1], "data", params[1].data.clone()),
                   lambda: setattr(copies[0], "data", copies[0].data.clone()),
                   lambda: params[0].set_(torch.zeros(300)), lambda: opt.params.__setitem__(0, torch.zeros(300)),
                   lambda: opt.state.__setitem__("exp_avg", opt.state["exp_avg"].clone()),
                   lambda: setattr(opt, "state", {k: v.clone() for k, v in reversed(opt.state.items())}),
                   lambda: setattr(opt, "step_dev", torch.zeros(1, dtype=torch.int64)), lambda: setattr(opt, "lr_dev", torch.ones(1))):
        keep += [t.data for t in opt._tensors()]
        change()
        opt.step(grads)
        check_table(api, opt, bits)
    assert opt.steps == 9 and len(api.calls) == 9


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_refuses_tensors_that_no_longer_fit(api, bits):
    buffers = []

    def at_the_same_address(o, name, list_of):
        """Storage of fewer values where the tensor's lay, as an allocator may give it."""
        t = list_of(o)[name]
        buffers.append(np.zeros(4096, np.uint8))
        t.data = torch.frombuffer(buffers[-1].data, dtype=t.dtype, count=t.numel())
        o._bind()
        t.data = torch.frombuffer(buffers[-1].data, dtype=t.dtype, count=t.numel() - 100)

    for change in (lambda o: at_the_same_address(o, 0, lambda o: o.params), lambda o: at_the_same_address(o, 1, lambda o: o.copies),
                   lambda o: at_the_same_address(o, "exp_avg_sq", lambda o: o.state),
                   lambda o: setattr(o.params[0], "data", o.params[0].data.double()),
                   lambda o: setattr(o.params[0], "data", torch.zeros(600)[::2]),
                   lambda o: setattr(o.copies[1], "data", o.params[1].data), lambda o: o.copies.pop(), lambda o: o.params.pop(),
                   lambda o: setattr(o.params[1], "data", o.params[0].data[100:]),                 # overlaps
                   lambda o: o.state.__setitem__("exp_avg", o.state["exp_avg"][:256]), lambda o: o.state.pop("exp_avg"),
                   lambda o: setattr(o, "lr_dev", torch.zeros(2))):
        params = [torch.ones(300), torch.ones(200)]
        opt = api.AdamW(params, copies=[p.bfloat16() for p in params], state_bits=bits, lr_dev=torch.zeros(1))
        change(opt)
        for _ in range(2):
            with pytest.raises(api.IstError):
                opt.step([torch.ones(300), torch.ones(200)])
        assert opt.steps == 0 and not api.calls


def test_a_refused_step_keeps_the_rate(api, monkeypatch):
    opt = api.AdamW([torch.ones(8)], lr=0.25)
    accepted = api._call

    def refuse(index, function, table_at, count, args, *rest):
        if args.lr != 0.125:
            raise api.IstError(api.IST_ERR_ARG, "lr must be finite")
        accepted(index, function, table_at, count, args, *rest)

    monkeypatch.setattr(api, "_call", refuse)
    with pytest.raises(api.IstError):
        opt.step([torch.ones(8)], lr=float("inf"))
    assert (opt.lr, opt.steps) == (0.25, 0)
    opt.step([torch.ones(8)], lr=0.125)
    assert (opt.lr, opt.steps) == (0.125, 1)


@pytest.mark.parametrize("eps, fine", [(2.0 ** -126, True), (2.0 ** 125, True), (2.0 ** 125 * (1 + 2.0 ** -23), False), (1e38, False),
                                       (2.0 ** -127, False), (float("inf"), False)])
def test_eps_has_a_reciprocal_in_fp32(api, eps, fine):
    """The divisor's reciprocal is taken, and is a normal number: one that is flushed to zero would stop the parameters.  A step
    without tensors enqueues nothing."""
    args = api.AdamWArgs(lr=1e-3, beta1=0.9, beta2=0.999, eps=eps, step=1, state_bits=32)
    assert api.lib.ist_adamw_step(None, 0, args, None, 0, None) == (api.IST_OK if fine else api.IST_ERR_ARG)
    assert fine or "eps" in api.lib.ist_last_error(None).decode()


def test_a_view_of_fewer_values_wants_gradients_of_the_old_size(api):
    params = [torch.ones(300), torch.ones(200)]
    opt = api.AdamW(params)
    params[0].data = params[0].data[:200]                     # the same memory, still all there
    with pytest.raises(api.IstError, match="sizes"):
        opt.step([torch.ones(200), torch.ones(200)])
    assert opt.steps == 0 and not api.calls


@pytest.mark.parametrize("bits", [32, 8])
def test_values_of_states_that_no_longer_fit_are_refused(api, bits):
    """The values are read by the sizes of one state: all have to fit."""
    for name in ["exp_avg", "exp_avg_sq"] + (["exp_avg_base", "exp_avg_sq_base"] if bits == 8 else []):
        opt = api.AdamW([torch.ones(300), torch.ones(200)], state_bits=bits)
        opt.state[name] = opt.state[name][:2]
        with pytest.raises(api.IstError, match=name):
            opt.state_values()
        assert not api.calls
