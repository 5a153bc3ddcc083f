"""Refusals of the operators without a context, checked without a device: every invalid argument is an error before
anything is enqueued, and the message says which."""
import ctypes
import math

import numpy as np
import pytest
import torch

P = 1 << 20            # an address that nothing here follows


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import build
    build.build()
    from paper_1910_02120_b200 import api as a
    return a


def _forward(api, x=P, x_type=0, x_stride=8, rows=4, cols=8, groups=2, weight=None, bias=None, eps=1e-5, y=2 * P, y_type=0,
             y_stride=8, mean=None, rstd=None):
    return api.lib.ist_layer_norm_forward(x, x_type, x_stride, rows, cols, groups, weight, bias, eps, y, y_type, y_stride, mean,
                                          rstd, None)


@pytest.mark.parametrize("bad, word", [
    (dict(x=None), "null"), (dict(y=None), "null"), (dict(x_type=2), "types"), (dict(y_type=-1), "types"),
    (dict(rows=-1), "rows"), (dict(rows=1 << 31, groups=1), "rows"), (dict(rows=(1 << 31) - 65535, groups=1), "rows"), (dict(cols=0), "cols"), (dict(cols=(1 << 30) + 1), "cols"),
    (dict(groups=0), "groups"), (dict(groups=3), "groups"), (dict(x_stride=7), "stride"), (dict(y_stride=0), "stride"),
    (dict(x_stride=(1 << 40) + 1), "stride"), (dict(rows=1 << 20, x_stride=1 << 40), "stride"), (dict(eps=0.0), "eps"),
    (dict(eps=math.inf), "eps"), (dict(eps=math.nan), "eps"), (dict(eps=-1.0), "eps"), (dict(x=P + 2), "aligned"),
    (dict(y=P + 1, y_type=1), "aligned"), (dict(weight=P + 2), "aligned"), (dict(y=P), "overlap"), (dict(y=P + 32), "overlap"),
    (dict(y=P - 48, y_type=1), "overlap"), (dict(bias=2 * P + 64), "overlap"), (dict(mean=2 * P + 124), "overlap"),
    (dict(mean=3 * P, rstd=3 * P + 12), "outputs overlap"), (dict(x_stride=16, y_stride=16, y=P + 28), "overlap"),
])
def test_forward_refuses(api, bad, word):
    assert _forward(api, **bad) == api.IST_ERR_ARG
    message = api.lib.ist_last_error(None).decode()
    assert message.startswith("ist_layer_norm_forward: ") and word in message, message


@pytest.mark.parametrize("good", [
    dict(x_stride=16, y_stride=16, y=P + 32),                       # rows side by side in one buffer
    dict(x_stride=16, y_stride=16, y=P - 32),
    dict(x_stride=32, y_stride=64, y=P + 32, y_type=1),
    dict(x_stride=32, y_stride=8, rows=1, groups=1, y=P + 32),
])
def test_rows_that_interleave_do_not_overlap(api, good):
    """Refused only for the last argument looked at (eps), so everything before it has passed; nothing is enqueued."""
    assert _forward(api, **good, eps=-1.0) == api.IST_ERR_ARG
    assert "eps" in api.lib.ist_last_error(None).decode()
    bad = {**good, "y": good["y"] + 4 * (1 if good["y"] < P else -1)}
    if good.get("rows") != 1:
        assert _forward(api, **bad) == api.IST_ERR_ARG and "overlap" in api.lib.ist_last_error(None).decode()


def test_no_rows_is_no_error(api):
    assert _forward(api, rows=0, x=None, y=None) == api.IST_OK
    assert api.lib.ist_adamw_step(None, 0, api.AdamWArgs(beta1=0.9, beta2=0.99, eps=1e-8, step=1, state_bits=32), None, 0, None) == api.IST_OK


def _backward(api, dy=P, dy_type=0, dy_stride=8, x=2 * P, x_type=0, x_stride=8, rows=4, cols=8, groups=2, weight=None, mean=3 * P,
              rstd=4 * P, dx=5 * P, dx_stride=8, dweight=6 * P, dbias=7 * P, ws=8 * P, ws_bytes=1 << 19):
    return api.lib.ist_layer_norm_backward(dy, dy_type, dy_stride, x, x_type, x_stride, rows, cols, groups, weight, mean, rstd, dx,
                                           dx_stride, dweight, dbias, ws, ws_bytes, None)


@pytest.mark.parametrize("bad, word", [
    (dict(dy=None), "null"), (dict(x=None), "null"), (dict(mean=None), "mean"), (dict(rstd=None), "rstd"), (dict(dy_type=3), "types"),
    (dict(dx=None, dweight=None, dbias=None), "no output"), (dict(groups=5), "groups"), (dict(dx_stride=4), "stride"),
    (dict(dx=P), "overlap"), (dict(dx=2 * P), "overlap"), (dict(dweight=7 * P), "overlap"), (dict(dbias=3 * P), "overlap"),
    (dict(dbias=7 * P + 2), "aligned"),
])
def test_backward_refuses(api, bad, word):
    assert _backward(api, **bad) == api.IST_ERR_ARG
    message = api.lib.ist_last_error(None).decode()
    assert message.startswith("ist_layer_norm_backward: ") and word in message, message


def test_backward_needs_its_workspace(api):
    big = dict(rows=4096, cols=1024, groups=2, dy=1 << 30, x=2 << 30, dx=3 << 30, dy_stride=1024, x_stride=1024, dx_stride=1024, ws=4 << 30)
    need = api.lib.ist_layer_norm_workspace_bytes(4096, 1024, 2)
    assert need > 0 and need % 8192 == 0
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=(4 << 30) + 8)):
        assert _backward(api, **{**big, "ws_bytes": need, **bad}) == api.IST_ERR_WORKSPACE
    assert _backward(api, **{**big, "ws_bytes": need, "dweight": 4 << 30}) == api.IST_ERR_ARG
    assert "overlap" in api.lib.ist_last_error(None).decode()
    for shape in ((-1, 8, 1), (4, 0, 1), (4, 8, 0), (4, 8, 3), (1 << 31, 8, 1), (0, 1 << 30, 1 << 20)):
        assert api.lib.ist_layer_norm_workspace_bytes(*shape) == 0
    assert api.lib.ist_layer_norm_workspace_bytes(4, 8, 2) == 0              # a few rows: one part, written where it belongs


def _table(api, count=1, **fields):
    t = np.zeros(count, api.ADAMW_TENSOR)
    for j in range(count):
        for k, name in enumerate(("param", "grad", "exp_avg", "exp_avg_sq", "exp_avg_base", "exp_avg_sq_base")):
            t[j][name] = (8 * j + k + 1) * P
    t["n"] = 100
    for k, v in fields.items():
        t[k] = v
    return t


def _args(api, **fields):
    return api.AdamWArgs(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=0.0, step=1, state_bits=8), **fields})


@pytest.mark.parametrize("bad, word", [
    (dict(state_bits=16), "state_bits"), (dict(grad_type=2), "types"), (dict(beta1=1.0), "beta"), (dict(beta2=-0.1), "beta"),
    (dict(beta1=math.nan), "beta"), (dict(eps=0.0), "eps"), (dict(eps=1e-60), "eps"), (dict(max_norm=-1.0), "max_norm"),
    (dict(max_norm=math.nan), "max_norm"), (dict(lr=math.inf), "lr"), (dict(step=0), "step"), (dict(step_dev=P + 4), "step_dev"),
    (dict(lr_dev=P + 2), "lr_dev"), (dict(norm_out_dev=P + 2), "norm_out_dev"),
])
def test_adamw_refuses_arguments(api, bad, word):
    t = _table(api)
    assert api.lib.ist_adamw_step(t.ctypes.data, 1, _args(api, **bad), P, 1 << 20, None) == api.IST_ERR_ARG
    message = api.lib.ist_last_error(None).decode()
    assert message.startswith("ist_adamw_step: ") and word in message, message


@pytest.mark.parametrize("bad, word", [
    (dict(param=0), "null"), (dict(exp_avg=0), "null"), (dict(exp_avg_sq=0), "null"), (dict(exp_avg_base=0), "base"),
    (dict(exp_avg_sq_base=0), "base"), (dict(n=-1), "n must"), (dict(n=(1 << 40) + 1), "n must"), (dict(param=P + 2), "aligned"),
    (dict(grad=P + 2), "aligned"), (dict(exp_avg_base=P + 1), "aligned"), (dict(param_bf16=P + 1), "aligned"),
    (dict(weight_decay=math.nan), "weight_decay"),
])
def test_adamw_refuses_tensors(api, bad, word):
    t = _table(api, 2)
    for k, v in bad.items():
        t[1][k] = v
    assert api.lib.ist_adamw_step(t.ctypes.data, 2, _args(api), P, 1 << 20, None) == api.IST_ERR_ARG
    message = api.lib.ist_last_error(None).decode()
    assert message.startswith("ist_adamw_step: tensor 1: ") and word in message, message


def test_adamw_refuses_calls(api):
    t = _table(api, 2, n=1 << 40)
    assert api.lib.ist_adamw_step(t.ctypes.data, 2, _args(api), None, 0, None) == api.IST_ERR_ARG       # 2^41 values
    assert api.lib.ist_adamw_step(None, 1, _args(api), None, 0, None) == api.IST_ERR_ARG
    assert api.lib.ist_adamw_step(t.ctypes.data, -1, _args(api), None, 0, None) == api.IST_ERR_ARG
    t = _table(api)
    need = api.lib.ist_adamw_workspace_bytes(1)
    for ws, size in ((None, need), (P, need - 1), (P + 8, need)):
        assert api.lib.ist_adamw_step(t.ctypes.data, 1, _args(api, max_norm=1.0), ws, size, None) == api.IST_ERR_WORKSPACE
    assert api.lib.ist_adamw_workspace_bytes(-1) == 0
    assert api.lib.ist_adamw_workspace_bytes(2000) > need


def test_state_values_refuses(api):
    f = api.lib.ist_adamw_state_values
    for args in ((None, P, None, None, 8, 0, P, None), (P, None, None, None, 8, 0, P, None), (None, None, P, None, 8, 0, None, P),
                 (P, P, None, None, -1, 0, P, None), (P, P, None, None, 8, 2, P, None), (P, P, None, None, 8, 0, P + 2, None),
                 (P, P + 1, None, None, 8, 0, P, None)):
        assert f(*args, None) == api.IST_ERR_ARG
    assert f(None, None, None, None, 0, 0, P, P, None) == api.IST_OK


def test_struct_layouts_match_the_header(api):
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "ist.h")).read(), flags=re.S)

    def names(struct):
        body = re.search(r"typedef struct %s \{(.*?)\}" % struct, header, re.S).group(1)
        return [n.strip(" *") for line in body.split(";") if line.strip() for n in re.sub(r"^\s*(const )?\w+", "", line.strip()).split(",")]

    assert names("ist_adamw_tensor") == list(api.ADAMW_TENSOR.names)
    assert names("ist_adamw_args") == [f[0] for f in api.AdamWArgs._fields_]
    assert api.ADAMW_TENSOR.itemsize == 72 and ctypes.sizeof(api.AdamWArgs) == 88


def test_tensors_of_the_cpu_are_refused(api):
    from paper_1910_02120_b200 import trunk
    x = torch.randn(4, 8)
    with pytest.raises(api.IstError, match="CUDA"):
        api.ist_layer_norm_forward(x)
    with pytest.raises(api.IstError, match="CUDA"):
        trunk.layer_norm(x.requires_grad_())
    with pytest.raises(api.IstError, match="CUDA"):
        api.ist_layer_norm_backward(x, x, None, x[:, 0], x[:, 0])
    with pytest.raises(api.IstError, match="CUDA"):
        api.AdamW([x])
    with pytest.raises(api.IstError, match="no parameters"):
        api.AdamW([])
