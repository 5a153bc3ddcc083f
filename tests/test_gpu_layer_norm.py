"""Layer norm's two passes against a plain implementation in 64 bits.

Tolerances.  u = 2^-24.  A sum of n values in an order that groups them has an error of at most (number of additions that
a value goes through) * u * sum |.|; a row's sums go through at most 16 additions in a thread and 10 across threads and
blocks, and the rest of the arithmetic is a handful of roundings, so 64 u covers them.  Rounding to the output's type adds half a
step, eps / 2 relative.  Sums over rows go through at most `rows` additions."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import api as a
    return a


def make_rows(rows, cols, dtype, gen, pad=0, shift=0.3, scale=0.7, offset=0):
    """A view with `pad` elements between its rows, starting `offset` elements into its buffer; the rest is NaN."""
    buf = torch.full((rows * (cols + pad) + offset + 16,), float("nan"), device=DEV, dtype=dtype)
    view = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * scale + shift)
    return view, buf


def vectors(groups, cols, gen):
    return (1 + 0.3 * torch.randn(groups, cols, generator=gen, device=DEV), 0.2 * torch.randn(groups, cols, generator=gen, device=DEV))


def each_row(v, groups, rows):
    return v.double().repeat_interleave(rows // groups, 0) if rows else v.double()[:0]


def forward64(x, w, b, eps, groups):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = 1 / (var + eps).sqrt()
    h = (x - mean) * rstd
    w = 1.0 if w is None else each_row(w, groups, len(x))
    b = 0.0 if b is None else each_row(b, groups, len(x))
    return h, h * w + b, mean[:, 0], rstd[:, 0], w, b


def check_forward(api, x, w, b, groups=1, eps=1e-5, y_dtype=None, **kw):
    y, mean, rstd = api.ist_layer_norm_forward(x, w, b, eps, groups=groups, y_dtype=y_dtype, **kw)
    h, ye, me, re, wr, br = forward64(x, w, b, eps, groups)
    sd = 1 / re[:, None]
    # the mean's own rounding and that of the differences weigh with the row's spread
    tol = 64 * U * ((h.abs() + 1) * (wr.abs() if torch.is_tensor(wr) else 1.0) + (br.abs() if torch.is_tensor(br) else 0.0))
    tol = tol + torch.finfo(y.dtype).eps / 2 * (ye.abs() + tol)
    assert y.dtype == (y_dtype or x.dtype) and y.shape == x.shape
    assert ((y.double() - ye).abs() <= tol).all(), float(((y.double() - ye).abs() / tol).max())
    assert ((mean.double() - me).abs() <= 64 * U * (me.abs() + sd[:, 0])).all()
    assert ((rstd.double() - re).abs() <= 64 * U * re).all()
    first = y.clone()                     # the same call without statistics, into the same place: the same bits
    bare, none, nothing = api.ist_layer_norm_forward(x, w, b, eps, groups=groups, y_dtype=y_dtype, want_stats=False, **kw)
    assert none is None and nothing is None and torch.equal(bare, first)
    return y, mean, rstd


def check_backward(api, dy, x, w, mean, rstd, groups=1, dx_view=None, **kw):
    rows, cols = x.shape
    dx, dw, db = api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=groups, dx=dx_view, **kw)
    d, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    g = d * (1.0 if w is None else each_row(w, groups, rows))
    gh = (g * h).mean(1, keepdim=True)
    want = r * (g - g.mean(1, keepdim=True) - h * gh)
    size = r * (g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True))
    tol = 64 * U * size
    if dx is not None:
        tol = tol + torch.finfo(dx.dtype).eps / 2 * (want.abs() + tol)
        if dx.dtype == BF16:
            tol = tol + 2.0 ** -134                                   # smallest bf16 numbers' half step
        assert dx.dtype == x.dtype and dx.shape == x.shape
        assert ((dx.double() - want).abs() <= tol).all(), float(((dx.double() - want).abs() / tol).max())
    per = rows // groups if groups else 0
    for got, terms in ((dw, d * h), (db, d)):
        if got is not None:
            t = terms.view(groups, per, cols)
            bound = (per + 64) * U * t.abs().sum(1)
            assert got.shape == (groups, cols)
            assert ((got.double() - t.sum(1)).abs() <= bound).all()
            # and as a whole: errors of additions are independent, far below the bound of one
            off, norm = (got.double() - t.sum(1)).norm(), t.abs().sum(1).norm()
            assert off <= 64 * U * norm
    return dx, dw, db


WIDTHS = [1, 2, 3, 7, 8, 31, 32, 33, 64, 100, 128, 129, 200, 255, 256, 257, 500, 512, 513, 768, 1000, 1001, 1024, 1025, 1500, 2048,
          2049, 3001, 4096, 4100, 5000, 8192, 8200, 10007, 16384, 16392, 20000, 32768, 33000, 50001, 65536, 65537, 70003]


@pytest.mark.parametrize("x_dtype, y_dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("cols", WIDTHS)
def test_widths(api, cols, x_dtype, y_dtype):
    gen = torch.Generator(device=DEV).manual_seed(cols)
    for groups, per, pad in ((1, 1, 0), (3, 5, 0), (2, 37, 8), (1, 64, 3)):
        rows = groups * per
        x, _ = make_rows(rows, cols, x_dtype, gen, pad)
        w, b = vectors(groups, cols, gen)
        y, mean, rstd = check_forward(api, x, w, b, groups, y_dtype=y_dtype)
        dy, _ = make_rows(rows, cols, y_dtype, gen, pad, shift=0.0, scale=1e-2)
        check_backward(api, dy, x, w, mean, rstd, groups)


@pytest.mark.parametrize("rows, groups", [(0, 1), (0, 3), (1, 1), (2, 2), (7, 7), (300, 1), (300, 300), (1200, 6), (5000, 1), (4099, 1), (20000, 4)])
@pytest.mark.parametrize("cols", [1, 24, 64, 1001, 1024])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_and_groups(api, rows, groups, cols, dtype):
    gen = torch.Generator(device=DEV).manual_seed(rows + cols)
    x, _ = make_rows(rows, cols, dtype, gen)
    w, b = vectors(groups, cols, gen)
    y, mean, rstd = check_forward(api, x, w, b, groups)
    assert y.shape == (rows, cols) and mean.shape == rstd.shape == (rows,)
    dy, _ = make_rows(rows, cols, F32, gen, shift=0.01, scale=1e-2)
    dx, dw, db = check_backward(api, dy, x, w, mean, rstd, groups)
    if rows == 0:
        assert not dw.any() and not db.any()


@pytest.mark.parametrize("x_dtype, y_dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("cols", [3, 16, 24, 33, 64, 100, 128, 250, 256, 500, 512, 700, 1000, 1001, 1024, 1500, 2048, 4001, 4096, 8192, 9000, 16384, 30001])
def test_many_rows(api, cols, x_dtype, y_dtype):
    """Enough rows for every block to go round its ring of stages several times, sites that end inside a tile among them."""
    gen = torch.Generator(device=DEV).manual_seed(cols)
    groups = 3
    rows = groups * (2 ** 24 // cols // groups)
    x, _ = make_rows(rows, cols, x_dtype, gen)
    w, b = vectors(groups, cols, gen)
    y, mean, rstd = check_forward(api, x, w, b, groups, y_dtype=y_dtype)
    dy, _ = make_rows(rows, cols, y_dtype, gen, shift=0.0, scale=1e-2)
    check_backward(api, dy, x, w, mean, rstd, groups)


@pytest.mark.parametrize("offset, pad", [(0, 1), (1, 0), (1, 1), (2, 2), (4, 4), (4, 0), (3, 5), (8, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [40, 320, 1000, 2100])
def test_strides_and_offsets(api, cols, dtype, offset, pad):
    """Rows that start anywhere; inputs and outputs are aligned differently, and what lies between the rows stays."""
    gen = torch.Generator(device=DEV).manual_seed(cols + offset * 100 + pad)
    rows, groups = 36, 2
    x, _ = make_rows(rows, cols, dtype, gen, pad, offset=offset)
    w, b = vectors(groups, cols, gen)
    _, mean, rstd = check_forward(api, x, w, b, groups)
    for other in (0, offset, 5):
        out, buf = make_rows(rows, cols, dtype, gen, pad, offset=other)
        check_forward(api, x, w, b, groups, y=out)
        api.ist_layer_norm_forward(x, w, b, groups=groups, y=out)
        assert int(buf.isnan().sum()) == buf.numel() - rows * cols
        dy, _ = make_rows(rows, cols, F32, gen, pad, shift=0.0, offset=other)
        out, buf = make_rows(rows, cols, dtype, gen, pad, offset=other)
        check_backward(api, dy, x, w, mean, rstd, groups, dx_view=out)
        assert int(buf.isnan().sum()) == buf.numel() - rows * cols


def test_vectors_that_start_anywhere(api):
    gen = torch.Generator(device=DEV).manual_seed(5)
    x, _ = make_rows(64, 512, F32, gen)
    flat = torch.randn(2 * 512 + 3, generator=gen, device=DEV)
    w, b = flat[1:513].view(1, 512), flat[515:1027].view(1, 512)
    y, mean, rstd = check_forward(api, x, w, b)
    dy, _ = make_rows(64, 512, F32, gen)
    check_backward(api, dy, x, w, mean, rstd)


@pytest.mark.parametrize("weight, bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("cols", [64, 1001, 4096, 40000])
def test_without_weight_or_bias(api, cols, weight, bias):
    gen = torch.Generator(device=DEV).manual_seed(cols)
    x, _ = make_rows(50, cols, BF16, gen)
    w, b = vectors(2, cols, gen)
    w, b = w if weight else None, b if bias else None
    y, mean, rstd = check_forward(api, x, w, b, 2)
    dy, _ = make_rows(50, cols, F32, gen, shift=0.0)
    check_backward(api, dy, x, w, mean, rstd, 2)


@pytest.mark.parametrize("cols", [64, 1000, 1001, 8192, 40000])
def test_only_what_is_wanted(api, cols):
    gen = torch.Generator(device=DEV).manual_seed(cols)
    x, _ = make_rows(48, cols, F32, gen)
    dy, _ = make_rows(48, cols, F32, gen)
    w, b = vectors(3, cols, gen)
    _, mean, rstd = api.ist_layer_norm_forward(x, w, b, groups=3)
    full = api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=3)
    for wanted in ((True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, False, True)):
        got = check_backward(api, dy, x, w, mean, rstd, 3, want_dx=wanted[0], want_dweight=wanted[1], want_dbias=wanted[2])
        for g, f, is_wanted in zip(got, full, wanted):
            assert (g is None) != is_wanted and (g is None or torch.equal(g, f))
    with pytest.raises(api.IstError, match="no output"):
        api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=3, want_dx=False, want_dweight=False, want_dbias=False)


@pytest.mark.parametrize("cols", [5, 64, 1001, 4096, 40000])
def test_rows_far_from_zero_and_constant_rows(api, cols):
    """A constant row has no spread, whatever its value; a common offset of a thousand spreads is taken out."""
    gen = torch.Generator(device=DEV).manual_seed(cols)
    w, b = vectors(1, cols, gen)
    x = torch.tensor([0.0, 1.0, -3.3, 1e4, 12345.678, 1e-20], device=DEV)[:, None].expand(6, cols).contiguous()
    y, mean, rstd = api.ist_layer_norm_forward(x, w, b)
    # the first mean is off by 64 u at most, and what is left of it is taken out to within 64 u of itself
    step = x.double().abs()[:, :1] * 64 * U
    assert ((y.double() - b.double()).abs() <= w.double().abs() * step * 64 * U / 1e-5 ** 0.5 + 2 * U * b.double().abs()).all()
    assert ((mean.double() - x[:, 0].double()).abs() <= 2 * U * x[:, 0].double().abs()).all()
    x = torch.randn(20, cols, generator=gen, device=DEV) + 1000.0
    check_forward(api, x, w, b)


@pytest.mark.parametrize("cols", [33, 64, 1001, 4096, 40000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_row_that_is_not_finite_stays_alone(api, cols, bad):
    gen = torch.Generator(device=DEV).manual_seed(cols)
    x, _ = make_rows(40, cols, F32, gen)
    w, b = vectors(2, cols, gen)
    clean, mean, rstd = api.ist_layer_norm_forward(x, w, b, groups=2)
    dirty = x.clone()
    dirty[7, cols // 2] = bad
    y, m, r = api.ist_layer_norm_forward(dirty, w, b, groups=2)
    assert y[7].isnan().all() and not m[7].isfinite()
    keep = torch.arange(40, device=DEV) != 7
    assert torch.equal(y[keep], clean[keep]) and torch.equal(m[keep], mean[keep]) and torch.equal(r[keep], rstd[keep])
    dy, _ = make_rows(40, cols, F32, gen)
    dx, dw, db = api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=2)
    dy2 = dy.clone()
    dy2[7, cols // 2] = bad
    dx2, dw2, db2 = api.ist_layer_norm_backward(dy2, x, w, mean, rstd, groups=2)
    assert not dx2[7].isfinite().any() and torch.equal(dx2[keep], dx[keep])
    other = torch.arange(cols, device=DEV) != cols // 2
    for a, c in ((dw2, dw), (db2, db)):
        assert torch.equal(a[1], c[1]) and torch.equal(a[0, other], c[0, other]) and not a[0, cols // 2].isfinite()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_one_element(api, dtype):
    """Their own mean: y is the bias, and nothing depends on x."""
    gen = torch.Generator(device=DEV).manual_seed(9)
    x, _ = make_rows(1000, 1, dtype, gen)
    w, b = vectors(4, 1, gen)
    y, mean, rstd = api.ist_layer_norm_forward(x, w, b, groups=4, y_dtype=F32)
    assert torch.equal(y, b.repeat_interleave(250, 0)) and torch.equal(mean, x[:, 0].float())
    dy, _ = make_rows(1000, 1, F32, gen)
    dx, dw, db = check_backward(api, dy, x, w, mean, rstd, 4)
    assert not dx.any() and not dw.any()


def test_same_bits_every_time(api):
    gen = torch.Generator(device=DEV).manual_seed(1)
    for rows, cols, groups in ((4096, 1024, 1), (1200, 1001, 6), (300, 16384, 2), (64, 40000, 1)):
        x, _ = make_rows(rows, cols, F32, gen)
        dy, _ = make_rows(rows, cols, F32, gen)
        w, b = vectors(groups, cols, gen)
        _, mean, rstd = api.ist_layer_norm_forward(x, w, b, groups=groups)
        first = api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=groups)
        for _ in range(5):
            again = api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=groups)
            assert all(torch.equal(a, f) for a, f in zip(again, first))


def test_offsets_past_32_bits(api):
    gen = torch.Generator(device=DEV).manual_seed(2)
    rows, cols, stride = 3, 1000, 2 ** 31 + 8
    buf = torch.empty(2 * stride + 2 * cols, dtype=BF16, device=DEV)
    x = buf.as_strided((rows, cols), (stride, 1))
    x.copy_(torch.randn(rows, cols, generator=gen, device=DEV))
    w, b = vectors(1, cols, gen)
    y, mean, rstd = check_forward(api, x, w, b)
    out = buf[cols:].as_strided((rows, cols), (stride, 1))
    check_forward(api, x, w, b, y=out)
    check_backward(api, y.float(), x, w, mean, rstd)
    check_backward(api, y, x.contiguous(), w, mean, rstd, dx_view=out)
    del buf, x, out
    torch.cuda.empty_cache()


def test_leading_dimensions(api):
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(4, 6, 5, 96, generator=gen, device=DEV)
    w, b = vectors(1, 96, gen)
    y, mean, rstd = api.ist_layer_norm_forward(x, w, b)
    assert y.shape == x.shape and mean.shape == (120,)
    flat, _, _ = api.ist_layer_norm_forward(x.view(-1, 96), w, b)
    assert torch.equal(y.view(-1, 96), flat)
    one, m, r = api.ist_layer_norm_forward(x[0, 0, 0], w, b)
    assert torch.equal(one, y[0, 0, 0]) and m.shape == (1,)
    part = x[..., :64]                                    # a common stride of 96
    yp, _, _ = api.ist_layer_norm_forward(part)
    assert torch.equal(yp, api.ist_layer_norm_forward(part.contiguous())[0])
    with pytest.raises(api.IstError, match="no common stride"):
        api.ist_layer_norm_forward(x[:, :3])


def test_refusals(api):
    x = torch.randn(8, 32, device=DEV)
    ok = torch.ones(32, device=DEV)
    for bad in (dict(weight=ok[:31]), dict(weight=ok.double()), dict(bias=torch.ones(64, device=DEV)[::2]), dict(groups=0),
                dict(groups=3), dict(groups=2, weight=ok), dict(y=x), dict(y=torch.empty(7, 32, device=DEV)), dict(eps=0.0),
                dict(weight=ok.cpu()), dict(y=torch.empty(8, 32, device=DEV), y_dtype=BF16), dict(groups=2 ** 32 + 1)):
        with pytest.raises(api.IstError):
            api.ist_layer_norm_forward(x, **bad)
    for bad in (x.double(), x.half(), x.int()):
        with pytest.raises(TypeError):
            api.ist_layer_norm_forward(bad)
    for bad in (x.t(), x[:, ::2], x[:1].expand(8, 32), x[:, :0], torch.tensor(1.0, device=DEV)):
        with pytest.raises(api.IstError):
            api.ist_layer_norm_forward(bad)
    y, mean, rstd = api.ist_layer_norm_forward(x)
    for bad in (dict(dx=x), dict(dx=y), dict(dx=torch.empty(8, 32, device=DEV, dtype=BF16)), dict(groups=3)):
        with pytest.raises(api.IstError):
            api.ist_layer_norm_backward(y, x, None, mean, rstd, **bad)
    for args in ((y[:4], x, None, mean, rstd), (y, x, None, mean[:4], rstd), (y, x, ok[:8], mean, rstd)):
        with pytest.raises(api.IstError):
            api.ist_layer_norm_backward(*args)


def test_other_streams_and_graphs(api):
    """Calls on a stream of their own, and two captured graphs that replay at the same time."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    x, _ = make_rows(2000, 1001, F32, gen)
    dy, _ = make_rows(2000, 1001, F32, gen)
    w, b = vectors(4, 1001, gen)
    y, mean, rstd = api.ist_layer_norm_forward(x, w, b, groups=4)
    want = api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y2, m2, r2 = api.ist_layer_norm_forward(x, w, b, groups=4, stream=side)
    got = api.ist_layer_norm_backward(dy, x, w, m2, r2, groups=4, stream=side)
    side.synchronize()
    assert torch.equal(y2, y) and all(torch.equal(a, c) for a, c in zip(got, want))
    graphs = []
    for k in range(2):
        xs, ds = x.clone(), dy.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            yk, mk, rk = api.ist_layer_norm_forward(xs, w, b, groups=4)
            outs = api.ist_layer_norm_backward(ds, xs, w, mk, rk, groups=4)
        graphs.append((g, xs, ds, yk, outs))
    scaled = dy * 0.5
    graphs[1][2].copy_(scaled)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        for (g, *_rest), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(graphs[0][3], y) and all(torch.equal(a, c) for a, c in zip(graphs[0][4], want))
    half = api.ist_layer_norm_backward(scaled, x, w, mean, rstd, groups=4)
    assert all(torch.equal(a, c) for a, c in zip(graphs[1][4], half))


def test_gradients_by_differences(api):
    """Central differences of a loss, computed in 64 bits with the definition, against the library's gradients."""
    gen = torch.Generator(device=DEV).manual_seed(6)
    x, _ = make_rows(6, 10, F32, gen)
    w, b = vectors(2, 10, gen)
    dy, _ = make_rows(6, 10, F32, gen, shift=0.0)
    _, mean, rstd = api.ist_layer_norm_forward(x, w, b, groups=2)
    dx, dw, db = api.ist_layer_norm_backward(dy, x, w, mean, rstd, groups=2)
    loss = lambda x, w, b: float((forward64(x, w, b, 1e-5, 2)[1] * dy.double()).sum())
    step = 1e-5                                         # second-order error about 1e-10 of third derivatives of size 10
    for t, grad in ((x, dx), (w, dw), (b, db)):
        t64 = [v.double().clone() for v in (x, w, b)]
        i = [v is t for v in (x, w, b)].index(True)
        for at in range(0, t.numel(), 7):
            flat = t64[i].view(-1)
            keep = float(flat[at])
            flat[at] = keep + step
            up = loss(*t64)
            flat[at] = keep - step
            down = loss(*t64)
            flat[at] = keep
            assert abs((up - down) / (2 * step) - float(grad.reshape(-1)[at])) <= 1e-5 * (1 + float(grad.abs().max()))


def test_autograd(api):
    from paper_1910_02120_b200 import trunk
    gen = torch.Generator(device=DEV).manual_seed(7)
    x = torch.randn(3, 8, 40, generator=gen, device=DEV).requires_grad_()
    w, b = (v.squeeze(0).requires_grad_() for v in vectors(1, 40, gen))
    out = trunk.layer_norm(x, w, b)
    (out * out).sum().backward()
    x64, w64, b64 = (v.detach().double().requires_grad_() for v in (x, w, b))
    h = (x64 - x64.mean(-1, keepdim=True)) / (x64.var(-1, correction=0, keepdim=True) + 1e-5).sqrt()
    o64 = h * w64 + b64
    (o64 * o64).sum().backward()
    for a, c in ((x, x64), (w, w64), (b, b64)):
        assert a.grad.shape == a.shape
        assert ((a.grad.double() - c.grad).abs() <= 256 * U * (c.grad.abs() + c.grad.abs().max())).all()
    w.grad = None
    trunk.layer_norm(x.detach(), w, None).sum().backward()               # an expanded gradient, only the weight's wanted
    assert w.grad is not None and w.grad.shape == w.shape
    with torch.no_grad():
        assert not trunk.layer_norm(x, w, b).requires_grad
    g, = torch.autograd.grad(trunk.layer_norm(x, w, b).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_autograd_captured_while_an_eager_graph_lives(api):
    """torch cannot capture the backward pass of leaves that a live eager graph leads to: the call is refused, the process and
    the leaves stay usable, and the same values behind leaves of their own are captured and replayed."""
    from paper_1910_02120_b200 import trunk
    gen = torch.Generator(device=DEV).manual_seed(8)
    x = torch.randn(64, 96, generator=gen, device=DEV).requires_grad_()
    w, b = (v.requires_grad_() for v in vectors(1, 96, gen))
    eager = trunk.layer_norm(x, w, b).square().sum()
    with pytest.raises(api.IstError, match="eager graph"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            trunk.layer_norm(x, w, b)
    own = [t.detach().requires_grad_() for t in (x, w, b)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(trunk.layer_norm(*own).square().sum(), own)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = torch.autograd.grad(trunk.layer_norm(*own).square().sum(), own)
    with torch.no_grad():
        x.mul_(1.5).add_(0.25)
    graph.replay()
    torch.cuda.synchronize()
    kept = [g.clone() for g in grads]
    del eager
    want = torch.autograd.grad(trunk.layer_norm(x, w, b).square().sum(), (x, w, b))
    assert all(torch.equal(a, c) for a, c in zip(kept, want))


def test_rows_side_by_side_in_one_buffer(api):
    """Inputs and outputs that take turns in a wider buffer."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    buf = torch.randn(500, 3 * 104, generator=gen, device=DEV)
    x, y, dx = buf[:, :100], buf[:, 104:204], buf[:, 208:308]
    w, b = vectors(2, 100, gen)
    y2, mean, rstd = check_forward(api, x, w, b, 2, y=y)
    assert y2 is y
    check_backward(api, y, x, w, mean, rstd, 2, dx_view=dx)
    with pytest.raises(api.IstError, match="overlap"):
        api.ist_layer_norm_forward(x, w, b, groups=2, y=buf[:, 96:196])


def test_the_first_call_of_a_process_may_be_captured():
    """Nothing has to be set up by an uncaptured call."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_1910_02120_b200 import api
x = torch.randn(300, 1001, device="cuda")
w = torch.randn(1, 1001, device="cuda")
p = [torch.zeros(5000, device="cuda")]
g = [torch.ones(5000, device="cuda")]
opt = api.AdamW(p, state_bits=8, max_norm=1.0)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y, mean, rstd = api.ist_layer_norm_forward(x, w)
    dx, dw, db = api.ist_layer_norm_backward(y, x, w, mean, rstd)
    norm = opt.step(g)
graph.replay()
torch.cuda.synchronize()
y2, mean, rstd = api.ist_layer_norm_forward(x, w)
assert torch.equal(y, y2) and torch.equal(dx, api.ist_layer_norm_backward(y, x, w, mean, rstd)[0])
assert abs(float(norm) - 5000 ** 0.5) < 1e-3 and float(p[0].abs().min()) > 0
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_autograd_of_sites_into_bf16(api):
    """Every site's weight and bias get their own gradients; the way back starts from a bf16 gradient."""
    from paper_1910_02120_b200 import trunk
    gen = torch.Generator(device=DEV).manual_seed(11)
    x = torch.randn(3 * 50, 136, generator=gen, device=DEV).requires_grad_()
    w, b = (v.requires_grad_() for v in vectors(3, 136, gen))
    y = trunk.layer_norm(x, w, b, groups=3, y_dtype=BF16)
    dy = torch.randn(150, 136, generator=gen, device=DEV).to(BF16)
    assert y.dtype == BF16
    y.backward(dy)
    x64, w64, b64 = (v.detach().double().requires_grad_() for v in (x, w, b))
    h = ((x64 - x64.mean(-1, keepdim=True)) / (x64.var(-1, correction=0, keepdim=True) + 1e-5).sqrt()).view(3, 50, 136)
    (h * w64[:, None] + b64[:, None]).view(150, 136).backward(dy.double())
    for a, c in ((x, x64), (w, w64), (b, b64)):
        assert a.grad.shape == a.shape
        assert ((a.grad.double() - c.grad).abs() <= 256 * U * (c.grad.abs() + c.grad.abs().max())).all()
