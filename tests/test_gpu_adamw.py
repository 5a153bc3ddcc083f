"""The AdamW step over many tensors against its definition in 64 bits, states in 32 and in 8 bits.

Tolerances.  u = 2^-24.  A moment is a sum of two products, each with a rounded coefficient and a rounded (clipped)
gradient: at most 8 u of the terms' magnitudes.  A parameter's change goes through a square root, a division and a handful of
products: 16 u of its magnitude, and 3 u of the parameter's for the two sums it is in.  An 8-bit code follows from 23 bits of the moment
and 20 random ones; where the moment's 8 u decide between two codes, either is right."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
BLOCK = 128
MASK = 2 ** 64 - 1


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import api as a
    return a


# --- SplitMix64 in numpy, and the 8-bit format in 64 bits ------------------------------------------------

def splitmix(seed, i):
    with np.errstate(over="ignore"):
        z = np.uint64(seed & MASK) + np.asarray(i, np.uint64) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def test_splitmix_is_the_published_generator():
    lines = [ln for ln in open(__file__.replace("test_gpu_adamw.py", "golden/splitmix64_seed1234567.txt")) if ln.strip() and ln[0].isdigit()]
    want = [int(ln.split()[-1]) for ln in lines]
    assert want and [int(splitmix(1234567, i + 1)) for i in range(len(want))] == want


def noise(seed, step, j, n, first=0):
    """(20 random bits for m, for v) of elements first .. first + n - 1 of tensor j; first is even."""
    key = int(splitmix(int(splitmix(seed, step)), j + 1))
    w = splitmix(key, np.arange(first // 2, (first + n + 1) // 2, dtype=np.uint64) + np.uint64(1))
    half = np.stack([w & np.uint64(0xffffffff), w >> np.uint64(32)], 1).reshape(-1)[:n].astype(np.int64)
    return (half & 0xffff) * 16 + 8, (half >> 16) * 16 + 8


def value(code):
    """The number whose fp32 pattern is code << 20, in 64 bits."""
    code = np.asarray(code, np.int64)
    e, k = code // 8, code % 8
    return np.where(e > 0, np.ldexp(8.0 + k, e - 130), np.ldexp(k * 1.0, -129))


def decode(codes, bases, signed):
    codes = codes.astype(np.int64)
    top = 127 if signed else 255
    k = codes & top
    x = np.where(k == 0, 0.0, value(np.repeat(bases.astype(np.int64), BLOCK)[:len(codes)] + k))
    x = np.where(k == top, np.nan if signed else np.inf, x)
    return np.where(codes > 127, -x, x) if signed else x


def place(x, r):
    """Where x > 0 lies on the grid of codes 1/2^20 apart, noise added: its integer part is the code."""
    f, e = np.frexp(x)
    normal = (e + 125.0) * 8 + f * 16
    return np.where(e + 126 > 0, normal, np.ldexp(x, 129)) + r / 2.0 ** 20


# --- the step -----------------------------------------------------------------------------------------------

def check_step(api, sizes, bits=32, grad=F32, copy=False, max_norm=None, steps=2, seed=3, first_step=0, offset=0, decay=0.01,
               scale=1e-3, skip=(), lr=1e-2, betas=(0.9, 0.999), eps=1e-8, tweak=None, gen_seed=0, **kw):
    gen = torch.Generator(device=DEV).manual_seed(gen_seed + len(sizes))
    flat = lambda dtype: torch.full((sum(n + offset for n in sizes) + 8,), float("nan"), dtype=dtype, device=DEV)

    def views(buf):
        out, at = [], offset
        for n in sizes:
            out.append(buf[at:at + n])
            at += n + offset
        return out

    pb, cb = flat(F32), flat(BF16)
    params, copies = views(pb), views(cb) if copy else None
    for p in params:
        p.normal_(0, 0.1, generator=gen)
    decays = [decay * (i % 2) for i in range(len(sizes))]
    opt = api.AdamW(params, lr=lr, betas=betas, eps=eps, weight_decay=decays, state_bits=bits, max_norm=max_norm, copies=copies, seed=seed,
                    step=first_step, **kw)
    for t in range(first_step + 1, first_step + steps + 1):
        gb = flat(grad)
        grads = views(gb)
        for i, g in enumerate(grads):
            g.copy_(torch.randn(g.shape, generator=gen, device=DEV) * scale * (i + 1))
            if i in skip:
                grads[i] = None
        if tweak:
            tweak(grads, t)
        before = [p.double().cpu().numpy() for p in params]
        old = {k: v.cpu().numpy().copy() for k, v in opt.state.items()}
        norm = opt.step(grads)
        clip = 1.0
        if max_norm is not None:
            want = math.sqrt(sum(float(g.double().square().sum()) for g in grads if g is not None))
            assert abs(float(norm) - want) <= 4 * U * want or not math.isfinite(want) and not math.isfinite(float(norm))
            clip = max_norm / want if want > max_norm else 1.0
        new = {k: v.cpu().numpy() for k, v in opt.state.items()}
        values = [v.cpu().numpy() for v in opt.state_values()] if bits == 8 else None
        for j, (n, at) in enumerate(zip(sizes, opt.offsets)):
            got = params[j].double().cpu().numpy()
            part = {k: (old[k][at // BLOCK:(at + n + BLOCK - 1) // BLOCK], new[k][at // BLOCK:(at + n + BLOCK - 1) // BLOCK]) if k.endswith("base")
                    else (old[k][at:at + n], new[k][at:at + n]) for k in old}
            if grads[j] is None:
                assert (got == before[j]).all() and all((a == b).all() for a, b in part.values())
                continue
            g = grads[j].double().cpu().numpy() * clip
            if bits == 8:
                m0 = decode(part["exp_avg"][0], part["exp_avg_base"][0], True)
                v0 = decode(part["exp_avg_sq"][0], part["exp_avg_sq_base"][0], False)
            else:
                m0, v0 = (part[k][0].astype(np.float64) for k in ("exp_avg", "exp_avg_sq"))
            with np.errstate(invalid="ignore", over="ignore"):
                m, v = betas[0] * m0 + (1 - betas[0]) * g, betas[1] * v0 + (1 - betas[1]) * g * g
                m_size = np.abs(betas[0] * m0) + np.abs((1 - betas[0]) * g)
                # an fp32 sum or product may be infinite where 64 bits reach further
                v = np.where(v > 3.4028235e38, np.inf, v)
                change = lr * (m / (1 - betas[0] ** t)) / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
                change_size = lr * (m_size / (1 - betas[0] ** t)) / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
                want = before[j] - lr * decays[j] * before[j] - change
                tol = 3 * U * (np.abs(before[j]) + np.abs(want)) + 16 * U * change_size + 2.0 ** -149
            fine = np.isfinite(want)
            assert (np.isnan(got) == np.isnan(want)).all()
            assert (np.abs(got - want) <= tol)[fine].all(), (j, float((np.abs(got - want) / tol)[fine].max()))
            if copy:
                c = copies[j].cpu()
                assert torch.equal(c.view(torch.int16)[torch.tensor(fine)], params[j].cpu().bfloat16().view(torch.int16)[torch.tensor(fine)])
            if bits == 32:
                tiny = 2.0 ** -148                                     # products below the normal numbers
                with np.errstate(invalid="ignore"):
                    assert (np.abs(part["exp_avg"][1] - m) <= 8 * U * m_size + tiny)[np.isfinite(m)].all()
                    assert (np.abs(part["exp_avg_sq"][1] - v) <= 8 * U * v + tiny)[np.isfinite(v)].all()
                    assert (np.isfinite(part["exp_avg"][1]) == np.isfinite(m)).all() and (np.isfinite(part["exp_avg_sq"][1]) == np.isfinite(v)).all()
            else:
                rm, rv = noise(seed, t, j, n)
                rel = 8 * U * np.divide(m_size, np.abs(m), out=np.ones(n), where=(m != 0) & np.isfinite(m))
                check_codes(m, rel, part["exp_avg"][1], part["exp_avg_base"][1], rm, True, (j, "m"))
                check_codes(v, np.full(n, 8 * U), part["exp_avg_sq"][1], part["exp_avg_sq_base"][1], rv, False, (j, "v"))
                for held, k, signed in ((values[0], "exp_avg", True), (values[1], "exp_avg_sq", False)):
                    want_values = decode(part[k][1], part[k + "_base"][1], signed)
                    assert np.array_equal(held[at:at + n].astype(np.float64), want_values, equal_nan=True)
    # what lies between the tensors is left as it was
    for buf, vs in ((pb, params), (cb, copies)):
        if vs:
            assert int(buf.isnan().sum()) >= buf.numel() - sum(sizes)
    return opt, params


def check_codes(x, rel, codes, bases, r, signed, what):
    """codes and bases hold the moments x, each known to within `rel` of itself and the roundings of fp32's denormal numbers:
    three of them, half of 2^-149 each, in products and a sum below 2^-126, where nothing relative holds."""
    n, top = len(x), 126 if signed else 254
    a = np.abs(x)
    with np.errstate(invalid="ignore"):
        least, most = np.maximum(a - rel * a - 2.0 ** -148, 0.0), a + rel * a + 2.0 ** -148
    blocks = lambda v: np.pad(np.where(np.isfinite(a), v, 0.0), (0, -n % BLOCK)).reshape(-1, BLOCK).max(1)
    lo, hi = (np.maximum(np.where(q > 0, np.floor(place(np.maximum(q, 1e-300), 0.0)), 0.0) + 1 - top, 0) for q in (blocks(least), blocks(most)))
    assert ((bases >= lo) & (bases <= hi)).all(), what
    base = np.repeat(bases.astype(np.int64), BLOCK)[:n]
    k = codes.astype(np.int64) & (127 if signed else 255)
    low, high = (np.minimum(np.floor(place(np.maximum(q, 1e-300), r)), 2039) - base for q in (least, most))
    low = np.maximum(low, 0 if signed else least > 0)          # a divisor does not vanish, if it has not in fp32
    high = np.maximum(high, 0 if signed else 1)
    ok = np.where(a > 0, (k >= low) & (k <= high), k == 0)
    ok = np.where(np.isfinite(a), ok, k == top + 1)
    assert ok.all(), (what, int((~ok).sum()), np.flatnonzero(~ok)[:5])
    # nearly all codes are decided by the moment alone
    if n >= 1000 and a.max() > 1e-35:
        assert (low == high)[np.isfinite(a)].mean() > 0.99, what
    if signed:
        sure = np.isfinite(a) & (least > 0)
        assert ((codes > 127) == ((x < 0) & (k > 0)))[sure].all(), what


SIZES = [1, 2, 3, 4, 5, 127, 128, 129, 255, 1000, 2047, 2048, 2049, 4096, 5001, 100000]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_sizes_and_offsets(api, bits, grad, offset):
    check_step(api, SIZES, bits, grad, copy=True, offset=offset, max_norm=0.5 if offset % 2 else None)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [1, 100, 128, 2048, 70001])
def test_a_single_tensor(api, bits, n):
    check_step(api, [n], bits, steps=3, max_norm=1e-3)


@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("offset", [0, 3])
def test_large_tensors(api, grad, offset):
    """More blocks of 128 values than the GPU holds at a time, several to a warp."""
    check_step(api, [5000001, 300, 4000000, 129], 8, grad, copy=True, offset=offset, max_norm=1.0, steps=1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [16, 17, 50, 51, 400, 401, 1300])
def test_many_tensors(api, bits, count):
    check_step(api, [1 + (7 * i) % 300 for i in range(count)], bits, steps=2, max_norm=2.0, scale=1e-4)


@pytest.mark.parametrize("bits", [32, 8])
def test_empty_tensors_and_missing_gradients(api, bits):
    check_step(api, [0, 5, 0, 300, 128, 0], bits, skip=(1, 4), max_norm=1.0)
    p = [torch.ones(4, device=DEV), torch.empty(0, device=DEV)]
    opt = api.AdamW(p, state_bits=bits, max_norm=1.0)
    assert float(opt.step([None, None])) == 0.0 and (p[0] == 1).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kw", [dict(first_step=100000), dict(betas=(0.0, 0.0)), dict(betas=(0.95, 0.99), eps=1e-4), dict(lr=0.0), dict(decay=0.0),
                                dict(scale=1e-12), dict(scale=1e-20), dict(scale=1e4), dict(max_norm=1e-12), dict(max_norm=math.inf)])
def test_arguments(api, bits, kw):
    check_step(api, [3000, 129], bits, **kw)


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_gradients_keep_zero_states(api, bits):
    def zero(grads, t):
        for g in grads:
            g.zero_()
    opt, params = check_step(api, [500, 128], bits, tweak=zero, steps=3, max_norm=1.0)
    assert all(not v.any() for v in opt.state.values())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3e30])
def test_values_that_are_not_finite_stay_alone(api, bits, bad):
    """They reach their own parameter and states, and no other value of the block."""
    def poison(grads, t):
        if t == 1:
            grads[0][200] = bad
    opt, params = check_step(api, [600, 100], bits, tweak=poison, steps=3)
    keep = torch.arange(600, device=DEV) != 200
    assert params[0][keep].isfinite().all() and params[1].isfinite().all()
    m, v = opt.state_values()
    keep = torch.arange(m.numel(), device=DEV) != 200
    assert m[keep].isfinite().all() and v[keep].isfinite().all() and not (m[200].isfinite() and v[200].isfinite())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_norms_that_are_not_finite(api, bad):
    p = [torch.ones(300, device=DEV), torch.ones(10, device=DEV)]
    g = [torch.full((300,), 1e-3, device=DEV), torch.full((10,), 1e-3, device=DEV)]
    g[0][5] = bad
    opt = api.AdamW(p, max_norm=1.0, weight_decay=0.0)
    norm = float(opt.step(g))
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    assert p[0][5].isnan() and int(p[0].isnan().sum()) == 1 and not p[1].isnan().any()
    assert torch.equal(p[1], torch.ones(10, device=DEV)) == math.isinf(bad)      # a factor of 0, or of 1


@pytest.mark.parametrize("scale", [1e-25, 1e-19, 1e19, 1e30])
def test_norms_whose_squares_leave_fp32(api, scale):
    g = torch.randn(5000, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)) * scale
    opt = api.AdamW([torch.zeros(5000, device=DEV)], max_norm=1.0)
    norm = float(opt.step([g]))
    want = float(g.double().norm())
    assert abs(norm - want) <= 4 * U * want


def test_rounding_of_8_bit_states_keeps_the_mean(api):
    """A second moment that decays by a thousandth per step, far less than half a step of its code, still falls as it should."""
    n, steps = 128 * 512, 300
    p = [torch.zeros(n, device=DEV)]
    g = torch.ones(n, device=DEV)
    opt = api.AdamW(p, state_bits=8, lr=0.0, seed=11)
    ref = api.AdamW([torch.zeros(n, device=DEV)], state_bits=32, lr=0.0)
    for o in (opt, ref):
        o.step([g])
    zero = torch.zeros(n, device=DEV)
    zero[::BLOCK] = 1.0                       # one value of a block keeps the block's base where it is
    for _ in range(steps):
        for o in (opt, ref):
            o.step([zero])
    keep = torch.arange(n, device=DEV) % BLOCK != 0
    got, want = opt.state_values()[1][keep].double(), ref.state["exp_avg_sq"][keep].double()
    # each rounding is off by an eighth of the value at most and has mean zero given what came before: standard deviation of a
    # walk of `steps` of them at most sqrt(steps) / 16, of the mean over n values a sqrt(n)-th of it
    assert abs(float(got.mean() / want.mean()) - 1) <= 6 * steps ** 0.5 / 16 / len(got) ** 0.5 + 300 * 8 * U


def test_device_step_and_rate_in_a_graph(api):
    """A captured step replayed: step number and learning rate come from the device; equal to eager steps."""
    for bits in (32, 8):
        runs = []
        for mode in ("eager", "graph"):
            gen = torch.Generator(device=DEV).manual_seed(5)
            params = [torch.randn(1000, generator=gen, device=DEV), torch.randn(77, generator=gen, device=DEV)]
            grads = [torch.empty_like(p) for p in params]
            new = lambda: [g.copy_(torch.randn(g.shape, generator=gen, device=DEV)) for g in grads]
            if mode == "eager":
                opt = api.AdamW(params, lr=0.01, state_bits=bits, max_norm=3.0, seed=9)
                for lr in (0.01, 0.01, 0.005, 0.02):
                    new()
                    opt.step(grads, lr=lr)
            else:
                count, rate = torch.zeros(1, dtype=torch.int64, device=DEV), torch.full((1,), 0.01, device=DEV)
                opt = api.AdamW(params, state_bits=bits, max_norm=3.0, seed=9, step_dev=count, lr_dev=rate)
                new()
                opt.step(grads)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    opt.step(grads)
                for lr in (0.01, 0.005, 0.02):
                    new()
                    rate.fill_(lr)
                    graph.replay()
                assert int(count) == 4
            runs.append((params, opt))
        for a, b in zip(runs[0][0], runs[1][0]):
            # the bias corrections are worked out on either side: an fp32 rounding apart at most
            assert ((a.double() - b.double()).abs() <= 4 * 64 * U * (0.02 + a.abs())).all()
        a, b = (r[1].state["exp_avg"] for r in runs)
        assert torch.equal(a, b)


def test_a_stream_of_its_own(api):
    gen = torch.Generator(device=DEV).manual_seed(6)
    g = torch.randn(100001, generator=gen, device=DEV)
    out = []
    for stream in (None, torch.cuda.Stream()):
        p = torch.ones(100001, device=DEV)
        torch.cuda.synchronize()
        opt = api.AdamW([p], max_norm=1.0, state_bits=8, stream=stream)
        torch.cuda.synchronize()
        norm = opt.step([g])
        m, v = opt.state_values(BF16)
        torch.cuda.synchronize()
        out.append((p, norm, m, v))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_same_bits_every_time(api):
    runs = []
    for _ in range(3):
        gen = torch.Generator(device=DEV).manual_seed(7)
        params = [torch.randn(n, generator=gen, device=DEV) for n in (300000, 77, 5000)]
        opt = api.AdamW(params, state_bits=8, max_norm=1.0, seed=1)
        for _ in range(3):
            opt.step([torch.randn(p.shape, generator=gen, device=DEV) for p in params])
        runs.append(params + list(opt.state.values()))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


@pytest.mark.parametrize("bits", [8, 32])
def test_offsets_past_32_bits(api, bits):
    """Values behind the 2^32nd of a tensor; the rest has no gradient to speak of and zero states."""
    n = 2 ** 32 + 300
    gen = torch.Generator(device=DEV).manual_seed(8)
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, dtype=BF16, device=DEV)
    tail = 2 ** 32 - 256
    g[tail:] = torch.randn(n - tail, generator=gen, device=DEV)
    opt = api.AdamW([p], state_bits=bits, seed=21, weight_decay=0.0, max_norm=1e9)
    norm = float(opt.step([g]))
    part = g[tail:].double()
    assert abs(norm - float(part.norm())) <= 4 * U * norm
    want = -1e-3 * part / (part.abs() + 1e-8)
    assert ((p[tail:].double() - want).abs() <= 16 * U * 1e-3).all()
    assert int((p[:tail] != 0).sum()) == 0
    if bits == 8:
        m, v = (opt.state[k][tail:n].cpu().numpy() for k in ("exp_avg", "exp_avg_sq"))
        mb, vb = (opt.state[k][tail // BLOCK:].cpu().numpy() for k in ("exp_avg_base", "exp_avg_sq_base"))
        rm, rv = noise(21, 1, 0, n - tail, tail)
        x = part.cpu().numpy()
        check_codes(0.1 * x, np.full(len(x), 8 * U), m, mb, rm, True, "m")
        check_codes(0.001 * x * x, np.full(len(x), 8 * U), v, vb, rv, False, "v")
    else:
        assert ((opt.state["exp_avg"][tail:n].double() - 0.1 * part).abs() <= 8 * U * part.abs()).all()
    del p, g, opt
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_code_has_its_value(api, dtype):
    """All codes under many bases, those of denormal values and of the largest among them."""
    bases = np.array([0, 1, 5, 100, 500, 1016, 1500, 1785, 1913], np.int16)
    codes = np.tile(np.arange(256, dtype=np.uint8), len(bases))
    per = np.repeat(bases, 2)
    opt = api.AdamW([torch.zeros(len(codes), device=DEV)], state_bits=8)
    opt.state["exp_avg"].copy_(torch.tensor(codes))
    opt.state["exp_avg_sq"].copy_(torch.tensor(codes))
    opt.state["exp_avg_base"].copy_(torch.tensor(per))
    opt.state["exp_avg_sq_base"].copy_(torch.tensor(per))
    m, v = (t.double().cpu().numpy() for t in opt.state_values(dtype))
    for got, signed in ((m, True), (v, False)):
        want = decode(codes, per, signed)
        with np.errstate(invalid="ignore"):
            sure = np.abs(want) <= 3.4e38
        assert np.array_equal(got[sure], want[sure]) and not np.isfinite(got[~sure]).any()


def test_refusals(api):
    p = torch.zeros(64, device=DEV)
    for bad in (dict(params=[p, p]), dict(params=[p[:40], p[30:]]), dict(params=[p.bfloat16()]), dict(params=[torch.zeros(8, 8, device=DEV).t()[:, :4]]),
                dict(params=[p], copies=[]), dict(params=[p], copies=[p]), dict(params=[p], weight_decay=[0.1, 0.1]), dict(params=[p], state_bits=4),
                dict(params=[p], state={}), dict(params=[p], state={"exp_avg": p, "exp_avg_sq": p}), dict(params=[p, torch.zeros(3)]),
                dict(params=[p], step_dev=torch.zeros(1, device=DEV)), dict(params=[p], lr_dev=torch.zeros(1))):
        with pytest.raises(api.IstError):
            api.AdamW(**bad)
    opt = api.AdamW([p, torch.zeros(3, device=DEV)])
    g = torch.ones(64, device=DEV)
    for bad in ([g], [g, g], [g, torch.ones(3)], [g, torch.ones(3, device=DEV).bfloat16()], [g, torch.ones(6, device=DEV)[::2]]):
        with pytest.raises(api.IstError):
            opt.step(bad)
    with pytest.raises(TypeError):
        opt.step([g.half(), None])
    with pytest.raises(api.IstError, match="eps"):
        api.AdamW([p], eps=0.0).step([g])
    with pytest.raises(TypeError):
        opt.state_values(torch.float16)
    assert not p.any() and opt.steps == 0


def test_a_step_tells_graphs_that_need_the_old_values(api):
    p = torch.ones(8, device=DEV, requires_grad=True)
    loss = (p * p).sum()
    api.AdamW([p]).step([torch.ones(8, device=DEV)])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_a_refused_step_is_no_step(api):
    count = torch.zeros(1, dtype=torch.int64, device=DEV)
    opt = api.AdamW([torch.ones(8, device=DEV)], eps=0.0, step_dev=count)
    with pytest.raises(api.IstError, match="eps"):
        opt.step([torch.ones(8, device=DEV)])
    assert int(count) == 0 and opt.steps == 0


def test_parameters_made_in_inference_mode(api):
    with torch.inference_mode():
        p = torch.ones(8, device=DEV)
        api.AdamW([p], weight_decay=0.0).step([torch.ones(8, device=DEV)])
    assert ((p - 0.999).abs() < 1e-6).all()
