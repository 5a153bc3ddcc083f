"""Operators that train a trunk in front of the partitioned layers, as measurable cases: layer norm's forward and
backward pass, and the AdamW step over many tensors with states in 32 or in 8 bits.

A case is a dict of plain values; "op" says which operator, and the rest its arguments:
  norm_forward, norm_backward
    rows, cols   size of the input        groups   sites: rows / groups rows each, every site its own weight and bias
    x, y, dy     element types            pad      elements between the rows of inputs and outputs
    stats        whether the forward pass also returns mean and reciprocal deviation (training) or not (serving)
  adamw
    net          "1024-4096-35": weights and biases of a fully connected network, or "72,8,64": tensor sizes
    sites        copies of the net, each with its own parameters
    bits         of a state: 32 or 8      grad     element type of the gradients
    copy         whether a bf16 operand copy of the parameters is kept
    packed       tensors lie one behind the other in one buffer, so that they start anywhere
    max_norm     bound of the global gradient norm, 0: none

`own` chooses between the framework's operators and their plain form in elementary torch operations.

States in 8 bits: a block of 128 values of a tensor shares an int16 `base`; a code c > 0 of seven bits (first moment,
which has a sign bit beside it) or eight (second moment) is the fp32 number with the bit pattern (base + c) << 20, code
0 is zero and the largest code stands for a value that is not finite.  Values are rounded to a neighbour at random,
with probabilities that keep the mean; the noise is SplitMix64's.
"""
import math

import torch

own = False

BLOCK = 128                       # values of an 8-bit state that share a base
EPS = 1e-5                        # of layer norm
BETA1, BETA2, ADAM_EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01
GOLDEN, MIX1, MIX2, MASK = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB, 2 ** 64 - 1
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _norm(name, op, rows, cols, groups=1, x="f32", y="f32", dy="f32", pad=0, stats=True):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "groups": groups, "x": x, "y": y, "dy": dy, "pad": pad,
            "stats": stats}


def _adamw(name, net, sites=1, bits=32, grad="f32", copy=False, packed=False, max_norm=0.0):
    return {"name": name, "op": "adamw", "net": net, "sites": sites, "bits": bits, "grad": grad, "copy": copy,
            "packed": packed, "max_norm": max_norm}


def listed():
    return [
        # features of four sites' trunks on their way into the head, one local step: latency counts
        _norm("norm-features", "norm_forward", 256, 64, groups=4),
        # rows of a speech network's round, 50 local steps of four sites
        _norm("norm-speech", "norm_forward", 51200, 1024, groups=4, x="bf16", y="bf16"),
        # nothing divides anything; fp32 features become the operands of a bf16 head
        _norm("norm-ragged", "norm_forward", 9600, 1001, groups=6, x="f32", y="bf16"),
        # rows as wide as the widest pixel network's hidden layer, scoring
        _norm("norm-wide", "norm_forward", 4096, 16384, groups=8, x="f32", y="bf16", stats=False),
        # the way back of the same four: the head's input gradient is fp32
        _norm("norm-features-grad", "norm_backward", 256, 64, groups=4),
        _norm("norm-speech-grad", "norm_backward", 51200, 1024, groups=4, x="bf16"),
        _norm("norm-ragged-grad", "norm_backward", 9600, 1001, groups=6, x="f32", dy="bf16"),
        _norm("norm-wide-grad", "norm_backward", 4096, 16384, groups=8, x="bf16", dy="bf16"),
        # a small convolutional trunk with a norm behind it, four sites, one local step
        _adamw("adamw-trunk", "72,8,12800,64,64,64", sites=4, max_norm=1.0),
        # the wide pixel network's middle: bf16 gradients, operands kept beside the masters
        _adamw("adamw-wide", "1024-16384-16384-10", grad="bf16", copy=True),
        # odd sizes one behind the other in one buffer, states in 8 bits
        _adamw("adamw8-ragged", "1001-5000-3001-77", bits=8, grad="bf16", packed=True),
        # a medium network, states in 8 bits, clipped gradients
        _adamw("adamw8-medium", "1024-8192-8192-100", bits=8, copy=True, max_norm=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(_moved(c) for c in listed() if _kind(c) == k) for k in ("norm_forward", "norm_backward", 32, 8)}
    while True:
        op = rng.choice(["norm_forward", "norm_backward", "adamw", "adamw"])
        if op == "adamw":
            if rng.random() < 0.5:
                multiple = rng.choice([1, 8, 64])
                dims = [max(4, _log(rng, 16, 8192) // multiple * multiple) for _ in range(rng.choice([2, 3, 4]))]
                net = "-".join(str(d) for d in dims + [_log(rng, 2, 200)])
            else:
                net = ",".join(str(_log(rng, 1, 2000000)) for _ in range(_log(rng, 1, 60)))
            c = _adamw("", net, _log(rng, 1, 8), rng.choice([32, 8]), rng.choice(["f32", "bf16"]), rng.random() < 0.4,
                       rng.random() < 0.4, rng.choice([0.0, 1.0]))
        else:
            groups = rng.choice([1, 1, 2, 4, 6, 8])
            multiple = rng.choice([1, 8, 64])
            cols = max(1, _log(rng, 1, 20000) // multiple * multiple)
            c = _norm("", op, groups * _log(rng, 1, 32768), cols, groups, rng.choice(["f32", "bf16"]),
                      rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]), rng.choice([0, 0, 8, 3]),
                      op == "norm_backward" or rng.random() < 0.6)
        if _moved(c) <= most[_kind(c)]:
            del c["name"]
            return c


def _kind(c):
    return c["bits"] if c["op"] == "adamw" else c["op"]


def _sizes(c):
    """Elements of each parameter tensor and its weight decay: none for vectors."""
    if "-" in c["net"]:
        dims = [int(d) for d in c["net"].split("-")]
        one = [n for i, o in zip(dims, dims[1:]) for n in (i * o, o)]
        decay = [d for _ in dims[1:] for d in (DECAY, 0.0)]
    else:
        one = [int(n) for n in c["net"].split(",")]
        decay = [DECAY if n > 64 else 0.0 for n in one]
    return one * c["sites"], decay * c["sites"]


def _moved(c):
    """Bytes that a pass reads and writes once."""
    if c["op"] == "adamw":
        n = sum(_sizes(c)[0])
        state = 16 if c["bits"] == 32 else 4 + 4 + 8 / BLOCK           # 8 bits: also the values it returns, in bf16
        return n * (8 + SIZE[c["grad"]] + state + 2 * c["copy"]) + 4 * (c["max_norm"] > 0)
    n, vectors = c["rows"] * c["cols"], 4 * c["groups"] * c["cols"]
    if c["op"] == "norm_forward":
        return n * (SIZE[c["x"]] + SIZE[c["y"]]) + 2 * vectors + 8 * c["rows"] * c["stats"]
    return n * (2 * SIZE[c["x"]] + SIZE[c["dy"]]) + 3 * vectors + 8 * c["rows"]


def work(case):
    if case["op"] == "adamw":
        return {"bytes": _moved(case), "flops": sum(_sizes(case)[0]) * (14 + 2 * (case["max_norm"] > 0))}
    return {"bytes": _moved(case), "flops": case["rows"] * case["cols"] * (8 if case["op"] == "norm_forward" else 14)}


# --- inputs ------------------------------------------------------------------------------------------

def _rows(case, kind, gen, scale, shift):
    """Rows as a user has them: a view of a wider buffer where they are padded."""
    cols = case["cols"]
    t = torch.randn(case["rows"], cols + case["pad"], generator=gen, device="cuda")
    t.mul_(scale).add_(shift)
    return t.to(TYPES[kind])[:, :cols]


def _offsets(sizes, packed):
    at, offsets = 0, []
    for n in sizes:
        offsets.append(at)
        at += n if packed else -(-n // 64) * 64
    return offsets, at


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] != "adamw":
        g, cols = case["groups"], case["cols"]
        s["weight"] = 1 + 0.2 * torch.randn(g, cols, generator=gen, device="cuda")
        s["bias"] = 0.1 * torch.randn(g, cols, generator=gen, device="cuda")
        s["x"] = _rows(case, case["x"], gen, 0.7, 0.3)
        if case["op"] == "norm_backward":                       # what the forward pass kept
            s["dy"] = _rows(case, case["dy"], gen, 1e-3, 0.0)
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = (x - s["mean"][:, None]).square_().mean(1).add_(EPS).rsqrt_()
        return s
    sizes, decay = _sizes(case)
    offsets, total = _offsets(sizes, case["packed"])
    scale = torch.rand(len(sizes), generator=gen, device="cuda").mul_(6).sub_(10).exp2_().tolist()    # each tensor's gradients
    views = lambda flat: [flat[o:o + n] for o, n in zip(offsets, sizes)]
    s["sizes"], s["decay"] = sizes, decay
    s["p"], s["g"] = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda", dtype=TYPES[case["grad"]])
    s["copy"] = torch.zeros(total, device="cuda", dtype=torch.bfloat16) if case["copy"] else None
    s["ps"], s["gs"] = views(s["p"]), views(s["g"])
    s["copies"] = views(s["copy"]) if case["copy"] else None
    # states: tensor after tensor, each on a multiple of 128 values
    s["room"] = [-(-n // BLOCK) * BLOCK for n in sizes]
    m, v = torch.zeros(sum(s["room"]), device="cuda"), torch.zeros(sum(s["room"]), device="cuda")
    at = 0
    for p, g, n, room, a in zip(s["ps"], s["gs"], sizes, s["room"], scale):
        p.normal_(0, 0.05, generator=gen)
        g.copy_(torch.randn(n, generator=gen, device="cuda").mul_(a))
        torch.randn(n, generator=gen, device="cuda", out=m[at:at + n]).mul_(0.3 * a)
        torch.randn(n, generator=gen, device="cuda", out=v[at:at + n]).square_().mul_(0.5).add_(0.5).mul_(a * a)
        at += room
    s["seed"], s["step"] = seed, 100
    s["state"] = {"exp_avg": m, "exp_avg_sq": v}
    if case["bits"] == 8:
        half = torch.full((1,), 0x80000, dtype=torch.int32, device="cuda")
        mc, mb = _encode(m, half, True)
        vc, vb = _encode(v, half, False)
        s["state"] = {"exp_avg": mc, "exp_avg_sq": vc, "exp_avg_base": mb, "exp_avg_sq_base": vb}
    if own:
        from paper_1910_02120_b200 import api
        s["opt"] = api.AdamW(s["ps"], lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=decay,
                             state_bits=case["bits"], max_norm=case["max_norm"] or None, copies=s["copies"],
                             state=s["state"], seed=seed, step=s["step"])
    return s


# --- one pass ------------------------------------------------------------------------------------------

def run(s):
    if s["op"] == "norm_forward":
        return _own_forward(s) if own else _plain_forward(s)
    if s["op"] == "norm_backward":
        return _own_backward(s) if own else _plain_backward(s)
    return _own_adamw(s) if own else _plain_adamw(s)


def _own_forward(s):
    from paper_1910_02120_b200 import api
    y, mean, rstd = api.ist_layer_norm_forward(s["x"], s["weight"], s["bias"], EPS, groups=s["groups"],
                                               y_dtype=TYPES[s["y"]], want_stats=s["stats"])
    return {"y": y, "mean": mean, "rstd": rstd} if s["stats"] else {"y": y}


def _own_backward(s):
    from paper_1910_02120_b200 import api
    dx, dweight, dbias = api.ist_layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], groups=s["groups"])
    return {"dx": dx, "dweight": dweight, "dbias": dbias}


def _own_adamw(s):
    norm = s["opt"].step(s["gs"])
    out = {"p": s["p"]}
    if s["bits"] == 8:
        out["m"], out["v"] = s["opt"].state_values(torch.bfloat16)
    else:
        out["m"], out["v"] = s["state"]["exp_avg"], s["state"]["exp_avg_sq"]
    if s["copies"]:
        out["copy"] = s["copy"]
    if norm is not None:
        out["norm"] = norm
    return out


def _plain_forward(s):
    x = s["x"].float()
    mean = x.sum(1, keepdim=True) / s["cols"]
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).sum(1, keepdim=True) / s["cols"] + EPS)
    xh = (d * rstd).view(s["groups"], -1, s["cols"])
    y = (xh * s["weight"][:, None] + s["bias"][:, None]).view(x.shape).to(TYPES[s["y"]])
    return {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]} if s["stats"] else {"y": y}


def _plain_backward(s):
    shape = (s["groups"], -1, s["cols"])
    dy = s["dy"].float().view(shape) if s["dy"].is_contiguous() else s["dy"].float().reshape(shape)
    rstd = s["rstd"].view(s["groups"], -1, 1)
    xh = (s["x"].float().reshape(shape) - s["mean"].view(s["groups"], -1, 1)) * rstd
    g = dy * s["weight"][:, None]
    dx = rstd * (g - g.sum(2, keepdim=True) / s["cols"] - xh * ((g * xh).sum(2, keepdim=True) / s["cols"]))
    return {"dx": dx.view(s["x"].shape).to(s["x"].dtype), "dweight": (dy * xh).sum(1), "dbias": dy.sum(1)}


def _splitmix(x):
    """SplitMix64's output function on int64 tensors (sums and products wrap)."""
    signed = lambda c: c - 2 ** 64 if c >= 2 ** 63 else c
    x = (x ^ ((x >> 30) & (2 ** 34 - 1))) * signed(MIX1)
    x = (x ^ ((x >> 27) & (2 ** 37 - 1))) * signed(MIX2)
    return x ^ ((x >> 31) & (2 ** 33 - 1))


def _output(seed, i):
    """The i-th output (i from 1) of a SplitMix64 generator seeded with `seed`, as a Python integer."""
    x = (seed + i * GOLDEN) & MASK
    x = ((x ^ (x >> 30)) * MIX1) & MASK
    x = ((x ^ (x >> 27)) * MIX2) & MASK
    return x ^ (x >> 31)


def _noise(seed, step, room):
    """20-bit noise for the first and the second moment of every value: two values share a word, of which the first takes
    the low half; a half's low 16 bits are the first moment's."""
    signed = lambda c: c - 2 ** 64 if c >= 2 ** 63 else c
    k = _output(seed, step)
    pairs = torch.tensor([r // 2 for r in room], device="cuda")
    key = torch.tensor([signed(_output(k, j + 1)) for j in range(len(room))], device="cuda")
    key = key - (pairs.cumsum(0) - pairs - 1) * signed(GOLDEN)
    word = torch.arange(sum(room) // 2, device="cuda") * signed(GOLDEN) + key.repeat_interleave(pairs)
    word = _splitmix(word)
    half = torch.stack([word & 0xffffffff, (word >> 32) & 0xffffffff], 1).view(-1)
    return ((half & 0xffff) * 16 + 8).int(), ((half >> 16) * 16 + 8).int()


def _encode(x, noise, signed):
    """8-bit codes and bases of an fp32 state."""
    top = 126 if signed else 254
    bits = x.abs().view(torch.int32)
    finite = bits < 0x7f800000
    base = torch.where(finite, bits, 0).view(-1, BLOCK).amax(1).bitwise_right_shift(20).add(1 - top).clamp(min=0)
    room = base.repeat_interleave(BLOCK)
    code = torch.minimum((bits + noise) >> 20, torch.tensor(2039, device="cuda", dtype=torch.int32)) - room
    code = code.clamp(min=0) if signed else torch.where(bits > 0, code.clamp(min=1), 0)
    code = torch.where(finite, code, top + 1)
    code = code + 128 * ((x < 0) & (code > 0)) if signed else code
    return code.to(torch.uint8), base.to(torch.int16)


def _decode(code, base, signed):
    c = code.int()
    top = 127 if signed else 255
    bits = (base.int().repeat_interleave(BLOCK) + (c & top)) << 20
    x = torch.where((c & top) == 0, 0, bits).view(torch.float32)
    x = torch.where((c & top) == top, math.nan if signed else math.inf, x)
    return torch.where(c > 127, -x, x) if signed else x


def _joined(parts, room):
    return torch.cat([torch.nn.functional.pad(t.float(), (0, r - t.numel())) for t, r in zip(parts, room)])


def _plain_adamw(s):
    s["step"] += 1
    state, room = s["state"], s["room"]
    p, g = _joined(s["ps"], room), _joined(s["gs"], room)
    norm = None
    if s["max_norm"]:
        norm = (g.double() * g).sum().sqrt()
        g = g * torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    m, v = state["exp_avg"], state["exp_avg_sq"]
    if s["bits"] == 8:
        m, v = _decode(m, state["exp_avg_base"], True), _decode(v, state["exp_avg_sq_base"], False)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    decay = torch.tensor(s["decay"], device="cuda").repeat_interleave(torch.tensor(room, device="cuda"))
    u = m / (1 - BETA1 ** s["step"]) / ((v / (1 - BETA2 ** s["step"])).sqrt() + ADAM_EPS)
    p = p - LR * decay * p - LR * u
    parts = [t[:n] for t, n in zip(p.split(room), s["sizes"])]
    [t.copy_(q) for t, q in zip(s["ps"], parts)]
    out = {"p": s["p"]}
    if s["bits"] == 8:
        a, b = _noise(s["seed"], s["step"], room)
        mc, mb = _encode(m, a, True)
        vc, vb = _encode(v, b, False)
        [state[k].copy_(t) for k, t in zip(("exp_avg", "exp_avg_base", "exp_avg_sq", "exp_avg_sq_base"), (mc, mb, vc, vb))]
        m, v = _decode(mc, mb, True).bfloat16(), _decode(vc, vb, False).bfloat16()
    else:
        state["exp_avg"].copy_(m)
        state["exp_avg_sq"].copy_(v)
        m, v = state["exp_avg"], state["exp_avg_sq"]
    out["m"], out["v"] = m, v
    if s["copies"]:
        [t.copy_(q) for t, q in zip(s["copies"], parts)]
        out["copy"] = s["copy"]
    if norm is not None:
        out["norm"] = norm.float().view(1)
    return out


# --- 64 bits ----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    out = {k: [] for k in (("y", "mean", "rstd") if case["op"] == "norm_forward" else ("dx", "dweight", "dbias"))}
    each = case["rows"] // case["groups"]
    for k in range(case["groups"]):                              # site by site
        at = slice(k * each, (k + 1) * each)
        x, w, b = s["x"][at].double(), s["weight"][k].double(), s["bias"][k].double()
        if case["op"] == "norm_forward":
            var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
            sd = (var + EPS).sqrt()
            parts = ((x - mean) / sd * w + b, mean[:, 0], 1 / sd[:, 0])
        else:
            dy, mean, rstd = s["dy"][at].double(), s["mean"][at, None].double(), s["rstd"][at, None].double()
            h = (x - mean) * rstd
            gw = torch.einsum("rc,rc,c,r->r", dy, h, w, torch.ones(each, device="cuda", dtype=torch.float64)) / case["cols"]
            gm = dy @ w / case["cols"]
            parts = ((dy * w - gm[:, None] - h * gw[:, None]) * rstd, torch.einsum("rc,rc->c", dy, h)[None], dy.sum(0)[None])
        for key, part in zip(out, parts):
            out[key].append(part)
    out = {k: torch.cat(v) for k, v in out.items()}
    return out if case["stats"] else {"y": out["y"]}


def _exact_value(k):
    return torch.ldexp(8.0 + (k % 8).double(), (k // 8 - 130).double())


def _exact_code(x, u, top, lift):
    """Values of doubles after rounding to three bits behind the leading one, `u` in [0, 1) deciding, in a block's range;
    what lies below the range is lifted into it or becomes zero."""
    f, e = torch.frexp(x)
    number = lambda k: (e.long() + 125) * 8 + torch.floor(k).long()        # place on the grid of all fp32 exponents
    largest = torch.where(x > 0, number(f * 16), 0).view(-1, BLOCK).amax(1)
    floor = (largest + 1 - top).clamp(min=0).repeat_interleave(BLOCK)
    k = number(f * 16 + u)
    return torch.where(x == 0, 0.0, torch.where(k - floor >= 1, _exact_value(k), _exact_value(floor + 1) if lift else 0.0))


def _exact_adamw(s):
    t, state = s["step"] + 1, s["state"]
    pad = lambda v, room: torch.nn.functional.pad(v.double(), (0, room - v.numel()))
    scale = 1.0
    norm = None
    if s["max_norm"]:
        norm = torch.stack([g.double().pow(2).sum() for g in s["gs"]]).sum().sqrt()
        scale = torch.clamp(s["max_norm"] / norm, max=1.0)
    new_p = torch.zeros_like(s["p"], dtype=torch.float64)
    ms, vs, at = [], [], 0
    offsets, _ = _offsets(s["sizes"], s["packed"])
    for j, (p, g, n, room) in enumerate(zip(s["ps"], s["gs"], s["sizes"], s["room"])):
        m, v = state["exp_avg"][at:at + room], state["exp_avg_sq"][at:at + room]
        if s["bits"] == 8:
            mb, vb = (state[k][at // BLOCK:(at + room) // BLOCK].long().repeat_interleave(BLOCK) for k in ("exp_avg_base", "exp_avg_sq_base"))
            mk, vk = mb + (m.long() & 127), vb + v.long()
            sign = 1.0 - 2.0 * (m > 127).double()
            m = torch.where((m & 127) == 0, 0.0, _exact_value(mk)) * sign
            v = torch.where(v == 0, 0.0, _exact_value(vk))
        at += room
        g = pad(g, room) * scale
        m = m.double() * BETA1 + g * (1 - BETA1)
        v = v.double() * BETA2 + g * g * (1 - BETA2)
        step = (m[:n] / (1 - BETA1 ** t)) / (torch.sqrt(v[:n] / (1 - BETA2 ** t)) + ADAM_EPS)
        new_p[offsets[j]:offsets[j] + n] = p.double() * (1 - LR * s["decay"][j]) - LR * step
        if s["bits"] == 8:
            key = _output(_output(s["seed"], t), j + 1)
            i = torch.arange(room // 2, device="cuda")
            signed = lambda c: c - 2 ** 64 if c >= 2 ** 63 else c
            word = _splitmix((i + 1) * signed(GOLDEN) + signed(key))
            u = torch.stack([word & 0xffff, (word >> 32) & 0xffff], 1).view(-1), torch.stack([(word >> 16) & 0xffff, (word >> 48) & 0xffff], 1).view(-1)
            u = [(16.0 * k.double() + 8) / 2 ** 20 for k in u]
            m, v = m.sign() * _exact_code(m.abs(), u[0], 126, False), _exact_code(v, u[1], 254, True)
        ms.append(m)
        vs.append(v)
    out = {"p": new_p, "m": torch.cat(ms), "v": torch.cat(vs)}
    if s["copies"]:
        out["copy"] = new_p
    if norm is not None:
        out["norm"] = norm.view(1)
    return out
