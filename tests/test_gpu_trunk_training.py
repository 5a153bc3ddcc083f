"""Layer norm, the partitioned head and AdamW as a trunk's training uses them: trunk features -> layer norm of all sites ->
one local step of the head, which returns its input gradient -> layer norm's way back -> AdamW over all sites' tensors."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def api():
    from paper_1910_02120_b200 import api as a
    return a


@pytest.mark.parametrize("precision, tol", [("fp32", 1e-4), ("bf16", 1e-1)])
def test_gradients_through_norm_and_head(api, precision, tol):
    """Against torch's autograd in 64 bits on each site's subnet.  The head's input gradient is good to 1e-4 of its size in fp32 and to
    1e-1 in bf16 (the bounds of its own test); layer norm's way back is linear in it, and adds roundings below 1e-5."""
    S, B, dims = 4, 64, [64, 256, 256, 10]
    gen = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)
    W = [rnd(dims[i], dims[i + 1]) * (2.0 / dims[i]) ** 0.5 for i in range(3)]
    b = [0.1 * rnd(dims[i + 1]) for i in range(3)]
    features = rnd(S * B, dims[0]) * 1.5 + 0.5
    weight, bias = 1 + 0.2 * rnd(S, dims[0]), 0.1 * rnd(S, dims[0])
    y = torch.randint(0, dims[-1], (S * B,), generator=gen, device=DEV, dtype=torch.int32)
    ctx = api.Ist(dims, S, api.IST_BF16 if precision == "bf16" else api.IST_FP32, B)
    ctx.bind_weights(W, b)
    ctx.partition(5)
    subnets = [[tuple(t.double() for t in ctx.get_subnet_params(layer, s)) for layer in (1, 2, 3)] for s in range(S)]
    rows, mean, rstd = api.ist_layer_norm_forward(features, weight, bias, groups=S,
                                                  y_dtype=torch.bfloat16 if precision == "bf16" else torch.float32)
    dx = torch.empty(S * B, dims[0], device=DEV)
    loss = ctx.local_steps(rows, y, 0.1, 1, B, dx_out=dx)
    dfeatures, dweight, dbias = api.ist_layer_norm_backward(dx, features, weight, mean, rstd, groups=S)
    ctx.reassemble()
    ctx.sync_status()
    f64, w64, b64 = (t.double().requires_grad_() for t in (features, weight, bias))
    f3 = f64.view(S, B, -1)
    a = (f3 - f3.mean(2, keepdim=True)) / (f3.var(2, correction=0, keepdim=True) + 1e-5).sqrt() * w64[:, None] + b64[:, None]
    losses = []
    for s in range(S):
        z = a[s]
        for layer, (Ws, bs) in enumerate(subnets[s]):
            z = z @ Ws + bs
            if layer < 2:
                z = z.relu()
        losses.append(torch.nn.functional.cross_entropy(z, y[s * B:(s + 1) * B].long()))
    sum(losses).backward()
    for s in range(S):
        assert abs(float(loss[s, 0]) - losses[s].item()) <= (1e-3 if precision == "bf16" else 1e-4) * max(1.0, losses[s].item())
    for got, want in ((dfeatures, f64.grad), (dweight, w64.grad), (dbias, b64.grad)):
        assert float((got.double() - want).norm() / want.norm()) <= tol
    # and the step that follows
    params, grads = [weight.clone(), bias.clone()], [dweight, dbias]
    before = [p.double() for p in params]
    api.AdamW(params, lr=0.01, weight_decay=0.0).step(grads)
    for p, q, g in zip(params, before, grads):
        g = g.double()
        assert ((p.double() - (q - 0.01 * g / (g.abs() + 1e-8))).abs() <= 2.0 ** -20 * (q.abs() + 0.01)).all()


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("options", [dict(norm=True), dict(optimizer="adamw", trunk_lr=0.003), dict(norm=True, optimizer="adamw", trunk_lr=0.003),
                                     dict(norm=True, optimizer="adamw8", trunk_lr=0.003), dict(norm=True, optimizer="adamw", trunk_lr=0.003, clip=1.0),
                                     dict(norm=True, optimizer="adamw8", trunk_lr=0.003, clip=1.0)])
def test_the_command_runs(precision, options):
    from paper_1910_02120_b200 import trunk_head
    records = trunk_head.train(rounds=3, S=4, K=4, B=64, precision=precision, seed=2, **options)
    assert len(records) == 3 and all(np.isfinite(r["subnet_loss"]) and 0 < r["subnet_loss"] < 20 for r in records)
    again = trunk_head.train(rounds=3, S=4, K=4, B=64, precision=precision, seed=2, **options)
    assert [r["round"] for r in again] == [1, 2, 3]


def test_the_command_refuses(api):
    from paper_1910_02120_b200 import trunk_head
    with pytest.raises(ValueError):
        trunk_head.train(rounds=1, optimizer="adam")
    with pytest.raises(ValueError):
        trunk_head.train(rounds=1, clip=1.0)


def test_without_options_as_before(api):
    """The loop as it was before norm and optimizer could be chosen, step by step: the same losses."""
    import copy
    from paper_1910_02120_b200 import trunk_head
    S, K, B, features, hidden, classes, lr, seed, rounds = 2, 3, 32, 64, 128, 10, 0.3, 4, 2
    got = [r["subnet_loss"] for r in trunk_head.train(rounds, S, K, B, features, hidden, classes, lr, "fp32", seed)]
    dev = torch.device(DEV)
    n = S * K * B * 4
    x_all, y_all = trunk_head.make_task(n, classes, seed, dev)
    dims = [features, hidden, hidden, classes]
    g = torch.Generator(device="cpu").manual_seed(seed + 1)
    Wd = [((torch.rand(dims[i], dims[i + 1], generator=g) * 2 - 1) * (6.0 / dims[i]) ** 0.5).to(dev) for i in range(3)]
    bd = [torch.zeros(dims[i + 1], device=dev) for i in range(3)]
    ctx = api.Ist(dims, S, api.IST_FP32, B, device=DEV)
    ctx.bind_weights(Wd, bd)
    trunk = trunk_head.make_trunk(features, seed, dev)
    want = []
    for r in range(rounds):
        perm = torch.randperm(n, generator=g)[: S * K * B].to(dev).view(S, K, B)
        copies = [copy.deepcopy(trunk) for _ in range(S)]
        ctx.partition(seed * 7919 + r)
        losses = []
        for k in range(K):
            rows = perm[:, k, :].reshape(-1)
            feats = [copies[s](x_all[rows[s * B:(s + 1) * B]]) for s in range(S)]
            X = torch.cat(feats).detach().contiguous()
            dx = torch.empty(S * B, features, dtype=torch.float32, device=dev)
            losses.append(ctx.local_steps(X, y_all[rows].contiguous(), lr, 1, B, dx_out=dx).mean().item())
            for s in range(S):
                copies[s].zero_grad()
                feats[s].backward(dx[s * B:(s + 1) * B])
                with torch.no_grad():
                    for p in copies[s].parameters():
                        p -= lr * p.grad
        ctx.reassemble()
        with torch.no_grad():
            for p, *ps in zip(trunk.parameters(), *[c.parameters() for c in copies]):
                p.copy_(torch.stack(ps).mean(0))
        want.append(sum(losses) / len(losses))
    # library convolutions may add in another order from call to call: an ulp or two per step
    assert all(abs(a - b) <= 1e-4 * b for a, b in zip(got, want)), (got, want)
