"""IST on the fully connected head of a network with a convolutional trunk (paper Sec. 2.2, "IST for
other architectures": the trunk is held whole by every site and trained by local SGD, its copies
averaged when the subnets are copied back; only the fully connected part is partitioned).

    python -m paper_1910_02120_b200.trunk_head --rounds 30

The head (partition, local steps, reassembly) runs in the CUDA library; the trunk is the caller's
part and is a small torch module here: one copy per subnet, which turns its subnet's images into
the head's input rows, receives the loss gradient with respect to those rows from
ist_local_steps_dx (one local step per call) and takes its own SGD step.  Synthetic images, a
synthetic teacher: a demonstration that the pieces fit, one JSON line per round.

    python -m paper_1910_02120_b200.trunk_head --trunk-norm --trunk-optimizer adamw8 --trunk-lr 0.003

puts a layer norm between trunk and head (one launch for all sites, each with its own weight and bias) and trains
trunk and norm by AdamW (one launch for all sites' tensors, states in 32 or 8 bits); both run in the CUDA library too.
"""
from __future__ import annotations

import argparse
import copy
import json
from typing import List

import torch

from . import api


def make_task(n: int, classes: int, seed: int, device):
    """Images [n][1][12][12] ~ N(0,1); labels from a fixed random convolution + linear teacher."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    x = torch.randn(n, 1, 12, 12, generator=g)
    k = torch.randn(4, 1, 3, 3, generator=g)
    a = torch.randn(4 * 5 * 5, classes, generator=g)
    f = torch.nn.functional.avg_pool2d(torch.tanh(torch.nn.functional.conv2d(x, k)), 2).flatten(1)
    return x.to(device), (f @ a).argmax(1).to(torch.int32).to(device)


def make_trunk(features: int, seed: int, device):
    torch.manual_seed(seed)
    return torch.nn.Sequential(torch.nn.Conv2d(1, 8, 3), torch.nn.ReLU(), torch.nn.AvgPool2d(2),
                               torch.nn.Flatten(), torch.nn.Linear(8 * 5 * 5, features)).to(device)


def make_optimizers(kind: str, sites: List[List[torch.Tensor]], lr: float, clip: float) -> List[api.AdamW]:
    """AdamW for the sites' tensors: one for all of them, or one per site where a site clips its gradients by itself.
    Vectors do not decay."""
    groups = [[p.detach() for p in site] for site in sites]
    if not clip:
        groups = [sum(groups, [])]
    return [api.AdamW(g, lr=lr, weight_decay=[0.01 if p.dim() > 1 else 0.0 for p in g], state_bits=8 if kind == "adamw8" else 32,
                      max_norm=clip or None, seed=i) for i, g in enumerate(groups)]


def train(rounds: int = 30, S: int = 4, K: int = 10, B: int = 64, features: int = 64, hidden: int = 256,
          classes: int = 10, lr: float = 0.3, precision: str = "fp32", seed: int = 1,
          device: str = "cuda:0", norm: bool = False, optimizer: str = "sgd", trunk_lr: float = None,
          clip: float = 0.0) -> List[dict]:
    """Runs `rounds` rounds; returns per round the mean loss of the subnets' local steps.  norm: a layer norm behind every
    site's trunk.  optimizer of trunks and norms: "sgd", "adamw" or "adamw8" (states in 8 bits), with learning rate trunk_lr (default lr);
    clip: bound of a site's gradient norm (AdamW; 0: none)."""
    if optimizer not in ("sgd", "adamw", "adamw8"):
        raise ValueError(f"unknown optimizer {optimizer}")
    if clip and optimizer == "sgd":
        raise ValueError("clip needs an AdamW optimizer")
    dev = torch.device(device)
    trunk_lr = lr if trunk_lr is None else trunk_lr
    n = S * K * B * 4
    x_all, y_all = make_task(n, classes, seed, dev)
    dims = [features, hidden, hidden, classes]
    g = torch.Generator(device="cpu").manual_seed(seed + 1)
    Wd = [((torch.rand(dims[i], dims[i + 1], generator=g) * 2 - 1) * (6.0 / dims[i]) ** 0.5).to(dev) for i in range(3)]
    bd = [torch.zeros(dims[i + 1], device=dev) for i in range(3)]
    prec = api.IST_BF16 if precision == "bf16" else api.IST_FP32
    ctx = api.Ist(dims, S, prec, B, device=device)
    ctx.bind_weights(Wd, bd)
    trunk = make_trunk(features, seed, dev)
    copies = [copy.deepcopy(trunk) for _ in range(S)]
    # every site's norm: row s belongs to site s
    weight, bias = torch.ones(S, features, device=dev), torch.zeros(S, features, device=dev)
    row_type = torch.bfloat16 if precision == "bf16" and features % 8 == 0 else torch.float32
    site_tensors = [list(copies[s].parameters()) + ([weight[s], bias[s]] if norm else []) for s in range(S)]
    opts = [] if optimizer == "sgd" else make_optimizers(optimizer, site_tensors, trunk_lr, clip)
    records = []
    for r in range(rounds):
        perm = torch.randperm(n, generator=g)[: S * K * B].to(dev).view(S, K, B)
        with torch.no_grad():                                  # the trunk goes to every site whole
            for c in copies:
                for p, q in zip(c.parameters(), trunk.parameters()):
                    p.copy_(q)
        ctx.partition(seed * 7919 + r)
        losses = []
        for k in range(K):
            rows = perm[:, k, :].reshape(-1)                   # [S][1][B]: one local step per call
            feats = [copies[s](x_all[rows[s * B:(s + 1) * B]]) for s in range(S)]
            X = torch.cat(feats).detach().contiguous()
            if norm:
                Xin, mean, rstd = api.ist_layer_norm_forward(X, weight, bias, groups=S, y_dtype=row_type)
            else:
                Xin = X.to(row_type)
            dx = torch.empty(S * B, features, dtype=torch.float32, device=dev)
            loss = ctx.local_steps(Xin, y_all[rows].contiguous(), lr, 1, B, dx_out=dx)
            losses.append(loss.mean().item())
            if norm:
                dx, dweight, dbias = api.ist_layer_norm_backward(dx, X, weight, mean, rstd, groups=S)
            grads = []
            for s in range(S):                                 # each site's trunk: its own step from its dX
                copies[s].zero_grad()
                feats[s].backward(dx[s * B:(s + 1) * B])
                grads.append([p.grad for p in copies[s].parameters()] + ([dweight[s], dbias[s]] if norm else []))
            if opts:
                for o, gs in zip(opts, grads if clip else [sum(grads, [])]):
                    o.step(gs)
            else:
                with torch.no_grad():
                    for tensors, gs in zip(site_tensors, grads):
                        for p, q in zip(tensors, gs):
                            p -= trunk_lr * q
        ctx.reassemble()
        ctx.sync_status()
        with torch.no_grad():                                  # the trunk's copies are averaged
            for p, *ps in zip(trunk.parameters(), *[c.parameters() for c in copies]):
                p.copy_(torch.stack(ps).mean(0))
            for v in (weight, bias):
                v.copy_(v.mean(0).expand_as(v).contiguous())
        records.append({"round": r + 1, "subnet_loss": sum(losses) / len(losses)})
    ctx.close()
    return records


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rounds", type=int, default=30)
    ap.add_argument("--S", type=int, default=4)
    ap.add_argument("--K", type=int, default=10)
    ap.add_argument("--B", type=int, default=64)
    ap.add_argument("--lr", type=float, default=0.3)
    ap.add_argument("--precision", default="fp32", choices=["bf16", "fp32"])
    ap.add_argument("--trunk-norm", action="store_true", help="a layer norm between trunk and head")
    ap.add_argument("--trunk-optimizer", default="sgd", choices=["sgd", "adamw", "adamw8"])
    ap.add_argument("--trunk-lr", type=float, default=None, help="learning rate of the trunk (default: --lr)")
    ap.add_argument("--trunk-clip", type=float, default=0.0, help="bound of a site's gradient norm (AdamW)")
    args = ap.parse_args()
    for rec in train(args.rounds, args.S, args.K, args.B, lr=args.lr, precision=args.precision, norm=args.trunk_norm,
                     optimizer=args.trunk_optimizer, trunk_lr=args.trunk_lr, clip=args.trunk_clip):
        print(json.dumps(rec))


if __name__ == "__main__":
    main()
