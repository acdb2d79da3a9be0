"""A training step of a small token model around gated experts that keeps its activations in 8 bits:

    x = scale * table[tokens]          dynb_embed            kept in 8 bits (dynb_store8) for the norm's gradient
    n = layer norm(x)                  dynb_layer_norm       kept in 8 bits for the experts' first layer's
    a = f(n Wg^T) (n Wu^T)             moe_gated             gate and up kept in 8 bits by the same kernel
    o = x + sum over uses of w a W2^T  moe_product
    loss = mean |o - target|^2 / 2

The backward pass restores n (dynb_load8) where a product wants it, and reads x and the pair (gate, up) as they were kept: dynb_layer_norm_backward and
moe_gated_grad take rows in 8 bits.  What waits for it takes d + d + 2 h k bytes a token and a sixteenth more for the scales; in bfloat16, with the hidden rows, it is
4 d + 6 h k.  The router (k largest logits of a token, softmax over them, the order of the uses), the loss and the update are torch's.

    python examples/train_gated_experts.py [steps]
"""
from __future__ import annotations

import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1707_02402_amd as dyn  # noqa: E402
from train_expert_layer import data  # noqa: E402

BF = torch.bfloat16


def make(V=4000, d=512, h=1024, E=64, seed=0):
    """The parameters, fp32: embedding table, norm's weight and bias, router, the experts' gate and up, and their second layer."""
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape, std: torch.randn(*shape, generator=g, device="cuda") * std
    return dict(table=normal(V, d, std=d ** -0.5), gamma=torch.ones(d, device="cuda"), beta=torch.zeros(d, device="cuda"), Wr=normal(E, d, std=d ** -0.5),
                W1=normal(E, 2, h, d, std=d ** -0.5), W2=normal(E, d, h, std=h ** -0.5))


def route(logits, k):
    """The k largest logits' experts and weights of every token, and the uses stacked by expert: offsets, perm and its inverse."""
    E, T = logits.shape[1], len(logits)
    kept, idx = torch.topk(logits, k, dim=1)
    expert = idx.reshape(-1)
    perm = torch.argsort(expert, stable=True)
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(T * k, device=perm.device)
    ends = torch.searchsorted(expert[perm].contiguous(), torch.arange(E, device=perm.device), right=True)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=perm.device), ends]).int()
    return dict(idx=idx, weight=torch.softmax(kept, 1), perm=perm.int(), inv=inv, offsets=offsets)


def forward(p, tokens, k, gate=dyn.MOE_GATE_SILU):
    """Returns the output rows and what the backward pass wants of the forward one."""
    w = {name: p[name].to(BF) for name in ("table", "Wr", "W1", "W2")}
    d, h, T = p["table"].shape[1], p["W1"].shape[2], len(tokens)
    x = dyn.dynb_embed(tokens, w["table"], scale=math.sqrt(d))
    n, mean, rstd = dyn.dynb_layer_norm(x, p["gamma"], p["beta"], want_stats=True)
    r = route(n.float() @ w["Wr"].float().t(), k)
    pre = dyn.Rows8(torch.empty(T * k, 2, h, dtype=torch.int8, device="cuda"), torch.empty(T * k, 2, (h + 31) // 32, dtype=BF, device="cuda"))
    a = dyn.moe_gated(n, w["W1"], r["offsets"], perm=r["perm"], k=k, gate=gate, pre=pre)
    y = dyn.moe_product(a, w["W2"], r["offsets"])
    used = y.float()[r["inv"]].view(T, k, d)
    out = (x.float() + (used * r["weight"][..., None]).sum(1)).to(BF)
    return out, dict(w=w, x=dyn.dynb_store8(x), n=dyn.dynb_store8(n), pre=pre, mean=mean, rstd=rstd, y=y, route=r, gate=gate)


def backward(p, tokens, k, kept, do):
    """Gradients (fp32) of the parameters for do, the loss's gradient by the output rows (bfloat16)."""
    w, r, T = kept["w"], kept["route"], len(tokens)
    V, d = p["table"].shape
    E, _, h, _ = p["W1"].shape
    M, off, perm = T * k, r["offsets"], r["perm"]
    token = (perm // k).long()
    n = dyn.dynb_load8(kept["n"])
    dy = (do[token].float() * r["weight"].reshape(M)[perm.long()][:, None]).to(BF)
    dpre, a = dyn.moe_gated_grad(dy, w["W2"], off, kept["pre"], gate=kept["gate"])
    dW2 = dyn.moe_product_grad_weight(dy, a, off)
    dW1 = dyn.moe_product_grad_weight(dpre.view(M, 2 * h), n, off, perm=perm, k=k).view(E, 2, h, d)
    drows = dyn.moe_product_grad_input(dpre.view(M, 2 * h), w["W1"].view(E, 2 * h, d), off)
    dn = drows[r["inv"]].float().view(T, k, d).sum(1)
    # the router: softmax over the k kept logits
    dweight = (kept["y"].float() * do[token].float()).sum(1)[r["inv"]].view(T, k)
    dkept = r["weight"] * (dweight - (r["weight"] * dweight).sum(1, keepdim=True))
    dlogits = torch.zeros(T, E, device="cuda").scatter_(1, r["idx"], dkept)
    dWr = dlogits.t() @ n.float()
    dn += dlogits @ w["Wr"].float()
    dx, dgamma, dbeta = dyn.dynb_layer_norm_backward(dn.to(BF), kept["x"], p["gamma"], kept["mean"], kept["rstd"])
    dtable = dyn.dynb_embed_backward(tokens, (dx.float() + do.float()).to(BF), V, scale=math.sqrt(d))
    return dict(table=dtable, gamma=dgamma, beta=dbeta, Wr=dWr, W1=dW1, W2=dW2)


def step(p, tokens, target, k=2, lr=0.5, max_norm=1.0):
    """One step of gradient descent; returns the loss and the norm that the gradients had."""
    o, kept = forward(p, tokens, k)
    diff = o.float() - target
    loss = diff.square().sum(1).mean() / 2
    grads = backward(p, tokens, k, kept, (diff / len(tokens)).to(BF))
    norm = dyn.dynb_clip_gradients(list(grads.values()), max_norm)
    for name, g in grads.items():
        p[name].add_(g, alpha=-lr)
    return loss, norm


def main(steps=20):
    V, d, T = 4000, 512, 8192
    p = make(V, d)
    for i in range(steps):
        tokens, target = data(V, d, T, 1000 + i)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        loss, norm = step(p, tokens, target)
        print(f"step {i:3d}  loss {float(loss):8.4f}  gradients' norm {float(norm):8.4f}  {(time.perf_counter() - t0) * 1e3:7.2f} ms", flush=True)


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20)
