"""A training step of a small token model around the expert layer, on the library's operators:

    x = scale * table[tokens]          dynb_embed            its gradient: dynb_embed_backward
    n = layer norm(x)                  dynb_layer_norm       dynb_layer_norm_backward
    o = x + experts(n)                 moe_forward           moe_product, moe_product_grad_input, moe_product_grad_weight
    loss = mean |o - target|^2 / 2
    all gradients down to a norm       dynb_clip_gradients

The forward pass keeps the layer's routing (moe_forward's aux) and nothing else of it: the backward pass makes the hidden rows again
with moe_product, as training with little memory does.  The router's few numbers (uses of a token, experts' logits), the loss and the
update are torch's; parameters are kept in fp32 and rounded to bfloat16 for the layer.

    python examples/train_expert_layer.py [steps]
"""
from __future__ import annotations

import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1707_02402_amd as dyn  # noqa: E402

BF = torch.bfloat16


def make(V=4000, d=512, h=1024, E=64, seed=0):
    """The parameters, fp32: embedding table, norm's weight and bias, gate, and the experts' two layers."""
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape, std: torch.randn(*shape, generator=g, device="cuda") * std
    return dict(table=normal(V, d, std=d ** -0.5), gamma=torch.ones(d, device="cuda"), beta=torch.zeros(d, device="cuda"), Wg=normal(E, d, std=d ** -0.5),
                W1=normal(E, h, d, std=(2.0 / d) ** 0.5), W2=normal(E, d, h, std=(0.2 / h) ** 0.5))


def forward(p, tokens, k):
    """Returns the output rows and what the backward pass wants of the forward one."""
    w = {name: p[name].to(BF) for name in ("table", "Wg", "W1", "W2")}
    d = p["table"].shape[1]
    x = dyn.dynb_embed(tokens, w["table"], scale=math.sqrt(d))
    n, mean, rstd = dyn.dynb_layer_norm(x, p["gamma"], p["beta"], want_stats=True)
    y, route = dyn.moe_forward(n, w["Wg"], None, None, w["W1"], w["W2"], k, want_aux=True)
    return x + y, dict(w=w, x=x, n=n, mean=mean, rstd=rstd, route=route)


def backward(p, tokens, k, kept, do):
    """Gradients (fp32) of the parameters for do, the loss's gradient by the output rows (bfloat16)."""
    w, n, r = kept["w"], kept["n"], kept["route"]
    V, d = p["table"].shape
    T, E, M = len(tokens), p["Wg"].shape[0], len(tokens) * k
    token = (r.perm // k).long()                                                          # whose use row r of the stacked rows is
    weight = r.topk_w.reshape(M)[r.perm.long()]
    # the experts: hidden rows and results again, then the two layers backwards
    hid = dyn.moe_product(n, w["W1"], r.offsets, perm=r.perm, k=k, relu=True)
    y = dyn.moe_product(hid, w["W2"], r.offsets)
    dy = (do[token].float() * weight[:, None]).to(BF)
    dhid = dyn.moe_product_grad_input(dy, w["W2"], r.offsets, act=hid)
    dW2 = dyn.moe_product_grad_weight(dy, hid, r.offsets)
    dW1 = dyn.moe_product_grad_weight(dhid, n, r.offsets, perm=r.perm, k=k)
    drows = dyn.moe_product_grad_input(dhid, w["W1"], r.offsets)
    dn = drows[r.inv.long()].float().view(T, k, d).sum(1)
    # the router: softmax over the k kept logits
    dweight = (y.float() * do[token].float()).sum(1)[r.inv.long()].view(T, k)
    dkept = r.topk_w * (dweight - (r.topk_w * dweight).sum(1, keepdim=True))
    dlogits = torch.zeros(T, E, device="cuda").scatter_(1, r.topk_idx.long(), dkept)
    dWg = dlogits.t() @ n.float()
    dn += dlogits @ w["Wg"].float()
    # the norm, the residual beside it, the embedding
    dx, dgamma, dbeta = dyn.dynb_layer_norm_backward(dn.to(BF), kept["x"], p["gamma"], kept["mean"], kept["rstd"])
    dtable = dyn.dynb_embed_backward(tokens, (dx.float() + do.float()).to(BF), V, scale=math.sqrt(d))
    return dict(table=dtable, gamma=dgamma, beta=dbeta, Wg=dWg, W1=dW1, W2=dW2)


def step(p, tokens, target, k=2, lr=0.5, max_norm=1.0):
    """One step of gradient descent; returns the loss and the norm that the gradients had."""
    o, kept = forward(p, tokens, k)
    diff = o.float() - target
    loss = diff.square().sum(1).mean() / 2
    grads = backward(p, tokens, k, kept, (diff / len(tokens)).to(BF))
    names = list(grads)
    norm = dyn.dynb_clip_gradients([grads[name] for name in names], max_norm)
    for name in names:
        p[name].add_(grads[name], alpha=-lr)
    return loss, norm


def data(V, d, T, seed):
    """Tokens by Zipf's law, some padding; a token's target is a vector of its own."""
    g = torch.Generator("cuda").manual_seed(seed)
    share = torch.arange(1, V + 1, device="cuda", dtype=torch.float64) ** -1.0
    tokens = torch.multinomial(share, T, replacement=True, generator=g).int()
    tokens[torch.rand(T, generator=g, device="cuda") < 0.02] = -1
    vectors = torch.randn(V + 1, d, generator=torch.Generator("cuda").manual_seed(99), device="cuda") * 0.5
    return tokens, vectors[tokens.long()]


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
