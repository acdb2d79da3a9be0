"""The operators together, as examples/train_expert_layer.py runs them: a step's gradients, and a loss that falls.

The reference is the step written out in 64 bits, expert by expert.  Without roundings it has to be what autograd gives (to 1e-9); rounding the tensors that
the step stores in bfloat16 (x, n, hidden rows, results and their gradients) at the same places it has to be what the operators give.  What is left between the
two are fp32 sums, off by some 1e-6: they move a stored number to its neighbour, 2^-7 of it away at most, where the sum lies that near to the middle between
two, which is one number in some thousand: 2^-7 / sqrt(1000) of a tensor's norm, 2.5e-4.  Six such tensors follow one another; the bound is 2^-8."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F8 = torch.bfloat16, torch.float64
BOUND = 2.0 ** -8


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_expert_layer
    return train_expert_layer


def norm_parts(x, eps=1e-5):
    centred = x - x.mean(1, keepdim=True)
    rstd = (centred.square().mean(1, keepdim=True) + eps).rsqrt()
    return centred * rstd, rstd


def written_out(p, tokens, idx, do, k, rnd):
    """Output rows and gradients of a step, routing idx [T,k] given; rnd: what storing a tensor does to it."""
    known, d, E = (tokens >= 0)[:, None], p["table"].shape[1], p["Wg"].shape[0]
    x = rnd(torch.where(known, p["table"][tokens.clamp(min=0).long()] * d ** 0.5, 0.0))
    xhat, rstd = norm_parts(x)
    n = rnd(xhat * p["gamma"] + p["beta"])
    weight = torch.softmax((n @ p["Wg"].t()).gather(1, idx), 1)
    y = torch.zeros(*idx.shape, d, dtype=F8, device="cuda")
    hid = torch.zeros(*idx.shape, p["W1"].shape[1], dtype=F8, device="cuda")
    uses = [torch.nonzero(idx == e, as_tuple=True) for e in range(E)]
    for e, (t, j) in enumerate(uses):
        hid[t, j] = rnd(torch.relu(n[t] @ p["W1"][e].t()))
        y[t, j] = rnd(hid[t, j] @ p["W2"][e].t())
    out = rnd(x + rnd((weight[..., None] * y).sum(1)))
    dy = rnd(weight[..., None] * do[:, None])
    dW1, dW2, drows = torch.zeros_like(p["W1"]), torch.zeros_like(p["W2"]), torch.zeros_like(y)
    for e, (t, j) in enumerate(uses):
        dhid = rnd((dy[t, j] @ p["W2"][e]) * (hid[t, j] > 0))
        dW2[e], dW1[e] = dy[t, j].t() @ hid[t, j], dhid.t() @ n[t]
        drows[t, j] = rnd(dhid @ p["W1"][e])
    dweight = (y * do[:, None]).sum(2)
    dlogits = torch.zeros(len(tokens), E, dtype=F8, device="cuda").scatter_(1, idx, weight * (dweight - (weight * dweight).sum(1, keepdim=True)))
    dn = rnd(drows.sum(1) + dlogits @ p["Wg"])
    g = dn * p["gamma"]
    dx = rnd(rnd(rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))) + do)
    dtable = torch.zeros_like(p["table"]).index_add_(0, tokens[known[:, 0]].long(), dx[known[:, 0]]) * d ** 0.5
    return out, dict(table=dtable, gamma=(dn * xhat).sum(0), beta=dn.sum(0), Wg=dlogits.t() @ n, W1=dW1, W2=dW2)


@pytest.mark.parametrize("V,d,h,E,T,k", [(300, 64, 96, 8, 500, 2), (2000, 128, 256, 40, 3000, 3), (50, 72, 40, 3, 37, 1)])
def test_gradients_of_a_step(example, V, d, h, E, T, k):
    p = {n: t.to(BF).float() for n, t in example.make(V, d, h, E, seed=V).items()}
    tokens, target = example.data(V, d, T, 5)
    o, kept = example.forward(p, tokens, k)
    do = ((o.float() - target) / T).to(BF)
    got = example.backward(p, tokens, k, kept, do)
    idx, q = kept["route"].topk_idx.long(), {n: t.double() for n, t in p.items()}
    off = lambda a, b: float((a.double() - b).norm() / b.norm().clamp(min=1e-30))
    # the reference against autograd
    plain_out, plain = written_out(q, tokens, idx, do.double(), k, lambda t: t)
    a = {n: t.clone().requires_grad_() for n, t in q.items()}
    x = torch.where((tokens >= 0)[:, None], a["table"][tokens.clamp(min=0).long()] * d ** 0.5, 0.0)
    n = torch.nn.functional.layer_norm(x, (d,), a["gamma"], a["beta"], 1e-5)
    weight, out = torch.softmax((n @ a["Wg"].t()).gather(1, idx), 1), x
    for e in range(E):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        out = out.index_add(0, t, weight[t, j][:, None] * (torch.relu(n[t] @ a["W1"][e].t()) @ a["W2"][e].t()))
    (out * do.double()).sum().backward()
    assert off(plain_out, out.detach()) < 1e-9
    for name in got:
        # (one use a token: its weight is 1 whatever the logits are, and the gate has no gradient)
        assert off(plain[name], a[name].grad) < 1e-9 or (name == "Wg" and k == 1), name
    # the operators against the reference
    ref_out, ref = written_out(q, tokens, idx, do.double(), k, lambda t: t.to(BF).double())
    assert off(o, ref_out) < BOUND
    for name, t in got.items():
        if name == "Wg" and k == 1:
            assert float(t.abs().max()) < 1e-6
        else:
            assert off(t, ref[name]) < BOUND, name


def test_the_loss_falls(example):
    p = example.make(500, 128, 256, 16, seed=3)
    losses = []
    for i in range(30):
        tokens, target = example.data(500, 128, 2048, 1000 + i)
        loss, norm = example.step(p, tokens, target, k=2, lr=1.0, max_norm=1.0)
        assert torch.isfinite(loss) and torch.isfinite(norm)
        losses.append(float(loss))
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5]), losses
