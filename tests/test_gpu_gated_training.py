"""The gated layer and the rows in 8 bits together, as examples/train_gated_experts.py runs them.

The reference is the step written out in 64 bits, expert by expert.  Without roundings it has to be what autograd gives (to 1e-9); rounding what the step stores,
to bfloat16 or to 8 bits, at the same places it has to be what the operators give.  What is left between the two are fp32 sums, off by some 1e-6: they move a stored number to
its neighbour where the sum lies that near to the middle between two.  In bfloat16 that is 2^-7 of one number in some thousand, 2.5e-4 of a tensor's norm; in 8 bits, whose step
is 1 / 127 of a block's largest, some 2 % of the norm of one number in ten thousand, 2e-4.  Eight such tensors follow one another; the bound is 2^-8."""
import os
import sys

import pytest
import torch

from tests.test_gpu_gated import gate_of
from tests.test_gpu_rows8 import to_eight, values
from tests.test_gpu_training import norm_parts

pytestmark = pytest.mark.gpu
BF, F8 = torch.bfloat16, torch.float64
BOUND = 2.0 ** -8


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_gated_experts
    return train_gated_experts


def eight(x):
    """What x comes back as from 8 bits."""
    return values(*to_eight(x.cpu())).to(x.device)


def written_out(p, tokens, idx, do, k, gate, rnd, kept):
    """Output rows and gradients of a step, routing idx [T,k] given; rnd: what storing a tensor does to it, kept: what keeping it for the backward pass does."""
    known, d, E = (tokens >= 0)[:, None], p["table"].shape[1], p["Wr"].shape[0]
    x = rnd(torch.where(known, p["table"][tokens.clamp(min=0).long()] * d ** 0.5, 0.0))
    xhat, rstd = norm_parts(x)
    n = rnd(xhat * p["gamma"] + p["beta"])
    weight = torch.softmax((n @ p["Wr"].t()).gather(1, idx), 1)
    T, h = len(tokens), p["W1"].shape[2]
    pre, act = torch.zeros(T, k, 2, h, dtype=F8, device="cuda"), torch.zeros(T, k, h, dtype=F8, device="cuda")
    y = torch.zeros(T, k, d, dtype=F8, device="cuda")
    uses = [torch.nonzero(idx == e, as_tuple=True) for e in range(E)]
    for e, (t, j) in enumerate(uses):
        pre[t, j] = torch.stack([n[t] @ p["W1"][e, 0].t(), n[t] @ p["W1"][e, 1].t()], 1)
        act[t, j] = rnd(gate_of(gate, pre[t, j, 0])[0] * pre[t, j, 1])
        y[t, j] = rnd(act[t, j] @ p["W2"][e].t())
    out = rnd(x + (weight[..., None] * y).sum(1))
    x8, n8, pre8 = kept(x), kept(n), kept(pre)
    mean = x.mean(1, keepdim=True)
    dy = rnd(weight[..., None] * do[:, None])
    dW1, dW2, drows = torch.zeros_like(p["W1"]), torch.zeros_like(p["W2"]), torch.zeros_like(y)
    for e, (t, j) in enumerate(uses):
        f, slope = gate_of(gate, pre8[t, j, 0])[:2]
        up, dact = pre8[t, j, 1], dy[t, j] @ p["W2"][e]
        dg, du, again = rnd(dact * up * slope), rnd(dact * f), rnd(f * up)
        dW2[e] = dy[t, j].t() @ again
        dW1[e, 0], dW1[e, 1] = dg.t() @ rnd(n8[t]), du.t() @ rnd(n8[t])
        drows[t, j] = rnd(dg @ p["W1"][e, 0] + du @ p["W1"][e, 1])
    dweight = (y * do[:, None]).sum(2)
    dlogits = torch.zeros(T, E, dtype=F8, device="cuda").scatter_(1, idx, weight * (dweight - (weight * dweight).sum(1, keepdim=True)))
    dn = rnd(drows.sum(1) + dlogits @ p["Wr"])
    g, hat = dn * p["gamma"], (x8 - mean) * rstd
    dx = rnd(rnd(rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))) + do)
    dtable = torch.zeros_like(p["table"]).index_add_(0, tokens[known[:, 0]].long(), dx[known[:, 0]]) * d ** 0.5
    return out, dict(table=dtable, gamma=(dn * hat).sum(0), beta=dn.sum(0), Wr=dlogits.t() @ rnd(n8), W1=dW1, W2=dW2)


@pytest.mark.parametrize("V,d,h,E,T,k,gate", [(300, 64, 96, 8, 500, 2, "silu"), (2000, 128, 256, 40, 3000, 3, "gelu"), (50, 72, 40, 3, 37, 1, "silu"), (200, 75, 101, 5, 260, 2, "gelu")])
def test_gradients_of_a_step(example, V, d, h, E, T, k, gate):
    p = {n: t.to(BF).float() for n, t in example.make(V, d, h, E, seed=V).items()}
    tokens, target = example.data(V, d, T, 5)
    o, kept = example.forward(p, tokens, k, gate=example.dyn.MOE_GATE_GELU if gate == "gelu" else example.dyn.MOE_GATE_SILU)
    do = ((o.float() - target) / T).to(BF)
    got = example.backward(p, tokens, k, kept, do)
    idx, q = kept["route"]["idx"], {n: t.double() for n, t in p.items()}
    off = lambda a, b: float((a.double() - b).norm() / b.norm().clamp(min=1e-30))
    # the reference against autograd
    plain_out, plain = written_out(q, tokens, idx, do.double(), k, gate, lambda t: t, lambda t: t)
    a = {n: t.clone().requires_grad_() for n, t in q.items()}
    x = torch.where((tokens >= 0)[:, None], a["table"][tokens.clamp(min=0).long()] * d ** 0.5, 0.0)
    n = torch.nn.functional.layer_norm(x, (d,), a["gamma"], a["beta"], 1e-5)
    weight, out = torch.softmax((n @ a["Wr"].t()).gather(1, idx), 1), x
    f = torch.nn.functional.silu if gate == "silu" else lambda t: torch.nn.functional.gelu(t, approximate="tanh")
    for e in range(E):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        out = out.index_add(0, t, weight[t, j][:, None] * ((f(n[t] @ a["W1"][e, 0].t()) * (n[t] @ a["W1"][e, 1].t())) @ a["W2"][e].t()))
    (out * do.double()).sum().backward()
    assert off(plain_out, out.detach()) < 1e-9
    for name in got:
        # (one use a token: its weight is 1 whatever the logits are, and the router has no gradient)
        assert off(plain[name], a[name].grad) < 1e-9 or (name == "Wr" and k == 1), name
    # the operators against the reference
    ref_out, ref = written_out(q, tokens, idx, do.double(), k, gate, lambda t: t.to(BF).double(), eight)
    assert off(o, ref_out) < BOUND
    for name, t in got.items():
        if name == "Wr" and k == 1:
            assert float(t.abs().max()) < 1e-6
        else:
            assert off(t, ref[name]) < BOUND, name


def test_steps_run(example):
    p = example.make(500, 128, 256, 16, seed=3)
    for i in range(3):
        tokens, target = example.data(500, 128, 2048, 1000 + i)
        loss, norm = example.step(p, tokens, target)
        assert torch.isfinite(loss) and torch.isfinite(norm) and float(norm) > 0
    assert all(torch.isfinite(t).all() for t in p.values())
