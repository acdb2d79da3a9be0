"""Gated expert layers, and activations that wait for the backward pass in 8 bits; the cases that their speed is measured on.

  gated         the first half of a gated feed-forward layer: rows of tokens, gathered and stacked by expert, times their
                expert's two matrices, out = f(gate) * up with f SiLU or GELU (its tanh form); with the pair (gate, up) in
                bfloat16 for the backward pass, or without it
  gated_grad    the gradient through the second layer's product and the gating at once: with dact = dout W, the gradients of
                gate and up, and f(gate) * up again for the second layer's weights' gradient
  gated_step8   both, as a training step runs them: the forward pass keeps (gate, up) in 8 bits, the backward pass reads them
  checkpoint8   rows of activations into 8 bits and back
  norm_grad8    the gradients of a layer norm whose input was kept in 8 bits

Rows in 8 bits: every 32 neighbours of a row (the last block may be shorter) share a scale s, a bfloat16, the largest magnitude
over 127 rounded up, and an element is the whole number nearest to x / s; both steps are fp32 arithmetic, rounded as it rounds.

Experts' loads follow Zipf's law, as routers' do, and some experts have no rows.  Widths are those of the benchmark
configurations' expert layers (512 -> 1024 with 256 experts and two uses of a token, 1024 -> 2048 with four), or drawn around them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                # False: the operators' plain forms; True: the framework's entry points

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
BLOCK = 32


# ------------------------------------------------------------------------------------------ the cases
def _gated(name, T, k, K, h, E, zipf, act="silu", keep=False, empty=0.0):
    return dict(name=name, kind="gated", T=T, k=k, K=K, h=h, E=E, zipf=zipf, act=act, keep=keep, empty=empty)


def _gated_grad(name, T, k, h, N, E, zipf, act="silu", pre="bf16", empty=0.0):
    return dict(name=name, kind="gated_grad", T=T, k=k, h=h, N=N, E=E, zipf=zipf, act=act, pre=pre, empty=empty)


def _gated_step8(name, T, k, K, h, N, E, zipf, act="silu", empty=0.0):
    return dict(name=name, kind="gated_step8", T=T, k=k, K=K, h=h, N=N, E=E, zipf=zipf, act=act, empty=empty)


def _rows(name, kind, T, d, dtype="bf16"):
    return dict(name=name, kind=kind, T=T, d=d, dtype=dtype)


def listed():
    return [
        # generation for one sequence: one token's two experts
        _gated("gated_2", 1, 2, 512, 1024, 256, 1.1),
        # generation for a few sequences through the large layer: most of the time is the experts' weights' way
        _gated("gated_148", 37, 4, 1024, 2048, 256, 1.1),
        # odd sizes: no row begins on a border of 16 bytes; training, the pair kept
        _gated("gated_3001_odd", 3001, 1, 777, 1001, 8, 0.5, act="gelu", keep=True),
        # a dense layer (one expert) in training
        _gated("gated_8192_dense", 8192, 1, 2048, 4096, 1, 0.0, act="gelu", keep=True),
        # crowded experts: a long prompt through the large layer
        _gated("gated_65536", 16384, 4, 1024, 2048, 64, 0.6, empty=0.05),
        # the small configuration's training batch, backward: few rows an expert
        _gated_grad("gated_grad_8192", 4096, 2, 1024, 512, 256, 1.1),
        # odd sizes from 8 bits
        _gated_grad("gated_grad_2999_odd", 2999, 1, 1001, 777, 8, 0.5, act="gelu", pre="i8"),
        # the large layer's batch forward and backward, the pair in 8 bits between
        _gated_step8("gated_step8_65536", 16384, 4, 1024, 2048, 1024, 64, 0.6, empty=0.05),
        # a few rows, where a launch is all there is
        _rows("checkpoint8_37x512", "checkpoint8", 37, 512),
        # the hidden rows of the large batch
        _rows("checkpoint8_65536x2048", "checkpoint8", 65536, 2048),
        # a batch of odd sizes in full precision
        _rows("norm_grad8_4097x777_f32", "norm_grad8", 4097, 777, dtype="f32"),
        # the large layer's batch
        _rows("norm_grad8_65536x1024", "norm_grad8", 65536, 1024),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Mostly a multiple of 64, sometimes of 8, sometimes anything."""
    n, form = _log_int(rng, lo, hi), rng.random()
    unit = 64 if form < 0.6 else 8 if form < 0.8 else 1
    return max(unit, n // unit * unit)


def draw(rng):
    kind = rng.choice(["gated", "gated", "gated", "gated_grad", "gated_grad", "gated_step8", "gated_step8", "checkpoint8", "norm_grad8"])
    while True:
        if kind in ("checkpoint8", "norm_grad8"):
            case = dict(kind=kind, T=_log_int(rng, 1, 65536), d=_width(rng, 32, 8192), dtype=rng.choice(["bf16", "bf16", "f32"]))
            fits = case["T"] * case["d"] <= 65536 * 1024
        else:
            E = _log_int(rng, 1, 1024)
            case = dict(kind=kind, T=_log_int(rng, 1, 16384), k=min(E, rng.choice([1, 2, 2, 4, 4])), h=_width(rng, 64, 4096), E=E,
                        zipf=round(rng.uniform(0.4, 1.2), 2), act=rng.choice(["silu", "silu", "gelu"]), empty=rng.choice([0.0, 0.05]) if E >= 64 else 0.0)
            if kind != "gated_grad":
                case["K"] = _width(rng, 64, 2048)
            if kind != "gated":
                case["N"] = _width(rng, 64, 2048)
            if kind == "gated":
                case["keep"] = rng.random() < 0.5
            if kind == "gated_grad":
                case["pre"] = rng.choice(["bf16", "i8"])
            wide = max(case.get("K", 0), case.get("N", 0))
            fits = (case["T"] * case["k"] * wide * case["h"] <= 65536 * 1024 * 2048 and E * wide * case["h"] <= 128 * 1024 * 2048 and
                    case["T"] * case["k"] * case["h"] <= 65536 * 2048)
        if fits:
            return case


# ------------------------------------------------------------------------------------------ inputs
def _generators(seed):
    return np.random.Generator(np.random.Philox(key=[seed, 31])), torch.Generator("cuda").manual_seed(seed * 1000003 + 31)


def _normal(g, *shape, dtype, std=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat, step = out.view(-1), 1 << 28
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda").mul_(std))
    return out


def _zipf(r, n, s, size):
    """`size` ids of 0 .. n - 1 with probabilities that fall as rank ** -s, the ranks dealt to the ids at random."""
    cum = np.cumsum(np.arange(1, n + 1, dtype=np.float64) ** -s)
    rank = np.minimum(np.searchsorted(cum, r.random(size) * cum[-1]), n - 1)
    return r.permutation(n)[rank]


def _eight(*shape):
    """Room for rows in 8 bits: the elements and the blocks' scales."""
    return dict(q=torch.empty(shape, dtype=torch.int8, device="cuda"),
                scale=torch.empty((*shape[:-1], (shape[-1] + BLOCK - 1) // BLOCK), dtype=torch.bfloat16, device="cuda"))


def _prepare_layer(case, seed):
    """The rows of all uses, stacked by expert: use a of token a // k stands where a stable sort by expert puts it."""
    r, g = _generators(seed)
    T, k, h, E = (case[x] for x in ("T", "k", "h", "E"))
    M, bf, kind = T * k, torch.bfloat16, case["kind"]
    live = max(1, E - int(round(E * case["empty"])))
    expert = r.permutation(E)[_zipf(r, live, case["zipf"], M)]
    counts = np.bincount(expert, minlength=E)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    st = dict(offsets=torch.from_numpy(offsets).cuda(), counts=counts.tolist(), k=k, act=case["act"], M=M, h=h, hidden=torch.empty((M, h), dtype=bf, device="cuda"))
    if kind != "gated_grad":
        st["perm"] = torch.from_numpy(np.argsort(expert, kind="stable").astype(np.int32)).cuda()
        st["x"] = _normal(g, T, case["K"], dtype=bf)
        st["W1"] = _normal(g, E, 2, h, case["K"], dtype=bf, std=math.sqrt(1.0 / case["K"]))
    if kind != "gated":
        st["dout"] = _normal(g, M, case["N"], dtype=bf, std=0.01)
        st["W2"] = _normal(g, E, case["N"], h, dtype=bf, std=math.sqrt(1.0 / h))
        st["dpre"] = torch.empty((M, 2, h), dtype=bf, device="cuda")
    if kind == "gated_step8":
        st.update(pre=_eight(M, 2, h), again=torch.empty((M, h), dtype=bf, device="cuda"))
    elif kind == "gated" and case["keep"]:
        st["pre"] = torch.empty((M, 2, h), dtype=bf, device="cuda")
    elif kind == "gated_grad":
        pre = _normal(g, M, 2, h, dtype=bf)              # what the forward pass left
        st["pre"] = _to_eight(pre) if case["pre"] == "i8" else pre
    return st


def _prepare_rows(case, seed):
    r, g = _generators(seed)
    T, d, dt = case["T"], case["d"], DTYPE[case["dtype"]]
    x = _normal(g, T, d, dtype=torch.float32)
    x.mul_(torch.rand((T, 1), generator=g, device="cuda") * 2 + 0.5).add_(torch.randn((T, 1), generator=g, device="cuda"))
    x.mul_(torch.randn((1, d), generator=g, device="cuda").mul_(0.5).exp_())             # channels of different sizes
    if case["kind"] == "checkpoint8":
        return dict(x=x.to(dt), out=torch.empty((T, d), dtype=dt, device="cuda"), kept=_eight(T, d))
    mean = x.mean(1)
    rstd = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt()
    return dict(kept=_to_eight(x), mean=mean, rstd=rstd, gamma=_normal(g, d, dtype=torch.float32, std=0.2).add_(1), dy=_normal(g, T, d, dtype=dt, std=0.1),
                out=torch.empty((T, d), dtype=dt, device="cuda"))


def prepare(case, seed):
    return dict((_prepare_rows if case["kind"] in ("checkpoint8", "norm_grad8") else _prepare_layer)(case, seed), kind=case["kind"])


# ------------------------------------------------------------------------------------------ plain forms
def _blocks(x):
    """x with its last axis in blocks, zeros behind its end."""
    d = x.shape[-1]
    pad = torch.zeros((*x.shape[:-1], -d % BLOCK), dtype=x.dtype, device=x.device)
    return torch.cat([x, pad], -1).unflatten(-1, (-1, BLOCK))


def _to_eight(x):
    b = _blocks(x.float())
    largest = b.abs().amax(-1)
    up = ((largest / torch.full_like(largest, 127.0)).view(torch.int32) + 0xffff) & -0x10000
    s = torch.where(torch.isfinite(largest), up.view(torch.float32).clamp(min=2.0 ** -126), math.nan)
    q = torch.where(torch.isfinite(largest)[..., None], (b * (1.0 / s)[..., None]).round(), 0.0)
    return dict(q=q.to(torch.int8).flatten(-2)[..., :x.shape[-1]].contiguous(), scale=s.to(torch.bfloat16))


def _from_eight(kept):
    return (_blocks(kept["q"].float()) * kept["scale"].float()[..., None]).flatten(-2)[..., :kept["q"].shape[-1]]


def _groups(counts):
    at = 0
    for e, n in enumerate(counts):
        if n:
            yield e, slice(at, at + n)
        at += n


def _sigma(st, g):
    """The gate's sigma and the derivative of its argument."""
    if st["act"] == "silu":
        return torch.sigmoid(g), 1.0
    a = 2.0 * math.sqrt(2.0 / math.pi)
    return torch.sigmoid(a * (g + 0.044715 * g * g * g)), a * (1.0 + 3 * 0.044715 * g * g)


def _plain_forward(st, pre):
    """out, and gate and up into `pre`, which has fp32 or another type."""
    hidden, h = torch.zeros_like(st["hidden"]), st["h"]
    for e, rows in _groups(st["counts"]):
        y = st["x"][st["perm"][rows].long() // st["k"]].float() @ st["W1"][e].view(2 * h, -1).float().t()
        g, u = y[:, :h], y[:, h:]
        hidden[rows] = (g * _sigma(st, g)[0] * u).to(hidden.dtype)
        if pre is not None:
            pre[rows] = y.view(-1, 2, h).to(pre.dtype)
    return hidden


def _plain_backward(st, pre):
    """Gradients of gate and up, and the hidden rows again, from gate and up in fp32."""
    hidden, dpre = torch.zeros_like(st["hidden"]), torch.zeros_like(st["dpre"])
    for e, rows in _groups(st["counts"]):
        dact = st["dout"][rows].float() @ st["W2"][e].float()
        g, u = pre[rows, 0], pre[rows, 1]
        s, slope = _sigma(st, g)
        dpre[rows, 0] = (dact * u * (s + g * s * (1.0 - s) * slope)).to(dpre.dtype)
        dpre[rows, 1] = (dact * g * s).to(dpre.dtype)
        hidden[rows] = (g * s * u).to(hidden.dtype)
    return dpre, hidden


def _plain_gated(st):
    if "pre" not in st:
        return _plain_forward(st, None)
    pre = torch.zeros_like(st["pre"])
    return _plain_forward(st, pre), pre


def _plain_gated_grad(st):
    return _plain_backward(st, _from_eight(st["pre"]) if isinstance(st["pre"], dict) else st["pre"].float())


def _plain_gated_step8(st):
    pre = torch.zeros((st["M"], 2, st["h"]), dtype=torch.float32, device="cuda")
    hidden = _plain_forward(st, pre)
    return (hidden, *_plain_backward(st, _from_eight(_to_eight(pre))))


def _plain_checkpoint8(st):
    return _from_eight(_to_eight(st["x"])).to(st["x"].dtype)


def _plain_norm_grad8(st):
    dy = st["dy"].float()
    xhat = (_from_eight(st["kept"]) - st["mean"][:, None]) * st["rstd"][:, None]
    g = dy * st["gamma"]
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * st["rstd"][:, None]
    return dx.to(st["dy"].dtype), (dy * xhat).sum(0), dy.sum(0)


PLAIN = dict(gated=_plain_gated, gated_grad=_plain_gated_grad, gated_step8=_plain_gated_step8, checkpoint8=_plain_checkpoint8, norm_grad8=_plain_norm_grad8)


# ------------------------------------------------------------------------------------------ the framework's
def _own(st):
    import paper_1707_02402_amd as dyn
    kind = st["kind"]
    rows8 = lambda kept: dyn.Rows8(kept["q"], kept["scale"])
    if kind == "checkpoint8":
        return dyn.dynb_load8(dyn.dynb_store8(st["x"], out=rows8(st["kept"])), out=st["out"])
    if kind == "norm_grad8":
        return dyn.dynb_layer_norm_backward(st["dy"], rows8(st["kept"]), st["gamma"], st["mean"], st["rstd"], dx=st["out"])
    gate = dyn.MOE_GATE_SILU if st["act"] == "silu" else dyn.MOE_GATE_GELU
    pre = rows8(st["pre"]) if isinstance(st.get("pre"), dict) else st.get("pre")
    if kind == "gated_grad":
        return dyn.moe_gated_grad(st["dout"], st["W2"], st["offsets"], pre, gate=gate, dpre=st["dpre"], hidden=st["hidden"])
    hidden = dyn.moe_gated(st["x"], st["W1"], st["offsets"], perm=st["perm"], k=st["k"], gate=gate, out=st["hidden"], pre=pre)
    if kind == "gated":
        return hidden if pre is None else (hidden, pre)
    return (hidden, *dyn.moe_gated_grad(st["dout"], st["W2"], st["offsets"], pre, gate=gate, dpre=st["dpre"], hidden=st["again"]))


def run(state):
    return _own(state) if own else PLAIN[state["kind"]](state)


# ------------------------------------------------------------------------------------------ in 64 bits
def _f32(x):
    """x, rounded as fp32 arithmetic rounds."""
    return x.to(torch.float32).to(torch.float64)


def _restored(x):
    """What rows x come back as from 8 bits, block after block; the two fp32 steps of the definition are rounded to 24 bits."""
    x, out = x.to(torch.float64), torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[-1], BLOCK):
        v = x[..., c:c + BLOCK]
        ratio = _f32(v.abs().max(-1, keepdim=True).values / 127.0)
        _, power = torch.frexp(ratio)                    # ratio = m * 2 ** power, m in [1/2, 1): eight bits of m, rounded up
        unit = torch.ldexp(torch.ones_like(ratio), power - 8)
        s = torch.ceil(ratio / unit) * unit
        s = torch.where(s < 2.0 ** -126, torch.full_like(s, 2.0 ** -126), s)
        out[..., c:c + BLOCK] = torch.round(_f32(v * _f32(torch.reciprocal(s)))) * s
    return out


def _values(kept):
    """Rows in 8 bits as the values they stand for."""
    s = kept["scale"].to(torch.float64).repeat_interleave(BLOCK, -1)
    return kept["q"].to(torch.float64) * s[..., :kept["q"].shape[-1]]


def _gate64(act, g):
    """f and f', from tanh."""
    if act == "silu":
        t = torch.tanh(0.5 * g)
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.25 * g * (1 - t * t)
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g ** 2)


def exact(case, seed):
    st, kind, f8 = prepare(case, seed), case["kind"], torch.float64
    if kind == "checkpoint8":
        return _restored(st["x"])
    if kind == "norm_grad8":
        d = case["d"]
        x, dy, rstd = _values(st["kept"]), st["dy"].to(f8), st["rstd"].to(f8)[:, None]
        h = (x - st["mean"].to(f8)[:, None]) * rstd
        p = torch.stack([dy @ st["gamma"].to(f8), (dy * h) @ st["gamma"].to(f8)], 1) / d
        dx = rstd * (dy * st["gamma"].to(f8) - p[:, :1] - h * p[:, 1:])
        return dx, torch.einsum("td,td->d", dy, h), torch.ones(len(x), dtype=f8, device="cuda") @ dy
    at, M, h = st["offsets"].cpu().tolist(), st["M"], st["h"]
    hidden, again = (torch.zeros((M, h), dtype=f8, device="cuda") for _ in range(2))
    pre, dpre = (torch.zeros((M, 2, h), dtype=f8, device="cuda") for _ in range(2))
    for e in range(case["E"]):
        lo, hi = at[e], at[e + 1]
        if lo == hi:
            continue
        if kind == "gated_grad":
            p = st["pre"]
            p = _values({n: t[lo:hi] for n, t in p.items()}) if isinstance(p, dict) else p[lo:hi].to(f8)
        else:
            x = st["x"].index_select(0, torch.div(st["perm"][lo:hi], st["k"], rounding_mode="floor")).to(f8)
            p = torch.stack([x @ st["W1"][e, 0].to(f8).t(), x @ st["W1"][e, 1].to(f8).t()], 1)
            hidden[lo:hi] = _gate64(case["act"], p[:, 0])[0] * p[:, 1]
            pre[lo:hi] = p
            if kind == "gated":
                continue
            p = _restored(p)
        f, slope = _gate64(case["act"], p[:, 0])
        dact = st["dout"][lo:hi].to(f8) @ st["W2"][e].to(f8)
        dpre[lo:hi] = torch.stack([dact * p[:, 1] * slope, dact * f], 1)
        again[lo:hi] = f * p[:, 1]
    if kind == "gated":
        return (hidden, pre) if case["keep"] else hidden
    return (dpre, again) if kind == "gated_grad" else (hidden, dpre, again)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def _expected_distinct(n, s, draws):
    """How many of n ids turn up in so many draws by Zipf's law."""
    p = np.arange(1, n + 1, dtype=np.float64) ** -s
    return float(-np.expm1(draws * np.log1p(-np.minimum(p / p.sum(), 1 - 1e-12))).sum())


def work(case):
    kind = case["kind"]
    if kind in ("checkpoint8", "norm_grad8"):
        T, d, e = case["T"], case["d"], 2 if case["dtype"] == "bf16" else 4
        eight = T * d + T * ((d + BLOCK - 1) // BLOCK) * 2
        if kind == "checkpoint8":
            return dict(bytes=2 * T * d * e + 2 * eight, flops=4 * T * d)
        return dict(bytes=2 * T * d * e + eight + 8 * T + 12 * d, flops=15 * T * d)
    T, k, h, E = (case[x] for x in ("T", "k", "h", "E"))
    M, K, N = T * k, case.get("K", 0), case.get("N", 0)
    live = max(1, E - int(round(E * case["empty"])))
    used = int(round(_expected_distinct(live, case["zipf"], M)))
    blocks = (h + BLOCK - 1) // BLOCK
    wide, eight = 4 * M * h, 2 * M * h + 4 * M * blocks          # gate and up in bfloat16, in 8 bits
    nbytes, flops = 4 * E, 0
    if kind != "gated_grad":
        nbytes += 2 * T * K + 4 * M + 2 * M * h + 4 * used * h * K + (wide if case.get("keep") else eight if kind == "gated_step8" else 0)
        flops += 4 * M * h * K + 8 * M * h
    if kind != "gated":
        nbytes += 2 * M * N + (eight if kind == "gated_step8" or case["pre"] == "i8" else wide) + wide + 2 * M * h + 2 * used * N * h
        flops += 2 * M * N * h + 16 * M * h
    return dict(bytes=nbytes, flops=flops)
