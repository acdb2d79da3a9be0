"""Whose memory the binding allocates.  torch hands out blocks that earlier work of the stream they are handed out on may still be using: what another
stream is to write first has to be that stream's.  Shown on the CPU with streams that only keep a list; on the GPU for the calls themselves."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_1707_02402_amd import binding


class Block:
    def __init__(self, owner):
        self.owner, self.users = owner, []

    def record_stream(self, stream):
        self.users.append(stream)


@pytest.fixture
def streams(monkeypatch):
    active = ["current"]

    @contextlib.contextmanager
    def switch(stream):
        active.append(stream)
        yield
        active.pop()

    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: active[-1])
    monkeypatch.setattr(torch.cuda, "stream", switch)
    monkeypatch.setattr(torch, "empty", lambda *_, **__: Block(active[-1]))
    monkeypatch.setattr(torch, "empty_like", lambda *_, **__: Block(active[-1]))
    return active


def test_memory_belongs_to_the_stream_of_the_work(streams):
    like = SimpleNamespace(dtype=torch.float32, device="cuda")
    for make in (lambda s: binding._scratch(100, "cuda", s), lambda s: binding._new(s, 3, 4, like=like), lambda s: binding._twin(s, None)):
        block = make("side")
        assert block.owner == "side" and block.users == ["current"]
        for same in (None, "current"):
            block = make(same)
            assert block.owner == "current" and block.users == []
    assert streams == ["current"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["dynb_embed", "dynb_embed_backward", "dynb_layer_norm", "dynb_layer_norm_backward", "moe_product", "moe_product_grad_input", "moe_product_grad_weight", "dynb_clip_gradients"])
def test_a_block_in_use_on_the_current_stream_is_not_written_from_another(name):
    """Blocks of every size that a call may ask for are given up while a long queue of fills still writes them: the call's results on another stream are
    the same all the same, when all is done."""
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as dyn
    g = torch.Generator("cuda").manual_seed(1)
    T, d, V = 4096, 256, 512
    bf = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)
    x, dy, table, W, tokens = bf(T, d), bf(T, d), bf(V, d), bf(4, d, d), torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    gamma, off = torch.ones(d, device="cuda"), torch.tensor([0, 1000, 1000, 3000, T], dtype=torch.int32, device="cuda")
    _, mean, rstd = dyn.dynb_layer_norm(x, gamma, want_stats=True)
    grads = [torch.randn(100_000, generator=g, device="cuda")]
    listed = dyn.GradTensors(grads, [torch.empty_like(grads[0])])
    calls = dict(dynb_embed=lambda s: dyn.dynb_embed(tokens, table, stream=s), dynb_embed_backward=lambda s: dyn.dynb_embed_backward(tokens, dy, V, stream=s),
                 dynb_layer_norm=lambda s: dyn.dynb_layer_norm(x, gamma, want_stats=True, stream=s),
                 dynb_layer_norm_backward=lambda s: dyn.dynb_layer_norm_backward(dy, x, gamma, mean, rstd, stream=s),
                 moe_product=lambda s: dyn.moe_product(x, W, off, stream=s), moe_product_grad_input=lambda s: dyn.moe_product_grad_input(dy, W, off, stream=s),
                 moe_product_grad_weight=lambda s: dyn.moe_product_grad_weight(dy, x, off, stream=s),
                 dynb_clip_gradients=lambda s: dyn.dynb_clip_gradients(listed, 1.0, stream=s))
    tensors = lambda r: list(r) if isinstance(r, tuple) else [r]
    want = [t.clone() for t in tensors(calls[name](None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (512, 512, 1024, 1024, 16384, 16384, 65536, 1 << 18, 1 << 19, 1 << 20, 1 << 21, 1 << 21, 1 << 22)]
    for _ in range(40):
        for t in busy:
            t.fill_(0x55)
    del busy, t
    got = tensors(calls[name](side))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
