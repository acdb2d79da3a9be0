"""dynb_clip_gradients against norms in 64 bits.  The squares are added up in fp64 (sums of 10^7 of them are off by 10^-9), so the norm is off by
its one rounding to fp32 and the factor by two more; what is stored in bfloat16 by 2^-8 of itself."""
import pytest
import torch

from tests.operator_util import U16, U32

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def check(dyn, grads, max_norm, into):
    want = torch.cat([t.double().cpu().reshape(-1) for t in grads] + [torch.zeros(0, dtype=torch.float64)])
    norm = float(want.square().sum().sqrt())
    factor = max_norm / norm if norm > max_norm else 1.0
    kept = [t.clone() for t in grads]
    if into == "place":
        got_norm, out = dyn.dynb_clip_gradients(grads, max_norm), grads
    else:
        out = [torch.full_like(t, float("nan")) for t in grads]
        got_norm = dyn.dynb_clip_gradients(dyn.GradTensors(grads, out), max_norm)
        assert all(torch.equal(a, b) for a, b in zip(kept, grads))
    assert abs(float(got_norm) - norm) <= 4 * U32 * norm
    for o, t in zip(out, kept):
        ref = t.double().cpu() * factor
        u = U16 if t.dtype == torch.bfloat16 else U32
        assert ((o.double().cpu() - ref).abs() <= (u + 8 * U32) * ref.abs() + 1e-38).all()
        if factor == 1.0:
            assert torch.equal(o, t)


@pytest.mark.parametrize("sizes", [[1], [3], [5, 1, 8], [1000], [4096, 4097, 7], [0, 12, 0], [100_003, 1, 64, 65, 2_000_001], [17] * 700, [1 << 20] * 3])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("into", ["place", "others"])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_norm_and_factor(dyn, sizes, dtype, into, max_norm):
    g = torch.Generator().manual_seed(len(sizes) + sum(sizes))
    kinds = [DT[dtype] if dtype != "mixed" else (DT["f32"] if i % 2 else DT["bf16"]) for i in range(len(sizes))]
    check(dyn, [torch.randn(n, generator=g).to(k).cuda() for n, k in zip(sizes, kinds)], max_norm, into)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tensors_between_borders(dyn, dtype):
    """Starts that are no multiple of 16 bytes, the same for gradient and result or not."""
    g = torch.Generator().manual_seed(2)
    for a, b in ((1, 1), (1, 3), (0, 5), (7, 0)):
        grad = torch.randn(10_000 + a, generator=g).to(DT[dtype]).cuda()[a:]
        buf = torch.full((10_020,), 7.0, dtype=DT[dtype], device="cuda")
        out = buf[b:b + grad.numel()]
        norm = float(dyn.dynb_clip_gradients(dyn.GradTensors([grad], [out]), 1.0))
        ref = grad.double() / norm
        assert ((out.double() - ref).abs() <= ((U16 if dtype == "bf16" else U32) + 8 * U32) * ref.abs()).all()
        assert (buf[:b] == 7).all() and (buf[b + grad.numel():] == 7).all()


def test_values_whose_squares_leave_fp32(dyn):
    for v in (1e25, 1e-30):
        t = torch.full((1000,), v, device="cuda")
        assert abs(float(dyn.dynb_clip_gradients([t], 1e-35 if v < 1 else 1.0)) / (float(torch.tensor(v)) * 1000 ** 0.5) - 1) < 1e-6
        assert torch.isfinite(t).all() and (t > 0).all()
        assert abs(float(t.double().square().sum().sqrt()) / (1e-35 if v < 1 else 1.0) - 1) < 1e-5


def test_norms_that_are_not_finite_leave_the_gradients(dyn):
    for bad in (float("inf"), float("nan")):
        t = [torch.ones(5000, device="cuda"), torch.ones(100, dtype=torch.bfloat16, device="cuda")]
        t[0][4321] = bad
        kept = [x.clone() for x in t]
        norm = float(dyn.dynb_clip_gradients(t, 1.0))
        assert norm != norm or norm == float("inf")
        assert all(torch.equal(torch.nan_to_num(a, nan=-3), torch.nan_to_num(b, nan=-3)) for a, b in zip(t, kept))


def test_no_tensors(dyn):
    assert float(dyn.dynb_clip_gradients([], 1.0)) == 0.0
    assert float(dyn.dynb_clip_gradients([torch.empty(0, device="cuda")], 1.0)) == 0.0


def test_norm_only(dyn):
    from paper_1707_02402_amd import binding as b
    t = torch.full((10_000,), 3.0, device="cuda")
    arr = (b._GradTensor * 1)((t.data_ptr(), None, t.numel(), 0))
    norm, ws = torch.empty((), device="cuda"), torch.empty(dyn.dynb_clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
    b._check(b.lib.dynb_clip_gradients(arr, 1, 1.0, norm.data_ptr(), ws.data_ptr(), ws.numel(), b._stream()))
    assert float(norm) == 300.0 and (t == 3).all()


def test_the_same_bits_on_other_streams_and_in_graphs(dyn):
    g = torch.Generator().manual_seed(6)
    grads = [torch.randn(n, generator=g).cuda() for n in (1_000_000, 77, 30_001)]
    out = [torch.empty_like(t) for t in grads]
    listed, norm = dyn.GradTensors(grads, out), torch.empty((), device="cuda")
    ws = torch.empty(dyn.dynb_clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
    dyn.dynb_clip_gradients(listed, 1.0, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    ref = [t.clone() for t in out] + [norm.clone()]
    side = torch.cuda.Stream()
    dyn.dynb_clip_gradients(listed, 1.0, norm=norm, workspace=ws, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, out + [norm]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dyn.dynb_clip_gradients(listed, 1.0, norm=norm, workspace=ws)
    for _ in range(3):
        for t in out:
            t.fill_(1)
        norm.fill_(1), ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, out + [norm]))
