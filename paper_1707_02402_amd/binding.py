"""ctypes binding of libdynbatch.so: same names as the C ABI, argument marshalling only.

PyTorch tensors provide device memory and the current HIP stream; every step of the two hot
paths runs inside the library's kernels.  There is no fallback: if the library has not been
built, importing this module raises.
"""
from __future__ import annotations

import ctypes as ct
import os
from types import SimpleNamespace
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdynbatch.so")

DYNB_F32, DYNB_BF16, DYNB_I8 = 0, 1, 2
DYNB_SCHED_IMPROVED, DYNB_SCHED_STANDARD, DYNB_SCHED_NAIVE, DYNB_SCHED_DEPTH = 0, 1, 2, 3
DYNB_PLAN_THROUGHPUT = 8
DYNB_PLAN_BALANCE = 4
DYNB_PLAN_PERSISTENT = 16
DYNB_PLAN_KEEP = 32
ERRORS = {-1: "DYNB_E_INVAL", -2: "DYNB_E_MALFORMED", -3: "DYNB_E_NOMEM", -4: "DYNB_E_WORKSPACE",
          -5: "DYNB_E_UNSUPPORTED", -6: "DYNB_E_HIP"}

EXPORTS = ["dynb_last_error", "dynbatch_plan", "dynbatch_plan_dag", "dynbatch_plan_view", "dynbatch_plan_free",
           "dynbatch_plan_device_bytes", "dynbatch_plan_upload", "dynbatch_workspace_bytes",
           "dynbatch_packed_weights_bytes", "dynbatch_pack_weights",
           "dynbatch_classify_workspace_bytes", "dynbatch_classify", "dynbatch_backward_workspace_bytes", "dynbatch_backward",
           "dynbatch_execute", "dynbatch_execute_check", "dynb_set_spin_limit", "moe_workspace_bytes", "moe_forward", "moe_forward_static", "moe_forward_naive",
           "moe_product", "moe_product_grad_input", "moe_product_grad_weight_workspace_bytes", "moe_product_grad_weight",
           "dynb_embed", "dynb_embed_backward_workspace_bytes", "dynb_embed_backward",
           "dynb_layer_norm", "dynb_layer_norm_backward_workspace_bytes", "dynb_layer_norm_backward",
           "dynb_clip_workspace_bytes", "dynb_clip_gradients",
           "moe_gated", "moe_gated_grad", "dynb_store8", "dynb_load8", "dynb_layer_norm_backward8",
           "dynb_timing_enable", "dynb_probe_mfma_bf16", "dynb_probe_copy", "dynb_probe_read",
           "dynb_timing_read"]


class DynbError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code
        self.name = ERRORS.get(code, str(code))


I32P = ct.POINTER(ct.c_int32)


class _PlanView(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("n_examples", "n_nodes", "n_levels", "n_buckets", "n_compute_nodes",
                                          "n_launches", "max_launch_nodes", "n_slots")] + \
               [(n, I32P) for n in ("node_level", "node_type", "child0", "child1", "root", "bucket_level",
                                    "bucket_type", "bucket_start", "bucket_count", "members", "in0", "in1", "out",
                                    "node_launch", "item_node")] + \
               [("n_tickets", ct.c_int32), ("tickets", I32P)] + \
               [(n, I32P) for n in ("grad_dst0", "grad_dst1", "fn_first", "fn_items")] + \
               [("n_types", ct.c_int32), ("n_wg_units", ct.c_int32), ("wg_units", I32P), ("wg_order", I32P)]


class _Shape(ct.Structure):
    _fields_ = [("C", ct.c_int32), ("H", ct.c_int32), ("W", ct.c_int32), ("dtype", ct.c_int32)]


class _Weights(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("w1", "b1", "w3a", "b3a", "w3b", "b3b", "packed")]


class _Grads(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("dfeats", "dw1", "db1", "dw3a", "db3a", "dw3b", "db3b")]


class _HeadShape(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("C", "H", "W", "dtype", "Cc", "F", "n_answers")]


class _HeadWeights(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("wc", "bc", "wf1", "bf1", "wf2", "bf2")]


class _MoeShape(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("T", "d", "h", "E", "k", "dtype")] + [("flags", ct.c_uint32)]


class _StageTime(ct.Structure):
    _fields_ = [("tag", ct.c_int32), ("units", ct.c_int32), ("ms", ct.c_float)]


class _MoeAux(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("logits", "topk_idx", "topk_w", "counts", "offsets", "perm", "inv")]


class _ProductShape(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("M", "K", "N", "E", "dtype")] + [("flags", ct.c_uint32)]


class _Groups(ct.Structure):
    _fields_ = [("offsets", ct.c_void_p), ("perm", ct.c_void_p), ("k", ct.c_int32), ("rows", ct.c_int32)]


class _EmbedShape(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("T", "V", "d", "dtype")] + [("scale", ct.c_float)]


class _NormShape(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("T", "d", "dtype")] + [("eps", ct.c_float)]


class _Rows8(ct.Structure):
    _fields_ = [("q", ct.c_void_p), ("q_stride", ct.c_int64), ("scale", ct.c_void_p), ("scale_stride", ct.c_int64)]


class _Rows8Shape(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("T", "d", "dtype")]


class _GatedShape(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in ("M", "K", "h", "E", "dtype")] + [("flags", ct.c_uint32)]


class _GatedPre(ct.Structure):
    _fields_ = [("rows", ct.c_void_p), ("stride", ct.c_int64), ("scale", ct.c_void_p), ("scale_stride", ct.c_int64), ("dtype", ct.c_int32)]


class _GradTensor(ct.Structure):
    _fields_ = [("grad", ct.c_void_p), ("out", ct.c_void_p), ("count", ct.c_int64), ("dtype", ct.c_int32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    L = ct.CDLL(LIB_PATH)
    L.dynb_last_error.restype = ct.c_char_p
    L.dynbatch_plan.argtypes = [I32P, I32P, ct.c_int32, ct.POINTER(ct.c_uint8), ct.c_int32, ct.c_uint32,
                                ct.POINTER(ct.c_void_p)]
    L.dynbatch_plan_dag.argtypes = [I32P, I32P, I32P, I32P, I32P, ct.c_int32, ct.POINTER(ct.c_uint8), ct.c_int32, ct.c_uint32,
                                    ct.POINTER(ct.c_void_p)]
    L.dynbatch_plan_view.argtypes = [ct.c_void_p, ct.POINTER(_PlanView)]
    L.dynbatch_plan_free.argtypes = [ct.c_void_p]
    L.dynbatch_plan_free.restype = None
    L.dynbatch_plan_device_bytes.argtypes = [ct.c_void_p]
    L.dynbatch_plan_device_bytes.restype = ct.c_size_t
    L.dynbatch_plan_upload.argtypes = [ct.c_void_p, ct.c_void_p, ct.c_size_t, ct.c_void_p]
    L.dynbatch_workspace_bytes.argtypes = [ct.c_void_p, ct.POINTER(_Shape)]
    L.dynbatch_workspace_bytes.restype = ct.c_size_t
    L.dynbatch_execute.argtypes = [ct.c_void_p, ct.POINTER(_Shape), ct.POINTER(_Weights), ct.c_void_p, ct.c_void_p,
                                   ct.c_void_p, ct.c_size_t, ct.c_void_p]
    L.dynbatch_backward_workspace_bytes.argtypes = [ct.c_void_p, ct.POINTER(_Shape)]
    L.dynbatch_backward_workspace_bytes.restype = ct.c_size_t
    L.dynbatch_backward.argtypes = [ct.c_void_p, ct.POINTER(_Shape), ct.POINTER(_Weights), ct.c_void_p, ct.c_void_p, ct.c_void_p,
                                    ct.c_void_p, ct.POINTER(_Grads), ct.c_void_p, ct.c_size_t, ct.c_void_p]
    L.dynbatch_classify_workspace_bytes.argtypes = [ct.POINTER(_HeadShape), ct.c_int32]
    L.dynbatch_classify_workspace_bytes.restype = ct.c_size_t
    L.dynbatch_classify.argtypes = [ct.POINTER(_HeadShape), ct.POINTER(_HeadWeights), ct.c_void_p, ct.c_int32, ct.c_void_p,
                                    ct.c_void_p, ct.c_void_p, ct.c_size_t, ct.c_void_p]
    L.dynbatch_execute_check.argtypes = [ct.c_void_p, ct.POINTER(_Shape), ct.c_void_p, ct.c_void_p]
    L.dynb_set_spin_limit.argtypes = [ct.c_int32]
    L.dynb_set_spin_limit.restype = ct.c_int32
    L.dynbatch_packed_weights_bytes.argtypes = [ct.POINTER(_Shape), ct.c_int32]
    L.dynbatch_packed_weights_bytes.restype = ct.c_size_t
    L.dynbatch_pack_weights.argtypes = [ct.POINTER(_Shape), ct.c_int32, ct.POINTER(_Weights), ct.c_void_p, ct.c_size_t,
                                        ct.c_void_p]
    L.moe_workspace_bytes.argtypes = [ct.POINTER(_MoeShape)]
    L.moe_workspace_bytes.restype = ct.c_size_t
    L.moe_forward.argtypes = [ct.POINTER(_MoeShape), ct.c_void_p, ct.c_void_p, ct.c_void_p, ct.c_void_p, ct.c_void_p,
                              ct.c_void_p, ct.c_void_p, ct.POINTER(_MoeAux), ct.c_void_p, ct.c_size_t, ct.c_void_p]
    L.moe_forward_naive.argtypes = L.moe_forward.argtypes + [ct.c_int32]
    L.moe_forward_static.argtypes = L.moe_forward.argtypes[:9] + [ct.c_void_p]
    VP, I64, SZ = ct.c_void_p, ct.c_int64, ct.c_size_t
    PS, GR, ES, NS = (ct.POINTER(t) for t in (_ProductShape, _Groups, _EmbedShape, _NormShape))
    L.moe_product.argtypes = [PS, GR, VP, I64, VP, VP, I64, VP]
    L.moe_product_grad_input.argtypes = [PS, GR, VP, I64, VP, VP, I64, VP, I64, VP]
    L.moe_product_grad_weight_workspace_bytes.argtypes = [PS]
    L.moe_product_grad_weight_workspace_bytes.restype = SZ
    L.moe_product_grad_weight.argtypes = [PS, GR, VP, I64, VP, I64, VP, ct.c_int32, VP, SZ, VP]
    L.dynb_embed.argtypes = [ES, VP, VP, VP, I64, VP]
    L.dynb_embed_backward_workspace_bytes.argtypes = [ES]
    L.dynb_embed_backward_workspace_bytes.restype = SZ
    L.dynb_embed_backward.argtypes = [ES, VP, VP, I64, VP, ct.c_int32, VP, SZ, VP]
    L.dynb_layer_norm.argtypes = [NS, VP, I64, VP, VP, VP, I64, VP, VP, VP]
    L.dynb_layer_norm_backward_workspace_bytes.argtypes = [NS]
    L.dynb_layer_norm_backward_workspace_bytes.restype = SZ
    L.dynb_layer_norm_backward.argtypes = [NS, VP, I64, VP, I64, VP, VP, VP, VP, I64, VP, VP, VP, SZ, VP]
    R8, R8S, GS, GP = (ct.POINTER(t) for t in (_Rows8, _Rows8Shape, _GatedShape, _GatedPre))
    L.dynb_layer_norm_backward8.argtypes = [NS, VP, I64, R8, VP, VP, VP, VP, I64, VP, VP, VP, SZ, VP]
    L.dynb_store8.argtypes = [R8S, VP, I64, R8, VP]
    L.dynb_load8.argtypes = [R8S, R8, VP, I64, VP]
    L.moe_gated.argtypes = [GS, GR, VP, I64, VP, VP, I64, GP, VP]
    L.moe_gated_grad.argtypes = [GS, GR, VP, I64, VP, GP, VP, I64, VP, I64, VP]
    L.dynb_clip_workspace_bytes.argtypes = []
    L.dynb_clip_workspace_bytes.restype = SZ
    L.dynb_clip_gradients.argtypes = [ct.POINTER(_GradTensor), ct.c_int32, ct.c_float, VP, VP, SZ, VP]
    L.dynb_probe_mfma_bf16.argtypes = [ct.c_int32, ct.c_int32, ct.c_void_p, ct.c_void_p, ct.POINTER(ct.c_double)]
    L.dynb_probe_copy.argtypes = [ct.c_void_p, ct.c_void_p, ct.c_size_t, ct.c_void_p]
    L.dynb_probe_read.argtypes = [ct.c_void_p, ct.c_size_t, ct.c_void_p, ct.c_void_p]
    L.dynb_timing_enable.argtypes = [ct.c_int]
    L.dynb_timing_read.argtypes = [ct.POINTER(_StageTime), ct.c_int32, ct.POINTER(ct.c_int32)]
    return L


lib = _load()


def _check(rc: int):
    if rc:
        raise DynbError(rc, lib.dynb_last_error().decode())


def _stream(stream=None):
    if stream is not None:
        return ct.c_void_p(stream.cuda_stream)
    import torch
    try:                                         # current_stream() builds an object: 2.6 us, more than the smallest kernels take
        c = torch._C
        return ct.c_void_p(c._cuda_getCurrentRawStream(c._cuda_getDevice()))
    except AttributeError:                       # neither is torch's public interface: a torch without them is asked the slower way
        return ct.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t):
    return None if t is None else ct.c_void_p(t.data_ptr())


def _made(stream, make):
    """make() for work on `stream` (None: the current one).  Memory that torch hands out may still be in use by earlier work of the
    stream it is handed out on, so it has to be the stream that the work runs on; the current one, where the caller goes on with a
    result, is made known, so that the block is not handed out again ahead of the work there."""
    if stream is None:
        return make()
    import torch
    current = torch.cuda.current_stream()
    if stream == current:
        return make()
    with torch.cuda.stream(stream):
        made = make()
    for t in made if isinstance(made, (tuple, list)) else (made,):
        t.record_stream(current)
    return made


def _scratch(nbytes: int, device, stream):
    """Device buffer the binding allocates on the caller's behalf."""
    import torch
    if stream is None:                           # (the usual case, without the detour)
        return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)
    return _made(stream, lambda: torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device))


# ------------------------------------------------------------------------------------------ planner
class Plan:
    """Owner of a dynb_plan*; keeps the uploaded index-list buffer alive."""

    def __init__(self, handle, B):
        self.handle = handle
        self.B = B
        self.dev_buf = None
        self._free = lib.dynbatch_plan_free      # kept here: module globals may be gone at interpreter shutdown

    def free(self):
        h, self.handle = getattr(self, "handle", None), None
        if h:
            self._free(h)

    def __del__(self):
        try:
            self.free()
        except Exception:                        # nothing useful can be done in a finalizer
            pass


def dynbatch_plan(prog, prog_off, arity, flags: int = DYNB_SCHED_IMPROVED) -> Plan:
    prog = np.ascontiguousarray(prog, dtype=np.int32)
    prog_off = np.ascontiguousarray(prog_off, dtype=np.int32)
    arity = np.ascontiguousarray(arity, dtype=np.uint8)
    h = ct.c_void_p()
    if len(prog) == 0:
        prog = np.zeros(1, np.int32)      # keep the pointer non-NULL; lengths come from prog_off
    _check(lib.dynbatch_plan(prog.ctypes.data_as(I32P), prog_off.ctypes.data_as(I32P), len(prog_off) - 1,
                             arity.ctypes.data_as(ct.POINTER(ct.c_uint8)), len(arity), flags, ct.byref(h)))
    return Plan(h, len(prog_off) - 1)


def dynbatch_plan_dag(node_type, arg0, arg1, node_off, root, arity, flags: int = DYNB_SCHED_IMPROVED) -> Plan:
    """Plan of a batch of dependency graphs (argument indices local to each example, -1 = none)."""
    a = [np.ascontiguousarray(v, dtype=np.int32) for v in (node_type, arg0, arg1, node_off, root)]
    arity = np.ascontiguousarray(arity, dtype=np.uint8)
    for i in range(3):
        if len(a[i]) == 0:
            a[i] = np.zeros(1, np.int32)  # keep the pointers non-NULL; lengths come from node_off
    h = ct.c_void_p()
    B = len(a[3]) - 1
    if len(a[4]) != B:
        raise ValueError("root must have one entry per example")
    _check(lib.dynbatch_plan_dag(*[v.ctypes.data_as(I32P) for v in a], B,
                                 arity.ctypes.data_as(ct.POINTER(ct.c_uint8)), len(arity), flags, ct.byref(h)))
    return Plan(h, B)


def dynbatch_plan_view(plan: Plan) -> SimpleNamespace:
    v = _PlanView()
    _check(lib.dynbatch_plan_view(plan.handle, ct.byref(v)))

    def arr(p, n):
        return np.ctypeslib.as_array(p, shape=(n,)).copy() if n > 0 else np.zeros(0, np.int32)

    N, nb, B = v.n_nodes, v.n_buckets, v.n_examples
    return SimpleNamespace(
        n_examples=B, n_nodes=N, n_levels=v.n_levels, n_buckets=nb, n_compute_nodes=v.n_compute_nodes,
        n_launches=v.n_launches, max_launch_nodes=v.max_launch_nodes, n_slots=v.n_slots,
        node_level=arr(v.node_level, N), node_type=arr(v.node_type, N), child0=arr(v.child0, N),
        child1=arr(v.child1, N), root=arr(v.root, B), bucket_level=arr(v.bucket_level, nb),
        bucket_type=arr(v.bucket_type, nb), bucket_start=arr(v.bucket_start, nb),
        bucket_count=arr(v.bucket_count, nb), members=arr(v.members, N), in0=arr(v.in0, N), in1=arr(v.in1, N),
        out=arr(v.out, N), node_launch=arr(v.node_launch, N), item_node=arr(v.item_node, v.n_compute_nodes),
        n_tickets=v.n_tickets, tickets=arr(v.tickets, v.n_tickets),
        grad_dst0=arr(v.grad_dst0, v.n_compute_nodes if v.grad_dst0 else 0),
        grad_dst1=arr(v.grad_dst1, v.n_compute_nodes if v.grad_dst1 else 0),
        fn_first=arr(v.fn_first, v.n_types + 1 if v.fn_first else 0),
        fn_items=arr(v.fn_items, v.n_compute_nodes if v.fn_items else 0),
        n_types=v.n_types, n_wg_units=v.n_wg_units,
        wg_units=arr(v.wg_units, 8 * v.n_wg_units if v.wg_units else 0).reshape(-1, 8),
        wg_order=arr(v.wg_order, v.n_wg_units if v.wg_order else 0))


def dynbatch_plan_device_bytes(plan: Plan) -> int:
    return int(lib.dynbatch_plan_device_bytes(plan.handle))


def dynbatch_plan_upload(plan: Plan, dev_buf=None, stream=None):
    import torch
    n = dynbatch_plan_device_bytes(plan)
    if dev_buf is None:
        dev_buf = _scratch(n, "cuda", stream)
    _check(lib.dynbatch_plan_upload(plan.handle, _ptr(dev_buf), dev_buf.numel() * dev_buf.element_size(), _stream(stream)))
    plan.dev_buf = dev_buf
    return dev_buf


# ------------------------------------------------------------------------------------------ executor
def _shape_of(feats) -> _Shape:
    import torch
    B, H, W, C = feats.shape
    if feats.dtype == torch.float32:
        dt = DYNB_F32
    elif feats.dtype == torch.bfloat16:
        dt = DYNB_BF16
    else:
        raise TypeError("feats must be float32 or bfloat16")
    return _Shape(C, H, W, dt)


def dynbatch_workspace_bytes(plan: Plan, C: int, H: int, W: int, dtype: int) -> int:
    return int(lib.dynbatch_workspace_bytes(plan.handle, ct.byref(_Shape(C, H, W, dtype))))


def _weights_struct(weights: dict) -> _Weights:
    return _Weights(*[(t.data_ptr() if t is not None else None) for t in
                      (weights.get(k) for k in ("w1", "b1", "w3a", "b3a", "w3b", "b3b", "packed"))])


def dynbatch_packed_weights_bytes(C: int, H: int, W: int, dtype: int, n_types: int) -> int:
    return int(lib.dynbatch_packed_weights_bytes(ct.byref(_Shape(C, H, W, dtype)), n_types))


def dynbatch_pack_weights(weights: dict, C: int, H: int, W: int, dtype: int, packed=None, stream=None):
    """One-time preparation: returns a device buffer to pass as weights["packed"]."""
    import torch
    n_types = int(weights["w3a"].shape[0])
    shape = _Shape(C, H, W, dtype)
    if packed is None:
        packed = _scratch(max(int(lib.dynbatch_packed_weights_bytes(ct.byref(shape), n_types)), 256), weights["w3a"].device, stream)
    w = _weights_struct({**weights, "packed": None})
    _check(lib.dynbatch_pack_weights(ct.byref(shape), n_types, ct.byref(w), _ptr(packed),
                                     packed.numel() * packed.element_size(), _stream(stream)))
    return packed


def dynbatch_execute(plan: Plan, weights: dict, feats, out=None, workspace=None, stream=None):
    """weights: dict with device tensors w1,b1,w3a,b3a,w3b,b3b (biases float32 or None; w1 may be None)
    and optionally packed (from dynbatch_pack_weights).
    feats: device [B,H,W,C] float32 or bfloat16, contiguous.  Returns out [B,H,W,C]."""
    import torch
    assert feats.is_cuda and feats.is_contiguous() and feats.shape[0] == plan.B
    shape = _shape_of(feats)
    for key in ("w1", "w3a", "w3b"):
        t = weights.get(key)
        assert t is None or (t.is_cuda and t.is_contiguous() and t.dtype == feats.dtype), key
    for key in ("b1", "b3a", "b3b"):
        t = weights.get(key)
        assert t is None or (t.is_cuda and t.is_contiguous() and t.dtype == torch.float32), key
    if out is None:
        out = _made(stream, lambda: torch.empty_like(feats))
    assert out.is_cuda and out.is_contiguous() and out.shape == feats.shape and out.dtype == feats.dtype
    if workspace is None:
        workspace = _scratch(lib.dynbatch_workspace_bytes(plan.handle, ct.byref(shape)), feats.device, stream)
    w = _weights_struct(weights)
    _check(lib.dynbatch_execute(plan.handle, ct.byref(shape), ct.byref(w), _ptr(feats), _ptr(out), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


def dynbatch_execute_check(plan: Plan, feats, workspace, stream=None) -> None:
    """After executing a DYNB_PLAN_PERSISTENT plan: waits for the stream and raises DynbError(DYNB_E_HIP) if a
    bounded wait of the dependency-driven kernel expired."""
    _check(lib.dynbatch_execute_check(plan.handle, ct.byref(_shape_of(feats)), _ptr(workspace), _stream(stream)))


def dynb_set_spin_limit(polls: int) -> int:
    return int(lib.dynb_set_spin_limit(int(polls)))


# ------------------------------------------------------------------------------------------ backward pass
def dynbatch_backward_workspace_bytes(plan: Plan, C: int, H: int, W: int, dtype: int) -> int:
    return int(lib.dynbatch_backward_workspace_bytes(plan.handle, ct.byref(_Shape(C, H, W, dtype))))


def dynbatch_backward(plan: Plan, weights: dict, feats, out, forward_workspace, dout, workspace=None, stream=None, grads=None) -> dict:
    """Backward pass of an executed DYNB_PLAN_KEEP plan.  dout: device float32 [B,H,W,C].  Returns a dict of device
    float32 tensors dfeats, dw1, db1, dw3a, db3a, dw3b, db3b in the shapes of feats and of the weights (`grads`: such
    a dict from an earlier call, to be overwritten)."""
    import torch
    shape = _shape_of(feats)
    assert dout.is_cuda and dout.is_contiguous() and dout.dtype == torch.float32 and dout.shape == feats.shape
    f32 = lambda *shape: _made(stream, lambda: torch.empty(shape, dtype=torch.float32, device=feats.device))
    C = shape.C
    n_types = weights["w3a"].shape[0]
    g = grads if grads is not None else dict(
        dfeats=f32(*feats.shape), dw3a=f32(*weights["w3a"].shape), dw3b=f32(*weights["w3b"].shape), db3a=f32(n_types, C),
        db3b=f32(n_types, C), dw1=f32(n_types, C, 2 * C), db1=f32(n_types, C))
    for k in ("dfeats", "dw1", "db1", "dw3a", "db3a", "dw3b", "db3b"):
        assert g[k].is_cuda and g[k].is_contiguous() and g[k].dtype == torch.float32
    if workspace is None:
        n = int(lib.dynbatch_backward_workspace_bytes(plan.handle, ct.byref(shape)))
        if n == 0:
            _check(lib.dynbatch_backward(plan.handle, ct.byref(shape), None, None, None, None, None, None, None, 0, None))
        workspace = _scratch(n, feats.device, stream)
    gs = _Grads(*[g[k].data_ptr() for k in ("dfeats", "dw1", "db1", "dw3a", "db3a", "dw3b", "db3b")])
    w = _weights_struct(weights)
    _check(lib.dynbatch_backward(plan.handle, ct.byref(shape), ct.byref(w), _ptr(feats), _ptr(out), _ptr(forward_workspace),
                                 _ptr(dout), ct.byref(gs), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                 _stream(stream)))
    return g


# ------------------------------------------------------------------------------------------ classifier head
def _head_shape(roots, head: dict) -> _HeadShape:
    import torch
    B, H, W, C = roots.shape
    dt = DYNB_F32 if roots.dtype == torch.float32 else DYNB_BF16
    Cc, F, A = head["wc"].shape[0], head["wf1"].shape[0], head["wf2"].shape[0]
    assert head["wc"].shape == (Cc, C) and head["wf1"].shape == (F, H * W * Cc) and head["wf2"].shape == (A, F)
    return _HeadShape(C, H, W, dt, Cc, F, A)


def dynbatch_classify_workspace_bytes(C, H, W, dtype, Cc, F, n_answers, B) -> int:
    return int(lib.dynbatch_classify_workspace_bytes(ct.byref(_HeadShape(C, H, W, dtype, Cc, F, n_answers)), B))


def dynbatch_classify(roots, head: dict, probs=None, want_logits: bool = False, workspace=None, stream=None):
    """roots: device [B,H,W,C] float32 or bfloat16 (the output of dynbatch_execute); head: dict of device tensors
    wc [Cc,C], wf1 [F,H*W*Cc], wf2 [A,F] in the dtype of roots and bc, bf1, bf2 float32 or None.
    Returns probs [B,A] float32 (and the logits if wanted)."""
    import torch
    assert roots.is_cuda and roots.is_contiguous() and roots.dtype in (torch.float32, torch.bfloat16)
    for key in ("wc", "wf1", "wf2"):
        assert head[key].is_cuda and head[key].is_contiguous() and head[key].dtype == roots.dtype, key
    for key in ("bc", "bf1", "bf2"):
        t = head.get(key)
        assert t is None or (t.is_cuda and t.is_contiguous() and t.dtype == torch.float32), key
    shape = _head_shape(roots, head)
    B, A = roots.shape[0], shape.n_answers
    rows = lambda: _made(stream, lambda: torch.empty((B, A), dtype=torch.float32, device=roots.device))
    if probs is None:
        probs = rows()
    logits = rows() if want_logits else None
    if workspace is None:
        workspace = _scratch(lib.dynbatch_classify_workspace_bytes(ct.byref(shape), B), roots.device, stream)
    w = _HeadWeights(*[(head.get(k).data_ptr() if head.get(k) is not None else None) for k in ("wc", "bc", "wf1", "bf1", "wf2", "bf2")])
    _check(lib.dynbatch_classify(ct.byref(shape), ct.byref(w), _ptr(roots), B, _ptr(probs), _ptr(logits), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)))
    return (probs, logits) if want_logits else probs


# ------------------------------------------------------------------------------------------ MoE
def moe_workspace_bytes(T: int, d: int, h: int, E: int, k: int, dtype: int = DYNB_BF16) -> int:
    return int(lib.moe_workspace_bytes(ct.byref(_MoeShape(T, d, h, E, k, dtype))))


MOE_STATIC_SCRATCH_BYTES = 48 << 20
MOE_SEPARATE_PERMUTE = 1


def moe_forward_static(x, Wg, Wn, noise, W1, W2, k: int, out, aux=None, stream=None):
    """moe_forward without a workspace: the library's built-in device array holds the scratch data and the
    call allocates nothing, so `out` (and the aux tensors, if wanted: a namespace like moe_forward returns)
    must be given."""
    T, d = x.shape
    E, h = W1.shape[0], W1.shape[1]
    shape = _MoeShape(T, d, h, E, k, DYNB_BF16)
    aux_c = None
    if aux is not None:
        aux_c = _MoeAux(*[getattr(aux, n).data_ptr() for n in
                          ("logits", "topk_idx", "topk_w", "counts", "offsets", "perm", "inv")])
    _check(lib.moe_forward_static(ct.byref(shape), _ptr(x), _ptr(Wg), _ptr(Wn), _ptr(noise), _ptr(W1), _ptr(W2),
                                  _ptr(out), ct.byref(aux_c) if aux_c is not None else None, _stream(stream)))
    return out


def moe_forward(x, Wg, Wn, noise, W1, W2, k: int, out=None, want_aux: bool = False, workspace=None, stream=None,
                naive_stride: int = 0, flags: int = 0):
    """x [T,d] bf16; Wg, Wn [E,d] bf16; noise [T,E] f32 or None; W1 [E,h,d]; W2 [E,d,h] bf16 (all device,
    contiguous).  Returns out [T,d] bf16, or (out, aux namespace of device tensors) if want_aux.
    naive_stride >= 1 calls moe_forward_naive (one expert call per use) instead."""
    import torch
    T, d = x.shape
    E, h = W1.shape[0], W1.shape[1]
    for t in (x, Wg, W1, W2):
        assert t.is_cuda and t.is_contiguous() and t.dtype == torch.bfloat16
    assert Wg.shape == (E, d) and W1.shape == (E, h, d) and W2.shape == (E, d, h)
    assert Wn is None or (Wn.is_cuda and Wn.is_contiguous() and Wn.dtype == torch.bfloat16 and Wn.shape == (E, d))
    assert noise is None or (noise.is_cuda and noise.is_contiguous() and noise.dtype == torch.float32
                             and noise.shape == (T, E))
    shape = _MoeShape(T, d, h, E, k, DYNB_BF16, flags)
    if out is None:
        out = _made(stream, lambda: torch.empty_like(x))
    if workspace is None:
        n = int(lib.moe_workspace_bytes(ct.byref(shape)))
        if n == 0:
            _check(lib.moe_forward(ct.byref(shape), None, None, None, None, None, None, None, None, None, 0, None))
        workspace = _scratch(n, x.device, stream)
    aux_t, aux_c = None, None
    if want_aux:
        names = ("logits", "topk_idx", "topk_w", "counts", "offsets", "perm", "inv")
        sizes = ((T, E), (T, k), (T, k), (E,), (E + 1,), (T * k,), (T * k,))
        aux_t = SimpleNamespace(**dict(zip(names, _made(stream, lambda: [
            torch.empty(size, dtype=torch.float32 if name in ("logits", "topk_w") else torch.int32, device=x.device)
            for name, size in zip(names, sizes)]))))
        aux_c = _MoeAux(*[getattr(aux_t, n).data_ptr() for n in names])
    args = (ct.byref(shape), _ptr(x), _ptr(Wg), _ptr(Wn), _ptr(noise), _ptr(W1), _ptr(W2), _ptr(out),
            ct.byref(aux_c) if aux_c is not None else None, _ptr(workspace),
            workspace.numel() * workspace.element_size(), _stream(stream))
    if naive_stride:
        _check(lib.moe_forward_naive(*args, naive_stride))
    else:
        _check(lib.moe_forward(*args))
    return (out, aux_t) if want_aux else out


MOE_KERNELS = ("gate_stream", "gate_small", "gate_big", "stream", "few1", "few2", "skinny1", "skinny2")


def dynb_moe_kernels(T: int, d: int, h: int, E: int, k: int, noisy: bool = False, flags: int = 0) -> set:
    """The kernels that moe_forward chooses for tensors on 16-byte borders (k_gate and k_grouped_gemm where none is named)."""
    bits = lib.dynb_moe_kernels(ct.byref(_MoeShape(T, d, h, E, k, DYNB_BF16, flags)), int(noisy))
    if bits < 0:
        _check(bits)
    return {name for i, name in enumerate(MOE_KERNELS) if bits >> i & 1}


# ------------------------------------------------------------------------------------------ products grouped by expert
MOE_PRODUCT_RELU = 1


_F32 = _BF16 = _I8 = _I32 = None                 # torch's, once a tensor has been met


def _meet_torch():
    global _F32, _BF16, _I8, _I32
    import torch
    _F32, _BF16, _I8, _I32 = torch.float32, torch.bfloat16, torch.int8, torch.int32


def _dtype_code(t) -> int:
    if _F32 is None:
        _meet_torch()
    dtype = t.dtype
    if dtype is _F32:
        return DYNB_F32
    assert dtype is _BF16, dtype
    return DYNB_BF16


def _rows(t, n: int, width: int, like=None) -> int:
    """Checks a tensor of n rows of `width` neighbouring elements; returns the elements from a row to the next."""
    stride = t.stride()
    assert t.is_cuda and t.shape == (n, width) and (width == 1 or stride[1] == 1), (t.shape, stride)
    assert like is None or t.dtype is like.dtype
    return stride[0] if n > 1 else max(stride[0], width)


def _new(stream, *shape, like, dtype=None):
    """An uninitialised result."""
    import torch
    if stream is None:                           # (the usual case, without the detour)
        return torch.empty(shape, dtype=dtype if dtype is not None else like.dtype, device=like.device)
    return _made(stream, lambda: torch.empty(shape, dtype=dtype if dtype is not None else like.dtype, device=like.device))


def _twin(stream, t):
    """Another one (in half of _new's time)."""
    import torch
    return torch.empty_like(t) if stream is None else _made(stream, lambda: torch.empty_like(t))


def _groups_struct(offsets, perm, k: int, M: int, rows: int) -> _Groups:
    if _I32 is None:
        _meet_torch()
    assert offsets.is_cuda and offsets.is_contiguous() and offsets.dtype is _I32
    if perm is None:
        return _Groups(offsets.data_ptr(), None, k, rows)
    assert perm.is_cuda and perm.is_contiguous() and perm.dtype is _I32 and perm.shape == (M,)
    return _Groups(offsets.data_ptr(), perm.data_ptr(), k, rows)


def moe_product(x, W, offsets, perm=None, k: int = 1, relu: bool = False, out=None, stream=None):
    """out[r] = f(x[row(r)] W_e^T) for the rows r of every group e.  x [rows,K], W [E,N,K] bf16; offsets [E+1] int32: group e is rows
    offsets[e] .. offsets[e+1]; perm [M] int32: row(r) = perm[r] // k, None: row(r) = r (moe_forward's aux gives offsets and perm
    in this form).  f: ReLU or nothing.  Returns out [M,N] bf16."""
    import torch
    E, N, K = W.shape
    M = x.shape[0] if perm is None else perm.shape[0]
    xs = _rows(x, x.shape[0], K)
    assert W.is_cuda and W.is_contiguous() and W.dtype == x.dtype == torch.bfloat16 and offsets.shape == (E + 1,)
    if out is None:
        out = _new(stream, M, N, like=x)
    os_ = _rows(out, M, N, x)
    g = _groups_struct(offsets, perm, k, M, x.shape[0])
    shape = _ProductShape(M, K, N, E, DYNB_BF16, MOE_PRODUCT_RELU if relu else 0)
    _check(lib.moe_product(ct.byref(shape), ct.byref(g), x.data_ptr(), xs, W.data_ptr(), out.data_ptr(), os_, _stream(stream)))
    return out


def moe_product_grad_input(dout, W, offsets, act=None, out=None, stream=None):
    """din[r] = dout[r] W_e for the rows r of every group e, set to 0 where `act` (the ReLU's results that the layer read, or None)
    is not positive.  dout [M,N], W [E,N,K], act [M,K] bf16; offsets as in moe_product.  Returns din [M,K] bf16."""
    import torch
    E, N, K = W.shape
    M = dout.shape[0]
    ds = _rows(dout, M, N)
    assert W.is_cuda and W.is_contiguous() and W.dtype == dout.dtype == torch.bfloat16 and offsets.shape == (E + 1,)
    as_ = 0 if act is None else _rows(act, M, K, dout)
    if out is None:
        out = _new(stream, M, K, like=dout)
    os_ = _rows(out, M, K, dout)
    g = _groups_struct(offsets, None, 1, M, M)
    shape = _ProductShape(M, K, N, E, DYNB_BF16, 0)
    _check(lib.moe_product_grad_input(ct.byref(shape), ct.byref(g), dout.data_ptr(), ds, W.data_ptr(),
                                      None if act is None else act.data_ptr(), as_, out.data_ptr(), os_, _stream(stream)))
    return out


def moe_product_grad_weight_workspace_bytes(M: int, K: int, N: int, E: int) -> int:
    return int(lib.moe_product_grad_weight_workspace_bytes(ct.byref(_ProductShape(M, K, N, E, DYNB_BF16, 0))))


def moe_product_grad_weight(dout, x, offsets, perm=None, k: int = 1, dW=None, grad_dtype: int = DYNB_F32, workspace=None, stream=None):
    """dW_e = sum over the rows r of group e of dout[r]^T x[row(r)] (0 for an empty group).  dout [M,N], x [rows,K] bf16; offsets, perm and
    k as in moe_product.  Returns dW [E,N,K] in grad_dtype (`dW`: such a tensor of an earlier call, float32 or bfloat16, to be overwritten)."""
    import torch
    M, N = dout.shape
    K, E = x.shape[1], offsets.shape[0] - 1
    ds, xs = _rows(dout, M, N), _rows(x, M if perm is None else x.shape[0], K, dout)
    assert dout.dtype == torch.bfloat16
    if dW is None:
        dW = _new(stream, E, N, K, like=x, dtype=torch.float32 if grad_dtype == DYNB_F32 else torch.bfloat16)
    assert dW.is_cuda and dW.is_contiguous() and dW.shape == (E, N, K)
    g = _groups_struct(offsets, perm, k, M, x.shape[0])
    shape = _ProductShape(M, K, N, E, DYNB_BF16, 0)
    if workspace is None:
        workspace = _scratch(lib.moe_product_grad_weight_workspace_bytes(ct.byref(shape)), x.device, stream)
    _check(lib.moe_product_grad_weight(ct.byref(shape), ct.byref(g), dout.data_ptr(), ds, x.data_ptr(), xs, dW.data_ptr(), _dtype_code(dW),
                                       workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream)))
    return dW


# ------------------------------------------------------------------------------------------ gated layers
MOE_GATE_SILU, MOE_GATE_GELU = 0, 1


def _pre_struct(pre, M: int, h: int) -> _GatedPre:
    eight = type(pre) is Rows8
    rows = pre.q if eight else pre
    s0, s1, s2 = rows.stride()
    assert rows.is_cuda and rows.shape == (M, 2, h) and s1 == h and (s2 == 1 or h == 1), (rows.shape, rows.stride())
    if M <= 1:
        s0 = max(s0, 2 * h)
    if _BF16 is None:
        _meet_torch()
    if not eight:
        assert rows.dtype is _BF16
        return _GatedPre(rows.data_ptr(), s0, None, 0, DYNB_BF16)
    scale, n = pre.scale, (h + 31) // 32
    c0, c1, c2 = scale.stride()
    assert rows.dtype is _I8 and scale.dtype is _BF16 and scale.is_cuda and scale.shape == (M, 2, n) and c1 == n and (c2 == 1 or n == 1), (scale.shape, scale.stride())
    return _GatedPre(rows.data_ptr(), s0, scale.data_ptr(), c0 if M > 1 else max(c0, 2 * n), DYNB_I8)


def moe_gated(x, W, offsets, perm=None, k: int = 1, gate: int = MOE_GATE_SILU, out=None, pre=None, stream=None):
    """out[r] = f(x[row(r)] Wg_e^T) (x[row(r)] Wu_e^T) for the rows r of every group e, f SiLU or GELU (tanh form).  x [rows,K], W [E,2,h,K] (Wg, Wu)
    bf16; offsets, perm and k as in moe_product.  pre: what to keep of gate and up for the backward pass, a bf16 tensor [M,2,h] or Rows8(q [M,2,h],
    scale [M,2,(h + 31) // 32]) to be written, or None.  Returns out [M,h] bf16."""
    E, two, h, K = W.shape
    n = x.shape[0]
    M = n if perm is None else perm.shape[0]
    xs = _rows(x, n, K)
    g = _groups_struct(offsets, perm, k, M, n)
    assert two == 2 and W.is_cuda and W.is_contiguous() and W.dtype is x.dtype is _BF16 and offsets.shape == (E + 1,)
    if out is None:
        out = _new(stream, M, h, like=x)
    _check(lib.moe_gated(_GatedShape(M, K, h, E, DYNB_BF16, gate), g, x.data_ptr(), xs, W.data_ptr(), out.data_ptr(), _rows(out, M, h, x),
                         None if pre is None else _pre_struct(pre, M, h), _stream(stream)))
    return out


def moe_gated_grad(dout, W, offsets, pre, gate: int = MOE_GATE_SILU, dpre=None, hidden=None, want_hidden: bool = True, stream=None):
    """Backward through the second layer's product and the gate: with dact[r] = dout[r] W_e, the gradients dact up f'(gate) and dact f(gate) of what was kept,
    and f(gate) up again, which the second layer's weights' gradient wants.  dout [M,N], W [E,N,h] bf16 (moe_product's second layer), pre as moe_gated kept
    it.  Returns (dpre [M,2,h], hidden [M,h]) bf16, or dpre alone without want_hidden.  dpre.view(M, 2 * h) and W.view(E, 2 * h, K) of moe_gated are what
    moe_product_grad_input and moe_product_grad_weight take."""
    E, N, h = W.shape
    M = dout.shape[0]
    ds = _rows(dout, M, N)
    g = _groups_struct(offsets, None, 1, M, M)
    assert W.is_cuda and W.is_contiguous() and W.dtype is dout.dtype is _BF16 and offsets.shape == (E + 1,)
    if dpre is None:
        dpre = _new(stream, M, 2, h, like=dout)
    assert type(dpre) is not Rows8
    d = _pre_struct(dpre, M, h)
    if hidden is None and want_hidden:
        hidden = _new(stream, M, h, like=dout)
    to, hs = (None, 0) if hidden is None else (hidden.data_ptr(), _rows(hidden, M, h, dout))
    _check(lib.moe_gated_grad(_GatedShape(M, N, h, E, DYNB_BF16, gate), g, dout.data_ptr(), ds, W.data_ptr(), _pre_struct(pre, M, h), d.rows, d.stride, to, hs, _stream(stream)))
    return dpre if hidden is None else (dpre, hidden)


# ------------------------------------------------------------------------------------------ rows in 8 bits
class Rows8(NamedTuple):
    """Rows of activations in 8 bits: q [...,d] int8, scale [...,(d + 31) // 32] bfloat16, a scale for every 32 neighbours of a row."""
    q: object
    scale: object


def _rows8_struct(r: Rows8, T: int, d: int) -> _Rows8:
    if _I8 is None:
        _meet_torch()
    q, scale = r
    assert q.dtype is _I8 and scale.dtype is _BF16
    return _Rows8(q.data_ptr(), _rows(q, T, d), scale.data_ptr(), _rows(scale, T, (d + 31) // 32))


def dynb_store8(x, out=None, stream=None) -> Rows8:
    """Rows x [T,d] float32 or bfloat16 in 8 bits, (q [T,d] int8, scale [T,(d + 31) // 32] bfloat16): s = max|x| / 127 of 32 neighbours, rounded up to a
    bfloat16, q = x / s rounded (both in fp32).  A block with an infinity or a NaN comes back as NaN."""
    T, d = x.shape
    xs = _rows(x, T, d)
    shape = _Rows8Shape(T, d, _dtype_code(x))
    if out is None:
        out = Rows8(_new(stream, T, d, like=x, dtype=_I8), _new(stream, T, (d + 31) // 32, like=x, dtype=_BF16))
    _check(lib.dynb_store8(shape, x.data_ptr(), xs, _rows8_struct(out, T, d), _stream(stream)))
    return out


def dynb_load8(rows: Rows8, out=None, dtype: int = DYNB_BF16, stream=None):
    """What rows in 8 bits stand for, q s.  Returns a tensor [T,d] of `dtype`, bfloat16 or float32 (`out`: such a tensor, to be overwritten)."""
    T, d = rows.q.shape
    r = _rows8_struct(rows, T, d)
    if out is None:
        assert dtype in (DYNB_F32, DYNB_BF16), dtype
        out = _new(stream, T, d, like=rows.q, dtype=_F32 if dtype == DYNB_F32 else _BF16)
    _check(lib.dynb_load8(_Rows8Shape(T, d, _dtype_code(out)), r, out.data_ptr(), _rows(out, T, d), _stream(stream)))
    return out


# ------------------------------------------------------------------------------------------ embeddings
def dynb_embed(tokens, table, scale: float = 1.0, out=None, stream=None):
    """out[t] = scale * table[tokens[t]], a row of zeros for a token outside [0, V).  tokens [T] int32, table [V,d] float32 or bfloat16
    (device, contiguous).  Returns out [T,d] in the table's dtype."""
    import torch
    T, (V, d) = tokens.shape[0], table.shape
    assert tokens.is_cuda and tokens.is_contiguous() and tokens.dtype == torch.int32 and tokens.dim() == 1
    assert table.is_cuda and table.is_contiguous()
    if out is None:
        out = _new(stream, T, d, like=table)
    os_ = _rows(out, T, d, table)
    shape = _EmbedShape(T, V, d, _dtype_code(table), scale)
    _check(lib.dynb_embed(ct.byref(shape), tokens.data_ptr(), table.data_ptr(), out.data_ptr(), os_, _stream(stream)))
    return out


def dynb_embed_backward_workspace_bytes(T: int, V: int, d: int, dtype: int) -> int:
    return int(lib.dynb_embed_backward_workspace_bytes(ct.byref(_EmbedShape(T, V, d, dtype, 1.0))))


def dynb_embed_backward(tokens, dout, V: int, scale: float = 1.0, dtable=None, grad_dtype: int = DYNB_F32, workspace=None, stream=None):
    """dtable[v] = scale * sum over t with tokens[t] = v of dout[t], every row written.  dout [T,d] float32 or bfloat16.  Returns dtable
    [V,d] in grad_dtype (`dtable`: such a tensor of an earlier call, float32 or bfloat16, to be overwritten)."""
    import torch
    T, d = dout.shape
    assert tokens.is_cuda and tokens.is_contiguous() and tokens.dtype == torch.int32 and tokens.shape == (T,)
    ds = _rows(dout, T, d)
    if dtable is None:
        dtable = _new(stream, V, d, like=dout, dtype=torch.float32 if grad_dtype == DYNB_F32 else torch.bfloat16)
    assert dtable.is_cuda and dtable.is_contiguous() and dtable.shape == (V, d)
    shape = _EmbedShape(T, V, d, _dtype_code(dout), scale)
    if workspace is None:
        workspace = _scratch(lib.dynb_embed_backward_workspace_bytes(ct.byref(shape)), dout.device, stream)
    _check(lib.dynb_embed_backward(ct.byref(shape), tokens.data_ptr(), dout.data_ptr(), ds, dtable.data_ptr(), _dtype_code(dtable),
                                   workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream)))
    return dtable


# ------------------------------------------------------------------------------------------ layer norm
def _fp32(t, n: int):
    if t is None:
        return None
    if _F32 is None:
        _meet_torch()
    assert t.is_cuda and t.dtype is _F32 and t.shape == (n,) and t.is_contiguous()
    return t.data_ptr()


def dynb_layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, out=None, want_stats: bool = False, stream=None):
    """Layer norm of the rows of x [T,d] (float32 or bfloat16); gamma, beta [d] float32 or None.  Returns y in the dtype of x, or
    (y, mean, rstd), mean and rstd [T] float32, if the backward pass will want them."""
    import torch
    T, d = x.shape
    xs = _rows(x, T, d)
    if out is None:
        out = _new(stream, T, d, like=x)
    ys = _rows(out, T, d, x)
    shape = _NormShape(T, d, _dtype_code(x), eps)
    if not want_stats:
        _check(lib.dynb_layer_norm(ct.byref(shape), x.data_ptr(), xs, _fp32(gamma, d), _fp32(beta, d), out.data_ptr(), ys, None, None, _stream(stream)))
        return out
    mean = _new(stream, T, like=x, dtype=torch.float32)
    rstd = _twin(stream, mean)
    _check(lib.dynb_layer_norm(ct.byref(shape), x.data_ptr(), xs, _fp32(gamma, d), _fp32(beta, d), out.data_ptr(), ys, mean.data_ptr(), rstd.data_ptr(),
                               _stream(stream)))
    return out, mean, rstd


def dynb_layer_norm_backward_workspace_bytes(T: int, d: int, dtype: int) -> int:
    return int(lib.dynb_layer_norm_backward_workspace_bytes(ct.byref(_NormShape(T, d, dtype, 0.0))))


def dynb_layer_norm_backward(dy, x, gamma, mean, rstd, dx=None, workspace=None, stream=None):
    """Gradients of dynb_layer_norm: dy, x [T,d], mean and rstd what it returned; x may be Rows8, the layer's input in 8 bits.  Returns (dx [T,d] in the dtype of
    dy, dgamma [d], dbeta [d] float32)."""
    T, d = dy.shape
    eight = type(x) is Rows8
    ds, xs = _rows(dy, T, d), 0 if eight else _rows(x, T, d, dy)
    if dx is None:
        dx = _new(stream, T, d, like=dy)
    dxs = _rows(dx, T, d, dy)
    shape = _NormShape(T, d, _dtype_code(dy), 0.0)
    dgamma = _new(stream, d, like=dy, dtype=_F32)
    dbeta = _twin(stream, dgamma)
    if workspace is None:
        workspace = _scratch(lib.dynb_layer_norm_backward_workspace_bytes(shape), dy.device, stream)
    rest = (_fp32(gamma, d), _fp32(mean, T), _fp32(rstd, T), dx.data_ptr(), dxs, dgamma.data_ptr(), dbeta.data_ptr(), workspace.data_ptr(), workspace.nbytes, _stream(stream))
    if eight:
        _check(lib.dynb_layer_norm_backward8(shape, dy.data_ptr(), ds, _rows8_struct(x, T, d), *rest))
    else:
        _check(lib.dynb_layer_norm_backward(shape, dy.data_ptr(), ds, x.data_ptr(), xs, *rest))
    return dx, dgamma, dbeta


# ------------------------------------------------------------------------------------------ clipping
class GradTensors:
    """A network's gradient tensors (device, contiguous, float32 or bfloat16) and where the clipped ones go (None: into the gradients
    themselves), marshalled once for the steps in which they stay where they are.  Keeps the tensors alive.  No two results may share
    memory: a gradient that several names stand for is listed once."""

    def __init__(self, grads, out=None):
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        assert len(self.grads) == len(self.out)
        for g, o in zip(self.grads, self.out):
            assert g.is_cuda and g.is_contiguous() and o.is_cuda and o.is_contiguous() and o.dtype == g.dtype and o.numel() == g.numel()
        listed = [(g.data_ptr(), o.data_ptr(), g.numel(), _dtype_code(g)) for g, o in zip(self.grads, self.out)]
        places = [t[1] for t in listed if t[2]]
        assert len(set(places)) == len(places), "two results at one place"
        self.array = (_GradTensor * max(len(self.grads), 1))(*listed)


def dynb_clip_workspace_bytes() -> int:
    return int(lib.dynb_clip_workspace_bytes())


def dynb_clip_gradients(grads, max_norm: float, norm=None, workspace=None, stream=None):
    """Scales the gradients (a list of tensors, in place, or a GradTensors) down to a norm of all of them together of max_norm, if that norm is
    finite and above it.  Returns the norm they had: one float32 on the device."""
    import torch
    t = grads if isinstance(grads, GradTensors) else GradTensors(grads)
    device = t.grads[0].device if t.grads else torch.device("cuda", torch.cuda.current_device())
    if norm is None:
        norm = _made(stream, lambda: torch.empty((), dtype=torch.float32, device=device))
    assert norm.is_cuda and norm.dtype == torch.float32 and norm.numel() == 1
    if workspace is None:
        workspace = _scratch(lib.dynb_clip_workspace_bytes(), device, stream)
    _check(lib.dynb_clip_gradients(t.array, len(t.grads), max_norm, norm.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                   _stream(stream)))
    return norm


# ------------------------------------------------------------------------------------------ timing
MOE_STAGES = ("gate", "topk", "sort", "permute", "ffn1", "ffn2", "combine")


def dynb_timing_enable(mode) -> None:
    """0/False off, 1/True one event per launch group or stage, 2 one event pair around all launch groups."""
    _check(lib.dynb_timing_enable(int(mode)))


def dynb_timing_read():
    """Stages of the last timed call: list of (tag, units, ms)."""
    n = ct.c_int32(0)
    _check(lib.dynb_timing_read(None, 0, ct.byref(n)))
    if n.value == 0:
        return []
    buf = (_StageTime * n.value)()
    _check(lib.dynb_timing_read(buf, n.value, ct.byref(n)))
    return [(b.tag, b.units, b.ms) for b in buf]


# ------------------------------------------------------------------------------------------ measurement helpers
def dynb_probe_mfma_bf16(iters: int, workgroups: int, sink, stream=None) -> float:
    """Enqueues the register-only MFMA loop; returns its flop count (time it with events on the stream)."""
    fl = ct.c_double(0.0)
    _check(lib.dynb_probe_mfma_bf16(iters, workgroups, _ptr(sink), _stream(stream), ct.byref(fl)))
    return fl.value


def dynb_probe_read(src, sink, stream=None) -> int:
    """Reads all of `src` (device tensor) and stores nothing; returns the number of bytes read."""
    n = src.numel() * src.element_size()
    _check(lib.dynb_probe_read(_ptr(src), n, _ptr(sink), _stream(stream)))
    return n


def dynb_probe_copy(dst, src, stream=None) -> int:
    """Enqueues the plain copy kernel over two equally sized device tensors; returns the bytes copied."""
    n = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == n
    _check(lib.dynb_probe_copy(_ptr(dst), _ptr(src), n, _stream(stream)))
    return n
