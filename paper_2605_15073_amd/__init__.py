"""Python binding of libcgtp (contracted Clebsch-Gordan products on MI355X).

Thin ctypes marshalling over the C ABI declared in ``include/cgtp.h``: every
step of the computation runs in the HIP kernels of ``libcgtp.so``. Tensors are
torch device tensors (torch provides device memory and streams only). If the
shared library is missing this module raises on first use; there is no CPU
fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcgtp.so")

CGTP_OK = 0
CGTP_ERR_ARG = -1
CGTP_ERR_WORKSPACE = -2
CGTP_ERR_CSR = -3
CGTP_ERR_HIP = -4
CGTP_ERR_UNSUPPORTED = -5
CGTP_F32 = 0
CGTP_F64 = 1
CGTP_BF16 = 2
CGTP_VALIDATE_CSR = 1
CGTP_EDGE_SEPARATED = 2
CGTP_TIME_STAGES = 4
CGTP_OP_ONSITE = 0
CGTP_OP_MESSAGE_PASS = 1
CGTP_OP_MESSAGE_PASS_TWO_SLOT = 2
CGTP_OP_ONSITE_GENERAL = 3
CGTP_OP_MESSAGE_PASS_GENERAL = 4
CGTP_OP_MESSAGE_PASS_FIELDS = 5
CGTP_OP_ONSITE_NBODY = 6
CGTP_MAX_NU = 8
CGTP_MAX_LMAX = 24
CGTP_MAX_GROUPS = 4096
CGTP_MAX_WIDTH = 65536
CGTP_MAX_ADAPTER_RANK = 64
CGTP_ADAMW_BLOCK = 256
CGTP_MAX_TOP_K = 64
CGTP_MAX_ROUTE_BLOCKS = 64
CGTP_SCORE_SOFTMAX = 0
CGTP_SCORE_SIGMOID = 1
CGTP_MAX_PER_ROW = 64
CGTP_ACT_NONE = 0
CGTP_ACT_SILU = 1
CGTP_ACT_GELU = 2
CGTP_ACT_RELU = 3

EXPORTED = ("cgtp_plan_create", "cgtp_plan_grid", "cgtp_workspace_bytes", "cgtp_onsite",
            "cgtp_message_pass", "cgtp_message_pass_two_slot", "cgtp_workspace_bytes_general",
            "cgtp_onsite_general", "cgtp_message_pass_general", "cgtp_message_pass_fields",
            "cgtp_workspace_bytes_nbody", "cgtp_onsite_nbody", "cgtp_stage_times",
            "cgtp_destroy", "cgtp_status_string", "cgtp_last_error", "cgtp_host_tables",
            "cgtp_onsite_noalloc", "cgtp_gather_probe", "cgtp_receiver_order",
            "cgtp_plan_set_receiver_order", "cgtp_group_rows_bytes", "cgtp_group_rows",
            "cgtp_grouped_linear", "cgtp_grouped_linear_grad_bytes", "cgtp_grouped_linear_grad",
            "cgtp_adapter_linear_bytes", "cgtp_adapter_linear", "cgtp_adapter_linear_grad_bytes",
            "cgtp_adapter_linear_grad", "cgtp_adamw_create", "cgtp_adamw_step",
            "cgtp_adamw_states", "cgtp_adamw_destroy", "cgtp_route_rows", "cgtp_route_rows_grad",
            "cgtp_grouped_layer", "cgtp_grouped_layer_grad_bytes", "cgtp_grouped_layer_grad",
            "cgtp_mix_rows", "cgtp_mix_rows_grad", "cgtp_adamw_grad_norm_bytes",
            "cgtp_adamw_grad_norm")
CGTP_NOALLOC_SCRATCH_BYTES = 64 << 20
ONSITE_STAGES = ("contract_operands", "grid_product_curl_analysis", "project")
ONSITE_GENERAL_STAGES = ("contract_a", "contract_b", "grid_product_curl_analysis",
                         "project_even", "project_odd")
MP_STAGES = ("contract_node", "sender_fields", "contract_edge_radial", "receiver", "analysis",
             "project_even", "project_odd")
NBODY_STAGES = ("contract_operands", "grid_product_analysis", "project")


class CgtpError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: status {status} ({detail})")
        self.status = status


class _Desc(ctypes.Structure):
    _fields_ = [("lmax", ctypes.c_int), ("channels", ctypes.c_int), ("rank", ctypes.c_int),
                ("n_theta", ctypes.c_int), ("n_phi", ctypes.c_int), ("dtype", ctypes.c_int),
                ("flags", ctypes.c_uint)]


class _AdamWTensor(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("param", "grad", "m", "v", "m_scale", "v_scale",
                                                "copy")] + [("n", ctypes.c_int64)])


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libcgtp.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libcgtp.so not found at {path}: build it with "
                           "`python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(path)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    lib.cgtp_plan_create.argtypes = [ctypes.POINTER(_Desc), ctypes.POINTER(vp)]
    lib.cgtp_plan_grid.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.cgtp_workspace_bytes.argtypes = [vp, i32, i64, i64, ctypes.POINTER(sz)]
    lib.cgtp_onsite.argtypes = [vp, i64] + [vp] * 8 + [vp, sz, vp]
    lib.cgtp_onsite_noalloc.argtypes = [vp, i64] + [vp] * 8 + [vp]
    lib.cgtp_gather_probe.argtypes = [vp, i64, i64, vp, vp, vp, sz, vp, vp]
    lib.cgtp_message_pass.argtypes = [vp, i64, i64] + [vp] * 11 + [vp, sz, vp]
    lib.cgtp_message_pass_two_slot.argtypes = [vp, i64, i64] + [vp] * 12 + [vp, sz, vp]
    lib.cgtp_workspace_bytes_general.argtypes = [vp, i32, i64, i64, i32, i32, i32,
                                                 ctypes.POINTER(sz)]
    lib.cgtp_onsite_general.argtypes = ([vp, i64] + [vp] * 4 + [i32, vp, vp, i32] + [vp] * 4
                                        + [vp, sz, vp])
    lib.cgtp_message_pass_general.argtypes = ([vp, i64, i64] + [vp] * 6 + [i32, vp, vp, i32]
                                              + [vp] * 4 + [vp, sz, vp])
    lib.cgtp_message_pass_fields.argtypes = lib.cgtp_message_pass_general.argtypes
    lib.cgtp_workspace_bytes_nbody.argtypes = [vp, i64, i32, ctypes.POINTER(sz)]
    lib.cgtp_onsite_nbody.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.cgtp_stage_times.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double), i32,
                                     ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.cgtp_destroy.argtypes = [vp]
    lib.cgtp_status_string.argtypes = [i32]
    lib.cgtp_status_string.restype = ctypes.c_char_p
    lib.cgtp_last_error.argtypes = []
    lib.cgtp_last_error.restype = ctypes.c_char_p
    lib.cgtp_host_tables.argtypes = [i32, i32, i32] + [vp] * 5
    lib.cgtp_receiver_order.argtypes = [i64, i64, vp, vp, vp, vp]
    lib.cgtp_plan_set_receiver_order.argtypes = [vp, i64, vp]
    f64, szp = ctypes.c_double, ctypes.POINTER(sz)
    lib.cgtp_group_rows_bytes.argtypes = [i64, i32, szp]
    lib.cgtp_group_rows.argtypes = [i64, i32] + [vp] * 4 + [sz, vp]
    rows = [i32, i64, i32, i32, i32]              # dtype, n_rows, n_groups, n_in, n_out
    lib.cgtp_grouped_linear.argtypes = rows + [vp] * 3 + [i64, vp, vp, i64, vp]
    lib.cgtp_grouped_linear_grad_bytes.argtypes = rows + [szp]
    lib.cgtp_grouped_linear_grad.argtypes = (rows + [vp] * 3 + [i64, vp, vp, i64, vp, i64, vp, vp]
                                             + [sz, vp])
    lib.cgtp_adapter_linear_bytes.argtypes = rows + [i32, szp]
    lib.cgtp_adapter_linear.argtypes = (rows + [i32] + [vp] * 3 + [i64] + [vp] * 5 + [i64, vp]
                                        + [sz, vp])
    lib.cgtp_adapter_linear_grad_bytes.argtypes = rows + [i32, szp]
    lib.cgtp_adapter_linear_grad.argtypes = (rows + [i32] + [vp] * 3 + [i64] + [vp] * 5
                                             + [i64, vp, i64] + [vp] * 3 + [sz, vp])
    lib.cgtp_adamw_create.argtypes = [i32, ctypes.POINTER(_AdamWTensor), i32, i32,
                                      ctypes.POINTER(vp)]
    lib.cgtp_adamw_step.argtypes = [vp] + [f64] * 5 + [i64, vp, vp]
    lib.cgtp_adamw_states.argtypes = [vp] * 4
    lib.cgtp_adamw_destroy.argtypes = [vp]
    lib.cgtp_adamw_grad_norm_bytes.argtypes = [vp, szp]
    lib.cgtp_adamw_grad_norm.argtypes = [vp, f64, vp, vp, vp, vp, sz, vp]
    f32, routed = ctypes.c_float, [i32, i64, i32, i32]   # dtype, n_rows, n_experts, top_k
    lib.cgtp_route_rows.argtypes = routed + [vp, i64, vp, i32, i32, i32, i32, f32, vp, vp, vp]
    lib.cgtp_route_rows_grad.argtypes = routed + [vp, i64, vp, vp, i32, i32, f32, vp, i64, vp]
    layer = rows + [i32]                          # per_row
    lib.cgtp_grouped_layer.argtypes = layer + [vp] * 3 + [i64, vp, vp, i32, vp, i64, vp, i64, vp, i64, vp]
    lib.cgtp_grouped_layer_grad_bytes.argtypes = layer + [i32, szp]
    lib.cgtp_grouped_layer_grad.argtypes = (layer + [vp] * 3 + [i64, vp, vp, i64, i32, vp, i64, vp, i64]
                                            + [vp] * 3 + [sz, vp])
    mixed = [i32, i64, i32, i32, vp, i64]         # dtype, n_rows, per_row, width, y or dout
    lib.cgtp_mix_rows.argtypes = mixed + [vp, vp, i64, vp, i64, vp]
    lib.cgtp_mix_rows_grad.argtypes = mixed + [vp, vp, i64, vp, i64, vp, vp]
    for name in ("cgtp_plan_create", "cgtp_plan_grid", "cgtp_workspace_bytes", "cgtp_onsite",
                 "cgtp_onsite_noalloc", "cgtp_gather_probe",
                 "cgtp_message_pass", "cgtp_message_pass_two_slot", "cgtp_stage_times",
                 "cgtp_destroy", "cgtp_host_tables", "cgtp_receiver_order",
                 "cgtp_plan_set_receiver_order", *(n for n in EXPORTED if n.startswith(
                     ("cgtp_group", "cgtp_adapter", "cgtp_adamw", "cgtp_route", "cgtp_mix")))):
        getattr(lib, name).restype = i32
    _lib = lib
    return lib


def _check(status: int, where: str):
    if status != CGTP_OK:
        lib = load_library()
        detail = lib.cgtp_last_error().decode() or lib.cgtp_status_string(status).decode()
        raise CgtpError(status, where, detail)


class Plan:
    """Owns a cgtp_plan handle (grid tables on the current device)."""

    def __init__(self, lmax: int, channels: int, rank: int, n_theta: int = 0, n_phi: int = 0,
                 dtype: str = "f32", flags: int = 0):
        lib = load_library()
        self.lmax, self.channels, self.rank = lmax, channels, rank
        self.dtype = dtype
        desc = _Desc(lmax, channels, rank, n_theta, n_phi,
                     CGTP_F64 if dtype == "f64" else CGTP_F32, flags)
        h = ctypes.c_void_p()
        _check(lib.cgtp_plan_create(ctypes.byref(desc), ctypes.byref(h)), "cgtp_plan_create")
        self.handle = h
        u, v = ctypes.c_int(), ctypes.c_int()
        _check(lib.cgtp_plan_grid(h, ctypes.byref(u), ctypes.byref(v)), "cgtp_plan_grid")
        self.n_theta, self.n_phi = u.value, v.value

    def close(self):
        if getattr(self, "handle", None):
            _check(load_library().cgtp_destroy(self.handle), "cgtp_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def plan_create(lmax: int, channels: int, rank: int, n_theta: int = 0, n_phi: int = 0,
                dtype: str = "f32", flags: int = 0) -> Plan:
    return Plan(lmax, channels, rank, n_theta, n_phi, dtype, flags)


def destroy(plan: Plan) -> None:
    plan.close()


def workspace_bytes(plan: Plan, op: int, n_nodes: int, n_edges: int = 0) -> int:
    out = ctypes.c_size_t()
    _check(load_library().cgtp_workspace_bytes(plan.handle, op, n_nodes, n_edges,
                                               ctypes.byref(out)), "cgtp_workspace_bytes")
    return out.value


def stage_times(plan: Plan, op: int):
    """cgtp_stage_times: ({stage name: summed ms}, number of calls) since the last query."""
    ms = (ctypes.c_double * 8)()
    ns, nc = ctypes.c_int(), ctypes.c_int()
    _check(load_library().cgtp_stage_times(plan.handle, op, ms, 8, ctypes.byref(ns),
                                           ctypes.byref(nc)), "cgtp_stage_times")
    names = (NBODY_STAGES if op == CGTP_OP_ONSITE_NBODY else
             ONSITE_STAGES if op == CGTP_OP_ONSITE else
             ONSITE_GENERAL_STAGES if op == CGTP_OP_ONSITE_GENERAL else MP_STAGES)
    return {names[i]: ms[i] for i in range(ns.value)}, nc.value


def _torch():
    import torch
    return torch


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream_handle(stream):
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _want(plan: Plan, name: str, t, shape, dtype=None):
    torch = _torch()
    dt = dtype or (torch.float64 if plan.dtype == "f64" else torch.float32)
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda or t.dtype != dt or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected contiguous {dt} device tensor of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def onsite(plan: Plan, A, B, U_A, U_B, U_out_even, U_out_odd, out_even=None, out_odd=None,
           workspace=None, stream=None):
    """cgtp_onsite. A, B [N, C, K]; U_* [L, C, R]; outputs [N, C, K] (allocated if not given
    and not explicitly skipped with out_even=False / out_odd=False)."""
    torch = _torch()
    N, C, K = A.shape
    L = plan.lmax + 1
    _want(plan, "A", A, (N, plan.channels, L * L))
    _want(plan, "B", B, A.shape)
    for nm, U in (("U_A", U_A), ("U_B", U_B)):
        _want(plan, nm, U, (L, plan.channels, plan.rank))
    outs = []
    for nm, o, U in (("out_even", out_even, U_out_even), ("out_odd", out_odd, U_out_odd)):
        if o is False:
            outs.append(None)
            continue
        _want(plan, nm.replace("out", "U_out"), U, (L, plan.channels, plan.rank))
        if o is None:
            o = torch.empty_like(A)
        _want(plan, nm, o, A.shape)
        outs.append(o)
    ws_ptr, ws_len = None, 0
    if workspace is not None:
        ws_ptr, ws_len = _ptr(workspace), workspace.numel() * workspace.element_size()
    _check(load_library().cgtp_onsite(plan.handle, N, _ptr(A), _ptr(B), _ptr(U_A), _ptr(U_B),
                                      _ptr(U_out_even), _ptr(U_out_odd), _ptr(outs[0]),
                                      _ptr(outs[1]), ws_ptr, ws_len, _stream_handle(stream)),
           "cgtp_onsite")
    return outs[0], outs[1]


def onsite_noalloc(plan: Plan, A, B, U_A, U_B, U_out_even, U_out_odd, out_even, out_odd,
                   stream=None):
    """cgtp_onsite_noalloc: cgtp_onsite on the library's fixed device scratch
    (CGTP_NOALLOC_SCRATCH_BYTES per GPU). The caller passes the outputs (either may be
    False to skip that slot); nothing is allocated, here or in the library."""
    N, C, K = A.shape
    L = plan.lmax + 1
    _want(plan, "A", A, (N, plan.channels, L * L))
    _want(plan, "B", B, A.shape)
    for nm, U in (("U_A", U_A), ("U_B", U_B)):
        _want(plan, nm, U, (L, plan.channels, plan.rank))
    outs = []
    for nm, o, U in (("out_even", out_even, U_out_even), ("out_odd", out_odd, U_out_odd)):
        if o is False:
            outs.append(None)
            continue
        _want(plan, nm.replace("out", "U_out"), U, (L, plan.channels, plan.rank))
        _want(plan, nm, o, A.shape)
        outs.append(o)
    _check(load_library().cgtp_onsite_noalloc(plan.handle, N, _ptr(A), _ptr(B), _ptr(U_A),
                                              _ptr(U_B), _ptr(U_out_even), _ptr(U_out_odd),
                                              _ptr(outs[0]), _ptr(outs[1]),
                                              _stream_handle(stream)),
           "cgtp_onsite_noalloc")
    return outs[0], outs[1]


def _host(a, dtype):
    """A contiguous numpy array of dtype on the host (from numpy or a torch tensor)."""
    if hasattr(a, "detach"):
        a = a.detach().cpu().numpy()
    return np.ascontiguousarray(a, dtype=dtype)


def receiver_order(row_ptr, col, edge_vec=None):
    """cgtp_receiver_order on the host: a locality-preserving permutation of the receivers
    of the CSR (row_ptr [N+1], col [E]), from the edge vectors [E, 3] if given, else the
    breadth-first order. Returns an int32 numpy array [N]."""
    rp = _host(row_ptr, np.int32)
    cl = _host(col, np.int32)
    N, E = rp.shape[0] - 1, cl.shape[0]
    ev = None if edge_vec is None else _host(edge_vec, np.float32)
    if ev is not None and ev.shape != (E, 3):
        raise ValueError(f"edge_vec: expected shape ({E}, 3), got {ev.shape}")
    out = np.empty(N, dtype=np.int32)
    vp = ctypes.c_void_p
    _check(load_library().cgtp_receiver_order(
        N, E, vp(rp.ctypes.data), vp(cl.ctypes.data),
        None if ev is None else vp(ev.ctypes.data), vp(out.ctypes.data)), "cgtp_receiver_order")
    return out


def set_receiver_order(plan: Plan, order=None) -> None:
    """cgtp_plan_set_receiver_order: run the plan's message-passing receivers in this order
    (a permutation of the N nodes; None restores the identity)."""
    lib = load_library()
    if order is None:
        _check(lib.cgtp_plan_set_receiver_order(plan.handle, 0, None),
               "cgtp_plan_set_receiver_order")
        return
    o = _host(order, np.int32)
    _check(lib.cgtp_plan_set_receiver_order(plan.handle, o.shape[0], ctypes.c_void_p(o.ctypes.data)),
           "cgtp_plan_set_receiver_order")


def gather_probe(plan: Plan, row_ptr, col, fields, sink, stream=None):
    """cgtp_gather_probe: replay the receiver's sender-field loads over fields (a device
    buffer of at least N R 3 UVs floats) for the CSR (row_ptr, col); sink: a device float."""
    torch = _torch()
    N = row_ptr.shape[0] - 1
    E = col.shape[0]
    _want(plan, "row_ptr", row_ptr, (N + 1,), torch.int32)
    _want(plan, "col", col, (E,), torch.int32)
    if not fields.is_cuda or not sink.is_cuda:
        raise ValueError("fields and sink must be device tensors")
    _check(load_library().cgtp_gather_probe(plan.handle, N, E, _ptr(row_ptr), _ptr(col),
                                            _ptr(fields), fields.numel() * fields.element_size(),
                                            _ptr(sink), _stream_handle(stream)),
           "cgtp_gather_probe")


def message_pass(plan: Plan, row_ptr, col, edge_unit, edge_radial, node_feat, U_E, U_I,
                 U_out_even, U_out_odd, out_even=None, out_odd=None, workspace=None,
                 stream=None, node_flip=None):
    """cgtp_message_pass (or cgtp_message_pass_two_slot when node_flip is given).
    row_ptr [N+1], col [E] int32; edge_unit [E, 3]; edge_radial [E, C, L];
    node_feat [N, C, K] (natural-parity slot); node_flip [N, C, K] (parity-flipped slot);
    U_* [L, C, R]; outputs [N, C, K]."""
    torch = _torch()
    N = node_feat.shape[0]
    E = col.shape[0]
    L = plan.lmax + 1
    _want(plan, "row_ptr", row_ptr, (N + 1,), torch.int32)
    _want(plan, "col", col, (E,), torch.int32)
    _want(plan, "edge_unit", edge_unit, (E, 3))
    _want(plan, "edge_radial", edge_radial, (E, plan.channels, L))
    _want(plan, "node_feat", node_feat, (N, plan.channels, L * L))
    if node_flip is not None:
        _want(plan, "node_flip", node_flip, (N, plan.channels, L * L))
    for nm, U in (("U_E", U_E), ("U_I", U_I)):
        _want(plan, nm, U, (L, plan.channels, plan.rank))
    outs = []
    for nm, o, U in (("out_even", out_even, U_out_even), ("out_odd", out_odd, U_out_odd)):
        if o is False:
            outs.append(None)
            continue
        _want(plan, nm.replace("out", "U_out"), U, (L, plan.channels, plan.rank))
        if o is None:
            o = torch.empty_like(node_feat)
        _want(plan, nm, o, node_feat.shape)
        outs.append(o)
    ws_ptr, ws_len = None, 0
    if workspace is not None:
        ws_ptr, ws_len = _ptr(workspace), workspace.numel() * workspace.element_size()
    lib = load_library()
    head = (plan.handle, N, E, _ptr(row_ptr), _ptr(col), _ptr(edge_unit), _ptr(edge_radial),
            _ptr(node_feat))
    tail = (_ptr(U_E), _ptr(U_I), _ptr(U_out_even), _ptr(U_out_odd), _ptr(outs[0]),
            _ptr(outs[1]), ws_ptr, ws_len, _stream_handle(stream))
    if node_flip is None:
        _check(lib.cgtp_message_pass(*head, *tail), "cgtp_message_pass")
    else:
        _check(lib.cgtp_message_pass_two_slot(*head, _ptr(node_flip), *tail),
               "cgtp_message_pass_two_slot")
    return outs[0], outs[1]


def workspace_bytes_general(plan: Plan, op: int, n_nodes: int, n_edges: int = 0, flips: int = 0,
                            in_blocks: int = 1, out_blocks: int = 1) -> int:
    """cgtp_workspace_bytes_general (flips: bit 0 first on-site operand, bit 1 second operand
    or node feature)."""
    out = ctypes.c_size_t()
    _check(load_library().cgtp_workspace_bytes_general(plan.handle, op, n_nodes, n_edges, flips,
                                                       in_blocks, out_blocks, ctypes.byref(out)),
           "cgtp_workspace_bytes_general")
    return out.value


def _blocks(plan: Plan, name: str, U, allowed):
    """Number of factor blocks of a stacked factor tensor: [L, C, R] is 1, [n, L, C, R] is n."""
    L = plan.lmax + 1
    base = (L, plan.channels, plan.rank)
    n = 1 if U is not None and U.dim() == 3 else (U.shape[0] if U is not None else 0)
    if n not in allowed:
        raise ValueError(f"{name}: expected {allowed} stacked blocks of {base}")
    _want(plan, name, U, base if n == 1 else (n,) + base)
    return n


def _outputs(plan: Plan, like, out_even, out_odd, U_out_even, U_out_odd):
    torch = _torch()
    outs, nout = [], set()
    for nm, o, U in (("out_even", out_even, U_out_even), ("out_odd", out_odd, U_out_odd)):
        if o is False:
            outs.append(None)
            continue
        nout.add(_blocks(plan, nm.replace("out", "U_out"), U, (1, 2)))
        if o is None:
            o = torch.empty_like(like)
        _want(plan, nm, o, like.shape)
        outs.append(o)
    if len(nout) != 1:
        raise ValueError("U_out_even and U_out_odd must have the same number of blocks")
    return outs, nout.pop()


def onsite_general(plan: Plan, A, B, U_A, U_B, U_out_even, U_out_odd, A_flip=None, B_flip=None,
                   out_even=None, out_odd=None, workspace=None, stream=None):
    """cgtp_onsite_general. A, B (and the flipped slots A_flip, B_flip) [N, C, K].
    U_A, U_B: [L, C, R], or stacked [2, L, C, R] (Gaunt, curl) or [4, L, C, R] (block
    2 * category + sector). U_out_even, U_out_odd: [L, C, R] or [2, L, C, R] (Gaunt, curl)."""
    N = A.shape[0]
    L = plan.lmax + 1
    _want(plan, "A", A, (N, plan.channels, L * L))
    for nm, X in (("B", B), ("A_flip", A_flip), ("B_flip", B_flip)):
        if X is not None or nm == "B":
            _want(plan, nm, X, A.shape)
    nin = _blocks(plan, "U_A", U_A, (1, 2, 4))
    if _blocks(plan, "U_B", U_B, (1, 2, 4)) != nin:
        raise ValueError("U_A and U_B must have the same number of blocks")
    outs, nout = _outputs(plan, A, out_even, out_odd, U_out_even, U_out_odd)
    ws_ptr, ws_len = None, 0
    if workspace is not None:
        ws_ptr, ws_len = _ptr(workspace), workspace.numel() * workspace.element_size()
    _check(load_library().cgtp_onsite_general(
        plan.handle, N, _ptr(A), _ptr(A_flip), _ptr(B), _ptr(B_flip), nin, _ptr(U_A), _ptr(U_B),
        nout, _ptr(U_out_even), _ptr(U_out_odd), _ptr(outs[0]), _ptr(outs[1]), ws_ptr, ws_len,
        _stream_handle(stream)), "cgtp_onsite_general")
    return outs[0], outs[1]


def message_pass_general(plan: Plan, row_ptr, col, edge_unit, edge_radial, node_feat, U_E, U_I,
                         U_out_even, U_out_odd, node_flip=None, out_even=None, out_odd=None,
                         workspace=None, stream=None):
    """cgtp_message_pass_general. Arguments as in message_pass; U_E, U_I and U_out_* stacked
    as in onsite_general."""
    torch = _torch()
    N = node_feat.shape[0]
    E = col.shape[0]
    L = plan.lmax + 1
    _want(plan, "row_ptr", row_ptr, (N + 1,), torch.int32)
    _want(plan, "col", col, (E,), torch.int32)
    _want(plan, "edge_unit", edge_unit, (E, 3))
    _want(plan, "edge_radial", edge_radial, (E, plan.channels, L))
    _want(plan, "node_feat", node_feat, (N, plan.channels, L * L))
    if node_flip is not None:
        _want(plan, "node_flip", node_flip, node_feat.shape)
    nin = _blocks(plan, "U_E", U_E, (1, 2, 4))
    if _blocks(plan, "U_I", U_I, (1, 2, 4)) != nin:
        raise ValueError("U_E and U_I must have the same number of blocks")
    outs, nout = _outputs(plan, node_feat, out_even, out_odd, U_out_even, U_out_odd)
    ws_ptr, ws_len = None, 0
    if workspace is not None:
        ws_ptr, ws_len = _ptr(workspace), workspace.numel() * workspace.element_size()
    _check(load_library().cgtp_message_pass_general(
        plan.handle, N, E, _ptr(row_ptr), _ptr(col), _ptr(edge_unit), _ptr(edge_radial),
        _ptr(node_feat), _ptr(node_flip), nin, _ptr(U_E), _ptr(U_I), nout, _ptr(U_out_even),
        _ptr(U_out_odd), _ptr(outs[0]), _ptr(outs[1]), ws_ptr, ws_len, _stream_handle(stream)),
        "cgtp_message_pass_general")
    return outs[0], outs[1]


def message_pass_fields(plan: Plan, row_ptr, col, edge_feat, node_feat, U_E, U_I, U_out_even,
                        U_out_odd, edge_flip=None, node_flip=None, out_even=None, out_odd=None,
                        workspace=None, stream=None):
    """cgtp_message_pass_fields (two parity-bearing fields). row_ptr [N+1], col [E] int32;
    edge_feat, edge_flip [E, C, K]; node_feat, node_flip [N, C, K]; factors stacked as in
    onsite_general."""
    torch = _torch()
    N = node_feat.shape[0]
    E = col.shape[0]
    L = plan.lmax + 1
    _want(plan, "row_ptr", row_ptr, (N + 1,), torch.int32)
    _want(plan, "col", col, (E,), torch.int32)
    _want(plan, "edge_feat", edge_feat, (E, plan.channels, L * L))
    if edge_flip is not None:
        _want(plan, "edge_flip", edge_flip, edge_feat.shape)
    _want(plan, "node_feat", node_feat, (N, plan.channels, L * L))
    if node_flip is not None:
        _want(plan, "node_flip", node_flip, node_feat.shape)
    nin = _blocks(plan, "U_E", U_E, (1, 2, 4))
    if _blocks(plan, "U_I", U_I, (1, 2, 4)) != nin:
        raise ValueError("U_E and U_I must have the same number of blocks")
    outs, nout = _outputs(plan, node_feat, out_even, out_odd, U_out_even, U_out_odd)
    ws_ptr, ws_len = None, 0
    if workspace is not None:
        ws_ptr, ws_len = _ptr(workspace), workspace.numel() * workspace.element_size()
    _check(load_library().cgtp_message_pass_fields(
        plan.handle, N, E, _ptr(row_ptr), _ptr(col), _ptr(edge_feat), _ptr(edge_flip),
        _ptr(node_feat), _ptr(node_flip), nin, _ptr(U_E), _ptr(U_I), nout, _ptr(U_out_even),
        _ptr(U_out_odd), _ptr(outs[0]), _ptr(outs[1]), ws_ptr, ws_len, _stream_handle(stream)),
        "cgtp_message_pass_fields")
    return outs[0], outs[1]


def nbody_grid(lmax: int, nu: int):
    """Smallest (n_theta, n_phi) on which cgtp_onsite_nbody is exact for nu operands."""
    deg = (nu + 1) * lmax
    return max(1, (deg + 2) // 2), deg + 1


def workspace_bytes_nbody(plan: Plan, n_nodes: int, nu: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().cgtp_workspace_bytes_nbody(plan.handle, n_nodes, nu,
                                                     ctypes.byref(out)),
           "cgtp_workspace_bytes_nbody")
    return out.value


def onsite_nbody(plan: Plan, X, U, U_out, out=None, workspace=None, stream=None):
    """cgtp_onsite_nbody. X: sequence of nu device tensors [N, C, K]; U: nu factor tensors
    [L, C, R]; U_out [L, C, R]. The plan's grid must be at least nbody_grid(lmax, nu)."""
    torch = _torch()
    nu = len(X)
    if nu != len(U) or nu < 1:
        raise ValueError("X and U must hold the same number (>= 1) of operands")
    L = plan.lmax + 1
    N = X[0].shape[0]
    for t in range(nu):
        _want(plan, f"X[{t}]", X[t], (N, plan.channels, L * L))
        _want(plan, f"U[{t}]", U[t], (L, plan.channels, plan.rank))
    _want(plan, "U_out", U_out, (L, plan.channels, plan.rank))
    if out is None:
        out = torch.empty_like(X[0])
    _want(plan, "out", out, X[0].shape)
    xs = (ctypes.c_void_p * nu)(*[x.data_ptr() for x in X])
    us = (ctypes.c_void_p * nu)(*[u.data_ptr() for u in U])
    ws_ptr, ws_len = None, 0
    if workspace is not None:
        ws_ptr, ws_len = _ptr(workspace), workspace.numel() * workspace.element_size()
    _check(load_library().cgtp_onsite_nbody(plan.handle, N, nu, ctypes.cast(xs, ctypes.c_void_p),
                                            ctypes.cast(us, ctypes.c_void_p), _ptr(U_out),
                                            _ptr(out), ws_ptr, ws_len, _stream_handle(stream)),
           "cgtp_onsite_nbody")
    return out


def host_tables(lmax: int, n_theta: int = 0, n_phi: int = 0):
    """fp64 grid tables (x, w, p, dp, q) as the plan builds them; host only."""
    import numpy as np

    lib = load_library()
    u, v = n_theta, n_phi
    if u == 0:
        u = (3 * lmax + 3) // 2
    if v == 0:
        v = 3 * lmax + 1
    P = (lmax + 1) * (lmax + 2) // 2
    x, w = np.zeros(u), np.zeros(u)
    p, dp = np.zeros((u, P)), np.zeros((u, P))
    q = np.zeros((v, 2 * lmax + 1))
    args = [ctypes.c_void_p(a.ctypes.data) for a in (x, w, p, dp, q)]
    _check(lib.cgtp_host_tables(lmax, n_theta, n_phi, *args), "cgtp_host_tables")
    return x, w, p, dp, q


# ---------------------------------------------------------------- row operators

def _row_dtype(name, t):
    torch = _torch()
    if t.dtype == torch.float32:
        return CGTP_F32
    if t.dtype == torch.bfloat16:
        return CGTP_BF16
    raise ValueError(f"{name}: expected float32 or bfloat16, got {t.dtype}")


def _want_rows(name, t, n, width, like):
    """[n, width] rows on like's device, of like's type, contiguous along the width; returns the
    row stride."""
    if t.shape == (n, width) and t.dtype == like.dtype and t.device == like.device:
        row, step = t.stride()
        if n <= 1:
            if step == 1 or width == 1 or n == 0:
                return width
        elif (step == 1 or width == 1) and row >= width:
            return row
    raise ValueError(f"{name}: expected {like.dtype} rows ({n}, {width}) on {like.device}, contiguous "
                     f"along the width, got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on "
                     f"{t.device}")


def _want_dev(name, t, shape, dtype, like):
    """A contiguous tensor on like's device, which is a GPU (checked by _row_call)."""
    if t.device != like.device or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} tensor of shape {tuple(shape)} on "
                         f"{like.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


@functools.lru_cache(maxsize=1)
def _current():
    """(handle of the current stream of a device, number of the current device). A Stream object costs a
    tenth of a small call, so torch's own handle of it is taken where this torch has such a call."""
    torch = _torch()
    return (getattr(torch._C, "_cuda_getCurrentRawStream",
                    lambda index: torch.cuda.current_stream(index).cuda_stream),
            getattr(torch._C, "_cuda_getDevice", lambda: torch.cuda.current_device()))


def _row_call(like, stream):
    """(handle of the stream that a call on like's device runs on, the stream if it is not the
    current one). Work on another stream waits for what the current one has pending, whether the call
    allocates or not; what reads its results is for the caller to order."""
    torch = _torch()
    if not like.is_cuda:
        raise ValueError(f"expected device tensors, got one on {like.device}")
    current = _current()[0](like.device.index)
    if stream is None or stream.cuda_stream == current:
        return current, None
    stream.wait_stream(torch.cuda.current_stream(like.device))
    return stream.cuda_stream, stream


def _new(shape, dtype, like):
    return _torch().empty(shape, dtype=dtype, device=like.device)


def _row_workspace(workspace, need, like):
    """(pointer, bytes, the tensor) of the caller's workspace or of a new one."""
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = _new((need,), _torch().uint8, like)
    elif workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on {like.device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


@functools.lru_cache(maxsize=1024)
def _bytes(name, *args):
    out = ctypes.c_size_t()
    _check(getattr(load_library(), name)(*args, ctypes.byref(out)), name)
    return out.value


def _run(name, like, side, tensors, *args):
    """The call on like's device. Pointers are integers or None. Where it runs on the stream side, the
    memory of its tensors is not reused before that stream is done with them."""
    torch = _torch()
    if side is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(side)
    if _current()[1]() == like.device.index:
        status = getattr(_lib, name)(*args)
    else:
        with torch.cuda.device(like.device):
            status = getattr(_lib, name)(*args)
    if status != CGTP_OK:
        _check(status, name)


def _addr(t):
    return None if t is None else t.data_ptr()


def _want_order(offsets, order, n, G, like):
    torch = _torch()
    _want_dev("offsets", offsets, (G + 1,), torch.int32, like)
    if order is not None:
        _want_dev("order", order, (n,), torch.int32, like)


def group_rows(ids, n_groups: int, offsets=None, order=None, workspace=None, stream=None):
    """cgtp_group_rows: (offsets [n_groups + 1], order [n]) of the rows with group ids [n] (int32;
    a row whose id is outside [0, n_groups) belongs to no group and comes last)."""
    torch = _torch()
    if ids.dim() != 1:
        raise ValueError(f"ids: expected one dimension, got {tuple(ids.shape)}")
    n = ids.shape[0]
    handle, side = _row_call(ids, stream)
    _want_dev("ids", ids, (n,), torch.int32, ids)
    need = _bytes("cgtp_group_rows_bytes", n, n_groups)
    if offsets is None:
        offsets = _new((n_groups + 1,), torch.int32, ids)
    if order is None:
        order = _new((n,), torch.int32, ids)
    _want_order(offsets, order, n, n_groups, ids)
    ws_ptr, ws_len, ws = _row_workspace(workspace, need, ids)
    _run("cgtp_group_rows", ids, side, (ids, offsets, order, ws), n, n_groups, ids.data_ptr(), offsets.data_ptr(), order.data_ptr(),
         ws_ptr, ws_len, handle)
    return offsets, order


def _linear_head(x, w, offsets, order, shared):
    if x.dim() != 2 or w.dim() != (2 if shared else 3):
        raise ValueError(f"x, w: expected 2 and {2 if shared else 3} dimensions, got "
                         f"{tuple(x.shape)} and {tuple(w.shape)}")
    load_library()
    n, (n_in, n_out) = x.shape[0], w.shape[-2:]
    G = offsets.shape[0] - 1
    _want_order(offsets, order, n, G, x)
    _want_dev("w", w, (n_in, n_out) if shared else (G, n_in, n_out), x.dtype, x)
    return _row_dtype("x", x), n, G, n_in, n_out, _want_rows("x", x, n, n_in, x)


def grouped_linear(x, w, offsets, order=None, y=None, stream=None):
    """cgtp_grouped_linear: y_i = w[g(i)]^T x_i (0 for a row of no group). x [n, n_in] and
    y [n, n_out] rows (any row stride), w [G, n_in, n_out]; offsets, order from group_rows (order
    None: the rows are sorted by group)."""
    dt, n, G, n_in, n_out, xs = _linear_head(x, w, offsets, order, False)
    handle, side = _row_call(x, stream)
    if y is None:
        y = _new((n, n_out), x.dtype, x)
    ys = _want_rows("y", y, n, n_out, x)
    _run("cgtp_grouped_linear", x, side, (x, w, offsets, order, y), dt, n, G, n_in, n_out, _addr(offsets), _addr(order), _addr(x),
         xs, _addr(w), _addr(y), ys, handle)
    return y


def _grad_out(name, out, shape, like, rows):
    """An output of a gradient call: allocated if None, skipped if False; (tensor, row stride)."""
    if out is False:
        return None, 0
    if out is None:
        return _new(shape, like.dtype, like), shape[-1] if rows else 0
    if rows:
        return out, _want_rows(name, out, *shape, like)
    _want_dev(name, out, shape, like.dtype, like)
    return out, 0


def grouped_linear_grad(x, w, dy, offsets, order=None, dx=None, dw=None, workspace=None,
                        stream=None):
    """cgtp_grouped_linear_grad: (dx [n, n_in], dw [G, n_in, n_out]) from dy [n, n_out]; an output
    given as False is skipped (None in its place)."""
    dt, n, G, n_in, n_out, xs = _linear_head(x, w, offsets, order, False)
    dys = _want_rows("dy", dy, n, n_out, x)
    handle, side = _row_call(x, stream)
    dx, dxs = _grad_out("dx", dx, (n, n_in), x, True)
    dw, _ = _grad_out("dw", dw, (G, n_in, n_out), x, False)
    ws_ptr, ws_len, ws = None, 0, None
    if dw is not None:
        need = _bytes("cgtp_grouped_linear_grad_bytes", dt, n, G, n_in, n_out)
        ws_ptr, ws_len, ws = _row_workspace(workspace, need, x)
    _run("cgtp_grouped_linear_grad", x, side, (x, w, dy, offsets, order, dx, dw, ws), dt, n, G, n_in, n_out, _addr(offsets), _addr(order),
         _addr(x), xs, _addr(w), _addr(dy), dys, _addr(dx), dxs, _addr(dw), ws_ptr, ws_len, handle)
    return dx, dw


def _adapter_head(x, w, a, b, offsets, order, scale):
    head = _linear_head(x, w, offsets, order, True)
    dt, n, G, n_in, n_out, xs = head
    if a.dim() != 3:
        raise ValueError(f"a: expected three dimensions, got {tuple(a.shape)}")
    r = a.shape[2]
    _want_dev("a", a, (G, n_in, r), x.dtype, x)
    _want_dev("b", b, (G, r, n_out), x.dtype, x)
    if scale is not None:
        _want_dev("scale", scale, (G,), _torch().float32, x)
    return head, r


def adapter_linear(x, w, a, b, offsets, order=None, scale=None, y=None, workspace=None,
                   stream=None):
    """cgtp_adapter_linear: y_i = w^T x_i + scale[g] b[g]^T (a[g]^T x_i), g = g(i). x [n, n_in] and
    y [n, n_out] rows, w [n_in, n_out] shared, a [G, n_in, r], b [G, r, n_out], scale [G] float32
    or None (1)."""
    (dt, n, G, n_in, n_out, xs), r = _adapter_head(x, w, a, b, offsets, order, scale)
    handle, side = _row_call(x, stream)
    if y is None:
        y = _new((n, n_out), x.dtype, x)
    ys = _want_rows("y", y, n, n_out, x)
    need = _bytes("cgtp_adapter_linear_bytes", dt, n, G, n_in, n_out, r)
    ws_ptr, ws_len, ws = _row_workspace(workspace, need, x)
    _run("cgtp_adapter_linear", x, side, (x, w, a, b, offsets, order, scale, y, ws), dt, n, G, n_in, n_out, r, _addr(offsets), _addr(order), _addr(x),
         xs, _addr(w), _addr(a), _addr(b), _addr(scale), _addr(y), ys, ws_ptr, ws_len, handle)
    return y


def adapter_linear_grad(x, w, a, b, dy, offsets, order=None, scale=None, dx=None, da=None, db=None,
                        workspace=None, stream=None):
    """cgtp_adapter_linear_grad: (dx, da, db) from dy [n, n_out], the shared projection frozen; an
    output given as False is skipped (None in its place)."""
    (dt, n, G, n_in, n_out, xs), r = _adapter_head(x, w, a, b, offsets, order, scale)
    dys = _want_rows("dy", dy, n, n_out, x)
    handle, side = _row_call(x, stream)
    dx, dxs = _grad_out("dx", dx, (n, n_in), x, True)
    da, _ = _grad_out("da", da, (G, n_in, r), x, False)
    db, _ = _grad_out("db", db, (G, r, n_out), x, False)
    need = _bytes("cgtp_adapter_linear_grad_bytes", dt, n, G, n_in, n_out, r)
    ws_ptr, ws_len, ws = _row_workspace(workspace, need, x)
    _run("cgtp_adapter_linear_grad", x, side, (x, w, a, b, dy, offsets, order, scale, dx, da, db, ws), dt, n, G, n_in, n_out, r, _addr(offsets), _addr(order),
         _addr(x), xs, _addr(w), _addr(a), _addr(b), _addr(scale), _addr(dy), dys, _addr(dx), dxs,
         _addr(da), _addr(db), ws_ptr, ws_len, handle)
    return dx, da, db


def _out_rows(name, out, n, width, like):
    """Rows that a call writes, allocated if None; (tensor, row stride)."""
    return (_new((n, width), like.dtype, like), width) if out is None else (out, _want_rows(name, out, n, width, like))


_SCORES = {"softmax": CGTP_SCORE_SOFTMAX, "sigmoid": CGTP_SCORE_SIGMOID}
_ACTIVATIONS = {None: CGTP_ACT_NONE, "silu": CGTP_ACT_SILU, "gelu": CGTP_ACT_GELU, "relu": CGTP_ACT_RELU}


def _choice(name, value, known):
    try:
        return known[value]
    except (KeyError, TypeError):
        raise ValueError(f"{name}: expected one of {list(known)}, got {value!r}") from None


def _route_head(logits, top_k, score):
    if logits.dim() != 2:
        raise ValueError(f"logits: expected two dimensions, got {tuple(logits.shape)}")
    load_library()
    n, E = logits.shape
    return (_row_dtype("logits", logits), n, E, top_k, _want_rows("logits", logits, n, E, logits),
            _choice("score", score, _SCORES))


def route_rows(logits, top_k: int, bias=None, score: str = "softmax", n_blocks: int = 1, keep_blocks=None,
               renormalize: bool = True, scale: float = 1.0, ids=None, weights=None, stream=None):
    """cgtp_route_rows: (ids [n, top_k] int32, weights [n, top_k] float32) of the experts that the rows of
    logits [n, E] are routed to: by "softmax" or "sigmoid" scores, with bias [E] float32 added for the choice
    alone, among the best keep_blocks (None: all) of n_blocks blocks of experts. ids.view(-1) is what group_rows
    orders."""
    torch = _torch()
    dt, n, E, k, ls, code = _route_head(logits, top_k, score)
    handle, side = _row_call(logits, stream)
    if bias is not None:
        _want_dev("bias", bias, (E,), torch.float32, logits)
    shape = (n, max(k, 0))
    if ids is None:
        ids = _new(shape, torch.int32, logits)
    else:
        _want_dev("ids", ids, shape, torch.int32, logits)
    if weights is None:
        weights = _new(shape, torch.float32, logits)
    else:
        _want_dev("weights", weights, shape, torch.float32, logits)
    _run("cgtp_route_rows", logits, side, (logits, bias, ids, weights), dt, n, E, k, _addr(logits), ls, _addr(bias), code,
         n_blocks, n_blocks if keep_blocks is None else keep_blocks, int(bool(renormalize)), scale, _addr(ids),
         _addr(weights), handle)
    return ids, weights


def route_rows_grad(logits, ids, dweights, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                    dlogits=None, stream=None):
    """cgtp_route_rows_grad: dlogits [n, E] from dweights [n, top_k] float32, with the ids, logits and options of
    the forward call."""
    torch = _torch()
    if ids.dim() != 2:
        raise ValueError(f"ids: expected two dimensions, got {tuple(ids.shape)}")
    dt, n, E, k, ls, code = _route_head(logits, ids.shape[1], score)
    handle, side = _row_call(logits, stream)
    _want_dev("ids", ids, (n, k), torch.int32, logits)
    _want_dev("dweights", dweights, (n, k), torch.float32, logits)
    dlogits, ds = _out_rows("dlogits", dlogits, n, E, logits)
    _run("cgtp_route_rows_grad", logits, side, (logits, ids, dweights, dlogits), dt, n, E, k, _addr(logits), ls, _addr(ids),
         _addr(dweights), code, int(bool(renormalize)), scale, _addr(dlogits), ds, handle)
    return dlogits


def _layer_head(x, w, offsets, order, per_row):
    if x.dim() != 2 or w.dim() != 3:
        raise ValueError(f"x, w: expected 2 and 3 dimensions, got {tuple(x.shape)} and {tuple(w.shape)}")
    load_library()
    t, (n_in, n_out) = x.shape[0], w.shape[-2:]
    n, G = t * per_row, offsets.shape[0] - 1
    _want_order(offsets, order, n, G, x)
    _want_dev("w", w, (G, n_in, n_out), x.dtype, x)
    return _row_dtype("x", x), t, n, G, n_in, n_out, _want_rows("x", x, t, n_in, x)


def grouped_layer(x, w, offsets, order=None, bias=None, activation=None, residual=None, per_row: int = 1, y=None,
                  z=False, stream=None):
    """cgtp_grouped_layer: y_i = act(w[g]^T x_t + bias[g]) + residual_i, g = g(i), t = i // per_row. x [t, n_in];
    residual and y [t * per_row, n_out] rows, w [G, n_in, n_out], bias [G, n_out]; activation None, "silu", "gelu"
    or "relu". offsets, order from group_rows over the t * per_row rows. With z None or a tensor, what the
    activation took is kept and (y, z) returned."""
    dt, t, n, G, n_in, n_out, xs = _layer_head(x, w, offsets, order, per_row)
    act = _choice("activation", activation, _ACTIVATIONS)
    handle, side = _row_call(x, stream)
    if bias is not None:
        _want_dev("bias", bias, (G, n_out), x.dtype, x)
    rs = 0 if residual is None else _want_rows("residual", residual, n, n_out, x)
    y, ys = _out_rows("y", y, n, n_out, x)
    kept, zs = _grad_out("z", z, (n, n_out), x, True)
    _run("cgtp_grouped_layer", x, side, (x, w, offsets, order, bias, residual, y, kept), dt, n, G, n_in, n_out, per_row,
         _addr(offsets), _addr(order), _addr(x), xs, _addr(w), _addr(bias), act, _addr(residual), rs, _addr(y), ys,
         _addr(kept), zs, handle)
    return y if kept is None else (y, kept)


def grouped_layer_grad(x, w, dy, offsets, order=None, z=None, activation=None, per_row: int = 1, dx=None, dw=None,
                       dbias=None, workspace=None, stream=None):
    """cgtp_grouped_layer_grad: (dx [t, n_in], dw [G, n_in, n_out], dbias [G, n_out]) from dy [t * per_row, n_out]
    and the z that the forward call kept (not needed without an activation); an output given as False is skipped
    (None in its place)."""
    dt, t, n, G, n_in, n_out, xs = _layer_head(x, w, offsets, order, per_row)
    act = _choice("activation", activation, _ACTIVATIONS)
    dys = _want_rows("dy", dy, n, n_out, x)
    if act == CGTP_ACT_NONE:
        z, zs = None, 0
    elif z is None:
        raise ValueError("z: needed where there is an activation")
    else:
        zs = _want_rows("z", z, n, n_out, x)
    handle, side = _row_call(x, stream)
    dx, dxs = _grad_out("dx", dx, (t, n_in), x, True)
    dw, _ = _grad_out("dw", dw, (G, n_in, n_out), x, False)
    dbias, _ = _grad_out("dbias", dbias, (G, n_out), x, False)
    need = _bytes("cgtp_grouped_layer_grad_bytes", dt, n, G, n_in, n_out, 1 if dx is None else per_row, act)
    ws_ptr, ws_len, ws = _row_workspace(workspace, need, x)
    _run("cgtp_grouped_layer_grad", x, side, (x, w, dy, z, offsets, order, dx, dw, dbias, ws), dt, n, G, n_in, n_out, per_row,
         _addr(offsets), _addr(order), _addr(x), xs, _addr(w), _addr(z), zs, act, _addr(dy), dys, _addr(dx), dxs,
         _addr(dw), _addr(dbias), ws_ptr, ws_len, handle)
    return dx, dw, dbias


def _mix_rows_of(name, y, per_row):
    if y.dim() != 2:
        raise ValueError(f"{name}: expected two dimensions, got {tuple(y.shape)}")
    if per_row < 1 or y.shape[0] % per_row != 0:
        raise ValueError(f"{name}: {y.shape[0]} rows are no multiple of per_row {per_row}")
    return y.shape[0] // per_row, y.shape[1]


def mix_rows(y, per_row: int, weights=None, residual=None, out=None, stream=None):
    """cgtp_mix_rows: out_t = residual_t + sum_j weights[t][j] y_(t per_row + j). y [t * per_row, width] rows,
    weights [t, per_row] float32 or None (1), residual and out [t, width] rows."""
    load_library()
    n, width = _mix_rows_of("y", y, per_row)
    dt, ys = _row_dtype("y", y), _want_rows("y", y, n * per_row, width, y)
    handle, side = _row_call(y, stream)
    if weights is not None:
        _want_dev("weights", weights, (n, per_row), _torch().float32, y)
    rs = 0 if residual is None else _want_rows("residual", residual, n, width, y)
    out, outs = _out_rows("out", out, n, width, y)
    _run("cgtp_mix_rows", y, side, (y, weights, residual, out), dt, n, per_row, width, _addr(y), ys, _addr(weights),
         _addr(residual), rs, _addr(out), outs, handle)
    return out


def mix_rows_grad(dout, per_row: int, weights=None, y=None, dy=None, dweights=None, stream=None):
    """cgtp_mix_rows_grad: (dy [t * per_row, width], dweights [t, per_row] float32) from dout [t, width]; an output
    given as False is skipped (None in its place). dweights needs y."""
    torch = _torch()
    load_library()
    if dout.dim() != 2:
        raise ValueError(f"dout: expected two dimensions, got {tuple(dout.shape)}")
    n, width = dout.shape
    dt, ds = _row_dtype("dout", dout), _want_rows("dout", dout, n, width, dout)
    handle, side = _row_call(dout, stream)
    if weights is not None:
        _want_dev("weights", weights, (n, per_row), torch.float32, dout)
    dy, dys = _grad_out("dy", dy, (n * per_row, width), dout, True)
    ys = 0
    if dweights is False:
        dweights = None
    else:
        if y is None:
            raise ValueError("y: needed for dweights")
        ys = _want_rows("y", y, n * per_row, width, dout)
        if dweights is None:
            dweights = _new((n, per_row), torch.float32, dout)
        else:
            _want_dev("dweights", dweights, (n, per_row), torch.float32, dout)
    _run("cgtp_mix_rows_grad", dout, side, (dout, weights, y, dy, dweights), dt, n, per_row, width, _addr(dout), ds,
         _addr(weights), _addr(y) if dweights is not None else None, ys, _addr(dy), dys, _addr(dweights), handle)
    return dy, dweights


class AdamWTensors:
    """Owns a cgtp_adamw handle over lists of device tensors, which it keeps alive: params (float32),
    grads (all float32 or all bfloat16), the moments m and v (float32; or int8 and uint8 with the
    float32 scales m_scale and v_scale, one per CGTP_ADAMW_BLOCK elements) and, if given, bfloat16
    copies of the parameters that each step writes. All contiguous, on one device; grads are read
    where they lie when a step runs."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None):
        torch = _torch()
        lists = [params, grads, m, v, m_scale, v_scale, copies]
        n = len(params)
        if n == 0 or any(x is not None and len(x) != n for x in lists):
            raise ValueError("params, grads, m, v (, scales, copies): lists of one length >= 1")
        if (m_scale is None) != (v_scale is None):
            raise ValueError("m_scale and v_scale: both or neither")
        if not params[0].is_cuda:
            raise ValueError(f"params[0]: expected a device tensor, got one on {params[0].device}")
        bits = 32 if m_scale is None else 8
        gdt = grads[0].dtype
        self.state_bits, self.device = bits, params[0].device
        code = _row_dtype("grads", grads[0])
        table = (_AdamWTensor * n)()
        for i in range(n):
            k = params[i].numel()
            shape, nb = params[i].shape, ((k + CGTP_ADAMW_BLOCK - 1) // CGTP_ADAMW_BLOCK,)
            _want_dev(f"params[{i}]", params[i], shape, torch.float32, params[0])
            _want_dev(f"grads[{i}]", grads[i], shape, gdt, params[0])
            _want_dev(f"m[{i}]", m[i], shape, torch.float32 if bits == 32 else torch.int8, params[0])
            _want_dev(f"v[{i}]", v[i], shape, torch.float32 if bits == 32 else torch.uint8,
                      params[0])
            row = dict(param=params[i], grad=grads[i], m=m[i], v=v[i])
            if bits == 8:
                _want_dev(f"m_scale[{i}]", m_scale[i], nb, torch.float32, params[0])
                _want_dev(f"v_scale[{i}]", v_scale[i], nb, torch.float32, params[0])
                row.update(m_scale=m_scale[i], v_scale=v_scale[i])
            if copies is not None:
                _want_dev(f"copies[{i}]", copies[i], shape, torch.bfloat16, params[0])
                row.update(copy=copies[i])
            for name, t in row.items():
                setattr(table[i], name, t.data_ptr())
            table[i].n = k
        self._keep = [list(x) for x in lists if x is not None]
        self.shapes = [p.shape for p in params]
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(load_library().cgtp_adamw_create(n, table, code, bits, ctypes.byref(h)),
                   "cgtp_adamw_create")
        self.handle = h
        need = ctypes.c_size_t()
        _check(load_library().cgtp_adamw_grad_norm_bytes(h, ctypes.byref(need)), "cgtp_adamw_grad_norm_bytes")
        # for adamw_grad_norm: like the tensors it serves one stream at a time, and lives until close() has waited
        self._norm_workspace = torch.empty(need.value, dtype=torch.uint8, device=self.device)

    def close(self):
        if getattr(self, "handle", None):
            with _torch().cuda.device(self.device):
                _check(load_library().cgtp_adamw_destroy(self.handle), "cgtp_adamw_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def adamw(tensors: AdamWTensors, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
          eps: float = 1e-8, weight_decay: float = 0.01, grad_scale=None, stream=None) -> None:
    """cgtp_adamw_step: update the tensors of the handle in place. step counts from 1; grad_scale: a
    device float32 tensor of one element that multiplies every gradient (clipping), or None. The
    handle's tensors live as long as it does, and closing it waits for the device."""
    first = tensors._keep[0][0]
    if grad_scale is not None:
        _want_dev("grad_scale", grad_scale, (1,), _torch().float32, first)
    handle, side = _row_call(first, stream)
    _run("cgtp_adamw_step", first, side, (grad_scale,), tensors.handle, lr, beta1, beta2, eps, weight_decay, step,
         _addr(grad_scale), handle)


def adamw_states(tensors: AdamWTensors, m_out=None, v_out=None, stream=None):
    """cgtp_adamw_states: the float32 values that 8-bit states stand for, as lists (m, v)."""
    torch = _torch()
    first = tensors._keep[0][0]
    handle, side = _row_call(first, stream)
    outs = []
    for name, given in (("m_out", m_out), ("v_out", v_out)):
        if given is None:
            given = [_new(shape, torch.float32, first) for shape in tensors.shapes]
        if len(given) != len(tensors.shapes):
            raise ValueError(f"{name}: expected {len(tensors.shapes)} tensors, got {len(given)}")
        for i, (t, shape) in enumerate(zip(given, tensors.shapes)):
            _want_dev(f"{name}[{i}]", t, shape, torch.float32, first)
        outs.append(given)
    arrays = [(ctypes.c_void_p * len(o))(*[t.data_ptr() for t in o]) for o in outs]
    _run("cgtp_adamw_states", first, side, (*outs[0], *outs[1]), tensors.handle, arrays[0], arrays[1], handle)
    return outs[0], outs[1]


def adamw_grad_norm(tensors: AdamWTensors, max_norm: float, grad_scale=None, norm=None, scale=None, workspace=None,
                    stream=None):
    """cgtp_adamw_grad_norm: (norm, scale), device float32 tensors of one element: the norm of all gradients of the
    handle times |grad_scale|, and grad_scale min(1, max_norm / norm), the grad_scale of the adamw call that
    follows. An output given as False is skipped (None in its place)."""
    torch = _torch()
    first = tensors._keep[0][0]
    handle, side = _row_call(first, stream)
    if grad_scale is not None:
        _want_dev("grad_scale", grad_scale, (1,), torch.float32, first)
    outs = []
    for name, out in (("norm", norm), ("scale", scale)):
        if out is None:
            out = _new((1,), torch.float32, first)
        elif out is not False:
            _want_dev(name, out, (1,), torch.float32, first)
        outs.append(None if out is False else out)
    ws_ptr, ws_len, ws = _row_workspace(tensors._norm_workspace if workspace is None else workspace, 0, first)
    _run("cgtp_adamw_grad_norm", first, side, (grad_scale, *outs, ws), tensors.handle, max_norm, _addr(grad_scale),
         _addr(outs[0]), _addr(outs[1]), ws_ptr, ws_len, handle)
    return tuple(outs)
