"""Thin ctypes binding over libnacho.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU, passes their
device pointers through the C ABI declared in include/nacho.h and returns the
status code handling to `_check`.  PyTorch is used for device memory and the
current stream; no step of the hot path runs in Python or in torch.

The library must have been built (`paper_2604_17198_amd.build.build()`); a
missing library is an error, there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import build as _build

F32, F64, BF16, F16 = 0, 1, 2, 3
DENSE, COMPRESSED, NONUNIQUE, SINGLETON = 0, 1, 2, 3
OP_PARTITION, OP_SPMV, OP_SPMM, OP_SPADD, OP_SPMUL = 0, 1, 2, 3, 4
MAX_OPERANDS, MAX_LEVELS = 8, 3

EXPORTS = [
    "nacho_version", "nacho_status_string", "nacho_num_partitions", "nacho_workspace_bytes",
    "nacho_partition", "nacho_spmv", "nacho_spmm", "nacho_spadd_k", "nacho_spmul_k", "nacho_workspace_parts",
    "nacho_validate", "nacho_profile_enable", "nacho_profile_read", "nacho_spmv_static",
    "nacho_static_scratch_bytes", "nacho_instrument", "nacho_instrument_record_bytes", "nacho_instrument_wait",
    "nacho_probe", "nacho_merge_wavefronts", "nacho_rowcost_partitions", "nacho_partition_rowcost",
    "nacho_spmv_rowcost", "nacho_partition_csr64", "nacho_spmv_fused", "nacho_spadd_fused",
    "nacho_distill_workspace_bytes", "nacho_distill", "nacho_distill_grad",
    "nacho_route_workspace_bytes", "nacho_route", "nacho_route_grad", "nacho_combine",
    "nacho_combine_grad", "nacho_experts_workspace_bytes", "nacho_experts", "nacho_experts_grad",
]


class NachoError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _Level(C.Structure):
    _fields_ = [("kind", C.c_int32), ("extent", C.c_int64), ("pos", C.c_void_p),
                ("crd", C.c_void_p), ("count", C.c_int64)]


class _Tensor(C.Structure):
    _fields_ = [("nlevels", C.c_int32), ("lvl", _Level * MAX_LEVELS), ("val", C.c_void_p)]


class _Parts(C.Structure):
    _fields_ = [("k", C.c_int32), ("d", C.c_int32), ("P", C.c_int64), ("coord", C.c_void_p),
                ("posn", C.c_void_p), ("cost", C.c_void_p)]


class _SparseOut(C.Structure):
    _fields_ = [("pos0", C.c_void_p), ("crd0", C.c_void_p), ("pos1", C.c_void_p),
                ("crd1", C.c_void_p), ("val", C.c_void_p), ("cap_rows", C.c_int64),
                ("cap_nnz", C.c_int64), ("counts", C.c_void_p), ("status", C.c_void_p),
                ("pos2", C.c_void_p), ("crd2", C.c_void_p), ("cap_fibres", C.c_int64)]


class _Routing(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pos", "expert", "gate", "slot", "expert_pos", "token", "counts", "lse",
                                          "balance", "routed")]


class _ExpertsLayer(C.Structure):
    _fields_ = [("expert_pos", C.c_void_p), ("token", C.c_void_p), ("n_experts", C.c_int64), ("n_slots", C.c_int64),
                ("n_tokens", C.c_int64), ("inner", C.c_int64), ("outer", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("w", C.c_void_p), ("ldw", C.c_int64), ("w_stride", C.c_int64), ("bias", C.c_void_p),
                ("bias_stride", C.c_int64), ("act", C.c_int32), ("dtype", C.c_int32)]


_lib = None
_libs = {}
_instrumented = False


def select_library(instrumented: bool):
    """Route all calls to libnacho.so (default) or to libnacho_instr.so, the instrumented build."""
    global _lib, _instrumented
    _instrumented = bool(instrumented)
    _lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None and _instrumented in _libs:
        _lib = _libs[_instrumented]
    if _lib is None:
        path = _build.LIB_INSTR if _instrumented else _build.LIB
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with `python -m paper_2604_17198_amd.build` "
                "(the HIP path has no fallback)")
        L = C.CDLL(path)
        L.nacho_status_string.restype = C.c_char_p
        L.nacho_num_partitions.restype = C.c_int64
        L.nacho_num_partitions.argtypes = [C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int64, C.c_int64]
        L.nacho_workspace_bytes.argtypes = [C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int64,
                                            C.c_int64, C.POINTER(C.c_size_t)]
        L.nacho_partition.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.nacho_spmv.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64,
                                 C.c_void_p, C.c_size_t, C.c_void_p]
        L.nacho_spmv_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p]
        L.nacho_static_scratch_bytes.restype = C.c_size_t
        L.nacho_spmm.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64,
                                 C.c_int32, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
        L.nacho_spadd_k.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int64, C.c_void_p,
                                    C.c_void_p, C.c_size_t, C.c_void_p]
        L.nacho_spmul_k.argtypes = L.nacho_spadd_k.argtypes
        L.nacho_spadd_fused.argtypes = L.nacho_spadd_k.argtypes
        L.nacho_workspace_parts.argtypes = [C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int64, C.c_int64,
                                            C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p]
        L.nacho_profile_read.argtypes = [C.c_void_p, C.c_void_p, C.c_int32]
        L.nacho_validate.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.nacho_instrument.argtypes = [C.c_void_p, C.c_int64]
        L.nacho_instrument_wait.argtypes = [C.c_int64]
        L.nacho_spmv_fused.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t,
                                       C.c_void_p]
        L.nacho_partition_csr64.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int64,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.nacho_rowcost_partitions.restype = C.c_int64
        L.nacho_rowcost_partitions.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int64]
        L.nacho_partition_rowcost.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p]
        L.nacho_spmv_rowcost.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int64,
                                         C.c_void_p, C.c_size_t, C.c_void_p]
        L.nacho_probe.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_int64, C.c_void_p]
        L.nacho_distill_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int32, C.POINTER(C.c_size_t)]
        L.nacho_distill.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_float, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
        L.nacho_distill_grad.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_float, C.c_void_p,
                                         C.c_void_p, C.c_int64, C.c_void_p]
        L.nacho_route_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int32, C.POINTER(C.c_size_t)]
        L.nacho_route.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.nacho_route_grad.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_int32,
                                       C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_int64, C.c_void_p]
        L.nacho_combine.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_int64,
                                    C.c_void_p, C.c_int64, C.c_void_p]
        L.nacho_combine_grad.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_int64,
                                         C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.nacho_experts_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
        L.nacho_experts.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]
        L.nacho_experts_grad.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                         C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t,
                                         C.c_void_p]
        _libs[_instrumented] = L
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().nacho_status_string(C.c_int32(status)).decode()


def _check(status: int, where: str):
    if status != 0:
        raise NachoError(status, where)


# (A small call takes the GPU five to ten microseconds, so what Python spends per call counts: addresses and the
# stream go through ctypes as plain integers, descriptors are passed by reference, and the current stream is asked
# for without building a torch Stream object around it -- 13 us per call before, of which the stream was a third.)
def _ptr(t):
    return None if t is None else t.data_ptr()


def _public_stream():
    return torch.cuda.current_stream().cuda_stream


def _raw_stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


# (torch's raw getters are private names: without them the public calls)
_stream = _raw_stream if all(hasattr(torch._C, n) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice")) else _public_stream
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def dtype_code(dt) -> int:
    if dt is torch.float32:
        return F32
    if dt is torch.float64:
        return F64
    raise TypeError(f"unsupported value type {dt}")


# --------------------------------------------------------------------------- #
# operand descriptors (host structs holding device pointers)
# --------------------------------------------------------------------------- #
class Operand:
    """Keeps the tensors alive and exposes the C descriptor."""

    def __init__(self, levels, val=None):
        self.keep = []
        c = _Tensor()
        c.nlevels = len(levels)
        for m, l in enumerate(levels):
            c.lvl[m].extent = int(l["extent"])
            if l["kind"] == "dense":
                c.lvl[m].kind = DENSE
                c.lvl[m].pos = None
                c.lvl[m].crd = None
                c.lvl[m].count = 0
            elif l["kind"] in ("nonunique", "singleton"):
                crd = l["crd"]
                assert crd.dtype == torch.int32
                self.keep.append(crd)
                c.lvl[m].kind = NONUNIQUE if l["kind"] == "nonunique" else SINGLETON
                c.lvl[m].pos = None
                c.lvl[m].crd = crd.data_ptr() if crd.numel() else None
                c.lvl[m].count = int(crd.numel())
            else:
                pos, crd = l["pos"], l["crd"]
                assert pos.dtype == torch.int32 and crd.dtype == torch.int32
                self.keep += [pos, crd]
                c.lvl[m].kind = COMPRESSED
                c.lvl[m].pos = pos.data_ptr()
                c.lvl[m].crd = crd.data_ptr() if crd.numel() else None
                c.lvl[m].count = int(crd.numel())
        if val is not None:
            self.keep.append(val)
            c.val = val.data_ptr() if val.numel() else None
        where = self.keep[0].device
        for t in self.keep:
            if t.device != where or not t.is_contiguous():
                raise ValueError(f"an operand's arrays: contiguous ones on one device are needed (here {where})")
        self.c = c
        self.nlevels = len(levels)
        self.nnz = int(levels[-1]["crd"].numel())
        self.val = val


def vector(idx, extent, val=None):
    pos = torch.tensor([0, idx.numel()], dtype=torch.int32, device=idx.device)
    return Operand([{"kind": "compressed", "extent": extent, "pos": pos, "crd": idx}], val)


def csr(pos, crd, n_rows, n_cols, val=None):
    return Operand([{"kind": "dense", "extent": n_rows},
                    {"kind": "compressed", "extent": n_cols, "pos": pos, "crd": crd}], val)


def dcsr(pos0, crd0, pos1, crd1, n_rows, n_cols, val=None):
    return Operand([{"kind": "compressed", "extent": n_rows, "pos": pos0, "crd": crd0},
                    {"kind": "compressed", "extent": n_cols, "pos": pos1, "crd": crd1}], val)


def csf3(pos0, crd0, pos1, crd1, pos2, crd2, shape, val=None):
    """Third-order tensor, three compressed levels (nacho_partition, nacho_spadd_k)."""
    return Operand([{"kind": "compressed", "extent": shape[0], "pos": pos0, "crd": crd0},
                    {"kind": "compressed", "extent": shape[1], "pos": pos1, "crd": crd1},
                    {"kind": "compressed", "extent": shape[2], "pos": pos2, "crd": crd2}], val)


def coo(rows, cols, n_rows, n_cols, val=None):
    """Coordinate list sorted by (row, column), no pair twice."""
    return Operand([{"kind": "nonunique", "extent": n_rows, "crd": rows},
                    {"kind": "singleton", "extent": n_cols, "crd": cols}], val)


_ARRAYS = [_Tensor * n for n in range(MAX_OPERANDS + 1)]


def _pack(ops):
    """The operands' descriptors as one C array (one operand: its descriptor itself)."""
    n = len(ops)
    if n == 1:
        return C.byref(ops[0].c)
    return (_ARRAYS[n] if n <= MAX_OPERANDS else _Tensor * n)(*[o.c for o in ops])


# --------------------------------------------------------------------------- #
# entry points
# --------------------------------------------------------------------------- #
def version() -> int:
    return int(lib().nacho_version())


def num_partitions(op, ops, dtype, n_dense=0, P=0) -> int:
    arr = _pack(ops)
    return int(lib().nacho_num_partitions(op, arr, len(ops), dtype, n_dense, P))


def workspace_bytes(op, ops, dtype, n_dense=0, P=0) -> int:
    n = C.c_size_t(0)
    arr = _pack(ops)
    _check(lib().nacho_workspace_bytes(op, arr, len(ops), dtype, n_dense, P,
                                       C.byref(n)), "nacho_workspace_bytes")
    return int(n.value)


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def nacho_partition(ops, P, queries=None, cost_scale=1):
    """Boundaries 0..P.  Returns dict(coord[P+1, d], posn[P+1, k, d] int32, cost[P+1] int64)
    as device tensors."""
    k, d = len(ops), ops[0].nlevels
    dev = ops[0].keep[0].device
    coord = torch.empty((P + 1, d), dtype=torch.int32, device=dev)
    posn = torch.empty((P + 1, k, d), dtype=torch.int32, device=dev)
    cost = torch.empty(P + 1, dtype=torch.int64, device=dev)
    parts = _Parts(k, d, P, coord.data_ptr(), posn.data_ptr(), cost.data_ptr())
    arr = _pack(ops)
    if queries is not None:
        assert queries.dtype == torch.int64 and queries.numel() == P + 1
    _check(lib().nacho_partition(arr, k, cost_scale, P, _ptr(queries),
                                 C.byref(parts), None, 0, _stream()), "nacho_partition")
    return {"coord": coord, "posn": posn, "cost": cost}


def nacho_partition_csr64(pos, crd, n_rows, n_cols, P):
    """All P+1 boundaries of one CSR operand with 64-bit positions (pos: int64 device tensor).
    Returns dict(coord int32 [P+1, 2], posn int64 [P+1, 2], cost int64 [P+1]); enqueues only."""
    dev = pos.device
    assert pos.dtype == torch.int64 and (crd is None or crd.dtype == torch.int32)
    nnz = int((pos[-1] - pos[0]).item())
    coord = torch.empty((P + 1, 2), dtype=torch.int32, device=dev)
    posn = torch.empty((P + 1, 2), dtype=torch.int64, device=dev)
    cost = torch.empty(P + 1, dtype=torch.int64, device=dev)
    _check(lib().nacho_partition_csr64(_ptr(pos), _ptr(crd), n_rows, n_cols, nnz, P, _ptr(coord), _ptr(posn),
                                       _ptr(cost), _stream()), "nacho_partition_csr64")
    return {"coord": coord, "posn": posn, "cost": cost}


def workspace_parts(op, ops, dtype, ws, n_dense=0, P=0):
    """The partition table a fused call keeps in its workspace `ws` (valid after the call ran):
    dict(coord[P+1, d], posn[P+1, k, d] int32, cost[P+1] int64) as copies, plus 'P' and 'grain'."""
    parts = _Parts()
    grain = C.c_int64(0)
    arr = _pack(ops)
    _check(lib().nacho_workspace_parts(op, arr, len(ops), dtype, n_dense, P, _ptr(ws),
                                       ws.numel(), C.byref(parts), C.byref(grain), _stream()),
           "nacho_workspace_parts")
    base = ws.data_ptr()
    k, d, Pe = parts.k, parts.d, int(parts.P)

    def view(ptr, count, dt, shape):
        off = ptr - base
        nbytes = count * (8 if dt == torch.int64 else 4)
        return ws[off:off + nbytes].view(dt).reshape(shape).clone()

    return {"coord": view(parts.coord, (Pe + 1) * d, torch.int32, (Pe + 1, d)),
            "posn": view(parts.posn, (Pe + 1) * k * d, torch.int32, (Pe + 1, k, d)),
            "cost": view(parts.cost, Pe + 1, torch.int64, (Pe + 1,)), "P": Pe, "grain": int(grain.value)}


def nacho_spmv(A: Operand, x, y=None, P=0, ws=None):
    """y = A x.  A is a CSR Operand with values; x, y device tensors of A's value type."""
    dt = dtype_code(x.dtype)
    if y is None:
        y = torch.empty(A.c.lvl[0].extent, dtype=x.dtype, device=x.device)
    if ws is None:
        ws = _workspace(workspace_bytes(OP_SPMV, [A], dt, 0, P), x.device)
    arr = _pack([A])
    _check(lib().nacho_spmv(arr, _ptr(x), _ptr(y), dt, P, _ptr(ws),
                            ws.numel(), _stream()), "nacho_spmv")
    return y


def nacho_spmv_fused(A: Operand, x, y, ws=None):
    """y = A x without a partition pass: the executing wavefronts search their own boundaries."""
    dt = dtype_code(x.dtype)
    if ws is None:
        ws = _workspace(workspace_bytes(OP_SPMV, [A], dt, 0, 0), x.device)
    arr = _pack([A])
    _check(lib().nacho_spmv_fused(arr, _ptr(x), _ptr(y), dt, _ptr(ws), ws.numel(), _stream()),
           "nacho_spmv_fused")
    return y


def nacho_spmv_static(A: Operand, x, y, P=0):
    """y = A x on the library's built-in scratch memory: no workspace, nothing allocated (y is the
    caller's)."""
    arr = _pack([A])
    _check(lib().nacho_spmv_static(arr, _ptr(x), _ptr(y), dtype_code(x.dtype), P,
                                   _stream()), "nacho_spmv_static")
    return y


def static_scratch_bytes() -> int:
    return int(lib().nacho_static_scratch_bytes())


def rowcost_partitions(A: Operand, dtype, row_cost, P=0) -> int:
    arr = _pack([A])
    return int(lib().nacho_rowcost_partitions(arr, dtype, row_cost, P))


def nacho_partition_rowcost(A: Operand, P, row_cost):
    """Boundaries 0..P of one CSR operand under the row-aware cost; result as nacho_partition."""
    dev = A.keep[0].device
    coord = torch.empty((P + 1, 2), dtype=torch.int32, device=dev)
    posn = torch.empty((P + 1, 1, 2), dtype=torch.int32, device=dev)
    cost = torch.empty(P + 1, dtype=torch.int64, device=dev)
    parts = _Parts(1, 2, P, coord.data_ptr(), posn.data_ptr(), cost.data_ptr())
    arr = _pack([A])
    _check(lib().nacho_partition_rowcost(arr, row_cost, P, C.byref(parts), _stream()),
           "nacho_partition_rowcost")
    return {"coord": coord, "posn": posn, "cost": cost}


def nacho_spmv_rowcost(A: Operand, x, y, row_cost, P=0, ws=None):
    """y = A x on partitions balanced by non-zeros + row_cost per row."""
    dt = dtype_code(x.dtype)
    Pe = rowcost_partitions(A, dt, row_cost, P)
    if ws is None:
        ws = _workspace(workspace_bytes(OP_SPMV, [A], dt, 0, Pe), x.device)
    arr = _pack([A])
    _check(lib().nacho_spmv_rowcost(arr, _ptr(x), _ptr(y), dt, row_cost, P, _ptr(ws),
                                    ws.numel(), _stream()), "nacho_spmv_rowcost")
    return y


def nacho_spmm(A: Operand, B, Cout=None, P=0, ws=None):
    """C = A B with B, C dense row-major device tensors."""
    dt = dtype_code(B.dtype)
    n = int(B.shape[1])
    if Cout is None:
        Cout = torch.empty((A.c.lvl[0].extent, n), dtype=B.dtype, device=B.device)
    if ws is None:
        ws = _workspace(workspace_bytes(OP_SPMM, [A], dt, n, P), B.device)
    arr = _pack([A])
    _check(lib().nacho_spmm(arr, _ptr(B), n, int(B.stride(0)), _ptr(Cout),
                            int(Cout.stride(0)), dt, P, _ptr(ws), ws.numel(), _stream()), "nacho_spmm")
    return Cout


class SparseOut:
    """Caller-allocated result arrays of nacho_spadd_k."""

    def __init__(self, fmt, cap_rows, cap_nnz, dtype, device, n_rows=0, cap_fibres=0):
        """fmt "csf3": cap_rows is the capacity in slices, cap_fibres in fibres."""
        i32 = dict(dtype=torch.int32, device=device)
        self.fmt = fmt
        self.pos0 = torch.zeros(2, **i32) if fmt in ("dcsr", "csf3") else None
        self.crd0 = None
        if fmt in ("dcsr", "csf3"):
            self.crd0 = torch.empty(max(cap_rows, 1), **i32)
        elif fmt == "coo":
            self.crd0 = torch.empty(max(cap_nnz, 1), **i32)      # the rows of the result's entries
        n_pos1 = {"vector": 2, "coo": 2, "csr": n_rows + 1, "dcsr": cap_rows + 1, "csf3": cap_rows + 1}[fmt]
        self.pos1 = torch.zeros(n_pos1, **i32)
        self.crd1 = torch.empty(max(cap_fibres if fmt == "csf3" else cap_nnz, 1), **i32)
        self.pos2 = torch.zeros(cap_fibres + 1, **i32) if fmt == "csf3" else None
        self.crd2 = torch.empty(max(cap_nnz, 1), **i32) if fmt == "csf3" else None
        self.val = torch.empty(max(cap_nnz, 1), dtype=dtype, device=device)
        self.counts = torch.zeros(3, dtype=torch.int64, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.c = _SparseOut(_ptr(self.pos0), _ptr(self.crd0), _ptr(self.pos1), _ptr(self.crd1),
                            _ptr(self.val), cap_rows, cap_nnz, _ptr(self.counts), _ptr(self.status),
                            _ptr(self.pos2), _ptr(self.crd2), cap_fibres)


def nacho_spadd_k(ops, out: SparseOut, P=0, ws=None):
    """Z = sum of the operands (union add).  Enqueues only; read out.counts / out.status after
    synchronising."""
    dt = dtype_code(ops[0].val.dtype)
    dev = ops[0].val.device
    if ws is None:
        ws = _workspace(workspace_bytes(OP_SPADD, ops, dt, 0, P), dev)
    arr = _pack(ops)
    _check(lib().nacho_spadd_k(arr, len(ops), dt, P, C.byref(out.c), _ptr(ws),
                               ws.numel(), _stream()), "nacho_spadd_k")
    return out


def nacho_spadd_fused(ops, out: SparseOut, P=0, ws=None):
    """nacho_spadd_k on sparse vectors without a partition pass: the workgroups of the merge kernel search
    their own boundaries.  Enqueues only."""
    dt = dtype_code(ops[0].val.dtype)
    dev = ops[0].val.device
    if ws is None:
        ws = _workspace(workspace_bytes(OP_SPADD, ops, dt, 0, P), dev)
    arr = _pack(ops)
    _check(lib().nacho_spadd_fused(arr, len(ops), dt, P, C.byref(out.c), _ptr(ws),
                                   ws.numel(), _stream()), "nacho_spadd_fused")
    return out


def nacho_spmul_k(ops, out: SparseOut, P=0, ws=None):
    """Z = product of the operands over the intersection of their coordinates (vectors, CSR, DCSR, COO).
    Enqueues only."""
    dt = dtype_code(ops[0].val.dtype)
    dev = ops[0].val.device
    if ws is None:
        ws = _workspace(workspace_bytes(OP_SPMUL, ops, dt, 0, P), dev)
    arr = _pack(ops)
    _check(lib().nacho_spmul_k(arr, len(ops), dt, P, C.byref(out.c), _ptr(ws),
                               ws.numel(), _stream()), "nacho_spmul_k")
    return out


# --------------------------------------------------------------------------- #
# operators that train models
# --------------------------------------------------------------------------- #
_MODEL_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def model_dtype_code(dt) -> int:
    code = _MODEL_TYPES.get(dt)
    if code is None:
        raise TypeError(f"unsupported value type {dt}")
    return code


# (What Python spends on a small call is most of its time: messages are put together only where something is wrong.)
def _need(ok, what):
    if not ok:
        raise ValueError(what)


_HOST = -1                                                   # the number of the device of tensors that are on no GPU


def _matrix(t, what, rows=None, cols=None, dtype=None, device=None):
    """A matrix whose rows are contiguous, of the given sizes where they are given; returns its leading dimension.  Without a
    device to be on it has to be on the current GPU."""
    if t.dim() != 2:
        raise ValueError(f"{what}: a matrix is needed, got {t.dim()} dimensions")
    r, c = t.shape
    ld, step = t.stride()
    if step != 1 and c > 1:
        raise ValueError(f"{what}: contiguous rows are needed")
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise ValueError(f"{what}: {r} x {c}, expected {rows} x {cols}")
    if device is None:
        number = t.get_device()
        if number == _HOST or number != _current_device():
            raise ValueError(f"{what}: on {t.device}, and not on the current GPU")
    elif t.dtype is not dtype or t.device != device:
        raise ValueError(f"{what}: {t.dtype} on {t.device}, expected {dtype} on {device}")
    return ld if r > 1 else (ld if ld > c else c)


def _vector_of(t, what, n, dtype, device):
    """A contiguous array of n elements, or None."""
    if t is not None and (t.numel() != n or t.dtype is not dtype or not t.is_contiguous() or t.device != device):
        raise ValueError(f"{what}: {n} contiguous elements of {dtype} on {device} are needed")
    return t


def _room(ws, device):
    """The bytes of a workspace that the caller brings."""
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"ws: contiguous memory on {device} is needed")
    return ws.numel()


def _floats(n, device):
    """A new array of n results (whatever the program's default type is)."""
    return torch.empty(n, dtype=torch.float32, device=device)


def _check_teacher(teacher, logits, weight):
    if teacher.nlevels != 2 or teacher.c.lvl[0].kind != DENSE or teacher.c.lvl[1].kind != COMPRESSED:
        raise NachoError(-2, "teacher: a CSR operand is needed")
    val = teacher.val                                        # (an operand's arrays are contiguous and on one device)
    if val is None or val.numel() != teacher.nnz or val.dtype is not torch.float32 or val.device != logits.device:
        raise ValueError(f"teacher: {teacher.nnz} values of torch.float32 on {logits.device} are needed")
    rows, cols = teacher.c.lvl[0].extent, teacher.c.lvl[1].extent
    _need(teacher.keep[0].numel() == rows + 1, "teacher: rows + 1 positions are needed")
    ld = _matrix(logits, "logits", rows, cols)
    _vector_of(weight, "weight", rows, torch.float32, logits.device)
    return rows, cols, ld


def nacho_distill(teacher: Operand, logits, temperature=1.0, weight=None, grad=None, loss=None, lse=None, ws=None):
    """Distillation loss of every row of `logits` against the teacher's stored logits (a CSR operand of
    float32 values).  Returns (loss[rows], lse[rows]); `grad`, when given, receives the logits' gradient."""
    dt = model_dtype_code(logits.dtype)
    rows, cols, ld = _check_teacher(teacher, logits, weight)
    dev = logits.device
    ldg = _matrix(grad, "grad", rows, cols, logits.dtype, dev) if grad is not None else 0
    loss = _vector_of(loss, "loss", rows, torch.float32, dev) if loss is not None else _floats(rows, dev)
    lse = _vector_of(lse, "lse", rows, torch.float32, dev) if lse is not None else _floats(rows, dev)
    if ws is None:
        n = C.c_size_t(0)
        _check(lib().nacho_distill_workspace_bytes(rows, cols, dt, C.byref(n)), "nacho_distill_workspace_bytes")
        room = n.value
        ws = _workspace(room, dev) if room else None
    else:
        room = _room(ws, dev)
    _check(lib().nacho_distill(_pack([teacher]), _ptr(logits), ld, dt, _ptr(weight), temperature, _ptr(loss), _ptr(lse),
                               _ptr(grad), ldg, _ptr(ws), room, _stream()), "nacho_distill")
    return loss, lse


def nacho_distill_grad(teacher: Operand, logits, lse, temperature=1.0, weight=None, grad=None):
    """Gradient of the logits from the lse of an earlier nacho_distill; `weight` is the factor of each row's loss times
    the gradient that arrives at it."""
    dt = model_dtype_code(logits.dtype)
    rows, cols, ld = _check_teacher(teacher, logits, weight)
    _vector_of(lse, "lse", rows, torch.float32, logits.device)
    if grad is None:
        grad = torch.empty((rows, cols), dtype=logits.dtype, device=logits.device)
    ldg = _matrix(grad, "grad", rows, cols, logits.dtype, logits.device)
    _check(lib().nacho_distill_grad(_pack([teacher]), _ptr(logits), ld, dt, _ptr(weight), temperature, _ptr(lse), _ptr(grad),
                                    ldg, _stream()), "nacho_distill_grad")
    return grad


class Routing:
    """The arrays nacho_route fills: the routing matrix by tokens (pos, expert, gate), by experts (expert_pos, token; slot:
    the place there of every entry), counts, lse, the balance loss and the number of tokens that store an entry."""

    def __init__(self, n_tokens, n_experts, top_k, device, normalise=False):
        self.n_tokens, self.n_experts, self.top_k, self.normalise = n_tokens, n_experts, top_k, normalise
        # one allocation for the whole numbers and one for the rest; the matrix's coordinates and values come first, where
        # they start at a multiple of 16 bytes
        room = n_tokens * top_k
        (self.expert, self.slot, self.token, self.pos, self.expert_pos, self.counts, self.routed), i = self._arrays(
            (room, room, room, n_tokens + 1, n_experts + 1, n_experts, 1), torch.int32, device)
        (self.gate, self.lse, self.balance), f = self._arrays((room, n_tokens, 1), torch.float32, device)
        self.c = _Routing(i[3], i[0], f[0], i[1], i[4], i[2], i[5], f[1], f[2], i[6])

    @staticmethod
    def _arrays(sizes, dtype, device):
        """Arrays of these numbers of 4-byte elements, and their addresses (one without an element has one too)."""
        whole = torch.empty(sum(sizes), dtype=dtype, device=device)
        at, starts = whole.data_ptr(), []
        for n in sizes:
            starts.append(at)
            at += 4 * n
        return torch.unsafe_split_with_sizes(whole, sizes), starts

    def matrix(self):
        """The gates as a CSR operand [tokens x experts] (of full rows: every place holds an entry)."""
        return csr(self.pos, self.expert, self.n_tokens, self.n_experts, self.gate)


def nacho_route(logits, top_k, normalise=False, keep=None, out=None, ws=None):
    """Routes every token to its top_k experts; `keep` (bool or uint8 [tokens]): tokens that take part.  Enqueues only."""
    dt, dev = model_dtype_code(logits.dtype), logits.device
    ld = _matrix(logits, "logits")
    tokens, experts = logits.shape
    if out is None:
        out = Routing(tokens, experts, top_k, dev)
    _need((out.n_tokens, out.n_experts, out.top_k) == (tokens, experts, top_k) and out.pos.device == dev,
          "out: made for other sizes or another device")
    out.normalise = bool(normalise)
    if keep is not None:
        _vector_of(keep, "keep", tokens, torch.bool if keep.dtype is torch.bool else torch.uint8, dev)
    if ws is None:
        n = C.c_size_t(0)
        _check(lib().nacho_route_workspace_bytes(tokens, experts, top_k, C.byref(n)), "nacho_route_workspace_bytes")
        room = n.value
        ws = _workspace(room, dev)
    else:
        room = _room(ws, dev)
    _check(lib().nacho_route(_ptr(logits), ld, tokens, experts, dt, top_k, out.normalise, _ptr(keep), C.byref(out.c),
                             _ptr(ws), room, _stream()), "nacho_route")
    return out


def nacho_route_grad(logits, routing: Routing, grad_gate=None, balance=0.0, keep=None, grad=None):
    """Gradient of the logits from that of the gates (by entry) and `balance` times that of the balance loss.  `keep` may
    be given as to nacho_route; tokens that it leaves out store nothing, which is how they are known."""
    dt, dev = model_dtype_code(logits.dtype), logits.device
    r = routing
    ld = _matrix(logits, "logits", r.n_tokens, r.n_experts)
    _need(r.pos.device == dev, "routing: on another device than the logits")
    _vector_of(grad_gate, "grad_gate", r.n_tokens * r.top_k, torch.float32, dev)
    if grad is None:
        grad = torch.empty((r.n_tokens, r.n_experts), dtype=logits.dtype, device=dev)
    ldg = _matrix(grad, "grad", r.n_tokens, r.n_experts, logits.dtype, dev)
    _check(lib().nacho_route_grad(_ptr(logits), ld, r.n_tokens, r.n_experts, dt, r.top_k, r.normalise, C.byref(r.c),
                                  _ptr(grad_gate), balance, _ptr(grad), ldg, _stream()), "nacho_route_grad")
    return grad


_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


def _stack(t, what, shape, dtype, device):
    """Matrices (or rows) of one size, each with contiguous rows: leading dimension and distance."""
    if tuple(t.shape) != shape or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{what}: {tuple(t.shape)} of {t.dtype} on {t.device}, expected {shape} of {dtype} on {device}")
    stride, cols = t.stride(), shape[-1]
    if stride[-1] != 1 and cols > 1:
        raise ValueError(f"{what}: contiguous rows are needed")
    if len(shape) == 2:
        return cols, stride[0] if shape[0] > 1 else max(cols, stride[0])
    ld = stride[1] if shape[1] > 1 else cols
    if ld < cols:
        raise ValueError(f"{what}: rows that do not overlap are needed")
    return ld, stride[0] if shape[0] > 1 else max(shape[1] * ld, stride[0])


def _layer(x, weight, expert_pos, token, bias, act):
    """The descriptor of a layer of experts, and its number of slots."""
    dtype, dev = x.dtype, x.device
    dt = model_dtype_code(dtype)
    if weight.dim() != 3:
        raise ValueError("weight: [experts, outer, inner] is needed")
    shape = tuple(weight.shape)
    experts, outer, inner = shape
    ldx = _matrix(x, "x", None, inner)
    ldw, stride = _stack(weight, "weight", shape, dtype, dev)
    _vector_of(expert_pos, "expert_pos", experts + 1, torch.int32, dev)
    bounds, tokens = expert_pos.data_ptr(), x.shape[0]
    if token is None:
        slots, where = tokens, None
    else:
        slots = token.numel()
        _vector_of(token, "token", slots, torch.int32, dev)
        where = token.data_ptr() or bounds                   # (an array without an element has no address)
    if act not in _ACTS:
        raise ValueError(f"act: one of {', '.join(_ACTS)}")
    gap = _stack(bias, "bias", (experts, outer), dtype, dev)[1] if bias is not None else 0
    return _ExpertsLayer(bounds, where, experts, slots, tokens, inner, outer, x.data_ptr(), ldx, weight.data_ptr(), ldw, stride,
                         _ptr(bias), gap, _ACTS[act], dt), slots


def nacho_experts(x, weight, expert_pos, token=None, bias=None, act="none", y=None, pre=None):
    """y[s] = act(x[token[s]] weight[e]^T + bias[e]) for the slots s = expert_pos[e] .. expert_pos[e+1] of every expert e
    (expert_pos, token: a Routing's).  `pre`, when given, receives the rows before the activation."""
    c, slots = _layer(x, weight, expert_pos, token, bias, act)
    outer = c.outer
    if y is None:
        y = torch.empty((slots, outer), dtype=x.dtype, device=x.device)
        ldy = outer
    else:
        ldy = _matrix(y, "y", slots, outer, x.dtype, x.device)
    ldpre = _matrix(pre, "pre", slots, outer, x.dtype, x.device) if pre is not None else 0
    _check(lib().nacho_experts(C.byref(c), _ptr(y), ldy, _ptr(pre), ldpre, _stream()), "nacho_experts")
    return y


def nacho_experts_grad(grad_y, x, weight, expert_pos, token=None, act="none", pre=None, grad_x=None, grad_weight=None,
                       grad_bias=None, ws=None):
    """(gradient of every slot's row of x, gradient of the weights); `grad_bias`, when given, receives the biases'.  A
    `grad_x` or `grad_weight` that is False is not wanted: it is not computed, and None is returned."""
    c, slots = _layer(x, weight, expert_pos, token, None, act)
    experts, outer, inner = weight.shape
    dev = x.device
    ldgy = _matrix(grad_y, "grad_y", slots, outer, x.dtype, dev)
    ldpre = _matrix(pre, "pre", slots, outer, x.dtype, dev) if pre is not None else 0
    if grad_x is False:
        grad_x = None
    elif grad_x is None:
        grad_x = torch.empty((slots, inner), dtype=x.dtype, device=dev)
    if grad_weight is False:
        grad_weight = None
    elif grad_weight is None:
        grad_weight = torch.empty((experts, outer, inner), dtype=x.dtype, device=dev)
    ldgx = _matrix(grad_x, "grad_x", slots, inner, x.dtype, dev) if grad_x is not None else 0
    ldgw, gap = _stack(grad_weight, "grad_weight", (experts, outer, inner), x.dtype, dev) if grad_weight is not None else (0, 0)
    gb = _stack(grad_bias, "grad_bias", (experts, outer), x.dtype, dev)[1] if grad_bias is not None else 0
    if ws is None:
        n = C.c_size_t(0)
        _check(lib().nacho_experts_workspace_bytes(C.byref(c), C.byref(n)), "nacho_experts_workspace_bytes")
        room = n.value
        ws = _workspace(room, dev) if room else None
    else:
        room = _room(ws, dev)
    _check(lib().nacho_experts_grad(C.byref(c), _ptr(grad_y), ldgy, _ptr(pre), ldpre, _ptr(grad_x), ldgx, _ptr(grad_weight),
                                    ldgw, gap, _ptr(grad_bias), gb, _ptr(ws), room, _stream()),
           "nacho_experts_grad")
    return grad_x, grad_weight


def _slots_of(pos, slot, gate, n_slots, device):
    """The routing matrix tokens x slots as a descriptor."""
    _need(pos.dtype is torch.int32 and pos.is_contiguous() and pos.numel() > 0 and pos.device == device,
          "pos: tokens + 1 contiguous int32 positions are needed on the rows' device")
    _vector_of(slot, "slot", slot.numel(), torch.int32, device)
    _vector_of(gate, "gate", slot.numel(), torch.float32, device)
    c = _Tensor()
    c.nlevels = 2
    c.lvl[0].kind, c.lvl[0].extent = DENSE, pos.numel() - 1
    low = c.lvl[1]
    low.kind, low.extent, low.pos, low.crd, low.count = COMPRESSED, n_slots, pos.data_ptr(), slot.data_ptr() or None, slot.numel()
    c.val = None if gate is None else gate.data_ptr() or None
    return c


def nacho_combine(pos, slot, y, gate=None, residual=None, out=None):
    """out[t] = residual[t] + sum over the entries of token t of gate * y[slot] (pos, slot, gate: a Routing's).  `out` may
    be `residual` itself."""
    dt, dev = model_dtype_code(y.dtype), y.device
    ldy = _matrix(y, "y")
    tokens, n = pos.numel() - 1, y.shape[1]
    ldr = _matrix(residual, "residual", tokens, n, y.dtype, dev) if residual is not None else 0
    if out is None:
        out = torch.empty((tokens, n), dtype=y.dtype, device=dev)
        ldo = n
    else:
        ldo = _matrix(out, "out", tokens, n, y.dtype, dev)
    c = _slots_of(pos, slot, gate, y.shape[0], dev)
    _check(lib().nacho_combine(C.byref(c), _ptr(y), ldy, n, dt, _ptr(residual), ldr, _ptr(out), ldo, _stream()),
           "nacho_combine")
    return out


def nacho_combine_grad(pos, slot, y, grad_out, gate=None, grad_y=None, grad_gate=None):
    """Gradients of y's rows and of the gates; rows of y that no entry names, and places of gates behind the last entry, are
    left as they are.  One that is False is not wanted: it is not computed, and None is returned."""
    dt, dev = model_dtype_code(y.dtype), y.device
    ldy = _matrix(y, "y")
    tokens, n = pos.numel() - 1, y.shape[1]
    ldg = _matrix(grad_out, "grad_out", tokens, n, y.dtype, dev)
    if grad_y is False:
        grad_y = None
    elif grad_y is None:
        grad_y = torch.empty((y.shape[0], n), dtype=y.dtype, device=dev)
    ldgy = _matrix(grad_y, "grad_y", y.shape[0], n, y.dtype, dev) if grad_y is not None else 0
    if grad_gate is False:
        grad_gate = None
    elif grad_gate is None:
        grad_gate = _floats(slot.numel(), dev)
    _vector_of(grad_gate, "grad_gate", slot.numel(), torch.float32, dev)
    c = _slots_of(pos, slot, gate, y.shape[0], dev)
    _check(lib().nacho_combine_grad(C.byref(c), _ptr(y), ldy, n, dt, _ptr(grad_out), ldg, _ptr(grad_y), ldgy,
                                    _ptr(grad_gate), _stream()), "nacho_combine_grad")
    return grad_y, grad_gate


def nacho_validate(ops):
    """Checks the operands' preconditions on the device.  Returns (status, (operand, level, position))
    after synchronising: status 0, or -1 with the place of one violation."""
    dev = ops[0].keep[0].device
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    info = torch.zeros(3, dtype=torch.int64, device=dev)
    arr = _pack(ops)
    _check(lib().nacho_validate(arr, len(ops), _ptr(status), _ptr(info), _stream()),
           "nacho_validate")
    torch.cuda.synchronize()
    return int(status.cpu()[0]), tuple(int(v) for v in info.cpu())


WAVE_RECORD = [("t_begin", "<u8"), ("t_end", "<u8"), ("cycles", "<u8"), ("items", "<u4"), ("rows", "<u4"),
               ("hw_id", "<u4"), ("xcc_id", "<u4")]


def instrument(records, capacity=None):
    """Instrumented library only: executing kernels log one WAVE_RECORD per wavefront into the
    device uint8 tensor `records` (None: stop logging)."""
    rb = int(lib().nacho_instrument_record_bytes())
    if records is None:
        _check(lib().nacho_instrument(None, 0), "nacho_instrument")
        return
    cap = records.numel() // rb if capacity is None else capacity
    _check(lib().nacho_instrument(_ptr(records), cap), "nacho_instrument")


def instrument_wait(workgroup):
    """Instrumented library only: the wait of this workgroup of the row loop of a DCSR product counts as run out (-1: none)."""
    _check(lib().nacho_instrument_wait(workgroup), "nacho_instrument_wait")


def merge_wavefronts() -> int:
    return int(lib().nacho_merge_wavefronts())


PROBE_READ, PROBE_COPY, PROBE_GATHER = 0, 1, 2


def probe(kind, dst, src, nbytes, gathers=0):
    """Enqueue one of the library's kernels of known traffic (see nacho_probe)."""
    _check(lib().nacho_probe(kind, _ptr(dst), _ptr(src), nbytes, gathers, _stream()), "nacho_probe")


def profile_enable(on: bool):
    lib().nacho_profile_enable(1 if on else 0)


def profile_read():
    """[(kernel name, ms)] of the last fused call (synchronises)."""
    ms = (C.c_float * 16)()
    names = (C.c_char_p * 16)()
    n = lib().nacho_profile_read(C.cast(ms, C.c_void_p), C.cast(names, C.c_void_p), 16)
    if n < 0:
        raise NachoError(n, "nacho_profile_read")
    return [(names[i].decode(), float(ms[i])) for i in range(min(n, 16))]
