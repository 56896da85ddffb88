"""ctypes binding of libgnnpre.so: one Python function per C entry point, same names.

Only argument marshalling happens here.  Tensors are torch tensors used as plain device (or
host) memory; every step of the computation runs inside the library's CUDA kernels.  If the
library has not been built, importing this module raises: there is no fallback.

`stream` (default: the current one) is where a call's kernels run.  What the caller brings is ordered with it by the caller; a call that
makes its result itself, checks its waits or converts indices has it wait for the current stream first.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Sequence

import torch

from . import build as _build

GNNPRE_OP_GCN_SYM, GNNPRE_OP_SAGE_MEAN, GNNPRE_OP_GIN_SUM = 0, 1, 2
GNNPRE_MEM_DEVICE, GNNPRE_MEM_HOST = 0, 1
GNNPRE_FLAG_LAUNCH_PER_BLOCK, GNNPRE_FLAG_SKIP_VALIDATION, GNNPRE_FLAG_NO_BULK_COPY = 1, 2, 4
GNNPRE_FLAG_BULK_COPY = 8
GNNPRE_MAX_HOPS = 64
GNNPRE_SCHEDULE_RESIDENT, GNNPRE_SCHEDULE_SLABS, GNNPRE_SCHEDULE_PANELS = 0, 1, 2


class gnnpre_csr_t(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("nnz", ctypes.c_int64), ("rowptr", ctypes.c_void_p),
                ("colidx", ctypes.c_void_p), ("mem", ctypes.c_int32)]


class gnnpre_plan_opts_t(ctypes.Structure):
    _fields_ = [("op", ctypes.c_int32), ("gin_eps", ctypes.c_float), ("feat_dim", ctypes.c_int64),
                ("budget_bytes", ctypes.c_int64), ("force_blocks", ctypes.c_int32),
                ("force_col_slabs", ctypes.c_int32), ("segment_edges", ctypes.c_int32),
                ("operands_mem", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("teleport_alpha", ctypes.c_float)]


class gnnpre_plan_info_t(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("nnz", ctypes.c_int64), ("nnz_tilde", ctypes.c_int64),
                ("feat_dim", ctypes.c_int64), ("op", ctypes.c_int32), ("b", ctypes.c_int32), ("c", ctypes.c_int32),
                ("slab_width", ctypes.c_int64), ("B_S", ctypes.c_int64), ("B_X", ctypes.c_int64),
                ("B_fixed", ctypes.c_int64), ("beta_S", ctypes.c_int64), ("beta_X", ctypes.c_int64),
                ("budget_bytes", ctypes.c_int64), ("device_bytes", ctypes.c_int64), ("host_bytes", ctypes.c_int64),
                ("num_segments", ctypes.c_int64), ("num_row_fixups", ctypes.c_int64),
                ("num_scratch_rows", ctypes.c_int64), ("segment_edges", ctypes.c_int32),
                ("structure_mem", ctypes.c_int32)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class gnnpre_block_info_t(ctypes.Structure):
    _fields_ = [("e_lo", ctypes.c_int64), ("e_hi", ctypes.c_int64), ("row_lo", ctypes.c_int32),
                ("row_hi", ctypes.c_int32), ("first_row_partial", ctypes.c_int32),
                ("last_row_partial", ctypes.c_int32)]


class gnnpre_stats_t(ctypes.Structure):
    _fields_ = [("hop_ms", ctypes.c_float * GNNPRE_MAX_HOPS), ("total_ms", ctypes.c_float),
                ("segments_ms", ctypes.c_float), ("h2d_bytes", ctypes.c_int64), ("d2h_bytes", ctypes.c_int64),
                ("kernel_launches", ctypes.c_int64), ("segments_launches", ctypes.c_int64),
                ("startup_ms", ctypes.c_float), ("drain_ms", ctypes.c_float), ("schedule", ctypes.c_int32),
                ("upload_slabs", ctypes.c_int32)]


class GnnpreError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        text = _lib.gnnpre_status_string(status).decode()
        detail = _lib.gnnpre_last_cuda_error().decode()
        super().__init__(f"{where}: {text} ({status})" + (f" [{detail}]" if detail and status == -7 else ""))


def _load() -> ctypes.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: run paper_2207_12000_b200.build.build() (needs nvcc); "
                          "there is no fallback implementation")
    lib = ctypes.CDLL(path)
    p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.gnnpre_degrees.argtypes = [ctypes.POINTER(gnnpre_csr_t), p, p]
    lib.gnnpre_build_plan.argtypes = [ctypes.POINTER(gnnpre_csr_t), p, ctypes.POINTER(gnnpre_plan_opts_t),
                                      ctypes.POINTER(p)]
    lib.gnnpre_plan_info.argtypes = [p, ctypes.POINTER(gnnpre_plan_info_t)]
    lib.gnnpre_plan_block.argtypes = [p, i32, ctypes.POINTER(gnnpre_block_info_t)]
    lib.gnnpre_plan_scales.argtypes = [p, p, p, p]
    lib.gnnpre_plan_support.argtypes = [p, p, p]
    lib.gnnpre_plan_hop_order.argtypes = [p, p]
    lib.gnnpre_propagate.argtypes = [p, p, i64, i32, i32, ctypes.POINTER(p), i64, i32, p,
                                     ctypes.POINTER(gnnpre_stats_t)]
    lib.gnnpre_hop_static.argtypes = [ctypes.POINTER(gnnpre_csr_t), i32, ctypes.c_float, i64, p, i64, p, i64, p]
    lib.gnnpre_lc_selftest_wait_timeout.argtypes = [p, i64, i64, i64, p, i64, i64, p, i64, p, ctypes.c_uint32, p]
    lib.gnnpre_propagate_weighted.argtypes = [p, p, i64, i32, ctypes.POINTER(ctypes.c_void_p), i64,
                                              ctypes.POINTER(ctypes.c_float), p, i64, p]
    lib.gnnpre_lc_first_layer.argtypes = [ctypes.POINTER(ctypes.c_void_p), i32, i64, i64, i64, p, i64, p, i64, i64,
                                          ctypes.c_uint64, i32, p, i64, i64, p, p]
    lib.gnnpre_embedding_lookup.argtypes = [p, i64, i64, i64, i32, p, i32, i64, ctypes.c_float, p, i64, p]
    lib.gnnpre_embedding_grad_workspace.argtypes = [i64, i64, i64]
    lib.gnnpre_embedding_grad_workspace.restype = i64
    lib.gnnpre_embedding_grad.argtypes = [p, i64, i32, p, i32, i64, i64, i64, ctypes.c_float, i32, p, i64, i32, p, i64, p]
    lib.gnnpre_orthogonalize_workspace.argtypes = [i64, i64, i64, i32]
    lib.gnnpre_orthogonalize_workspace.restype = i64
    lib.gnnpre_orthogonalize.argtypes = [p, i64, i64, i64, i64, i64, i32, i32, ctypes.POINTER(ctypes.c_float), ctypes.c_float,
                                         ctypes.c_float, p, i64, i64, p, i64, p, p]
    lib.gnnpre_orthogonalize_selftest_wait_timeout.argtypes = [p, i64, i64, p, p, i64, p, ctypes.c_uint32, p]
    lib.gnnpre_lc_first_layer_grad_workspace.argtypes = [i32, i64, i64, i64]
    lib.gnnpre_lc_first_layer_grad_workspace.restype = i64
    lib.gnnpre_lc_first_layer_grad.argtypes = [ctypes.POINTER(ctypes.c_void_p), i32, i64, i64, i64, p, i64, p, i64, i64, p, i64, i64,
                                               ctypes.c_uint64, i64, i32, p, i64, p, i64, p, p]
    lib.gnnpre_lc_grad_selftest_wait_timeout.argtypes = [p, i64, i64, i64, p, i64, i64, p, i64, p, i64, p, ctypes.c_uint32, p]
    lib.gnnpre_normalize.argtypes = [p, p, i32, p]
    lib.gnnpre_solve_normalisation_blocks.argtypes = [i64] * 8 + [ctypes.POINTER(i64)]
    lib.gnnpre_selftest_wait_timeout.argtypes = [p, ctypes.c_uint32, p]
    lib.gnnpre_selftest_wait_timeout_async.argtypes = [p, ctypes.c_uint32, p]
    lib.gnnpre_plan_status.argtypes = [p, p]
    lib.gnnpre_gather_ceiling.argtypes = [p, p, i64, p, p]
    lib.gnnpre_describe_panels.argtypes = [i64, i64, i32, p, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.gnnpre_inject_alloc_failure.argtypes = [i64, i64]
    lib.gnnpre_plan_destroy.argtypes = [p]
    lib.gnnpre_plan_destroy.restype = None
    lib.gnnpre_solve_budget.argtypes = [i64] * 8 + [ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.gnnpre_status_string.argtypes = [ctypes.c_int]
    lib.gnnpre_status_string.restype = ctypes.c_char_p
    lib.gnnpre_last_cuda_error.restype = ctypes.c_char_p
    return lib


_lib = _load()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise GnnpreError(status, where)


def _mem_of(t: torch.Tensor) -> int:
    return GNNPRE_MEM_DEVICE if t.is_cuda else GNNPRE_MEM_HOST


def _csr(rowptr: torch.Tensor, colidx: torch.Tensor) -> gnnpre_csr_t:
    assert rowptr.dtype == torch.int64 and colidx.dtype == torch.int32
    assert rowptr.is_contiguous() and colidx.is_contiguous() and rowptr.device == colidx.device
    return gnnpre_csr_t(rowptr.numel() - 1, colidx.numel(), rowptr.data_ptr(), colidx.data_ptr(), _mem_of(rowptr))


# The current stream's handle without building a torch.cuda.Stream around it (3.2 us a call).
_raw_stream = torch._C._cuda_getCurrentRawStream


def _stream_ptr(stream) -> int:
    if stream is None:
        return _raw_stream(torch.cuda.current_device())
    return stream.cuda_stream


def _torch_stream(stream):
    """`stream` as torch's own, also where it is another library's object that has a handle only."""
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)


def _on(stream):
    """Where a call takes and fills what it makes for itself (workspace, converted indices, error word): on the stream that its kernels
    run on, whose order then covers a block from its last use to its next."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(_torch_stream(stream))


def _wait_for_current(stream) -> None:
    if stream is not None:
        _torch_stream(stream).wait_stream(torch.cuda.current_stream())


def _results(count: int, shape, dtype, device, stream) -> list[torch.Tensor]:
    """Results that the caller did not bring, from the current stream's memory.  If the kernels run on another stream, that one waits for
    the current one, whose work may still use the blocks, and the allocator is told of their use there."""
    made = [torch.empty(shape, dtype=dtype, device=device) for _ in range(count)]
    if stream is not None and made and made[0].is_cuda:
        _wait_for_current(stream)
        for out in made:
            out.record_stream(_torch_stream(stream))
    return made


def _result(shape, dtype, device, stream) -> torch.Tensor:
    return _results(1, shape, dtype, device, stream)[0]


def _error_word(device, stream) -> torch.Tensor:
    """Of a checked call, which runs after what the current stream has been given."""
    _wait_for_current(stream)
    with _on(stream):
        return torch.zeros(1, dtype=torch.int32, device=device)


def _check_waits(flag: torch.Tensor, stream, where: str) -> None:
    """Synchronises with the call that was given `flag` and raises if a wait of it ran out."""
    with _on(stream):
        ran_out = int(flag.item()) != 0
    if ran_out:
        raise GnnpreError(-8, where)


def _pointers(tensors):
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def gnnpre_degrees(rowptr: torch.Tensor, colidx: torch.Tensor, stream=None) -> torch.Tensor:
    csr = _csr(rowptr, colidx)
    deg = _result((csr.n,), torch.int32, rowptr.device, stream)
    _check(_lib.gnnpre_degrees(ctypes.byref(csr), deg.data_ptr(), _stream_ptr(stream)), "gnnpre_degrees")
    return deg


class Plan:
    """Owns a gnnpre_plan_t*; destroyed with the object."""

    def __init__(self, handle: int, keepalive=None, nnz_tilde: int | None = None):
        self._h = ctypes.c_void_p(handle)
        self._keepalive = keepalive
        self._nnz_tilde = nnz_tilde

    @property
    def nnz_tilde(self) -> int:
        """Edges of the operator's support."""
        if self._nnz_tilde is None:
            self._nnz_tilde = gnnpre_plan_info(self)["nnz_tilde"]
        return self._nnz_tilde

    @property
    def handle(self):
        return self._h

    def info(self) -> dict:
        return gnnpre_plan_info(self)

    def close(self):
        if self._h:
            _lib.gnnpre_plan_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def gnnpre_build_plan(rowptr: torch.Tensor, colidx: torch.Tensor, op: int, feat_dim: int, *, degrees=None,
                      gin_eps: float = 0.0, budget_bytes: int = 0, force_blocks: int = 0, force_col_slabs: int = 0,
                      segment_edges: int = 0, operands_mem: int = GNNPRE_MEM_DEVICE, flags: int = 0,
                      teleport_alpha: float = 0.0) -> Plan:
    csr = _csr(rowptr, colidx)
    opts = gnnpre_plan_opts_t(op, gin_eps, feat_dim, budget_bytes, force_blocks, force_col_slabs, segment_edges,
                              operands_mem, flags, teleport_alpha)
    if degrees is not None:
        assert degrees.dtype == torch.int32 and degrees.device == rowptr.device and degrees.is_contiguous()
    out = ctypes.c_void_p()
    _check(_lib.gnnpre_build_plan(ctypes.byref(csr), degrees.data_ptr() if degrees is not None else None,
                                  ctypes.byref(opts), ctypes.byref(out)), "gnnpre_build_plan")
    return Plan(out.value, nnz_tilde=csr.nnz + (0 if op == GNNPRE_OP_SAGE_MEAN else csr.n))


def gnnpre_plan_info(plan: Plan) -> dict:
    info = gnnpre_plan_info_t()
    _check(_lib.gnnpre_plan_info(plan.handle, ctypes.byref(info)), "gnnpre_plan_info")
    return info.as_dict()


def gnnpre_plan_block(plan: Plan, l: int) -> dict:
    blk = gnnpre_block_info_t()
    _check(_lib.gnnpre_plan_block(plan.handle, l, ctypes.byref(blk)), "gnnpre_plan_block")
    return {k: getattr(blk, k) for k, _ in blk._fields_}


def gnnpre_plan_scales(plan: Plan):
    """(degrees int32, rscale fp32, cscale fp32) as host tensors."""
    n = gnnpre_plan_info(plan)["n"]
    deg = torch.empty(n, dtype=torch.int32)
    r = torch.empty(n, dtype=torch.float32)
    c = torch.empty(n, dtype=torch.float32)
    _check(_lib.gnnpre_plan_scales(plan.handle, deg.data_ptr(), r.data_ptr(), c.data_ptr()), "gnnpre_plan_scales")
    return deg, r, c


def gnnpre_plan_support(plan: Plan):
    """(rowptr int64 [n+1], colidx int32 [nnz_tilde]) of the operator's support, as host tensors."""
    info = gnnpre_plan_info(plan)
    rp = torch.empty(info["n"] + 1, dtype=torch.int64)
    ci = torch.empty(info["nnz_tilde"], dtype=torch.int32)
    _check(_lib.gnnpre_plan_support(plan.handle, rp.data_ptr(), ci.data_ptr()), "gnnpre_plan_support")
    return rp, ci


def gnnpre_plan_hop_order(plan: Plan):
    """int64 [num_segments] on the host: the first edge of each segment, in the order a whole hop takes them."""
    first = torch.empty(gnnpre_plan_info(plan)["num_segments"], dtype=torch.int64)
    _check(_lib.gnnpre_plan_hop_order(plan.handle, first.data_ptr()), "gnnpre_plan_hop_order")
    return first


def gnnpre_propagate(plan: Plan, X: torch.Tensor, K: int, out: Sequence[torch.Tensor] | None = None, *,
                     stream=None, want_stats: bool = False):
    """out[k-1] = A^ applied k times to X.  X and out are fp32 row-major views (stride(1) == 1) on the
    device, or host tensors (preferably pinned) for the streamed path.  Returns (out, stats-or-None)."""
    shape, xs = X.shape, X.stride()
    assert X.dtype is torch.float32 and len(shape) == 2 and xs[1] == 1
    n, F = shape
    on_device = X.is_cuda
    if out is None:
        Fp = (F + 3) // 4 * 4  # the library works on whole groups of 4 columns
        if on_device:
            out = [t[:, :F] for t in _results(K, (n, Fp), torch.float32, X.device, stream)]
        else:
            out = [torch.empty((n, Fp), dtype=torch.float32, pin_memory=True)[:, :F] for _ in range(K)]
    assert len(out) == K
    ldo, out_device = F, on_device
    if K > 0:
        os, out_device = out[0].stride(), out[0].is_cuda
        ldo = os[0]
        assert os[1] == 1
        for o in out:
            assert o.dtype is torch.float32 and o.shape == shape and o.stride() == os and o.is_cuda == out_device
    stats = gnnpre_stats_t() if want_stats else None
    _check(_lib.gnnpre_propagate(plan.handle, X.data_ptr(), xs[0], GNNPRE_MEM_DEVICE if on_device else GNNPRE_MEM_HOST, K,
                                 _pointers(out) if K > 0 else (ctypes.c_void_p * 1)(), ldo,
                                 GNNPRE_MEM_DEVICE if out_device else GNNPRE_MEM_HOST,
                                 _stream_ptr(stream), ctypes.byref(stats) if want_stats else None),
           "gnnpre_propagate")
    return list(out), stats


def gnnpre_hop_static(rowptr: torch.Tensor, colidx: torch.Tensor, op: int, X: torch.Tensor, out: torch.Tensor, *,
                      gin_eps: float = 0.0, stream=None) -> torch.Tensor:
    """out = A^ X in one call that allocates nothing (the caller supplies `out`); device tensors only."""
    assert X.dtype == torch.float32 and X.dim() == 2 and X.stride(1) == 1 and X.is_cuda
    assert out.dtype == torch.float32 and out.shape == X.shape and out.stride(1) == 1 and out.is_cuda
    csr = _csr(rowptr, colidx)
    _check(_lib.gnnpre_hop_static(ctypes.byref(csr), op, gin_eps, X.shape[1], X.data_ptr(), X.stride(0),
                                  out.data_ptr(), out.stride(0), _stream_ptr(stream)), "gnnpre_hop_static")
    return out


def gnnpre_lc_selftest_wait_timeout(hop: torch.Tensor, Wt: torch.Tensor, polls: int = 200, stream=None) -> int:
    """Status of a first-layer launch whose waits are made to run out (expected: -8, GNNPRE_ERR_TIMEOUT)."""
    n, F = hop.shape
    H = Wt.shape[0]
    Y = _result((min(n, 128), H), torch.float32, hop.device, stream)
    flag = _error_word(hop.device, stream)
    return int(_lib.gnnpre_lc_selftest_wait_timeout(hop.data_ptr(), n, F, hop.stride(0), Wt.data_ptr(), H, Wt.stride(0),
                                                    Y.data_ptr(), Y.stride(0), flag.data_ptr(), polls, _stream_ptr(stream)))


def gnnpre_propagate_weighted(plan: Plan, X: torch.Tensor, gamma, *, out=None, Z: torch.Tensor | None = None,
                              keep_hops: bool = True, stream=None):
    """K = len(gamma) - 1 hops and Z = gamma[0] X + sum_k gamma[k] X_k, all on the device.
    Returns (hops, Z); with keep_hops=False two buffers alternate and hops holds only the last two."""
    K = len(gamma) - 1
    assert X.is_cuda and X.dtype == torch.float32 and X.dim() == 2 and X.stride(1) == 1
    n, F = X.shape
    Fp = (F + 3) // 4 * 4
    if out is None:
        nbuf = K if keep_hops else min(K, 2)
        bufs = [t[:, :F] for t in _results(nbuf, (n, Fp), torch.float32, X.device, stream)]
        out = [bufs[k % nbuf] for k in range(K)]
    if Z is None:
        Z = _result((n, Fp), torch.float32, X.device, stream)[:, :F]
    for o in list(out) + [Z]:
        assert o.is_cuda and o.dtype == torch.float32 and o.shape == (n, F) and o.stride(1) == 1
    assert all(o.stride(0) == out[0].stride(0) for o in out)
    ptrs = _pointers(out)
    g = (ctypes.c_float * (K + 1))(*[float(v) for v in gamma])
    _check(_lib.gnnpre_propagate_weighted(plan.handle, X.data_ptr(), X.stride(0), K, ptrs, out[0].stride(0), g,
                                          Z.data_ptr(), Z.stride(0), _stream_ptr(stream)), "gnnpre_propagate_weighted")
    return list(out), Z


GNNPRE_LC_TF32, GNNPRE_LC_TF32X3 = 0, 1


def _int32_rows(batch: torch.Tensor, n: int, stream) -> torch.Tensor:
    """int64 row indices as the library takes them: what lies outside [0, n) still does (2^32 + 5 is not row 5)."""
    _wait_for_current(stream)
    with _on(stream):
        return batch.clamp(-1, n).to(torch.int32)


def _hop_pitch(n: int, F: int, pitch: int) -> int:
    """Leading dimension of hop matrices; a matrix of one row may have any, so it gets one that the library takes."""
    return pitch if n > 1 else (F + 3) // 4 * 4


def gnnpre_lc_first_layer(hops, batch, Wt: torch.Tensor, *, relu_mask: int = 0, precision: int = GNNPRE_LC_TF32,
                          out: torch.Tensor | None = None,
                          concat: bool = False, check: bool = True, stream=None) -> torch.Tensor:
    """act(hops[k][batch] @ Wt.T) for every hop on the tensor cores (Eq. 9's first dense stage).

    hops: list of device fp32 [n, F] matrices with one common row stride; batch: device int32 row indices
    or None (all rows); Wt: device fp32 [H, F].  Returns [K, B, H], or [B, K*H] with concat=True.
    precision: GNNPRE_LC_TF32 (tf32 operands) or GNNPRE_LC_TF32X3 (split operands, fp32-like accuracy).
    With check=True the call synchronises and raises if a device-side wait ran out."""
    K = len(hops)
    shape, hs = hops[0].shape, hops[0].stride()
    n, F = shape
    assert hs[1] == 1
    for h in hops:
        assert h.is_cuda and h.dtype is torch.float32 and h.shape == shape and h.stride() == hs
    H, ws = Wt.shape[0], Wt.stride()
    assert Wt.is_cuda and Wt.dtype is torch.float32 and Wt.shape == (H, F) and ws[1] == 1
    if batch is None:
        B, bptr = n, None
    else:
        if batch.dtype is torch.int64:  # the default index type of the host framework; the library takes int32
            batch = _int32_rows(batch, n, stream)
        assert batch.is_cuda and batch.dtype is torch.int32 and batch.dim() == 1 and batch.is_contiguous()
        B, bptr = batch.shape[0], batch.data_ptr()
    if out is None:
        out = _result((B, K * H) if concat else (K, B, H), torch.float32, Wt.device, stream)
    os = out.stride()
    if concat:
        assert out.shape == (B, K * H) and os[1] == 1
        ldy, hop_stride = os[0], H
    else:
        assert out.shape == (K, B, H) and os[2] == 1
        ldy, hop_stride = (os[1], os[0]) if B > 0 else (H, 0)
    flag = _error_word(Wt.device, stream) if check else None
    _check(_lib.gnnpre_lc_first_layer(_pointers(hops), K, n, F, _hop_pitch(n, F, hs[0]), bptr, B, Wt.data_ptr(), H, ws[0],
                                      relu_mask, precision, out.data_ptr(), ldy, hop_stride,
                                      flag.data_ptr() if check else None, _stream_ptr(stream)), "gnnpre_lc_first_layer")
    if check:
        _check_waits(flag, stream, "gnnpre_lc_first_layer")
    return out


GNNPRE_F32, GNNPRE_BF16, GNNPRE_F16 = 0, 1, 2
GNNPRE_I32, GNNPRE_I64 = 0, 1
_DTYPES = {torch.float32: GNNPRE_F32, torch.bfloat16: GNNPRE_BF16, torch.float16: GNNPRE_F16}
_ID_TYPES = {torch.int32: GNNPRE_I32, torch.int64: GNNPRE_I64}


def _on_current_device(*tensors) -> None:
    """The library launches on the current device's stream: operands of another device (or of the host: -1) are refused."""
    current = torch.cuda.current_device()
    for t in tensors:
        assert t.get_device() == current


def _workspace(given: torch.Tensor | None, size: int, where: str, device, stream) -> torch.Tensor:
    if size < 0:
        raise GnnpreError(size, where)
    if given is None:
        with _on(stream):
            return torch.empty(size, dtype=torch.uint8, device=device)
    assert given.dtype is torch.uint8 and given.is_contiguous() and given.numel() >= size
    return given


def gnnpre_embedding_lookup(table: torch.Tensor, ids: torch.Tensor, *, scale: float = 1.0, out: torch.Tensor | None = None,
                            stream=None) -> torch.Tensor:
    """scale * table[ids] ([N, D]); an id outside the table (padding) gives a row of zeros.

    table: device fp32, bf16 or fp16 [V, D] with stride(1) == 1; ids: device int32 or int64 [N]; out: of table's type, by default with
    rows that start on 16-byte boundaries, as gnnpre_propagate and gnnpre_lc_first_layer want them."""
    V, D = table.shape
    (N,) = ids.shape
    dtype, id_type = _DTYPES.get(table.dtype), _ID_TYPES.get(ids.dtype)
    assert dtype is not None and id_type is not None and ids.is_contiguous()
    if out is None:
        whole = 16 // table.element_size()
        out = _result((N, (D + whole - 1) // whole * whole), table.dtype, table.device, stream)
        if D % whole:
            out = out[:, :D]
    (ldt, one), (ldo, also_one) = table.stride(), out.stride()
    assert out.dtype is table.dtype and out.shape == (N, D) and (D == 1 or one == 1 == also_one)
    # (the library launches on the current device's stream: operands of another device, or of the host, are refused)
    device = torch.cuda.current_device()
    assert table.get_device() == device == ids.get_device() and out.get_device() == device
    _check(_lib.gnnpre_embedding_lookup(table.data_ptr(), V, D, ldt if V > 1 else max(ldt, D), dtype, ids.data_ptr(), id_type, N, scale,
                                        out.data_ptr(), ldo if N > 1 else max(ldo, D),
                                        _raw_stream(device) if stream is None else stream.cuda_stream), "gnnpre_embedding_lookup")
    return out


def gnnpre_embedding_grad_workspace(num_rows: int, dim: int, count: int) -> int:
    """Bytes of workspace that gnnpre_embedding_grad needs for `count` ids into a [num_rows, dim] table."""
    size = _lib.gnnpre_embedding_grad_workspace(num_rows, dim, count)
    if size < 0:
        raise GnnpreError(size, "gnnpre_embedding_grad_workspace")
    return size


def gnnpre_embedding_grad(d_out: torch.Tensor, ids: torch.Tensor, num_rows: int, *, scale: float = 1.0, out: torch.Tensor | None = None,
                          accumulate: bool = False, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Gradient of gnnpre_embedding_lookup in its table: row v is scale * (sum of the rows of d_out whose id is v), [num_rows, D].

    d_out: device fp32, bf16 or fp16 [N, D]; out: of d_out's type or fp32 (the default).  With accumulate=True it is added to
    out (rows that no id asks for stay untouched).  workspace: uint8 tensor of gnnpre_embedding_grad_workspace bytes, for callers
    that keep one; otherwise one is taken from torch's allocator."""
    N, D = d_out.shape
    dtype, id_type = _DTYPES.get(d_out.dtype), _ID_TYPES.get(ids.dtype)
    assert dtype is not None and id_type is not None and ids.shape == (N,) and ids.is_contiguous()
    assert out is not None or not accumulate
    if out is None:
        out = _result((num_rows, D), torch.float32, d_out.device, stream)
    (ldd, one), (ldt, also_one) = d_out.stride(), out.stride()
    to = _DTYPES.get(out.dtype)
    assert to in (dtype, GNNPRE_F32) and out.shape == (num_rows, D) and (D == 1 or one == 1 == also_one)
    room = _workspace(workspace, _lib.gnnpre_embedding_grad_workspace(num_rows, D, N), "gnnpre_embedding_grad", d_out.device, stream)
    device = torch.cuda.current_device()
    assert d_out.get_device() == device == ids.get_device() and out.get_device() == device == room.get_device()
    _check(_lib.gnnpre_embedding_grad(d_out.data_ptr(), ldd if N > 1 else max(ldd, D), dtype, ids.data_ptr(), id_type, N, num_rows, D, scale,
                                      int(accumulate), out.data_ptr(), ldt if num_rows > 1 else max(ldt, D), to, room.data_ptr(),
                                      room.numel(), _raw_stream(device) if stream is None else stream.cuda_stream),
           "gnnpre_embedding_grad")
    return out


def gnnpre_lc_first_layer_grad_workspace(num_hops: int, batch_size: int, feat_dim: int, hidden: int) -> int:
    """Bytes of workspace that gnnpre_lc_first_layer_grad needs."""
    size = _lib.gnnpre_lc_first_layer_grad_workspace(num_hops, batch_size, feat_dim, hidden)
    if size < 0:
        raise GnnpreError(size, "gnnpre_lc_first_layer_grad_workspace")
    return size


def gnnpre_lc_first_layer_grad(hops, batch, dY: torch.Tensor, *, Y: torch.Tensor | None = None, relu_mask: int = 0,
                               out: torch.Tensor | None = None, accumulate: bool = False, concat: bool = False,
                               workspace: torch.Tensor | None = None, check: bool = True, stream=None) -> torch.Tensor:
    """Gradient of gnnpre_lc_first_layer in its weight, [H, F]: sum over the hops of dZ_k.T @ hops[k][batch], dZ_k = dY_k where Y_k > 0
    for the hops of relu_mask, dY_k for the others.

    hops, batch as in the forward call; dY and Y (its result; needed with relu_mask) are [K, B, H], or [B, K*H] with concat=True.  With
    accumulate=True the gradient is added to out.  workspace: uint8 tensor of gnnpre_lc_first_layer_grad_workspace bytes, for callers
    that keep one.  With check=True the call synchronises and raises if a device-side wait ran out."""
    K = len(hops)
    shape, hs = hops[0].shape, hops[0].stride()
    n, F = shape
    device = torch.cuda.current_device()
    assert hs[1] == 1 or F == 1
    for h in hops:
        assert h.dtype is torch.float32 and h.shape == shape and h.stride() == hs and h.get_device() == device
    if batch is None:
        N, bptr = n, None
    else:
        if batch.dtype is torch.int64:
            batch = _int32_rows(batch, n, stream)
        (N,) = batch.shape
        assert batch.dtype is torch.int32 and batch.is_contiguous() and batch.get_device() == device
        bptr = batch.data_ptr()
    last = dY.shape[-1]
    H = last // K if concat else last
    want = (N, K * H) if concat else (K, N, H)
    layout = []  # leading dimension, distance between the hops
    for t in (dY,) if Y is None else (dY, Y):
        ts = t.stride()
        assert t.dtype is torch.float32 and t.shape == want and ts[-1] == 1 and t.get_device() == device
        ld = ts[-2] if N > 1 else max(ts[-2], want[-1])
        layout.append((ld, H if concat else ts[0]))
    assert Y is not None or not relu_mask
    if Y is None:
        layout.append((0, 0))
    assert out is not None or not accumulate
    if out is None:
        out = _result((H, F), torch.float32, dY.device, stream)
    ldw, one = out.stride()
    assert out.dtype is torch.float32 and out.shape == (H, F) and (one == 1 or F == 1) and out.get_device() == device
    room = _workspace(workspace, _lib.gnnpre_lc_first_layer_grad_workspace(K, N, F, H), "gnnpre_lc_first_layer_grad", dY.device, stream)
    assert room.get_device() == device
    flag = _error_word(dY.device, stream) if check else None
    _check(_lib.gnnpre_lc_first_layer_grad(_pointers(hops), K, n, F, _hop_pitch(n, F, hs[0]), bptr, N, dY.data_ptr(), *layout[0],
                                           Y.data_ptr() if Y is not None else None, *layout[1], relu_mask, H, int(accumulate), out.data_ptr(),
                                           ldw, room.data_ptr(), room.numel(), flag.data_ptr() if check else None,
                                           _raw_stream(device) if stream is None else stream.cuda_stream), "gnnpre_lc_first_layer_grad")
    if check:
        _check_waits(flag, stream, "gnnpre_lc_first_layer_grad")
    return out


def gnnpre_lc_grad_selftest_wait_timeout(hop: torch.Tensor, dY: torch.Tensor, polls: int = 200, stream=None) -> int:
    """Status of a weight gradient whose waits are made to run out (expected: -8, GNNPRE_ERR_TIMEOUT)."""
    n, F = hop.shape
    H = dY.shape[1]
    assert dY.shape[0] == n
    out = _result((H, F), torch.float32, hop.device, stream)
    room = _workspace(None, gnnpre_lc_first_layer_grad_workspace(1, n, F, H), "gnnpre_lc_grad_selftest_wait_timeout", hop.device, stream)
    flag = _error_word(hop.device, stream)
    _on_current_device(hop, dY)
    return int(_lib.gnnpre_lc_grad_selftest_wait_timeout(hop.data_ptr(), n, F, hop.stride(0), dY.data_ptr(), dY.stride(0), H,
                                                         out.data_ptr(), F, room.data_ptr(), room.numel(), flag.data_ptr(), polls,
                                                         _stream_ptr(stream)))


def gnnpre_orthogonalize_workspace(batch: int, rows: int, cols: int, steps: int) -> int:
    """Bytes of workspace that gnnpre_orthogonalize needs for `batch` matrices of [rows, cols]."""
    size = _lib.gnnpre_orthogonalize_workspace(batch, rows, cols, steps)
    if size < 0:
        raise GnnpreError(size, "gnnpre_orthogonalize_workspace")
    return size


def gnnpre_orthogonalize(G: torch.Tensor, *, steps: int = 5, coeffs=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, scale: float = 1.0,
                         out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, check: bool = True,
                         stream=None) -> torch.Tensor:
    """scale * X after `steps` steps X <- (a I + b A + c A^2) X, A = X X^T, from X = G / (||G||_F + eps): an update with its singular
    values brought to about one size.

    G: device fp32, bf16 or fp16 [rows, cols] or [batch, rows, cols] with stride 1 along the columns; out: of its type and shape, may
    be G.  workspace: uint8 tensor of gnnpre_orthogonalize_workspace bytes, for callers that keep one.  With check=True the call
    synchronises and raises if a device-side wait ran out."""
    assert G.dim() in (2, 3) and G.dtype in _DTYPES
    if out is None:
        out = _result(G.shape, G.dtype, G.device, stream)
    assert out.dtype is G.dtype and out.shape == G.shape
    a, o = (t if t.dim() == 3 else t.unsqueeze(0) for t in (G, out))
    n, rows, cols = a.shape
    assert (a.stride(2) == 1 or cols == 1) and (o.stride(2) == 1 or cols == 1)
    _on_current_device(G, out)
    size = _lib.gnnpre_orthogonalize_workspace(n, rows, cols, steps)
    room = _workspace(workspace, size, "gnnpre_orthogonalize", G.device, stream)
    _on_current_device(room)
    flag = _error_word(G.device, stream) if check else None
    ld = [max(t.stride(1), cols) if rows == 1 else t.stride(1) for t in (a, o)]
    _check(_lib.gnnpre_orthogonalize(a.data_ptr(), rows, cols, ld[0], a.stride(0), n, _DTYPES[G.dtype], steps,
                                     (ctypes.c_float * 3)(*[float(c) for c in coeffs]), eps, scale, o.data_ptr(), ld[1], o.stride(0),
                                     room.data_ptr(), room.numel(), flag.data_ptr() if check else None, _stream_ptr(stream)),
           "gnnpre_orthogonalize")
    if check:
        _check_waits(flag, stream, "gnnpre_orthogonalize")
    return out


def gnnpre_orthogonalize_selftest_wait_timeout(G: torch.Tensor, polls: int = 200, stream=None) -> int:
    """Status of products whose waits are made to run out (expected: -8, GNNPRE_ERR_TIMEOUT)."""
    rows, cols = G.shape
    assert G.dtype is torch.float32 and G.is_contiguous()
    out = _result(G.shape, G.dtype, G.device, stream)
    room = _workspace(None, gnnpre_orthogonalize_workspace(1, rows, cols, 1), "gnnpre_orthogonalize_selftest_wait_timeout", G.device, stream)
    flag = _error_word(G.device, stream)
    _on_current_device(G)
    return int(_lib.gnnpre_orthogonalize_selftest_wait_timeout(G.data_ptr(), rows, cols, out.data_ptr(), room.data_ptr(), room.numel(),
                                                               flag.data_ptr(), polls, _stream_ptr(stream)))


def gnnpre_normalize(plan: Plan, out: torch.Tensor | None = None, *, host: bool = False, stream=None) -> torch.Tensor:
    """fp32 value of every edge of the support (order of gnnpre_plan_support), on the device or in host memory."""
    m = plan.nnz_tilde
    if out is None:
        out = torch.empty(m, dtype=torch.float32, pin_memory=True) if host else _result((m,), torch.float32, "cuda", stream)
    assert out.dtype == torch.float32 and out.numel() == m and out.is_contiguous()
    _check(_lib.gnnpre_normalize(plan.handle, out.data_ptr(), _mem_of(out), _stream_ptr(stream)), "gnnpre_normalize")
    return out


def gnnpre_solve_normalisation_blocks(B_A, B_S, B_D, alpha_A, alpha_S, alpha_D, B_GPU, max_a):
    a = ctypes.c_int64()
    rc = _lib.gnnpre_solve_normalisation_blocks(B_A, B_S, B_D, alpha_A, alpha_S, alpha_D, B_GPU, max_a, ctypes.byref(a))
    if rc == -6:
        return -1
    _check(rc, "gnnpre_solve_normalisation_blocks")
    return a.value


def gnnpre_selftest_wait_timeout(plan: Plan, polls: int = 200, stream=None) -> int:
    """Status of a device wait that is made to run out (expected: -8, GNNPRE_ERR_TIMEOUT)."""
    return int(_lib.gnnpre_selftest_wait_timeout(plan.handle, polls, _stream_ptr(stream)))


def gnnpre_selftest_wait_timeout_async(plan: Plan, polls: int = 200, stream=None) -> None:
    """Enqueues the wait that runs out; gnnpre_plan_status then reports it once."""
    _check(_lib.gnnpre_selftest_wait_timeout_async(plan.handle, polls, _stream_ptr(stream)),
           "gnnpre_selftest_wait_timeout_async")


def gnnpre_plan_status(plan: Plan, stream=None) -> int:
    """Synchronises `stream` and returns 0, or -8 (GNNPRE_ERR_TIMEOUT) once if a kernel of the plan gave up a wait."""
    return int(_lib.gnnpre_plan_status(plan.handle, _stream_ptr(stream)))


def gnnpre_gather_ceiling(plan: Plan, X: torch.Tensor, sink: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Enqueues the fetches of one hop (rows summed plainly, nothing stored but one float per segment): the
    yardstick the segment kernels are measured against when X fits the L2.  Returns the sink buffer."""
    assert X.is_cuda and X.dtype == torch.float32 and X.dim() == 2 and X.stride(1) == 1
    nseg = gnnpre_plan_info(plan)["num_segments"]
    if sink is None:
        sink = _result((max(nseg, 1),), torch.float32, X.device, stream)
    assert sink.is_cuda and sink.dtype == torch.float32 and sink.numel() >= nseg and sink.is_contiguous()
    _check(_lib.gnnpre_gather_ceiling(plan.handle, X.data_ptr(), X.stride(0), sink.data_ptr(), _stream_ptr(stream)),
           "gnnpre_gather_ceiling")
    return sink


def gnnpre_describe_panels(feat_dim: int, slab_width: int, K: int):
    """(number of upload slabs, list of jobs) of the narrow-first panel schedule; a job is a dict with keys
    k, lo, hi, upload, drain_lo, drain_hi.  Host only."""
    ns, nj = ctypes.c_int32(), ctypes.c_int32()
    _check(_lib.gnnpre_describe_panels(feat_dim, slab_width, K, None, 0, ctypes.byref(ns), ctypes.byref(nj)),
           "gnnpre_describe_panels")
    buf = (ctypes.c_int32 * (6 * max(nj.value, 1)))()
    _check(_lib.gnnpre_describe_panels(feat_dim, slab_width, K, buf, nj.value, ctypes.byref(ns), ctypes.byref(nj)),
           "gnnpre_describe_panels")
    keys = ("k", "lo", "hi", "upload", "drain_lo", "drain_hi")
    return ns.value, [dict(zip(keys, buf[6 * i:6 * i + 6])) for i in range(nj.value)]


def gnnpre_inject_alloc_failure(device_countdown: int = -1, host_countdown: int = -1) -> None:
    """Test hook: the library's (countdown + 1)-th next allocation of that kind is reported as failed; -1 disarms."""
    _check(_lib.gnnpre_inject_alloc_failure(device_countdown, host_countdown), "gnnpre_inject_alloc_failure")


def gnnpre_release_cached_memory() -> None:
    """Frees the device memory that a closed plan left for the next one (at most 128 MB per device)."""
    _check(_lib.gnnpre_release_cached_memory(), "gnnpre_release_cached_memory")


def gnnpre_solve_budget(B_S, B_X, B_fixed, beta_S, beta_X, B_GPU, max_b, max_c):
    b, c = ctypes.c_int64(), ctypes.c_int64()
    rc = _lib.gnnpre_solve_budget(B_S, B_X, B_fixed, beta_S, beta_X, B_GPU, max_b, max_c, ctypes.byref(b),
                                  ctypes.byref(c))
    if rc == -6:
        return None
    _check(rc, "gnnpre_solve_budget")
    return b.value, c.value


def gnnpre_status_string(status: int) -> str:
    return _lib.gnnpre_status_string(status).decode()


def exported_symbols():
    return ["gnnpre_degrees", "gnnpre_build_plan", "gnnpre_plan_info", "gnnpre_plan_block", "gnnpre_plan_scales",
            "gnnpre_plan_support", "gnnpre_plan_hop_order", "gnnpre_propagate", "gnnpre_propagate_weighted", "gnnpre_hop_static", "gnnpre_lc_first_layer", "gnnpre_lc_selftest_wait_timeout", "gnnpre_normalize",
            "gnnpre_embedding_lookup", "gnnpre_embedding_grad_workspace", "gnnpre_embedding_grad",
            "gnnpre_lc_first_layer_grad_workspace", "gnnpre_lc_first_layer_grad", "gnnpre_lc_grad_selftest_wait_timeout",
            "gnnpre_orthogonalize_workspace", "gnnpre_orthogonalize", "gnnpre_orthogonalize_selftest_wait_timeout",
            "gnnpre_solve_normalisation_blocks", "gnnpre_selftest_wait_timeout", "gnnpre_selftest_wait_timeout_async",
            "gnnpre_plan_status", "gnnpre_inject_alloc_failure", "gnnpre_gather_ceiling", "gnnpre_describe_panels", "gnnpre_plan_destroy", "gnnpre_release_cached_memory", "gnnpre_solve_budget",
            "gnnpre_status_string", "gnnpre_last_cuda_error"]
