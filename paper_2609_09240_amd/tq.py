"""ctypes binding of libtq.so — argument marshalling only.

Each function has the name of the C entry point it calls (include/tq.h) and
takes torch tensors that already live on the GPU; torch provides device
memory and the current HIP stream, every step of the computation runs in the
library's kernels.  There is no fallback: if libtq.so is missing, every call
raises.
"""

import contextlib
import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtq.so")

ABI_VERSION = 7
GROUP = 128
GROUP_BYTES = 26
OUT_FP16 = 0
OUT_FP32 = 1
MAX_GROUPED = 8
MAX_BATCH = 64
Q4_MAX_BATCH = 64
KV_MAX_ROWS = 1024
WORKSPACE_COUNT_BYTES = 16384   # at the front of a 4-bit operator's workspace

STATUS = {0: "TQ_OK", 1: "TQ_ERR_NULL", 2: "TQ_ERR_SHAPE", 3: "TQ_ERR_ALIGN",
          4: "TQ_ERR_UNSUPPORTED", 5: "TQ_ERR_HIP"}


class TqError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}")


class TqMatrix(ctypes.Structure):
    _fields_ = [
        ("n_out", ctypes.c_int64),
        ("n_in", ctypes.c_int64),
        ("group", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("codes0", ctypes.c_void_p),
        ("scale0", ctypes.c_void_p),
        ("nnz1", ctypes.c_int64),
        ("rowptr1", ctypes.c_void_p),
        ("gidx1", ctypes.c_void_p),
        ("codes1", ctypes.c_void_p),
        ("offset1", ctypes.c_void_p),
        ("scale1", ctypes.c_void_p),
        ("rowptr1_host", ctypes.c_void_p),
        ("offset0", ctypes.c_void_p),
    ]


class TqStage(ctypes.Structure):
    _fields_ = [
        ("mats", ctypes.POINTER(TqMatrix)),
        ("n", ctypes.c_int32),
        ("flags", ctypes.c_int32),
        ("x", ctypes.c_void_p),
        ("ys", ctypes.POINTER(ctypes.c_void_p)),
    ]


class TqChainInfo(ctypes.Structure):
    _fields_ = [
        ("n_stages", ctypes.c_int32),
        ("n_workgroups", ctypes.c_int32),
        ("lds_bytes", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("plan_bytes", ctypes.c_int64),
        ("sync_bytes", ctypes.c_int64),
    ]


class TqQ4Matrix(ctypes.Structure):
    _fields_ = [
        ("n_out", ctypes.c_int64),
        ("n_in", ctypes.c_int64),
        ("group", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("codes", ctypes.c_void_p),
        ("params", ctypes.c_void_p),
    ]


class TqKvCache(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("group", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("n_seqs", ctypes.c_int32),
        ("max_pages", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("n_pages", ctypes.c_int64),
        ("data", ctypes.c_void_p),
        ("pages", ctypes.c_void_p),
        ("lens", ctypes.c_void_p),
        ("refs", ctypes.c_void_p),
    ]


class TqKvRows(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("token_stride", ctypes.c_int64),
        ("head_stride", ctypes.c_int64),
    ]


class TqKvAttn(ctypes.Structure):
    _fields_ = [
        ("n_rows", ctypes.c_int32),
        ("n_tokens", ctypes.c_int32),
        ("max_q", ctypes.c_int32),
        ("n_heads", ctypes.c_int32),
        ("max_len", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("flags", ctypes.c_int32),
        ("seqs", ctypes.c_void_p),
        ("cu_q", ctypes.c_void_p),
        ("q", TqKvRows),
        ("o", ctypes.c_void_p),
        ("lse", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
    ]


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        mp = ctypes.POINTER(TqMatrix)
        qp, cp, rp = ctypes.POINTER(TqQ4Matrix), ctypes.POINTER(TqKvCache), ctypes.POINTER(TqKvRows)
        sigs = {
            "tq_abi_version": ([], ctypes.c_int),
            "tq_status_string": ([ctypes.c_int], ctypes.c_char_p),
            "tq_pack": ([vp, i64, i32, vp, vp, vp], ctypes.c_int),
            "tq_unpack": ([vp, i64, i32, vp, vp, vp], ctypes.c_int),
            "tq_validate": ([vp, i64, i32, vp, vp], ctypes.c_int),
            "tq_unpack_fp16": ([mp, vp, vp], ctypes.c_int),
            "tq_gemv": ([mp, vp, vp, i32, vp], ctypes.c_int),
            "tq_gemv_grouped": ([mp, i32, vp, ctypes.POINTER(ctypes.c_void_p), i32, vp], ctypes.c_int),
            "tq_gemm_smallbatch": ([mp, vp, i32, vp, i32, vp], ctypes.c_int),
            "tq_ternarize": ([vp, i64, i32, vp, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp], ctypes.c_int),
            "tq_select_workspace_bytes": ([i64], ctypes.c_size_t),
            "tq_select_two_plane": ([vp, i64, i32, i64, vp, vp, vp, vp, ctypes.c_size_t, vp], ctypes.c_int),
            "tq_select_two_plane_noalloc": ([vp, i64, i32, i64, vp, vp, vp, vp], ctypes.c_int),
            "tq_chain_plan": ([ctypes.POINTER(TqStage), i32, ctypes.POINTER(TqChainInfo), vp, ctypes.c_size_t],
                              ctypes.c_int),
            "tq_chain_sync_init": ([vp, ctypes.POINTER(TqChainInfo), vp], ctypes.c_int),
            "tq_gemv_chain": ([vp, vp, ctypes.POINTER(TqChainInfo), vp], ctypes.c_int),
            "tq_q4_code_bytes": ([i64, i64], ctypes.c_size_t),
            "tq_q4_param_bytes": ([i64, i64, i32], ctypes.c_size_t),
            "tq_q4_quantize": ([vp, i64, qp, vp, vp, vp], ctypes.c_int),
            "tq_q4_unpack_fp16": ([qp, vp, vp], ctypes.c_int),
            "tq_q4_workspace_bytes": ([qp, i32], ctypes.c_size_t),
            "tq_q4_gemm": ([qp, vp, i64, i32, vp, i32, vp, ctypes.c_size_t, vp], ctypes.c_int),
            "tq_kv_page_bytes": ([cp], ctypes.c_size_t),
            "tq_kv_extend": ([cp, vp, vp, i32, vp, vp, vp], ctypes.c_int),
            "tq_kv_free": ([cp, vp, i32, vp, vp], ctypes.c_int),
            "tq_kv_workspace_bytes": ([cp, i32], ctypes.c_size_t),
            "tq_kv_fork": ([cp, vp, vp, i32, vp, vp, ctypes.c_size_t, vp], ctypes.c_int),
            "tq_kv_compact": ([cp, vp, vp, ctypes.c_size_t, vp], ctypes.c_int),
            "tq_kv_copy_pages": ([cp, vp, vp, i32, vp, vp], ctypes.c_int),
            "tq_kv_append": ([cp, i32, vp, vp, vp, i32, i32, i32, rp, rp, vp, vp], ctypes.c_int),
            "tq_kv_read": ([cp, i32, vp, vp, vp, i32, i32, i32, vp, vp, vp], ctypes.c_int),
            "tq_kv_attention_workspace_bytes": ([cp, ctypes.POINTER(TqKvAttn)], ctypes.c_size_t),
            "tq_kv_attention": ([cp, i32, ctypes.POINTER(TqKvAttn), vp], ctypes.c_int),
        }
        for name, (args, res) in sigs.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        if L.tq_abi_version() != ABI_VERSION:
            raise RuntimeError(f"{LIB_PATH} implements ABI {L.tq_abi_version()}, the binding expects "
                               f"{ABI_VERSION}: rebuild it with __graft_entry__.build()")
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()   # (ctypes converts the int)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    # The raw handle of torch.cuda.current_stream(), without building the
    # Stream object: 0.5 us a call where that took 2.8.
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _used_on(stream, *tensors):
    """Tensors that a launch on `stream` reads or writes: when that is not the
    current stream, tell the caching allocator not to reuse their memory
    before the stream's work is done."""
    if stream is not None and stream != torch.cuda.current_stream():
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _after_current(stream):
    """Order `stream` after the work queued so far on the current stream
    (uploads made with .to(device) run there)."""
    if stream is not None and stream != torch.cuda.current_stream():
        stream.wait_stream(torch.cuda.current_stream())


def _host_copy(t, stream):
    """Host copy of a device tensor written on `stream`."""
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    return t.cpu()


def _check(status, where):
    if status != 0:
        raise TqError(status, where)


def _cuda(t, dtype, name):
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on the GPU")


# --------------------------------------------------------------------------
# Device-resident packed linear.
# --------------------------------------------------------------------------

@dataclass
class PackedLinear:
    """A packed linear in device memory (the buffers tq_matrix points at)."""
    n_out: int
    n_in: int
    codes0: torch.Tensor          # uint8 [26 * N * G]
    scale0: torch.Tensor          # float16 [N, G]
    rowptr1: torch.Tensor = None  # int32 [N + 1]
    gidx1: torch.Tensor = None    # int16 [nnz1] (uint16 values)
    codes1: torch.Tensor = None   # uint8 [26 * nnz1]
    offset1: torch.Tensor = None  # float16 [nnz1]
    scale1: torch.Tensor = None   # float16 [nnz1]
    rowptr1_host: torch.Tensor = None  # optional host copy of rowptr1 (int32, CPU)
    offset0: torch.Tensor = None  # optional float16 [N, G]: an offset on every group

    @property
    def nnz1(self):
        return 0 if self.gidx1 is None else int(self.gidx1.numel())

    @property
    def n_groups(self):
        return self.n_out * (self.n_in // GROUP)

    def struct(self):
        m = TqMatrix()
        m.n_out, m.n_in, m.group, m.reserved = self.n_out, self.n_in, GROUP, 0
        m.codes0 = self.codes0.data_ptr()
        m.scale0 = self.scale0.data_ptr()
        m.nnz1 = self.nnz1
        if self.nnz1:
            m.rowptr1 = self.rowptr1.data_ptr()
            m.gidx1 = self.gidx1.data_ptr()
            m.codes1 = self.codes1.data_ptr()
            m.offset1 = self.offset1.data_ptr()
            m.scale1 = self.scale1.data_ptr()
            if self.rowptr1_host is not None:
                m.rowptr1_host = self.rowptr1_host.data_ptr()
        if self.offset0 is not None:
            m.offset0 = self.offset0.data_ptr()
        return m

    def nbytes(self):
        """Bytes of the packed weights (codes, scales, plane-1 records, CSR)."""
        ng = self.n_groups
        b = GROUP_BYTES * ng + 2 * ng
        if self.offset0 is not None:
            b += 2 * ng
        if self.nnz1:
            b += 4 * (self.n_out + 1) + 32 * self.nnz1
        return b

    @classmethod
    def from_inputs(cls, inp, device="cuda", stream=None, host_rowptr=True):
        """Upload unpacked inputs (trits, scales, CSR) and pack them on the GPU.
        With host_rowptr the row pointers are also kept in host memory (see
        tq_matrix.rowptr1_host)."""
        dev = torch.device(device)
        t0 = torch.from_numpy(inp.t0.reshape(-1, GROUP)).to(dev)
        _after_current(stream)
        codes0 = tq_pack(t0, stream=stream)
        _used_on(stream, t0)
        del t0
        kw = {}
        if inp.nnz1:
            t1 = torch.from_numpy(inp.t1.reshape(-1, GROUP)).to(dev)
            _after_current(stream)
            _used_on(stream, t1)
            kw = dict(
                rowptr1=torch.from_numpy(inp.rowptr1).to(dev),
                gidx1=torch.from_numpy(inp.gidx1.view("int16")).to(dev),
                codes1=tq_pack(t1, stream=stream),
                offset1=torch.from_numpy(inp.mu1).to(dev),
                scale1=torch.from_numpy(inp.s1).to(dev),
            )
            if host_rowptr:
                kw["rowptr1_host"] = torch.from_numpy(inp.rowptr1.astype("int32")).contiguous()
        if getattr(inp, "mu0", None) is not None:
            kw["offset0"] = torch.from_numpy(inp.mu0).to(dev)
        return cls(inp.n_out, inp.n_in, codes0, torch.from_numpy(inp.s0).to(dev), **kw)


# --------------------------------------------------------------------------
# Entry points (same names as the C ABI).
# --------------------------------------------------------------------------

def tq_abi_version():
    return lib().tq_abi_version()


def tq_status_string(status):
    return lib().tq_status_string(status).decode()


def tq_pack(trits, codes=None, d_err=None, stream=None):
    """int8 trits [n, 128] -> uint8 codes [26 n] (split layout)."""
    _cuda(trits, torch.int8, "trits")
    n = trits.numel() // GROUP
    if codes is None:
        codes = torch.empty(GROUP_BYTES * n, dtype=torch.uint8, device=trits.device)
    _check(lib().tq_pack(_ptr(trits), n, GROUP, _ptr(codes), _ptr(d_err), _stream(stream)), "tq_pack")
    return codes


def tq_unpack(codes, n_groups, trits=None, d_err=None, stream=None):
    """uint8 codes [26 n] -> int8 trits [n, 128]."""
    _cuda(codes, torch.uint8, "codes")
    if trits is None:
        trits = torch.empty((n_groups, GROUP), dtype=torch.int8, device=codes.device)
    _check(lib().tq_unpack(_ptr(codes), n_groups, GROUP, _ptr(trits), _ptr(d_err), _stream(stream)),
           "tq_unpack")
    return trits


def tq_validate(codes, n_groups, d_err=None, stream=None):
    """Adds the number of invalid bytes to d_err (int32 [1]); returns d_err."""
    _cuda(codes, torch.uint8, "codes")
    if d_err is None:
        d_err = torch.zeros(1, dtype=torch.int32, device=codes.device)
    _check(lib().tq_validate(_ptr(codes), n_groups, GROUP, _ptr(d_err), _stream(stream)), "tq_validate")
    return d_err


def tq_unpack_fp16(mat, w=None, stream=None):
    """Dense fp16 W^ [N, K] in the fixed fp32 evaluation order."""
    if w is None:
        w = torch.empty((mat.n_out, mat.n_in), dtype=torch.float16, device=mat.codes0.device)
    m = mat.struct()
    _check(lib().tq_unpack_fp16(ctypes.byref(m), _ptr(w), _stream(stream)), "tq_unpack_fp16")
    return w


def _out(n, shape, out_f32, device):
    return torch.empty(shape, dtype=torch.float32 if out_f32 else torch.float16, device=device)


def tq_gemv(mat, x, y=None, out_f32=False, stream=None):
    """y = W^ x for fp16 x [K]; y fp16 [N] (or fp32)."""
    _cuda(x, torch.float16, "x")
    if y is None:
        y = _out(mat.n_out, (mat.n_out,), out_f32, x.device)
    m = mat.struct()
    _check(lib().tq_gemv(ctypes.byref(m), _ptr(x), _ptr(y), OUT_FP32 if out_f32 else OUT_FP16,
                         _stream(stream)), "tq_gemv")
    return y


def tq_gemv_grouped(mats, x, ys=None, out_f32=False, stream=None):
    """[W_i^ x for each matrix] in one launch (all matrices share K)."""
    _cuda(x, torch.float16, "x")
    n = len(mats)
    if ys is None:
        ys = [_out(m.n_out, (m.n_out,), out_f32, x.device) for m in mats]
    arr = (TqMatrix * n)(*[m.struct() for m in mats])
    yp = (ctypes.c_void_p * n)(*[y.data_ptr() for y in ys])
    _check(lib().tq_gemv_grouped(arr, n, _ptr(x), yp, OUT_FP32 if out_f32 else OUT_FP16,
                                 _stream(stream)), "tq_gemv_grouped")
    return ys


class Chain:
    """A planned chain of dependent grouped GEMVs (tq_chain_plan) with its
    device plan and sync block.  ``stages`` is a list of (matrices, x, ys):
    stage s computes tq_gemv_grouped(matrices, x) into ys and reads x only
    after stage s - 1 has finished.  Every tensor named here must outlive the
    chain."""

    def __init__(self, stages, out_f32=False, stream=None):
        import numpy as np
        self._keep = []
        arr = (TqStage * len(stages))()
        for st, (mats, x, ys) in zip(arr, stages):
            _cuda(x, torch.float16, "x")
            m = (TqMatrix * len(mats))(*[mm.struct() for mm in mats])
            yp = (ctypes.c_void_p * len(ys))(*[y.data_ptr() for y in ys])
            self._keep += [m, yp, x, list(mats), list(ys)]
            st.mats = ctypes.cast(m, ctypes.POINTER(TqMatrix))
            st.n = len(mats)
            st.flags = OUT_FP32 if out_f32 else OUT_FP16
            st.x = x.data_ptr()
            st.ys = ctypes.cast(yp, ctypes.POINTER(ctypes.c_void_p))
        self.info = TqChainInfo()
        _check(lib().tq_chain_plan(arr, len(stages), ctypes.byref(self.info), None, 0), "tq_chain_plan")
        host = np.zeros(self.info.plan_bytes, dtype=np.uint8)
        _check(lib().tq_chain_plan(arr, len(stages), ctypes.byref(self.info), host.ctypes.data_as(ctypes.c_void_p),
                                   host.nbytes), "tq_chain_plan")
        dev = stages[0][1].device
        self.plan = torch.from_numpy(host).to(dev)
        self.sync = torch.empty(self.info.sync_bytes, dtype=torch.uint8, device=dev)
        _check(lib().tq_chain_sync_init(_ptr(self.sync), ctypes.byref(self.info), _stream(stream)),
               "tq_chain_sync_init")

    def run(self, stream=None):
        """tq_gemv_chain: every stage, in order, in one launch."""
        _check(lib().tq_gemv_chain(_ptr(self.plan), _ptr(self.sync), ctypes.byref(self.info), _stream(stream)),
               "tq_gemv_chain")

    def error_flag(self, stream=None):
        """The sync block's sticky error word (nonzero after a call whose
        waits gave up)."""
        return int(_host_copy(self.sync[8:12], stream).view(torch.int32).item())


def tq_gemm_smallbatch(mat, X, Y=None, out_f32=False, stream=None):
    """Y = X W^T for fp16 X [B, K]; Y [B, N]."""
    _cuda(X, torch.float16, "X")
    B = X.shape[0]
    if Y is None:
        Y = _out(mat.n_out, (B, mat.n_out), out_f32, X.device)
    m = mat.struct()
    _check(lib().tq_gemm_smallbatch(ctypes.byref(m), _ptr(X), B, _ptr(Y), OUT_FP32 if out_f32 else OUT_FP16,
                                    _stream(stream)), "tq_gemm_smallbatch")
    return Y


def tq_ternarize(w, rec_index=None, nnz=0, iters=4, t0=None, s0=None, t1=None, offset1=None, scale1=None,
                 energy=None, want_energy=True, offset0=None, group_offsets=False, stream=None):
    """E2M-ATQ ternarisation of fp16 groups w [n, 128] (see include/tq.h).
    Returns (t0, s0, t1, offset1, scale1, energy, offset0); t1/offset1/scale1
    have nnz rows, energy is fp64 [n] (None unless requested), offset0 is
    fp16 [n] with ``group_offsets`` (or when passed in), else None."""
    _cuda(w, torch.float16, "w")
    n = w.numel() // GROUP
    dev = w.device
    if t0 is None:
        t0 = torch.empty((n, GROUP), dtype=torch.int8, device=dev)
    if s0 is None:
        s0 = torch.empty(n, dtype=torch.float16, device=dev)
    if nnz > 0:
        if t1 is None:
            t1 = torch.empty((nnz, GROUP), dtype=torch.int8, device=dev)
        if offset1 is None:
            offset1 = torch.empty(nnz, dtype=torch.float16, device=dev)
        if scale1 is None:
            scale1 = torch.empty(nnz, dtype=torch.float16, device=dev)
    if rec_index is not None:
        _cuda(rec_index, torch.int32, "rec_index")
    if want_energy and energy is None:
        energy = torch.empty(n, dtype=torch.float64, device=dev)
    if group_offsets and offset0 is None:
        offset0 = torch.empty(n, dtype=torch.float16, device=dev)
    _check(lib().tq_ternarize(_ptr(w), n, GROUP, _ptr(rec_index), nnz, iters, _ptr(t0), _ptr(s0), _ptr(t1),
                              _ptr(offset1), _ptr(scale1), _ptr(offset0), _ptr(energy), _stream(stream)),
           "tq_ternarize")
    return t0, s0, t1, offset1, scale1, energy, offset0


def tq_select_workspace_bytes(n_groups):
    return int(lib().tq_select_workspace_bytes(n_groups))


def tq_select_two_plane(energy, n_out, groups_per_row, nnz, rec_index=None, rowptr1=None, gidx1=None,
                        workspace=None, stream=None):
    """The nnz groups with the largest energy (fp64 [n_out * groups_per_row],
    on the GPU), ties to the lower flat index, and their plane-1 CSR: returns
    (rec_index int32 [n], rowptr1 int32 [n_out + 1], gidx1 int16 [nnz] holding
    uint16 group indices)."""
    _cuda(energy, torch.float64, "energy")
    n = n_out * groups_per_row
    dev = energy.device
    if rec_index is None:
        rec_index = torch.empty(n, dtype=torch.int32, device=dev)
    if rowptr1 is None:
        rowptr1 = torch.empty(n_out + 1, dtype=torch.int32, device=dev)
    if gidx1 is None:
        gidx1 = torch.empty(nnz, dtype=torch.int16, device=dev)
    if workspace is None:
        workspace = torch.empty(tq_select_workspace_bytes(n), dtype=torch.uint8, device=dev)
    _check(lib().tq_select_two_plane(_ptr(energy), n_out, groups_per_row, nnz, _ptr(rec_index), _ptr(rowptr1),
                                     _ptr(gidx1) if nnz else None, _ptr(workspace), workspace.numel(),
                                     _stream(stream)), "tq_select_two_plane")
    _used_on(stream, energy, rec_index, rowptr1, gidx1, workspace)
    return rec_index, rowptr1, gidx1


def tq_select_two_plane_noalloc(energy, n_out, groups_per_row, nnz, rec_index, rowptr1, gidx1, stream=None):
    """tq_select_two_plane on the library's static scratch: the caller
    passes every output buffer and nothing is allocated."""
    _cuda(energy, torch.float64, "energy")
    _check(lib().tq_select_two_plane_noalloc(_ptr(energy), n_out, groups_per_row, nnz, _ptr(rec_index),
                                             _ptr(rowptr1), _ptr(gidx1) if nnz else None, _stream(stream)),
           "tq_select_two_plane_noalloc")
    return rec_index, rowptr1, gidx1


def quantize_linear(W, f2=0.1, iters=4, host_rowptr=True, group_offsets=False, stream=None):
    """Packed linear from dense fp16 weights W [N, K] on the GPU: one-plane
    fits rank the groups (tq_ternarize), the top floor(f2 * N * K / 128) get
    two planes (tq_select_two_plane), then tq_ternarize and tq_pack produce
    the stored planes (section 4.2 and section 12).  With ``group_offsets``
    every group carries an offset (offset0), the paper's own representation
    of section 3, eq. 3."""
    import math
    _cuda(W, torch.float16, "W")
    N, K = W.shape
    if K % GROUP:
        raise ValueError("K must be a multiple of 128")
    ng = K // GROUP
    groups = W.reshape(N * ng, GROUP)
    _after_current(stream)
    # The ranking fit: with offsets its refinement decides the energy.
    ranking = tq_ternarize(groups, iters=iters if group_offsets else 0, group_offsets=group_offsets,
                           stream=stream)
    energy = ranking[5]
    nnz = int(math.floor(f2 * N * ng))
    rec, rowptr, gidx = tq_select_two_plane(energy, N, ng, nnz, stream=stream)
    _used_on(stream, groups, *[t for t in ranking if t is not None])
    t0, s0, t1, mu, s1, _, mu0 = tq_ternarize(groups, rec_index=rec, nnz=nnz, iters=iters, want_energy=False,
                                              group_offsets=group_offsets, stream=stream)
    codes0 = tq_pack(t0, stream=stream)
    _used_on(stream, rec, t0, t1, s0, mu, s1, mu0)
    kw = {}
    if nnz:
        kw = dict(rowptr1=rowptr, gidx1=gidx, codes1=tq_pack(t1, stream=stream), offset1=mu, scale1=s1)
        if host_rowptr:
            kw["rowptr1_host"] = _host_copy(rowptr, stream).contiguous()
    if group_offsets:
        kw["offset0"] = mu0.reshape(N, ng)
    return PackedLinear(N, K, codes0, s0.reshape(N, ng), **kw)


# --------------------------------------------------------------------------
# Products with 4-bit weights.
# --------------------------------------------------------------------------

class _Workspaces:
    """Workspaces whose counts are zeros between calls: one per stream, kept
    with the handle that owns it and made anew, larger, when a call needs more.
    Under graph capture every call gets one of its own from the graph's memory,
    its counts filled in the graph: a replay may come when the stream's buffer
    has been replaced, or run beside a call that uses it."""

    __slots__ = ("device", "by_stream")

    def __init__(self, device):
        self.device, self.by_stream = device, {}

    def _new(self, need):
        ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        ws[:WORKSPACE_COUNT_BYTES].zero_()
        return ws

    def get(self, need, stream):
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            if torch.cuda.is_current_stream_capturing():
                return self._new(need)
            key = _stream(stream)
            ws = self.by_stream.get(key)
            if ws is None or ws.numel() < need:
                ws = self.by_stream[key] = self._new(need)
        return ws


class Q4Linear:
    """A matrix of 4-bit weights in device memory (the buffers tq_q4_matrix
    points at): codes uint8, params float16, both flat and in the library's
    layout.  The buffers are fixed when it is made; their contents may
    change."""

    __slots__ = ("n_out", "n_in", "group", "codes", "params", "_ref", "_ws")

    def __init__(self, n_out, n_in, group, codes, params):
        _cuda(codes, torch.uint8, "codes")
        _cuda(params, torch.float16, "params")
        nc, np_ = lib().tq_q4_code_bytes(n_out, n_in), lib().tq_q4_param_bytes(n_out, n_in, group)
        if nc == 0 or np_ == 0:
            raise TqError(4, "Q4Linear")
        if codes.numel() != nc or 2 * params.numel() != np_:
            raise ValueError(f"codes and params must hold {nc} and {np_} bytes")
        self.n_out, self.n_in, self.group, self.codes, self.params = n_out, n_in, group, codes, params
        self._ref = ctypes.pointer(TqQ4Matrix(n_out, n_in, group, 0, codes.data_ptr(), params.data_ptr()))
        self._ws = _Workspaces(codes.device)

    @classmethod
    def empty(cls, n_out, n_in, group=GROUP, device="cuda"):
        """Buffers for a matrix, not yet written."""
        nc, np_ = lib().tq_q4_code_bytes(n_out, n_in), lib().tq_q4_param_bytes(n_out, n_in, group)
        return cls(n_out, n_in, group, torch.empty(nc, dtype=torch.uint8, device=device),
                   torch.empty(np_ // 2, dtype=torch.float16, device=device))

    def nbytes(self):
        return self.codes.numel() + 2 * self.params.numel()


def _fp16_rows(t, name):
    """fp16 [rows, K] on the GPU with adjacent elements; any row stride."""
    if not (t.is_cuda and t.dtype == torch.float16 and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1)):
        raise ValueError(f"{name} must be a float16 matrix on the GPU with adjacent elements in a row")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def tq_q4_quantize(w, group=GROUP, mat=None, stream=None):
    """Q4Linear of dense fp16 weights w [N, K]."""
    ldw = _fp16_rows(w, "w")
    if mat is None:
        mat = Q4Linear.empty(w.shape[0], w.shape[1], group, w.device)
    elif (mat.n_out, mat.n_in) != tuple(w.shape):
        raise ValueError("w does not have the shape of mat")
    _check(lib().tq_q4_quantize(_ptr(w), ldw, mat._ref, _ptr(mat.codes), _ptr(mat.params), _stream(stream)),
           "tq_q4_quantize")
    _used_on(stream, w, mat.codes, mat.params)
    return mat


def tq_q4_unpack_fp16(mat, w=None, stream=None):
    """Dense fp16 [N, K] of a Q4Linear."""
    if w is None:
        w = torch.empty((mat.n_out, mat.n_in), dtype=torch.float16, device=mat.codes.device)
    _out_buffer(w, (mat.n_out, mat.n_in), torch.float16, "w")
    _check(lib().tq_q4_unpack_fp16(mat._ref, _ptr(w), _stream(stream)), "tq_q4_unpack_fp16")
    _used_on(stream, w, mat.codes, mat.params)
    return w


def _out_buffer(t, shape, dtype, name):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}")
    _cuda(t, dtype, name)


def tq_q4_workspace_bytes(mat, B):
    """Workspace with which tq_q4_gemm of B rows is fastest."""
    return int(lib().tq_q4_workspace_bytes(mat._ref, B))


def tq_q4_gemm(mat, X, Y=None, out_f32=False, workspace=None, stream=None):
    """Y = X W^T for fp16 X [B, K] (or x [K]), B up to Q4_MAX_BATCH; Y [B, N]
    (or [N]).  A workspace of the caller's has zeros in its first
    WORKSPACE_COUNT_BYTES before its first call."""
    one = X.dim() == 1
    if one:
        X = X.unsqueeze(0)
    ldx = _fp16_rows(X, "X")
    B = X.shape[0]
    if X.shape[1] != mat.n_in:
        raise ValueError(f"X must have {mat.n_in} columns")
    dtype = torch.float32 if out_f32 else torch.float16
    shape = (mat.n_out,) if one else (B, mat.n_out)
    if Y is None:
        Y = torch.empty(shape, dtype=dtype, device=X.device)
    else:
        _out_buffer(Y, shape, dtype, "Y")
    if workspace is not None:
        _cuda(workspace, torch.uint8, "workspace")
    elif B > 16:
        need = lib().tq_q4_workspace_bytes(mat._ref, B)
        workspace = mat._ws.get(need, stream) if need else None
    _check(lib().tq_q4_gemm(mat._ref, X.data_ptr(), ldx, B, Y.data_ptr(), OUT_FP32 if out_f32 else OUT_FP16,
                            _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)),
           "tq_q4_gemm")
    if stream is not None:
        _used_on(stream, X, Y, workspace, mat.codes, mat.params)
    return Y


# --------------------------------------------------------------------------
# The key/value cache held in 4 bits.
# --------------------------------------------------------------------------

class KVCache:
    """A paged 4-bit key/value cache in device memory (the buffers tq_kv_cache
    points at): data uint8 [n_layers, n_pages, page_bytes], pages int32
    [n_seqs, max_pages] (-1: none), lens int32 [n_seqs], refs int32 [n_pages].
    The buffers are fixed when it is made; their contents belong to the
    calls below.  One cache serves one stream at a time: calls on another
    one are the caller's to order."""

    __slots__ = ("data", "pages", "lens", "refs", "n_kv_heads", "head_dim", "page_size", "group", "_ref", "_ws")

    def __init__(self, data, pages, lens, refs, n_kv_heads, head_dim, page_size=64, group=64):
        _cuda(data, torch.uint8, "data")
        for t, name in ((pages, "pages"), (lens, "lens"), (refs, "refs")):
            _cuda(t, torch.int32, name)
        if data.dim() != 3 or pages.dim() != 2 or lens.shape != pages.shape[:1] or refs.shape != data.shape[1:2]:
            raise ValueError("data [layers, n_pages, page_bytes], pages [n_seqs, max_pages], lens [n_seqs] and "
                             "refs [n_pages] do not fit each other")
        c = TqKvCache(data.shape[0], n_kv_heads, head_dim, group, page_size, pages.shape[0], pages.shape[1], 0,
                      data.shape[1], data.data_ptr(), pages.data_ptr(), lens.data_ptr(), refs.data_ptr())
        ref = ctypes.pointer(c)
        want = lib().tq_kv_page_bytes(ref)
        if want == 0:
            raise TqError(4, "KVCache")
        if data.shape[2] != want:
            raise ValueError(f"a page has {want} bytes")
        self.data, self.pages, self.lens, self.refs = data, pages, lens, refs
        self.n_kv_heads, self.head_dim, self.page_size, self.group = n_kv_heads, head_dim, page_size, group
        self._ref = ref
        self._ws = _Workspaces(data.device)

    @classmethod
    def empty(cls, n_layers, n_pages, n_seqs, max_pages, n_kv_heads, head_dim, page_size=64, group=64,
              device="cuda"):
        """A cache with every slot empty and every page free."""
        c = TqKvCache(n_layers, n_kv_heads, head_dim, group, page_size, n_seqs, max_pages, 0, n_pages)
        pb = lib().tq_kv_page_bytes(ctypes.byref(c))
        if pb == 0:
            raise TqError(4, "KVCache")
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.empty((n_layers, n_pages, pb), dtype=torch.uint8, device=device),
                   torch.full((n_seqs, max_pages), -1, **i32), torch.zeros(n_seqs, **i32), torch.zeros(n_pages, **i32),
                   n_kv_heads, head_dim, page_size, group)

    def attention_workspace(self, need, stream=None):
        """The workspace of at least `need` bytes that tq_kv_attention uses on a
        stream (the current one without) unless it is given one; while that
        stream is being captured, a new one for the graph."""
        return self._ws.get(need, stream)

    def _buffers(self):
        return self.data, self.pages, self.lens, self.refs


def _i32(t, n, name):
    """An int32 vector of n elements on the GPU, or None."""
    if t is None:
        return None
    if t.dim() != 1 or t.numel() != n:
        raise ValueError(f"{name} must have {n} elements")
    _cuda(t, torch.int32, name)
    return t.data_ptr()


def _n_rows(cache, seqs, cu):
    if seqs is not None:
        return seqs.numel()
    return cu.numel() - 1 if cu is not None else cache.lens.numel()


def tq_kv_extend(cache, cu_new=None, seqs=None, starts=None, d_err=None, stream=None):
    """Room for new tokens: row i (slot seqs[i], or slot i) gets
    cu_new[i + 1] - cu_new[i] of them (one without cu_new).  Returns starts,
    the lengths before, -1 for a row that got none."""
    n = _n_rows(cache, seqs, cu_new)
    if starts is None:
        starts = torch.empty(n, dtype=torch.int32, device=cache.lens.device)
    _check(lib().tq_kv_extend(cache._ref, _i32(seqs, n, "seqs"), _i32(cu_new, n + 1, "cu_new"), n,
                              _i32(starts, n, "starts"), _i32(d_err, 1, "d_err"), _stream(stream)), "tq_kv_extend")
    _used_on(stream, seqs, cu_new, starts, d_err, *cache._buffers())
    return starts


def tq_kv_free(cache, seqs=None, d_err=None, stream=None):
    """Empty the slots seqs (every slot without)."""
    n = _n_rows(cache, seqs, None)
    _check(lib().tq_kv_free(cache._ref, _i32(seqs, n, "seqs"), n, _i32(d_err, 1, "d_err"), _stream(stream)),
           "tq_kv_free")
    _used_on(stream, seqs, d_err, *cache._buffers())


def _workspace(workspace, need, device):
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    _cuda(workspace, torch.uint8, "workspace")
    return workspace


def tq_kv_workspace_bytes(cache, n_rows=0):
    """Workspace of tq_kv_fork of n_rows rows, or of tq_kv_compact."""
    return int(lib().tq_kv_workspace_bytes(cache._ref, n_rows))


def tq_kv_fork(cache, parents, children, d_err=None, workspace=None, stream=None):
    """Empty slots children[i] become copies of slots parents[i]."""
    n = parents.numel()
    workspace = _workspace(workspace, tq_kv_workspace_bytes(cache, n), cache.lens.device)
    _check(lib().tq_kv_fork(cache._ref, _i32(parents, n, "parents"), _i32(children, n, "children"), n,
                            _i32(d_err, 1, "d_err"), workspace.data_ptr(), workspace.numel(), _stream(stream)),
           "tq_kv_fork")
    _used_on(stream, parents, children, d_err, workspace, *cache._buffers())


def tq_kv_compact(cache, n_live=None, workspace=None, stream=None):
    """Move the pages in use to the front of the pool; n_live (int32 [1])
    gets their number."""
    workspace = _workspace(workspace, tq_kv_workspace_bytes(cache), cache.lens.device)
    _check(lib().tq_kv_compact(cache._ref, _i32(n_live, 1, "n_live"), workspace.data_ptr(), workspace.numel(),
                               _stream(stream)), "tq_kv_compact")
    _used_on(stream, n_live, workspace, *cache._buffers())


def tq_kv_copy_pages(cache, src, dst, d_err=None, stream=None):
    """Copy pages src[i] -> dst[i] in all layers."""
    n = src.numel()
    _check(lib().tq_kv_copy_pages(cache._ref, _i32(src, n, "src"), _i32(dst, n, "dst"), n, _i32(d_err, 1, "d_err"),
                                  _stream(stream)), "tq_kv_copy_pages")
    _used_on(stream, src, dst, d_err, *cache._buffers())


def _kv_rows(t, heads, d, name):
    """fp16 [T, heads, D] on the GPU as tq_kv_rows, any strides but the last."""
    if not (t.is_cuda and t.dtype == torch.float16 and t.dim() == 3 and t.shape[2] == d and t.stride(2) == 1):
        raise ValueError(f"{name} must be float16 [tokens, heads, {d}] on the GPU with adjacent channels")
    if heads is not None and t.shape[1] != heads:
        raise ValueError(f"{name} must have {heads} heads")
    return TqKvRows(t.data_ptr(), t.stride(0), t.stride(1))


def _fits(bits):
    """Numbers that are passed as 32 bits, or'ed together: ctypes would cut those
    that do not fit without a word.  Where one of them hides behind a negative
    one, a number with bit 31 set is passed, which the library refuses."""
    if bits >> 31 not in (0, -1):
        raise ValueError("a number does not fit 32 bits")


def _most(given, cu, n_tokens):
    """Tokens of a row at most, as the caller says or as there can be."""
    return given if given is not None else (n_tokens if cu is not None else 1)


def tq_kv_append(cache, layer, k, v, starts, seqs=None, cu_new=None, max_new=None, d_err=None, stream=None):
    """Quantise keys and values k, v [T, n_kv_heads, D] into the cache at the
    positions that tq_kv_extend gave (starts); row i's tokens are cu_new[i] ..
    cu_new[i + 1] - 1 (token i without cu_new).  max_new: what no row has more
    of; tokens past it are left out.  Without it as many as there are tokens,
    which is right and starts more workgroups than a number that fits."""
    n = starts.numel()
    max_new = _most(max_new, cu_new, k.shape[0])
    _fits(layer | max_new)
    if k.shape != v.shape:
        raise ValueError("k and v must have the same shape")
    kr = _kv_rows(k, cache.n_kv_heads, cache.head_dim, "k")
    vr = _kv_rows(v, cache.n_kv_heads, cache.head_dim, "v")
    _check(lib().tq_kv_append(cache._ref, layer, _i32(seqs, n, "seqs"), _i32(starts, n, "starts"),
                              _i32(cu_new, n + 1, "cu_new"), n, k.shape[0], max_new, kr, vr,
                              _i32(d_err, 1, "d_err"), _stream(stream)), "tq_kv_append")
    _used_on(stream, k, v, starts, seqs, cu_new, d_err, *cache._buffers())


def tq_kv_read(cache, layer, starts, n_tokens, seqs=None, cu_new=None, max_new=None, k=None, v=None, stream=None):
    """fp16 keys and values [n_tokens, n_kv_heads, D] of cached tokens; rows,
    positions and max_new as in tq_kv_append.  Tokens that no row has are not
    written."""
    n = starts.numel()
    max_new = _most(max_new, cu_new, n_tokens)
    _fits(layer | max_new | n_tokens)
    shape = (n_tokens, cache.n_kv_heads, cache.head_dim)
    if k is None:
        k = torch.empty(shape, dtype=torch.float16, device=cache.lens.device)
    if v is None:
        v = torch.empty(shape, dtype=torch.float16, device=cache.lens.device)
    _out_buffer(k, shape, torch.float16, "k")
    _out_buffer(v, shape, torch.float16, "v")
    _check(lib().tq_kv_read(cache._ref, layer, _i32(seqs, n, "seqs"), _i32(starts, n, "starts"),
                            _i32(cu_new, n + 1, "cu_new"), n, n_tokens, max_new, k.data_ptr(), v.data_ptr(),
                            _stream(stream)), "tq_kv_read")
    _used_on(stream, k, v, starts, seqs, cu_new, *cache._buffers())
    return k, v


def tq_kv_attention_workspace_bytes(cache, n_rows, n_heads, n_tokens=None, max_q=1, max_len=0, window=0):
    """Workspace of tq_kv_attention for n_rows rows of n_tokens queries together
    (max_q a row without), 0 where it uses none."""
    T = n_rows * max_q if n_tokens is None else n_tokens
    _fits(n_rows | T | max_q | n_heads | max_len | window)
    # (Slots that are not read here: more rows than slots are allowed where rows name theirs.)
    a = TqKvAttn(n_rows, T, max_q, n_heads, max_len, window, 1.0, OUT_FP16, cache.lens.data_ptr())
    return int(lib().tq_kv_attention_workspace_bytes(cache._ref, a))


def tq_kv_attention(cache, layer, q, seqs=None, cu_q=None, max_q=None, max_len=0, scale=None, window=0, o=None,
                    lse=None, out_f32=False, want_lse=False, workspace=None, stream=None):
    """Attention of q [T, n_heads, D], the last tokens of their slots, over the
    cache: o [T, n_heads, D] (fp16 or fp32), and with want_lse also the log of
    the softmax's sum, fp32 [T, n_heads].  scale: 1 / sqrt(D) without.  max_q:
    what no row has more queries of (the tokens past it are not computed);
    without it as many as there are tokens, which is right and may be slower
    than a number that fits.  Tokens that no row has are not written.  A
    workspace of the caller's has zeros in its first WORKSPACE_COUNT_BYTES
    before its first call."""
    T, n_heads, D = q.shape
    n = seqs.numel() if seqs is not None else (cu_q.numel() - 1 if cu_q is not None else T)
    if cu_q is None and n != T:
        raise ValueError("without cu_q, q must have one token a row")
    max_q = _most(max_q, cu_q, T)
    _fits(layer | max_q | max_len | window)
    qr = _kv_rows(q, None, cache.head_dim, "q")
    dtype = torch.float32 if out_f32 else torch.float16
    if o is None:
        o = torch.empty((T, n_heads, D), dtype=dtype, device=q.device)
    else:
        _out_buffer(o, (T, n_heads, D), dtype, "o")
    if lse is None:
        if want_lse:
            lse = torch.empty((T, n_heads), dtype=torch.float32, device=q.device)
    else:
        _out_buffer(lse, (T, n_heads), torch.float32, "lse")
    a = TqKvAttn(n, T, max_q, n_heads, max_len, window, D ** -0.5 if scale is None else scale,
                 OUT_FP32 if out_f32 else OUT_FP16, _i32(seqs, n, "seqs"), _i32(cu_q, n + 1, "cu_q"), qr,
                 o.data_ptr(), None if lse is None else lse.data_ptr(), None, 0)
    need = lib().tq_kv_attention_workspace_bytes(cache._ref, a)
    if need:
        if workspace is None:
            workspace = cache.attention_workspace(need, stream)
        else:
            _cuda(workspace, torch.uint8, "workspace")
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    _check(lib().tq_kv_attention(cache._ref, layer, a, _stream(stream)), "tq_kv_attention")
    _used_on(stream, q, seqs, cu_q, o, lse, workspace, *cache._buffers())
    return (o, lse) if lse is not None else o
