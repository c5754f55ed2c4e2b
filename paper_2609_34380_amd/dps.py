"""Python binding of libdps (include/dps.h): argument marshalling only.

Every computation runs in the HIP kernels of libdps.so; this module turns
torch tensors into device pointers, passes torch's current HIP stream, and
turns status codes into exceptions.  PyTorch provides device memory and
streams, nothing else.  If libdps.so is not built, the first call raises.
"""
import collections
import ctypes
import functools
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdps.so")

MODE_FULL = 0
MODE_FAST = 1
ENC_E5M2 = 0
ENC_E4M3 = 1
ACT_FP16 = 0
ACT_FP8_ROWSCALE = 1

_STATUS = {0: "DPS_OK", 1: "DPS_ERR_INVALID_ARG", 2: "DPS_ERR_ALIGNMENT",
           3: "DPS_ERR_UNSUPPORTED", 4: "DPS_ERR_WORKSPACE", 5: "DPS_ERR_HIP",
           6: "DPS_ERR_NO_SPACE", 7: "DPS_ERR_TIMEOUT"}
ERR_NO_SPACE = 6
UNIT_FREE, UNIT_BACKED, UNIT_AVAIL, UNIT_FULL, UNIT_RESTORING = 0, 1, 2, 3, 4

EXPORTED = ("dps_select_enc", "dps_split", "dps_merge", "dps_restore", "dps_backup", "dps_quant_rows_e4m3", "dps_workspace_bytes",
            "dps_plan_info", "dps_linear", "dps_linear_static", "dps_linear_grouped", "dps_status_str", "dps_last_error",
            "dps_sum_create", "dps_sum_destroy", "dps_sum_alloc", "dps_sum_free",
            "dps_sum_restore_begin", "dps_sum_restore_done", "dps_sum_mode",
            "dps_sum_unit_state", "dps_sum_unit_of", "dps_sum_counts", "dps_sum_slots",
            "dps_vmm_granularity", "dps_vmm_create", "dps_vmm_kv_view", "dps_vmm_unit_bytes",
            "dps_vmm_map_residual", "dps_vmm_remap", "dps_vmm_unmap_residual", "dps_vmm_destroy",
            "dps_vmm_last_error", "dps_restore_worker_create", "dps_restore_worker_kick",
            "dps_restore_worker_wait_idle", "dps_restore_worker_restored",
            "dps_restore_worker_destroy", "dps_restore_worker_last_error",
            "dps_kv_map", "dps_kv_store", "dps_attn_workspace_bytes", "dps_attn_decode",
            "dps_kv_fork_workspace_bytes", "dps_kv_fork", "dps_kv_copy", "dps_kv_remap",
            "dps_attn_shared_workspace_bytes", "dps_attn_shared",
            "dps_beam_workspace_bytes", "dps_beam_select", "dps_sum_compact")


class DpsError(RuntimeError):
    def __init__(self, status, detail):
        self.status = status
        self.name = _STATUS.get(status, str(status))
        super().__init__("%s: %s" % (self.name, detail))


class CResidual(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("pool_bytes", ctypes.c_int64),
                ("slots", ctypes.c_void_p), ("n_chunks", ctypes.c_int64),
                ("log2_chunk", ctypes.c_int32)]


class CRestoreTarget(ctypes.Structure):
    _fields_ = [("backup", ctypes.c_void_p), ("numel", ctypes.c_int64), ("res", CResidual)]


class CWeight(ctypes.Structure):
    _fields_ = [("hi", ctypes.c_void_p), ("res", CResidual), ("experts", ctypes.c_int64),
                ("n", ctypes.c_int64), ("k", ctypes.c_int64), ("enc", ctypes.c_int32)]


class CKvCache(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("pool_bytes", ctypes.c_int64),
                ("block_stride", ctypes.c_int64), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_tokens", ctypes.c_int32),
                ("type", ctypes.c_int32), ("k_scale", ctypes.c_float),
                ("v_scale", ctypes.c_float)]


class CKvStep(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("q_start", ctypes.c_void_p),
                ("seq_len", ctypes.c_void_p), ("counts", ctypes.c_void_p),
                ("pos", ctypes.c_void_p), ("slot", ctypes.c_void_p), ("req", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p)]


class CKvStoreArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("heads", ctypes.c_int64), ("qkv", ctypes.c_void_p),
                ("qkv_stride", ctypes.c_int64), ("slot", ctypes.c_void_p),
                ("pos", ctypes.c_void_p), ("rope", ctypes.c_void_p), ("max_pos", ctypes.c_int64),
                ("rot", ctypes.c_int32), ("adjacent", ctypes.c_int32),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("type", ctypes.c_int32), ("q_out", ctypes.c_void_p),
                ("q_out_stride", ctypes.c_int64), ("k_out", ctypes.c_void_p),
                ("k_out_stride", ctypes.c_int64)]


class CAttnArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("heads", ctypes.c_int64), ("q", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("table", ctypes.c_void_p),
                ("requests", ctypes.c_int64), ("table_cols", ctypes.c_int64),
                ("req", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("window", ctypes.c_int32),
                ("type", ctypes.c_int32), ("scale", ctypes.c_float), ("out", ctypes.c_void_p),
                ("out_stride", ctypes.c_int64), ("lse", ctypes.c_void_p)]


class CKvForked(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("table", ctypes.c_void_p), ("seq_len", ctypes.c_void_p),
                ("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("tokens", ctypes.c_void_p),
                ("freed", ctypes.c_void_p), ("n_freed", ctypes.c_int64),
                ("counts", ctypes.c_void_p)]


class CBeamArgs(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("beams", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("logits", ctypes.c_void_p), ("logits_stride", ctypes.c_int64),
                ("type", ctypes.c_int32), ("end", ctypes.c_int32), ("score", ctypes.c_void_p),
                ("done", ctypes.c_void_p), ("keep", ctypes.c_int64),
                ("new_score", ctypes.c_void_p), ("parent", ctypes.c_void_p),
                ("token", ctypes.c_void_p), ("new_done", ctypes.c_void_p)]


_lib = None


def load_library(path=LIB_PATH):
    """Load libdps.so and declare its C signatures.  Raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("libdps.so is not built (%s); run __graft_entry__.build() or "
                           "python -m paper_2609_34380_amd.csrc.build" % path)
    lib = ctypes.CDLL(path)
    P, I64, I32, U32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32
    ST = ctypes.c_int
    lib.dps_select_enc.argtypes = [P, I64, P, P]
    lib.dps_select_enc.restype = ST
    lib.dps_split.argtypes = [ctypes.c_int, P, I64, P, ctypes.POINTER(CResidual), P]
    lib.dps_split.restype = ST
    lib.dps_merge.argtypes = [ctypes.c_int, P, ctypes.POINTER(CResidual), I64, P, P]
    lib.dps_merge.restype = ST
    lib.dps_restore.argtypes = [P, I64, ctypes.POINTER(CResidual), P, I64, I64, I64, P]
    lib.dps_restore.restype = ST
    lib.dps_backup.argtypes = [ctypes.POINTER(CResidual), P, I64, P, I64, P]
    lib.dps_backup.restype = ST
    lib.dps_quant_rows_e4m3.argtypes = [P, I64, I64, P, P, P]
    lib.dps_quant_rows_e4m3.restype = ST
    lib.dps_workspace_bytes.argtypes = [ctypes.c_int, U32, I64, I64, I64, I64]
    lib.dps_workspace_bytes.restype = ctypes.c_size_t
    lib.dps_plan_info.argtypes = [ctypes.c_int, U32, I64, I64, I64, I64, I32, P]
    lib.dps_plan_info.restype = ST
    lib.dps_linear.argtypes = [ctypes.c_int, U32, P, I64, ctypes.POINTER(CWeight), P, P,
                               ctypes.c_size_t, P]
    lib.dps_linear.restype = ST
    lib.dps_linear_static.argtypes = [ctypes.c_int, U32, P, I64, ctypes.POINTER(CWeight), P, P]
    lib.dps_linear_static.restype = ST
    lib.dps_linear_grouped.argtypes = [ctypes.c_int, U32, P, P, I64, ctypes.POINTER(CWeight),
                                       P, P, ctypes.c_size_t, P]
    lib.dps_linear_grouped.restype = ST
    PI64 = ctypes.POINTER(I64)
    lib.dps_sum_create.argtypes = [I64, I64, I64, ctypes.POINTER(P)]
    lib.dps_sum_create.restype = ST
    lib.dps_sum_destroy.argtypes = [P]
    lib.dps_sum_destroy.restype = None
    lib.dps_sum_alloc.argtypes = [P, I64, P]
    lib.dps_sum_alloc.restype = ST
    lib.dps_sum_free.argtypes = [P, P, I64, ctypes.POINTER(I32)]
    lib.dps_sum_free.restype = ST
    lib.dps_sum_restore_begin.argtypes = [P, PI64, PI64]
    lib.dps_sum_restore_begin.restype = ST
    lib.dps_sum_restore_done.argtypes = [P, I64]
    lib.dps_sum_restore_done.restype = ST
    lib.dps_sum_mode.argtypes = [P]
    lib.dps_sum_mode.restype = I32
    lib.dps_sum_unit_state.argtypes = [P, I64]
    lib.dps_sum_unit_state.restype = I32
    lib.dps_sum_unit_of.argtypes = [P, I64]
    lib.dps_sum_unit_of.restype = I64
    lib.dps_sum_counts.argtypes = [P, P]
    lib.dps_sum_counts.restype = ST
    lib.dps_sum_slots.argtypes = [P, I64, I64, I64, P]
    lib.dps_sum_slots.restype = ST
    lib.dps_vmm_granularity.argtypes = [PI64]
    lib.dps_vmm_granularity.restype = ST
    lib.dps_vmm_create.argtypes = [I64, I64, ctypes.POINTER(P)]
    lib.dps_vmm_create.restype = ST
    lib.dps_vmm_kv_view.argtypes = [P]
    lib.dps_vmm_kv_view.restype = P
    lib.dps_vmm_unit_bytes.argtypes = [P]
    lib.dps_vmm_unit_bytes.restype = I64
    lib.dps_vmm_map_residual.argtypes = [P, P, I64, ctypes.POINTER(P)]
    lib.dps_vmm_map_residual.restype = ST
    lib.dps_vmm_remap.argtypes = [P, P, I64, I32]
    lib.dps_vmm_remap.restype = ST
    lib.dps_vmm_unmap_residual.argtypes = [P, P]
    lib.dps_vmm_unmap_residual.restype = ST
    lib.dps_vmm_destroy.argtypes = [P]
    lib.dps_vmm_destroy.restype = None
    lib.dps_vmm_last_error.argtypes = []
    lib.dps_vmm_last_error.restype = ctypes.c_char_p
    lib.dps_restore_worker_create.argtypes = [P, P, I64, I64, I64, ctypes.POINTER(P)]
    lib.dps_restore_worker_create.restype = ST
    lib.dps_restore_worker_kick.argtypes = [P]
    lib.dps_restore_worker_kick.restype = ST
    lib.dps_restore_worker_wait_idle.argtypes = [P, I64]
    lib.dps_restore_worker_wait_idle.restype = ST
    lib.dps_restore_worker_restored.argtypes = [P]
    lib.dps_restore_worker_restored.restype = I64
    lib.dps_restore_worker_destroy.argtypes = [P]
    lib.dps_restore_worker_destroy.restype = None
    lib.dps_restore_worker_last_error.argtypes = []
    lib.dps_restore_worker_last_error.restype = ctypes.c_char_p
    # descriptors as pointers: a structure by reference, or its bytes
    lib.dps_kv_map.argtypes = [P, P, I64, I32, P, I64, P, I64, P, P]
    lib.dps_kv_map.restype = ST
    lib.dps_kv_store.argtypes = [P, ctypes.POINTER(CKvCache), P]
    lib.dps_kv_store.restype = ST
    lib.dps_attn_workspace_bytes.argtypes = [I64, I64, I64, I64]
    lib.dps_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.dps_attn_decode.argtypes = [P, ctypes.POINTER(CKvCache), P, ctypes.c_size_t, P]
    lib.dps_attn_decode.restype = ST
    lib.dps_kv_fork_workspace_bytes.argtypes = [I64, I64]
    lib.dps_kv_fork_workspace_bytes.restype = ctypes.c_size_t
    lib.dps_kv_fork.argtypes = [P, P, I64, I32, P, I64, P, I64, I64, P, P, ctypes.c_size_t, P]
    lib.dps_kv_fork.restype = ST
    lib.dps_kv_copy.argtypes = [ctypes.POINTER(CKvCache), P, P, P, I64, P, P]
    lib.dps_kv_copy.restype = ST
    lib.dps_kv_remap.argtypes = [P, I64, P, P, I64, P]
    lib.dps_kv_remap.restype = ST
    lib.dps_attn_shared_workspace_bytes.argtypes = [I64, I64, I64, I64, I64]
    lib.dps_attn_shared_workspace_bytes.restype = ctypes.c_size_t
    lib.dps_attn_shared.argtypes = [P, ctypes.POINTER(CKvCache), P, P, I64, P, ctypes.c_size_t, P]
    lib.dps_attn_shared.restype = ST
    lib.dps_beam_workspace_bytes.argtypes = [I64, I64, I64, I64]
    lib.dps_beam_workspace_bytes.restype = ctypes.c_size_t
    lib.dps_beam_select.argtypes = [P, P, ctypes.c_size_t, P]
    lib.dps_beam_select.restype = ST
    lib.dps_sum_compact.argtypes = [P, I64, P, P, PI64]
    lib.dps_sum_compact.restype = ST
    lib.dps_status_str.argtypes = [ST]
    lib.dps_status_str.restype = ctypes.c_char_p
    lib.dps_last_error.argtypes = []
    lib.dps_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status):
    if status != 0:
        detail = _lib.dps_last_error().decode()
        raise DpsError(status, detail)


def _stream():
    """The raw handle of torch's current stream on the current device (an int;
    building torch's Stream object costs a microsecond a call).  Callers hold
    device tensors, so the runtime is initialised."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _require_cuda(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("libdps works on device tensors only")


class Residual:
    """Residual plane of one tensor: a shared pool (uint8 device tensor) plus
    the int32 device table slots[chunk] = pool slot of that chunk."""

    def __init__(self, pool, slots, log2_chunk):
        _require_cuda(pool, slots)
        assert pool.dtype == torch.uint8 and slots.dtype == torch.int32
        self.pool = pool
        self.slots = slots
        self.log2_chunk = int(log2_chunk)

    def c(self):
        return CResidual(self.pool.data_ptr(), self.pool.numel(), self.slots.data_ptr(),
                         self.slots.numel(), self.log2_chunk)


def _null_residual():
    return CResidual(None, 0, None, 0, 0)


class NestedWeight:
    """A nested weight: upper-byte plane hi ([n][k] or [experts][n][k], uint8),
    its residual (None when only fast mode will be used) and the encoding
    (ENC_E5M2 or ENC_E4M3) both were split with."""

    def __init__(self, hi, residual, enc=ENC_E5M2):
        _require_cuda(hi)
        assert hi.dtype == torch.uint8 and hi.is_contiguous()
        assert enc in (ENC_E5M2, ENC_E4M3)
        self.hi = hi
        self.residual = residual
        self.enc = enc
        if hi.dim() == 2:
            self.experts, self.n, self.k = 1, hi.shape[0], hi.shape[1]
        elif hi.dim() == 3:
            self.experts, self.n, self.k = hi.shape
        else:   # a plain byte plane (split / merge only)
            self.experts, self.n, self.k = 1, 1, hi.numel()
        self._c = None

    def c(self):
        if self._c is None:
            res = self.residual.c() if self.residual is not None else _null_residual()
            self._c = CWeight(self.hi.data_ptr(), res, self.experts, self.n, self.k, self.enc)
            self._ref = ctypes.byref(self._c)
        return self._c

    def ref(self):
        """byref(c()), made once: the descriptor as the C calls take it."""
        if self._c is None:
            self.c()
        return self._ref


def select_enc(w, out=None):
    """Per-layer encoding for FP16 weights w (dps_select_enc): an int32 device
    tensor of one element holding ENC_E4M3 or ENC_E5M2 once the stream runs."""
    lib = load_library()
    _require_cuda(w)
    assert w.dtype == torch.float16 and w.is_contiguous()
    if out is None:
        out = torch.empty(1, dtype=torch.int32, device=w.device)
    _check(lib.dps_select_enc(_ptr(w), w.numel(), _ptr(out), _stream()))
    return out


def split(w, residual, hi=None, enc=ENC_E5M2):
    """FP16 weights -> NestedWeight; the residual bytes are written into
    residual.pool through its chunk table (dps_split)."""
    lib = load_library()
    _require_cuda(w)
    assert w.dtype == torch.float16 and w.is_contiguous()
    if hi is None:
        hi = torch.empty(w.shape, dtype=torch.uint8, device=w.device)
    res = residual.c()
    _check(lib.dps_split(enc, _ptr(w), w.numel(), _ptr(hi), ctypes.byref(res), _stream()))
    return NestedWeight(hi, residual, enc)


def merge(nw, out=None):
    """NestedWeight -> the FP16 weights its two parts describe (dps_merge)."""
    lib = load_library()
    if out is None:
        out = torch.empty(nw.hi.shape, dtype=torch.float16, device=nw.hi.device)
    res = nw.residual.c()
    _check(lib.dps_merge(nw.enc, _ptr(nw.hi), ctypes.byref(res), nw.hi.numel(), _ptr(out),
                         _stream()))
    return out


COPY_BYTES = 4 << 20   # restore copy size used in the paper


def _host_slots(residual, slots_host):
    if slots_host is None:
        slots_host = residual.slots.cpu()
    assert slots_host.dtype == torch.int32 and not slots_host.is_cuda
    return slots_host.contiguous()


def backup(residual, numel, out=None, slots_host=None, copy_bytes=COPY_BYTES):
    """The residual's logical byte stream copied into host memory (dps_backup).
    out: a uint8 CPU tensor of numel bytes, pinned for asynchronous copies
    (a new pinned tensor by default).  Completion follows the current stream."""
    lib = load_library()
    slots_host = _host_slots(residual, slots_host)
    if out is None:
        out = torch.empty(numel, dtype=torch.uint8, pin_memory=True)
    assert out.dtype == torch.uint8 and not out.is_cuda and out.numel() >= numel
    res = residual.c()
    _check(lib.dps_backup(ctypes.byref(res), _ptr(slots_host), numel, _ptr(out), copy_bytes,
                          _stream()))
    return out


def restore(backup_host, residual, numel=None, chunk_begin=0, chunk_end=None, slots_host=None,
            copy_bytes=COPY_BYTES):
    """Copy logical chunks [chunk_begin, chunk_end) of the residual stream from
    the host backup into the pool (dps_restore), on the current stream."""
    lib = load_library()
    assert backup_host.dtype == torch.uint8 and not backup_host.is_cuda
    numel = backup_host.numel() if numel is None else numel
    slots_host = _host_slots(residual, slots_host)
    if chunk_end is None:
        chunk_end = -(-numel // (1 << residual.log2_chunk))
    res = residual.c()
    _check(lib.dps_restore(_ptr(backup_host), numel, ctypes.byref(res), _ptr(slots_host),
                           chunk_begin, chunk_end, copy_bytes, _stream()))


def quant_rows_e4m3(x):
    """FP16 [m][k] -> (E4M3 codes uint8 [m][k], float32 power-of-two row scale [m])."""
    lib = load_library()
    _require_cuda(x)
    assert x.dtype == torch.float16 and x.dim() == 2 and x.is_contiguous()
    m, k = x.shape
    xq = torch.empty((m, k), dtype=torch.uint8, device=x.device)
    scale = torch.empty(m, dtype=torch.float32, device=x.device)
    _check(lib.dps_quant_rows_e4m3(_ptr(x), m, k, _ptr(xq), _ptr(scale), _stream()))
    return xq, scale


def workspace_bytes(mode, act, rows, n, k, experts=1):
    lib = load_library()
    return lib.dps_workspace_bytes(mode, act, rows, n, k, experts)


KERNEL_NAMES = {0: "gemv", 1: "rows", 2: "decode", 3: "gemm_f16", 4: "gemm_fp8"}


def plan_info(mode, act, rows, n, k, experts=1, log2_chunk=21):
    """The launch plan of a linear call (dps_plan_info): a dict with the
    kernel family, weight rows and token rows per block tile, K splits and
    K elements per split."""
    lib = load_library()
    info = (ctypes.c_int64 * 5)()
    _check(lib.dps_plan_info(mode, _act_flag(act), rows, n, k, experts, log2_chunk, info))
    return {"kernel": KERNEL_NAMES[info[0]], "tile_rows": info[1], "tile_tokens": info[2],
            "splits": info[3], "ksplit": info[4]}


def _act_flag(act):
    if act in ("fp16", ACT_FP16):
        return ACT_FP16
    if act in ("fp8", ACT_FP8_ROWSCALE):
        return ACT_FP8_ROWSCALE
    raise ValueError("act must be 'fp16' or 'fp8'")


@functools.lru_cache(maxsize=1024)
def _workspace_need(mode, flag, rows, n, k, experts, device_index):
    """workspace_bytes() of a shape on the current device (the plan depends
    on the device's CU count alone)."""
    return workspace_bytes(mode, flag, rows, n, k, experts)


def _workspace(mode, flag, rows, nw, device, workspace):
    need = _workspace_need(mode, flag, rows, nw.n, nw.k, nw.experts, torch.cuda.current_device())
    if need == 0:
        return None, 0
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, workspace.numel()


def linear(x, nw, mode, act="fp16", out=None, workspace=None):
    """Y = X . W^T through dps_linear; mode MODE_FULL or MODE_FAST."""
    lib = _lib or load_library()
    if not x.is_cuda:
        _require_cuda(x)
    assert x.dtype == torch.float16 and x.dim() == 2 and x.is_contiguous()
    flag = _act_flag(act)
    m = x.shape[0]
    if out is None:
        out = x.new_empty((m, nw.n))
    ws, ws_bytes = _workspace(mode, flag, m, nw, x.device, workspace)
    status = lib.dps_linear(mode, flag, x.data_ptr(), m, nw.ref(), out.data_ptr(), _ptr(ws),
                            ws_bytes, _stream())
    if status:
        _check(status)
    return out


STATIC_SCRATCH_BYTES = 64 << 20   # DPS_STATIC_SCRATCH_BYTES


def linear_static(x, nw, mode, act="fp16", out=None):
    """Y = X . W^T through dps_linear_static: the library's static device
    scratch instead of a workspace, so the call allocates nothing (beyond
    `out` when it is not given)."""
    lib = load_library()
    _require_cuda(x)
    assert x.dtype == torch.float16 and x.dim() == 2 and x.is_contiguous()
    flag = _act_flag(act)
    m = x.shape[0]
    if out is None:
        out = torch.empty((m, nw.n), dtype=torch.float16, device=x.device)
    _check(lib.dps_linear_static(mode, flag, _ptr(x), m, nw.ref(), _ptr(out),
                                 _stream()))
    return out


def linear_grouped(x_sorted, offsets, nw, mode, act="fp16", out=None, workspace=None):
    """MoE grouped linear through dps_linear_grouped; offsets is an int32
    device tensor of experts + 1 row offsets."""
    lib = load_library()
    _require_cuda(x_sorted, offsets)
    assert offsets.dtype == torch.int32 and offsets.numel() == nw.experts + 1
    flag = _act_flag(act)
    rows = x_sorted.shape[0]
    if out is None:
        out = torch.empty((rows, nw.n), dtype=torch.float16, device=x_sorted.device)
    ws, ws_bytes = _workspace(mode, flag, rows, nw, x_sorted.device, workspace)
    _check(lib.dps_linear_grouped(mode, flag, _ptr(x_sorted), _ptr(offsets), rows,
                                  nw.ref(), _ptr(out), _ptr(ws), ws_bytes, _stream()))
    return out


def make_residual(numel, log2_chunk, device, slots=None, pool=None):
    """A residual for `numel` weights: by default a pool of exactly the chunks
    needed with the identity table."""
    c = 1 << log2_chunk
    n_chunks = max(1, -(-numel // c))
    if slots is None:
        slots = torch.arange(n_chunks, dtype=torch.int32)
    slots = slots.to(device=device, dtype=torch.int32)
    if pool is None:
        pool = torch.zeros(max(n_chunks, int(slots.max().item()) + 1) * c, dtype=torch.uint8,
                           device=device)
    return Residual(pool, slots, log2_chunk)


# ---- paged KV cache ---------------------------------------------------------------

KV_F16, KV_BF16, KV_E4M3 = 0, 1, 2
_KV_TYPES = {torch.float16: KV_F16, torch.bfloat16: KV_BF16, torch.float8_e4m3fn: KV_E4M3}


def _require(cond, what):
    if not cond:
        raise ValueError(what)


def _require_int(name, t, dtype, dim):
    """An index array as the kernels take it: dtype, contiguous, on the device."""
    if not (t.dtype == dtype and t.dim() == dim and t.is_cuda and t.is_contiguous()):
        raise ValueError("%s must be a contiguous %d-d %s device tensor" % (name, dim, dtype))


class KvCache:
    """One layer's paged KV cache over `pool` (a contiguous device tensor, e.g.
    VmmRegion.kv): block b at byte offset + b * block_stride, block_tokens tokens of
    kv_heads key and value heads of head_dim (block_bytes in all; layout as
    dps_kv_cache in include/dps.h).  dtype: torch.float16, bfloat16 or
    float8_e4m3fn (values / k_scale and v_scale).  By default blocks follow
    one another from the pool's start."""

    def __init__(self, pool, block_tokens, kv_heads, head_dim, dtype, k_scale=1.0, v_scale=1.0,
                 offset=0, block_stride=None):
        _require(dtype in _KV_TYPES, "dtype must be float16, bfloat16 or float8_e4m3fn")
        _require(pool.is_cuda and pool.is_contiguous(), "pool must be a contiguous device tensor")
        _require(0 < block_tokens <= 256 and 0 < kv_heads <= 4096 and 0 < head_dim <= 256,
                 "block_tokens, kv_heads or head_dim is out of range")
        self.pool = pool
        self.block_tokens, self.kv_heads = int(block_tokens), int(kv_heads)
        self.head_dim, self.dtype = int(head_dim), dtype
        self.type = _KV_TYPES[dtype]
        self.block_bytes = 2 * self.kv_heads * self.block_tokens * self.head_dim * dtype.itemsize
        self.block_stride = self.block_bytes if block_stride is None else int(block_stride)
        nbytes = pool.numel() * pool.element_size()
        _require(0 <= offset <= nbytes, "offset is outside the pool")
        self.n_blocks = 0
        if self.block_stride > 0 and nbytes - offset >= self.block_bytes:
            self.n_blocks = (nbytes - offset - self.block_bytes) // self.block_stride + 1
        self.c = CKvCache(pool.data_ptr() + offset, nbytes - offset, self.block_stride,
                          self.kv_heads, self.head_dim, self.block_tokens, self.type,
                          float(k_scale), float(v_scale))
        self.ref = ctypes.byref(self.c)


def _packer(cls):
    """The bytes of a C structure from its fields in order: filling a ctypes
    structure costs several times as much, on calls that take microseconds."""
    codes = {ctypes.c_void_p: "P", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f"}
    made = struct.Struct("@" + "".join(codes[t] for _, t in cls._fields_) + "0q")
    assert made.size == ctypes.sizeof(cls)
    return made.pack


_pack_step, _pack_store, _pack_attn = (_packer(c) for c in (CKvStep, CKvStoreArgs, CAttnArgs))
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32
_ACT_TYPES = {torch.float16: KV_F16, torch.bfloat16: KV_BF16}


class KvMap(collections.namedtuple("KvMap", "q_start seq_len counts pos slot req kv_len")):
    """What kv_map writes: int32 q_start [requests + 1], seq_len [requests], counts
    [2] (new tokens, blocks taken), and per row of the step int32 pos, int64 slot,
    int32 req and kv_len (see dps_kv_step in include/dps.h)."""

    def step(self, requests):
        """The descriptor (bytes) of these buffers, checked and made once."""
        if self.__dict__.get("_requests") != requests:
            for name, t in zip(self._fields, self):
                _require_int(name, t, _I64 if name == "slot" else _I32, 1)
            rows = self.pos.shape[0]
            _require(self.q_start.shape[0] == requests + 1 and self.counts.shape[0] == 2 and
                     self.seq_len.shape[0] == requests and self.slot.shape[0] == rows and
                     self.req.shape[0] == rows and self.kv_len.shape[0] == rows,
                     "out does not fit the requests, or its rows differ")
            self._step = _pack_step(rows, *[t.data_ptr() for t in self])
            self._requests = requests
        return self._step


def make_kv_map(requests, rows, device):
    """Buffers for kv_map of up to `rows` rows; a graph's step keeps them."""
    i32 = functools.partial(torch.empty, dtype=_I32, device=device)
    return KvMap(i32(requests + 1), i32(requests), i32(2), i32(rows),
                 torch.empty(rows, dtype=_I64, device=device), i32(rows), i32(rows))


def kv_map(ctx_len, new_len, fresh, table, block_tokens, rows=None, out=None):
    """Block tables and slot maps of a step (dps_kv_map): every request of ctx_len
    cached and new_len new tokens (int32 device tensors) takes the blocks it needs
    from `fresh` (int32 block ids) into its row of `table` (int32 [requests][columns],
    updated in place).  rows: room for new tokens (without out); returns a KvMap."""
    lib = _lib or load_library()
    for t, dim in ((ctx_len, 1), (new_len, 1), (fresh, 1), (table, 2)):
        if not (t.dtype is _I32 and t.is_cuda and t.is_contiguous() and t.dim() == dim):
            _require_int("ctx_len, new_len and fresh (1-d) and table (2-d)", t, _I32, dim)
    requests = ctx_len.shape[0]
    held, cols = table.shape
    if not (new_len.shape[0] == requests == held):
        raise ValueError("ctx_len, new_len and table differ in requests")
    if not 0 < block_tokens <= 256:
        raise ValueError("block_tokens is out of range")
    if out is None:
        _require(rows is not None and rows >= 0, "rows (or out) is needed")
        out = make_kv_map(requests, rows, ctx_len.device)
    status = lib.dps_kv_map(ctx_len.data_ptr(), new_len.data_ptr(), requests, block_tokens,
                            fresh.data_ptr(), fresh.shape[0], table.data_ptr(), cols,
                            out.step(requests), _stream())
    if status:
        _check(status)
    return out


def _row_stride(name, t, rows, heads, dim, dtype):
    """The row stride in elements of a [rows][heads * dim] or [rows][heads][dim]
    device tensor whose rows are contiguous."""
    width = heads * dim
    if t.is_contiguous() and t.shape in ((rows, heads, dim), (rows, width)) and \
            t.dtype is dtype and t.is_cuda:
        return width
    inner = t.stride(-1) == 1 and (t.dim() == 2 or heads <= 1 or t.stride(1) == dim)
    if not (t.shape in ((rows, heads, dim), (rows, width)) and inner and t.dtype == dtype and
            t.is_cuda):
        raise ValueError("%s must be %d device rows of %d x %d contiguous %s" %
                         (name, rows, heads, dim, dtype))
    return t.stride(0) if rows > 1 else width


def kv_store(qkv, cache, slot, heads, pos=None, rope=None, q_weight=None, k_weight=None, eps=1e-6,
             adjacent=False, q_out=None, k_out=None):
    """Head norms (with q_weight and k_weight, [head_dim]) and rotation of the query
    and key heads of qkv ([rows][(heads + 2 kv_heads) * head_dim], FP16 or BF16), keys
    and values into `cache` at int64 `slot` [rows] (distinct; negative: not stored), in
    one pass (dps_kv_store).  rope: float32 [max_pos][rot], rot / 2 cosines then sines, at the
    int32 positions `pos`; adjacent: pairs (2i, 2i + 1) instead of (i, i + rot / 2).
    Returns the queries [rows][heads][head_dim] (q_out).  k_out: the finished keys
    [rows][kv_heads][head_dim] as well."""
    lib = _lib or load_library()
    rows, dim, kv_heads = qkv.shape[0], cache.head_dim, cache.kv_heads
    dtype = qkv.dtype
    kind = _ACT_TYPES.get(dtype)
    if kind is None:
        raise ValueError("qkv must be float16 or bfloat16")
    stride = _row_stride("qkv", qkv, rows, heads + 2 * kv_heads, dim, dtype)
    if not (slot.dtype is _I64 and slot.is_cuda and slot.is_contiguous() and slot.shape == (rows,)):
        raise ValueError("slot must be a contiguous int64 device tensor, one entry a row")
    at = table = None
    max_pos = rot = 0
    if rope is not None:
        if not (rope.is_cuda and rope.dtype is _F32 and rope.dim() == 2 and rope.is_contiguous()):
            raise ValueError("rope must be a contiguous float32 device tensor [max_pos][rot]")
        if not (pos is not None and pos.dtype is _I32 and pos.is_cuda and pos.is_contiguous() and
                pos.shape == (rows,)):
            raise ValueError("a rotation needs pos, contiguous int32, one entry a row")
        max_pos, rot = rope.shape
        at, table = pos.data_ptr(), rope.data_ptr()
    wq = wk = None
    if q_weight is not None or k_weight is not None:
        for w in (q_weight, k_weight):
            if not (w is not None and w.is_cuda and w.dtype is dtype and w.is_contiguous() and
                    w.shape == (dim,)):
                raise ValueError("q_weight and k_weight must be [head_dim] of qkv's dtype, both")
        wq, wk = q_weight.data_ptr(), k_weight.data_ptr()
    if q_out is None:
        q_out = torch.empty((rows, heads, dim), dtype=dtype, device=qkv.device)
    q_stride = _row_stride("q_out", q_out, rows, heads, dim, dtype)
    kp, k_stride = None, 0
    if k_out is not None:
        kp, k_stride = k_out.data_ptr(), _row_stride("k_out", k_out, rows, kv_heads, dim, dtype)
    args = _pack_store(rows, heads, qkv.data_ptr(), stride, slot.data_ptr(), at or 0, table or 0,
                       max_pos, rot, 1 if adjacent else 0, wq or 0, wk or 0, eps, kind,
                       q_out.data_ptr(), q_stride, kp or 0, k_stride)
    status = lib.dps_kv_store(args, cache.ref, _stream())
    if status:
        _check(status)
    return q_out


def attn_workspace_bytes(cache, rows, heads):
    """Workspace of attn_decode for up to `rows` rows of `heads` query heads."""
    lib = _lib or load_library()
    return lib.dps_attn_workspace_bytes(rows, heads, cache.kv_heads, cache.head_dim)


def attn_decode(q, cache, table, kv_len, req=None, scale=None, window=0, out=None, lse=None,
                workspace=None):
    """Attention of one new token a row over the paged cache (dps_attn_decode): row j
    of q ([rows][heads][head_dim]) attends positions 0 .. kv_len[j] - 1 (the last
    `window` of them if window > 0) of request req[j] (j without req), whose blocks
    are table[req[j]].  Rows of one request (a prompt's) share no loads: each reads its
    tokens anew.  scale: of the scores, 1 / sqrt(head_dim) by default.  lse:
    float32 [rows][heads] for the log of the sums.  Returns out (q's shape)."""
    lib = _lib or load_library()
    if q.dim() != 3:
        raise ValueError("q must be [rows][heads][head_dim]")
    rows, heads, dim = q.shape
    dtype = q.dtype
    kind = _ACT_TYPES.get(dtype)
    if kind is None or dim != cache.head_dim:
        raise ValueError("q must be float16 or bfloat16, of the cache's head_dim")
    q_stride = _row_stride("q", q, rows, heads, dim, dtype)
    if not (table.dtype is _I32 and table.is_cuda and table.is_contiguous() and table.dim() == 2):
        raise ValueError("table must be a contiguous int32 device tensor [requests][columns]")
    if not (kv_len.dtype is _I32 and kv_len.is_cuda and kv_len.is_contiguous() and
            kv_len.shape == (rows,)):
        raise ValueError("kv_len must be a contiguous int32 device tensor, one entry a row")
    rp = lp = 0
    if req is not None:
        if not (req.dtype is _I32 and req.is_cuda and req.is_contiguous() and req.shape == (rows,)):
            raise ValueError("req must be a contiguous int32 device tensor, one entry a row")
        rp = req.data_ptr()
    if out is None:
        out = torch.empty((rows, heads, dim), dtype=dtype, device=q.device)
    out_stride = _row_stride("out", out, rows, heads, dim, dtype)
    if lse is not None:
        if not (lse.dtype is _F32 and lse.is_cuda and lse.is_contiguous() and
                lse.shape == (rows, heads)):
            raise ValueError("lse must be a contiguous float32 device tensor [rows][heads]")
        lp = lse.data_ptr()
    if window < 0:
        raise ValueError("window is negative")
    if workspace is None:
        need = lib.dps_attn_workspace_bytes(rows, heads, cache.kv_heads, dim)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    elif not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous device tensor")
    requests, cols = table.shape
    args = _pack_attn(rows, heads, q.data_ptr(), q_stride, table.data_ptr(), requests, cols, rp,
                      kv_len.data_ptr(), min(window, 0x7fffffff), kind,
                      dim ** -0.5 if scale is None else scale, out.data_ptr(), out_stride, lp)
    status = lib.dps_attn_decode(args, cache.ref, workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream())
    if status:
        _check(status)
    return out


# ---- sequences that branch --------------------------------------------------------

BEAM_F16, BEAM_BF16, BEAM_F32 = 0, 1, 2
_BEAM_TYPES = {torch.float16: BEAM_F16, torch.bfloat16: BEAM_BF16, torch.float32: BEAM_F32}
_pack_forked, _pack_beam = _packer(CKvForked), _packer(CBeamArgs)


def _ints(name, t, dim=1):
    """An int32 array of the current device, as the kernels take it."""
    if not (t.dtype is _I32 and t.is_cuda and t.is_contiguous() and t.dim() == dim):
        _require_int(name, t, _I32, dim)
    _here(name, t)


def _here(name, t):
    """The calls go to the current device's stream."""
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError("%s is not on the current device" % name)


def _scratch(workspace, need, like):
    """The workspace of a call: the caller's, or one of `need` bytes."""
    if workspace is None:
        return torch.empty(max(need, 1), dtype=torch.uint8, device=like.device)
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous device tensor")
    _here("workspace", workspace)
    return workspace


class KvFork(collections.namedtuple("KvFork", "table seq_len src dst tokens freed counts")):
    """What kv_fork writes, int32: table [rows][columns] and seq_len [rows] of the new
    rows; the copies to make, src, dst and tokens [rows]; freed blocks; counts [2]
    (copies, blocks freed).  See dps_kv_forked in include/dps.h."""

    def descriptor(self):
        """The descriptor (bytes) of these buffers, checked and made once."""
        made = self.__dict__.get("_made")
        if made is None:
            for name, t in zip(self._fields, self):
                _ints(name, t, 2 if name == "table" else 1)
            rows = self.table.shape[0]
            for name in ("seq_len", "src", "dst", "tokens"):
                _require(getattr(self, name).shape == (rows,), "%s differs in rows" % name)
            _require(self.counts.shape == (2,), "counts must hold two values")
            made = self._made = _pack_forked(
                rows, *[t.data_ptr() for t in self[:6]], self.freed.shape[0],
                self.counts.data_ptr())
        _here("out", self.table)
        return made


def make_kv_fork(rows, columns, n_freed, device):
    """Buffers for kv_fork: rows of the step to come, room for n_freed freed blocks."""
    i32 = functools.partial(torch.empty, dtype=_I32, device=device)
    return KvFork(i32((rows, columns)), i32(rows), i32(rows), i32(rows), i32(rows), i32(n_freed),
                  i32(2))


def kv_fork_workspace_bytes(rows, n_blocks):
    """Workspace of kv_fork for `rows` new rows over a cache of n_blocks blocks."""
    lib = _lib or load_library()
    return lib.dps_kv_fork_workspace_bytes(rows, n_blocks)


def kv_fork(parent, seq_len, table, fresh, block_tokens, n_blocks, out=None, workspace=None):
    """Block tables after rows have branched, ended or changed places (dps_kv_fork):
    new row r goes on from row parent[r] of `table` (int32 [old rows][columns], lengths
    seq_len), an empty row where that is -1.  Whole blocks are shared; of a last block
    with room in it every child but the first takes a copy, in a block off `fresh`,
    which kv_copy makes (tokens=f.tokens, count=f.counts).  n_blocks: of the cache.
    Returns a KvFork (out); its table is not `table`."""
    lib = _lib or load_library()
    for name, t, dim in (("parent", parent, 1), ("seq_len", seq_len, 1), ("fresh", fresh, 1),
                         ("table", table, 2)):
        _ints(name, t, dim)
    rows, (old_rows, cols) = parent.shape[0], table.shape
    if seq_len.shape[0] != old_rows:
        raise ValueError("seq_len and table differ in rows")
    if not 0 < block_tokens <= 256:
        raise ValueError("block_tokens is out of range")
    if out is None:
        out = make_kv_fork(rows, cols, min(n_blocks, old_rows * cols), table.device)
    elif out.table.shape != (rows, cols):
        raise ValueError("out does not fit the rows, or the table's columns")
    made = out.descriptor()
    ws = _scratch(workspace, lib.dps_kv_fork_workspace_bytes(rows, n_blocks), table)
    status = lib.dps_kv_fork(parent.data_ptr(), seq_len.data_ptr(), old_rows, block_tokens,
                             table.data_ptr(), cols, fresh.data_ptr(), fresh.shape[0], n_blocks,
                             made, ws.data_ptr(), ws.numel() * ws.element_size(), _stream())
    if status:
        _check(status)
    return out


def kv_copy(cache, src, dst, tokens=None, count=None):
    """Copies of cache blocks (dps_kv_copy): the first tokens[i] tokens (all by default)
    of block src[i] to block dst[i], int32 device tensors; count: an int32 device
    tensor whose first value says how many of the pairs there are (KvFork.counts).
    Every dst is named once, and is no src."""
    lib = _lib or load_library()
    _ints("src", src)
    _ints("dst", dst)
    n = src.shape[0]
    if dst.shape[0] != n:
        raise ValueError("src and dst differ in length")
    tp = cp = None
    if tokens is not None:
        _ints("tokens", tokens)
        if tokens.shape[0] != n:
            raise ValueError("src and tokens differ in length")
        tp = tokens.data_ptr()
    if count is not None:
        _ints("count", count)
        if count.shape[0] < 1:
            raise ValueError("count is empty")
        cp = count.data_ptr()
    status = lib.dps_kv_copy(cache.ref, src.data_ptr(), dst.data_ptr(), tp, n, cp, _stream())
    if status:
        _check(status)


def kv_remap(table, src, dst):
    """Block ids src[i] (ascending) of the table become dst[i], in place (dps_kv_remap):
    the tables of a cache whose blocks kv_copy has moved."""
    lib = _lib or load_library()
    _ints("table", table, table.dim())
    _ints("src", src)
    _ints("dst", dst)
    if src.shape != dst.shape:
        raise ValueError("src and dst differ in length")
    status = lib.dps_kv_remap(table.data_ptr(), table.numel(), src.data_ptr(), dst.data_ptr(),
                              src.shape[0], _stream())
    if status:
        _check(status)
    return table


def attn_shared_workspace_bytes(cache, rows, heads, groups):
    """Workspace of attn_shared for `rows` rows of `heads` query heads in `groups` groups
    (whoever calls with several sizes takes the largest of theirs)."""
    lib = _lib or load_library()
    return lib.dps_attn_shared_workspace_bytes(rows, groups, heads, cache.kv_heads, cache.head_dim)


def attn_shared(q, cache, table, kv_len, group_start, shared_len, req=None, scale=None, out=None,
                lse=None, workspace=None):
    """attn_decode of rows that share prefixes (dps_attn_shared): rows group_start[g] ..
    group_start[g + 1] - 1 (int32 [groups + 1], ascending) have their first shared_len[g]
    tokens (int32 [groups]) in common (in the same blocks or in copies, as kv_fork leaves
    them), which are read once for all of them.  Rows in no group, and rows shorter than their
    group's prefix, attend their tokens by themselves.  Other arguments and the result
    are attn_decode's."""
    lib = _lib or load_library()
    if q.dim() != 3:
        raise ValueError("q must be [rows][heads][head_dim]")
    rows, heads, dim = q.shape
    dtype = q.dtype
    kind = _ACT_TYPES.get(dtype)
    if kind is None or dim != cache.head_dim:
        raise ValueError("q must be float16 or bfloat16, of the cache's head_dim")
    q_stride = _row_stride("q", q, rows, heads, dim, dtype)
    _here("q", q)
    for name, t, n in (("table", table, 2), ("kv_len", kv_len, 1), ("group_start", group_start, 1),
                       ("shared_len", shared_len, 1)):
        _ints(name, t, n)
    groups = shared_len.shape[0]
    if kv_len.shape[0] != rows or group_start.shape[0] != groups + 1:
        raise ValueError("kv_len has an entry a row, group_start one more than shared_len")
    rp = lp = 0
    if req is not None:
        _ints("req", req)
        if req.shape[0] != rows:
            raise ValueError("req has an entry a row")
        rp = req.data_ptr()
    if out is None:
        out = torch.empty((rows, heads, dim), dtype=dtype, device=q.device)
    out_stride = _row_stride("out", out, rows, heads, dim, dtype)
    _here("out", out)
    if lse is not None:
        if not (lse.dtype is _F32 and lse.is_cuda and lse.is_contiguous() and
                lse.shape == (rows, heads)):
            raise ValueError("lse must be a contiguous float32 device tensor [rows][heads]")
        _here("lse", lse)
        lp = lse.data_ptr()
    if workspace is None:
        need = lib.dps_attn_shared_workspace_bytes(rows, groups, heads, cache.kv_heads, dim)
        workspace = _scratch(None, need, q)
    else:
        _scratch(workspace, 0, q)
    requests, cols = table.shape
    args = _pack_attn(rows, heads, q.data_ptr(), q_stride, table.data_ptr(), requests, cols, rp,
                      kv_len.data_ptr(), 0, kind, dim ** -0.5 if scale is None else scale,
                      out.data_ptr(), out_stride, lp)
    status = lib.dps_attn_shared(args, cache.ref, group_start.data_ptr(), shared_len.data_ptr(),
                                 groups, workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream())
    if status:
        _check(status)
    return out


class BeamStep(collections.namedtuple("BeamStep", "score parent token done")):
    """What beam_select writes, [batch][keep]: float32 score, int32 parent (a row of the
    step) and token, uint8 done."""

    def checked(self, shape):
        if self.__dict__.get("_shape") != shape:
            for name, t, dtype in zip(self._fields, self, (_F32, _I32, _I32, torch.uint8)):
                _require(t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.shape == shape,
                         "%s must be a contiguous %s device tensor of %s" % (name, dtype, shape))
                _here(name, t)
            self._shape = shape
        _here("out", self.score)
        return self


def make_beam_step(batch, keep, device):
    """Buffers for beam_select."""
    new = functools.partial(torch.empty, (batch, keep), device=device)
    return BeamStep(new(dtype=_F32), new(dtype=_I32), new(dtype=_I32), new(dtype=torch.uint8))


def beam_workspace_bytes(batch, beams, vocab, keep):
    """Workspace of beam_select."""
    lib = _lib or load_library()
    return lib.dps_beam_workspace_bytes(batch, beams, vocab, keep)


def beam_select(logits, score, beams, keep=None, done=None, end=-1, out=None, workspace=None):
    """The next beams (dps_beam_select) of logits [batch * beams][vocab] (FP16, BF16 or
    FP32, rows contiguous): the `keep` (`beams` by default) best of score[row] +
    log_softmax(logits[row])[token] for each request, best first, of equal ones those
    of the lowest row and token.  score: float32, one a row; done: uint8, one a row:
    the beam has ended and stands for itself with the token `end`.  Returns a BeamStep
    (out); places without a candidate have score -inf, parent and token -1.  (Different
    logits of a row count as equal ones in any order where 64 bits cannot tell their scores
    apart.)"""
    lib = _lib or load_library()
    kind = _BEAM_TYPES.get(logits.dtype)
    if kind is None or logits.dim() != 2 or not logits.is_cuda:
        raise ValueError("logits must be float16, bfloat16 or float32 device rows")
    rows, vocab = logits.shape
    keep = beams if keep is None else keep
    if beams < 1 or rows % beams:
        raise ValueError("rows must be a multiple of beams")
    stride = vocab
    if not logits.is_contiguous():
        if logits.stride(1) != 1 and vocab > 1:
            raise ValueError("the rows of logits must be contiguous")
        stride = logits.stride(0) if rows > 1 else vocab
    _here("logits", logits)
    if not (score.dtype is _F32 and score.is_cuda and score.is_contiguous() and
            score.shape == (rows,)):
        raise ValueError("score must be a contiguous float32 device tensor, one entry a row")
    _here("score", score)
    dp = 0
    if done is not None:
        if not (done.dtype in (torch.uint8, torch.bool) and done.is_cuda and
                done.is_contiguous() and done.shape == (rows,)):
            raise ValueError("done must be a contiguous uint8 device tensor, one entry a row")
        _here("done", done)
        dp = done.data_ptr()
    batch = rows // beams
    if out is None:
        _require(0 < keep <= 256, "keep must be in 1..256")
        out = make_beam_step(batch, keep, logits.device)
    out.checked((batch, keep))
    ws = _scratch(workspace, lib.dps_beam_workspace_bytes(batch, beams, vocab, keep), logits)
    args = _pack_beam(batch, beams, vocab, logits.data_ptr(), stride, kind, end, score.data_ptr(),
                      dp, keep, out.score.data_ptr(), out.parent.data_ptr(), out.token.data_ptr(),
                      out.done.data_ptr())
    status = lib.dps_beam_select(args, ws.data_ptr(), ws.numel() * ws.element_size(), _stream())
    if status:
        _check(status)
    return out


class SumManager:
    """The SUM manager's unit bookkeeping (dps_sum_*): n_units units of
    blocks_per_unit KV blocks, residual r initially bound to unit r."""

    COUNT_NAMES = ("free", "backed", "avail", "full", "restoring", "stale", "evicted",
                   "free_blocks")

    def __init__(self, n_units, blocks_per_unit, n_res):
        lib = load_library()
        h = ctypes.c_void_p()
        _check(lib.dps_sum_create(n_units, blocks_per_unit, n_res, ctypes.byref(h)))
        self._h = h
        self.n_units, self.blocks_per_unit, self.n_res = n_units, blocks_per_unit, n_res

    def close(self):
        if self._h:
            _lib.dps_sum_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def alloc(self, n):
        """n block ids (a list), or None when the request does not fit."""
        out = (ctypes.c_int64 * max(n, 1))()
        st = _lib.dps_sum_alloc(self._h, n, out)
        if st == ERR_NO_SPACE:
            return None
        _check(st)
        return list(out[:n])

    def free(self, blocks):
        """Free the listed blocks; returns True when restoration should wake."""
        arr = (ctypes.c_int64 * max(len(blocks), 1))(*blocks)
        wake = ctypes.c_int32(0)
        _check(_lib.dps_sum_free(self._h, arr, len(blocks), ctypes.byref(wake)))
        return bool(wake.value)

    def compact(self, max_moves):
        """Moves that empty whole units (dps_sum_compact): two lists of block ids, src
        (ascending) and dst, whoever holds them.  dst is allocated from now on; src is freed
        by the caller, with free(), once the blocks are copied (kv_copy) and no table names
        it (kv_remap); of a move that the caller leaves out, dst is."""
        arr = ctypes.c_int64 * max(max_moves, 1)
        src, dst, n = arr(), arr(), ctypes.c_int64(0)
        _check(_lib.dps_sum_compact(self._h, max_moves, src, dst, ctypes.byref(n)))
        return list(src[:n.value]), list(dst[:n.value])

    def restore_begin(self):
        """(residual, unit) now held for a restore, or None."""
        r, u = ctypes.c_int64(), ctypes.c_int64()
        _check(_lib.dps_sum_restore_begin(self._h, ctypes.byref(r), ctypes.byref(u)))
        return None if r.value < 0 else (r.value, u.value)

    def restore_done(self, residual):
        _check(_lib.dps_sum_restore_done(self._h, residual))

    @property
    def mode(self):
        return _lib.dps_sum_mode(self._h)

    def unit_state(self, unit):
        return _lib.dps_sum_unit_state(self._h, unit)

    def unit_of(self, residual):
        return _lib.dps_sum_unit_of(self._h, residual)

    def counts(self):
        c = (ctypes.c_int64 * 8)()
        _check(_lib.dps_sum_counts(self._h, c))
        return dict(zip(self.COUNT_NAMES, c[:]))

    def slots(self, residual, chunks_per_unit, n_chunks):
        """Host int32 slot table of the residual in its unit."""
        out = torch.empty(max(n_chunks, 1), dtype=torch.int32)
        _check(_lib.dps_sum_slots(self._h, residual, chunks_per_unit, n_chunks,
                                  ctypes.c_void_p(out.data_ptr())))
        return out[:n_chunks]


class _DeviceBytes:
    """A __cuda_array_interface__ over device bytes the library mapped, so
    torch can view them (torch.as_tensor) without owning them."""

    def __init__(self, ptr, nbytes):
        self.__cuda_array_interface__ = {"shape": (int(nbytes),), "typestr": "|u1",
                                         "data": (int(ptr), False), "version": 3,
                                         "strides": None}


def _check_vmm(status):
    if status != 0:
        raise DpsError(status, _lib.dps_vmm_last_error().decode())


def vmm_granularity():
    """Minimum VMM allocation granularity of the current device, bytes."""
    lib = load_library()
    g = ctypes.c_int64()
    _check_vmm(lib.dps_vmm_granularity(ctypes.byref(g)))
    return g.value


class VmmRegion:
    """The shared region through the HIP virtual memory API (dps_vmm_*):
    n_units physical units of unit_bytes, all mapped into the KV view
    (`kv`, a uint8 device tensor over n_units * unit_bytes), and residual
    views mapping chosen units in chunk order.  The tensors returned view
    memory the region owns: drop them before unmapping or closing."""

    def __init__(self, n_units, unit_bytes, device=None):
        lib = load_library()
        self.device = torch.device(device) if device is not None else torch.device(
            "cuda", torch.cuda.current_device())
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check_vmm(lib.dps_vmm_create(n_units, unit_bytes, ctypes.byref(h)))
        self._h = h
        self.n_units, self.unit_bytes = int(n_units), int(unit_bytes)
        self.log2_unit = self.unit_bytes.bit_length() - 1
        self.kv = torch.as_tensor(_DeviceBytes(lib.dps_vmm_kv_view(h), n_units * unit_bytes),
                                  device=self.device)

    def map_residual(self, units):
        """A residual view (uint8 device tensor of len(units) * unit_bytes)
        whose piece i maps unit units[i]."""
        arr = (ctypes.c_int32 * len(units))(*[int(u) for u in units])
        va = ctypes.c_void_p()
        _check_vmm(_lib.dps_vmm_map_residual(self._h, arr, len(units), ctypes.byref(va)))
        return torch.as_tensor(_DeviceBytes(va.value, len(units) * self.unit_bytes),
                               device=self.device)

    def remap(self, view, piece, unit):
        _check_vmm(_lib.dps_vmm_remap(self._h, ctypes.c_void_p(view.data_ptr()), int(piece),
                                      int(unit)))

    def unmap(self, view):
        _check_vmm(_lib.dps_vmm_unmap_residual(self._h, ctypes.c_void_p(view.data_ptr())))

    def residual(self, view):
        """The Residual descriptor of a view: the view as its pool, the
        identity chunk table, chunks of one unit."""
        n = view.numel() // self.unit_bytes
        slots = torch.arange(n, dtype=torch.int32, device=self.device)
        return Residual(view, slots, self.log2_unit)

    def close(self):
        if self._h:
            self.kv = None
            _lib.dps_vmm_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class RestoreWorker:
    """The SUM manager's restore worker (dps_restore_worker_*): a native
    thread that, when kicked, restores every evicted residual the manager
    hands out -- rewrites its device chunk table to the new unit, copies the
    host backup in on its own stream, reports the restore done.
    targets[r] = (backup pinned uint8 CPU tensor, numel, Residual) of the
    manager's residual r; the tensors must outlive the worker."""

    def __init__(self, sum_manager, targets, chunks_per_unit, copy_bytes=COPY_BYTES):
        lib = load_library()
        arr = (CRestoreTarget * len(targets))()
        for i, (bk, numel, res) in enumerate(targets):
            assert bk.dtype == torch.uint8 and not bk.is_cuda and bk.numel() >= numel
            arr[i] = CRestoreTarget(bk.data_ptr(), int(numel), res.c())
        self._keep = (sum_manager, targets)
        h = ctypes.c_void_p()
        rc = lib.dps_restore_worker_create(sum_manager._h, arr, len(targets), chunks_per_unit,
                                           copy_bytes, ctypes.byref(h))
        if rc != 0:
            raise DpsError(rc, lib.dps_restore_worker_last_error().decode())
        self._h = h

    def kick(self):
        _check(_lib.dps_restore_worker_kick(self._h))

    def wait_idle(self, timeout_ms=60000):
        rc = _lib.dps_restore_worker_wait_idle(self._h, int(timeout_ms))
        if rc != 0:
            raise DpsError(rc, _lib.dps_restore_worker_last_error().decode())

    @property
    def restored(self):
        return _lib.dps_restore_worker_restored(self._h)

    def close(self):
        if self._h:
            _lib.dps_restore_worker_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
