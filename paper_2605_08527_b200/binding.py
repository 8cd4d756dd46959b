"""Python binding of the C-ABI library: same names as include/marlaas.h, argument marshalling only.

Every step of the layer runs in the library's CUDA kernels; torch is used here for device memory
(tensors own the buffers) and for the current stream.  There is no CPU fallback: if the library is
missing or the device is not a B200-class (sm_100) GPU, the calls raise.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmarlaas.so")

MARLAAS_OK = 0
MARLAAS_ERR_INVALID_ARG = -1
MARLAAS_ERR_BAD_SEGMENT_TABLE = -2
MARLAAS_ERR_UNKNOWN_TENANT = -3
MARLAAS_ERR_RANK_TOO_LARGE = -4
MARLAAS_ERR_POOL_FULL = -5
MARLAAS_ERR_UNSUPPORTED_DEVICE = -6
MARLAAS_ERR_CUDA = -7
MARLAAS_ERR_DEVICE_TIMEOUT = -8
MARLAAS_ERR_DEVICE_BAD_INDEX = -9
MARLAAS_ERR_WORKSPACE_TOO_SMALL = -10

MARLAAS_FLAG_ACCUMULATE = 1
MARLAAS_FLAG_HOST_TABLE = 2
MARLAAS_FLAG_VALIDATE_SYNC = 4
MARLAAS_FLAG_CUDA_CORE_PATH = 8
MARLAAS_FLAG_REUSE_PLAN = 16
MARLAAS_FLAG_OVERLAP_PREVIOUS = 32
MARLAAS_FLAG_TOKEN_MEAN = 64
MARLAAS_FLAG_NO_STD = 128
MARLAAS_FLAG_RMS_NORM = 256

MARLAAS_DTYPE_BF16 = 0
MARLAAS_DTYPE_F32 = 1
MARLAAS_MAX_VOCABULARY = 262144
MARLAAS_POLICY_STATS = 8
MARLAAS_MAX_NORM_WIDTH = 16384
MARLAAS_MAX_HEAD_WIDTH = 65536
MARLAAS_HEAD_STATS = 4

EXPORTED_SYMBOLS = [
    "marlaas_adapter_pool_storage_bytes", "marlaas_adapter_pool_create", "marlaas_adapter_pool_destroy",
    "marlaas_adapter_pool_register", "marlaas_adapter_pool_unregister", "marlaas_adapter_pool_lookup",
    "marlaas_adapter_pool_export", "marlaas_adapter_pool_rank_stride", "marlaas_lora_workspace_bytes",
    "marlaas_lora_forward_workspace_bytes", "marlaas_debug_wait_runs_out", "marlaas_lora_forward_multi",
    "marlaas_lora_forward", "marlaas_lora_backward", "marlaas_lora_build_index", "marlaas_check_status",
    "marlaas_last_error", "marlaas_kernel_launch_count", "marlaas_kernel_timing_begin", "marlaas_kernel_timing_end",
    "marlaas_lora_static_workspace_limit", "marlaas_lora_forward_static_ws", "marlaas_adapter_pool_adamw_commit",
    "marlaas_lora_forward_workspace_min_bytes", "marlaas_adapter_pool_storage_bytes_segmented", "marlaas_adapter_pool_create_segmented", "marlaas_adapter_pool_parts",
    "marlaas_policy_workspace_bytes", "marlaas_group_advantages", "marlaas_token_logprobs", "marlaas_policy_loss",
    "marlaas_adamw_compact_state_bytes", "marlaas_adapter_pool_adamw_compact_commit", "marlaas_adamw_compact_state_export",
    "marlaas_adapter_pool_store", "marlaas_layer_norm_workspace_bytes", "marlaas_layer_norm", "marlaas_layer_norm_backward",
    "marlaas_head_cross_entropy_workspace_bytes", "marlaas_head_cross_entropy", "marlaas_lora_dropout_workspace_bytes",
    "marlaas_lora_forward_dropout", "marlaas_lora_backward_dropout",
]


class MarlaasError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"marlaas status {status}: {message}")
        self.status = status


class marlaas_adamw_t(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
                ("weight_decay", ctypes.c_float), ("grad_scale", ctypes.c_float), ("step", ctypes.c_int64)]


class marlaas_policy_loss_t(ctypes.Structure):
    _fields_ = [("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float), ("kl_coef", ctypes.c_float),
                ("entropy_coef", ctypes.c_float), ("inv_temperature", ctypes.c_float), ("grad_scale", ctypes.c_float)]


class marlaas_dropout_t(ctypes.Structure):
    _fields_ = [("rates", ctypes.c_void_p), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64)]


class marlaas_segments_t(ctypes.Structure):
    _fields_ = [("num_segments", ctypes.c_int32), ("seg_offsets", ctypes.c_void_p), ("seg_slot", ctypes.c_void_p)]


_lib: Optional[ctypes.CDLL] = None


def load_library() -> ctypes.CDLL:
    """dlopen the in-tree libmarlaas.so (built by paper_2605_08527_b200/build.py); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise MarlaasError(MARLAAS_ERR_CUDA, f"{LIB_PATH} is not built; run `python -m paper_2605_08527_b200.build` "
                           "(needs nvcc); there is no fallback path")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u32, u64, f32, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                                       ctypes.c_uint64, ctypes.c_float, ctypes.c_size_t)
    P = ctypes.POINTER
    L.marlaas_adapter_pool_storage_bytes.restype = sz
    L.marlaas_adapter_pool_storage_bytes.argtypes = [i64, i64, i32, i32]
    L.marlaas_adapter_pool_create.restype = i32
    L.marlaas_adapter_pool_create.argtypes = [P(vp), ctypes.c_int, i64, i64, i32, i32, vp, sz, vp]
    L.marlaas_adapter_pool_destroy.restype = i32
    L.marlaas_adapter_pool_destroy.argtypes = [vp]
    L.marlaas_adapter_pool_storage_bytes_segmented.restype = sz
    L.marlaas_adapter_pool_storage_bytes_segmented.argtypes = [i64, i32, P(i64), i32, i32]
    L.marlaas_adapter_pool_create_segmented.restype = i32
    L.marlaas_adapter_pool_create_segmented.argtypes = [P(vp), ctypes.c_int, i64, i32, P(i64), i32, i32, vp, sz, vp]
    L.marlaas_adapter_pool_parts.restype = i32
    L.marlaas_adapter_pool_parts.argtypes = [vp]
    L.marlaas_adapter_pool_register.restype = i32
    L.marlaas_adapter_pool_register.argtypes = [vp, u64, u64, i32, f32, vp, vp, P(i32), vp]
    L.marlaas_adapter_pool_unregister.restype = i32
    L.marlaas_adapter_pool_unregister.argtypes = [vp, u64, vp]
    L.marlaas_adapter_pool_lookup.restype = i32
    L.marlaas_adapter_pool_lookup.argtypes = [vp, u64, P(i32), P(i32), P(f32), P(u64)]
    L.marlaas_adapter_pool_export.restype = i32
    L.marlaas_adapter_pool_export.argtypes = [vp, i32, vp, vp, vp]
    L.marlaas_adapter_pool_adamw_commit.restype = i32
    L.marlaas_adapter_pool_adamw_commit.argtypes = [vp, i32, P(u64), P(u64)] + [P(vp)] * 8 + [P(marlaas_adamw_t), vp]
    L.marlaas_adapter_pool_rank_stride.restype = i32
    L.marlaas_adapter_pool_rank_stride.argtypes = [vp]
    L.marlaas_lora_workspace_bytes.restype = sz
    L.marlaas_lora_workspace_bytes.argtypes = [vp, i64]
    L.marlaas_lora_forward_workspace_bytes.restype = sz
    L.marlaas_lora_forward_workspace_bytes.argtypes = [vp, i64]
    L.marlaas_lora_forward_workspace_min_bytes.restype = sz
    L.marlaas_lora_forward_workspace_min_bytes.argtypes = [vp, i64]
    L.marlaas_lora_forward.restype = i32
    L.marlaas_lora_forward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, P(marlaas_segments_t), vp, vp, sz, u32, vp]
    L.marlaas_lora_static_workspace_limit.restype = sz
    L.marlaas_lora_static_workspace_limit.argtypes = []
    L.marlaas_lora_forward_static_ws.restype = i32
    L.marlaas_lora_forward_static_ws.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, P(marlaas_segments_t), vp, u32, vp]
    L.marlaas_lora_backward.restype = i32
    L.marlaas_lora_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp,
                                        P(marlaas_segments_t), vp, vp, sz, u32, vp]
    L.marlaas_lora_build_index.restype = i32
    L.marlaas_lora_build_index.argtypes = [vp, i64, P(marlaas_segments_t), vp, vp, vp, vp, vp, sz, u32, vp]
    L.marlaas_check_status.restype = i32
    L.marlaas_check_status.argtypes = [vp, vp]
    L.marlaas_lora_forward_multi.restype = i32
    L.marlaas_lora_forward_multi.argtypes = [ctypes.c_int32, vp, ctypes.c_uint32, vp]
    L.marlaas_debug_wait_runs_out.restype = i32
    L.marlaas_debug_wait_runs_out.argtypes = [vp, ctypes.c_uint64, vp]
    L.marlaas_kernel_timing_begin.restype = i32
    L.marlaas_kernel_timing_begin.argtypes = [vp]
    L.marlaas_kernel_timing_end.restype = i32
    L.marlaas_kernel_timing_end.argtypes = [vp, P(f32), P(i32)]
    L.marlaas_policy_workspace_bytes.restype = sz
    L.marlaas_policy_workspace_bytes.argtypes = [vp, i64, i32, i32]
    L.marlaas_group_advantages.restype = i32
    L.marlaas_group_advantages.argtypes = [vp, i64, P(marlaas_segments_t), vp, i32, vp, vp, f32, vp, vp, vp, vp, sz, u32, vp]
    L.marlaas_token_logprobs.restype = i32
    L.marlaas_token_logprobs.argtypes = [vp, i64, i64, vp, i64, i32, vp, f32, vp, vp, u32, vp]
    L.marlaas_policy_loss.restype = i32
    L.marlaas_policy_loss.argtypes = [vp, i64, i64, vp, i64, i32, vp, P(marlaas_segments_t), vp, vp, vp, vp,
                                      P(marlaas_policy_loss_t), vp, i64, vp, vp, vp, sz, u32, vp]
    L.marlaas_adamw_compact_state_bytes.restype = sz
    L.marlaas_adamw_compact_state_bytes.argtypes = [i64]
    L.marlaas_adapter_pool_adamw_compact_commit.restype = i32
    L.marlaas_adapter_pool_adamw_compact_commit.argtypes = [vp, i32, P(u64), P(u64)] + [P(vp)] * 6 + [P(i32), P(marlaas_adamw_t), u64, vp]
    L.marlaas_adamw_compact_state_export.restype = i32
    L.marlaas_adamw_compact_state_export.argtypes = [vp, i64, vp, vp, vp, vp]
    L.marlaas_adapter_pool_store.restype = i32
    L.marlaas_adapter_pool_store.argtypes = [vp, P(vp), P(vp)]
    L.marlaas_layer_norm_workspace_bytes.restype = sz
    L.marlaas_layer_norm_workspace_bytes.argtypes = [vp, i64, i64, i32, i32]
    L.marlaas_layer_norm.restype = i32
    L.marlaas_layer_norm.argtypes = [vp, i64, i64, vp, i64, P(marlaas_segments_t), vp, vp, f32, vp, i64, vp, vp, vp, sz, u32, vp]
    L.marlaas_layer_norm_backward.restype = i32
    L.marlaas_layer_norm_backward.argtypes = [vp, i64, i64, vp, i64, vp, i64, P(marlaas_segments_t), vp, vp, vp, vp, i64, vp, vp, vp, sz, u32, vp]
    L.marlaas_head_cross_entropy_workspace_bytes.restype = sz
    L.marlaas_head_cross_entropy_workspace_bytes.argtypes = [vp, i64, i64, i64, i32, i32]
    L.marlaas_head_cross_entropy.restype = i32
    L.marlaas_head_cross_entropy.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, vp, P(marlaas_segments_t), vp, f32, f32, vp, i64, vp, vp,
                                             vp, sz, u32, vp]
    L.marlaas_lora_dropout_workspace_bytes.restype = sz
    L.marlaas_lora_dropout_workspace_bytes.argtypes = [vp, i64]
    L.marlaas_lora_forward_dropout.restype = i32
    L.marlaas_lora_forward_dropout.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, P(marlaas_segments_t), P(marlaas_dropout_t), vp, vp, sz, u32, vp]
    L.marlaas_lora_backward_dropout.restype = i32
    L.marlaas_lora_backward_dropout.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, P(marlaas_segments_t), P(marlaas_dropout_t),
                                                vp, vp, sz, u32, vp]
    L.marlaas_last_error.restype = ctypes.c_char_p
    L.marlaas_last_error.argtypes = []
    L.marlaas_kernel_launch_count.restype = u64
    L.marlaas_kernel_launch_count.argtypes = []
    _lib = L
    return L


def _check(rc: int) -> None:
    if rc != MARLAAS_OK:
        raise MarlaasError(rc, load_library().marlaas_last_error().decode())


def _current() -> int:
    """The current device's current stream, without the Stream object (a few microseconds) that torch.cuda makes for it."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        return ctypes.c_void_p(_current())
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _on_stream(stream, call, *args, **kwargs):
    """`call` with `stream` made the current one, so that what it allocates is memory of that stream: a block of the stream that
    is current now may still be in use by work there.  What the call returns may be used, and let go, on either."""
    before = torch.cuda.current_stream()
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream))
    with torch.cuda.stream(stream):
        out = call(*args, **kwargs)
    todo = [out]
    while todo:
        t = todo.pop()
        if isinstance(t, (tuple, list)):
            todo += t
        elif t is not None:
            t.record_stream(stream)
            t.record_stream(before)
    return out


def _dptr(t: Optional[torch.Tensor]) -> ctypes.c_void_p:
    return ctypes.c_void_p(None if t is None else t.data_ptr())


def marlaas_last_error() -> str:
    return load_library().marlaas_last_error().decode()


def marlaas_kernel_launch_count() -> int:
    return int(load_library().marlaas_kernel_launch_count())


class marlaas_forward_call_t(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("T", ctypes.c_int64), ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64),
                ("seg", ctypes.c_void_p), ("h_save", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class Segments:
    """The token-to-adapter segment table of one mixed batch (int32 tensors, on the device or -- with
    MARLAAS_FLAG_HOST_TABLE -- on the host)."""

    def __init__(self, seg_offsets: torch.Tensor, seg_slot: torch.Tensor):
        assert seg_offsets.dtype == torch.int32 and seg_slot.dtype == torch.int32
        assert seg_offsets.is_contiguous() and seg_slot.is_contiguous()
        assert seg_offsets.numel() == seg_slot.numel() + 1
        assert seg_offsets.device == seg_slot.device
        self.seg_offsets, self.seg_slot = seg_offsets, seg_slot
        self.on_host = seg_offsets.device.type == "cpu"
        self.c = marlaas_segments_t(seg_slot.numel(), seg_offsets.data_ptr(), seg_slot.data_ptr())
        self.ref = ctypes.byref(self.c)
        self.num_segments = seg_slot.numel()

    @property
    def flags(self) -> int:
        return MARLAAS_FLAG_HOST_TABLE if self.on_host else 0


class AdapterPool:
    """marlaas_pool_t plus the torch tensor that owns its device storage.  With `parts` (the widths of several
    projections that read the same activations) the pool is made by marlaas_adapter_pool_create_segmented and d_out
    is their sum."""

    def __init__(self, d_in: int, d_out: int, max_rank: int, capacity: int, device="cuda:0", stream=None,
                 parts: Optional[Sequence[int]] = None):
        L = load_library()
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise MarlaasError(MARLAAS_ERR_UNSUPPORTED_DEVICE, "the layer runs on a CUDA device only")
        idx = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self.parts = None if parts is None else [int(p) for p in parts]
        if self.parts is not None:
            assert d_out == sum(self.parts)
        self.n_parts = 1 if self.parts is None else len(self.parts)
        self.d_in, self.d_out, self.max_rank, self.capacity = d_in, d_out, max_rank, capacity
        if self.parts is None:
            nbytes = L.marlaas_adapter_pool_storage_bytes(d_in, d_out, max_rank, capacity)
        else:
            widths = (ctypes.c_int64 * len(self.parts))(*self.parts)
            nbytes = L.marlaas_adapter_pool_storage_bytes_segmented(d_in, len(self.parts), widths, max_rank, capacity)
        if nbytes == 0:
            raise MarlaasError(MARLAAS_ERR_INVALID_ARG, "invalid pool dimensions")
        self.index = idx
        with torch.cuda.device(idx):
            self.storage = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            h = ctypes.c_void_p()
            if self.parts is None:
                _check(L.marlaas_adapter_pool_create(ctypes.byref(h), idx, d_in, d_out, max_rank, capacity,
                                                     _dptr(self.storage), nbytes, _stream(stream)))
            else:
                _check(L.marlaas_adapter_pool_create_segmented(ctypes.byref(h), idx, d_in, len(self.parts), widths, max_rank,
                                                               capacity, _dptr(self.storage), nbytes, _stream(stream)))
        self.handle = h
        self.rank_stride = int(L.marlaas_adapter_pool_rank_stride(h))
        self._workspaces = {}
        self._captured_workspaces = []
        self._policy_last = None
        self._step_bytes = {}               # workspace sizes of calls around the layer, by their sizes
        self._store = None

    def close(self):
        if getattr(self, "handle", None):
            load_library().marlaas_adapter_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, T: int) -> torch.Tensor:
        """A cached workspace tensor large enough for T tokens (one per pool; not for overlapping calls, and so not for graphs
        that run at the same time).  A buffer that a captured call was given stays as long as the pool, since its graph goes on
        using it when a larger batch has replaced it here."""
        need = marlaas_lora_workspace_bytes(self, T)
        ws = self._workspaces.get("ws")
        if ws is None or ws.numel() < need:
            ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            self._workspaces["ws"], self._workspace_stream = ws, torch._C._cuda_getCurrentRawStream(self.index)
        elif torch._C._cuda_getCurrentRawStream(self.index) != self._workspace_stream:
            ws.record_stream(torch.cuda.current_stream(self.index))
        if torch._C._cuda_isCurrentStreamCapturing() and not any(ws is w for w in self._captured_workspaces):
            self._captured_workspaces.append(ws)
        return ws

    def policy_workspace(self, T: int, num_segments: int, num_groups: int = 0, stream=None, handle=None) -> torch.Tensor:
        """A workspace tensor for marlaas_group_advantages and marlaas_policy_loss, cached per stream (`handle`: what
        _current() gives, if it is known).  A call that is being captured gets one of its own from the graph's memory, as
        torch's own operations get theirs; a capture that torch.cuda.graph does not make has to pass a workspace."""
        if stream is not None:
            return _on_stream(stream, self.policy_workspace, T, num_segments, num_groups)
        if torch._C._cuda_isCurrentStreamCapturing():
            return torch.empty(max(marlaas_policy_workspace_bytes(self, T, num_segments, num_groups), 256), dtype=torch.uint8, device=self.device)
        key = (T, num_segments, num_groups, _current() if handle is None else handle)
        last = self._policy_last
        if last is not None and last[0] == key:
            return last[1]
        need = max(marlaas_policy_workspace_bytes(self, T, num_segments, num_groups), 256)
        where = ("policy", key[3])
        ws = self._workspaces.get(where)
        if ws is None or ws.numel() < need:
            ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            self._workspaces[where] = ws
        self._policy_last = (key, ws)
        return ws

    def step_workspace(self, handle: int, workspace_bytes, *sizes) -> torch.Tensor:
        """Scratch for the calls around a training step's layers, at least workspace_bytes(self, *sizes), cached per stream (`handle`:
        the pool's device's current one).  A call that is being captured gets one of its own from the graph's memory."""
        need = self._step_bytes.get((workspace_bytes, sizes))
        if need is None:
            if len(self._step_bytes) >= 4096:
                self._step_bytes.clear()
            need = self._step_bytes[workspace_bytes, sizes] = max(workspace_bytes(self, *sizes), 256)
        if torch._C._cuda_isCurrentStreamCapturing():
            return torch.empty(need, dtype=torch.uint8, device=self.device)
        ws = self._workspaces.get(("step", handle))
        if ws is None or ws.numel() < need:
            ws = self._workspaces[("step", handle)] = torch.empty(need, dtype=torch.uint8, device=self.device)
        return ws

    def store(self):
        """Views of the pool's bf16 rows: At [n_parts][capacity * rank_stride][d_in] and Bs [capacity * rank_stride][d_out]
        (not to be written)."""
        if self._store is not None:
            return self._store
        at, bs = ctypes.c_void_p(), ctypes.c_void_p()
        _check(load_library().marlaas_adapter_pool_store(self.handle, ctypes.byref(at), ctypes.byref(bs)))
        rows, base, flat = self.capacity * self.rank_stride, self.storage.data_ptr(), self.storage
        def view(p, *shape):
            n = 2
            for d in shape:
                n *= d
            return flat[p.value - base:p.value - base + n].view(torch.bfloat16).view(*shape)
        self._store = view(at, self.n_parts, rows, self.d_in), view(bs, rows, self.d_out)
        return self._store


def marlaas_adapter_pool_register(pool: AdapterPool, tenant_id: int, version: int, rank: int, alpha: float,
                                  A: Optional[torch.Tensor], B: Optional[torch.Tensor], stream=None) -> int:
    if rank > 0 and pool.parts is not None:
        # one pair per projection, handed to the library as blocks one after another
        assert len(A) == pool.n_parts and len(B) == pool.n_parts
        for p in range(pool.n_parts):
            assert tuple(A[p].shape) == (pool.d_in, rank) and tuple(B[p].shape) == (rank, pool.parts[p])
        A = torch.cat([a.contiguous().reshape(-1) for a in A])
        B = torch.cat([b.contiguous().reshape(-1) for b in B])
        assert A.dtype == torch.bfloat16 and B.dtype == torch.bfloat16 and A.device == pool.device and B.device == pool.device
    elif rank > 0:
        assert A.dtype == torch.bfloat16 and B.dtype == torch.bfloat16 and A.is_contiguous() and B.is_contiguous()
        assert tuple(A.shape) == (pool.d_in, rank) and tuple(B.shape) == (rank, pool.d_out)
        assert A.device == pool.device and B.device == pool.device
    slot = ctypes.c_int32(-1)
    _check(load_library().marlaas_adapter_pool_register(pool.handle, tenant_id, version, rank, alpha, _dptr(A), _dptr(B),
                                                        ctypes.byref(slot), _stream(stream)))
    return int(slot.value)


def marlaas_adapter_pool_adamw_commit(pool: AdapterPool, tenant_ids: Sequence[int], dA, dB, A, B, m_A, v_A, m_B, v_B, *,
                                      lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                                      weight_decay: float = 0.0, grad_scale: float = 1.0, step: int = 1,
                                      new_versions: Optional[Sequence[int]] = None, stream=None) -> None:
    """AdamW on the fp32 masters of the listed tenants and commit of their bf16 rounding into the pool.  Each of the
    eight arguments dA .. v_B is a list (one entry per tenant) of contiguous fp32 device tensors, updated in place
    (A, m_A, v_A: [d_in][rank]; B, m_B, v_B: [rank][d_out])."""
    n = len(tenant_ids)
    tables = []
    for name, lst in (("dA", dA), ("dB", dB), ("A", A), ("B", B), ("m_A", m_A), ("v_A", v_A), ("m_B", m_B), ("v_B", v_B)):
        assert len(lst) == n, name
        tab = (ctypes.c_void_p * max(n, 1))()
        for i, t in enumerate(lst):
            assert t.dtype == torch.float32 and t.is_contiguous() and t.device == pool.device, name
            tab[i] = t.data_ptr()
        tables.append(tab)
    ids = (ctypes.c_uint64 * max(n, 1))(*tenant_ids)
    vers = None if new_versions is None else (ctypes.c_uint64 * max(n, 1))(*new_versions)
    hp = marlaas_adamw_t(lr, beta1, beta2, eps, weight_decay, grad_scale, step)
    _check(load_library().marlaas_adapter_pool_adamw_commit(pool.handle, n, ids, vers, *tables, ctypes.byref(hp),
                                                            _stream(stream)))


def marlaas_adapter_pool_unregister(pool: AdapterPool, tenant_id: int, stream=None) -> None:
    _check(load_library().marlaas_adapter_pool_unregister(pool.handle, tenant_id, _stream(stream)))


def marlaas_adapter_pool_lookup(pool: AdapterPool, tenant_id: int):
    s, r, sc, v = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_float(), ctypes.c_uint64()
    _check(load_library().marlaas_adapter_pool_lookup(pool.handle, tenant_id, ctypes.byref(s), ctypes.byref(r),
                                                      ctypes.byref(sc), ctypes.byref(v)))
    return int(s.value), int(r.value), float(sc.value), int(v.value)


def marlaas_adapter_pool_export(pool: AdapterPool, slot: int, rank: int, stream=None):
    """The slot's adapter in the caller's layout; for a pool over several projections, two lists (one A and one B per
    projection)."""
    if stream is not None:
        return _on_stream(stream, marlaas_adapter_pool_export, pool, slot, rank)
    A = torch.empty((pool.n_parts * pool.d_in, rank), dtype=torch.bfloat16, device=pool.device)
    B = torch.empty(rank * pool.d_out, dtype=torch.bfloat16, device=pool.device)
    _check(load_library().marlaas_adapter_pool_export(pool.handle, slot, _dptr(A), _dptr(B), _stream(stream)))
    if pool.parts is None:
        return A, B.view(rank, pool.d_out)
    As = [A[p * pool.d_in:(p + 1) * pool.d_in] for p in range(pool.n_parts)]
    Bs, o = [], 0
    for w in pool.parts:
        Bs.append(B[o:o + rank * w].view(rank, w))
        o += rank * w
    return As, Bs


def marlaas_lora_workspace_bytes(pool: AdapterPool, T: int) -> int:
    return int(load_library().marlaas_lora_workspace_bytes(pool.handle, T))


def marlaas_lora_forward_workspace_bytes(pool: AdapterPool, T: int) -> int:
    return int(load_library().marlaas_lora_forward_workspace_bytes(pool.handle, T))


def marlaas_lora_forward_workspace_min_bytes(pool: AdapterPool, T: int) -> int:
    return int(load_library().marlaas_lora_forward_workspace_min_bytes(pool.handle, T))


def _mat(t: torch.Tensor, cols: int, name: str):
    assert t.dtype == torch.bfloat16 and t.dim() == 2 and t.shape[1] == cols and t.stride(1) == 1, name
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), cols)


def marlaas_lora_forward(pool: AdapterPool, x: torch.Tensor, W: torch.Tensor, seg: Segments,
                         y: Optional[torch.Tensor] = None, h_save: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, flags: int = 0, stream=None) -> torch.Tensor:
    if stream is not None:
        return _on_stream(stream, marlaas_lora_forward, pool, x, W, seg, y, h_save, workspace, flags)
    T = x.shape[0]
    if y is None:
        y = torch.empty((T, pool.d_out), dtype=torch.bfloat16, device=x.device)
    ws = workspace if workspace is not None else pool.workspace(T)
    ldx, ldw, ldy = _mat(x, pool.d_in, "x"), _mat(W, pool.d_out, "W"), _mat(y, pool.d_out, "y")
    assert W.shape[0] == pool.d_in
    if h_save is not None:
        assert h_save.dtype == torch.float32 and h_save.is_contiguous() and h_save.numel() == pool.n_parts * T * pool.rank_stride
    _check(load_library().marlaas_lora_forward(pool.handle, T, _dptr(x), ldx, _dptr(W), ldw, _dptr(y), ldy,
                                               ctypes.byref(seg.c), _dptr(h_save), _dptr(ws), ws.numel(),
                                               flags | seg.flags, _stream(stream)))
    return y


def marlaas_lora_forward_multi(calls, flags: int = 0, stream=None):
    """Independent forward calls as one (see marlaas.h): `calls` is a list of dicts with the keyword arguments of
    marlaas_lora_forward (pool, x, W, seg, and y / h_save / workspace, which must be distinct per call; missing y and
    workspace are allocated).  Returns the list of outputs."""
    if stream is not None:
        return _on_stream(stream, marlaas_lora_forward_multi, calls, flags)
    n = len(calls)
    arr = (marlaas_forward_call_t * max(n, 1))()
    keep, ys = [], []
    fl = flags
    for i, c in enumerate(calls):
        pool, x, W, seg = c["pool"], c["x"], c["W"], c["seg"]
        T = x.shape[0]
        y = c.get("y")
        if y is None:
            y = torch.empty((T, pool.d_out), dtype=torch.bfloat16, device=x.device)
        ws = c.get("workspace")
        if ws is None:
            ws = torch.empty(max(marlaas_lora_forward_workspace_bytes(pool, T), 256), dtype=torch.uint8, device=x.device)
        hs = c.get("h_save")
        if hs is not None:
            assert hs.dtype == torch.float32 and hs.is_contiguous() and hs.numel() == pool.n_parts * T * pool.rank_stride
        assert W.shape[0] == pool.d_in
        arr[i] = marlaas_forward_call_t(pool.handle, T, _dptr(x), _mat(x, pool.d_in, "x"), _dptr(W), _mat(W, pool.d_out, "W"),
                                        _dptr(y), _mat(y, pool.d_out, "y"), ctypes.cast(ctypes.byref(seg.c), ctypes.c_void_p),
                                        _dptr(hs), _dptr(ws), ws.numel())
        fl |= seg.flags
        keep.append((ws, hs, seg))
        ys.append(y)
    _check(load_library().marlaas_lora_forward_multi(n, ctypes.cast(arr, ctypes.c_void_p), fl, _stream(stream)))
    return ys


def marlaas_lora_static_workspace_limit() -> int:
    return int(load_library().marlaas_lora_static_workspace_limit())


def marlaas_lora_forward_static_ws(pool: AdapterPool, x: torch.Tensor, W: torch.Tensor, seg: Segments,
                                   y: torch.Tensor, h_save: Optional[torch.Tensor] = None, flags: int = 0,
                                   stream=None) -> torch.Tensor:
    """Forward for callers that may not allocate on the device: the scratch is the library's built-in array, and
    this wrapper allocates nothing either (y is the caller's).  Raises for batches beyond the array's size."""
    T = x.shape[0]
    ldx, ldw, ldy = _mat(x, pool.d_in, "x"), _mat(W, pool.d_out, "W"), _mat(y, pool.d_out, "y")
    assert W.shape[0] == pool.d_in and y.shape[0] == T
    if h_save is not None:
        assert h_save.dtype == torch.float32 and h_save.is_contiguous() and h_save.numel() == pool.n_parts * T * pool.rank_stride
    _check(load_library().marlaas_lora_forward_static_ws(pool.handle, T, _dptr(x), ldx, _dptr(W), ldw, _dptr(y), ldy,
                                                         ctypes.byref(seg.c), _dptr(h_save), flags | seg.flags,
                                                         _stream(stream)))
    return y


def _ptr_table(ts: Optional[Sequence[Optional[torch.Tensor]]], cap: int):
    if ts is None:
        return None
    tab = (ctypes.c_void_p * cap)()
    for i in range(cap):
        t = ts[i] if i < len(ts) else None
        if t is not None:
            assert t.dtype == torch.float32 and t.is_contiguous()
            tab[i] = t.data_ptr()
    return tab


def marlaas_lora_backward(pool: AdapterPool, x: torch.Tensor, W: torch.Tensor, dy: torch.Tensor, seg: Segments,
                          dx: Optional[torch.Tensor] = None, dA: Optional[Sequence[Optional[torch.Tensor]]] = None,
                          dB: Optional[Sequence[Optional[torch.Tensor]]] = None,
                          h_saved: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                          flags: int = 0, stream=None) -> None:
    if stream is not None:
        return _on_stream(stream, marlaas_lora_backward, pool, x, W, dy, seg, dx, dA, dB, h_saved, workspace, flags)
    T = dy.shape[0]
    ws = workspace if workspace is not None else pool.workspace(T)
    ldx = _mat(x, pool.d_in, "x") if x is not None else 0
    ldw, lddy = _mat(W, pool.d_out, "W"), _mat(dy, pool.d_out, "dy")
    lddx = _mat(dx, pool.d_in, "dx") if dx is not None else 0
    ta, tb = _ptr_table(dA, pool.capacity), _ptr_table(dB, pool.capacity)
    _check(load_library().marlaas_lora_backward(pool.handle, T, _dptr(x), ldx, _dptr(W), ldw, _dptr(dy), lddy,
                                                _dptr(dx), lddx, ta, tb, ctypes.byref(seg.c), _dptr(h_saved),
                                                _dptr(ws), ws.numel(), flags | seg.flags, _stream(stream)))


def marlaas_lora_build_index(pool: AdapterPool, T: int, seg: Segments, workspace: Optional[torch.Tensor] = None,
                             flags: int = 0, stream=None):
    if stream is not None:
        return _on_stream(stream, marlaas_lora_build_index, pool, T, seg, workspace, flags)
    dev = pool.device
    tok_slot = torch.empty(max(T, 1), dtype=torch.int32, device=dev)
    slot_count = torch.empty(pool.capacity + 1, dtype=torch.int32, device=dev)
    slot_offset = torch.empty(pool.capacity + 2, dtype=torch.int32, device=dev)
    perm = torch.empty(max(T, 1), dtype=torch.int32, device=dev)
    ws = workspace if workspace is not None else pool.workspace(T)
    _check(load_library().marlaas_lora_build_index(pool.handle, T, ctypes.byref(seg.c), _dptr(tok_slot),
                                                   _dptr(slot_count), _dptr(slot_offset), _dptr(perm), _dptr(ws),
                                                   ws.numel(), flags | seg.flags, _stream(stream)))
    return tok_slot[:T], slot_count, slot_offset, perm[:T]


def marlaas_check_status(pool: AdapterPool, stream=None) -> None:
    _check(load_library().marlaas_check_status(pool.handle, _stream(stream)))


def marlaas_debug_wait_runs_out(pool: AdapterPool, limit_ns: int = 1_000_000, stream=None) -> None:
    """Diagnostic: one small CTA lets a bounded wait run out; the next marlaas_check_status raises DEVICE_TIMEOUT."""
    _check(load_library().marlaas_debug_wait_runs_out(pool.handle, int(limit_ns), _stream(stream)))


def marlaas_kernel_timing_begin(pool: AdapterPool) -> None:
    _check(load_library().marlaas_kernel_timing_begin(pool.handle))


def marlaas_kernel_timing_end(pool: AdapterPool):
    """(summed device milliseconds, launches) of the dominant kernel since marlaas_kernel_timing_begin."""
    ms, n = ctypes.c_float(), ctypes.c_int32()
    _check(load_library().marlaas_kernel_timing_end(pool.handle, ctypes.byref(ms), ctypes.byref(n)))
    return float(ms.value), int(n.value)


# ---- the policy update around the layer ----

def _f32(t: torch.Tensor, n: int, name: str, device: int) -> int:
    assert t.dtype is torch.float32 and t.get_device() == device and t.is_contiguous() and t.numel() == n, name
    return t.data_ptr()


def _i32(t: torch.Tensor, n: int, name: str, device: int) -> int:
    assert t.dtype is torch.int32 and t.get_device() == device and t.is_contiguous() and t.numel() == n, name
    return t.data_ptr()


_DTYPES = {torch.bfloat16: MARLAAS_DTYPE_BF16, torch.float32: MARLAAS_DTYPE_F32}


def _rows(t: torch.Tensor, V: int, name: str, device: int) -> int:
    """Leading dimension of a [T][V] matrix of logits or of their gradient."""
    assert t.dim() == 2 and t.shape[1] == V and (V == 1 or t.stride(1) == 1) and t.get_device() == device, name
    # (torch is free with the stride of a single row)
    return t.stride(0) if t.shape[0] > 1 else (V + 7) // 8 * 8


def marlaas_policy_workspace_bytes(pool: AdapterPool, T: int, num_segments: int, num_groups: int = 0) -> int:
    return int(load_library().marlaas_policy_workspace_bytes(pool.handle, T, num_segments, num_groups))


def marlaas_group_advantages(pool: AdapterPool, seg: Segments, rewards: torch.Tensor, group_offsets: torch.Tensor,
                             targets: torch.Tensor, *, eps: float = 1e-6, seq_adv: Optional[torch.Tensor] = None,
                             adv: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                             workspace: Optional[torch.Tensor] = None, flags: int = 0, stream=None):
    """(seq_adv [S], adv [T], weight [T]) of a batch whose sequences are the segments of `seg`; group_offsets lives where
    the segment table does.  Outputs that are not given are allocated."""
    if stream is not None:
        return _on_stream(stream, marlaas_group_advantages, pool, seg, rewards, group_offsets, targets, eps=eps, seq_adv=seq_adv, adv=adv,
                          weight=weight, workspace=workspace, flags=flags)
    T, S, G, dev = targets.numel(), seg.num_segments, group_offsets.numel() - 1, pool.index
    if seq_adv is None:
        seq_adv = rewards.new_empty(S)
    if adv is None:
        adv = rewards.new_empty(T)
    if weight is None:
        weight = rewards.new_empty(T)
    handle = _current()
    ws = workspace if workspace is not None else pool.policy_workspace(T, S, G, None, handle)
    _check(load_library().marlaas_group_advantages(
        pool.handle, T, seg.ref, _f32(rewards, S, "rewards", dev), G, _i32(group_offsets, G + 1, "group_offsets (where the segment table is)", -1 if seg.on_host else dev),
        _i32(targets, T, "targets", dev), eps, _f32(seq_adv, S, "seq_adv", dev), _f32(adv, T, "adv", dev), _f32(weight, T, "weight", dev),
        ws.data_ptr(), ws.numel(), flags | seg.flags, handle))
    return seq_adv, adv, weight


def marlaas_token_logprobs(pool: AdapterPool, logits: torch.Tensor, targets: torch.Tensor, *, inv_temperature: float = 1.0,
                           logp: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                           with_entropy: bool = False, flags: int = 0, stream=None):
    """logp [T] of the targets (negative = ignored), and with `with_entropy` or `entropy` (logp, entropy)."""
    if stream is not None:
        return _on_stream(stream, marlaas_token_logprobs, pool, logits, targets, inv_temperature=inv_temperature, logp=logp, entropy=entropy,
                          with_entropy=with_entropy, flags=flags)
    (T, V), dev = logits.shape, pool.index
    if logp is None:
        logp = torch.empty(T, dtype=torch.float32, device=logits.device)
    if entropy is None and with_entropy:
        entropy = torch.empty(T, dtype=torch.float32, device=logits.device)
    assert logits.dtype in _DTYPES, "logits"
    _check(load_library().marlaas_token_logprobs(
        pool.handle, T, V, logits.data_ptr(), _rows(logits, V, "logits", dev), _DTYPES[logits.dtype], _i32(targets, T, "targets", dev),
        inv_temperature, _f32(logp, T, "logp", dev), None if entropy is None else _f32(entropy, T, "entropy", dev), flags, _current()))
    return logp if entropy is None else (logp, entropy)


def marlaas_policy_loss(pool: AdapterPool, logits: torch.Tensor, targets: torch.Tensor, seg: Segments, old_logp: torch.Tensor,
                        adv: torch.Tensor, weight: torch.Tensor, *, ref_logp: Optional[torch.Tensor] = None,
                        dlogits: Optional[torch.Tensor] = None, logp: Optional[torch.Tensor] = None,
                        stats: Optional[torch.Tensor] = None, clip_low: float = 0.2, clip_high: float = 0.2,
                        kl_coef: float = 0.0, entropy_coef: float = 0.0, inv_temperature: float = 1.0, grad_scale: float = 1.0,
                        workspace: Optional[torch.Tensor] = None, flags: int = 0, stream=None) -> torch.Tensor:
    """Clipped policy loss with KL and entropy terms: returns stats [capacity + 1][8] (see marlaas.h; column 0 is the loss
    per slot) and writes its gradient by the logits to `dlogits` (which may be `logits` itself) if given."""
    if stream is not None:
        return _on_stream(stream, marlaas_policy_loss, pool, logits, targets, seg, old_logp, adv, weight, ref_logp=ref_logp, dlogits=dlogits,
                          logp=logp, stats=stats, clip_low=clip_low, clip_high=clip_high, kl_coef=kl_coef, entropy_coef=entropy_coef,
                          inv_temperature=inv_temperature, grad_scale=grad_scale, workspace=workspace, flags=flags)
    (T, V), dev = logits.shape, pool.index
    if stats is None:
        assert not (flags & MARLAAS_FLAG_ACCUMULATE), "stats to add to"
        stats = adv.new_empty((pool.capacity + 1, MARLAAS_POLICY_STATS))
    assert logits.dtype in _DTYPES, "logits"
    lddl = 0
    if dlogits is not None:
        assert dlogits.dtype == logits.dtype and dlogits.shape[0] == T, "dlogits"
        lddl = _rows(dlogits, V, "dlogits", dev)
    handle = _current()
    ws = workspace if workspace is not None else pool.policy_workspace(T, seg.num_segments, 0, None, handle)
    hp = marlaas_policy_loss_t(clip_low, clip_high, kl_coef, entropy_coef, inv_temperature, grad_scale)
    _check(load_library().marlaas_policy_loss(
        pool.handle, T, V, logits.data_ptr(), _rows(logits, V, "logits", dev), _DTYPES[logits.dtype], _i32(targets, T, "targets", dev),
        seg.ref, _f32(old_logp, T, "old_logp", dev), None if ref_logp is None else _f32(ref_logp, T, "ref_logp", dev),
        _f32(adv, T, "adv", dev), _f32(weight, T, "weight", dev), ctypes.byref(hp), None if dlogits is None else dlogits.data_ptr(), lddl,
        None if logp is None else _f32(logp, T, "logp", dev), _f32(stats, (pool.capacity + 1) * MARLAAS_POLICY_STATS, "stats", dev),
        ws.data_ptr(), ws.numel(), flags | seg.flags, handle))
    return stats


def marlaas_adamw_compact_state_bytes(n: int) -> int:
    return int(load_library().marlaas_adamw_compact_state_bytes(n))


def compact_state(pool: AdapterPool, rank: int):
    """Zeroed 8-bit moments (state_A, state_B) of one tenant's adapter of the given rank."""
    widths = pool.parts if pool.parts is not None else [pool.d_out]
    a = pool.n_parts * marlaas_adamw_compact_state_bytes(pool.d_in * rank)
    b = sum(marlaas_adamw_compact_state_bytes(rank * w) for w in widths)
    return tuple(torch.zeros(n, dtype=torch.uint8, device=pool.device) for n in (a, b))


class CompactAdamWTables:
    """The tensors of marlaas_adapter_pool_adamw_compact_commit, one entry per listed tenant: gradients and masters
    (contiguous fp32) and 8-bit states (contiguous uint8, see compact_state).  Made once for buffers that stay in place from
    step to step; keeps them alive."""

    def __init__(self, pool: AdapterPool, tenant_ids: Sequence[int], dA, dB, A, B, state_A, state_B):
        n = self.n = len(tenant_ids)
        self.tensors = (list(dA), list(dB), list(A), list(B), list(state_A), list(state_B))
        widths = pool.parts if pool.parts is not None else [pool.d_out]
        ranks = [marlaas_adapter_pool_lookup(pool, t)[1] for t in tenant_ids]
        self.tables = []
        for k, (name, lst) in enumerate(zip(("dA", "dB", "A", "B", "state_A", "state_B"), self.tensors)):
            assert len(lst) == n, name
            tab = (ctypes.c_void_p * max(n, 1))()
            for i, t in enumerate(lst):
                r = ranks[i]
                if k < 4:
                    need = pool.n_parts * pool.d_in * r if k % 2 == 0 else r * pool.d_out
                    ok = t.dtype == torch.float32 and t.numel() == need
                else:
                    need = (pool.n_parts * marlaas_adamw_compact_state_bytes(pool.d_in * r) if k == 4 else
                            sum(marlaas_adamw_compact_state_bytes(r * w) for w in widths))
                    ok = t.dtype == torch.uint8 and t.numel() == need
                assert ok and t.is_contiguous() and t.device == pool.device, f"{name}[{i}]"
                tab[i] = t.data_ptr()
            self.tables.append(tab)
        self.ids = (ctypes.c_uint64 * max(n, 1))(*tenant_ids)
        self.ranks = (ctypes.c_int32 * max(n, 1))(*ranks)


def marlaas_adapter_pool_adamw_compact_commit(pool: AdapterPool, tables: CompactAdamWTables, *, lr: float, beta1: float = 0.9,
                                              beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
                                              grad_scale: float = 1.0, step: int = 1, seed: int = 0,
                                              new_versions: Optional[Sequence[int]] = None, stream=None) -> None:
    """AdamW with 8-bit moments on the masters of the listed tenants, and commit of their bf16 rounding into the pool.
    A tenant whose rank has changed since the tables were made is refused.  A captured commit repeats its step number, rates and
    random bits at every replay, and raises the version once, when it is captured."""
    vers = None if new_versions is None else (ctypes.c_uint64 * max(tables.n, 1))(*new_versions)
    hp = marlaas_adamw_t(lr, beta1, beta2, eps, weight_decay, grad_scale, step)
    _check(load_library().marlaas_adapter_pool_adamw_compact_commit(pool.handle, tables.n, tables.ids, vers, *tables.tables,
                                                                    tables.ranks, ctypes.byref(hp), seed, _stream(stream)))


def marlaas_adamw_compact_state_export(pool: AdapterPool, state: torch.Tensor, m: Optional[torch.Tensor] = None,
                                       v: Optional[torch.Tensor] = None, stream=None):
    """fp32 (m, v) that the blocks of `state` stand for (256 elements per block, those past a matrix's end are 0)."""
    if stream is not None:
        return _on_stream(stream, marlaas_adamw_compact_state_export, pool, state, m, v)
    assert state.dtype == torch.uint8 and state.is_contiguous() and state.numel() % 528 == 0 and state.device == pool.device
    blocks, dev = state.numel() // 528, pool.index
    if m is None:
        m = torch.empty(256 * blocks, dtype=torch.float32, device=pool.device)
    if v is None:
        v = torch.empty(256 * blocks, dtype=torch.float32, device=pool.device)
    _check(load_library().marlaas_adamw_compact_state_export(pool.handle, blocks, state.data_ptr(), _f32(m, 256 * blocks, "m", dev),
                                                             _f32(v, 256 * blocks, "v", dev), _current()))
    return m, v


# ---- around the adapted projections of a training step ----

def _bf16_rows(t: torch.Tensor, T: int, cols: int, name: str, device: int) -> int:
    """Leading dimension of a bf16 [T][cols] matrix."""
    strides = t.stride()
    assert t.dtype is torch.bfloat16 and t.shape == (T, cols) and t.get_device() == device and (cols == 1 or strides[1] == 1), name
    return strides[0] if T > 1 else -(-cols // 8) * 8


def marlaas_lora_dropout_workspace_bytes(pool: AdapterPool, T: int) -> int:
    return int(load_library().marlaas_lora_dropout_workspace_bytes(pool.handle, T))


def _drop(pool: AdapterPool, rates: torch.Tensor, seed: int, offset: int) -> marlaas_dropout_t:
    assert 0 <= seed < 1 << 64 and 0 <= offset < 1 << 64, "seed and offset are 64-bit numbers"
    return marlaas_dropout_t(_f32(rates, pool.capacity, "rates", pool.index), seed, offset)


def marlaas_lora_forward_dropout(pool: AdapterPool, x: torch.Tensor, W: torch.Tensor, seg: Segments, rates: torch.Tensor, seed: int,
                                 offset: int = 0, y: Optional[torch.Tensor] = None, h_save: Optional[torch.Tensor] = None,
                                 workspace: Optional[torch.Tensor] = None, flags: int = 0, stream=None) -> torch.Tensor:
    """marlaas_lora_forward with dropout in the adapters: `rates` fp32 [capacity] per slot, masks from (seed, offset)."""
    if stream is not None:
        return _on_stream(stream, marlaas_lora_forward_dropout, pool, x, W, seg, rates, seed, offset, y, h_save, workspace, flags)
    T, dev = x.shape[0], pool.index
    y = torch.empty((T, pool.d_out), dtype=torch.bfloat16, device=x.device) if y is None else y
    handle = torch._C._cuda_getCurrentRawStream(dev)
    ws = pool.step_workspace(handle, marlaas_lora_dropout_workspace_bytes, T) if workspace is None else workspace
    drop = _drop(pool, rates, seed, offset)
    _check(load_library().marlaas_lora_forward_dropout(
        pool.handle, T, x.data_ptr(), _bf16_rows(x, T, pool.d_in, "x", dev), W.data_ptr(), _bf16_rows(W, pool.d_in, pool.d_out, "W", dev),
        y.data_ptr(), _bf16_rows(y, T, pool.d_out, "y", dev), seg.ref, ctypes.byref(drop),
        None if h_save is None else _f32(h_save, pool.n_parts * T * pool.rank_stride, "h_save", dev), ws.data_ptr(), ws.numel(),
        flags | seg.flags, handle))
    return y


def marlaas_lora_backward_dropout(pool: AdapterPool, x: Optional[torch.Tensor], W: torch.Tensor, dy: torch.Tensor, seg: Segments,
                                  rates: torch.Tensor, seed: int, offset: int = 0, dx: Optional[torch.Tensor] = None,
                                  dA: Optional[Sequence[Optional[torch.Tensor]]] = None, dB: Optional[Sequence[Optional[torch.Tensor]]] = None,
                                  h_saved: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, flags: int = 0,
                                  stream=None) -> None:
    """marlaas_lora_backward with the masks of the forward call (the same rates, seed and offset)."""
    if stream is not None:
        return _on_stream(stream, marlaas_lora_backward_dropout, pool, x, W, dy, seg, rates, seed, offset, dx, dA, dB, h_saved, workspace, flags)
    T, dev = dy.shape[0], pool.index
    handle = torch._C._cuda_getCurrentRawStream(dev)
    ws = pool.step_workspace(handle, marlaas_lora_dropout_workspace_bytes, T) if workspace is None else workspace
    drop = _drop(pool, rates, seed, offset)
    _check(load_library().marlaas_lora_backward_dropout(
        pool.handle, T, None if x is None else x.data_ptr(), 0 if x is None else _bf16_rows(x, T, pool.d_in, "x", dev), W.data_ptr(),
        _bf16_rows(W, pool.d_in, pool.d_out, "W", dev), dy.data_ptr(), _bf16_rows(dy, T, pool.d_out, "dy", dev),
        None if dx is None else dx.data_ptr(), 0 if dx is None else _bf16_rows(dx, T, pool.d_in, "dx", dev),
        _ptr_table(dA, pool.capacity), _ptr_table(dB, pool.capacity), seg.ref, ctypes.byref(drop),
        None if h_saved is None else _f32(h_saved, pool.n_parts * T * pool.rank_stride, "h_saved", dev), ws.data_ptr(), ws.numel(),
        flags | seg.flags, handle))


def marlaas_layer_norm_workspace_bytes(pool: AdapterPool, T: int, d: int, num_segments: int, backward: bool) -> int:
    return int(load_library().marlaas_layer_norm_workspace_bytes(pool.handle, T, d, num_segments, int(backward)))


def marlaas_layer_norm(pool: AdapterPool, x: torch.Tensor, seg: Segments, gain: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                       eps: float = 1e-5, y: Optional[torch.Tensor] = None, mean: Optional[torch.Tensor] = None,
                       rstd: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, flags: int = 0, stream=None):
    """(y, mean [T], rstd [T]) of the rows of x with the gain and bias [capacity + 1][d] of their tenants (the last row: slot
    -1).  Outputs that are not given are allocated."""
    if stream is not None:
        return _on_stream(stream, marlaas_layer_norm, pool, x, seg, gain, bias, eps=eps, y=y, mean=mean, rstd=rstd, workspace=workspace,
                          flags=flags)
    (T, d), dev = x.shape, pool.index
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if y is None else y
    mean = torch.empty(T, dtype=torch.float32, device=x.device) if mean is None else mean
    rstd = torch.empty(T, dtype=torch.float32, device=x.device) if rstd is None else rstd
    handle = torch._C._cuda_getCurrentRawStream(dev)
    ws = workspace
    if ws is None and seg.on_host:
        ws = pool.step_workspace(handle, marlaas_layer_norm_workspace_bytes, T, d, seg.num_segments, False)
    params = (pool.capacity + 1) * d
    _check(load_library().marlaas_layer_norm(
        pool.handle, T, d, x.data_ptr(), _bf16_rows(x, T, d, "x", dev), seg.ref, _f32(gain, params, "gain", dev),
        None if bias is None else _f32(bias, params, "bias", dev), eps, y.data_ptr(), _bf16_rows(y, T, d, "y", dev), _f32(mean, T, "mean", dev),
        _f32(rstd, T, "rstd", dev), None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), flags | seg.flags, handle))
    return y, mean, rstd


def marlaas_layer_norm_backward(pool: AdapterPool, x: torch.Tensor, dy: torch.Tensor, seg: Segments, gain: torch.Tensor,
                                mean: Optional[torch.Tensor], rstd: torch.Tensor, *, dx: Optional[torch.Tensor] = None,
                                dgain: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                                workspace: Optional[torch.Tensor] = None, flags: int = 0, stream=None) -> None:
    """Writes those of dx, dgain, dbias ([capacity + 1][d]) that are given."""
    if stream is not None:
        return _on_stream(stream, marlaas_layer_norm_backward, pool, x, dy, seg, gain, mean, rstd, dx=dx, dgain=dgain, dbias=dbias,
                          workspace=workspace, flags=flags)
    (T, d), dev = x.shape, pool.index
    params = (pool.capacity + 1) * d
    handle = torch._C._cuda_getCurrentRawStream(dev)
    ws = workspace
    if ws is None:
        ws = pool.step_workspace(handle, marlaas_layer_norm_workspace_bytes, T, d, seg.num_segments, True)
    _check(load_library().marlaas_layer_norm_backward(
        pool.handle, T, d, x.data_ptr(), _bf16_rows(x, T, d, "x", dev), dy.data_ptr(), _bf16_rows(dy, T, d, "dy", dev), seg.ref,
        _f32(gain, params, "gain", dev), None if mean is None else _f32(mean, T, "mean", dev), _f32(rstd, T, "rstd", dev),
        None if dx is None else dx.data_ptr(), 0 if dx is None else _bf16_rows(dx, T, d, "dx", dev),
        None if dgain is None else _f32(dgain, params, "dgain", dev), None if dbias is None else _f32(dbias, params, "dbias", dev),
        ws.data_ptr(), ws.numel(), flags | seg.flags, handle))


def marlaas_head_cross_entropy_workspace_bytes(pool: AdapterPool, T: int, d: int, V: int, num_segments: int, with_gradient: bool) -> int:
    return int(load_library().marlaas_head_cross_entropy_workspace_bytes(pool.handle, T, d, V, num_segments, int(with_gradient)))


def marlaas_head_cross_entropy(pool: AdapterPool, x: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, seg: Optional[Segments] = None, *,
                               weight: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, logp: Optional[torch.Tensor] = None,
                               stats: Optional[torch.Tensor] = None, inv_temperature: float = 1.0, grad_scale: float = 1.0,
                               workspace: Optional[torch.Tensor] = None, flags: int = 0, stream=None):
    """(logp [T], stats [capacity + 1][4]) of the targets under softmax(inv_temperature x W), and the weighted loss's gradient by x
    in `dx` (which may be `x` itself) if given.  Without `seg` there are no stats: (logp, None)."""
    if stream is not None:
        return _on_stream(stream, marlaas_head_cross_entropy, pool, x, W, targets, seg, weight=weight, dx=dx, logp=logp, stats=stats,
                          inv_temperature=inv_temperature, grad_scale=grad_scale, workspace=workspace, flags=flags)
    (T, d), V, dev = x.shape, W.shape[1], pool.index
    if logp is None:
        logp = torch.empty(T, dtype=torch.float32, device=x.device)
    if seg is None:
        assert stats is None, "stats need the segment table"
    elif stats is None:
        assert not (flags & MARLAAS_FLAG_ACCUMULATE), "stats to add to"
        stats = torch.empty((pool.capacity + 1, MARLAAS_HEAD_STATS), dtype=torch.float32, device=x.device)
    S = 0 if seg is None else seg.num_segments
    handle = torch._C._cuda_getCurrentRawStream(dev)
    ws = workspace
    if ws is None:
        ws = pool.step_workspace(handle, marlaas_head_cross_entropy_workspace_bytes, T, d, V, S, dx is not None)
    _check(load_library().marlaas_head_cross_entropy(
        pool.handle, T, d, V, x.data_ptr(), _bf16_rows(x, T, d, "x", dev), W.data_ptr(), _bf16_rows(W, d, V, "W", dev),
        _i32(targets, T, "targets", dev), None if seg is None else seg.ref, None if weight is None else _f32(weight, T, "weight", dev),
        inv_temperature, grad_scale, None if dx is None else dx.data_ptr(), 0 if dx is None else _bf16_rows(dx, T, d, "dx", dev),
        _f32(logp, T, "logp", dev), None if stats is None else _f32(stats, (pool.capacity + 1) * MARLAAS_HEAD_STATS, "stats", dev),
        ws.data_ptr(), ws.numel(), flags | (0 if seg is None else seg.flags), handle))
    return logp, stats
