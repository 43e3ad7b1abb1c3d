"""ctypes binding of libdecode_attn.so: argument marshalling only.

Every function has the name of the C entry point it calls.  torch supplies
device memory (tensors), their data pointers and the current HIP stream;
every step of the computation runs in the library's HIP kernels.  torch is
imported before the library is loaded so that both resolve the same HIP
runtime (libamdhip64.so.7).  A missing library raises; there is no fallback.
"""

from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence, Tuple

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdecode_attn.so")
HEAD_DIM = 128
MAX_SPLITS = 64
KV4_TILE_BYTES = 4352  # 32 keys of one KV head in the 4-bit cache
MAX_REQUESTS = 4096    # of one da_extend_tables call
MAX_AXES = 4           # of da_append_kv_axes
MAX_NEW_TOKENS = 1 << 28  # rows of one
ARRIVAL_BYTES = 1 << 20  # counters at the end of a workspace
INT_MAX = 2 ** 31 - 1
DEALT_MIN_KEYS = 2561  # da_prefers_dealt never holds for shorter batches: no need to ask

DA_OK = 0
DA_ERR_NULL = -1
DA_ERR_SHAPE = -2
DA_ERR_UNSUPPORTED = -3
DA_ERR_SPLITS = -4
DA_ERR_ALIGN = -5
DA_ERR_WORKSPACE = -6
DA_ERR_HIP = -7
DA_ERR_ARG = -8

POLICY_MI355X = 0
POLICY_PAPER = 1
POLICY_EVOLVED = 2
POLICY_STREAMED = 3
POLICY_TABLE = 4
POLICY_TABLE_STREAMED = 5

# Every symbol include/decode_attn.h declares.
EXPORTS = (
    "da_choose_splits", "da_model_time", "da_make_plan", "da_workspace_bytes", "da_split_bounds", "da_decode_attn",
    "da_decode_attn_planned", "da_decode_attn_noalloc", "da_decode_attn_paged", "da_decode_attn_paged_planned", "da_schedule_max_bytes",
    "da_make_schedule", "da_schedule_workspace_bytes",
    "da_decode_attn_scheduled", "da_decode_attn_dealt", "da_dealt_workspace_bytes", "da_prefers_dealt",
    "da_decode_attn_window", "da_window_keys", "da_extend_tables", "da_append_kv", "da_append_kv4", "da_read_kv4",
    "da_append_kv_axes", "da_append_kv4_axes", "da_add_key_weights", "da_evict_kv", "da_evict_workspace_bytes",
    "da_decode_attn_prefix", "da_prefix_workspace_bytes", "da_decode_attn_kv4", "da_kv4_workspace_bytes",
    "da_split_partials", "da_combine_splits", "da_device_info", "da_strerror",
    "da_last_error",
)


class DaPlan(ctypes.Structure):
    _fields_ = [
        ("num_splits", ctypes.c_int32),
        ("pack_gqa", ctypes.c_int32),
        ("heads_per_tile", ctypes.c_int32),
        ("tiles", ctypes.c_int32),
        ("grid", ctypes.c_int32),
        ("num_cus", ctypes.c_int32),
        ("group_waves", ctypes.c_int32),
        ("kv_fetch", ctypes.c_int32),
        ("kv_nontemporal", ctypes.c_int32),
        ("v_slices", ctypes.c_int32),
        ("combine", ctypes.c_int32),
        ("wg_per_cu", ctypes.c_int32),
    ]

    def as_dict(self) -> dict:
        return {name: int(getattr(self, name)) for name, _ in self._fields_}


class DaSchedule(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in (
        "B", "H_Q", "H_KV", "L_K_max", "pack_gqa", "heads_per_tile", "tiles", "num_items", "chunk_tiles",
        "max_splits", "state_rows", "num_cus", "kv_fetch", "seq_offset", "meta_bytes", "kv_nontemporal",
        "combine")]

    def as_dict(self) -> dict:
        return {name: int(getattr(self, name)) for name, _ in self._fields_}


class DecodeAttnError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{message} (code {code})")
        self.code = code


_lib: Optional[ctypes.CDLL] = None

_I = ctypes.c_int
_P = ctypes.c_void_p
_F = ctypes.c_float
_Z = ctypes.c_size_t
_L = ctypes.c_int64


def _hip_runtimes_loaded() -> List[str]:
    paths = set()
    try:
        with open("/proc/self/maps") as f:
            for line in f:
                if "libamdhip64.so" in line:
                    paths.add(line.split()[-1])
    except OSError:
        pass
    return sorted(paths)


def load() -> ctypes.CDLL:
    """Load the built library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_00028_amd.build` "
                           "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    runtimes = _hip_runtimes_loaded()
    if len(runtimes) > 1:
        raise RuntimeError(f"two HIP runtimes are loaded ({runtimes}); torch must be imported first")
    lib.da_choose_splits.argtypes = [_I, _I, _I, _I, _I, _I, _I, _I, ctypes.POINTER(DaPlan)]
    lib.da_choose_splits.restype = _I
    lib.da_model_time.argtypes = [_I] * 10
    lib.da_model_time.restype = ctypes.c_double
    lib.da_make_plan.argtypes = [_I, _I, _I, _I, _I, _I, _I, _I, _I, _I, ctypes.POINTER(DaPlan)]
    lib.da_make_plan.restype = _I
    lib.da_workspace_bytes.argtypes = [_I, _I, _I, _I]
    lib.da_workspace_bytes.restype = _Z
    lib.da_split_bounds.argtypes = [_I, _I, ctypes.POINTER(ctypes.c_int32)]
    lib.da_split_bounds.restype = _I
    lib.da_decode_attn.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _I, _I, _P, _Z, _P]
    lib.da_decode_attn.restype = _I
    lib.da_decode_attn_planned.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, ctypes.POINTER(DaPlan),
                                           _P, _Z, _P]
    lib.da_decode_attn_planned.restype = _I
    lib.da_decode_attn_noalloc.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _I, _I, _P]
    lib.da_decode_attn_noalloc.restype = _I
    lib.da_decode_attn_paged.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _F, _I, _I,
                                         _P, _Z, _P]
    lib.da_decode_attn_paged.restype = _I
    lib.da_decode_attn_paged_planned.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _F,
                                                 ctypes.POINTER(DaPlan), _P, _Z, _P]
    lib.da_decode_attn_paged_planned.restype = _I
    lib.da_schedule_max_bytes.argtypes = [_I, _I, _I, _I]
    lib.da_schedule_max_bytes.restype = _Z
    lib.da_make_schedule.argtypes = [_P, _I, _I, _I, _I, _I, _I, _I, _I, _I, _P, _Z, ctypes.POINTER(DaSchedule)]
    lib.da_make_schedule.restype = _I
    lib.da_schedule_workspace_bytes.argtypes = [ctypes.POINTER(DaSchedule)]
    lib.da_schedule_workspace_bytes.restype = _Z
    lib.da_decode_attn_scheduled.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _P, _P, _I, _F,
                                             ctypes.POINTER(DaSchedule), _P, _P, _Z, _P]
    lib.da_decode_attn_scheduled.restype = _I
    lib.da_dealt_workspace_bytes.argtypes = [_I, _I, _I, _I]
    lib.da_dealt_workspace_bytes.restype = _Z
    lib.da_prefers_dealt.argtypes = [_I, _I, _I, _I, ctypes.c_int64, _I]
    lib.da_prefers_dealt.restype = _I
    lib.da_decode_attn_dealt.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _P, _P, _I, _I, _I, _I, _I, _F,
                                         ctypes.c_int64, _P, _Z, _P]
    lib.da_decode_attn_dealt.restype = _I
    lib.da_decode_attn_window.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _P, _P, _I, _I, _I, _I, _I, _F, _I, _I,
                                          _I, _I, _P, _Z, _P]
    lib.da_decode_attn_window.restype = _I
    lib.da_window_keys.argtypes = [_I, _I, _I]
    lib.da_window_keys.restype = _I
    lib.da_extend_tables.argtypes = [_P] * 10 + [_I] * 6 + [_P]
    lib.da_extend_tables.restype = _I
    lib.da_append_kv.argtypes = [_P, _L, _P, _L, _P, _L, _P, _P, _F, _P, _I, _I, _I, _P, _P, _P, _P, _P, _L, _I, _I,
                                 _I, _I, _P]
    lib.da_append_kv.restype = _I
    lib.da_append_kv4.argtypes = [_P, _L, _P, _L, _P, _L, _P, _P, _F, _P, _I, _I, _I, _P, _P, _P, _P, _I, _I, _I, _I,
                                  _I, _I, _P]
    lib.da_append_kv4.restype = _I
    lib.da_append_kv_axes.argtypes = [_P, _L, _P, _L, _P, _L, _P, _P, _F, _P, _I, _I, _I, ctypes.c_char_p, _I, _P, _P, _P,
                                      _P, _P, _L, _I, _I, _I, _I, _P]
    lib.da_append_kv_axes.restype = _I
    lib.da_append_kv4_axes.argtypes = [_P, _L, _P, _L, _P, _L, _P, _P, _F, _P, _I, _I, _I, ctypes.c_char_p, _I, _P, _P,
                                       _P, _P, _I, _I, _I, _I, _I, _I, _P]
    lib.da_append_kv4_axes.restype = _I
    lib.da_read_kv4.argtypes = [_P, _P, _P, _P, _I, _I, _I, _I, _I, _P]
    lib.da_read_kv4.restype = _I
    lib.da_decode_attn_kv4.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _F, _I, _I, _I, _P, _Z,
                                       _P]
    lib.da_decode_attn_kv4.restype = _I
    lib.da_kv4_workspace_bytes.argtypes = [_I] * 4 + [_L] + [_I] * 4
    lib.da_kv4_workspace_bytes.restype = _Z
    lib.da_decode_attn_prefix.argtypes = [_P] * 9 + [_I] * 9 + [_F, _I, _P, _Z, _P]
    lib.da_decode_attn_prefix.restype = _I
    lib.da_prefix_workspace_bytes.argtypes = [_I] * 5
    lib.da_prefix_workspace_bytes.restype = _Z
    lib.da_add_key_weights.argtypes = [_P] * 7 + [_L] + [_I] * 8 + [_F, _F, _P]
    lib.da_add_key_weights.restype = _I
    lib.da_evict_kv.argtypes = [_P] * 9 + [_L] + [_P] * 4 + [_I] * 11 + [_P, _Z, _P]
    lib.da_evict_kv.restype = _I
    lib.da_evict_workspace_bytes.argtypes = [_I] * 4
    lib.da_evict_workspace_bytes.restype = _Z
    lib.da_split_partials.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _I, _I, _P]
    lib.da_split_partials.restype = _I
    lib.da_combine_splits.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, _I, _P]
    lib.da_combine_splits.restype = _I
    lib.da_device_info.argtypes = [ctypes.POINTER(_I), ctypes.POINTER(_I)]
    lib.da_device_info.restype = _I
    lib.da_strerror.argtypes = [_I]
    lib.da_strerror.restype = ctypes.c_char_p
    lib.da_last_error.argtypes = []
    lib.da_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != DA_OK:
        lib = load()
        msg = (lib.da_last_error() or b"").decode() or lib.da_strerror(rc).decode()
        raise DecodeAttnError(rc, msg)


def da_strerror(code: int) -> str:
    return load().da_strerror(code).decode()


def da_last_error() -> str:
    return (load().da_last_error() or b"").decode()


def da_device_info() -> Tuple[int, bool]:
    cus, is950 = _I(0), _I(0)
    _check(load().da_device_info(ctypes.byref(cus), ctypes.byref(is950)))
    return cus.value, bool(is950.value)


def da_choose_splits(B: int, H_Q: int, H_KV: int, L_K_max: int, d: int = HEAD_DIM, num_cus: int = 0,
                     cu_margin: int = 0, policy: int = POLICY_MI355X) -> DaPlan:
    plan = DaPlan()
    _check(load().da_choose_splits(*map(_int, (B, H_Q, H_KV, L_K_max, d, num_cus, cu_margin, policy)),
                                   ctypes.byref(plan)))
    return plan


def da_model_time(policy: int, B: int, H_Q: int, H_KV: int, L_K: int, heads_per_tile: int, num_splits: int,
                  v_slices: int = 1, combine: int = 0, num_cus: int = 256) -> float:
    """The planner's modelled microseconds per call (-1 for no launch)."""
    return float(load().da_model_time(*map(_int, (policy, B, H_Q, H_KV, L_K, heads_per_tile, num_splits, v_slices,
                                                  combine, num_cus))))


def da_make_plan(B: int, H_Q: int, H_KV: int, L_K_max: int, d: int = HEAD_DIM, num_splits: int = 0,
                 pack_gqa: int = -1, num_cus: int = 0, cu_margin: int = 0, policy: int = POLICY_MI355X) -> DaPlan:
    plan = DaPlan()
    _check(load().da_make_plan(*map(_int, (B, H_Q, H_KV, L_K_max, d, num_splits, pack_gqa, num_cus, cu_margin, policy)),
                               ctypes.byref(plan)))
    return plan


def da_workspace_bytes(B: int, H_Q: int, d: int, num_splits: int) -> int:
    return int(load().da_workspace_bytes(_int(B), _int(H_Q), _int(d), _int(num_splits)))


def da_dealt_workspace_bytes(B: int, H_Q: int, H_KV: int, num_cus: int = 0) -> int:
    return int(load().da_dealt_workspace_bytes(_int(B), _int(H_Q), _int(H_KV), _int(num_cus)))


def da_prefers_dealt(B: int, H_Q: int, H_KV: int, L_K_max: int, keys: int = 0, num_cus: int = 0) -> bool:
    return bool(load().da_prefers_dealt(_int(B), _int(H_Q), _int(H_KV), _int(L_K_max), keys, _int(num_cus)))


def da_split_bounds(L: int, num_splits: int) -> List[int]:
    cuts = (ctypes.c_int32 * (min(num_splits, MAX_SPLITS) + 1))() if num_splits >= 0 else None
    _check(load().da_split_bounds(_int(L), _int(num_splits), cuts))
    return list(cuts)


def _int(x: int) -> int:
    """x as a C int: ctypes would wrap a number past it around to some other one,
    where the largest is refused, or bounds as much."""
    return x if -INT_MAX <= x <= INT_MAX else INT_MAX if x > 0 else -INT_MAX


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    # an empty tensor has no storage: NULL (the library reads nothing there)
    return None if t is None or t.numel() == 0 else t.data_ptr()


# The handle of a device's current stream without a Stream object around it (0.1 us instead of 1.9).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(dev: torch.device, stream) -> int:
    if stream is None:
        if _raw_stream is not None and dev.index is not None:
            return _raw_stream(dev.index)
        return torch.cuda.current_stream(dev).cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _on(dev: torch.device, handle: int) -> torch.cuda.Stream:
    return torch.cuda.ExternalStream(handle, device=dev) if handle else torch.cuda.default_stream(dev)


def _capturing(dev: torch.device, stream) -> bool:
    """Whether a call's stream (None: the current one) is being captured into a graph."""
    if stream is None and dev.index == torch.cuda.current_device():
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.stream(_on(dev, _stream(dev, stream))):
        return torch.cuda.is_current_stream_capturing()


def _fresh(dev: torch.device, stream, make):
    """make(): new tensors for a call on `stream` (None: the current one) to write.
    Of that stream's memory: a block of the current one's may be waiting for work
    queued there, and would go to another tensor there while the call still runs."""
    if stream is None or _stream(dev, stream) == _stream(dev, None):
        return make()
    with torch.cuda.stream(_on(dev, _stream(dev, stream))):
        return make()


def _new_out(q: torch.Tensor, stream) -> torch.Tensor:
    return _fresh(q.device, stream, lambda: torch.empty_like(q, memory_format=torch.contiguous_format))


def _bf16_cuda(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, names=("q", "k", "v")) -> None:
    bf16 = torch.bfloat16
    if (q.dtype is bf16 and k.dtype is bf16 and v.dtype is bf16 and q.is_contiguous() and k.is_contiguous()
            and v.is_contiguous() and q.is_cuda and k.is_cuda and v.is_cuda):
        return
    for name, t in zip(names, (q, k, v)):
        if t.dtype != bf16 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"{name} must be a contiguous bfloat16 CUDA tensor")


def _shapes(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu: Optional[torch.Tensor],
            L_K_max: Optional[int]) -> Tuple[int, int, int, int, int]:
    _bf16_cuda(q, k, v)
    ks = k.shape
    if ks != v.shape:
        raise ValueError("k and v shapes differ")
    B, H_Q, d = q.shape
    if cu is None:
        if len(ks) != 4 or ks[0] != B or ks[3] != d:
            raise ValueError("k must be [B, L_K, H_KV, d]")
        L = ks[1]
        H_KV = ks[2]
        if L_K_max is not None and L_K_max != L:
            raise ValueError("L_K_max must equal k.shape[1] for the fixed layout")
        L_K_max = L
    else:
        if cu.dtype != torch.int32 or not cu.is_contiguous() or cu.numel() != B + 1 or not cu.is_cuda:
            raise ValueError("cu_seqlens_k must be a contiguous int32 CUDA tensor of B+1 entries")
        if k.dim() != 3 or k.shape[2] != d:
            raise ValueError("varlen k must be [sum L_b, H_KV, d]")
        H_KV = k.shape[1]
        if L_K_max is None:
            raise ValueError("L_K_max (the host-known longest sequence) is required with cu_seqlens_k")
    return B, H_Q, H_KV, _int(int(L_K_max)), d


_workspaces: Dict[Tuple[int, int], torch.Tensor] = {}
# Workspaces replaced by a larger one.  They are never freed: a HIP graph
# captured earlier keeps their addresses, and kernels queued on a stream
# other than torch's current one may still be using them, so returning them
# to the caching allocator could hand live memory to another tensor.
_retired: List[torch.Tensor] = []


def workspace_for(dev: torch.device, stream_handle: int, nbytes: int) -> torch.Tensor:
    """A workspace of at least nbytes, cached per (device, stream).  Calls on
    one stream run in order, so they can share it.  It is zero-filled when
    allocated: the chunk-state regions need no initialisation (every call
    writes what it reads), and the arrival counters of single-launch plans
    start at zero and are left at zero by every call.  A cache that has to
    grow keeps its old buffer alive for the life of the process."""
    index = dev.index if dev.index is not None else (torch.cuda.current_device() if dev.type == "cuda" else -1)
    key = (index, stream_handle)
    ws = _workspaces.get(key)
    if ws is None or ws.numel() < nbytes:
        if ws is not None:
            _retired.append(ws)
        ws = _workspaces[key] = _zeros_before(dev, stream_handle, max(nbytes, 256))
    return ws


def _zeros_before(dev: torch.device, stream_handle: int, nbytes: int) -> torch.Tensor:
    """nbytes zero bytes for the next kernel on the stream of this handle."""
    make = lambda: torch.zeros(nbytes, dtype=torch.uint8, device=dev)  # noqa: E731
    if dev.type != "cuda" or stream_handle == _stream(dev, None):
        return make()
    own, cur = _on(dev, stream_handle), torch.cuda.current_stream(dev)
    own_captures, cur_captures = _capturing(dev, own), _capturing(dev, cur)
    if cur_captures and not own_captures:
        # a fill on the current stream would be recorded for the graph's replays and not run now
        with torch.cuda.stream(own):
            return make()
    ws = make()  # on the current stream
    # A captured stream may not wait for one outside its graph; such a fill runs
    # now, the graph's first replay later.
    if own_captures == cur_captures:
        own.wait_stream(cur)
    return ws


def _offered(workspace: Optional[torch.Tensor], dev: torch.device, s_handle: int) -> Optional[torch.Tensor]:
    """The workspace to offer an entry point that plans for itself: the
    caller's, or the one cached for this stream as it is.  Only where the plan
    needs a larger one, which the entry point finds before it launches
    anything, is the plan made here too and the cached one grown."""
    return _usable(workspace, dev) if workspace is not None else _workspaces.get((dev.index, s_handle))


def _usable(workspace: torch.Tensor, dev: torch.device) -> torch.Tensor:
    """A caller's workspace, whose bytes a kernel on `dev` may write from its address on."""
    if workspace.get_device() != dev.index or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}, got one on {workspace.device}")
    return workspace


def _nbytes(t: Optional[torch.Tensor]) -> int:
    return t.numel() * t.element_size() if t is not None else 0


def _deals(B: int, H_Q: int, H_KV: int, L: int, keys: int, dev: torch.device, stream) -> bool:
    """Whether a batch whose lengths the device holds goes to
    da_decode_attn_dealt.  Not while a graph is captured: its replays follow
    other lengths, for which L_K_max is a bound and not the longest sequence
    (78 sequences of 100-550 keys under L_K_max 32768: 8.2 us, dealt 14.9),
    and a workspace allocated then would be cleared by the replays only."""
    return load().da_prefers_dealt(B, H_Q, H_KV, L, keys, 0) != 0 and not _capturing(dev, stream)


def da_decode_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens_k: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None, *,
                   L_K_max: Optional[int] = None, softmax_scale: float = 0.0, num_splits: int = 0,
                   pack_gqa: int = -1, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """O = softmax(scale q K^T) V for one decode step; returns `out`.  A packed
    batch with nothing forced and no workspace passed goes to
    da_decode_attn_dealt where that pays, outside graph capture."""
    B, H_Q, H_KV, L, d = _shapes(q, k, v, cu_seqlens_k, L_K_max)
    if (cu_seqlens_k is not None and workspace is None and num_splits <= 0 and pack_gqa == -1
            and L >= DEALT_MIN_KEYS and d == HEAD_DIM and _deals(B, H_Q, H_KV, L, k.shape[0], q.device, stream)):
        return da_decode_attn_dealt(q, k, v, L, cu_seqlens_k, out=out, lse_out=lse_out, softmax_scale=softmax_scale,
                                    stream=stream)
    dev = q.device
    if out is None:
        out = _new_out(q, stream)
    s_handle = _stream(dev, stream)
    ws = _offered(workspace, dev, s_handle)
    while True:
        rc = load().da_decode_attn(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens_k), _ptr(out), _ptr(lse_out),
                                   B, H_Q, H_KV, L, d, float(softmax_scale), _int(int(num_splits)), _int(int(pack_gqa)),
                                   _ptr(ws), _nbytes(ws), s_handle)
        if rc != DA_ERR_WORKSPACE or workspace is not None:
            break
        plan = da_make_plan(B, H_Q, H_KV, L, d, num_splits, pack_gqa)
        workspace = ws = workspace_for(dev, s_handle, da_workspace_bytes(B, H_Q, d, plan.num_splits))
    _check(rc)
    return out


def da_decode_attn_planned(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: DaPlan,
                           cu_seqlens_k: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                           lse_out: Optional[torch.Tensor] = None, *, L_K_max: Optional[int] = None,
                           softmax_scale: float = 0.0, workspace: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """da_decode_attn with a plan made beforehand (da_make_plan /
    da_choose_splits, any policy or cu_margin), run exactly as it is."""
    B, H_Q, H_KV, L, d = _shapes(q, k, v, cu_seqlens_k, L_K_max)
    dev = q.device
    if out is None:
        out = _new_out(q, stream)
    s_handle = _stream(dev, stream)
    if workspace is None:
        nbytes = da_workspace_bytes(B, H_Q, d, plan.num_splits)
        if nbytes:
            workspace = workspace_for(dev, s_handle, nbytes)
    else:
        _usable(workspace, dev)
    ws_ptr = _ptr(workspace)
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(load().da_decode_attn_planned(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens_k), _ptr(out), _ptr(lse_out),
                                         B, H_Q, H_KV, L, d, float(softmax_scale), ctypes.byref(plan),
                                         ws_ptr, ws_bytes, s_handle))
    return out


def da_decode_attn_noalloc(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                           cu_seqlens_k: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                           lse_out: Optional[torch.Tensor] = None, *, L_K_max: Optional[int] = None,
                           softmax_scale: float = 0.0, num_splits: int = 0, pack_gqa: int = -1,
                           stream=None) -> torch.Tensor:
    """da_decode_attn with no workspace: the library's fixed per-device
    scratch holds the chunk states.  Pass `out` to make the call allocate
    nothing at all."""
    B, H_Q, H_KV, L, d = _shapes(q, k, v, cu_seqlens_k, L_K_max)
    if out is None:
        out = _new_out(q, stream)
    _check(load().da_decode_attn_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens_k), _ptr(out), _ptr(lse_out),
                                         B, H_Q, H_KV, L, d, float(softmax_scale), _int(int(num_splits)),
                                         _int(int(pack_gqa)),
                                         _stream(q.device, stream)))
    return out


def _paged_args(q, k_cache, v_cache, block_table, seq_lens):
    """Check a paged call's tensors; (B, H_Q, H_KV, d, page_size, max_pages, num_pages)."""
    _bf16_cuda(q, k_cache, v_cache, ("q", "k_cache", "v_cache"))
    for name, t in (("block_table", block_table), ("seq_lens", seq_lens)):
        if t.dtype != torch.int32 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
    if k_cache.shape != v_cache.shape or k_cache.dim() != 4:
        raise ValueError("k_cache and v_cache must both be [num_pages, page_size, H_KV, d]")
    B, H_Q, d = q.shape
    num_pages, page_size, H_KV, dk = k_cache.shape
    if dk != d or block_table.dim() != 2 or block_table.shape[0] != B or seq_lens.numel() != B:
        raise ValueError("block_table must be [B, max_pages], seq_lens [B], and the head dims must agree")
    return B, H_Q, H_KV, d, page_size, _int(block_table.shape[1]), num_pages


def da_decode_attn_paged(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
                         seq_lens: torch.Tensor, L_K_max: int, out: Optional[torch.Tensor] = None,
                         lse_out: Optional[torch.Tensor] = None, *, softmax_scale: float = 0.0, num_splits: int = 0,
                         pack_gqa: int = -1, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Decode attention over a paged KV cache; returns `out`.
    k_cache, v_cache: [num_pages, page_size, H_KV, d] bf16; block_table: [B, max_pages] int32;
    seq_lens: [B] int32; L_K_max: host-known longest sequence.  A batch with
    nothing forced and no workspace passed goes to da_decode_attn_dealt where
    that pays, outside graph capture."""
    B, H_Q, H_KV, d, page_size, max_pages, num_pages = _paged_args(q, k_cache, v_cache, block_table, seq_lens)
    if (workspace is None and num_splits <= 0 and pack_gqa == -1 and L_K_max >= DEALT_MIN_KEYS and d == HEAD_DIM
            and _deals(B, H_Q, H_KV, _int(int(L_K_max)), num_pages * page_size, q.device, stream)):
        return da_decode_attn_dealt(q, k_cache, v_cache, L_K_max, None, block_table, seq_lens, out, lse_out,
                                    softmax_scale=softmax_scale, stream=stream)
    dev = q.device
    if out is None:
        out = _new_out(q, stream)
    s_handle = _stream(dev, stream)
    L = _int(int(L_K_max))
    ws = _offered(workspace, dev, s_handle)
    while True:
        rc = load().da_decode_attn_paged(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(seq_lens),
                                         _ptr(out), _ptr(lse_out), B, H_Q, H_KV, page_size, max_pages, num_pages, L,
                                         d, float(softmax_scale), _int(int(num_splits)), _int(int(pack_gqa)), _ptr(ws),
                                         _nbytes(ws), s_handle)
        if rc != DA_ERR_WORKSPACE or workspace is not None:
            break
        plan = da_make_plan(B, H_Q, H_KV, L, d, num_splits, pack_gqa)
        workspace = ws = workspace_for(dev, s_handle, da_workspace_bytes(B, H_Q, d, plan.num_splits))
    _check(rc)
    return out


def da_decode_attn_paged_planned(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                                 block_table: torch.Tensor, seq_lens: torch.Tensor, L_K_max: int, plan: DaPlan,
                                 out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None, *,
                                 softmax_scale: float = 0.0, workspace: Optional[torch.Tensor] = None,
                                 stream=None) -> torch.Tensor:
    """da_decode_attn_paged with a plan made beforehand, run exactly as it is."""
    B, H_Q, H_KV, d, page_size, max_pages, num_pages = _paged_args(q, k_cache, v_cache, block_table, seq_lens)
    dev = q.device
    if out is None:
        out = _new_out(q, stream)
    s_handle = _stream(dev, stream)
    if workspace is None:
        nbytes = da_workspace_bytes(B, H_Q, d, plan.num_splits)
        if nbytes:
            workspace = workspace_for(dev, s_handle, nbytes)
    else:
        _usable(workspace, dev)
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(load().da_decode_attn_paged_planned(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table),
                                               _ptr(seq_lens), _ptr(out), _ptr(lse_out), B, H_Q, H_KV, page_size,
                                               max_pages, num_pages, _int(int(L_K_max)), d, float(softmax_scale),
                                               ctypes.byref(plan), _ptr(workspace), ws_bytes, s_handle))
    return out


def da_schedule_max_bytes(B: int, H_Q: int, H_KV: int, pack_gqa: int = -1) -> int:
    return int(load().da_schedule_max_bytes(_int(B), _int(H_Q), _int(H_KV), _int(pack_gqa)))


def da_make_schedule(seq_lens: Sequence[int], H_Q: int, H_KV: int, L_K_max: Optional[int] = None,
                     d: int = HEAD_DIM, pack_gqa: int = -1, num_cus: int = 0, cu_margin: int = 0,
                     chunk_tiles: int = 0) -> Tuple[DaSchedule, torch.Tensor]:
    """Per-sequence schedule from host-known lengths: (DaSchedule, metadata
    bytes as a CPU uint8 tensor to copy to the device)."""
    lens = torch.as_tensor(list(seq_lens) if not isinstance(seq_lens, torch.Tensor) else seq_lens.cpu(),
                           dtype=torch.int32).contiguous()
    B = lens.numel()
    if L_K_max is None:
        L_K_max = int(lens.max()) if B else 0
    cap = da_schedule_max_bytes(B, H_Q, H_KV, pack_gqa)
    meta = torch.zeros(max(cap, 16), dtype=torch.uint8)
    sched = DaSchedule()
    _check(load().da_make_schedule(lens.data_ptr() if B else None,
                                   *map(_int, (B, H_Q, H_KV, int(L_K_max), d, pack_gqa, num_cus, cu_margin,
                                               chunk_tiles)),
                                   meta.data_ptr(), meta.numel(), ctypes.byref(sched)))
    return sched, meta[: sched.meta_bytes].clone()


def da_schedule_workspace_bytes(sched: DaSchedule) -> int:
    return int(load().da_schedule_workspace_bytes(ctypes.byref(sched)))


def da_decode_attn_scheduled(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, sched: DaSchedule,
                             meta_dev: torch.Tensor, cu_seqlens_k: Optional[torch.Tensor] = None,
                             block_table: Optional[torch.Tensor] = None, seq_lens: Optional[torch.Tensor] = None,
                             out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None, *,
                             softmax_scale: float = 0.0, workspace: Optional[torch.Tensor] = None,
                             stream=None) -> torch.Tensor:
    """Decode attention driven by a per-sequence schedule; returns `out`.
    Contiguous K/V (fixed, or varlen with cu_seqlens_k) when block_table is
    None, else paged: k, v [num_pages, page_size, H_KV, d] with block_table
    [B, max_pages] and seq_lens [B]."""
    _bf16_cuda(q, k, v)
    if meta_dev.dtype != torch.uint8 or not meta_dev.is_cuda or meta_dev.numel() < sched.meta_bytes:
        raise ValueError("meta_dev must be a CUDA uint8 tensor holding the schedule's metadata")
    B, H_Q, d = q.shape
    if B != sched.B or H_Q != sched.H_Q:
        raise ValueError("q does not match the schedule")
    page_size = max_pages = num_pages = 0
    if block_table is not None:
        for name, t in (("block_table", block_table), ("seq_lens", seq_lens)):
            if t is None or t.dtype != torch.int32 or not t.is_contiguous() or not t.is_cuda:
                raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
        num_pages, page_size = k.shape[0], k.shape[1]
        max_pages = block_table.shape[1]
    dev = q.device
    if out is None:
        out = _new_out(q, stream)
    s_handle = _stream(dev, stream)
    if workspace is None:
        nbytes = da_schedule_workspace_bytes(sched)
        if nbytes:
            workspace = workspace_for(dev, s_handle, nbytes)
    else:
        _usable(workspace, dev)
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(load().da_decode_attn_scheduled(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens_k), _ptr(block_table),
                                           _ptr(seq_lens), page_size, max_pages, num_pages, _ptr(out),
                                           _ptr(lse_out), d, float(softmax_scale), ctypes.byref(sched),
                                           _ptr(meta_dev), _ptr(workspace), ws_bytes, s_handle))
    return out


def da_decode_attn_dealt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, L_K_max: int,
                         cu_seqlens_k: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                         seq_lens: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                         lse_out: Optional[torch.Tensor] = None, *, softmax_scale: float = 0.0,
                         workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Decode attention over a batch of mixed lengths, its tiles shared evenly
    among the CUs on the device; returns `out`.  Packed K/V with cu_seqlens_k
    when block_table is None, else paged.  da_decode_attn and
    da_decode_attn_paged come here by themselves where it pays."""
    page_size = max_pages = num_pages = keys = 0
    if block_table is None:
        if cu_seqlens_k is None:
            raise ValueError("cu_seqlens_k, or block_table and seq_lens, are required")
        B, H_Q, H_KV, L, d = _shapes(q, k, v, cu_seqlens_k, L_K_max)
        keys = k.shape[0]
    else:
        B, H_Q, H_KV, d, page_size, max_pages, num_pages = _paged_args(q, k, v, block_table, seq_lens)
        L = _int(int(L_K_max))
    dev = q.device
    if out is None:
        out = _new_out(q, stream)
    s_handle = _stream(dev, stream)
    if workspace is None:
        workspace = workspace_for(dev, s_handle, da_dealt_workspace_bytes(B, H_Q, H_KV))
    else:
        _usable(workspace, dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(load().da_decode_attn_dealt(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens_k), _ptr(block_table),
                                       _ptr(seq_lens), page_size, max_pages, num_pages, _ptr(out), _ptr(lse_out),
                                       B, H_Q, H_KV, L, d, float(softmax_scale), keys, _ptr(workspace), ws_bytes,
                                       s_handle))
    return out


def da_split_partials(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                      cu_seqlens_k: Optional[torch.Tensor] = None, o_part: Optional[torch.Tensor] = None,
                      m_part: Optional[torch.Tensor] = None, l_part: Optional[torch.Tensor] = None, *,
                      num_splits: int, pack_gqa: int, L_K_max: Optional[int] = None,
                      softmax_scale: float = 0.0, stream=None):
    """Per-chunk partial states (o_part [s,B,H_Q,d], m_part, l_part [s,B,H_Q])."""
    B, H_Q, H_KV, L, d = _shapes(q, k, v, cu_seqlens_k, L_K_max)
    dev = q.device
    new = lambda *shape: _fresh(dev, stream, lambda: torch.empty(shape, dtype=torch.float32, device=dev))  # noqa: E731
    if o_part is None:
        o_part = new(num_splits, B, H_Q, d)
    if m_part is None:
        m_part = new(num_splits, B, H_Q)
    if l_part is None:
        l_part = new(num_splits, B, H_Q)
    _check(load().da_split_partials(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens_k), _ptr(o_part), _ptr(m_part),
                                    _ptr(l_part), B, H_Q, H_KV, L, d, float(softmax_scale), _int(int(num_splits)),
                                    _int(int(pack_gqa)), _stream(dev, stream)))
    return o_part, m_part, l_part


def da_combine_splits(o_part: torch.Tensor, m_part: torch.Tensor, l_part: torch.Tensor,
                      out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None, *,
                      stream=None) -> torch.Tensor:
    """Log-sum-exp merge of partial states; returns `out` (bf16 [B,H_Q,d])."""
    for name, t in (("o_part", o_part), ("m_part", m_part), ("l_part", l_part)):
        if t.dtype != torch.float32 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"{name} must be a contiguous float32 CUDA tensor")
    s, B, H_Q, d = o_part.shape
    if tuple(m_part.shape) != (s, B, H_Q) or tuple(l_part.shape) != (s, B, H_Q):
        raise ValueError("m_part and l_part must be [s, B, H_Q]")
    dev = o_part.device
    if out is None:
        out = _fresh(dev, stream, lambda: torch.empty((B, H_Q, d), dtype=torch.bfloat16, device=dev))
    _check(load().da_combine_splits(_ptr(o_part), _ptr(m_part), _ptr(l_part), _ptr(out), _ptr(lse_out), s, B, H_Q,
                                    d, _stream(dev, stream)))
    return out


# ---------------------------------------------------------------- a step's cache: tables, rows, windows, 4 bits

_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_BF16, _I32, _F32 = torch.bfloat16, torch.int32, torch.float32


def _on_device(dev: torch.device, fn, *args, **kw):
    """fn(*args, **kw) with `dev` the current device (the library launches on that one)."""
    with torch.cuda.device(dev):
        return fn(*args, **kw)


_captures = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None) or torch.cuda.is_current_stream_capturing
# (device, stream) -> (capture, workspace): of the capture that is under way there, or was last
_graph_workspaces: Dict[Tuple[int, int], Tuple[int, torch.Tensor]] = {}


def _offered_now(dev: torch.device, stream, handle: int) -> Tuple[Optional[torch.Tensor], int]:
    """The workspace to offer a call on the current device that passes none, and
    the number of the capture it is part of, or 0.  Outside graph capture it is
    the one cached for the stream.  A captured call takes one out of its graph's
    memory (torch.cuda.graph's; a capture made by other means passes its own),
    shared by the calls captured on that stream and cleared by each replay, so that
    graphs with pools of their own can be replayed in any order, beside each other
    and beside the stream's own calls.  Graphs that share a pool are replayed one
    after the other, as torch asks of them.  The last one of a stream is held until
    another graph is captured there, and its pool with it."""
    if not (_captures() if stream is None else _capturing(dev, stream)):
        return _workspaces.get((dev.index, handle)), 0
    status, number = ctypes.c_int(), ctypes.c_ulonglong()
    if load().hipStreamGetCaptureInfo(_P(handle), ctypes.byref(status), ctypes.byref(number)):
        raise DecodeAttnError(DA_ERR_HIP, "the stream's capture has no number")
    capture, ws = _graph_workspaces.get((dev.index, handle), (0, None))
    return (ws if capture == number.value + 1 else None), number.value + 1


def _grown(dev: torch.device, handle: int, capture: int, nbytes: int) -> torch.Tensor:
    """A larger workspace than the one offered."""
    if not capture:
        return workspace_for(dev, handle, nbytes)
    with torch.cuda.stream(_on(dev, handle)):
        ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        ws[-ARRIVAL_BYTES:].zero_()
    _graph_workspaces[dev.index, handle] = (capture, ws)
    return ws


def _need(name: str, t: torch.Tensor, dtype: torch.dtype, shape: Tuple[int, ...], dev: torch.device) -> None:
    # dev: a CUDA device (get_device: -1 on the CPU), and cheaper to compare by its number
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev.index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {tuple(shape)} on {dev}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")


def _outputs(q: torch.Tensor, out: Optional[torch.Tensor], lse_out: Optional[torch.Tensor], stream) -> torch.Tensor:
    if out is None:
        # q is contiguous
        out = torch.empty_like(q) if stream is None else _new_out(q, stream)
    else:
        _need("out", out, _BF16, q.shape, q.device)
    if lse_out is not None:
        _need("lse_out", lse_out, _F32, q.shape[:2], q.device)
    return out


def _one_device(dev: torch.device, *tensors: Optional[torch.Tensor]) -> None:
    index = dev.index
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError(f"the call's tensors must be on one device, got {dev} and {t.device}")


def da_window_keys(L_K_max: int, window: int, sinks: int = 0) -> int:
    return int(load().da_window_keys(_int(L_K_max), _int(window), _int(sinks)))


def da_decode_attn_window(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, window: int, sinks: int = 0,
                          cu_seqlens_k: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                          seq_lens: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                          lse_out: Optional[torch.Tensor] = None, *, L_K_max: Optional[int] = None,
                          softmax_scale: float = 0.0, num_splits: int = 0, pack_gqa: int = -1,
                          workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Decode attention that sees the last `window` keys of each sequence and
    its first `sinks` keys; returns `out`.  K and V as for da_decode_attn (fixed,
    or packed with cu_seqlens_k), or with block_table and seq_lens paged."""
    dev = q.device
    window, sinks, num_splits, pack_gqa = _int(window), _int(sinks), _int(num_splits), _int(pack_gqa)
    page_size = max_pages = num_pages = 0
    if (cu_seqlens_k if block_table is not None else seq_lens) is not None:
        raise ValueError("seq_lens are the lengths of a paged batch (block_table), cu_seqlens_k those of a packed one")
    if block_table is None:
        B, H_Q, H_KV, L, d = _shapes(q, k, v, cu_seqlens_k, L_K_max)
    else:
        if seq_lens is None or L_K_max is None:
            raise ValueError("seq_lens and L_K_max (the host-known longest sequence) are required with block_table")
        B, H_Q, H_KV, d, page_size, max_pages, num_pages = _paged_args(q, k, v, block_table, seq_lens)
        L = _int(int(L_K_max))
    _one_device(dev, k, v, cu_seqlens_k, block_table, seq_lens)
    if dev.index != _get_device():
        return _on_device(dev, da_decode_attn_window, q, k, v, window, sinks, cu_seqlens_k, block_table, seq_lens, out,
                          lse_out, L_K_max=L_K_max, softmax_scale=softmax_scale, num_splits=num_splits,
                          pack_gqa=pack_gqa, workspace=workspace, stream=stream)
    out = _outputs(q, out, lse_out, stream)
    s_handle = _stream(dev, stream)
    ws, capture = (_usable(workspace, dev), 0) if workspace is not None else _offered_now(dev, stream, s_handle)
    while True:
        rc = load().da_decode_attn_window(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(cu_seqlens_k), _ptr(block_table), _ptr(seq_lens), page_size,
            max_pages, num_pages, out.data_ptr(), _ptr(lse_out), B, H_Q, H_KV, L, d, softmax_scale, window, sinks,
            num_splits, pack_gqa, _ptr(ws), _nbytes(ws), s_handle)
        if rc != DA_ERR_WORKSPACE or workspace is not None:
            break
        plan = da_make_plan(B, H_Q, H_KV, da_window_keys(L, window, sinks), d, num_splits, pack_gqa)
        workspace = ws = _grown(dev, s_handle, capture, da_workspace_bytes(B, H_Q, d, plan.num_splits))
    if rc:
        _check(rc)
    return out


def da_extend_tables(lens: torch.Tensor, new_lens: torch.Tensor, free_pages: torch.Tensor, taken: torch.Tensor,
                     block_table: torch.Tensor, page_size: int, num_pages: int, max_tokens: int,
                     lens_out: Optional[torch.Tensor] = None, taken_out: Optional[torch.Tensor] = None,
                     cu_new: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                     positions: Optional[torch.Tensor] = None, *, stream=None) -> Tuple[torch.Tensor, ...]:
    """Block tables and slots of a step from request lengths; returns
    (lens_out, taken_out, cu_new, slots, positions), new tensors where none are
    passed.  All int32 on one device: lens and new_lens [B]; free_pages: page
    ids, of which `taken` [1] are in use; block_table [B, max_pages], whose
    entries of new pages are written; slots and positions [max_tokens].
    lens_out may be lens and taken_out may be taken.  After the first request
    that the list cannot serve no later one gets a page."""
    dev = lens.device
    if (lens.dim() != 1 or free_pages.dim() != 1 or block_table.dim() != 2 or not 0 <= max_tokens <= MAX_NEW_TOKENS
            or not lens.is_cuda):
        raise ValueError("lens and free_pages must have one dimension, block_table two, on the GPU, and max_tokens "
                         f"must be in [0, {MAX_NEW_TOKENS}]")
    B = lens.shape[0]
    num_free = free_pages.shape[0]
    max_pages = block_table.shape[1]
    one, rows = (B,), (max_tokens,)
    _need("lens", lens, _I32, one, dev)
    _need("new_lens", new_lens, _I32, one, dev)
    _need("free_pages", free_pages, _I32, (num_free,), dev)
    _need("taken", taken, _I32, (1,), dev)
    _need("block_table", block_table, _I32, (B, max_pages), dev)
    if dev.index != _get_device():
        return _on_device(dev, da_extend_tables, lens, new_lens, free_pages, taken, block_table, page_size, num_pages,
                          max_tokens, lens_out, taken_out, cu_new, slots, positions, stream=stream)
    sizes = (B, 1, B + 1, max_tokens, max_tokens)
    given = (lens_out, taken_out, cu_new, slots, positions)
    new = None
    if not any(t is not None for t in given):
        new = _fresh(dev, stream, lambda: torch.empty(2 * B + 2 + 2 * max_tokens, dtype=_I32, device=dev))
        at = new.data_ptr()
        ptrs = (at, at + 4 * B, at + 4 * B + 4, at + 8 * B + 8, at + 8 * B + 8 + 4 * max_tokens)
    else:
        for name, t, n in zip(("lens_out", "taken_out", "cu_new", "slots", "positions"), given, sizes):
            if t is not None:
                _need(name, t, _I32, (n,), dev)
        mine = given
        given = _fresh(dev, stream, lambda: tuple(torch.empty(n, dtype=_I32, device=dev) if t is None else t
                                                  for t, n in zip(mine, sizes)))
        ptrs = tuple(_ptr(t) for t in given)
    rc = load().da_extend_tables(lens.data_ptr(), new_lens.data_ptr(), free_pages.data_ptr(), taken.data_ptr(),
                                 block_table.data_ptr(), *ptrs, B, _int(page_size), _int(max_pages), _int(num_pages),
                                 _int(num_free), max_tokens, _stream(dev, stream))
    if rc:
        _check(rc)
    return given if new is None else new.split_with_sizes(sizes)


def _rows(name: str, t: torch.Tensor, dev: torch.device) -> Tuple[int, torch.Size]:
    """Token stride and shape of q, k or v [N, heads, d]: heads dense, tokens any distance apart."""
    shape = t.shape
    if len(shape) == 3:
        stride = t.stride()
        if ((stride[2] == 1 or shape[2] == 1) and (stride[1] == shape[2] or shape[1] == 1) and t.dtype is _BF16
                and t.get_device() == dev.index):
            return (stride[0] if shape[0] > 1 else 0), shape
    raise ValueError(f"{name} must be a bfloat16 tensor [N, heads, d] on {dev} whose heads are dense")


def _append_args(q, k, v, positions, slots, rope, q_weight, k_weight, eps, neighbours, q_out, stream, axes=None):
    """Check what the append calls share; (their leading arguments, N, H_Q, H_KV, d, q_out)."""
    dev = k.device
    if not k.is_cuda:
        raise ValueError("k must be on the GPU")
    k_stride, shape = _rows("k", k, dev)
    v_stride, v_shape = _rows("v", v, dev)
    if v_shape != shape:
        raise ValueError("k and v shapes differ")
    N, H_KV, d = shape
    q_stride = H_Q = rope_rows = rope_dim = 0
    if q is not None:
        q_stride, q_shape = _rows("q", q, dev)
        H_Q = q_shape[1]
        if q_shape[0] != N or q_shape[2] != d:
            raise ValueError("q must be [N, H_Q, d] with k's N and d")
        if q_out is None:
            q_out = _fresh(dev, stream, lambda: torch.empty(q_shape, dtype=_BF16, device=dev))
        else:
            _need("q_out", q_out, _BF16, q_shape, dev)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if q_weight is not None:
        _need("q_weight", q_weight, _BF16, (d,), dev)
    if k_weight is not None:
        _need("k_weight", k_weight, _BF16, (d,), dev)
    if rope is None:
        positions = None
    else:
        if rope.dim() != 2 or rope.numel() == 0 or positions is None:
            raise ValueError("rope must be [positions, rope_dim], not empty, and needs positions")
        rope_rows, rope_dim = rope.shape
        _need("rope", rope, _F32, rope.shape, dev)
        if axes is None:
            _need("positions", positions, _I32, (N,), dev)
        else:
            if positions.dim() != 2 or not 1 <= positions.shape[0] <= MAX_AXES or len(axes) != rope_dim // 2:
                raise ValueError(f"positions must be [1 to {MAX_AXES} axes, N], and axes name one for each of the "
                                 "rope_dim / 2 pairs")
            _need("positions", positions, _I32, (positions.shape[0], N), dev)
    if slots is not None:
        _need("slots", slots, _I32, (N,), dev)
    return (q.data_ptr() if H_Q and N else None, q_stride, k.data_ptr(), k_stride, v.data_ptr(), v_stride,
            q_weight.data_ptr() if q_weight is not None else None,
            k_weight.data_ptr() if k_weight is not None else None, eps,
            rope.data_ptr() if rope is not None else None, rope_rows, rope_dim, 1 if neighbours else 0,
            *(() if axes is None else (axes, positions.shape[0])),
            positions.data_ptr() if positions is not None else None, slots.data_ptr() if slots is not None else None,
            q_out.data_ptr() if H_Q and N else None), N, H_Q, H_KV, d, q_out


def da_append_kv(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor],
                 slots: Optional[torch.Tensor], k_cache: torch.Tensor, v_cache: torch.Tensor, *,
                 rope: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, neighbours: bool = False,
                 q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """Norms of q and k per head, rotation by position, and k and v into the
    rows `slots` of a bf16 cache; returns q_out (None without q).
    q [N, H_Q, d], k, v [N, H_KV, d]: slices of one projection's output will do;
    caches [..., H_KV, d] (page pools, or sequences), rows counted over the
    leading dims; rope fp32 [positions, rope_dim]: cosines, then sines."""
    dev = k.device
    if k.is_cuda and dev.index != _get_device():
        return _on_device(dev, da_append_kv, q, k, v, positions, slots, k_cache, v_cache, rope=rope, q_weight=q_weight,
                          k_weight=k_weight, eps=eps, neighbours=neighbours, q_out=q_out, stream=stream)
    args, N, H_Q, H_KV, d, q_out = _append_args(q, k, v, positions, slots, rope, q_weight, k_weight, eps, neighbours,
                                                q_out, stream)
    shape = k_cache.shape
    if len(shape) < 3 or shape[-2] != H_KV or shape[-1] != d:
        raise ValueError("k_cache must be [..., H_KV, d]")
    _need("k_cache", k_cache, _BF16, shape, dev)
    _need("v_cache", v_cache, _BF16, shape, dev)
    rc = load().da_append_kv(*args, k_cache.data_ptr(), v_cache.data_ptr(),
                             k_cache.numel() // (H_KV * d) if H_KV * d else 0, N, H_Q, H_KV, d, _stream(dev, stream))
    if rc:
        _check(rc)
    return q_out


def _kv4_cache(cache: torch.Tensor) -> Tuple[int, int, int]:
    """(num_pages, H_KV, page_size) of a 4-bit cache."""
    shape = cache.shape
    if (len(shape) != 4 or cache.dtype is not torch.uint8 or shape[3] != KV4_TILE_BYTES or not cache.is_contiguous()
            or not cache.is_cuda):
        raise ValueError("cache must be a contiguous uint8 CUDA tensor [num_pages, H_KV, page_size / 32, "
                         f"{KV4_TILE_BYTES}]")
    return shape[0], shape[1], 32 * shape[2]


def da_append_kv4(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor],
                  slots: Optional[torch.Tensor], cache: torch.Tensor, *, rope: Optional[torch.Tensor] = None,
                  q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  neighbours: bool = False, q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """da_append_kv into a 4-bit cache, uint8 [num_pages, H_KV, page_size / 32, 4352]; returns q_out."""
    dev = k.device
    if k.is_cuda and dev.index != _get_device():
        return _on_device(dev, da_append_kv4, q, k, v, positions, slots, cache, rope=rope, q_weight=q_weight,
                          k_weight=k_weight, eps=eps, neighbours=neighbours, q_out=q_out, stream=stream)
    args, N, H_Q, H_KV, d, q_out = _append_args(q, k, v, positions, slots, rope, q_weight, k_weight, eps, neighbours,
                                                q_out, stream)
    num_pages, heads, page_size = _kv4_cache(cache)
    if heads != H_KV:
        raise ValueError(f"the cache has {heads} KV heads, k {H_KV}")
    _one_device(dev, cache)
    rc = load().da_append_kv4(*args, cache.data_ptr(), page_size, num_pages, N, H_Q, H_KV, d, _stream(dev, stream))
    if rc:
        _check(rc)
    return q_out


def _axis_bytes(axes, rope) -> bytes:
    if rope is None:
        raise ValueError("rope is required")
    return axes if isinstance(axes, bytes) else bytes(list(axes))  # of an array its numbers, not its memory


def da_append_kv_axes(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor,
                      slots: Optional[torch.Tensor], k_cache: torch.Tensor, v_cache: torch.Tensor, *,
                      rope: torch.Tensor, axes: Sequence[int], q_weight: Optional[torch.Tensor] = None,
                      k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, neighbours: bool = False,
                      q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """da_append_kv for positions [A, N] on up to four axes: pair i of the
    rotation turns by the position on axis axes[i] (rope_dim / 2 whole numbers
    below A; bytes save the conversion); returns q_out."""
    dev = k.device
    if k.is_cuda and dev.index != _get_device():
        return _on_device(dev, da_append_kv_axes, q, k, v, positions, slots, k_cache, v_cache, rope=rope, axes=axes,
                          q_weight=q_weight, k_weight=k_weight, eps=eps, neighbours=neighbours, q_out=q_out,
                          stream=stream)
    args, N, H_Q, H_KV, d, q_out = _append_args(q, k, v, positions, slots, rope, q_weight, k_weight, eps, neighbours,
                                                q_out, stream, _axis_bytes(axes, rope))
    shape = k_cache.shape
    if len(shape) < 3 or shape[-2] != H_KV or shape[-1] != d:
        raise ValueError("k_cache must be [..., H_KV, d]")
    _need("k_cache", k_cache, _BF16, shape, dev)
    _need("v_cache", v_cache, _BF16, shape, dev)
    rc = load().da_append_kv_axes(*args, k_cache.data_ptr(), v_cache.data_ptr(),
                                  k_cache.numel() // (H_KV * d) if H_KV * d else 0, N, H_Q, H_KV, d,
                                  _stream(dev, stream))
    if rc:
        _check(rc)
    return q_out


def da_append_kv4_axes(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor,
                       slots: Optional[torch.Tensor], cache: torch.Tensor, *, rope: torch.Tensor, axes: Sequence[int],
                       q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                       eps: float = 1e-6, neighbours: bool = False, q_out: Optional[torch.Tensor] = None,
                       stream=None) -> Optional[torch.Tensor]:
    """da_append_kv_axes into a 4-bit cache (da_append_kv4); returns q_out."""
    dev = k.device
    if k.is_cuda and dev.index != _get_device():
        return _on_device(dev, da_append_kv4_axes, q, k, v, positions, slots, cache, rope=rope, axes=axes,
                          q_weight=q_weight, k_weight=k_weight, eps=eps, neighbours=neighbours, q_out=q_out,
                          stream=stream)
    args, N, H_Q, H_KV, d, q_out = _append_args(q, k, v, positions, slots, rope, q_weight, k_weight, eps, neighbours,
                                                q_out, stream, _axis_bytes(axes, rope))
    num_pages, heads, page_size = _kv4_cache(cache)
    if heads != H_KV:
        raise ValueError(f"the cache has {heads} KV heads, k {H_KV}")
    _one_device(dev, cache)
    rc = load().da_append_kv4_axes(*args, cache.data_ptr(), page_size, num_pages, N, H_Q, H_KV, d, _stream(dev, stream))
    if rc:
        _check(rc)
    return q_out


def da_read_kv4(cache: torch.Tensor, slots: Optional[torch.Tensor] = None, *,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """K and V bf16 [N, H_KV, 128] of the rows `slots` of a 4-bit cache (None: all its rows)."""
    num_pages, H_KV, page_size = _kv4_cache(cache)
    dev = cache.device
    if slots is None:
        N = num_pages * page_size
    else:
        if slots.dim() != 1:
            raise ValueError("slots must have one dimension")
        N = slots.shape[0]
        _need("slots", slots, _I32, (N,), dev)
    if dev.index != _get_device():
        return _on_device(dev, da_read_kv4, cache, slots, stream=stream)
    k, v = _fresh(dev, stream, lambda: torch.empty((2, N, H_KV, HEAD_DIM), dtype=_BF16, device=dev)).unbind(0)
    rc = load().da_read_kv4(cache.data_ptr(), _ptr(slots), k.data_ptr(), v.data_ptr(), N, H_KV, page_size, num_pages,
                            HEAD_DIM, _stream(dev, stream))
    if rc:
        _check(rc)
    return k, v


def da_kv4_workspace_bytes(B: int, H_Q: int, H_KV: int, L_K_max: int, pool_keys: int = 0, window: int = 0,
                           sinks: int = 0, num_splits: int = 0, num_cus: int = 0) -> int:
    return int(load().da_kv4_workspace_bytes(_int(B), _int(H_Q), _int(H_KV), _int(L_K_max),
                                             max(0, min(pool_keys, 2 ** 63 - 1)), _int(window), _int(sinks),
                                             _int(num_splits), _int(num_cus)))


def da_decode_attn_kv4(q: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor,
                       L_K_max: int, window: int = 0, sinks: int = 0, out: Optional[torch.Tensor] = None,
                       lse_out: Optional[torch.Tensor] = None, *, softmax_scale: float = 0.0, num_splits: int = 0,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Decode attention over a paged cache of 4-bit values (da_append_kv4);
    returns `out`.  block_table, seq_lens and L_K_max as for
    da_decode_attn_paged; window (0: none) and sinks as for
    da_decode_attn_window."""
    dev = q.device
    if q.dim() != 3 or q.dtype is not _BF16 or not q.is_contiguous() or not q.is_cuda:
        raise ValueError("q must be a contiguous bfloat16 CUDA tensor [B, H_Q, d]")
    num_pages, H_KV, page_size = _kv4_cache(cache)
    B, H_Q, d = q.shape
    window, sinks, num_splits = _int(window), _int(sinks), _int(num_splits)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    _need("block_table", block_table, _I32, (B, max_pages), dev)
    max_pages = _int(max_pages)
    _need("seq_lens", seq_lens, _I32, (B,), dev)
    _one_device(dev, cache)
    if dev.index != _get_device():
        return _on_device(dev, da_decode_attn_kv4, q, cache, block_table, seq_lens, L_K_max, window, sinks, out, lse_out,
                          softmax_scale=softmax_scale, num_splits=num_splits, workspace=workspace, stream=stream)
    out = _outputs(q, out, lse_out, stream)
    s_handle = _stream(dev, stream)
    L = _int(int(L_K_max))
    ws, capture = (_usable(workspace, dev), 0) if workspace is not None else _offered_now(dev, stream, s_handle)
    while True:
        rc = load().da_decode_attn_kv4(q.data_ptr(), cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                                       out.data_ptr(), _ptr(lse_out), B, H_Q, H_KV, page_size, max_pages, num_pages, L, d,
                                       softmax_scale, window, sinks, num_splits, _ptr(ws), _nbytes(ws), s_handle)
        if rc != DA_ERR_WORKSPACE or workspace is not None:
            break
        workspace = ws = _grown(dev, s_handle, capture,
                                da_kv4_workspace_bytes(B, H_Q, H_KV, L, num_pages * page_size, window, sinks, num_splits))
    if rc:
        _check(rc)
    return out


# ---------------------------------------------------------------- a shared and bounded cache
# (an empty tensor's data_ptr() is 0: NULL)


def _paged_pool(name: str, cache: torch.Tensor, dev: torch.device) -> Tuple[int, int, int, int]:
    """(num_pages, page_size, H_KV, d) of a bf16 page pool."""
    shape = cache.shape
    if len(shape) != 4:
        raise ValueError(f"{name} must be [num_pages, page_size, H_KV, d]")
    _need(name, cache, _BF16, shape, dev)
    return shape


def _table_args(block_table: torch.Tensor, seq_lens: torch.Tensor, B: int, dev: torch.device) -> int:
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    _need("block_table", block_table, _I32, (B, max_pages), dev)
    _need("seq_lens", seq_lens, _I32, (B,), dev)
    return _int(max_pages)


def da_prefix_workspace_bytes(B: int, G: int, H_Q: int, H_KV: int, num_cus: int = 0) -> int:
    return int(load().da_prefix_workspace_bytes(_int(B), _int(G), _int(H_Q), _int(H_KV), _int(num_cus)))


def da_decode_attn_prefix(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
                          seq_lens: torch.Tensor, cu_groups: torch.Tensor, prefix_lens: torch.Tensor, L_K_max: int,
                          out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None, *,
                          softmax_scale: float = 0.0, chunk_keys: int = 0, workspace: Optional[torch.Tensor] = None,
                          stream=None) -> torch.Tensor:
    """Decode attention over a paged cache in which groups of sequences begin with
    the same keys, which are read once a group; returns `out`.  Group i is the
    sequences [cu_groups[i], cu_groups[i + 1]), whose first prefix_lens[i] keys are
    the same; block_table and seq_lens hold whole sequences, as for
    da_decode_attn_paged.  A batch too small to gain by it is read as it is, unless
    chunk_keys is given (negative: chunks of a chosen length)."""
    dev = q.device
    if q.dim() != 3 or q.dtype is not _BF16 or not q.is_contiguous() or not q.is_cuda:
        raise ValueError("q must be a contiguous bfloat16 CUDA tensor [B, H_Q, d]")
    B, H_Q, d = q.shape
    num_pages, page_size, H_KV, dk = _paged_pool("k_cache", k_cache, dev)
    if dk != d:
        raise ValueError(f"k_cache has head dim {dk}, q {d}")
    _need("v_cache", v_cache, _BF16, k_cache.shape, dev)
    max_pages = _table_args(block_table, seq_lens, B, dev)
    if prefix_lens.dim() != 1:
        raise ValueError("prefix_lens must have one dimension")
    G = prefix_lens.shape[0]
    _need("prefix_lens", prefix_lens, _I32, (G,), dev)
    _need("cu_groups", cu_groups, _I32, (G + 1,), dev)
    if dev.index != _get_device():
        return _on_device(dev, da_decode_attn_prefix, q, k_cache, v_cache, block_table, seq_lens, cu_groups, prefix_lens,
                          L_K_max, out, lse_out, softmax_scale=softmax_scale, chunk_keys=chunk_keys,
                          workspace=workspace, stream=stream)
    out = _outputs(q, out, lse_out, stream)
    s_handle = _stream(dev, stream)
    L, chunk_keys = _int(int(L_K_max)), _int(int(chunk_keys))
    ws, capture = (_usable(workspace, dev), 0) if workspace is not None else _offered_now(dev, stream, s_handle)
    while True:
        rc = load().da_decode_attn_prefix(
            q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
            cu_groups.data_ptr(), prefix_lens.data_ptr(), out.data_ptr(), _ptr(lse_out), B, G, H_Q, H_KV, _int(page_size),
            max_pages, _int(num_pages), L, d, softmax_scale, chunk_keys, _ptr(ws), _nbytes(ws), s_handle)
        if rc != DA_ERR_WORKSPACE or workspace is not None:
            break
        workspace = ws = _grown(dev, s_handle, capture, da_prefix_workspace_bytes(B, G, H_Q, H_KV))
    if rc:
        _check(rc)
    return out


def da_add_key_weights(q: torch.Tensor, k_cache: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor,
                       lse: torch.Tensor, weights: torch.Tensor, L_K_max: int, decay: float = 1.0,
                       weights_out: Optional[torch.Tensor] = None, *, softmax_scale: float = 0.0,
                       stream=None) -> torch.Tensor:
    """The attention weight of every key, summed over the heads that share it:
    weights_out = decay weights + sum over heads of exp(scale q k - lse); returns
    weights_out, which is `weights` where none is passed.  q [B, H_Q, d], lse
    [B, H_Q] of the attention call, weights fp32 [B, H_KV, at least L_K_max]."""
    dev = q.device
    if q.dim() != 3 or q.dtype is not _BF16 or not q.is_contiguous() or not q.is_cuda:
        raise ValueError("q must be a contiguous bfloat16 CUDA tensor [B, H_Q, d]")
    B, H_Q, d = q.shape
    num_pages, page_size, H_KV, dk = _paged_pool("k_cache", k_cache, dev)
    if dk != d:
        raise ValueError(f"k_cache has head dim {dk}, q {d}")
    max_pages = _table_args(block_table, seq_lens, B, dev)
    _need("lse", lse, _F32, (B, H_Q), dev)
    if weights.dim() != 3:
        raise ValueError("weights must be [B, H_KV, keys]")
    stride = weights.shape[2]
    _need("weights", weights, _F32, (B, H_KV, stride), dev)
    if weights_out is None:
        weights_out = weights
    else:
        _need("weights_out", weights_out, _F32, (B, H_KV, stride), dev)
    if dev.index != _get_device():
        return _on_device(dev, da_add_key_weights, q, k_cache, block_table, seq_lens, lse, weights, L_K_max, decay,
                          weights_out, softmax_scale=softmax_scale, stream=stream)
    rc = load().da_add_key_weights(
        q.data_ptr(), k_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), lse.data_ptr(), weights.data_ptr(),
        weights_out.data_ptr(), stride, B, H_Q, H_KV, _int(page_size), max_pages, _int(num_pages), _int(int(L_K_max)), d,
        softmax_scale, decay, _stream(dev, stream))
    if rc:
        _check(rc)
    return weights_out


def da_evict_workspace_bytes(B: int, H_KV: int, L_K_max: int, budget: int) -> int:
    return int(load().da_evict_workspace_bytes(_int(B), _int(H_KV), _int(L_K_max), _int(budget)))


def da_evict_kv(k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor,
                totals: torch.Tensor, weights: torch.Tensor, positions: torch.Tensor, budget: int, L_K_max: int, *,
                sinks: int = 0, recent: int = 0, free_pages: Optional[torch.Tensor] = None,
                taken: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
                weights_out: Optional[torch.Tensor] = None, positions_out: Optional[torch.Tensor] = None,
                taken_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Sequences of more than `budget` keys keep that many, of each KV head those
    of the first `sinks` and the last `recent` positions and the largest weights;
    rows move within the caches; returns (lens_out, weights_out, positions_out,
    taken_out), which are seq_lens, weights, positions and taken where none are
    passed.  totals int32 [B]: tokens each sequence has had; weights fp32 and
    positions int32 [B, H_KV, at least L_K_max] (-1: where no eviction has placed
    the row); free_pages and taken: da_extend_tables's, to which pages go back.  A
    sequence of more than L_K_max keys stays as it is."""
    dev = k_cache.device
    if not k_cache.is_cuda:
        raise ValueError("k_cache must be on the GPU")
    num_pages, page_size, H_KV, d = _paged_pool("k_cache", k_cache, dev)
    _need("v_cache", v_cache, _BF16, k_cache.shape, dev)
    B = seq_lens.shape[0] if seq_lens.dim() == 1 else 0
    max_pages = _table_args(block_table, seq_lens, B, dev)
    _need("totals", totals, _I32, (B,), dev)
    if weights.dim() != 3:
        raise ValueError("weights must be [B, H_KV, keys]")
    shape = (B, H_KV, weights.shape[2])
    _need("weights", weights, _F32, shape, dev)
    _need("positions", positions, _I32, shape, dev)
    if (free_pages is None) != (taken is None) or (taken_out is not None and taken is None):
        raise ValueError("free_pages and taken go together, and taken_out with them")
    num_free = 0
    if free_pages is not None:
        num_free = _int(free_pages.numel())
        _need("free_pages", free_pages, _I32, (num_free,), dev)
        _need("taken", taken, _I32, (1,), dev)
    outs = []
    for name, t, own, dtype in (("lens_out", lens_out, seq_lens, _I32), ("weights_out", weights_out, weights, _F32),
                                ("positions_out", positions_out, positions, _I32),
                                ("taken_out", taken_out, taken, _I32)):
        if t is None:
            t = own
        else:
            _need(name, t, dtype, own.shape, dev)
        outs.append(t)
    if dev.index != _get_device():
        return _on_device(dev, da_evict_kv, k_cache, v_cache, block_table, seq_lens, totals, weights, positions, budget,
                          L_K_max, sinks=sinks, recent=recent, free_pages=free_pages, taken=taken, lens_out=outs[0],
                          weights_out=outs[1], positions_out=outs[2], taken_out=outs[3], workspace=workspace,
                          stream=stream)
    budget, L = _int(int(budget)), _int(int(L_K_max))
    s_handle = _stream(dev, stream)
    ws, capture = (_usable(workspace, dev), 0) if workspace is not None else _offered_now(dev, stream, s_handle)
    while True:
        rc = load().da_evict_kv(
            k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), totals.data_ptr(),
            weights.data_ptr(), positions.data_ptr(), outs[1].data_ptr(), outs[2].data_ptr(), shape[2], outs[0].data_ptr(),
            _ptr(free_pages), _ptr(taken), _ptr(outs[3]), num_free, B, H_KV, _int(page_size), max_pages, _int(num_pages),
            L, d, budget, _int(int(sinks)), _int(int(recent)), _ptr(ws), _nbytes(ws), s_handle)
        if rc != DA_ERR_WORKSPACE or workspace is not None:
            break
        workspace = ws = _grown(dev, s_handle, capture, da_evict_workspace_bytes(B, H_KV, L, budget))
    if rc:
        _check(rc)
    return tuple(outs)
