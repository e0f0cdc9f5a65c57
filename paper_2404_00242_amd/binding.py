"""ctypes binding over libdeft's C ABI (see include/deft.h).

Argument marshalling only: the plan is built by the library's host code, every
step of the attention path runs in the library's HIP kernels.  PyTorch supplies
device memory and the stream.  There is no fallback: if libdeft.so is missing or
a call fails, an exception is raised.
"""

from __future__ import annotations

import array
import ctypes
import os
import struct
from typing import NamedTuple

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# DEFT_LIB lets a developer point the binding at another build of the same library (A/B timing runs)
LIB_PATH = os.environ.get("DEFT_LIB") or os.path.join(_PKG, "libdeft.so")

DEFT_OUT_BF16 = 0
DEFT_OUT_F32 = 1
# deft_plan flags: how the tree's KV is partitioned and grouped with queries
DEFT_SPLIT_FLATTEN = 0
DEFT_SPLIT_NODE = 1
DEFT_SPLIT_NODE_CHUNK = 2
DEFT_GROUP_QUERY = 3
DEFT_SPLIT_BALANCED = 4  # or rows_per_query(Hq // Hkv) to it
DEFT_PRECISE_WEIGHTS = 0x100  # or-ed to a mode: two-term softmax weights in every group
SPLIT_MODES = {"flatten": DEFT_SPLIT_FLATTEN, "node": DEFT_SPLIT_NODE, "node_chunk": DEFT_SPLIT_NODE_CHUNK,
               "query": DEFT_GROUP_QUERY, "balanced": DEFT_SPLIT_BALANCED}


def rows_per_query(g: int) -> int:
    """DEFT_ROWS_PER_QUERY(g): the flag bits that tell DEFT_SPLIT_BALANCED how many query heads share a KV head"""
    return (int(g) & 0xFFF) << 16

EXPORTS = (
    "deft_plan", "deft_plan_paged", "deft_plan_update", "deft_plan_paged_update", "deft_suggest_chunk_size", "deft_plan_view", "deft_plan_rows", "deft_plan_device_bytes", "deft_plan_upload", "deft_workspace_bytes",
    "deft_tree_attn_decode", "deft_tree_attn_decode_static", "deft_stage1_partial_attention", "deft_stage2_global_reduction",
    "deft_tree_attn_decode_q8", "deft_kv_rows", "deft_kv_copies", "deft_kv_list_device_bytes", "deft_kv_list_upload", "deft_kv_list_destroy",
    "deft_kv_store_q8", "deft_kv_load_q8", "deft_kv_copy_pages", "deft_compact_pages",
    "deft_hbm_read_probe", "deft_plan_destroy", "deft_strerror", "deft_last_hip_error",
)

_i32p = ctypes.POINTER(ctypes.c_int32)
_u64p = ctypes.POINTER(ctypes.c_uint64)

_VIEW_SCALARS = ("chunk_size", "n_nodes", "nq", "n_flat", "n_chunks", "n_segs", "n_slots", "n_mask_words")
# name -> (ctype pointer, length as a function of the scalars)
_VIEW_ARRAYS = (
    ("q_order", _i32p, lambda s: s["nq"]),
    ("node_q_lo", _i32p, lambda s: s["n_nodes"]),
    ("node_q_hi", _i32p, lambda s: s["n_nodes"]),
    ("chunk_seg_ptr", _i32p, lambda s: s["n_chunks"] + 1),
    ("seg_tok_begin", _i32p, lambda s: s["n_segs"]),
    ("seg_len", _i32p, lambda s: s["n_segs"]),
    ("seg_qlo", _i32p, lambda s: s["n_segs"]),
    ("seg_qhi", _i32p, lambda s: s["n_segs"]),
    ("seg_node", _i32p, lambda s: s["n_segs"]),
    ("chunk_qlo", _i32p, lambda s: s["n_chunks"]),
    ("chunk_qhi", _i32p, lambda s: s["n_chunks"]),
    ("chunk_slot_base", _i32p, lambda s: s["n_chunks"] + 1),
    ("seg_mask_ptr", _i32p, lambda s: s["n_segs"] + 1),
    ("seg_mask", _u64p, lambda s: s["n_mask_words"]),
    ("q_part_ptr", _i32p, lambda s: s["nq"] + 1),
    ("q_part_chunk", _i32p, lambda s: s["n_slots"]),
    ("q_part_slot", _i32p, lambda s: s["n_slots"]),
)


class _PlanView(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in _VIEW_SCALARS] + [(n, t) for n, t, _ in _VIEW_ARRAYS]


class DeftError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(what)


_lib = None
_torch = None  # imported by the first call that needs device memory: planning alone does without


def _get_torch():
    global _torch
    if _torch is None:
        import torch

        _torch = torch
    return _torch


def load_library():
    """Loads libdeft.so (built by paper_2404_00242_amd.build); raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2404_00242_amd.build` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, c32, csz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    lib.deft_plan.restype = ctypes.c_int
    # int32 arrays go in as plain addresses (_address): a typed ctypes pointer costs 2 us an array to make
    lib.deft_plan.argtypes = [vp, vp, vp, c32, vp, c32, c32, c32, ctypes.c_uint32, ctypes.POINTER(vp)]
    lib.deft_plan_paged.restype = ctypes.c_int
    lib.deft_plan_paged.argtypes = [vp, vp, c32, c32, vp, vp, c32, vp, c32, c32, ctypes.c_uint32, ctypes.POINTER(vp)]
    lib.deft_plan_update.restype = ctypes.c_int
    lib.deft_plan_update.argtypes = [vp] + lib.deft_plan.argtypes
    lib.deft_plan_paged_update.restype = ctypes.c_int
    lib.deft_plan_paged_update.argtypes = [vp] + lib.deft_plan_paged.argtypes
    lib.deft_suggest_chunk_size.restype = ctypes.c_int32
    lib.deft_suggest_chunk_size.argtypes = [vp, vp, c32, vp, c32, c32, c32, ctypes.c_uint32]
    lib.deft_plan_view.restype = ctypes.c_int
    lib.deft_plan_view.argtypes = [vp, ctypes.POINTER(_PlanView)]
    lib.deft_plan_rows.restype = ctypes.c_int64
    lib.deft_plan_rows.argtypes = [vp]
    lib.deft_plan_device_bytes.restype = csz
    lib.deft_plan_device_bytes.argtypes = [vp, c32, c32]
    lib.deft_plan_upload.restype = ctypes.c_int
    lib.deft_plan_upload.argtypes = [vp, c32, c32, vp, csz, vp]
    lib.deft_workspace_bytes.restype = csz
    lib.deft_workspace_bytes.argtypes = [vp, c32, c32, c32]
    lib.deft_tree_attn_decode.restype = ctypes.c_int
    lib.deft_tree_attn_decode.argtypes = [vp, vp, vp, vp, vp, vp, c32, c32, c32, ctypes.c_float, ctypes.c_uint32,
                                          vp, csz, vp]
    lib.deft_tree_attn_decode_static.restype = ctypes.c_int
    lib.deft_tree_attn_decode_static.argtypes = [vp, vp, vp, vp, vp, vp, c32, c32, c32, ctypes.c_float, ctypes.c_uint32,
                                                 vp]
    lib.deft_stage1_partial_attention.restype = ctypes.c_int
    lib.deft_stage1_partial_attention.argtypes = [vp, vp, vp, vp, vp, c32, c32, c32, ctypes.c_float, vp, csz, vp]
    lib.deft_stage2_global_reduction.restype = ctypes.c_int
    lib.deft_stage2_global_reduction.argtypes = [vp, vp, vp, c32, c32, c32, ctypes.c_float, ctypes.c_uint32, vp, csz,
                                                 vp]
    cache = vp  # (the bytes of a deft_cache_q8_t: _pack_cache)
    lib.deft_tree_attn_decode_q8.restype = ctypes.c_int
    lib.deft_tree_attn_decode_q8.argtypes = [vp, vp, vp, cache, vp, c32, ctypes.c_float, ctypes.c_uint32, vp, csz, vp]
    lib.deft_kv_rows.restype = ctypes.c_int
    lib.deft_kv_rows.argtypes = [vp, c32, c32, c32, ctypes.POINTER(vp)]
    lib.deft_kv_copies.restype = ctypes.c_int
    lib.deft_kv_copies.argtypes = [vp, vp, c32, c32, ctypes.POINTER(vp)]
    lib.deft_kv_list_device_bytes.restype = csz
    lib.deft_kv_list_device_bytes.argtypes = [vp]
    lib.deft_kv_list_upload.restype = ctypes.c_int
    lib.deft_kv_list_upload.argtypes = [vp, vp, csz, vp]
    lib.deft_kv_list_destroy.restype = None
    lib.deft_kv_list_destroy.argtypes = [vp]
    lib.deft_kv_store_q8.restype = ctypes.c_int
    lib.deft_kv_store_q8.argtypes = [vp, vp, vp, vp, ctypes.c_int64, ctypes.c_int64, cache, vp]
    lib.deft_kv_load_q8.restype = ctypes.c_int
    lib.deft_kv_load_q8.argtypes = [vp, vp, cache, vp, vp, vp]
    lib.deft_kv_copy_pages.restype = ctypes.c_int
    lib.deft_kv_copy_pages.argtypes = [vp, vp, vp, vp, c32, vp]
    lib.deft_compact_pages.restype = ctypes.c_int
    lib.deft_compact_pages.argtypes = [vp, vp, c32, vp, c32, vp, vp, vp, ctypes.POINTER(c32)]
    lib.deft_hbm_read_probe.restype = ctypes.c_int
    lib.deft_hbm_read_probe.argtypes = [vp, csz, vp, vp]
    lib.deft_plan_destroy.restype = None
    lib.deft_plan_destroy.argtypes = [vp]
    lib.deft_capture_id.restype = ctypes.c_uint64
    lib.deft_capture_id.argtypes = [vp]
    lib.deft_strerror.restype = ctypes.c_char_p
    lib.deft_strerror.argtypes = [ctypes.c_int]
    lib.deft_last_hip_error.restype = ctypes.c_char_p
    lib.deft_last_hip_error.argtypes = []
    _lib = lib
    return lib


def _check(status: int, what: str):
    if status != 0:
        lib = load_library()
        msg = lib.deft_strerror(status).decode()
        if status == -4:
            msg += " (" + lib.deft_last_hip_error().decode() + ")"
        raise DeftError(status, f"{what}: {msg} [{status}]")


def _i32(x):
    return np.ascontiguousarray(np.asarray(x), dtype=np.int32).reshape(-1)


def _indices(x, what: str):
    """_i32 of whole numbers that int32 holds: others are refused and not cut short."""
    a = np.asarray(x)
    if a.dtype != np.int32 and a.size:
        if a.dtype.kind not in "iu" or int(a.min()) < -(1 << 31) or int(a.max()) >= 1 << 31:
            raise DeftError(-1, f"{what}: rows, pages and tables are whole numbers of 32 bits")
    return _i32(a)


def _size(x, what: str) -> int:
    """A number of rows or pages, the same."""
    n = int(x)
    if not -(1 << 31) <= n < 1 << 31:
        raise DeftError(-1, f"{what}: sizes are whole numbers of 32 bits")
    return n


def _address(x):
    """Address of an _i32 array's data, None for an empty one."""
    return x.__array_interface__["data"][0] if x.size else None


class _Images:
    """Device images of a plan or a list, torch uint8 tensors, by a key.

    An upload only enqueues the copy, on the stream of the call that needs the image first.  An event recorded behind it is kept
    until it has passed, and a call on another stream makes that stream wait for it; the allocator is told of every stream that
    uses the image.  A graph that is captured before the copy has landed uploads an image of its own, once: no eager call may
    use that one, which holds nothing before a replay.  (Of a stream that is itself being captured the runtime does not say
    whether an earlier event has passed.  Its upload came before the capture, and torch.cuda.graph begins one by waiting for the
    device.)"""

    class _Image:
        __slots__ = ("tensor", "event", "first", "streams")  # first: the upload's stream; streams: those that need do nothing more

    def __init__(self):
        self.of = {}  # key, or (key, capture) -> _Image

    def get(self, key, index, raw, capture, nbytes, upload):
        torch = _get_torch()
        x = self.of.get(key)
        own = capture and (x is None or not self._landed(x))
        if own:
            key = key, capture
            x = self.of.get(key)
        on = _torch_stream(raw, index)
        if x is None:
            x = self._Image()
            with torch.cuda.device(index), torch.cuda.stream(on):  # (its memory goes to no other tensor while that stream uses it)
                n = nbytes()
                x.tensor, x.event = torch.empty(n, dtype=torch.uint8, device=torch.device("cuda", index)), torch.cuda.Event()
                upload(x.tensor.data_ptr(), n)
                x.event.record(on)
            x.first, x.streams = raw, {raw}
            self.of[key] = x
        elif raw not in x.streams:
            if own or not self._landed(x):
                on.wait_event(x.event)
            if own or not capture:
                x.streams.add(raw)
            if not capture:
                x.tensor.record_stream(on)
        return x.tensor

    @staticmethod
    def _landed(x):
        if x.event is None or (x.first and _capture(x.first)):
            return True
        if x.event.query():
            x.event = None
        return x.event is None


class Plan:
    """Owns a deft_plan_t handle and, per Hq/Hkv ratio, the device image uploaded for it."""

    def __init__(self, handle, nq=None):
        self._h = handle
        self._images = _Images()  # by (G, device index)
        self._workspaces = {}  # (Hq, Hkv, d, device index, stream, capture) -> torch uint8 tensor
        self._view = None
        self._nq = nq          # queries, and rows a KV cache must have; a plan never changes
        self._rows = None

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.deft_plan_destroy(h)

    @property
    def handle(self):
        return self._h

    def view(self) -> dict:
        """The canonical plan as numpy arrays (copies), keyed like include/deft.h's deft_plan_view_t."""
        if self._view is None:
            v = _PlanView()
            _check(load_library().deft_plan_view(self._h, ctypes.byref(v)), "deft_plan_view")
            out = {n: int(getattr(v, n)) for n in _VIEW_SCALARS}
            for name, ctype, length in _VIEW_ARRAYS:
                n = length(out)
                ptr = getattr(v, name)
                dt = np.uint64 if ctype is _u64p else np.int32
                out[name] = np.ctypeslib.as_array(ptr, shape=(n,)).copy() if n > 0 else np.zeros(0, dtype=dt)
            self._view = out
        return self._view

    def limits(self):
        """(queries of the plan, rows a KV cache must have for it)"""
        if self._rows is None:
            if self._nq is None:
                self._nq = self.view()["nq"]
            self._rows = int(load_library().deft_plan_rows(self._h))
        return self._nq, self._rows

    def device_bytes(self, Hq: int, Hkv: int) -> int:
        return int(load_library().deft_plan_device_bytes(self._h, Hq, Hkv))

    def workspace_bytes(self, Hq: int, Hkv: int, d: int) -> int:
        return int(load_library().deft_workspace_bytes(self._h, Hq, Hkv, d))

    def image(self, Hq: int, Hkv: int, device, stream=None):
        """Device image for this Hq/Hkv ratio, uploaded on first use (memory comes from torch); see _Images.  The plan has to live
        as long as a graph that uses it."""
        torch = _get_torch()
        index = torch.device(device).index
        if index is None:
            index = torch.cuda.current_device()
        raw = _raw_stream(stream, index)
        return self._image(Hq, Hkv, index, raw, _capture(raw) if raw else 0)

    def _image(self, Hq, Hkv, index, raw, capture):
        def nbytes():
            n = self.device_bytes(Hq, Hkv)
            if n == 0:
                raise DeftError(-1, "deft_plan_device_bytes: invalid Hq/Hkv")
            return n

        def upload(at, n):
            _check(_lib.deft_plan_upload(self._h, Hq, Hkv, at, n, raw), "deft_plan_upload")

        return self._images.get((Hq // Hkv, index), index, raw, capture, nbytes, upload)

    def workspace(self, Hq: int, Hkv: int, d: int, device, stream=None):
        """The workspace of calls on a stream (default: torch's current stream).  Calls of two streams may overlap, and so may
        replays of two graphs and eager calls: each stream has a workspace of its own, and each capture on it another, which a
        graph's replays need the plan for."""
        torch = _get_torch()
        index = torch.device(device).index
        if index is None:
            index = torch.cuda.current_device()
        raw = _raw_stream(stream, index)
        return self._workspace(Hq, Hkv, d, index, raw, _capture(raw) if raw else 0)

    def _workspace(self, Hq, Hkv, d, index, raw, capture):
        key = (Hq, Hkv, d, index, raw, capture)
        ws = self._workspaces.get(key)
        if ws is None:
            nbytes = self.workspace_bytes(Hq, Hkv, d)
            if nbytes == 0:
                raise DeftError(-1, "deft_workspace_bytes: invalid head shape")
            torch = _get_torch()
            with torch.cuda.stream(_torch_stream(raw, index)):  # (nothing else is given its memory while that stream uses it)
                ws = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", index))
            self._workspaces[key] = ws
        return ws


def _raw_stream(stream, index: int) -> int:
    """Handle of a stream given as a torch stream, as a handle, or as None: the current stream of device `index`."""
    if stream is None:
        return _get_torch()._C._cuda_getCurrentRawStream(index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _capture(raw: int) -> int:
    """Number of the capture that a stream other than the null stream is in, 0 if it is in none."""
    return load_library().deft_capture_id(raw)


_streams = {}  # (handle, device index) -> torch's object for it


def _torch_stream(raw: int, index: int):
    """The stream of a handle, for torch."""
    stream = _streams.get((raw, index))
    if stream is None:
        cuda = _get_torch().cuda
        stream = _streams[raw, index] = cuda.ExternalStream(raw, device=index) if raw else cuda.default_stream(index)
    return stream


def _result(raw: int, index: int, shape, dtype):
    """Memory for what a call writes on a stream that is not torch's current one: it goes to no tensor of the current stream, and
    comes from none whose work there is still to come.  The caller has it on the current stream, and the allocator is told.  (4 us
    of the host's; a call that is given its output does without.)"""
    torch = _get_torch()
    if _elsewhere(index):
        with torch.cuda.device(index):
            return _result(raw, index, shape, dtype)
    on = _torch_stream(raw, index)
    # (as torch.cuda.stream does it, 4 us less)
    here, set_stream = torch._C._cuda_getCurrentStream(index), torch._C._cuda_setStream
    set_stream(stream_id=on.stream_id, device_index=on.device_index, device_type=on.device_type)
    try:
        out = torch.empty(shape, dtype=dtype, device=on.device)
    finally:
        set_stream(stream_id=here[0], device_index=here[1], device_type=here[2])
    out.record_stream(_torch_stream(torch._C._cuda_getCurrentRawStream(index), index))
    return out


def deft_suggest_chunk_size(node_tok_len, node_parent, query_node, Hq: int, Hkv: int, flags: int = 0) -> int:
    """Chunk size S_t suited to this tree for the split named by flags (about two equal stage-1 tasks per
    compute unit)."""
    nl, par, qn = _i32(node_tok_len), _i32(node_parent), _i32(query_node)
    rc = load_library().deft_suggest_chunk_size(_address(nl), _address(par), nl.size, _address(qn), qn.size, int(Hq),
                                                int(Hkv), int(flags))
    if rc < 0:
        _check(rc, "deft_suggest_chunk_size")
    return int(rc)


def deft_plan(node_tok_begin, node_tok_len, node_parent, query_node, ntok: int, chunk_size: int = 0,
              flags: int = 0, prev: "Plan | None" = None) -> Plan:
    """QKV Preparation Phase (Algorithm 3): builds the flattened chunk / bit-mask plan on the host.
    prev: the plan of an earlier version of the tree (deft_plan_update: same result, less work)."""
    lib = load_library()
    nb, nl, par, qn = _i32(node_tok_begin), _i32(node_tok_len), _i32(node_parent), _i32(query_node)
    if not (nb.size == nl.size == par.size):
        raise DeftError(-1, "deft_plan: node table columns differ in length")
    out = ctypes.c_void_p()
    args = (_address(nb), _address(nl), _address(par), nb.size, _address(qn), qn.size, int(ntok), int(chunk_size),
            int(flags), ctypes.byref(out))
    if prev is None:
        _check(lib.deft_plan(*args), "deft_plan")
    else:
        _check(lib.deft_plan_update(prev.handle, *args), "deft_plan_update")
    return Plan(out, qn.size)


def deft_plan_paged(node_page_ptr, page_ids, page_size: int, n_pool_pages: int, node_tok_len, node_parent,
                    query_node, chunk_size: int = 0, flags: int = 0, prev: "Plan | None" = None) -> Plan:
    """QKV Preparation Phase over a paged KV pool (K/V are [n_pool_pages * page_size, Hkv, d]).
    prev: the plan of an earlier version of the tree (deft_plan_paged_update: same result, less work)."""
    lib = load_library()
    pp, pg, nl, par, qn = (_i32(x) for x in (node_page_ptr, page_ids, node_tok_len, node_parent, query_node))
    if not (nl.size == par.size == pp.size - 1):
        raise DeftError(-1, "deft_plan_paged: node table columns differ in length")
    out = ctypes.c_void_p()
    args = (_address(pp), _address(pg), int(page_size), int(n_pool_pages), _address(nl), _address(par), nl.size,
            _address(qn), qn.size, int(chunk_size), int(flags), ctypes.byref(out))
    if prev is None:
        _check(lib.deft_plan_paged(*args), "deft_plan_paged")
    else:
        _check(lib.deft_plan_paged_update(prev.handle, *args), "deft_plan_paged_update")
    return Plan(out, qn.size)


KV_STAGGER_BYTES = 512  # V pool's base relative to the K pool's, modulo 1 KiB


def alloc_kv_cache(n_rows: int, Hkv: int, d: int, device="cuda"):
    """Uninitialised K and V pools [n_rows, Hkv, d] (bf16), carved from one allocation so that the V pool
    starts KV_STAGGER_BYTES past a 1 KiB boundary and the K pool on one.

    Placement only, no arithmetic: on MI355X a compute unit reads fastest when the rows it has in flight
    differ in address bits 7..9.  K and V rows of one head sit at the same offset of their pools, so with
    both pools on the same alignment every row a workgroup streams shares those bits; half a KiB between
    the pools' alignments spreads them (measured on the few-shot benchmark: stage 1 30.5 -> 29.4 us).
    Any 16-byte aligned K and V are accepted by the kernels; this is merely the fast layout."""
    import torch

    pool = n_rows * Hkv * d * 2
    k_span = -(-pool // 1024) * 1024
    buf = torch.empty(1024 + k_span + KV_STAGGER_BYTES + pool, dtype=torch.uint8, device=device)
    k_off = (-buf.data_ptr()) % 1024
    v_off = k_off + k_span + KV_STAGGER_BYTES
    k = buf[k_off:k_off + pool].view(torch.bfloat16).view(n_rows, Hkv, d)
    v = buf[v_off:v_off + pool].view(torch.bfloat16).view(n_rows, Hkv, d)
    return k, v


def deft_tree_attn_decode(plan: Plan, q, k, v, out=None, scale: float = 0.0, out_dtype=None, workspace=None,
                          stream=None):
    """Attention Calculation Phase (Algorithm 4) on the GPU.

    q [nq,Hq,d], k/v [ntok,Hkv,d]: contiguous bf16 CUDA(HIP) tensors.  Returns o [nq,Hq,d] (bf16, or
    float32 when out_dtype / out says so), in the caller's query order.  Asynchronous on `stream`
    (default: torch's current stream); the current stream has to wait for another one before it reads o.
    """
    torch = _torch or _get_torch()
    bf16 = torch.bfloat16
    if not (q.is_cuda and k.is_cuda and v.is_cuda):
        raise DeftError(-1, "deft_tree_attn_decode: q, k, v must be device tensors (there is no CPU path)")
    if not (q.dtype == k.dtype == v.dtype == bf16 and q.dim() == k.dim() == v.dim() == 3 and q.is_contiguous()
            and k.is_contiguous() and v.is_contiguous()):
        for name, t in (("q", q), ("k", k), ("v", v)):
            if t.dtype != bf16 or not t.is_contiguous() or t.dim() != 3:
                raise DeftError(-1, f"deft_tree_attn_decode: {name} must be a contiguous 3-d bf16 tensor")
    nq, Hq, d = q.shape
    ntok, Hkv, d2 = shape = k.shape
    if v.shape != shape or d2 != d:
        raise DeftError(-1, "deft_tree_attn_decode: k and v must both be [ntok, Hkv, d]")
    plan_nq, plan_rows = plan.limits()
    if nq != plan_nq:
        raise DeftError(-1, "deft_tree_attn_decode: q has a different number of queries than the plan")
    if plan_rows > ntok:
        raise DeftError(-1, "deft_tree_attn_decode: the plan addresses rows beyond the KV cache")
    dev = q.device
    index = dev.index
    raw = _raw_stream(stream, index)
    if out is None and stream is not None and raw != torch._C._cuda_getCurrentRawStream(index):
        out = _result(raw, index, (nq, Hq, d), out_dtype or bf16)
    elif out is None:
        # (empty_like costs half a microsecond less than naming shape, type and device; its format is named because a q of one
        # query, sliced from a wider tensor, is contiguous under strides that the output should not have; of a q that is a
        # subclass of Tensor it would make another)
        dense = torch.contiguous_format
        if type(q) is not torch.Tensor:
            out = torch.empty((nq, Hq, d), dtype=out_dtype or bf16, device=dev)
        elif out_dtype is None or out_dtype == bf16:
            out = torch.empty_like(q, memory_format=dense)
        else:
            out = torch.empty_like(q, dtype=out_dtype, memory_format=dense)
    elif out.shape != (nq, Hq, d) or not out.is_contiguous() or out.device != dev:
        raise DeftError(-1, "deft_tree_attn_decode: out must be a contiguous [nq, Hq, d] tensor on q's device")
    if out.dtype == bf16:
        flags = DEFT_OUT_BF16
    elif out.dtype == torch.float32:
        flags = DEFT_OUT_F32
    else:
        raise DeftError(-1, "deft_tree_attn_decode: out must be bf16 or float32")
    capture = _capture(raw) if raw else 0
    image = plan._images.of.get((Hq // Hkv, index))
    img = image.tensor if image is not None and not capture and raw in image.streams else plan._image(Hq, Hkv, index, raw, capture)
    ws = workspace
    if ws is None:
        ws = plan._workspaces.get((Hq, Hkv, d, index, raw, capture))
        if ws is None:
            ws = plan._workspace(Hq, Hkv, d, index, raw, capture)
    rc = (_lib or load_library()).deft_tree_attn_decode(
        plan._h, img.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), Hq, Hkv, d, float(scale), flags,
        ws.data_ptr(), ws.numel() * ws.element_size(), raw)
    if rc != 0:
        _check(rc, "deft_tree_attn_decode")
    return out


# ---- the cache in 8 bits ----

MAX_BLOCK_ROWS = 64
_BLOCK_ROWS = (1, 2, 4, 8, 16, 32, 64)
MIN_SCALE_BYTE = 10  # the smallest scale, 2^(10 - 127): of blocks that hold nothing yet


class CacheQ8(NamedTuple):
    """A KV cache in 8-bit floating point (see deft_cache_q8_t): a row's K and V are its e4m3 values times the scale of its
    block of `block_rows` rows and of the KV head, a power of two.  `alloc_kv_cache_q8` makes one."""

    k: "torch.Tensor"        # float8_e4m3fn [n_rows, Hkv, d]
    v: "torch.Tensor"
    k_scale: "torch.Tensor"  # float8_e8m0fnu [ceil(n_rows / block_rows), Hkv], beginning at a multiple of 4 bytes
    v_scale: "torch.Tensor"
    block_rows: int = 32


def alloc_kv_cache_q8(n_rows: int, Hkv: int, d: int, block_rows: int = 32, device="cuda") -> CacheQ8:
    """An empty 8-bit cache.  `block_rows` is a power of two up to 64.  A block must belong to one node, since a store takes the
    rows of a block behind those that it writes for empty and may change their scale: choose pages of a multiple of it, with a
    contiguous cache begin nodes at multiples of it or take 1.  K and V come from one allocation and are staggered as in alloc_kv_cache."""
    import torch

    if block_rows < 1 or block_rows > MAX_BLOCK_ROWS or block_rows & (block_rows - 1):
        raise DeftError(-1, f"alloc_kv_cache_q8: block_rows must be a power of two up to {MAX_BLOCK_ROWS}")
    pool, blocks = n_rows * Hkv * d, -(-n_rows // block_rows)
    k_span = -(-pool // 1024) * 1024
    buf = torch.empty(1024 + k_span + KV_STAGGER_BYTES + pool, dtype=torch.uint8, device=device)
    k_off = (-buf.data_ptr()) % 1024
    v_off = k_off + k_span + KV_STAGGER_BYTES
    k, v = (buf[off:off + pool].view(torch.float8_e4m3fn).view(n_rows, Hkv, d) for off in (k_off, v_off))
    scales = [torch.full((blocks, Hkv), MIN_SCALE_BYTE, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu) for _ in range(2)]
    return CacheQ8(k, v, *scales, block_rows)


_pack_cache = struct.Struct("4P4i").pack  # deft_cache_q8_t


def _cache_args(cache: CacheQ8, what: str):
    """(a deft_cache_q8_t, its device's index, n_rows, Hkv, d) of a cache that is one."""
    torch = _torch or _get_torch()
    k, v, ks, vs, block = cache
    block = int(block)
    index = k.get_device()
    if index < 0 or not index == v.get_device() == ks.get_device() == vs.get_device():
        raise DeftError(-1, f"{what}: the cache must be on one device (there is no CPU path)")
    shape = k.shape
    if not (k.dtype == v.dtype == torch.float8_e4m3fn and len(shape) == 3 and v.shape == shape and k.is_contiguous() and v.is_contiguous()):
        raise DeftError(-1, f"{what}: k and v of the cache must both be contiguous [n_rows, Hkv, d] float8_e4m3fn tensors")
    if not 0 < block <= MAX_BLOCK_ROWS or block & (block - 1):
        raise DeftError(-1, f"{what}: block_rows must be a power of two up to {MAX_BLOCK_ROWS}")
    n_rows, Hkv, d = shape
    if n_rows >= 1 << 31 or Hkv >= 1 << 31 or d >= 1 << 31:
        raise DeftError(-1, f"{what}: a cache's sizes are whole numbers of 32 bits")
    blocks = ks.shape
    if not (ks.dtype == vs.dtype == torch.float8_e8m0fnu and blocks == vs.shape and blocks == (-(-n_rows // block), Hkv) and ks.is_contiguous()
            and vs.is_contiguous()):
        raise DeftError(-1, f"{what}: the scales must both be contiguous [ceil(n_rows / block_rows), Hkv] float8_e8m0fnu tensors")
    ksp, vsp = ks.data_ptr(), vs.data_ptr()
    if (ksp | vsp) & 3:
        raise DeftError(-1, f"{what}: the scales must begin at a multiple of 4 bytes")
    return _pack_cache(k.data_ptr(), v.data_ptr(), ksp, vsp, n_rows, Hkv, d, block), index, n_rows, Hkv, d


def _elsewhere(index: int) -> bool:
    """Whether the current device is another one: a call then makes its tensors' device the current one, and starts again."""
    return (_torch or _get_torch())._C._cuda_getDevice() != index


class KVList:
    """Owns a deft_kv_list_t handle (cache rows or copies of pages) and its device images.  Like a plan it is made once for
    the calls of all layers."""

    def __init__(self, handle, n: int, pool: int, block_rows: int = 0):
        self._h = handle
        self._images = _Images()  # by device index
        self.n, self.pool, self.block_rows = n, pool, block_rows

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.deft_kv_list_destroy(h)

    @property
    def handle(self):
        return self._h

    def image(self, device, stream=None):
        """Device image of the list, uploaded on first use; see _Images.  The list has to live as long as a graph that uses it."""
        torch = _torch or _get_torch()
        index = torch.device(device).index
        if index is None:
            index = torch.cuda.current_device()
        return self._image(index, _raw_stream(stream, index))

    def _image(self, index: int, raw: int):
        capture = _capture(raw) if raw else 0
        image = self._images.of.get(index)
        if image is not None and not capture and raw in image.streams:
            return image.tensor

        def upload(at, n):
            _check(_lib.deft_kv_list_upload(self._h, at, n, raw), "deft_kv_list_upload")

        return self._images.get(index, index, raw, capture, lambda: int(load_library().deft_kv_list_device_bytes(self._h)), upload)


def deft_kv_rows(rows, n_pool_rows: int, block_rows: int = 32) -> KVList:
    """The rows of an 8-bit cache that tokens 0, 1, ... go to or come from, for deft_kv_store_q8 and deft_kv_load_q8."""
    r, pool, block = _indices(rows, "deft_kv_rows"), _size(n_pool_rows, "deft_kv_rows"), _size(block_rows, "deft_kv_rows")
    out = ctypes.c_void_p()
    _check(load_library().deft_kv_rows(_address(r), r.size, pool, block, ctypes.byref(out)), "deft_kv_rows")
    return KVList(out, r.size, pool, block)


def deft_kv_copies(src, dst, n_pool_pages: int) -> KVList:
    """Copies of pages for deft_kv_copy_pages: page dst[i] becomes what page src[i] held, for all i at once."""
    a, b, pool = _indices(src, "deft_kv_copies"), _indices(dst, "deft_kv_copies"), _size(n_pool_pages, "deft_kv_copies")
    if a.size != b.size:
        raise DeftError(-1, "deft_kv_copies: src and dst differ in length")
    out = ctypes.c_void_p()
    _check(load_library().deft_kv_copies(_address(a), _address(b), a.size, pool, ctypes.byref(out)), "deft_kv_copies")
    return KVList(out, a.size, pool)


def deft_compact_pages(node_page_ptr, page_ids, n_pool_pages: int, node_parent):
    """(new page_ids, src, dst): the copies that put every node's pages in a row, nodes depth-first, from page 0 on."""
    pp, pg, par = (_indices(x, "deft_compact_pages") for x in (node_page_ptr, page_ids, node_parent))
    if pp.size != par.size + 1 or (pp.size and int(pp[-1]) != pg.size):
        raise DeftError(-1, "deft_compact_pages: tables differ in length")
    new, src, dst = (np.zeros(max(1, pg.size), dtype=np.int32) for _ in range(3))
    n = ctypes.c_int32()
    _check(load_library().deft_compact_pages(_address(pp), _address(pg), _size(n_pool_pages, "deft_compact_pages"), _address(par), par.size, _address(new), _address(src),
                                             _address(dst), ctypes.byref(n)), "deft_compact_pages")
    return new[:pg.size], src[:n.value], dst[:n.value]


def _rows_for(rows: KVList, cache: CacheQ8, what: str):
    args = _cache_args(cache, what)
    if rows.block_rows != cache.block_rows or rows.pool > args[2]:
        raise DeftError(-1, f"{what}: the list is one of copies, or for a larger cache or other blocks")
    return args


def deft_kv_store_q8(rows: KVList, k, v, cache: CacheQ8, stream=None) -> None:
    """Stores the K and V of new tokens, bf16 [n, Hkv, d], into the rows of the list.  Tokens may lie apart (slices of a fused
    projection's output), by a multiple of 16 bytes; the heads of one may not.  A block is filled from its first row on: rows of it
    behind the lowest one written, other than those of the list, hold nothing afterwards.  Asynchronous on `stream`."""
    torch = _torch or _get_torch()
    c, index, _, Hkv, d = _rows_for(rows, cache, "deft_kv_store_q8")
    n, bf16, strides = rows.n, torch.bfloat16, []
    shape = (n, Hkv, d)
    for t in (k, v):
        if t.dtype != bf16 or t.shape != shape or t.get_device() != index:
            raise DeftError(-1, f"deft_kv_store_q8: k and v must be bf16 [{n}, {Hkv}, {d}] tensors on the cache's device")
        token, head, one = t.stride()
        if n and (one != 1 or (Hkv > 1 and head != d)):
            raise DeftError(-1, "deft_kv_store_q8: the heads of a token must be contiguous")
        strides.append(token if n > 1 else Hkv * d)  # (one token's stride says nothing)
    if n == 0:
        return
    if _elsewhere(index):
        with torch.cuda.device(index):
            return deft_kv_store_q8(rows, k, v, cache, stream)
    raw = _raw_stream(stream, index)
    rc = _lib.deft_kv_store_q8(rows._h, rows._image(index, raw).data_ptr(), k.data_ptr(), v.data_ptr(), strides[0], strides[1], c, raw)
    if rc != 0:
        _check(rc, "deft_kv_store_q8")


def deft_kv_load_q8(rows: KVList, cache: CacheQ8, k=None, v=None, stream=None):
    """(k, v), bf16 [n, Hkv, d]: the values of the list's rows.  Asynchronous on `stream`; the current stream has to wait for
    another one before it reads them."""
    torch = _torch or _get_torch()
    c, index, _, Hkv, d = _rows_for(rows, cache, "deft_kv_load_q8")
    shape, bf16 = (rows.n, Hkv, d), torch.bfloat16
    raw = _raw_stream(stream, index)
    elsewhere = stream is not None and raw != torch._C._cuda_getCurrentRawStream(index)
    if k is None:
        k = _result(raw, index, shape, bf16) if elsewhere else torch.empty(shape, dtype=bf16, device=cache.k.device)
    elif k.dtype != bf16 or k.shape != shape or not k.is_contiguous() or k.get_device() != index:
        raise DeftError(-1, f"deft_kv_load_q8: k must be a contiguous bf16 [{rows.n}, {Hkv}, {d}] tensor on the cache's device")
    if v is None:
        v = _result(raw, index, shape, bf16) if elsewhere else torch.empty(shape, dtype=bf16, device=cache.k.device)
    elif v.dtype != bf16 or v.shape != shape or not v.is_contiguous() or v.get_device() != index:
        raise DeftError(-1, f"deft_kv_load_q8: v must be a contiguous bf16 [{rows.n}, {Hkv}, {d}] tensor on the cache's device")
    if rows.n == 0:
        return k, v
    if _elsewhere(index):
        with torch.cuda.device(index):
            return deft_kv_load_q8(rows, cache, k, v, stream)
    rc = _lib.deft_kv_load_q8(rows._h, rows._image(index, raw).data_ptr(), c, k.data_ptr(), v.data_ptr(), raw)
    if rc != 0:
        _check(rc, "deft_kv_load_q8")
    return k, v


def deft_kv_copy_pages(copies: KVList, pools, stream=None, page_size=None) -> None:
    """Makes the copies of the list in every pool, in place.  pools: CacheQ8s, whose pages have to be whole blocks, and contiguous
    device tensors of any type, each the n_pool_pages pages of one K or V cache, or of an 8-bit cache's scales.  How many rows a
    page has follows from a pool's size; with page_size it is checked (a first dimension of n_pool_pages * page_size rows, or of their
    blocks' scales).  Asynchronous on `stream`."""
    if copies.block_rows:
        raise DeftError(-1, "deft_kv_copy_pages: the list is one of rows, not of copies")
    pages, pools = copies.pool, list(pools)
    if CacheQ8 in map(type, pools):
        pools = [x for t in pools for x in (_pages_of_cache(t, pages, page_size) if type(t) is CacheQ8 else (t,))]
    if not pools:
        return
    e8m0 = (_torch or _get_torch()).float8_e8m0fnu
    if page_size is not None or e8m0 in [t.dtype for t in pools]:
        for t in pools:
            _check_pool(t, pages, page_size, t.dtype is e8m0 and t.dim() == 2)
    sizes = [t.nbytes for t in pools]
    for nbytes in set(sizes):
        if pages == 0 or nbytes == 0 or nbytes % pages:
            raise DeftError(-1, "deft_kv_copy_pages: a pool is not a whole number of bytes for each of the list's pages")
    index, *others = {t.get_device() for t in pools}
    if others or index < 0 or not all([t.is_contiguous() for t in pools]):
        raise DeftError(-1, "deft_kv_copy_pages: pools must be contiguous tensors on one device (there is no CPU path)")
    if _elsewhere(index):
        with (_torch or _get_torch()).cuda.device(index):
            return deft_kv_copy_pages(copies, pools, stream)
    raw = _raw_stream(stream, index)
    at, per_page = array.array("Q", [t.data_ptr() for t in pools]), array.array("q", [n // pages for n in sizes])
    rc = load_library().deft_kv_copy_pages(copies._h, copies._image(index, raw).data_ptr(), at.buffer_info()[0], per_page.buffer_info()[0], len(pools), raw)
    if rc != 0:
        _check(rc, "deft_kv_copy_pages")


def _pages_of_cache(cache: CacheQ8, pages: int, page_size):
    """A cache's four pools, where it is that many pages of whole blocks."""
    rows = _cache_args(cache, "deft_kv_copy_pages")[2]
    if pages == 0 or rows % pages or rows // pages % cache.block_rows or (page_size is not None and rows != pages * page_size):
        raise DeftError(-1, "deft_kv_copy_pages: a cache is not a whole number of blocks for each of the list's pages, or of other pages")
    return cache[:4]


def _check_pool(t, pages: int, page_size, scales: bool):
    rows = t.shape[0] if t.dim() else 0
    if scales:  # [blocks, Hkv]
        whole = pages > 0 and rows > 0 and rows % pages == 0
        if not whole or (page_size is not None and (pages * page_size % rows or pages * page_size // rows not in _BLOCK_ROWS)):
            raise DeftError(-1, "deft_kv_copy_pages: scales are not a whole number of blocks for each of the list's pages, or of other pages")
    elif page_size is not None and rows != pages * page_size:
        raise DeftError(-1, f"deft_kv_copy_pages: a pool's first dimension is not that of {pages} pages of {page_size} rows")


def deft_tree_attn_decode_q8(plan: Plan, q, cache: CacheQ8, out=None, scale: float = 0.0, out_dtype=None, workspace=None, stream=None):
    """deft_tree_attn_decode over an 8-bit cache.

    q [nq,Hq,d]: contiguous bf16.  Returns o [nq,Hq,d] (bf16, or float32 when out_dtype / out says so: then with softmax weights
    in two terms throughout).  Asynchronous on `stream` (default: torch's current stream); the current stream has to wait for
    another one before it reads o.
    """
    torch = _torch or _get_torch()
    bf16 = torch.bfloat16
    c, index, n_rows, Hkv, d = _cache_args(cache, "deft_tree_attn_decode_q8")
    if q.dtype != bf16 or q.dim() != 3 or not q.is_contiguous() or q.get_device() != index:
        raise DeftError(-1, "deft_tree_attn_decode_q8: q must be a contiguous 3-d bf16 tensor on the cache's device")
    shape = nq, Hq, dq = q.shape
    if dq != d:
        raise DeftError(-1, "deft_tree_attn_decode_q8: q and the cache differ in d")
    if Hkv == 0 or Hq == 0 or Hq % Hkv:
        raise DeftError(-1, "deft_tree_attn_decode_q8: Hq must be a multiple of Hkv")
    plan_nq, plan_rows = plan.limits()
    if nq != plan_nq:
        raise DeftError(-1, "deft_tree_attn_decode_q8: q has a different number of queries than the plan")
    if plan_rows > n_rows:
        raise DeftError(-1, "deft_tree_attn_decode_q8: the plan addresses rows beyond the KV cache")
    raw = _raw_stream(stream, index)
    if out is None and stream is not None and raw != torch._C._cuda_getCurrentRawStream(index):
        out = _result(raw, index, shape, out_dtype or bf16)
    elif out is None:  # (see deft_tree_attn_decode)
        if type(q) is torch.Tensor and (out_dtype is None or out_dtype == bf16):
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        else:
            out = torch.empty(shape, dtype=out_dtype or bf16, device=q.device)
    elif out.shape != shape or not out.is_contiguous() or out.get_device() != index:
        raise DeftError(-1, "deft_tree_attn_decode_q8: out must be a contiguous [nq, Hq, d] tensor on q's device")
    if out.dtype == bf16:
        flags = DEFT_OUT_BF16
    elif out.dtype == torch.float32:
        flags = DEFT_OUT_F32
    else:
        raise DeftError(-1, "deft_tree_attn_decode_q8: out must be bf16 or float32")
    if _elsewhere(index):
        with torch.cuda.device(index):
            return deft_tree_attn_decode_q8(plan, q, cache, out, scale, None, workspace, stream)
    capture = _capture(raw) if raw else 0
    image = plan._images.of.get((Hq // Hkv, index))
    img = image.tensor if image is not None and not capture and raw in image.streams else plan._image(Hq, Hkv, index, raw, capture)
    ws = workspace
    if ws is None:
        ws = plan._workspaces.get((Hq, Hkv, d, index, raw, capture))
        if ws is None:
            ws = plan._workspace(Hq, Hkv, d, index, raw, capture)
    rc = (_lib or load_library()).deft_tree_attn_decode_q8(
        plan._h, img.data_ptr(), q.data_ptr(), c, out.data_ptr(), Hq, float(scale), flags, ws.data_ptr(), ws.numel() * ws.element_size(), raw)
    if rc != 0:
        _check(rc, "deft_tree_attn_decode_q8")
    return out
