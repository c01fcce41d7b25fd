"""Binding of libgkv.so: the same names as include/gkv.h, argument marshalling only (by ctypes; a decode step's calls by the
extension csrc/gkv_call.cpp).

Every step of the path runs in the CUDA kernels behind the C ABI.  PyTorch is used for device
memory (the arena, inputs, outputs) and for the current CUDA stream.  If the library is missing
or a CUDA device is needed and absent, calls fail loudly; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np
import torch

from . import build as _build

GKV_ABI_VERSION = 1
POLICY_STAIRCASE, POLICY_RD, POLICY_EXTERNAL = 0, 1, 2
REDUCE_MAX, REDUCE_SUM = 0, 1
TENSOR_K, TENSOR_V = 0, 1
OK = 0
ERR_INVALID_ARG, ERR_ARENA_TOO_SMALL, ERR_CTX_FULL, ERR_BAD_STATE, ERR_UNSUPPORTED = -1, -2, -3, -4, -5
ERR_RANGE, ERR_BUDGET, ERR_CUDA = -6, -7, -8

EXPORTS = [
    "gkv_query_arena_bytes", "gkv_create", "gkv_destroy", "gkv_release_host_memory", "gkv_append_demote", "gkv_decode_attn",
    "gkv_decode_attn_observe", "gkv_debug_export_mass", "gkv_debug_export_bounds", "gkv_rd_reallocate", "gkv_debug_device_plan",
    "gkv_debug_replan_levels",
    "gkv_quest_select", "gkv_quest_select_static", "gkv_debug_export_boxes", "gkv_debug_export_scores", "gkv_bits_report",
    "gkv_debug_export_block", "gkv_debug_export_residual", "gkv_debug_export_units",
    "gkv_prompt_attn", "gkv_prompt_workspace_bytes", "gkv_prompt_mass", "gkv_chunk_attn", "gkv_chunk_workspace_bytes",
    "gkv_debug_export_levels", "gkv_debug_plan_levels", "gkv_ctx_len", "gkv_strerror", "gkv_last_cuda_error",
]


class GkvConfig(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("abi_version", C.c_uint32),
        ("n_layers", C.c_int32), ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("d_k", C.c_int32), ("d_v", C.c_int32), ("v_aliases_k", C.c_int32), ("max_ctx", C.c_int32),
        ("block_tokens", C.c_int32), ("group", C.c_int32), ("page_tokens", C.c_int32), ("policy", C.c_int32),
        ("stair_tokens", C.c_int32 * 4), ("n_sink_blocks", C.c_int32), ("retire_after", C.c_int32),
        ("rd_budget_bpv", C.c_float), ("residual_fraction", C.c_float), ("quest_reduce", C.c_int32),
        ("monotone_in_age", C.c_int32), ("softmax_scale", C.c_float),
    ]


class GkvBits(C.Structure):
    _fields_ = [
        ("values", C.c_uint64), ("code_bits", C.c_uint64), ("param_bits", C.c_uint64), ("exact_bits", C.c_uint64),
        ("centroid_bits", C.c_uint64), ("tail_bits", C.c_uint64), ("residual_bits", C.c_uint64),
        ("residual_index_bits", C.c_uint64), ("box_bits", C.c_uint64), ("resident_bits", C.c_uint64),
        ("meta_bits", C.c_uint64), ("last_read_bits", C.c_uint64), ("blocks_by_level", C.c_uint64 * 5),
        ("bpv_resident", C.c_double), ("bpv_paper", C.c_double), ("bpv_read", C.c_double),
    ]


class GkvPrompt(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("abi_version", C.c_uint32),
        ("n_seqs", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("offsets", C.c_void_p),
        ("q_stride", C.c_int64), ("k_stride", C.c_int64), ("v_stride", C.c_int64), ("out_stride", C.c_int64),
        ("softmax_scale", C.c_float),
    ]


class GkvError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status} ({strerror(status)})")
        self.status = status


_lib = None
_call = None       # the extension that makes a decode step's calls (csrc/gkv_call.cpp)


def lib_path() -> str:
    return os.path.join(os.path.dirname(os.path.abspath(__file__)), "libgkv.so")


def load():
    """Load libgkv.so and the extension (building them is the job of ``build()`` / ``__graft_entry__.build``)."""
    global _lib, _call
    if _lib is not None:
        return _lib
    for path in (lib_path(), _build.CALL_LIB):
        if not os.path.exists(path):
            raise FileNotFoundError(f"{path} is missing: run `python -m paper_2608_23599_b200.build` first")
    lib = C.CDLL(lib_path())
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    lib.gkv_query_arena_bytes.argtypes = [C.POINTER(GkvConfig), C.POINTER(sz)]
    lib.gkv_create.argtypes = [C.POINTER(GkvConfig), vp, sz, C.POINTER(vp)]
    lib.gkv_destroy.argtypes = [vp]
    lib.gkv_release_host_memory.argtypes = [C.POINTER(sz)]
    lib.gkv_append_demote.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp]
    lib.gkv_decode_attn.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp]
    lib.gkv_decode_attn_observe.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp]
    lib.gkv_debug_export_bounds.argtypes = [vp, i32, vp]
    lib.gkv_debug_export_mass.argtypes = [vp, i32, vp]
    lib.gkv_rd_reallocate.argtypes = [vp, i32, vp]
    lib.gkv_debug_device_plan.argtypes = [vp, i32, vp, vp, vp, vp]
    lib.gkv_debug_replan_levels.argtypes = [C.POINTER(GkvConfig), i32, i32, C.POINTER(C.c_float), C.POINTER(C.c_float),
                                            C.POINTER(C.c_int8), C.POINTER(C.c_int8), C.POINTER(i32)]
    lib.gkv_quest_select.argtypes = [vp, i32, vp, i32, vp, C.POINTER(i32), vp]
    lib.gkv_debug_export_boxes.argtypes = [vp, i32, i32, i32, vp, vp, i32, C.POINTER(i32)]
    lib.gkv_debug_export_scores.argtypes = [vp, i32, vp, vp, vp]
    lib.gkv_quest_select_static.argtypes = [vp, i32, vp, i32, vp, C.POINTER(i32), vp]
    lib.gkv_chunk_attn.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.gkv_chunk_workspace_bytes.argtypes = [vp, i32, i32, C.POINTER(sz)]
    lib.gkv_prompt_attn.argtypes = [C.POINTER(GkvPrompt), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.gkv_prompt_workspace_bytes.argtypes = [C.POINTER(GkvPrompt), C.POINTER(sz)]
    lib.gkv_prompt_mass.argtypes = [C.POINTER(GkvPrompt), vp, vp, vp, i32, vp, vp]
    lib.gkv_bits_report.argtypes = [vp, i32, C.POINTER(GkvBits)]
    lib.gkv_debug_export_block.argtypes = [vp, i32, i32, i32, i32, i32, C.POINTER(i32), vp, vp, vp, vp, C.POINTER(i32)]
    lib.gkv_debug_export_residual.argtypes = [vp, i32, i32, i32, vp, i32, C.POINTER(i32)]
    lib.gkv_debug_export_units.argtypes = [vp, i32, vp, i32, C.POINTER(i32)]
    lib.gkv_debug_export_levels.argtypes = [vp, i32, i32, i32, vp, i32, C.POINTER(i32)]
    lib.gkv_debug_plan_levels.argtypes = [C.POINTER(GkvConfig), i32, i32, C.POINTER(C.c_float), C.POINTER(C.c_float),
                                          C.POINTER(C.c_int8), C.POINTER(i32)]
    lib.gkv_ctx_len.argtypes = [vp, i32, C.POINTER(i32)]
    lib.gkv_strerror.argtypes = [C.c_int]
    lib.gkv_strerror.restype = C.c_char_p
    lib.gkv_last_cuda_error.argtypes = [vp]
    for name in EXPORTS:
        if name != "gkv_strerror":
            getattr(lib, name).restype = C.c_int
    from . import _gkv_call
    _gkv_call.bind(*(C.cast(f, vp).value for f in (lib.gkv_append_demote, lib.gkv_decode_attn, lib.gkv_decode_attn_observe,
                                                   lib.gkv_quest_select)), vp)
    _gkv_call.bind_rows(*(C.cast(f, vp).value for f in (lib.gkv_prompt_attn, lib.gkv_prompt_workspace_bytes, lib.gkv_prompt_mass, lib.gkv_chunk_attn)),
                        torch.Tensor, torch.bfloat16, torch.float32, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream,
                        torch._C._cuda_isCurrentStreamCapturing)
    _lib, _call = lib, _gkv_call
    return lib


def _loaded():
    load()
    return _call


def strerror(status: int) -> str:
    return load().gkv_strerror(status).decode()


def make_config(n_layers, batch, n_q_heads, n_kv_heads, d_k, d_v, max_ctx, *, v_aliases_k=0, page_tokens=0,
                policy=POLICY_STAIRCASE, stair_tokens=(-1, 0, 0, 0), n_sink_blocks=0, retire_after=0,
                rd_budget_bpv=0.0, residual_fraction=0.0, quest_reduce=REDUCE_MAX, monotone_in_age=1,
                softmax_scale=0.0) -> GkvConfig:
    cfg = GkvConfig()
    cfg.struct_size = C.sizeof(GkvConfig)
    cfg.abi_version = GKV_ABI_VERSION
    cfg.n_layers, cfg.batch, cfg.n_q_heads, cfg.n_kv_heads = n_layers, batch, n_q_heads, n_kv_heads
    cfg.d_k, cfg.d_v, cfg.v_aliases_k, cfg.max_ctx = d_k, d_v, v_aliases_k, max_ctx
    cfg.block_tokens, cfg.group, cfg.page_tokens, cfg.policy = 64, 32, page_tokens, policy
    cfg.stair_tokens = (C.c_int32 * 4)(*stair_tokens)
    cfg.n_sink_blocks, cfg.retire_after = n_sink_blocks, retire_after
    cfg.rd_budget_bpv, cfg.residual_fraction = rd_budget_bpv, residual_fraction
    cfg.quest_reduce, cfg.monotone_in_age, cfg.softmax_scale = quest_reduce, monotone_in_age, softmax_scale
    return cfg


def config_from_workload(w, n_layers: Optional[int] = None) -> GkvConfig:
    return make_config(n_layers or w.n_layers, w.batch, w.n_q_heads, w.n_kv_heads, w.d_k, w.d_v, w.max_ctx,
                       v_aliases_k=w.v_aliases_k, page_tokens=w.page_tokens, policy=w.policy,
                       stair_tokens=tuple(w.stair_tokens), n_sink_blocks=w.n_sink_blocks,
                       retire_after=w.retire_after, rd_budget_bpv=w.rd_budget_bpv,
                       residual_fraction=w.residual_fraction, quest_reduce=getattr(w, "quest_reduce", REDUCE_MAX),
                       softmax_scale=w.softmax_scale)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    return t if isinstance(t, int) else t.data_ptr()


def _stream() -> int:
    # torch.cuda.current_stream().cuda_stream without the Stream object in between
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(rc: int, what: str, allow=()):
    if rc != OK and rc not in allow:
        raise GkvError(rc, what)
    return rc


def gkv_query_arena_bytes(cfg: GkvConfig) -> int:
    out = C.c_size_t(0)
    _check(load().gkv_query_arena_bytes(C.byref(cfg), C.byref(out)), "gkv_query_arena_bytes")
    return out.value


def gkv_release_host_memory() -> int:
    """Frees the page-locked host memory that closed caches have left for later ones; returns the bytes."""
    out = C.c_size_t(0)
    _check(load().gkv_release_host_memory(C.byref(out)), "gkv_release_host_memory")
    return out.value


def gkv_debug_plan_levels(cfg: GkvConfig, n_closed: int, n_tail: int = 0, mass=None, rng=None):
    """Host-only level plan of one stream (no device needed): (levels int8 [n_closed], budget_miss)."""
    levels = np.zeros(max(n_closed, 1), dtype=np.int8)
    miss = C.c_int32(0)
    fp = C.POINTER(C.c_float)
    m = None if mass is None else np.ascontiguousarray(mass, dtype=np.float32)
    r = None if rng is None else np.ascontiguousarray(rng, dtype=np.float32)
    _check(load().gkv_debug_plan_levels(C.byref(cfg), n_closed, n_tail,
                                        None if m is None else m.ctypes.data_as(fp),
                                        None if r is None else r.ctypes.data_as(fp),
                                        levels.ctypes.data_as(C.POINTER(C.c_int8)), C.byref(miss)),
           "gkv_debug_plan_levels")
    return levels[:n_closed], bool(miss.value)


def gkv_debug_replan_levels(cfg: GkvConfig, n_tail: int, mass, rng, prev):
    """Host-only plan of a decode-time re-allocation of one stream: (levels int8 [n_closed], budget_miss)."""
    m = np.ascontiguousarray(mass, dtype=np.float32)
    r = np.ascontiguousarray(rng, dtype=np.float32)
    pv = np.ascontiguousarray(prev, dtype=np.int8)
    n = len(pv)
    levels = np.zeros(n, dtype=np.int8)
    miss = C.c_int32(0)
    fp, bp = C.POINTER(C.c_float), C.POINTER(C.c_int8)
    _check(load().gkv_debug_replan_levels(C.byref(cfg), n, n_tail, m.ctypes.data_as(fp), r.ctypes.data_as(fp),
                                          pv.ctypes.data_as(bp), levels.ctypes.data_as(bp), C.byref(miss)),
           "gkv_debug_replan_levels")
    return levels, bool(miss.value)


def _rows(t, name, dtype, shape=None):
    """A tensor [rows][heads][128] whose heads follow one another; returns the distance of its rows."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda or t.dim() != 3 or t.shape[2] != 128:
        raise ValueError(f"{name}: a CUDA {dtype} tensor [rows][heads][128] is needed")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.numel() and (t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != 128)):
        raise ValueError(f"{name}: the heads of a row have to follow one another")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1] * 128:
        raise ValueError(f"{name}: rows that share memory")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * 128


def _floats(t, name, n, shape=None):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.numel() < n or (
            shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name}: a contiguous CUDA float32 tensor {list(shape) if shape is not None else [n]} is needed")


def _ints(x, name):
    a = np.asarray(x)
    if a.size and (a.dtype.kind not in "iu" or a.min() < -2 ** 31 or a.max() >= 2 ** 31):
        raise ValueError(f"{name}: whole numbers of 32 bits are needed")
    return np.ascontiguousarray(a, dtype=np.int32)


def _keep_space(spaces, key, kept):
    """Keeps a stream's workspace, of at most four streams (the memory of the oldest goes back to torch's allocator, in the order of its stream)."""
    spaces.pop(key, None)
    while len(spaces) >= 4:
        spaces.pop(next(iter(spaces)))
    spaces[key] = kept


def _prompt(q, k, offsets, softmax_scale, *more):
    off = _ints(offsets, "offsets")
    if off.ndim != 1 or off.size < 1:
        raise ValueError("offsets: n_seqs + 1 row numbers are needed")
    if off[-1] > q.shape[0]:
        raise ValueError(f"offsets: end at row {off[-1]} of {q.shape[0]}")
    if any(t is not None and t.device != q.device for t in (k, *more)):
        raise ValueError("all tensors have to be on one device")
    d = GkvPrompt()
    d.struct_size, d.abi_version = C.sizeof(GkvPrompt), GKV_ABI_VERSION
    d.n_seqs, d.n_q_heads, d.n_kv_heads, d.head_dim = off.size - 1, q.shape[1], k.shape[1], q.shape[2]
    d.offsets, d.softmax_scale = off.ctypes.data, softmax_scale
    return d, off


def _on(device, call):
    """call(stream) with `device` current, on its current stream."""
    if device.index == torch._C._cuda_getDevice():
        return call(_stream())
    with torch.cuda.device(device):
        return call(_stream())


_prompt_spaces = {}      # workspaces of prompt attention, one per stream (whose calls follow one another)


def _prompt_space(device, need):
    """(address, bytes, owner): the stream's workspace, or, while it is captured, memory of the graph's own."""
    with torch.cuda.device(device):
        key = 64 * _stream() + device.index
        captured = torch._C._cuda_isCurrentStreamCapturing()
        kept = None if captured else _prompt_spaces.get(key)
        if kept is None or kept[1] < need:
            kept = None
            if not captured:                 # (the small one goes before the large one comes)
                _prompt_spaces.pop(key, None)
            t = torch.empty(need, dtype=torch.uint8, device=device)
            kept = t.data_ptr(), need, t
            if not captured:
                _keep_space(_prompt_spaces, key, kept)
    return kept


def gkv_prompt_attn(q, k, v, out, offsets, lse=None, softmax_scale=0.0):
    """Causal attention of packed prompts: q, out cuda bf16 [rows][n_q_heads][128], k, v cuda bf16 [rows][n_kv_heads][128]
    (rows may be slices of a fused projection), offsets: host row numbers, sequence s = rows [offsets[s], offsets[s + 1]);
    lse: cuda fp32 [rows][n_q_heads] or None.  Rows of no sequence are left as they are; a sequence's own values have to be finite."""
    rc = (_call or _loaded()).prompt_attn(q, k, v, out, offsets, lse, softmax_scale, _prompt_spaces)
    if rc is not NotImplemented and rc > 0:      # bytes of workspace
        rc = _call.prompt_attn(q, k, v, out, offsets, lse, softmax_scale, _prompt_space(q.device, rc))
    if rc == OK:
        return rc
    if rc is not NotImplemented:
        return _check(rc, "gkv_prompt_attn")
    qs, ks = _rows(q, "q", torch.bfloat16), _rows(k, "k", torch.bfloat16)
    vs, os_ = _rows(v, "v", torch.bfloat16, k.shape), _rows(out, "out", torch.bfloat16, q.shape)
    if k.shape[0] != q.shape[0]:
        raise ValueError(f"k: {k.shape[0]} rows, not {q.shape[0]}")
    if lse is not None:
        _floats(lse, "lse", 0, q.shape[:2])
    d, _keep = _prompt(q, k, offsets, softmax_scale, v, out, lse)
    d.q_stride, d.k_stride, d.v_stride, d.out_stride = qs, ks, vs, os_
    need = C.c_size_t(0)
    _check(load().gkv_prompt_workspace_bytes(C.byref(d), C.byref(need)), "gkv_prompt_workspace_bytes")

    def call(st):
        ws = _prompt_space(q.device, need.value) if need.value else (None, 0)
        return load().gkv_prompt_attn(C.byref(d), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), ws[0], ws[1], st)
    rc = _on(q.device, call)
    return rc if rc == OK else _check(rc, "gkv_prompt_attn")


def gkv_prompt_mass(q, k, lse, mass, offsets, n_obs, softmax_scale=0.0):
    """Attention masses of prompt tokens under the newest n_obs queries of their sequence: q, k, offsets as for
    gkv_prompt_attn, lse the log-sum-exp that it wrote; mass: cuda fp32, [n_kv_heads][length] sequence after sequence (for
    sequences of one length the token_mass that gkv_append_demote takes)."""
    rc = (_call or _loaded()).prompt_mass(q, k, lse, mass, mass.dim() if isinstance(mass, torch.Tensor) else 0, offsets, n_obs, softmax_scale)
    if rc == OK:
        return rc
    if rc is not NotImplemented:
        return _check(rc, "gkv_prompt_mass")
    qs, ks = _rows(q, "q", torch.bfloat16), _rows(k, "k", torch.bfloat16)
    if k.shape[0] != q.shape[0]:
        raise ValueError(f"k: {k.shape[0]} rows, not {q.shape[0]}")
    _floats(lse, "lse", 0, q.shape[:2])
    d, off = _prompt(q, k, offsets, softmax_scale, lse, mass)
    _floats(mass, "mass", int(off[-1] - off[0]) * k.shape[1])
    d.q_stride, d.k_stride = qs, ks
    rc = _on(q.device, lambda st: load().gkv_prompt_mass(C.byref(d), _ptr(q), _ptr(k), _ptr(lse), n_obs, _ptr(mass), st))
    return rc if rc == OK else _check(rc, "gkv_prompt_mass")


class Cache:
    """Owner of a gkv_cache handle and of the torch arena behind it."""

    def __init__(self, cfg: GkvConfig, arena_bytes: Optional[int] = None, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("gkv needs a CUDA device: there is no CPU fallback")
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = gkv_query_arena_bytes(cfg) if arena_bytes is None else arena_bytes
        self.arena = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.arena.data_ptr()
        self._arena_ptr = (base + 255) // 256 * 256
        h = C.c_void_p()
        _check(load().gkv_create(C.byref(cfg), self._arena_ptr, nbytes, C.byref(h)), "gkv_create")
        self.handle = h
        self._chunk_spaces = {}

    def close(self):
        self._chunk_spaces = {}
        if getattr(self, "handle", None):
            load().gkv_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    stream_handle = None   # set to a cudaStream_t (int) to skip the per-call look-up of torch's current stream

    def _st(self) -> int:
        return self.stream_handle if self.stream_handle is not None else _stream()

    def gkv_append_demote(self, layer, k_new, v_new, token_mass=None, level_plan=None, n_new=None):
        """k_new/v_new: cuda bf16 [B][n_new][Hkv][d]; token_mass cuda fp32 [B][Hkv][n_new];
        level_plan: host int8 numpy [B][Hkv][n_new // 64].  Device buffers may be given as tensors or as
        plain integer device addresses (then pass n_new): a serving loop that calls once per layer and step
        keeps its addresses instead of building tensor views."""
        if n_new is None:
            n_new = k_new.shape[1]
        plan_ptr = None
        if level_plan is not None:
            self._plan_keep = level_plan = level_plan.astype("int8", copy=False)
            plan_ptr = level_plan.ctypes.data
        rc = _call.append(self.handle, layer, k_new, v_new, n_new, token_mass, plan_ptr, self._st())
        if rc is NotImplemented:
            rc = load().gkv_append_demote(self.handle, layer, _ptr(k_new), _ptr(v_new), n_new, _ptr(token_mass), plan_ptr, self._st())
        return rc if rc == OK else _check(rc, "gkv_append_demote", allow=(ERR_RANGE, ERR_BUDGET))

    def gkv_decode_attn(self, layer, q, out, lse=None, page_idx=None, n_sel=0):
        rc = _call.decode(self.handle, layer, q, page_idx, n_sel, out, lse, self._st())
        if rc is NotImplemented:
            rc = load().gkv_decode_attn(self.handle, layer, _ptr(q), _ptr(page_idx), n_sel, _ptr(out), _ptr(lse), self._st())
        return rc if rc == OK else _check(rc, "gkv_decode_attn")

    def gkv_decode_attn_observe(self, layer, q, out, lse=None, block_mass=None, certificate=None):
        """Full-context decode that also observes the attention mass of every block and updates the
        cache's running masses (block_mass: device fp32 [batch][n_kv_heads][ceil(ctx / 64)] or None;
        certificate: device fp32 [batch][n_q_heads] or None, the error certificate of this query)."""
        rc = _call.observe(self.handle, layer, q, out, lse, block_mass, certificate, self._st())
        if rc is NotImplemented:
            rc = load().gkv_decode_attn_observe(self.handle, layer, _ptr(q), _ptr(out), _ptr(lse), _ptr(block_mass),
                                                _ptr(certificate), self._st())
        return rc if rc == OK else _check(rc, "gkv_decode_attn_observe")

    def gkv_chunk_workspace_bytes(self, layer, n_new) -> int:
        n = C.c_size_t(0)
        _check(load().gkv_chunk_workspace_bytes(self.handle, layer, n_new, C.byref(n)), "gkv_chunk_workspace_bytes")
        return n.value

    def gkv_chunk_attn(self, layer, q, k_new, v_new, out, lse=None, lengths=None, workspace=None):
        """Attention of n_new new tokens per sequence over the cache and, causally, over one another; the cache stays as it is.
        q, out: cuda bf16 [B][n_new][Hq][128]; k_new, v_new: cuda bf16 [B][n_new][Hkv][128]; lse: cuda fp32 [B][n_new][Hq] or
        None; lengths: host ints [B] (rows from there on are left as they are) or None; workspace: a cuda tensor of
        gkv_chunk_workspace_bytes bytes, or None (one per stream is kept; a captured call has one of its graph's own)."""
        cfg = self.cfg
        ws, keep = (workspace, None) if workspace is not None else self._chunk_workspace(layer, q)
        if isinstance(ws, torch.Tensor):
            ws = (ws.data_ptr(), ws.numel() * ws.element_size()) if ws.device == self.arena.device and ws.is_contiguous() else None
        if ws is not None:
            rc = _call.chunk(self.handle, layer, q, k_new, v_new, out, lse, lengths, ws[0], ws[1], cfg.batch, cfg.n_q_heads, cfg.n_kv_heads,
                             self.stream_handle, self.arena.device.index)
            if rc == OK:
                return rc
            if rc is not NotImplemented:
                return _check(rc, "gkv_chunk_attn")
        # the long way: names what is wrong, takes lengths of any kind, and a device that is not the current one
        b, hq, hkv, dev = cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, self.arena.device
        n = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 4 else 0
        for t, name, h, dt in ((q, "q", hq, torch.bfloat16), (k_new, "k_new", hkv, torch.bfloat16), (v_new, "v_new", hkv, torch.bfloat16),
                               (out, "out", hq, torch.bfloat16), (lse, "lse", hq, torch.float32)):
            if t is None and name == "lse":
                continue
            shape = (b, n, h) if name == "lse" else (b, n, h, 128)
            if not isinstance(t, torch.Tensor) or tuple(t.shape) != shape or t.dtype != dt or t.device != dev or not t.is_contiguous():
                raise ValueError(f"{name}: a contiguous {dt} tensor {list(shape)} on {dev} is needed")
        if ws is None:
            raise ValueError(f"workspace: a contiguous tensor on {dev} is needed")
        ln = None
        if lengths is not None:
            ln = _ints(lengths, "lengths")
            if ln.shape != (b,):
                raise ValueError(f"lengths: {b} of them are needed")

        def call(st):
            return load().gkv_chunk_attn(self.handle, layer, _ptr(q), _ptr(k_new), _ptr(v_new), n, None if ln is None else ln.ctypes.data,
                                         _ptr(out), _ptr(lse), ws[0], ws[1], st if self.stream_handle is None else self.stream_handle)
        rc = _on(dev, call)
        return rc if rc == OK else _check(rc, "gkv_chunk_attn")

    def _chunk_workspace(self, layer, q):
        """(address, bytes) of a workspace for a chunk like q, and its owner.  One is kept per stream, whose calls follow one another; a captured
        call gets memory of its graph's own."""
        n = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 4 else 0
        if n == 0:
            return (None, 0), None
        need = self.gkv_chunk_workspace_bytes(layer, n)
        dev, handle = self.arena.device, self.stream_handle
        st = torch._C._cuda_getCurrentRawStream(dev.index) if handle is None else handle
        capturing = torch._C._cuda_isCurrentStreamCapturing()
        if handle is not None and handle != torch._C._cuda_getCurrentRawStream(dev.index):
            with torch.cuda.stream(torch.cuda.ExternalStream(handle, device=dev)):
                if torch._C._cuda_isCurrentStreamCapturing():
                    raise ValueError("workspace: a call that is captured on a stream other than torch's has to bring its own")
            capturing = False
        kept = None if capturing else self._chunk_spaces.get(st)
        if kept is None or kept[0][1] < need:
            kept = None
            if not capturing:                # (the small one goes before the large one comes)
                self._chunk_spaces.pop(st, None)
            with torch.cuda.device(dev):
                if handle is None:
                    t = torch.empty(need, dtype=torch.uint8, device=dev)
                else:      # memory that is free again in the order of the stream that uses it
                    with torch.cuda.stream(torch.cuda.ExternalStream(handle, device=dev)):
                        t = torch.empty(need, dtype=torch.uint8, device=dev)
            kept = (t.data_ptr(), need), t
            if not capturing:
                _keep_space(self._chunk_spaces, st, kept)
        return kept

    def gkv_debug_export_bounds(self, layer):
        """Per-block certificate bounds as numpy [batch][n_kv_heads][n_closed][4] (kappa, delta, max |v|, 0)."""
        n = self.gkv_ctx_len(layer) // 64
        out = np.zeros((self.cfg.batch, self.cfg.n_kv_heads, n, 4), dtype=np.float32)
        _check(load().gkv_debug_export_bounds(self.handle, layer, out.ctypes.data_as(C.c_void_p)), "gkv_debug_export_bounds")
        return out

    def gkv_debug_device_plan(self, layer):
        """(levels int8, mass fp32, range fp32) as numpy [batch][n_kv_heads][n_closed]: the plan the device
        allocator makes now and the numbers it was made from; flag: a stream missed the budget."""
        n = self.gkv_ctx_len(layer) // 64
        shp = (self.cfg.batch, self.cfg.n_kv_heads, n)
        lv, ms, rg = np.zeros(shp, np.int8), np.zeros(shp, np.float32), np.zeros(shp, np.float32)
        rc = load().gkv_debug_device_plan(self.handle, layer, lv.ctypes.data_as(C.c_void_p), ms.ctypes.data_as(C.c_void_p),
                                          rg.ctypes.data_as(C.c_void_p), self._st())
        _check(rc, "gkv_debug_device_plan", allow=(ERR_BUDGET,))
        return lv, ms, rg, rc == ERR_BUDGET

    def gkv_rd_reallocate(self, layer):
        """Decode-time re-allocation of an RD-policy layer from the running block masses."""
        return _check(load().gkv_rd_reallocate(self.handle, layer, self._st()), "gkv_rd_reallocate",
                      allow=(ERR_RANGE, ERR_BUDGET))

    def gkv_debug_export_mass(self, layer):
        """Running block masses of a layer as a numpy array [batch][n_kv_heads][ceil(ctx / 64)]."""
        n_items = (self.gkv_ctx_len(layer) + 63) // 64
        out = np.zeros((self.cfg.batch, self.cfg.n_kv_heads, n_items), dtype=np.float32)
        _check(load().gkv_debug_export_mass(self.handle, layer, out.ctypes.data_as(C.c_void_p)), "gkv_debug_export_mass")
        return out

    def gkv_debug_export_boxes(self, layer, b, kv_head):
        """Page boxes of one stream: (lo, hi) uint16 arrays [n_pages][d_k] of bf16 bits."""
        page = self.cfg.page_tokens
        cap = (self.gkv_ctx_len(layer) // 64) * (64 // page) if page > 0 else 0
        lo = np.zeros((max(cap, 1), self.cfg.d_k), dtype=np.uint16)
        hi = np.zeros((max(cap, 1), self.cfg.d_k), dtype=np.uint16)
        n = C.c_int32(0)
        _check(load().gkv_debug_export_boxes(self.handle, layer, b, kv_head, lo.ctypes.data_as(C.c_void_p),
                                             hi.ctypes.data_as(C.c_void_p), cap, C.byref(n)), "gkv_debug_export_boxes")
        return lo[: n.value], hi[: n.value]

    def gkv_debug_export_scores(self, layer, q):
        """Page scores of every stream for query q: float32 [batch][n_kv_heads][n_pages]."""
        page = self.cfg.page_tokens
        n_pages = (self.gkv_ctx_len(layer) // 64) * (64 // page) if page > 0 else 0
        out = np.zeros((self.cfg.batch, self.cfg.n_kv_heads, n_pages), dtype=np.float32)
        _check(load().gkv_debug_export_scores(self.handle, layer, _ptr(q), out.ctypes.data_as(C.c_void_p), self._st()),
               "gkv_debug_export_scores")
        return out

    def gkv_quest_select(self, layer, q, budget_tokens, page_idx_out) -> int:
        res = _call.select(self.handle, layer, q, budget_tokens, page_idx_out, self._st())
        if res is NotImplemented:
            n = C.c_int32(0)
            rc = load().gkv_quest_select(self.handle, layer, _ptr(q), budget_tokens, _ptr(page_idx_out), C.byref(n), self._st())
            res = rc, n.value
        if res[0] != OK:
            _check(res[0], "gkv_quest_select")
        return res[1]

    def gkv_quest_select_static(self, layer, q, budget_tokens, page_idx_out) -> int:
        """gkv_quest_select with its score scratch in the library's fixed device array: for callers
        that must not trigger any device allocation.  Same arguments and results."""
        n = C.c_int32(0)
        _check(load().gkv_quest_select_static(self.handle, layer, _ptr(q), budget_tokens, _ptr(page_idx_out),
                                              C.byref(n), self._st()), "gkv_quest_select_static")
        return n.value

    def gkv_bits_report(self, layer=-1) -> GkvBits:
        out = GkvBits()
        # the warnings (a saturated or oversized scale, a missed budget) do not fail the call; the last one is kept
        self.last_report_status = _check(load().gkv_bits_report(self.handle, layer, C.byref(out)), "gkv_bits_report",
                                         allow=(ERR_RANGE, ERR_BUDGET))
        return out

    def gkv_ctx_len(self, layer) -> int:
        n = C.c_int32(0)
        _check(load().gkv_ctx_len(self.handle, layer, C.byref(n)), "gkv_ctx_len")
        return n.value

    def gkv_debug_export_levels(self, layer, b, kv_head):
        import numpy as np
        cap = (self.cfg.max_ctx + 63) // 64
        lv = np.zeros(cap, dtype=np.int8)
        n = C.c_int32(0)
        _check(load().gkv_debug_export_levels(self.handle, layer, b, kv_head, lv.ctypes.data, cap, C.byref(n)),
               "gkv_debug_export_levels")
        return lv[: n.value].astype(np.int32)

    def gkv_debug_export_residual(self, layer, b, kv_head):
        import numpy as np
        cap = self.cfg.max_ctx
        idx = np.zeros(cap, dtype=np.int32)
        n = C.c_int32(0)
        _check(load().gkv_debug_export_residual(self.handle, layer, b, kv_head, idx.ctypes.data, cap, C.byref(n)),
               "gkv_debug_export_residual")
        return idx[: n.value]

    def gkv_debug_export_units(self, layer):
        """Work lists of the last full read: int32 [n][6] of (warp, head group, first item, tile mask, run, cost)."""
        n = C.c_int32(0)
        _check(load().gkv_debug_export_units(self.handle, layer, None, 0, C.byref(n)), "gkv_debug_export_units", allow=(ERR_INVALID_ARG,))
        out = np.zeros((n.value, 6), dtype=np.int32)
        _check(load().gkv_debug_export_units(self.handle, layer, out.ctypes.data, n.value, C.byref(n)), "gkv_debug_export_units")
        return out

    def gkv_debug_export_block(self, layer, b, kv_head, block, which):
        """Returns dict(level, codes u8 [64][d], scale/zero uint16 fp16 bits, rows uint16 bf16 bits, n_rows)."""
        import numpy as np
        d = self.cfg.d_k if which == TENSOR_K else self.cfg.d_v
        codes = np.zeros((64, d), dtype=np.uint8)
        npar = 2 * d if which == TENSOR_K else 64 * (d // 32)
        scale = np.zeros(npar, dtype=np.uint16)
        zero = np.zeros(npar, dtype=np.uint16)
        rows = np.zeros((64, d), dtype=np.uint16)
        level = C.c_int32(0)
        n_rows = C.c_int32(0)
        _check(load().gkv_debug_export_block(self.handle, layer, b, kv_head, block, which, C.byref(level),
                                             codes.ctypes.data, scale.ctypes.data, zero.ctypes.data,
                                             rows.ctypes.data, C.byref(n_rows)), "gkv_debug_export_block")
        shape = (2, d) if which == TENSOR_K else (64, d // 32)
        return dict(level=level.value, codes=codes, scale=scale.reshape(shape), zero=zero.reshape(shape),
                    rows=rows, n_rows=n_rows.value)


def build(force: bool = False, verbose: bool = False) -> str:
    return _build.build(force=force, verbose=verbose)
