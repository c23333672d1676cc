"""ctypes binding of libqevict.so (include/qevict.h), same names as the C ABI.

Argument marshalling only: every step of the decode path runs in the HIP
kernels of the library.  PyTorch supplies device memory (the workspace and the
tensors) and the HIP stream.  Importing this module does not need a GPU;
creating a cache does, and there is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import dataclasses
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqevict.so")

ABI_VERSION = 4
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_BAD_STATE, ERR_NONFINITE, \
    ERR_CAPACITY, ERR_DEVICE = 0, -1, -2, -3, -4, -5, -6, -7
TIER_UNUSED, TIER_OPEN, TIER_FULL, TIER_QUANT, TIER_EVICTED = 0, 1, 2, 3, 4
LEDGER_NONE, LEDGER_ACTIVE, LEDGER_DORMANT = 0, 1, 2
BITS_MIXED_4_2 = 42
OUT_F32, OUT_BF16 = 0, 1
FLAG_NO_PROMOTION, FLAG_DEBUG_MASSES, FLAG_ASYNC_ROUTING = 0x1, 0x2, 0x4
FLAG_ROUTING_QUEUE_WAIT, FLAG_ROUTING_DEVICE_WAIT = 0x8, 0x10
KERNEL_ATTEND, KERNEL_MERGE, KERNEL_RETIER, KERNEL_MIGRATE = range(4)
SCORE_CUMULATIVE, SCORE_DECAY, SCORE_KEY_NORM, SCORE_PNORM = 0, 1, 2, 3
BLOCK_TOKENS = 64
INT32_MAX = 2 ** 31 - 1

# exported symbols declared in include/qevict.h
SYMBOLS = (
    "qevict_workspace_size", "qevict_cache_init", "qevict_cache_destroy", "qevict_prefill_assign",
    "qevict_decode_attend", "qevict_retier", "qevict_quantize_window", "qevict_promote_window",
    "qevict_get_state", "qevict_export_window", "qevict_debug_shift_keys", "qevict_debug_masses",
    "qevict_debug_last_masses", "qevict_debug_routing_gate", "qevict_routing_order",
    "qevict_profile_enable", "qevict_profile_read", "qevict_last_attend_bytes", "qevict_join_routing",
    "qevict_status_string", "qevict_last_error", "qevict_prefill_scores_scratch_size",
    "qevict_prefill_scores", "qevict_capacities_for_budget", "qevict_memory_report",
    "qevict_prefill_scores_noalloc", "qevict_prompt_attend", "qevict_block_store", "qevict_block_fetch",
    "qevict_block_workspace_size", "qevict_block_attend",
)


class QEvictError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"qevict status {status}: {message}")
        self.status = status


class _Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "abi_version", "batch", "num_layers", "num_q_heads", "num_kv_heads", "head_dim",
        "window_tokens", "group_size", "quant_bits", "sink_tokens", "recent_tokens", "max_context",
        "capacity_full", "capacity_quant", "retier_interval", "out_dtype")] + [
        ("flags", ctypes.c_uint32), ("softmax_scale", ctypes.c_float), ("num_splits", ctypes.c_int32),
        ("score_mode", ctypes.c_int32), ("score_decay", ctypes.c_float), ("score_p", ctypes.c_float),
        ("rope_base", ctypes.c_float)]


class _PromptConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "abi_version", "num_seqs", "total_tokens", "num_q_heads", "num_kv_heads", "head_dim")] + [
        ("softmax_scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
            "q_token_stride", "q_head_stride", "k_token_stride", "k_head_stride", "v_token_stride",
            "v_head_stride", "out_token_stride", "out_head_stride")]


class _BlockConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "abi_version", "batch", "num_q_heads", "num_kv_heads", "head_dim", "max_context", "num_pages")] + [
        ("softmax_scale", ctypes.c_float)]


class _BlockLayer(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "lens")]


class MemoryReport(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "sink", "recent", "full", "quant_codes", "quant_meta", "position", "ledger", "total")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class RetierStats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "promotions", "admissions_full", "first_quantizations", "reactivations", "evictions",
        "n_full", "n_quant_int4", "n_quant_int2")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


@dataclasses.dataclass
class Config:
    batch: int
    num_q_heads: int
    num_kv_heads: int
    window_tokens: int
    quant_bits: int
    max_context: int
    capacity_full: int
    capacity_quant: int
    num_layers: int = 1
    head_dim: int = 128
    group_size: int = 0          # 0: window_tokens (32 for 8-token windows)
    sink_tokens: int = 0
    recent_tokens: int = 0
    retier_interval: int = 1
    out_dtype: int = OUT_F32
    flags: int = 0
    softmax_scale: float = 0.0
    num_splits: int = 0
    score_mode: int = SCORE_CUMULATIVE
    score_decay: float = 0.0
    score_p: float = 0.0
    rope_base: float = 0.0

    def to_c(self) -> _Config:
        c = _Config()
        c.abi_version = ABI_VERSION
        for f in dataclasses.fields(self):
            setattr(c, f.name, getattr(self, f.name))
        if not self.group_size:   # the value group: 32 channels for 8-token windows, else W
            c.group_size = 32 if self.window_tokens == 8 else self.window_tokens
        return c


_lib = None


def load_library(path: str | None = None):
    """Load libqevict.so (built in-tree); raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with `python -m paper_2608_05326_amd.build`")
    # torch carries its own HIP runtime: load it first so that the library binds
    # to the runtime torch's device memory and streams come from (loaded the
    # other way round, creating a cache fails with "no ROCm-capable device")
    import torch  # noqa: F401
    lib = ctypes.CDLL(p)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    P = ctypes.POINTER
    sig = {
        "qevict_workspace_size": [P(_Config), P(ctypes.c_size_t)],
        "qevict_cache_init": [P(_Config), vp, ctypes.c_size_t, vp, P(vp)],
        "qevict_cache_destroy": [vp],
        "qevict_prefill_assign": [vp, i32, vp, vp, i32, vp],
        "qevict_decode_attend": [vp, i32, vp, vp, vp, vp],
        "qevict_retier": [vp, i32, P(RetierStats)],
        "qevict_quantize_window": [vp, i32, i32, i32],
        "qevict_promote_window": [vp, i32, i32, i32],
        "qevict_get_state": [vp, i32, i32, vp, vp, vp, vp, i32, P(i32)],
        "qevict_export_window": [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp],
        "qevict_debug_shift_keys": [vp, i32, i32, i32, vp],
        "qevict_debug_masses": [vp, i32, vp, i32],
        "qevict_debug_last_masses": [vp, i32, vp],
        "qevict_debug_routing_gate": [vp, i64, i32],
        "qevict_routing_order": [vp, P(i32)],
        "qevict_profile_enable": [vp, i32],
        "qevict_profile_read": [vp, i32, P(ctypes.c_double), P(i64)],
        "qevict_last_attend_bytes": [vp, i32, P(i64)],
        "qevict_join_routing": [vp],
        "qevict_prefill_scores_scratch_size": [P(_Config), i32, i32, P(ctypes.c_size_t)],
        "qevict_prefill_scores": [vp, vp, i32, vp, i32, vp, ctypes.c_size_t, vp],
        "qevict_capacities_for_budget": [P(_Config), i64, i32, P(i32), P(i32)],
        "qevict_memory_report": [vp, i32, i32, P(MemoryReport)],
        "qevict_prefill_scores_noalloc": [vp, vp, i32, vp, i32, vp],
        "qevict_prompt_attend": [P(_PromptConfig), vp, vp, vp, vp, vp, vp],
        "qevict_block_store": [P(_BlockConfig), P(_BlockLayer), vp, i64, i64, vp, i64, i64, vp, i32, vp],
        "qevict_block_fetch": [P(_BlockConfig), P(_BlockLayer), vp, i64, i64, vp, i64, i64, vp, i32, vp],
        "qevict_block_workspace_size": [P(_BlockConfig), P(ctypes.c_size_t)],
        "qevict_block_attend": [P(_BlockConfig), P(_BlockLayer), vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = i32
    lib.qevict_status_string.argtypes = [i32]
    lib.qevict_status_string.restype = ctypes.c_char_p
    lib.qevict_last_error.argtypes = []
    lib.qevict_last_error.restype = ctypes.c_char_p
    if path is None:
        _lib = lib
    return lib


def _check(lib, status: int):
    if status != OK:
        raise QEvictError(status, lib.qevict_last_error().decode())


def workspace_size(cfg: Config) -> int:
    lib = load_library()
    n = ctypes.c_size_t()
    _check(lib, lib.qevict_workspace_size(ctypes.byref(cfg.to_c()), ctypes.byref(n)))
    return n.value


def capacities_for_budget(cfg: Config, budget_bytes: int, q_permille: int) -> tuple[int, int]:
    """(K_f, K_q) from a per-layer, per-sequence byte budget and quantized share q (thousandths)."""
    lib = load_library()
    kf, kq = ctypes.c_int32(), ctypes.c_int32()
    _check(lib, lib.qevict_capacities_for_budget(ctypes.byref(cfg.to_c()), budget_bytes, q_permille,
                                                 ctypes.byref(kf), ctypes.byref(kq)))
    return kf.value, kq.value


def prefill_scores_scratch_size(cfg: Config, prompt_len: int, n_obs: int) -> int:
    lib = load_library()
    n = ctypes.c_size_t()
    _check(lib, lib.qevict_prefill_scores_scratch_size(ctypes.byref(cfg.to_c()), prompt_len, n_obs,
                                                       ctypes.byref(n)))
    return n.value


def _ptr(t, torch_dtype=None, name="tensor", shape=None):
    """Device address of a contiguous tensor; with `shape`, the tensor must hold
    exactly that many elements (the kernels read and write whole extents)."""
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    if torch_dtype is not None and t.dtype != torch_dtype:
        raise ValueError(f"{name} must be {torch_dtype}, got {t.dtype}")
    if shape is not None and t.numel() != math.prod(shape):
        raise ValueError(f"{name} must hold {' x '.join(map(str, shape))} values, "
                         f"got shape {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


class Cache:
    """One tiered KV cache (all layers and sequences) in a torch-owned workspace."""

    def __init__(self, cfg: Config, device="cuda", stream=None):
        import torch

        self.torch = torch
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.workspace = torch.empty(workspace_size(cfg), dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        _check(self.lib, self.lib.qevict_cache_init(
            ctypes.byref(cfg.to_c()), ctypes.c_void_p(self.workspace.data_ptr()),
            self.workspace.numel(), ctypes.c_void_p(self.stream.cuda_stream), ctypes.byref(h)))
        self.handle = h
        gr = cfg.group_size or (32 if cfg.window_tokens == 8 else cfg.window_tokens)
        self.n_cap = -(-(cfg.max_context - cfg.sink_tokens) // cfg.window_tokens)
        self._gr = gr

    # -- lifecycle --
    def close(self):
        if getattr(self, "handle", None):
            self.lib.qevict_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _c(self, status):
        _check(self.lib, status)

    # -- the decode path --
    def prefill_assign(self, layer: int, k, v, init_scores=None):
        """k, v: bf16 [B, H_kv, T, d]; init_scores: float32 [B, n_w] (None with
        the key-norm score)."""
        t = self.torch
        c = self.cfg
        if k.dim() != 4:
            raise ValueError(f"k must be [B, H_kv, T, d], got shape {tuple(k.shape)}")
        T = k.shape[2]
        kv = (c.batch, c.num_kv_heads, T, c.head_dim)
        n_w = max(0, -(-(T - c.sink_tokens) // c.window_tokens))
        sc = None if init_scores is None or init_scores.numel() == 0 else \
            _ptr(init_scores, t.float32, "init_scores", (c.batch, n_w))
        self._c(self.lib.qevict_prefill_assign(
            self.handle, layer, _ptr(k, t.bfloat16, "k", kv), _ptr(v, t.bfloat16, "v", kv), T, sc))

    def prefill_scores(self, q_obs, k, scores=None, scratch=None):
        """Initial window scores from the observation queries' attention.
        q_obs: bf16 [B, H_q, n_obs, d]; k: bf16 [B, H_kv, T, d]; returns float32
        [B, n_w] (written into `scores` when given)."""
        t = self.torch
        cfg = self.cfg
        B, n_obs, T = cfg.batch, q_obs.shape[2], k.shape[2]
        if tuple(q_obs.shape) != (B, cfg.num_q_heads, n_obs, cfg.head_dim):
            raise ValueError(f"q_obs shape {tuple(q_obs.shape)}")
        if tuple(k.shape) != (B, cfg.num_kv_heads, T, cfg.head_dim):
            raise ValueError(f"k shape {tuple(k.shape)}")
        n_w = max(0, -(-(T - cfg.sink_tokens) // cfg.window_tokens))
        if scores is None:
            scores = t.empty((B, n_w), dtype=t.float32, device=self.device)
        if scores.numel() != B * n_w:
            raise ValueError(f"scores must hold {B} x {n_w} values")
        need = prefill_scores_scratch_size(cfg, T, n_obs)
        if scratch is None:
            scratch = t.empty(need, dtype=t.uint8, device=self.device)
        self._c(self.lib.qevict_prefill_scores(
            self.handle, _ptr(q_obs, t.bfloat16, "q_obs"), n_obs, _ptr(k, t.bfloat16, "k"), T,
            _ptr(scratch, None, "scratch"), scratch.numel() * scratch.element_size(),
            _ptr(scores, t.float32, "scores") if n_w else None))
        return scores

    def prefill_scores_noalloc(self, q_obs, k, scores):
        """qevict_prefill_scores on the library's fixed per-device scratch (no
        scratch argument; the call allocates nothing).  q_obs: bf16
        [B, H_q, n_obs, d]; k: bf16 [B, H_kv, T, d]; scores: float32 [B, n_w]."""
        t = self.torch
        cfg = self.cfg
        B, n_obs, T = cfg.batch, q_obs.shape[2], k.shape[2]
        if tuple(q_obs.shape) != (B, cfg.num_q_heads, n_obs, cfg.head_dim):
            raise ValueError(f"q_obs shape {tuple(q_obs.shape)}")
        if tuple(k.shape) != (B, cfg.num_kv_heads, T, cfg.head_dim):
            raise ValueError(f"k shape {tuple(k.shape)}")
        n_w = max(0, -(-(T - cfg.sink_tokens) // cfg.window_tokens))
        self._c(self.lib.qevict_prefill_scores_noalloc(
            self.handle, _ptr(q_obs, t.bfloat16, "q_obs"), n_obs, _ptr(k, t.bfloat16, "k"), T,
            _ptr(scores, t.float32, "scores", (B, n_w)) if n_w else None))
        return scores

    def memory_report(self, layer: int, seq: int) -> dict:
        """Persistent cache bytes of one (layer, sequence), by component."""
        m = MemoryReport()
        self._c(self.lib.qevict_memory_report(self.handle, layer, seq, ctypes.byref(m)))
        return m.as_dict()

    def decode_attend(self, layer: int, q, k_new, v_new, out):
        t = self.torch
        c = self.cfg
        odt = t.bfloat16 if c.out_dtype == OUT_BF16 else t.float32
        qs, ks = (c.batch, c.num_q_heads, c.head_dim), (c.batch, c.num_kv_heads, c.head_dim)
        self._c(self.lib.qevict_decode_attend(
            self.handle, layer, _ptr(q, t.bfloat16, "q", qs), _ptr(k_new, t.bfloat16, "k_new", ks),
            _ptr(v_new, t.bfloat16, "v_new", ks), _ptr(out, odt, "out", qs)))

    def retier(self, layer: int, stats: bool = False):
        if stats:
            s = RetierStats()
            self._c(self.lib.qevict_retier(self.handle, layer, ctypes.byref(s)))
            return s.as_dict()
        self._c(self.lib.qevict_retier(self.handle, layer, None))
        return None

    def join_routing(self):
        """Order the cache stream after all routing enqueued so far (async routing)."""
        self._c(self.lib.qevict_join_routing(self.handle))

    def quantize_window(self, layer: int, seq: int, window: int):
        self._c(self.lib.qevict_quantize_window(self.handle, layer, seq, window))

    def promote_window(self, layer: int, seq: int, window: int):
        self._c(self.lib.qevict_promote_window(self.handle, layer, seq, window))

    # -- inspection --
    def get_state(self, layer: int, seq: int) -> dict:
        cap = self.n_cap
        tiers = np.zeros(cap, np.int8)
        scores = np.zeros(cap, np.float32)
        ledger = np.zeros(cap, np.int8)
        bits = np.zeros(cap, np.int8)
        n = ctypes.c_int32()
        self._c(self.lib.qevict_get_state(
            self.handle, layer, seq, tiers.ctypes.data_as(ctypes.c_void_p),
            scores.ctypes.data_as(ctypes.c_void_p), ledger.ctypes.data_as(ctypes.c_void_p),
            bits.ctypes.data_as(ctypes.c_void_p), cap, ctypes.byref(n)))
        m = n.value
        return dict(tiers=tiers[:m], scores=scores[:m], ledger=ledger[:m], bits=bits[:m], n=m)

    def export_window(self, layer: int, seq: int, window: int, quant=True, full=False) -> dict:
        h, w, d = self.cfg.num_kv_heads, self.cfg.window_tokens, self.cfg.head_dim
        gr = self._gr
        out = {}
        ptrs = [None] * 6
        if quant:
            out["codes_k"] = np.zeros((h, w, d), np.uint8)
            out["codes_v"] = np.zeros((h, w, d), np.uint8)
            out["meta_k"] = np.zeros((h, 2, 1, d), np.uint16)   # one key group per channel
            out["meta_v"] = np.zeros((h, 2, w, d // gr), np.uint16)
            for i, k in enumerate(("codes_k", "codes_v", "meta_k", "meta_v")):
                ptrs[i] = out[k].ctypes.data_as(ctypes.c_void_p)
        if full:
            out["full_k"] = np.zeros((h, w, d), np.uint16)
            out["full_v"] = np.zeros((h, w, d), np.uint16)
            ptrs[4] = out["full_k"].ctypes.data_as(ctypes.c_void_p)
            ptrs[5] = out["full_v"].ctypes.data_as(ctypes.c_void_p)
        self._c(self.lib.qevict_export_window(self.handle, layer, seq, window, *ptrs))
        return out

    def debug_shift_keys(self, layer: int, seq: int, window: int, delta):
        dlt = np.ascontiguousarray(delta, dtype=np.float32)
        if dlt.size != self.cfg.num_kv_heads * self.cfg.head_dim:
            raise ValueError(f"delta must hold H_kv x d values, got shape {dlt.shape}")
        self._c(self.lib.qevict_debug_shift_keys(self.handle, layer, seq, window,
                                                 dlt.ctypes.data_as(ctypes.c_void_p)))

    ROUTING_SYNC, ROUTING_GATE, ROUTING_QUEUE_WAIT = 0, 1, 2

    def routing_order(self) -> int:
        o = ctypes.c_int32()
        self._c(self.lib.qevict_routing_order(self.handle, ctypes.byref(o)))
        return o.value

    def debug_routing_gate(self, timeout_us: int, release: bool):
        self._c(self.lib.qevict_debug_routing_gate(self.handle, int(timeout_us), int(bool(release))))

    def debug_last_masses(self, layer: int) -> np.ndarray:
        c = self.cfg
        m = np.zeros((c.batch, c.num_q_heads, self.n_cap + 1), np.float32)
        self._c(self.lib.qevict_debug_last_masses(self.handle, layer, m.ctypes.data_as(ctypes.c_void_p)))
        return m

    def debug_masses(self, layer: int) -> np.ndarray:
        c = self.cfg
        m = np.zeros((c.batch, c.num_q_heads, self.n_cap + 1), np.float32)
        self._c(self.lib.qevict_debug_masses(self.handle, layer, m.ctypes.data_as(ctypes.c_void_p),
                                             self.n_cap))
        return m

    def profile_enable(self, on: bool = True):
        self._c(self.lib.qevict_profile_enable(self.handle, 1 if on else 0))

    def profile_read(self, kernel: int):
        ms, n = ctypes.c_double(), ctypes.c_int64()
        self._c(self.lib.qevict_profile_read(self.handle, kernel, ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value

    def last_attend_bytes(self, layer: int) -> int:
        n = ctypes.c_int64()
        self._c(self.lib.qevict_last_attend_bytes(self.handle, layer, ctypes.byref(n)))
        return n.value


# ------------------------------------------- prompts and the 8-bit block cache
# (these calls cost the GPU a few microseconds when they are small, so their marshalling
# asks each tensor for its shape, strides and device index once)
def _rows(t, torch, index, name, heads=None, tokens=None, dim=None):
    """Address and (token, head) strides of a packed bf16 tensor [tokens, heads, d] on
    device `index`."""
    if t.get_device() != index or index < 0:
        raise ValueError(f"{name} must be on device cuda:{index}, got {t.device}")
    if t.dtype is not torch.bfloat16:
        raise ValueError(f"{name} must be torch.bfloat16, got {t.dtype}")
    sh = t.shape
    if len(sh) != 3 or (heads is not None and sh[1] != heads) or (tokens is not None and sh[0] != tokens) or \
            (dim is not None and sh[2] != dim):
        raise ValueError(f"{name} must be [{'T' if tokens is None else tokens}, "
                         f"{'H' if heads is None else heads}, {'d' if dim is None else dim}], "
                         f"got shape {tuple(sh)}")
    if sh[0] > INT32_MAX or sh[1] > INT32_MAX:   # (rows that repeat one can be as many)
        raise ValueError(f"{name}: rows and heads must be below 2^31, got shape {tuple(sh)}")
    st = t.stride()
    if st[2] != 1 and sh[2] > 1:
        raise ValueError(f"{name}: the channels of a row must be contiguous")
    # the stride of a dimension of size 1 is never used (and may be anything)
    return t.data_ptr(), st[0] if sh[0] > 1 else 0, st[1] if sh[1] > 1 else 0


def _int32(t, torch, index, name, n):
    if t.get_device() != index or t.dtype is not torch.int32 or t.dim() != 1 or t.shape[0] != n or \
            not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of {n} entries on device cuda:{index}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    if n > INT32_MAX:
        raise ValueError(f"{name} must have fewer than 2^31 entries, got {n}")
    return t.data_ptr()


def _check_stream(stream, index):
    """A kernel on another device's stream would run there, on addresses of this one."""
    if stream.device.index != index:
        raise ValueError(f"the stream belongs to device {stream.device}, the tensors to cuda:{index}")


def _launch(lib, torch, index, stream, fn, *args):
    """A handle-free call with the device of its tensors current (kernels run on the
    current device), on `stream` or torch's current one there."""
    if stream is not None:
        _check_stream(stream, index)
    before = torch.cuda.current_device()
    if before != index:
        torch.cuda.set_device(index)
    try:
        st = stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(index)
        status = fn(*args, st)
    finally:
        if before != index:
            torch.cuda.set_device(before)
    if status != OK:
        _check(lib, status)


def prompt_attend(q, k, v, cu_tokens, out=None, softmax_scale: float = 0.0, stream=None):
    """Causal attention of packed prompts: prompt s is rows cu_tokens[s] ..
    cu_tokens[s + 1] - 1, each token attends to the tokens of its prompt up to itself.
    q: bf16 [T, H_q, d]; k, v: bf16 [T, H_kv, d]; any strides that are multiples of 8
    elements with the channels contiguous (slices of a fused projection, transposed
    [H, T, d] tensors).  cu_tokens: int32 [n + 1] on the device.  Returns out, bf16
    [T, H_q, d]; rows behind the last prompt are left as they were (undefined in an out
    that is allocated here).  No gradient is recorded.  Runs on `stream`, by default
    torch's current one, as a torch operation under torch.cuda.stream(stream) does: what it
    takes has to be ready there and stay allocated until it is done, and an out that is
    allocated here belongs to that stream."""
    lib = load_library()
    import torch
    index = q.get_device()
    qp, q_st, q_sh = _rows(q, torch, index, "q")
    T, hq, d = q.shape
    kp, k_st, k_sh = _rows(k, torch, index, "k", None, T, d)
    hkv = k.shape[1]
    vp, v_st, v_sh = _rows(v, torch, index, "v", hkv, T, d)
    if out is None:
        # from the pool of the stream that writes it: elsewhere pending work may still use it
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            out = torch.empty((T, hq, d), dtype=torch.bfloat16, device=q.device)
    op, o_st, o_sh = _rows(out, torch, index, "out", hq, T, d)
    n = cu_tokens.numel() - 1
    cu = _int32(cu_tokens, torch, index, "cu_tokens", n + 1)
    c = _PromptConfig(ABI_VERSION, n, T, hq, hkv, d, softmax_scale, q_st, q_sh, k_st, k_sh, v_st, v_sh,
                      o_st, o_sh)
    _launch(lib, torch, index, stream, lib.qevict_prompt_attend, ctypes.byref(c), qp, kp, vp, cu, op)
    return out


@dataclasses.dataclass
class BlockConfig:
    batch: int
    num_q_heads: int
    num_kv_heads: int
    max_context: int
    num_pages: int = 0           # 0: a page for every block of every place
    num_layers: int = 1
    head_dim: int = 128
    softmax_scale: float = 0.0


class BlockCache:
    """8-bit paged cache of sequences of different lengths (every token is kept; int8
    codes with one scale per 64-token block and KV head, the open block in bf16).

    Its state is plain tensors that the program may read, fill and share:
      k_codes [L, pages, H_kv, 64, d], v_codes [L, pages, H_kv, d, 64]   int8
      k_scale, v_scale [L, pages, H_kv]                                  float32
      k_tail, v_tail [L, batch, H_kv, 64, d]                             bf16, open blocks
      table [batch, ceil(max_context / 64)]  int32  page of each block, the same in all layers
      lens [batch]                           int32  tokens held; negative: no sequence
    An entry of table outside 0 .. pages - 1 means that the block has no page: its tokens
    take no part.  With num_pages = 0 place s owns pages s * n .. s * n + n - 1, n the
    columns of the table; otherwise the table starts at -1 and the program assigns pages
    (before the block they are for is complete).  lens starts at -1: the program sets it after
    storing a prompt and advances it after each step (advance()).

    Assigning to one of them copies into it.  Steps of one cache share its workspace and open
    blocks: they run one after the other.

    Calls run on torch's current stream unless the cache was given one.  With one of its own,
    everything the cache enqueues is on that stream: its state's first contents, store, attend,
    fetch and advance(); an assigned value is copied there after the current stream's work so
    far, and the current stream waits for the copy.  The tensors that a call takes have to be
    ready on that stream, a program that reads or changes the state tensors in place does so
    on it, or orders its streams with it, and a graph of the calls is captured on it."""

    def __init__(self, cfg: BlockConfig, device="cuda", stream=None):
        import torch

        self.torch = torch
        self.lib = load_library()
        self.cfg = cfg
        dev = torch.device(device)
        if dev.type != "cuda":
            raise ValueError(f"a block cache needs a GPU, got device {dev}")
        if cfg.batch < 1 or cfg.max_context < 1 or cfg.num_layers < 1 or cfg.num_kv_heads < 1 or \
                cfg.num_pages < 0:
            raise ValueError("batch, max_context, num_layers and num_kv_heads must be positive")
        if max(cfg.batch, cfg.max_context, cfg.num_pages, cfg.num_q_heads, cfg.num_kv_heads,
               cfg.head_dim) > INT32_MAX:   # the C ABI's fields, which ctypes would cut to their low bits
            raise ValueError("sizes must be below 2^31")
        if dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        if stream is not None:
            _check_stream(stream, dev.index)
        self.device = dev
        self.stream = stream
        L, B, h, d, n = cfg.num_layers, cfg.batch, cfg.num_kv_heads, cfg.head_dim, BLOCK_TOKENS
        cols = -(-cfg.max_context // n)
        pages = cfg.num_pages or B * cols
        self.num_pages = pages
        self._c = _BlockConfig(ABI_VERSION, B, cfg.num_q_heads, h, d, cfg.max_context, pages, cfg.softmax_scale)
        need = ctypes.c_size_t()
        _check(self.lib, self.lib.qevict_block_workspace_size(ctypes.byref(self._c), ctypes.byref(need)))
        z = torch.zeros
        with self._on_stream():   # (its memory is then reused in that stream's order, too)
            self._state = dict(
                k_codes=z((L, pages, h, n, d), dtype=torch.int8, device=dev),
                v_codes=z((L, pages, h, d, n), dtype=torch.int8, device=dev),
                k_scale=z((L, pages, h), dtype=torch.float32, device=dev),
                v_scale=z((L, pages, h), dtype=torch.float32, device=dev),
                k_tail=z((L, B, h, n, d), dtype=torch.bfloat16, device=dev),
                v_tail=z((L, B, h, n, d), dtype=torch.bfloat16, device=dev),
                table=torch.full((B, cols), -1, dtype=torch.int32, device=dev),
                lens=torch.full((B,), -1, dtype=torch.int32, device=dev))
            if not cfg.num_pages:
                self._state["table"].copy_(torch.arange(pages, dtype=torch.int32).view(B, cols))
            self.workspace = torch.empty(need.value, dtype=torch.uint8, device=dev)
        current = self._other_stream()
        if current is not None:
            current.wait_stream(stream)
        self._layers = [_BlockLayer(*[
            (t if name in ("table", "lens") else t[i]).data_ptr() for name, t in self._state.items()])
            for i in range(L)]

    def _on_stream(self):
        """Context of the cache's own tensor work: its stream, where it was given one."""
        return contextlib.nullcontext() if self.stream is None else self.torch.cuda.stream(self.stream)

    def _other_stream(self):
        """torch's current stream where that is not the one the cache was given, else None."""
        if self.stream is None:
            return None
        current = self.torch.cuda.current_stream(self.device)
        return None if current == self.stream else current

    def _assign(self, name, value):
        current = self._other_stream()
        if current is not None:
            self.stream.wait_stream(current)
        with self._on_stream():
            self._state[name].copy_(value)
        if current is not None:
            current.wait_stream(self.stream)

    def _call(self, fn, layer: int, *args):
        if not 0 <= layer < self.cfg.num_layers:
            raise ValueError(f"layer {layer} out of range")
        _launch(self.lib, self.torch, self.device.index, self.stream, fn, ctypes.byref(self._c),
                ctypes.byref(self._layers[layer]), *args)

    def _packed(self, k, v, cu_tokens):
        t, c, i = self.torch, self.cfg, self.device.index
        kr = _rows(k, t, i, "k", c.num_kv_heads, None, c.head_dim)
        vr = _rows(v, t, i, "v", c.num_kv_heads, k.shape[0], c.head_dim)
        return (*kr, *vr, _int32(cu_tokens, t, i, "cu_tokens", c.batch + 1), k.shape[0])

    def store(self, layer: int, k, v, cu_tokens):
        """Stores packed prompts: rows cu_tokens[s] .. cu_tokens[s + 1] - 1 of k, v (bf16
        [T, H_kv, d], strides as in prompt_attend) become the tokens of place s; a place
        without rows keeps what it holds."""
        self._call(self.lib.qevict_block_store, layer, *self._packed(k, v, cu_tokens))

    def fetch(self, layer: int, k, v, cu_tokens):
        """Writes the tokens of every place (at most lens[s] of them) to its rows of k, v
        (bf16 [T, H_kv, d]); other rows are left as they were."""
        self._call(self.lib.qevict_block_fetch, layer, *self._packed(k, v, cu_tokens))

    def attend(self, layer: int, q, k_new, v_new, out):
        """One decode step: appends token lens[s] of every place and attends with it.
        q: bf16 [batch, H_q, d]; k_new, v_new: bf16 [batch, H_kv, d]; out: bf16 like q."""
        p = []
        for x, name, heads in ((q, "q", self.cfg.num_q_heads), (k_new, "k_new", self.cfg.num_kv_heads),
                               (v_new, "v_new", self.cfg.num_kv_heads), (out, "out", self.cfg.num_q_heads)):
            if x.get_device() != self.device.index or x.dtype is not self.torch.bfloat16 or \
                    x.shape != (self.cfg.batch, heads, self.cfg.head_dim) or not x.is_contiguous():
                raise ValueError(f"{name} must be a contiguous bf16 tensor of shape "
                                 f"{(self.cfg.batch, heads, self.cfg.head_dim)} on {self.device}, got {x.dtype} "
                                 f"{tuple(x.shape)} on {x.device}")
            p.append(x.data_ptr())
        self._call(self.lib.qevict_block_attend, layer, *p, self.workspace.data_ptr(), self.workspace.numel())

    def advance(self):
        """After a step's last layer: lens + 1 where a place holds a sequence that has room."""
        with self._on_stream():
            self.lens += ((self.lens >= 0) & (self.lens < self.cfg.max_context)).to(self.lens.dtype)


def _state_tensor(name):
    def get(self):
        return self._state[name]

    def put(self, value):   # assignment writes into the tensor the kernels read
        if value is not self._state[name]:
            self._assign(name, value)
    return property(get, put)


for _name, _ in _BlockLayer._fields_:
    setattr(BlockCache, _name, _state_tensor(_name))
