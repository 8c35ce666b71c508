"""Thin Python binding of liblookat.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/lookat.h)
and hands it raw device pointers of torch CUDA tensors; no step of the method
runs in Python or in torch.  There is no CPU path: a missing library or a
tensor that is not on a CUDA device raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblookat.so")
LIB_DEBUG_PATH = os.path.join(_PKG, "liblookat_debug.so")      # the build whose attend kernels check the codes they read

EXPORTS = [
    "lookat_create", "lookat_destroy", "lookat_last_error", "lookat_is_debug_build", "lookat_fit_codebooks",
    "lookat_encode_keys", "lookat_build_lut", "lookat_attend", "lookat_attend_static", "lookat_attend_pqv",
    "lookat_attend_prefill", "lookat_decode_step", "lookat_decode_step_host",
    "lookat_kernel_launches", "lookat_probe_read_bandwidth", "lookat_selftest_timeout", "lookat_set_prefill_form", "lookat_set_timing", "lookat_attend_kernel_ms", "lookat_attend_kernel_stats",
    # include/lookat_gpt2.h
    "lookat_gpt2_create", "lookat_gpt2_destroy", "lookat_gpt2_last_error", "lookat_gpt2_set_weights", "lookat_gpt2_prefill",
    "lookat_gpt2_decode", "lookat_gpt2_layer_state", "lookat_gpt2_position", "lookat_gpt2_kernel_launches",
    "lookat_gpt2_set_profile", "lookat_gpt2_profile", "lookat_gpt2_use_q8_cache", "lookat_gpt2_fork", "lookat_gpt2_q8_state",
    "lookat_linear", "lookat_linear_qkv", "lookat_layernorm", "lookat_embed", "lookat_causal_attention", "lookat_argmax",
    # include/lookat_q8.h
    "lookat_q8_append", "lookat_attend_q8", "lookat_pages_extend", "lookat_pages_fork", "lookat_pages_compact",
    # include/lookat_serve.h
    "lookat_rope_table", "lookat_rope", "lookat_attend_packed", "lookat_q8_append_packed", "lookat_beam_select",
]

STATUS = {0: "LOOKAT_OK", 1: "LOOKAT_ERR_INVALID_ARG", 2: "LOOKAT_ERR_UNSUPPORTED",
          3: "LOOKAT_ERR_CUDA", 4: "LOOKAT_ERR_NOMEM", 5: "LOOKAT_ERR_TIMEOUT"}


class LookatError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class lookat_config(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("d_k", ctypes.c_int32), ("d_v", ctypes.c_int32), ("m", ctypes.c_int32),
                ("K", ctypes.c_int32), ("scale", ctypes.c_float)]


class lookat_gpt2_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layer", "n_head", "d_model", "vocab", "n_pos", "m", "K", "fit_iters",
                                              "keep_prompt_keys")]


LAYER_FIELDS = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_g", "ln2_b", "w_fc", "b_fc", "w_pr", "b_pr")


class lookat_gpt2_layer(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in LAYER_FIELDS]


class lookat_q8_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("k_amax", ctypes.c_void_p), ("v", ctypes.c_void_p), ("v_amax", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("page", ctypes.c_int32), ("format", ctypes.c_int32)]


class lookat_page_state(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("tables", "seq_lens", "refs", "free_list", "n_free")] + \
               [(n, ctypes.c_int32) for n in ("B", "max_pages", "n_pages", "page")]


class lookat_page_pool(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("page_bytes", ctypes.c_int64)]


class lookat_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class lookat_rope_config(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32)] + \
               [(n, ctypes.c_double) for n in ("base", "factor", "original_len", "low", "high")]


class lookat_beam_state(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("scores", "lengths", "finished", "tokens")] + \
               [(n, ctypes.c_int32) for n in ("groups", "beams", "max_len")]


_libs = {}


def load_library(debug: bool = False) -> ctypes.CDLL:
    """Loads liblookat.so (built by paper_2601_10155_b200.build), or its debug build; raises if absent."""
    if debug in _libs:
        return _libs[debug]
    path = LIB_DEBUG_PATH if debug else LIB_PATH
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: run `python -m paper_2601_10155_b200.build{' --debug' if debug else ''}` (needs nvcc). "
            "There is no fallback path.")
    lib = ctypes.CDLL(path)
    vp, i32, i64, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64
    lib.lookat_create.argtypes = [ctypes.POINTER(lookat_config), ctypes.c_int, vp, ctypes.POINTER(vp)]
    lib.lookat_create.restype = ctypes.c_int
    lib.lookat_destroy.argtypes = [vp]
    lib.lookat_destroy.restype = None
    lib.lookat_last_error.argtypes = [vp]
    lib.lookat_last_error.restype = ctypes.c_char_p
    lib.lookat_fit_codebooks.argtypes = [vp, vp, i32, i64, i32, u64, vp, vp, vp]
    lib.lookat_fit_codebooks.restype = ctypes.c_int
    lib.lookat_encode_keys.argtypes = [vp, vp, i32, i64, vp, vp, i64, i64, vp]
    lib.lookat_encode_keys.restype = ctypes.c_int
    lib.lookat_build_lut.argtypes = [vp, vp, i32, vp, vp]
    lib.lookat_build_lut.restype = ctypes.c_int
    lib.lookat_attend.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, vp, i32, vp, vp]
    lib.lookat_attend.restype = ctypes.c_int
    lib.lookat_attend_static.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, vp, i32, vp, vp]
    lib.lookat_attend_static.restype = ctypes.c_int
    lib.lookat_attend_pqv.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, vp, vp]
    lib.lookat_attend_pqv.restype = ctypes.c_int
    lib.lookat_attend_prefill.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, vp, vp]
    lib.lookat_attend_prefill.restype = ctypes.c_int
    lib.lookat_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, i64, i32, vp]
    lib.lookat_decode_step.restype = ctypes.c_int
    lib.lookat_decode_step_host.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, i64, i64, i32, vp]
    lib.lookat_decode_step_host.restype = ctypes.c_int
    lib.lookat_kernel_launches.argtypes = [vp]
    lib.lookat_kernel_launches.restype = ctypes.c_uint64
    lib.lookat_probe_read_bandwidth.argtypes = [vp, vp, ctypes.c_uint64, i32, ctypes.POINTER(ctypes.c_double)]
    lib.lookat_probe_read_bandwidth.restype = i32
    lib.lookat_selftest_timeout.argtypes = [vp]
    lib.lookat_selftest_timeout.restype = i32
    lib.lookat_set_prefill_form.argtypes = [vp, i32]
    lib.lookat_set_prefill_form.restype = i32
    lib.lookat_set_timing.argtypes = [vp, i32]
    lib.lookat_set_timing.restype = None
    lib.lookat_attend_kernel_ms.argtypes = [vp]
    lib.lookat_attend_kernel_ms.restype = ctypes.c_double
    lib.lookat_attend_kernel_stats.argtypes = [vp, ctypes.POINTER(ctypes.c_double)]
    lib.lookat_attend_kernel_stats.restype = i32
    # the GPT-2 harness (include/lookat_gpt2.h)
    lib.lookat_gpt2_create.argtypes = [ctypes.POINTER(lookat_gpt2_config), ctypes.c_int, vp, i32, i32, ctypes.POINTER(vp)]
    lib.lookat_gpt2_create.restype = i32
    lib.lookat_gpt2_destroy.argtypes = [vp]
    lib.lookat_gpt2_destroy.restype = None
    lib.lookat_gpt2_last_error.argtypes = [vp]
    lib.lookat_gpt2_last_error.restype = ctypes.c_char_p
    lib.lookat_gpt2_set_weights.argtypes = [vp, vp, vp, vp, vp, ctypes.POINTER(lookat_gpt2_layer)]
    lib.lookat_gpt2_set_weights.restype = i32
    lib.lookat_gpt2_prefill.argtypes = [vp, vp, i32, u64, vp]
    lib.lookat_gpt2_prefill.restype = i32
    lib.lookat_gpt2_decode.argtypes = [vp, vp, vp, vp, vp]
    lib.lookat_gpt2_decode.restype = i32
    lib.lookat_gpt2_layer_state.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp)]
    lib.lookat_gpt2_layer_state.restype = i32
    lib.lookat_gpt2_position.argtypes = [vp]
    lib.lookat_gpt2_position.restype = i32
    lib.lookat_gpt2_kernel_launches.argtypes = [vp]
    lib.lookat_gpt2_kernel_launches.restype = ctypes.c_uint64
    lib.lookat_gpt2_set_profile.argtypes = [vp, i32]
    lib.lookat_gpt2_set_profile.restype = None
    lib.lookat_gpt2_profile.argtypes = [vp, ctypes.POINTER(ctypes.c_double)]
    lib.lookat_gpt2_profile.restype = i32
    lib.lookat_gpt2_use_q8_cache.argtypes = [vp, i32, i32]
    lib.lookat_gpt2_use_q8_cache.restype = i32
    lib.lookat_gpt2_fork.argtypes = [vp, vp]
    lib.lookat_gpt2_fork.restype = i32
    lib.lookat_gpt2_q8_state.argtypes = [vp, i32, ctypes.POINTER(lookat_q8_cache), ctypes.POINTER(lookat_page_state)]
    lib.lookat_gpt2_q8_state.restype = i32
    lib.lookat_linear.argtypes = [vp, vp, i32, vp, vp, i64, i32, i32, i32, vp, vp, i32]
    lib.lookat_linear.restype = i32
    lib.lookat_linear_qkv.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, i64, i64, vp, i64, i64, vp, i64, i64]
    lib.lookat_linear_qkv.restype = i32
    lib.lookat_layernorm.argtypes = [vp, vp, vp, vp, i64, i32, vp]
    lib.lookat_layernorm.restype = i32
    lib.lookat_embed.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]
    lib.lookat_embed.restype = i32
    lib.lookat_causal_attention.argtypes = [vp, vp, vp, vp, i32, i32, i32, i64, vp]
    lib.lookat_causal_attention.restype = i32
    lib.lookat_argmax.argtypes = [vp, vp, i32, i32, vp]
    lib.lookat_argmax.restype = i32
    # the 8-bit paged cache (include/lookat_q8.h)
    lib.lookat_q8_append.argtypes = [vp, ctypes.POINTER(lookat_q8_cache), vp, vp, i32, i32, vp, i32, vp, vp]
    lib.lookat_q8_append.restype = i32
    lib.lookat_attend_q8.argtypes = [vp, ctypes.POINTER(lookat_q8_cache), vp, i32, i32, vp, i32, vp, vp, i32]
    lib.lookat_attend_q8.restype = i32
    lib.lookat_pages_extend.argtypes = [vp, ctypes.POINTER(lookat_page_state), vp, ctypes.POINTER(lookat_page_pool), i32]
    lib.lookat_pages_extend.restype = i32
    lib.lookat_pages_fork.argtypes = [vp, ctypes.POINTER(lookat_page_state), vp]
    lib.lookat_pages_fork.restype = i32
    lib.lookat_pages_compact.argtypes = [vp, ctypes.POINTER(lookat_page_state), ctypes.POINTER(lookat_page_pool), i32, vp]
    lib.lookat_pages_compact.restype = i32
    # what runs around it (include/lookat_serve.h)
    rows = ctypes.POINTER(lookat_rows)
    lib.lookat_rope_table.argtypes = [ctypes.POINTER(lookat_rope_config), ctypes.POINTER(u64), ctypes.POINTER(ctypes.c_float)]
    lib.lookat_rope_table.restype = i32
    lib.lookat_rope.argtypes = [vp, rows, rows, i64, vp, vp, i32, i32, ctypes.c_float, rows, rows]
    lib.lookat_rope.restype = i32
    lib.lookat_attend_packed.argtypes = [vp, rows, rows, rows, i64, i32, vp, rows]
    lib.lookat_attend_packed.restype = i32
    lib.lookat_q8_append_packed.argtypes = [vp, ctypes.POINTER(lookat_q8_cache), rows, rows, i64, i32, vp, vp, i32, vp]
    lib.lookat_q8_append_packed.restype = i32
    lib.lookat_beam_select.argtypes = [vp, ctypes.POINTER(lookat_beam_state), vp, i64, i32, i32, ctypes.c_double, vp, vp]
    lib.lookat_beam_select.restype = i32
    lib.lookat_is_debug_build.argtypes = []
    lib.lookat_is_debug_build.restype = i32
    _libs[debug] = lib
    return lib


def _dev(t, dtype, name, shape=None):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (the library has no CPU path)")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _host(t, dtype, name, shape):
    if not isinstance(t, torch.Tensor) or t.is_cuda:
        raise TypeError(f"{name} must be a host tensor")
    if t.dtype != dtype or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be contiguous {dtype} of shape {tuple(shape)}")
    return t.data_ptr()


def _on(t, dtype, name, device, shape=None):
    """_dev, and the tensor lies on the context's device."""
    if isinstance(t, torch.Tensor) and t.get_device() == device.index and t.dtype is dtype and t.is_contiguous() and \
            (shape is None or t.shape == shape):
        return t.data_ptr()                                     # (what the lines below check, at less cost)
    p = _dev(t, dtype, name, shape)
    if t is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the context on {device}")
    return p


def _fill(rows, t, name, device, shape):
    """fp16 [tokens][heads][d] with dense vectors into a lookat_rows; a view of a wider tensor will do."""
    if not (isinstance(t, torch.Tensor) and t.get_device() == device.index and t.dtype is torch.float16 and t.shape == shape):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a CUDA tensor (the library has no CPU path)")
        if t.dtype is not torch.float16:
            raise TypeError(f"{name} must have dtype torch.float16, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
        raise ValueError(f"{name} is on {t.device}, the context on {device}")
    rows.data = t.data_ptr()
    rows.token_stride, rows.head_stride, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"{name}: a vector's elements must lie next to each other")
    return rows


class _RowArgs(threading.local):
    """What calls that take packed rows fill in: each thread has its own, since a call gives others way."""

    def __init__(self):
        self.r = [lookat_rows() for _ in range(4)]


class RopeTable:
    """The speeds of rotary positions (include/lookat_serve.h): turns per position of each pair on the device, and the factor on
    cosines and sines.  scaling: none, linear, base, bands or ramp."""

    SCALINGS = ("none", "linear", "base", "bands", "ramp")

    def __init__(self, rotary_dim, base=10000.0, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0, device="cuda"):
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling must be one of {self.SCALINGS}, got {scaling!r}")
        cfg = lookat_rope_config(rotary_dim, self.SCALINGS.index(scaling), base, factor, original_len, low, high)
        turns, amplitude = (ctypes.c_uint64 * max(1, rotary_dim // 2))(), ctypes.c_float()
        st = load_library().lookat_rope_table(ctypes.byref(cfg), turns, ctypes.byref(amplitude))
        if st != 0:
            raise LookatError(st, "lookat_rope_table: settings out of range")
        self.rotary_dim, self.amplitude = rotary_dim, amplitude.value
        self.host = list(turns)                                 # fractions of 2^64
        self.turns = torch.tensor([t - (1 << 64) if t >> 63 else t for t in self.host], dtype=torch.int64, device=device)
        self.pointer, self.device = self.turns.data_ptr(), self.turns.device


class BeamState:
    """The beams of a batch (include/lookat_serve.h): scores fp32, lengths and finished int32 [groups][beams], tokens int32
    [groups][beams][max_len] or None."""

    def __init__(self, scores, lengths, finished, tokens=None):
        if not isinstance(scores, torch.Tensor) or scores.dim() != 2:
            raise ValueError("scores must have shape [groups][beams]")
        shape, dev, i32 = tuple(scores.shape), scores.device, torch.int32
        if tokens is not None and tokens.dim() != 3:
            raise ValueError("tokens must have shape [groups][beams][max_len]")
        self.scores, self.lengths, self.finished, self.tokens = scores, lengths, finished, tokens
        self.groups, self.beams, self.rows, self.device = *shape, shape[0] * shape[1], dev
        max_len = 0 if tokens is None else tokens.shape[2]
        self.c = lookat_beam_state(_dev(scores, torch.float32, "scores"), _on(lengths, i32, "lengths", dev, shape), _on(finished, i32, "finished", dev, shape),
                                   None if max_len == 0 else _on(tokens, i32, "tokens", dev, (*shape, max_len)), *shape, max_len)

    @classmethod
    def empty(cls, groups, beams, max_len, device="cuda"):
        """Beams before their first step: only the first of each group counts."""
        scores = torch.full((groups, beams), -math.inf, dtype=torch.float32, device=device)
        scores[:, 0] = 0.0
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        return cls(scores, z(groups, beams), z(groups, beams), z(groups, beams, max_len) if max_len else None)


class Q8Cache:
    """The arrays of an 8-bit paged cache (include/lookat_q8.h), checked once: k [n_pages][H_kv][page][d_k] and v
    [n_pages][H_kv][page][d_v], int8 or float8_e4m3fn, k_amax and v_amax fp32 [n_pages][H_kv]."""

    def __init__(self, k, k_amax, v, v_amax):
        if not isinstance(k, torch.Tensor) or k.dtype not in (torch.int8, torch.float8_e4m3fn):
            raise TypeError("k must be an int8 or float8_e4m3fn tensor")
        if k.dim() != 4:
            raise ValueError(f"k must have shape [n_pages][H_kv][page][d_k], got {tuple(k.shape)}")
        n_pages, H, page, d_k = k.shape
        if v.dim() != 4:
            raise ValueError(f"v must have shape [n_pages][H_kv][page][d_v], got {tuple(v.shape)}")
        self.k, self.k_amax, self.v, self.v_amax = k, k_amax, v, v_amax
        self.n_pages, self.page, self.device = n_pages, page, k.device
        self.heads = (H, d_k, v.shape[3])
        self.c = lookat_q8_cache(_dev(k, k.dtype, "k"), _on(k_amax, torch.float32, "k_amax", k.device, (n_pages, H)),
                                 _on(v, k.dtype, "v", k.device, (n_pages, H, page, v.shape[3])),
                                 _on(v_amax, torch.float32, "v_amax", k.device, (n_pages, H)),
                                 n_pages, page, 0 if k.dtype == torch.int8 else 1)

    @classmethod
    def empty(cls, n_pages, n_kv_heads, page, d_k, d_v, dtype=torch.int8, device="cuda"):
        """A cache of unwritten pages."""
        return cls(torch.zeros((n_pages, n_kv_heads, page, d_k), dtype=torch.uint8, device=device).view(dtype),
                   torch.zeros((n_pages, n_kv_heads), dtype=torch.float32, device=device),
                   torch.zeros((n_pages, n_kv_heads, page, d_v), dtype=torch.uint8, device=device).view(dtype),
                   torch.zeros((n_pages, n_kv_heads), dtype=torch.float32, device=device))

    def pools(self):
        """The arrays that are kept by pages (for lookat_pages_extend and lookat_pages_compact)."""
        return [self.k, self.k_amax, self.v, self.v_amax]


class PageState:
    """The pages of a batch (include/lookat_q8.h): int32 tensors tables [B][max_pages], seq_lens [B], refs [n_pages],
    free_list [n_pages], n_free [1]."""

    def __init__(self, tables, seq_lens, refs, free_list, n_free, page):
        if tables.dim() != 2 or refs.dim() != 1:
            raise ValueError("tables must have shape [B][max_pages], refs [n_pages]")
        B, max_pages = tables.shape
        n_pages, i32, dev = refs.shape[0], torch.int32, tables.device
        self.tables, self.seq_lens, self.refs, self.free_list, self.n_free = tables, seq_lens, refs, free_list, n_free
        self.B, self.max_pages, self.n_pages, self.page, self.device = B, max_pages, n_pages, page, dev
        self.c = lookat_page_state(_dev(tables, i32, "tables"), _on(seq_lens, i32, "seq_lens", dev, (B,)), _on(refs, i32, "refs", dev),
                                   _on(free_list, i32, "free_list", dev, (n_pages,)), _on(n_free, i32, "n_free", dev, (1,)),
                                   B, max_pages, n_pages, page)

    @classmethod
    def empty(cls, B, max_pages, n_pages, page, device="cuda"):
        """B empty rows over n_pages free pages (page 0 on top of the free list)."""
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        return cls(torch.full((B, max_pages), -1, dtype=torch.int32, device=device), z(B), z(n_pages),
                   torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device),
                   torch.full((1,), n_pages, dtype=torch.int32, device=device), page)


class PagePools:
    """Arrays that are kept by pages: tensors whose first dim is the page."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.n_pages = self.tensors[0].shape[0] if self.tensors else None
        self.device = self.tensors[0].device if self.tensors else None
        self.c = (lookat_page_pool * max(1, len(self.tensors)))()
        for i, t in enumerate(self.tensors):
            if t.dim() < 1 or t.shape[0] != self.n_pages:
                raise ValueError(f"pool {i} has {tuple(t.shape)}, not {self.n_pages} pages")
            self.c[i] = lookat_page_pool(_on(t, t.dtype, f"pool {i}", self.device), t.numel() // max(1, t.shape[0]) * t.element_size())


_NO_POOLS = PagePools(())


class Lookat:
    """A library context for one attention shape on one device and stream.

    Method names and argument order are those of the C entry points.
    """

    def __init__(self, n_q_heads, n_kv_heads, d_k, d_v, m, K=256, scale=0.0, device=0, stream=None, debug=False):
        self._lib = load_library(debug)
        self._h = None
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the LOOKAT library runs on the GPU only")
        self.cfg = lookat_config(n_q_heads, n_kv_heads, d_k, d_v, m, K, scale)
        self.device = torch.device("cuda", device)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        self.stream = stream
        h = ctypes.c_void_p()
        st = self._lib.lookat_create(ctypes.byref(self.cfg), device, ctypes.c_void_p(stream.cuda_stream),
                                     ctypes.byref(h))
        if st != 0:
            raise LookatError(st, "lookat_create rejected the configuration or the device")
        self._h = h
        self._shape, self._kv_shape = (n_q_heads, n_kv_heads, d_k, d_v), (n_kv_heads, d_k, d_v)
        self._raw_stream = stream.cuda_stream
        self._row_args = _RowArgs()
        self.scale = scale if scale > 0 else 1.0 / math.sqrt(d_k)

    # -- helpers ---------------------------------------------------------------
    @property
    def d_sub(self):
        return self.cfg.d_k // self.cfg.m

    @property
    def g(self):
        return self.cfg.n_q_heads // self.cfg.n_kv_heads

    def _check(self, st):
        if st != 0:
            raise LookatError(st, self._lib.lookat_last_error(self._h).decode())

    def lookat_last_error(self) -> str:
        return self._lib.lookat_last_error(self._h).decode()

    def close(self):
        if self._h is not None:
            self._lib.lookat_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C entry points ------------------------------------------------------
    def lookat_fit_codebooks(self, keys, iters, seed=0, init=None, codebooks=None, distortion=None,
                             want_distortion=False):
        c = self.cfg
        B, H, n, d_k = keys.shape
        if codebooks is None:
            codebooks = torch.empty((c.n_kv_heads, c.m, c.K, self.d_sub), dtype=torch.float32, device=self.device)
        if distortion is None and want_distortion:
            distortion = torch.empty((c.n_kv_heads, c.m, iters + 1), dtype=torch.float64, device=self.device)
        self._check(self._lib.lookat_fit_codebooks(
            self._h, _dev(keys, torch.float16, "keys", (B, c.n_kv_heads, n, c.d_k)), B, n, iters, seed,
            _dev(init, torch.float32, "init", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(distortion, torch.float64, "distortion", (c.n_kv_heads, c.m, iters + 1))))
        return (codebooks, distortion) if distortion is not None else codebooks

    def lookat_encode_keys(self, keys, codebooks, codes=None, L_max=None, pos=0, near_ties=None):
        c = self.cfg
        B, H, n, d_k = keys.shape
        if L_max is None:
            L_max = codes.shape[2] if codes is not None else pos + n
        if codes is None:
            codes = torch.zeros((B, c.n_kv_heads, L_max, c.m), dtype=torch.uint8, device=self.device)
        self._check(self._lib.lookat_encode_keys(
            self._h, _dev(keys, torch.float16, "keys", (B, c.n_kv_heads, n, c.d_k)), B, n,
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codes, torch.uint8, "codes", (B, c.n_kv_heads, L_max, c.m)), L_max, pos,
            _dev(near_ties, torch.int64, "near_ties", (1,))))
        return codes

    def lookat_build_lut(self, q, codebooks, lut=None):
        c = self.cfg
        B = q.shape[0]
        if lut is None:
            lut = torch.empty((B, c.n_q_heads, c.m, c.K), dtype=torch.float32, device=self.device)
        self._check(self._lib.lookat_build_lut(
            self._h, _dev(q, torch.float16, "q", (B, c.n_q_heads, c.d_k)), B,
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(lut, torch.float32, "lut", (B, c.n_q_heads, c.m, c.K))))
        return lut

    def lookat_attend(self, codes, v, lut=None, q=None, codebooks=None, seq_lens=None, n_splits=0,
                      out=None, scores_out=None):
        c = self.cfg
        B, H, L_max, m = codes.shape
        if out is None:
            out = torch.empty((B, c.n_q_heads, c.d_v), dtype=torch.float32, device=self.device)
        self._check(self._lib.lookat_attend(
            self._h, _dev(lut, torch.float32, "lut", (B, c.n_q_heads, c.m, c.K)),
            _dev(q, torch.float16, "q", (B, c.n_q_heads, c.d_k)),
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codes, torch.uint8, "codes", (B, c.n_kv_heads, L_max, c.m)),
            _dev(v, torch.float16, "v", (B, c.n_kv_heads, L_max, c.d_v)), B, L_max,
            _dev(seq_lens, torch.int32, "seq_lens", (B,)), n_splits,
            _dev(out, torch.float32, "out", (B, c.n_q_heads, c.d_v)),
            _dev(scores_out, torch.float32, "scores_out", (B, c.n_q_heads, L_max))))
        return out

    def lookat_attend_pqv(self, codes, v_codebooks, v_codes, lut=None, q=None, codebooks=None, seq_lens=None, out=None):
        """Decode attention with product-quantised values as well (weights from the key codes, output from the
        weight histogram over the value codes)."""
        c = self.cfg
        B, H, L_max, m = codes.shape
        _, m_v, K_v, d_vsub = v_codebooks.shape
        if out is None:
            out = torch.empty((B, c.n_q_heads, c.d_v), dtype=torch.float32, device=self.device)
        self._check(self._lib.lookat_attend_pqv(
            self._h, _dev(lut, torch.float32, "lut", (B, c.n_q_heads, c.m, c.K)),
            _dev(q, torch.float16, "q", (B, c.n_q_heads, c.d_k)),
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codes, torch.uint8, "codes", (B, c.n_kv_heads, L_max, c.m)),
            _dev(v_codebooks, torch.float32, "v_codebooks", (c.n_kv_heads, m_v, K_v, c.d_v // m_v)),
            _dev(v_codes, torch.uint8, "v_codes", (B, c.n_kv_heads, L_max, m_v)), m_v, K_v, B, L_max,
            _dev(seq_lens, torch.int32, "seq_lens", (B,)),
            _dev(out, torch.float32, "out", (B, c.n_q_heads, c.d_v))))
        return out

    def lookat_attend_static(self, codes, v, lut=None, q=None, codebooks=None, seq_lens=None, n_splits=0,
                             out=None, scores_out=None):
        """lookat_attend for callers that cannot let the library allocate device memory (a process whose
        own pool owns the device, a latency-critical loop): the kernel's scratch is a fixed array inside
        the library.  `out` should be passed in by such callers; it is created here only for convenience."""
        c = self.cfg
        B, H, L_max, m = codes.shape
        if out is None:
            out = torch.empty((B, c.n_q_heads, c.d_v), dtype=torch.float32, device=self.device)
        self._check(self._lib.lookat_attend_static(
            self._h, _dev(lut, torch.float32, "lut", (B, c.n_q_heads, c.m, c.K)),
            _dev(q, torch.float16, "q", (B, c.n_q_heads, c.d_k)),
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codes, torch.uint8, "codes", (B, c.n_kv_heads, L_max, c.m)),
            _dev(v, torch.float16, "v", (B, c.n_kv_heads, L_max, c.d_v)), B, L_max,
            _dev(seq_lens, torch.int32, "seq_lens", (B,)), n_splits,
            _dev(out, torch.float32, "out", (B, c.n_q_heads, c.d_v)),
            _dev(scores_out, torch.float32, "scores_out", (B, c.n_q_heads, L_max))))
        return out

    def lookat_attend_prefill(self, q, codebooks, codes, v, q_pos0=0, out=None, scores_out=None):
        c = self.cfg
        B, H, L_max, m = codes.shape
        L_q = q.shape[2]
        if out is None:
            out = torch.empty((B, c.n_q_heads, L_q, c.d_v), dtype=torch.float32, device=self.device)
        self._check(self._lib.lookat_attend_prefill(
            self._h, _dev(q, torch.float16, "q", (B, c.n_q_heads, L_q, c.d_k)),
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codes, torch.uint8, "codes", (B, c.n_kv_heads, L_max, c.m)),
            _dev(v, torch.float16, "v", (B, c.n_kv_heads, L_max, c.d_v)), B, L_q, L_max, q_pos0,
            _dev(out, torch.float32, "out", (B, c.n_q_heads, L_q, c.d_v)),
            _dev(scores_out, torch.float32, "scores_out", (B, c.n_q_heads, L_q, L_max))))
        return out

    def lookat_decode_step(self, q, k_new, codebooks, codes, v, pos, out=None, n_splits=0):
        c = self.cfg
        B, H, L_max, m = codes.shape
        if out is None:
            out = torch.empty((B, c.n_q_heads, c.d_v), dtype=torch.float32, device=self.device)
        self._check(self._lib.lookat_decode_step(
            self._h, _dev(q, torch.float16, "q", (B, c.n_q_heads, c.d_k)),
            _dev(k_new, torch.float16, "k_new", (B, c.n_kv_heads, c.d_k)),
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codes, torch.uint8, "codes", (B, c.n_kv_heads, L_max, c.m)),
            _dev(v, torch.float16, "v", (B, c.n_kv_heads, L_max, c.d_v)), B, L_max, pos, n_splits,
            _dev(out, torch.float32, "out", (B, c.n_q_heads, c.d_v))))
        return out

    def lookat_decode_step_host(self, q_host, k_new_host, v_new_host, codebooks, codes, v, pos, out_host,
                                n_splits=0):
        c = self.cfg
        B, H, L_max, m = codes.shape
        self._check(self._lib.lookat_decode_step_host(
            self._h, _host(q_host, torch.float16, "q_host", (B, c.n_q_heads, c.d_k)),
            _host(k_new_host, torch.float16, "k_new_host", (B, c.n_kv_heads, c.d_k)),
            _host(v_new_host, torch.float16, "v_new_host", (B, c.n_kv_heads, c.d_v)), B,
            _dev(codebooks, torch.float32, "codebooks", (c.n_kv_heads, c.m, c.K, self.d_sub)),
            _dev(codes, torch.uint8, "codes", (B, c.n_kv_heads, L_max, c.m)),
            _dev(v, torch.float16, "v", (B, c.n_kv_heads, L_max, c.d_v)), L_max, pos, n_splits,
            _host(out_host, torch.float32, "out_host", (B, c.n_q_heads, c.d_v))))
        return out_host

    def _empty(self, shape, strides, dtype):
        """A result that the caller did not give.  Its memory comes from the stream that writes it: what another stream had freed
        may still be in use there.  The caller's stream is recorded, where the result goes next."""
        dev = self.device
        if torch._C._cuda_getCurrentRawStream(dev.index) == self._raw_stream:
            return torch.empty_strided(shape, strides, dtype=dtype, device=dev)            # (takes half the time of empty)
        caller = torch.cuda.current_stream(dev)
        with torch.cuda.stream(self.stream):
            out = torch.empty_strided(shape, strides, dtype=dtype, device=dev)
        out.record_stream(caller)
        return out

    # -- the 8-bit paged cache (include/lookat_q8.h) --------------------------------
    def _q8(self, cache, tables, seq_lens):
        if cache.heads != self._kv_shape:
            raise ValueError(f"the cache holds (heads, d_k, d_v) = {cache.heads}, the context {self._kv_shape}")
        if cache.device != self.device:
            raise ValueError(f"the cache is on {cache.device}, the context on {self.device}")
        if tables.dim() != 2:
            raise ValueError(f"tables must have shape [B][max_pages], got {tuple(tables.shape)}")
        B, max_pages = tables.shape
        return B, max_pages, _on(tables, torch.int32, "tables", self.device), _on(seq_lens, torch.int32, "seq_lens", self.device, (B,))

    def lookat_q8_append(self, cache, k_new, v_new, tables, seq_lens, n_new=None):
        """Quantises the last n_new[b] (None: n) tokens of every row into its pages; k_new [B][H_kv][n][d_k]."""
        _, H, d_k, d_v = self._shape
        dev = self.device
        B, max_pages, tb, sl = self._q8(cache, tables, seq_lens)
        n = k_new.shape[2] if k_new.dim() == 4 else 0
        st = self._lib.lookat_q8_append(
            self._h, cache.c, _on(k_new, torch.float16, "k_new", dev, (B, H, n, d_k)), _on(v_new, torch.float16, "v_new", dev, (B, H, n, d_v)),
            B, n, tb, max_pages, sl, None if n_new is None else _on(n_new, torch.int32, "n_new", dev, (B,)))
        if st:
            self._check(st)

    def lookat_attend_q8(self, cache, q, tables, seq_lens, out=None, out_fp16=False):
        """Attention of the queries at the rows' last positions over the 8-bit cache; q [B][H_q][L_q][d_k] or, for one
        token per row, [B][H_q][d_k]."""
        H, _, d_k, d_v = self._shape
        dev = self.device
        B, max_pages, tb, sl = self._q8(cache, tables, seq_lens)
        one = q.dim() == 3
        L_q = 1 if one else q.shape[2]
        pq = _on(q, torch.float16, "q", dev, (B, H, d_k) if one else (B, H, L_q, d_k))
        dtype = torch.float16 if out_fp16 else torch.float32
        shape = (B, H, d_v) if one else (B, H, L_q, d_v)
        if out is None:
            n = L_q * d_v
            out = self._empty(shape, (H * d_v, d_v, 1) if one else (H * n, n, d_v, 1), dtype)
            po = out.data_ptr()
        else:
            po = _on(out, dtype, "out", dev, shape)
        st = self._lib.lookat_attend_q8(self._h, cache.c, pq, B, L_q, tb, max_pages, sl, po, 1 if out_fp16 else 0)
        if st:
            self._check(st)
        return out

    def _pages(self, state, pools):
        if state.device != self.device:
            raise ValueError(f"the page state is on {state.device}, the context on {self.device}")
        if not isinstance(pools, PagePools):
            pools = PagePools(() if pools is None else pools)
        if pools.tensors and (pools.n_pages != state.n_pages or pools.device != self.device):
            raise ValueError(f"the pools have {pools.n_pages} pages on {pools.device}, the state {state.n_pages} on {state.device}")
        return pools

    def lookat_pages_extend(self, state, n_new, pools):
        """Pages for n_new[b] more tokens per row (n_new all 0 afterwards if there are too few); pools: the tensors kept
        by pages, a PagePools of them, or None."""
        pools = self._pages(state, pools)
        self._check(self._lib.lookat_pages_extend(self._h, state.c, _on(n_new, torch.int32, "n_new", self.device, (state.B,)),
                                                  pools.c, len(pools.tensors)))

    def lookat_pages_fork(self, state, parents):
        """Row b continues from row parents[b]; -1 empties it."""
        self._pages(state, _NO_POOLS)
        self._check(self._lib.lookat_pages_fork(self._h, state.c, _on(parents, torch.int32, "parents", self.device, (state.B,))))

    def lookat_pages_compact(self, state, pools, remap=None):
        """Live pages into the lowest ids; remap: optional int32 [n_pages] that gets each page's new id (-1: not live)."""
        pools = self._pages(state, pools)
        self._check(self._lib.lookat_pages_compact(self._h, state.c, pools.c, len(pools.tensors),
                                                   _on(remap, torch.int32, "remap", self.device, (state.n_pages,))))

    # -- what runs around it (include/lookat_serve.h) --------------------------------
    def lookat_rope(self, q, k, positions, table, interleaved=False, q_out=None, k_out=None):
        """Rotary positions of q [tokens][H_q][d_k] and k [tokens][H_kv][d_k] (either may be None); new tensors unless results are
        given, which may be q and k themselves."""
        H, H_kv, d, _ = self._shape
        dev = self.device
        if q is None and k is None:
            raise ValueError("q and k are both None")
        if (q is None and q_out is not None) or (k is None and k_out is not None):
            raise ValueError("a result without its input")
        T = (k if q is None else q).shape[0]
        if table.device != dev:
            raise ValueError(f"the table is on {table.device}, the context on {dev}")
        r = self._row_args.r
        in_q = in_k = to_q = to_k = None
        if q is not None:
            shape = (T, H, d)
            if q_out is None:
                q_out = self._empty(shape, (H * d, d, 1), torch.float16)
            in_q, to_q = _fill(r[0], q, "q", dev, shape), _fill(r[1], q_out, "q_out", dev, shape)
        if k is not None:
            shape = (T, H_kv, d)
            if k_out is None:
                k_out = self._empty(shape, (H_kv * d, d, 1), torch.float16)
            in_k, to_k = _fill(r[2], k, "k", dev, shape), _fill(r[3], k_out, "k_out", dev, shape)
        st = self._lib.lookat_rope(self._h, in_q, in_k, T, _on(positions, torch.int32, "positions", dev, (T,)), table.pointer, table.rotary_dim,
                                   1 if interleaved else 0, table.amplitude, to_q, to_k)
        if st:
            self._check(st)
        return q_out, k_out

    def lookat_attend_packed(self, q, k, v, starts, out=None):
        """Exact causal attention of packed prompts: q [tokens][H_q][d_k], k [tokens][H_kv][d_k], v [tokens][H_kv][d_v], row b the
        tokens starts[b] .. starts[b + 1] - 1; tokens of no row keep what `out` held."""
        H, H_kv, d_k, d_v = self._shape
        dev, r = self.device, self._row_args.r
        T, n = q.shape[0], starts.shape[0]
        shape = (T, H, d_v)
        if out is None:
            out = self._empty(shape, (H * d_v, d_v, 1), torch.float16)
        st = self._lib.lookat_attend_packed(self._h, _fill(r[0], q, "q", dev, (T, H, d_k)), _fill(r[1], k, "k", dev, (T, H_kv, d_k)),
                                            _fill(r[2], v, "v", dev, (T, H_kv, d_v)), T, n - 1, _on(starts, torch.int32, "starts", dev, (n,)),
                                            _fill(r[3], out, "out", dev, shape))
        if st:
            self._check(st)
        return out

    def lookat_q8_append_packed(self, cache, k, v, starts, tables, seq_lens):
        """Quantises the packed tokens starts[b] .. starts[b + 1] - 1 as the newest of row b; k [tokens][H_kv][d_k]."""
        _, H, d_k, d_v = self._shape
        dev, r = self.device, self._row_args.r
        B, max_pages, tb, sl = self._q8(cache, tables, seq_lens)
        T = k.shape[0]
        st = self._lib.lookat_q8_append_packed(self._h, cache.c, _fill(r[0], k, "k", dev, (T, H, d_k)), _fill(r[1], v, "v", dev, (T, H, d_v)), T, B,
                                               _on(starts, torch.int32, "starts", dev, (B + 1,)), tb, max_pages, sl)
        if st:
            self._check(st)

    def lookat_beam_select(self, state, logits, eos=-1, length_penalty=0.0, next_ids=None, parents=None):
        """One step of beam search over logits [groups * beams][vocab] (rows may lie further apart); the state moves in place.
        Returns (next_ids, parents), int32 [groups * beams]."""
        dev, rows, i32 = self.device, state.rows, torch.int32
        if state.device != dev:
            raise ValueError(f"the beams are on {state.device}, the context on {dev}")
        if not isinstance(logits, torch.Tensor) or not logits.is_cuda or logits.dtype is not torch.float32:
            raise TypeError("logits must be a CUDA tensor of dtype torch.float32")
        if logits.get_device() != dev.index or logits.dim() != 2 or logits.shape[0] != rows or logits.shape[1] < 1 or \
                (logits.shape[1] > 1 and logits.stride(1) != 1):
            raise ValueError(f"logits must have shape [{rows}][vocab] with dense rows on {dev}")
        vocab = logits.shape[1]
        if next_ids is None:
            next_ids = self._empty((rows,), (1,), i32)
        if parents is None:
            parents = self._empty((rows,), (1,), i32)
        st = self._lib.lookat_beam_select(self._h, state.c, logits.data_ptr(), logits.stride(0) if rows > 1 else vocab, vocab, eos, length_penalty,
                                          _on(next_ids, i32, "next_ids", dev, (rows,)), _on(parents, i32, "parents", dev, (rows,)))
        if st:
            self._check(st)
        return next_ids, parents

    def lookat_kernel_launches(self) -> int:
        return int(self._lib.lookat_kernel_launches(self._h))

    def lookat_probe_read_bandwidth(self, buf, reps=5):
        """GB/s of a read-only streaming pass over the device tensor `buf` (measurement aid)."""
        out = ctypes.c_double(0.0)
        self._check(self._lib.lookat_probe_read_bandwidth(self._h, ctypes.c_void_p(buf.data_ptr()),
                                                          ctypes.c_uint64(buf.numel() * buf.element_size()), int(reps),
                                                          ctypes.byref(out)))
        return out.value

    def lookat_selftest_timeout(self):
        self._check(self._lib.lookat_selftest_timeout(self._h))

    def lookat_set_prefill_form(self, form):
        """form: 'auto', 'tables' or 'contraction' (or the header's integer values)."""
        code = {"auto": 0, "tables": 1, "contraction": 2}.get(form, form)
        self._check(self._lib.lookat_set_prefill_form(self._h, int(code)))

    def lookat_set_timing(self, launches):
        """launches >= 1: time up to that many attend launches from now on (True = 64); 0 / False: stop."""
        self._lib.lookat_set_timing(self._h, 64 if launches is True else int(launches))

    def lookat_attend_kernel_stats(self):
        """{'n', 'min', 'median', 'max', 'mean'} of the timed attend launches in milliseconds, or None."""
        st = (ctypes.c_double * 4)()
        n = int(self._lib.lookat_attend_kernel_stats(self._h, st))
        return None if n == 0 else {"n": n, "min": st[0], "median": st[1], "max": st[2], "mean": st[3]}

    def lookat_attend_kernel_ms(self) -> float:
        return float(self._lib.lookat_attend_kernel_ms(self._h))


    # -- the GPT-2 harness's kernels one by one (include/lookat_gpt2.h) ------------
    def lookat_linear(self, x, w_t, bias=None, gelu=False, residual=None, out=None, out_fp16=True):
        M, K = x.shape
        N = w_t.shape[0]
        if out is None:
            out = torch.empty((M, N), dtype=torch.float16 if out_fp16 else torch.float32, device=self.device)
        if x.dtype not in (torch.float16, torch.float32):
            raise TypeError("x must be fp16 or fp32")
        self._check(self._lib.lookat_linear(
            self._h, _dev(x, x.dtype, "x", (M, K)), 1 if x.dtype == torch.float32 else 0, _dev(w_t, torch.float16, "w_t", (N, K)),
            _dev(bias, torch.float16, "bias", (N,)), M, N, K, 1 if gelu else 0, _dev(residual, torch.float32, "residual", (M, N)),
            _dev(out, torch.float16 if out_fp16 else torch.float32, "out", (M, N)), 1 if out_fp16 else 0))
        return out

    def lookat_linear_qkv(self, x, w_t, bias, B, T, n_head, q, k, v, q_off=0, k_off=0, v_off=0):
        d = n_head * 64
        self._check(self._lib.lookat_linear_qkv(
            self._h, _dev(x, torch.float16, "x", (B * T, d)), _dev(w_t, torch.float16, "w_t", (3 * d, d)),
            _dev(bias, torch.float16, "bias", (3 * d,)), B, T, n_head,
            _dev(q, torch.float16, "q"), q.shape[2], q_off, _dev(k, torch.float16, "k"), k.shape[2], k_off,
            _dev(v, torch.float16, "v"), v.shape[2], v_off))
        return q, k, v

    def lookat_layernorm(self, x, gain, bias, out=None):
        rows, d = x.shape
        if out is None:
            out = torch.empty((rows, d), dtype=torch.float16, device=self.device)
        self._check(self._lib.lookat_layernorm(self._h, _dev(x, torch.float32, "x"), _dev(gain, torch.float16, "gain", (d,)),
                                               _dev(bias, torch.float16, "bias", (d,)), rows, d, _dev(out, torch.float16, "out", (rows, d))))
        return out

    def lookat_embed(self, ids, wte, wpe, pos0=0, out=None):
        B, T = ids.shape
        vocab, d = wte.shape
        if out is None:
            out = torch.empty((B, T, d), dtype=torch.float32, device=self.device)
        self._check(self._lib.lookat_embed(self._h, _dev(ids, torch.int32, "ids"), _dev(wte, torch.float16, "wte"),
                                           _dev(wpe, torch.float16, "wpe"), B, T, pos0, d, vocab, _dev(out, torch.float32, "out", (B, T, d))))
        return out

    def lookat_causal_attention(self, q, k, v, out=None):
        B, H, T, dh = q.shape
        if out is None:
            out = torch.empty((B, T, H * dh), dtype=torch.float16, device=self.device)
        self._check(self._lib.lookat_causal_attention(self._h, _dev(q, torch.float16, "q", (B, H, T, 64)), _dev(k, torch.float16, "k", (B, H, T, 64)),
                                                      _dev(v, torch.float16, "v"), B, H, T, v.shape[2], _dev(out, torch.float16, "out", (B, T, H * 64))))
        return out

    def lookat_argmax(self, logits, out=None):
        rows, n = logits.shape
        if out is None:
            out = torch.empty((rows,), dtype=torch.int32, device=self.device)
        self._check(self._lib.lookat_argmax(self._h, _dev(logits, torch.float32, "logits"), rows, n, _dev(out, torch.int32, "out", (rows,))))
        return out


class LookatGpt2:
    """The GPT-2 decoder harness (include/lookat_gpt2.h): argument marshalling only.  `weights` is the dict of fp16
    numpy arrays the seeded generator makes; they are uploaded once and kept alive here."""

    def __init__(self, weights, B, capacity, m, K, fit_iters, device=0, stream=None, keep_prompt_keys=False):
        self._lib = load_library()
        self._h = None
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the LOOKAT library runs on the GPU only")
        self.device = torch.device("cuda", device)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        self.stream = stream
        w = weights
        self.cfg = lookat_gpt2_config(w["n_layer"], w["n_head"], w["d_model"], w["vocab"], w["n_pos"], m, K, fit_iters,
                                      1 if keep_prompt_keys else 0)
        self.B, self.capacity = B, capacity
        h = ctypes.c_void_p()
        st = self._lib.lookat_gpt2_create(ctypes.byref(self.cfg), device, ctypes.c_void_p(stream.cuda_stream), B, capacity, ctypes.byref(h))
        if st != 0:
            raise LookatError(st, "lookat_gpt2_create rejected the configuration or ran out of memory")
        self._h = h
        up = lambda a: torch.from_numpy(a).to(self.device)
        self._keep = {k: up(w[k]) for k in ("wte", "wpe", "lnf_g", "lnf_b")}
        self._layers = [{k: up(lw[k]) for k in LAYER_FIELDS} for lw in w["layers"]]
        arr = (lookat_gpt2_layer * w["n_layer"])()
        for l, lw in enumerate(self._layers):
            for k in LAYER_FIELDS:
                setattr(arr[l], k, lw[k].data_ptr())
        self._check(self._lib.lookat_gpt2_set_weights(self._h, self._keep["wte"].data_ptr(), self._keep["wpe"].data_ptr(),
                                                      self._keep["lnf_g"].data_ptr(), self._keep["lnf_b"].data_ptr(), arr))

    def _check(self, st):
        if st != 0:
            raise LookatError(st, self.lookat_gpt2_last_error())

    def lookat_gpt2_last_error(self) -> str:
        """The last call's error, or what the model's kernels have found (after a synchronisation)."""
        return self._lib.lookat_gpt2_last_error(self._h).decode()

    def close(self):
        if self._h is not None:
            self._lib.lookat_gpt2_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def lookat_gpt2_prefill(self, ids, seed=0, want_hidden=False):
        B, T = ids.shape
        hidden = torch.empty((B, T, self.cfg.d_model), dtype=torch.float32, device=self.device) if want_hidden else None
        self._check(self._lib.lookat_gpt2_prefill(self._h, _dev(ids, torch.int32, "ids", (self.B, T)), T, seed,
                                                  None if hidden is None else hidden.data_ptr()))
        return hidden

    def lookat_gpt2_decode(self, ids, want_hidden=False, want_logits=False, want_next=False, logits=None, next_ids=None):
        hidden = torch.empty((self.B, self.cfg.d_model), dtype=torch.float32, device=self.device) if want_hidden else None
        if want_logits and logits is None:
            logits = torch.empty((self.B, self.cfg.vocab), dtype=torch.float32, device=self.device)
        if want_next and next_ids is None:
            next_ids = torch.empty((self.B,), dtype=torch.int32, device=self.device)
        self._check(self._lib.lookat_gpt2_decode(self._h, _dev(ids, torch.int32, "ids", (self.B,)),
                                                 None if hidden is None else hidden.data_ptr(),
                                                 None if logits is None else logits.data_ptr(),
                                                 None if next_ids is None else next_ids.data_ptr()))
        return hidden, logits, next_ids

    def lookat_gpt2_layer_state(self, layer, T=None):
        """(codebooks, codes, values, prompt_keys) of a layer as torch views of the model's own device memory."""
        ptrs = [ctypes.c_void_p() for _ in range(4)]
        self._check(self._lib.lookat_gpt2_layer_state(self._h, layer, *[ctypes.byref(p) for p in ptrs]))
        c = self.cfg

        def view(ptr, shape, dtype):
            if not ptr.value:
                return None
            self.stream.synchronize()
            typestr = {torch.float32: "<f4", torch.float16: "<f2", torch.uint8: "|u1"}[dtype]
            return torch.as_tensor(_RawDeviceArray(ptr.value, shape, typestr), device=self.device).clone()
        H, cap = c.n_head, self.capacity
        return (view(ptrs[0], (H, c.m, c.K, 64 // c.m), torch.float32), view(ptrs[1], (self.B, H, cap, c.m), torch.uint8),
                view(ptrs[2], (self.B, H, cap, 64), torch.float16),
                view(ptrs[3], (self.B, H, T, 64), torch.float16) if T else None)

    def lookat_gpt2_use_q8_cache(self, page=16, dtype=torch.int8):
        """The 8-bit paged cache in place of codes and fp16 values; before the first prompt."""
        if dtype not in (torch.int8, torch.float8_e4m3fn):
            raise TypeError("dtype must be int8 or float8_e4m3fn")
        self._check(self._lib.lookat_gpt2_use_q8_cache(self._h, page, 0 if dtype == torch.int8 else 1))

    def lookat_gpt2_fork(self, parents):
        """Row b continues from row parents[b] (int32 [B], each in 0..B-1; else from itself, with a finding)."""
        self._check(self._lib.lookat_gpt2_fork(self._h, _on(parents, torch.int32, "parents", self.device, (self.B,))))

    def lookat_gpt2_q8_state(self, layer):
        """(k, k_amax, v, v_amax, tables, seq_lens, refs, free_list, n_free) of a layer's 8-bit cache and the batch's pages,
        copied; k and v as bytes."""
        q, ps, c = lookat_q8_cache(), lookat_page_state(), self.cfg
        self._check(self._lib.lookat_gpt2_q8_state(self._h, layer, ctypes.byref(q), ctypes.byref(ps)))
        self.stream.synchronize()
        view = lambda ptr, shape, t: torch.as_tensor(_RawDeviceArray(ptr, shape, t), device=self.device).clone()  # noqa: E731
        rows = (q.n_pages, c.n_head, q.page, 64)
        return (view(q.k, rows, "|u1"), view(q.k_amax, rows[:2], "<f4"), view(q.v, rows, "|u1"), view(q.v_amax, rows[:2], "<f4"),
                view(ps.tables, (ps.B, ps.max_pages), "<i4"), view(ps.seq_lens, (ps.B,), "<i4"), view(ps.refs, (ps.n_pages,), "<i4"),
                view(ps.free_list, (ps.n_pages,), "<i4"), view(ps.n_free, (1,), "<i4"))

    def lookat_gpt2_set_profile(self, enabled: bool):
        self._lib.lookat_gpt2_set_profile(self._h, 1 if enabled else 0)

    def lookat_gpt2_profile(self):
        """(steps, {category: milliseconds}) of the decode steps made since profiling was switched on."""
        names = ("embed", "layernorm", "qkv", "attention", "out_proj", "mlp", "lm_head")
        ms = (ctypes.c_double * len(names))()
        steps = int(self._lib.lookat_gpt2_profile(self._h, ms))
        return steps, {n: ms[i] for i, n in enumerate(names)}

    def lookat_gpt2_position(self) -> int:
        return int(self._lib.lookat_gpt2_position(self._h))

    def lookat_gpt2_kernel_launches(self) -> int:
        return int(self._lib.lookat_gpt2_kernel_launches(self._h))


class _RawDeviceArray:
    """A device array of the library seen through the CUDA array interface (no copy, no ownership)."""

    def __init__(self, ptr: int, shape, typestr: str):
        self.__cuda_array_interface__ = {"shape": tuple(int(x) for x in shape), "typestr": typestr, "data": (int(ptr), False),
                                         "version": 2, "strides": None}


# ---- byte accounting of the method (Section 3.4 "Compression Ratio", Section 3.1) ----
def key_bytes_per_token(m: int) -> int:
    """A compressed key is m uint8 indices."""
    return m


def key_compression_ratio(d_k: int, m: int) -> float:
    """fp16 key (2*d_k bytes) over its m code bytes."""
    return 2.0 * d_k / m


def lut_entries(m: int, K: int = 256) -> int:
    return m * K


def kv_cache_bytes_fp16(H: int, L: int, d_k: int) -> int:
    """Uncompressed fp16 KV cache: 2*H*d_k values per token, 2 bytes each."""
    return 4 * H * L * d_k


def attend_bytes_per_token_kvhead(m: int, d_v: int) -> int:
    """What one attend pass must read per cached token and KV head: m code bytes + fp16 V row."""
    return m + 2 * d_v
