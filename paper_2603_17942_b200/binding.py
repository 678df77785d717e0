"""ctypes binding of ``libesp_b200.so`` -- argument marshalling only.

Function names mirror ``include/esp.h``.  PyTorch appears here only as the
owner of device memory and streams: tensors are turned into raw pointers and
the library does all the work.  There is no CPU fallback; if the library is
missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Dict, List, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libesp_b200.so")

ESP_MAX_ROWS = 128
ESP_MAX_PROBES = 8
ESP_MAX_KPRIME = 32
ESP_PREFILL_CHUNK = 120
ESP_MAX_UNREAD_STEPS = 1024

ERRORS = {0: "ESP_OK", -1: "ESP_E_BADCFG", -2: "ESP_E_WORKSPACE", -3: "ESP_E_PROMPT", -4: "ESP_E_FULL",
          -5: "ESP_E_DEVICE", -6: "ESP_E_CUDA", -7: "ESP_E_STATE", -8: "ESP_E_ARG"}

EXPORTS = ["esp_workspace_bytes", "esp_init", "esp_prefill", "esp_step", "esp_step_async", "esp_read", "esp_set_mask", "esp_set_tree",
           "esp_debug_state", "esp_debug_capture", "esp_debug_set_gemm", "esp_debug_set_layer_kernel", "esp_debug_layer_timeline", "esp_step_profiled", "esp_get_stats",
           "esp_debug_wait_selftest", "esp_debug_gumbel", "esp_free",
           "esp_tree_attention_scratch_bytes", "esp_tree_attention", "esp_tree_attention_status", "esp_tree_attention_static", "esp_gemm_scratch_bytes",
           "esp_gemm_bf16",
           "esp_rope_frequencies", "esp_rope_table_bytes", "esp_rope_table", "esp_qk_norm_rope", "esp_paged_append",
           "esp_paged_attention_scratch_bytes", "esp_paged_attention", "esp_paged_status"]

__all__ = ["EspError", "esp_model_cfg", "esp_spec_cfg", "esp_weights", "esp_stats", "load_library", "model_cfg",
           "spec_cfg", "Handle", "esp_heads", "esp_paged_cache", "esp_paged_batch", "esp_rope_cfg", "rope_cfg", "PagedCache", "PagedBatch", "ESP_ROPE_MAX_DIM", "ESP_MAX_ROWS", "ESP_MAX_PROBES", "ESP_MAX_KPRIME", "ESP_PREFILL_CHUNK", "ESP_MAX_UNREAD_STEPS", "ESP_STATIC_SCRATCH_BYTES", "EXPORTS", "LIB_PATH", "KINDS"] + EXPORTS


class EspError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where} failed: {ERRORS.get(code, code)}")
        self.code = code


class esp_model_cfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn",
                                              "vocab", "dtype", "tied_embeddings", "qk_norm")] + \
               [("rope_base", ctypes.c_float), ("rms_eps", ctypes.c_float), ("max_seq_len", ctypes.c_int32),
                ("max_batch", ctypes.c_int32)]


class esp_spec_cfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_probes", "topk", "max_nodes", "expand_width", "n_anchor",
                                              "prune_parent", "prune_root", "ema_per_token")] + [("lam", ctypes.c_float)] + \
               [("static_widths", ctypes.c_int32 * ESP_MAX_PROBES), ("mask_init", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("seed_lo", ctypes.c_uint32), ("seed_hi", ctypes.c_uint32)]


_PP = ctypes.POINTER(ctypes.c_void_p)


class esp_weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("lm_head", ctypes.c_void_p), ("final_norm", ctypes.c_void_p)] + \
               [(n, _PP) for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "norm_attn", "norm_ffn",
                                   "q_norm", "k_norm")]


class esp_stats(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int64), ("emitted", ctypes.c_int64), ("accept_hist", ctypes.c_int64 * (ESP_MAX_PROBES + 1)),
                ("device_error", ctypes.c_int32), ("kernels_per_step", ctypes.c_int32), ("rows_hist", ctypes.c_int64 * 4)]


class esp_heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("n_heads", ctypes.c_int32)]


class esp_paged_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("page_stride", "token_stride", "head_stride")] + \
               [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")]


class esp_paged_batch(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_new", ctypes.c_int32), ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("table_pages", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("status", ctypes.c_void_p)]


class esp_rope_cfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rotary_dim", "interleaved", "scaling", "original_len")] + \
               [(n, ctypes.c_float) for n in ("base", "factor", "low", "high", "amplitude")]


_lib = None
_P, _I, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
# (with the types declared once, a call hands over plain numbers: a call per layer has no time for wrapping each argument)
_ARGTYPES = {
    "esp_rope_frequencies": [_P, _P],
    "esp_rope_table_bytes": [_P, _P],
    "esp_rope_table": [_P, _P, ctypes.c_size_t, _P],
    "esp_qk_norm_rope": [_I, _I, _I, _P, _P, _P, _P, _F, _P, _P, _P, _P, _P, _P],
    "esp_paged_append": [_I, _P, _P, _P, _P, _P, _P, _P, _F, _P, _P, _P, _P, _P],
    "esp_paged_attention_scratch_bytes": [_I, _I, _P],
    "esp_paged_attention": [_I, _P, _P, _P, _P, _I, _F, _P, _P, _P, ctypes.c_size_t, _P],
    "esp_paged_status": [_P, _P, _P],
}


def load_library(path: Optional[str] = None):
    """dlopen the CUDA library (raises OSError if it was not built)."""
    global _lib
    if _lib is None or path is not None:
        p = path or LIB_PATH
        if not os.path.exists(p):
            raise OSError(f"{p} not found: build it with `python -m paper_2603_17942_b200.build` "
                          f"(there is no fallback implementation)")
        lib = ctypes.CDLL(p)
        for name in EXPORTS:
            getattr(lib, name).restype = None if name == "esp_free" else ctypes.c_int
        for name, types in _ARGTYPES.items():
            getattr(lib, name).argtypes = types
        if path is not None:
            return lib
        _lib = lib
    return _lib


def _check(rc: int, where: str):
    if rc != 0:
        raise EspError(rc, where)


def _vp(x) -> ctypes.c_void_p:
    if x is None:
        return ctypes.c_void_p(None)
    if hasattr(x, "data_ptr"):
        return ctypes.c_void_p(x.data_ptr())
    if isinstance(x, np.ndarray):
        return ctypes.c_void_p(x.ctypes.data)
    return ctypes.c_void_p(int(x))


def model_cfg(shape, max_seq_len: int, max_batch: int = 1) -> esp_model_cfg:
    """esp_model_cfg from any object with the shape fields (see synth.ModelShape)."""
    return esp_model_cfg(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn,
                         shape.vocab, 0 if shape.dtype == "fp32" else 1, int(bool(shape.tied)), int(bool(shape.qk_norm)),
                         float(shape.rope_base), float(shape.rms_eps), int(max_seq_len), int(max_batch))


def spec_cfg(n_probes=0, topk=1, max_nodes=1, expand_width=1, n_anchor=0, prune_parent=True, prune_root=False,
             ema_per_token=True, lam=0.1, static_widths=(), mask_init=0, temperature=0.0, seed=0) -> esp_spec_cfg:
    widths = (ctypes.c_int32 * ESP_MAX_PROBES)(*[int(w) for w in static_widths])
    return esp_spec_cfg(n_probes, topk, max_nodes, expand_width, n_anchor, int(prune_parent), int(prune_root),
                        int(ema_per_token), float(lam), widths, int(mask_init), float(temperature),
                        int(seed) & 0xffffffff, (int(seed) >> 32) & 0xffffffff)


# ---------------------------------------------------------------- raw calls (same names as the header)
def esp_workspace_bytes(model: esp_model_cfg, spec: esp_spec_cfg) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().esp_workspace_bytes(ctypes.byref(model), ctypes.byref(spec), ctypes.byref(out)), "esp_workspace_bytes")
    return out.value


def esp_init(model: esp_model_cfg, spec: esp_spec_cfg, weights: esp_weights, workspace, workspace_bytes: int, stream=None):
    h = ctypes.c_void_p(None)
    _check(load_library().esp_init(ctypes.byref(model), ctypes.byref(spec), ctypes.byref(weights), _vp(workspace),
                                   ctypes.c_size_t(workspace_bytes), _vp(stream), ctypes.byref(h)), "esp_init")
    return h


def esp_prefill(h, seq: int, prompt: np.ndarray) -> int:
    prompt = np.ascontiguousarray(prompt, dtype=np.int32)
    first = ctypes.c_int32(-1)
    _check(load_library().esp_prefill(h, ctypes.c_int32(seq), _vp(prompt), ctypes.c_int32(len(prompt)), ctypes.byref(first)), "esp_prefill")
    return first.value


def esp_step(h, tokens_out: np.ndarray, n_out: np.ndarray):
    _check(load_library().esp_step(h, _vp(tokens_out), _vp(n_out)), "esp_step")


def esp_step_async(h):
    _check(load_library().esp_step_async(h), "esp_step_async")


def esp_read(h, tokens_out: np.ndarray, n_out: np.ndarray):
    _check(load_library().esp_read(h, _vp(tokens_out), _vp(n_out)), "esp_read")


def esp_set_mask(h, seq: int, mask):
    mask = np.ascontiguousarray(mask, dtype=np.float32)
    _check(load_library().esp_set_mask(h, ctypes.c_int32(seq), _vp(mask)), "esp_set_mask")


def esp_set_tree(h, seq: int, tokens, parents):
    tokens = np.ascontiguousarray(tokens, dtype=np.int32)
    parents = np.ascontiguousarray(parents, dtype=np.int32)
    _check(load_library().esp_set_tree(h, ctypes.c_int32(seq), _vp(tokens), _vp(parents), ctypes.c_int32(len(tokens))), "esp_set_tree")


def esp_debug_state(h, seq: int, d_model: int, n_probes: int = 1) -> Dict[str, object]:
    R, KP = ESP_MAX_ROWS, ESP_MAX_KPRIME
    out = {"row_token": np.zeros(R, np.int32), "row_parent": np.zeros(R, np.int32), "row_depth": np.zeros(R, np.int32),
           "topk_ids": np.zeros((R, KP), np.int32), "topk_vals": np.zeros((R, KP), np.float32),
           "lse": np.zeros(R, np.float32), "mask_vec": np.zeros((max(n_probes, 1), d_model), np.float32)}
    nn, nr, L = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(load_library().esp_debug_state(h, ctypes.c_int32(seq), _vp(out["row_token"]), _vp(out["row_parent"]),
                                          _vp(out["row_depth"]), ctypes.byref(nn), ctypes.byref(nr), ctypes.byref(L),
                                          _vp(out["topk_ids"]), _vp(out["topk_vals"]), _vp(out["lse"]), _vp(out["mask_vec"])),
           "esp_debug_state")
    out.update(n_nodes=nn.value, n_rows=nr.value, L=L.value)
    return out


def esp_debug_capture(h, logits=None, hidden=None):
    _check(load_library().esp_debug_capture(h, _vp(logits), _vp(hidden)), "esp_debug_capture")


def esp_debug_set_gemm(h, impl: int):
    _check(load_library().esp_debug_set_gemm(h, ctypes.c_int32(impl)), "esp_debug_set_gemm")


def esp_debug_set_layer_kernel(h, mode: int):
    """1: one kernel per operation (default), 0: all decoder layers in one persistent cooperative kernel."""
    _check(load_library().esp_debug_set_layer_kernel(h, ctypes.c_int32(mode)), "esp_debug_set_layer_kernel")


def esp_debug_layer_timeline(h, n_layers: int) -> np.ndarray:
    """Global-timer stamps (ns) of the last profiled step: [n_layers][10 barriers][8 words] (see esp.h)."""
    out = np.zeros(n_layers * 80, np.uint64)
    n = ctypes.c_int32(0)
    _check(load_library().esp_debug_layer_timeline(h, _vp(out), ctypes.c_int32(out.size), ctypes.byref(n)), "esp_debug_layer_timeline")
    return out[:n.value].reshape(-1, 10, 8)


KINDS = ("norm_and_partial_consumers", "qkv_gemm", "tree_attention", "o_gemm", "gateup_gemm", "down_gemm", "lmhead_topk", "select_tree")


def esp_step_profiled(h, tokens_out: np.ndarray, n_out: np.ndarray) -> Dict[str, float]:
    ms = np.zeros(8, np.float32)
    _check(load_library().esp_step_profiled(h, _vp(ms), _vp(tokens_out), _vp(n_out)), "esp_step_profiled")
    return {k: float(v) for k, v in zip(KINDS, ms)}


def esp_get_stats(h) -> esp_stats:
    st = esp_stats()
    _check(load_library().esp_get_stats(h, ctypes.byref(st)), "esp_get_stats")
    return st


def esp_debug_wait_selftest(scratch, stream=None) -> int:
    """Runs the bounded-wait self-test; returns the device status code the kernel recorded (1 = timed out)."""
    st = ctypes.c_int32(-1)
    _check(load_library().esp_debug_wait_selftest(_vp(scratch), _vp(stream), ctypes.byref(st)), "esp_debug_wait_selftest")
    return st.value


def esp_debug_gumbel(seed: int, position: int, n_tokens: int, noise_out, stream=None):
    _check(load_library().esp_debug_gumbel(ctypes.c_uint32(seed & 0xffffffff), ctypes.c_uint32((seed >> 32) & 0xffffffff),
                                           ctypes.c_uint32(position), ctypes.c_int32(n_tokens), _vp(noise_out), _vp(stream)),
           "esp_debug_gumbel")


def esp_free(h):
    load_library().esp_free(h)


def esp_tree_attention_scratch_bytes(batch: int, n_q_heads: int, head_dim: int, cap: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().esp_tree_attention_scratch_bytes(ctypes.c_int32(batch), ctypes.c_int32(n_q_heads),
                                                           ctypes.c_int32(head_dim), ctypes.c_int32(cap), ctypes.byref(out)),
           "esp_tree_attention_scratch_bytes")
    return out.value


def esp_tree_attention(dtype: int, batch: int, n_rows: int, L: int, cap: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                       dcap: int, q, kcache, vcache, anc, depth, out, scratch, scratch_bytes: int, stream=None):
    _check(load_library().esp_tree_attention(
        ctypes.c_int32(dtype), ctypes.c_int32(batch), ctypes.c_int32(n_rows), ctypes.c_int32(L), ctypes.c_int32(cap),
        ctypes.c_int32(n_q_heads), ctypes.c_int32(n_kv_heads), ctypes.c_int32(head_dim), ctypes.c_int32(dcap), _vp(q),
        _vp(kcache), _vp(vcache), _vp(anc), _vp(depth), _vp(out), _vp(scratch), ctypes.c_size_t(scratch_bytes), _vp(stream)),
        "esp_tree_attention")


ESP_STATIC_SCRATCH_BYTES = 32 << 20


def esp_tree_attention_static(dtype: int, batch: int, n_rows: int, L: int, cap: int, n_q_heads: int, n_kv_heads: int,
                              head_dim: int, dcap: int, q, kcache, vcache, anc, depth, out, stream=None):
    """esp_tree_attention with the library's built-in 32 MiB scratch array: no scratch argument, no allocation."""
    _check(load_library().esp_tree_attention_static(
        ctypes.c_int32(dtype), ctypes.c_int32(batch), ctypes.c_int32(n_rows), ctypes.c_int32(L), ctypes.c_int32(cap),
        ctypes.c_int32(n_q_heads), ctypes.c_int32(n_kv_heads), ctypes.c_int32(head_dim), ctypes.c_int32(dcap), _vp(q),
        _vp(kcache), _vp(vcache), _vp(anc), _vp(depth), _vp(out), _vp(stream)), "esp_tree_attention_static")


def esp_tree_attention_status(scratch=None, stream=None) -> int:
    """Device status word of the last tree attention on `scratch` (None: on the built-in array); raises EspError(ESP_E_DEVICE) if set."""
    st = ctypes.c_int32(0)
    _check(load_library().esp_tree_attention_status(_vp(scratch), _vp(stream), ctypes.byref(st)), "esp_tree_attention_status")
    return st.value


def esp_gemm_scratch_bytes() -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().esp_gemm_scratch_bytes(ctypes.byref(out)), "esp_gemm_scratch_bytes")
    return out.value


def esp_gemm_bf16(impl: int, rows: int, n_out: int, k_in: int, x, w, y, scratch, scratch_bytes: int, stream=None):
    _check(load_library().esp_gemm_bf16(ctypes.c_int32(impl), ctypes.c_int32(rows), ctypes.c_int32(n_out), ctypes.c_int32(k_in),
                                        _vp(x), _vp(w), _vp(y), _vp(scratch), ctypes.c_size_t(scratch_bytes), _vp(stream)),
           "esp_gemm_bf16")


# ---------------------------------------------------------------- operators over a paged key/value cache
# These take the tensors themselves ([tokens, heads, head_dim], the last dimension dense) and read shapes, strides and types off them; what does not
# fit together raises EspError(ESP_E_ARG) before the library is called.  They run on `stream` (a torch stream or its address), by default on torch's current one.
ESP_ROPE_MAX_DIM = 256
ROPE_SCALINGS = ("none", "linear", "base", "rotations", "index")


def _i32(x, where: str, name: str) -> int:
    """x where the library takes 32 bits (ctypes would cut the rest off)."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise EspError(-8, f"{where} ({name}: {x} is more than 32 bits hold)")
    return x


def rope_cfg(rotary_dim: int, base: float = 10000.0, interleaved: bool = False, scaling: str = "none", factor: float = 1.0, original_len: int = 8192,
             low: float = 1.0, high: Optional[float] = None, amplitude: float = 1.0) -> esp_rope_cfg:
    """esp_rope_cfg.  scaling: none, linear, base, rotations or index (see esp.h); high: turns above which a pair is kept, by default 4 for
    "rotations" and 32 for "index"."""
    if scaling not in ROPE_SCALINGS:
        raise EspError(-1, f"rope_cfg(scaling={scaling!r})")
    if high is None:
        high = 32.0 if scaling == "index" else 4.0
    return esp_rope_cfg(_i32(rotary_dim, "rope_cfg", "rotary_dim"), int(bool(interleaved)), ROPE_SCALINGS.index(scaling), _i32(original_len, "rope_cfg", "original_len"), base, factor,
                        low, high, amplitude)


def esp_rope_frequencies(rope: esp_rope_cfg) -> np.ndarray:
    """Radians per position of every rotated pair (fp64)."""
    out = np.zeros(ESP_ROPE_MAX_DIM // 2, np.float64)
    _check(load_library().esp_rope_frequencies(ctypes.byref(rope), out.ctypes.data), "esp_rope_frequencies")
    return out[:rope.rotary_dim // 2].copy()


def esp_rope_table_bytes(rope: esp_rope_cfg) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().esp_rope_table_bytes(ctypes.byref(rope), ctypes.byref(out)), "esp_rope_table_bytes")
    return out.value


def _need(ok: bool, where: str, what: str):
    if not ok:
        raise EspError(-8, f"{where} ({what})")


_torch = None
_DTYPES: Dict[object, int] = {}        # torch dtype -> dtype of the library


def _on_current_device(device: int, where: str):
    """The tensors' device (their get_device()) has to be the current one: the library launches there."""
    global _torch
    if _torch is None:
        import torch
        _DTYPES.update({torch.float32: 0, torch.bfloat16: 1})
        _torch = torch
    if device < 0 or device != _torch.cuda.current_device():
        raise EspError(-8, f"{where} (tensors on device {device}, which is not the current one)")


def esp_rope_table(rope: esp_rope_cfg, table, stream=None):
    """Fills `table` (a CUDA tensor of esp_rope_table_bytes bytes or more), once per configuration."""
    _on_current_device(table.get_device(), "esp_rope_table")
    _need(table.is_contiguous(), "esp_rope_table", "table: not dense")
    _check(load_library().esp_rope_table(ctypes.byref(rope), table.data_ptr(), table.numel() * table.element_size(), _stream(stream)), "esp_rope_table")


def _stream(stream):
    """Address of a stream; None: the current one, on which the call's tensors are used."""
    if stream is None:
        stream = _torch.cuda.current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


_pack_heads = struct.Struct("Pqqi4x").pack        # the bytes of an esp_heads: a quarter of the time that filling the struct takes
assert struct.calcsize("Pqqi4x") == ctypes.sizeof(esp_heads)


def _heads(x, tokens: int, dim: int, dtype, device: int, where: str, name: str):
    """x [tokens, heads, head_dim] as the bytes of an esp_heads; None stays None.  (A call per layer: nothing here is formatted unless it fails.)"""
    if x is None:
        return None
    shape, stride = x.shape, x.stride()
    if len(shape) != 3 or shape[0] != tokens or shape[2] != dim or x.dtype is not dtype or x.get_device() != device or (stride[2] != 1 and dim != 1):
        raise EspError(-8, f"{where} ({name}: {tuple(shape)} {x.dtype} on {x.device}, strides {stride}; wanted [{tokens}, heads, {dim}] {dtype} on device {device}, "
                           f"last dimension dense)")
    return _pack_heads(x.data_ptr(), stride[0], stride[1], shape[1])


def _vector(x, n: int, dtypes, device: int, where: str, name: str):
    """Address of a dense tensor of n elements (None: NULL)."""
    if x is None:
        return None
    if x.numel() != n or x.dtype not in dtypes or x.get_device() != device or not x.is_contiguous():
        raise EspError(-8, f"{where} ({name}: {tuple(x.shape)} {x.dtype} on {x.device}; wanted {n} dense elements of {dtypes} on device {device})")
    return x.data_ptr()


class PagedCache:
    """Pages of keys and values.  k, v [pages, kv_heads, page_size, head_dim] (order "head") or [pages, page_size, kv_heads, head_dim] (order "token"),
    fp32 or bf16, any strides that both share with a dense last dimension.  Keeps the tensors alive."""

    def __init__(self, k, v, order: str = "head"):
        where = "PagedCache"
        _need(order in ("head", "token"), where, f"order {order!r}")
        _need(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and k.device == v.device, where, "k and v differ")
        _need(str(k.dtype) in ("torch.float32", "torch.bfloat16") and (k.stride(3) == 1 or k.shape[3] == 1), where, "type, or last dimension not dense")
        h, s = (1, 2) if order == "head" else (2, 1)
        self.k, self.v, self.order = k, v, order
        self.dtype, self.device, self.head_dim = k.dtype, k.get_device(), k.shape[3]
        sizes = [_i32(k.shape[i], where, "pages, page_size, kv_heads, head_dim") for i in (0, s, h, 3)]
        self.c = esp_paged_cache(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(s), k.stride(h), *sizes,
                                 0 if str(k.dtype) == "torch.float32" else 1)
        self.ref = ctypes.byref(self.c)


class PagedBatch:
    """The sequences of a call: q_start [batch + 1], kv_len [batch], page_table [batch, pages] int32 on the GPU (their contents are read when a call runs),
    max_new: most new tokens of a sequence, status: an int32 tensor of one element or None.  Keeps the tensors alive."""

    def __init__(self, q_start, kv_len, page_table, max_new: int, status=None):
        where = "PagedBatch"
        n = kv_len.numel()
        _need(page_table.dim() == 2 and page_table.shape[0] == n and q_start.numel() == n + 1, where, "q_start, kv_len and page_table do not fit together")
        for t in (q_start, kv_len, status):
            _need(t is None or (str(t.dtype) == "torch.int32" and t.is_contiguous() and t.get_device() == page_table.get_device()), where, "int32, dense, one device")
        _need(str(page_table.dtype) == "torch.int32" and (page_table.stride(1) == 1 or page_table.shape[1] <= 1) and
              (page_table.stride(0) >= page_table.shape[1] or n <= 1), where, "page_table: int32 rows")
        _need(status is None or status.numel() >= 1, where, "status")
        self.q_start, self.kv_len, self.page_table, self.status = q_start, kv_len, page_table, status
        self.device = page_table.get_device()
        row = _i32(page_table.shape[1], where, "page_table")
        self.c = esp_paged_batch(_i32(n, where, "batch"), _i32(max_new, where, "max_new"), q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), row,
                                 _i32(page_table.stride(0), where, "page_table") if n > 1 else row,
                                 None if status is None else status.data_ptr())
        self.ref = ctypes.byref(self.c)


def esp_qk_norm_rope(q, k, q_out, k_out, rope: Optional[esp_rope_cfg] = None, rope_table=None, positions=None, q_gain=None, k_gain=None, eps: float = 1e-6,
                     stream=None):
    """Per-head RMSNorm (where a gain is given) and rotation (where `rope` is) of q and k into q_out and k_out; one pair may be None."""
    where = "esp_qk_norm_rope"
    x = k if q is None else q
    _need(x is not None and x.dim() == 3, where, "q or k [tokens, heads, head_dim]")
    n, _, d = x.shape
    n, d = _i32(n, where, "tokens"), _i32(d, where, "head_dim")
    dev = x.get_device()
    _on_current_device(dev, where)
    dt = x.dtype
    _need(dt in _DTYPES, where, "fp32 or bf16")
    _check(load_library().esp_qk_norm_rope(
        _DTYPES[dt], n, d, _heads(q, n, d, dt, dev, where, "q"), _heads(k, n, d, dt, dev, where, "k"), _vector(q_gain, d, (dt,), dev, where, "q_gain"),
        _vector(k_gain, d, (dt,), dev, where, "k_gain"), eps, None if rope is None else ctypes.byref(rope), _table(rope, rope_table, dev, where),
        _vector(positions, n, (_torch.int32,), dev, where, "positions"), _heads(q_out, n, d, dt, dev, where, "q_out"),
        _heads(k_out, n, d, dt, dev, where, "k_out"), _stream(stream)), where)


def _table(rope, table, device: int, where: str):
    if rope is None or table is None:
        return None
    _need(table.get_device() == device and table.numel() * table.element_size() >= 4 * rope.rotary_dim, where, "rope_table")
    return table.data_ptr()


def esp_paged_append(cache: PagedCache, batch: PagedBatch, k, v, rope: Optional[esp_rope_cfg] = None, rope_table=None, positions=None, k_gain=None, q=None,
                     q_out=None, q_gain=None, eps: float = 1e-6, stream=None):
    """Appends the new tokens' k (normed and rotated as asked) and v to the pages; with q, norms and rotates the queries into q_out in the same launch."""
    where = "esp_paged_append"
    n = _i32(k.shape[0], where, "tokens")
    dev, dt, d = cache.device, cache.dtype, cache.head_dim
    _on_current_device(dev, where)
    _need(batch.device == dev, where, "cache and batch on one device")
    _check(load_library().esp_paged_append(
        n, cache.ref, batch.ref, _heads(k, n, d, dt, dev, where, "k"), _heads(v, n, d, dt, dev, where, "v"), _heads(q, n, d, dt, dev, where, "q"),
        _vector(q_gain, d, (dt,), dev, where, "q_gain"), _vector(k_gain, d, (dt,), dev, where, "k_gain"), eps,
        None if rope is None else ctypes.byref(rope), _table(rope, rope_table, dev, where), _vector(positions, n, (_torch.int32,), dev, where, "positions"),
        _heads(q_out, n, d, dt, dev, where, "q_out"), _stream(stream)), where)


def esp_paged_attention_scratch_bytes(n_q_heads: int, head_dim: int) -> int:
    out = ctypes.c_size_t(0)
    where = "esp_paged_attention_scratch_bytes"
    _check(load_library().esp_paged_attention_scratch_bytes(_i32(n_q_heads, where, "n_q_heads"), _i32(head_dim, where, "head_dim"), ctypes.byref(out)), where)
    return out.value


def esp_paged_attention(cache: PagedCache, batch: PagedBatch, q, out, scratch, scratch_bytes: int, anc=None, window: int = 0, scale: float = 0.0, lse=None,
                        stream=None):
    """Attention of the new tokens over the pages into `out`: causal, with a window, or with the ancestor masks `anc` [tokens, 2] (64-bit words) of draft trees."""
    where = "esp_paged_attention"
    n, window = _i32(q.shape[0], where, "tokens"), _i32(window, where, "window")
    dev, dt, d = cache.device, cache.dtype, cache.head_dim
    _on_current_device(dev, where)
    _need(batch.device == dev and scratch.get_device() == dev, where, "cache, batch and scratch on one device")
    _need(scratch.numel() * scratch.element_size() >= scratch_bytes and scratch.is_contiguous(), where, "scratch_bytes")
    _check(load_library().esp_paged_attention(
        n, cache.ref, batch.ref, _heads(q, n, d, dt, dev, where, "q"), _vector(anc, 2 * n, (_torch.int64, _torch.uint64), dev, where, "anc"), window, scale,
        _heads(out, n, d, dt, dev, where, "out"), None if lse is None else _vector(lse, n * q.shape[1], (_torch.float32,), dev, where, "lse"),
        scratch.data_ptr(), scratch_bytes, _stream(stream)), where)


def esp_paged_status(batch: PagedBatch, stream=None) -> int:
    """The batch's status word (0); raises EspError(ESP_E_DEVICE) if a kernel has set it."""
    _need(batch.status is not None, "esp_paged_status", "the batch has no status word")
    _on_current_device(batch.device, "esp_paged_status")           # (whose current stream is waited for)
    st = ctypes.c_int32(0)
    _check(load_library().esp_paged_status(batch.status.data_ptr(), _stream(stream), ctypes.byref(st)), "esp_paged_status")
    return st.value


# ---------------------------------------------------------------- convenience: a handle that keeps its tensors alive
class Handle:
    """esp_init + the tensors it points at.  ``weights`` is a dict of CUDA tensors (see synth.make_weights)."""

    def __init__(self, shape, spec: esp_spec_cfg, weights: Dict[str, object], max_seq_len: int, max_batch: int = 1, stream=None):
        import torch
        self.shape, self.spec = shape, spec
        self.model = model_cfg(shape, max_seq_len, max_batch)
        self.weights = weights
        self.max_batch = max_batch
        w = esp_weights()
        w.embed, w.lm_head, w.final_norm = weights["embed"].data_ptr(), weights["lm_head"].data_ptr(), weights["final_norm"].data_ptr()
        self._arrays = []
        for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "norm_attn", "norm_ffn", "q_norm", "k_norm"):
            arr = (ctypes.c_void_p * shape.n_layers)(*[t.data_ptr() for t in weights[n]])
            self._arrays.append(arr)
            setattr(w, n, ctypes.cast(arr, _PP))
        self._w = w
        self.workspace_bytes = esp_workspace_bytes(self.model, spec)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=weights["embed"].device)
        self.stream = stream
        sp = stream.cuda_stream if stream is not None else None
        self.h = esp_init(self.model, spec, w, self.workspace, self.workspace_bytes, sp)
        self.tokens_out = np.zeros((max_batch, ESP_MAX_PROBES + 1), np.int32)
        self.n_out = np.zeros(max_batch, np.int32)

    def prefill(self, prompt, seq: int = 0) -> int:
        return esp_prefill(self.h, seq, prompt)

    def step(self, seq: int = 0) -> List[int]:
        esp_step(self.h, self.tokens_out, self.n_out)
        return [int(t) for t in self.tokens_out[seq, :self.n_out[seq]]]

    def step_async(self):
        esp_step_async(self.h)

    def read(self, seq: int = 0) -> List[int]:
        esp_read(self.h, self.tokens_out, self.n_out)
        return [int(t) for t in self.tokens_out[seq, :self.n_out[seq]]]

    def generate(self, prompt, max_new: int, seq: int = 0) -> List[int]:
        out = [self.prefill(prompt, seq)]
        while len(out) < max_new:
            out.extend(self.step(seq))
        return out[:max_new]

    def set_tree(self, tokens, parents, seq: int = 0):
        esp_set_tree(self.h, seq, tokens, parents)

    def set_mask(self, mask, seq: int = 0):
        esp_set_mask(self.h, seq, mask)

    def state(self, seq: int = 0):
        return esp_debug_state(self.h, seq, self.shape.d_model, self.spec.n_probes)

    def stats(self) -> esp_stats:
        return esp_get_stats(self.h)

    def close(self):
        if self.h is not None:
            esp_free(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
