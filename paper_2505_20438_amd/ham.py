"""Thin ctypes binding of libham (include/ham.h): argument marshalling only.

Every step of the decode loop runs in the library's HIP kernels; this module
passes device pointers (from torch tensors) and the caller's HIP stream.
It fails loudly when the compiled library is missing: there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libham.so")

HAM_OK, HAM_EINVAL, HAM_ENOMEM, HAM_EHIP, HAM_ESTATE, HAM_ECAP = 0, -1, -2, -3, -4, -5
HAM_F32, HAM_BF16 = 0, 1
HAM_STOP_HEAD, HAM_STOP_TOKEN, HAM_STOP_FORCED, HAM_STOP_FORCED_TOKEN = 0, 1, 2, 3

(HAM_PROF_QKV, HAM_PROF_O, HAM_PROF_GU, HAM_PROF_DOWN, HAM_PROF_MICRO, HAM_PROF_EMBED, HAM_PROF_HEAD0, HAM_PROF_HEADK,
 HAM_PROF_ATTN, HAM_PROF_NORM) = range(10)
HAM_PROF_KINDS = 10
HAM_KV8_BLOCK = 32

EXPORTED = ("ham_weights_bytes", "ham_state_bytes", "ham_workspace_bytes", "ham_init_weights",
            "ham_prefill", "ham_prefill_embeds", "ham_state_info", "ham_macro_step", "ham_kv_stats", "ham_set_debug", "ham_steps_done",
            "ham_tensor_info", "ham_set_graph", "ham_profile", "ham_profile_read", "ham_last_error", "ham_destroy",
            "ham_op_attention_workspace_bytes", "ham_op_decode_attention", "ham_op_attention_step",
            "ham_op_attention_step_splits", "ham_state_save", "ham_state_restore", "ham_op_attention_step_noalloc",
            "ham_op_attention_step_noalloc_max_bytes", "ham_op_kv8_cache_bytes", "ham_op_kv8_workspace_bytes",
            "ham_op_kv8_info", "ham_op_kv8_append", "ham_op_kv8_pack", "ham_op_kv8_select", "ham_op_kv8_attention",
            "ham_op_paged_pool_bytes", "ham_op_paged_workspace_bytes", "ham_op_paged_append", "ham_op_paged_attention",
            "ham_op_paged_prompt", "ham_op_paged_advance", "ham_op_paged_compact")


class HamConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "ffn_dim", "vocab",
        "embed_layers", "micro_layers", "max_group", "n_ctx_layers")] + [
        ("ctx_layers", ctypes.c_int32 * 8)] + [(n, ctypes.c_int32) for n in ("stop_mode", "stop_id")] + [
        ("stop_conf", ctypes.c_float), ("rope_theta", ctypes.c_float), ("norm_eps", ctypes.c_float),
        ("dtype", ctypes.c_int32), ("max_batch", ctypes.c_int32), ("max_prompt", ctypes.c_int32),
        ("max_steps", ctypes.c_int32)]


class HamKvStats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "kv_len", "prompt_slots", "gen_slots", "tokens", "groups", "done")] + [
        ("len_hist", ctypes.c_int32 * 5), ("device_error", ctypes.c_int32)]

    def as_dict(self) -> dict:
        d = {n: getattr(self, n) for n, _ in self._fields_ if n != "len_hist"}
        d["len_hist"] = list(self.len_hist)
        return d


class HamProfT(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_int32), ("ms", ctypes.c_double), ("bytes", ctypes.c_double)]


class HamKv8Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "rows", "n_heads", "n_kv_heads", "head_dim", "slots_cap")]


class HamPagedShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "rows", "n_heads", "n_kv_heads", "head_dim", "page_slots", "n_pages",
                                              "row_pages")]


class HamError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libham error {code}: {msg}")
        self.code = code


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libham.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: build it with `python -m paper_2505_20438_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32, SZ, U64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_uint64
    cfgp = ctypes.POINTER(HamConfig)
    for n in ("ham_weights_bytes", "ham_state_bytes", "ham_workspace_bytes"):
        getattr(lib, n).argtypes = [cfgp]
        getattr(lib, n).restype = SZ
    lib.ham_init_weights.argtypes = [cfgp, U64, P, SZ, P, SZ, P, SZ, P, ctypes.POINTER(P)]
    lib.ham_prefill.argtypes = [P, I32, P, I32, P, P, P, P, P]
    lib.ham_prefill_embeds.argtypes = [P, I32, P, P, I32, P, P, P, P, P]
    lib.ham_state_info.argtypes = [cfgp, I32, ctypes.POINTER(SZ), ctypes.POINTER(SZ), ctypes.POINTER(I32)]
    lib.ham_macro_step.argtypes = [P, P, P, P, P]
    lib.ham_kv_stats.argtypes = [P, ctypes.POINTER(HamKvStats)]
    lib.ham_set_debug.argtypes = [P, P, SZ]
    lib.ham_steps_done.argtypes = [P]
    lib.ham_tensor_info.argtypes = [cfgp, I32, ctypes.POINTER(SZ)] + [ctypes.POINTER(I32)] * 6
    lib.ham_profile.argtypes = [P, I32]
    lib.ham_set_graph.argtypes = [P, I32]
    lib.ham_profile_read.argtypes = [P, ctypes.POINTER(HamProfT), I32]
    lib.ham_op_attention_workspace_bytes.argtypes = [I32, I32, I32, I32]
    lib.ham_op_attention_workspace_bytes.restype = SZ
    lib.ham_op_decode_attention.argtypes = [I32, I32, I32, I32, I32, I32, P, P, P, P, P, I32, P, P, SZ, P]
    lib.ham_op_decode_attention.restype = I32
    lib.ham_op_attention_step.argtypes = [I32, I32, I32, I32, I32, I32, P, P, P, P, P, P, P, P, I32, P, P, P, SZ, P]
    lib.ham_op_attention_step.restype = I32
    lib.ham_op_attention_step_noalloc.argtypes = [I32, I32, I32, I32, I32, I32, P, P, P, P, P, P, P, P, I32, P, P, P]
    lib.ham_op_attention_step_noalloc.restype = I32
    lib.ham_op_attention_step_noalloc_max_bytes.argtypes = []
    lib.ham_op_attention_step_noalloc_max_bytes.restype = SZ
    lib.ham_op_attention_step_splits.argtypes = [I32, I32, I32, I32, I32]
    lib.ham_op_attention_step_splits.restype = I32
    k8 = ctypes.POINTER(HamKv8Shape)
    for n in ("ham_op_kv8_cache_bytes", "ham_op_kv8_workspace_bytes"):
        getattr(lib, n).argtypes = [k8]
        getattr(lib, n).restype = SZ
    lib.ham_op_kv8_info.argtypes = [k8] + [ctypes.POINTER(SZ)] * 4
    lib.ham_op_kv8_append.argtypes = [k8, I32, P, P, P, P, P, P, SZ, P, P, P]
    lib.ham_op_kv8_pack.argtypes = [k8, P, P, I32, P, I32, P, SZ, P, P]
    lib.ham_op_kv8_select.argtypes = [k8, P, P, SZ, P, P, I32, I32, I32, I32, P, P, P, P, SZ, P]
    lib.ham_op_kv8_attention.argtypes = [k8, P, P, SZ, P, P, I32, P, P, I32, P, P, P, SZ, P]
    pg = ctypes.POINTER(HamPagedShape)
    for n in ("ham_op_paged_pool_bytes", "ham_op_paged_workspace_bytes"):
        getattr(lib, n).argtypes = [pg]
        getattr(lib, n).restype = SZ
    lib.ham_op_paged_append.argtypes = [pg, I32, P, P, P, P, P, P, P, SZ, P, P, P]
    lib.ham_op_paged_attention.argtypes = [pg, P, P, SZ, P, P, P, I32, P, P, P, SZ, P]
    lib.ham_op_paged_prompt.argtypes = [pg, I32, P, P, P, SZ, P, P, I32, P, P, P, SZ, P]
    lib.ham_op_paged_advance.argtypes = [pg, I32, P, P, P, P, P, P, P, SZ, P, P, SZ, P]
    lib.ham_op_paged_compact.argtypes = [pg, I32, P, P, P, P, SZ, P, P, P, P, SZ, P]
    lib.ham_state_save.argtypes = [P, P, SZ]
    lib.ham_state_restore.argtypes = [P, P, SZ]
    lib.ham_last_error.restype = ctypes.c_char_p
    lib.ham_destroy.argtypes = [P]
    lib.ham_destroy.restype = None
    for n in ("ham_init_weights", "ham_prefill", "ham_prefill_embeds", "ham_state_info", "ham_macro_step", "ham_kv_stats", "ham_set_debug",
              "ham_steps_done", "ham_tensor_info", "ham_set_graph", "ham_profile", "ham_profile_read",
              "ham_state_save", "ham_state_restore", "ham_op_kv8_info", "ham_op_kv8_append", "ham_op_kv8_pack",
              "ham_op_kv8_select", "ham_op_kv8_attention", "ham_op_paged_append", "ham_op_paged_attention", "ham_op_paged_prompt",
              "ham_op_paged_advance", "ham_op_paged_compact"):
        getattr(lib, n).restype = I32
    _lib = lib
    return lib


def check(rc: int) -> None:
    if rc != HAM_OK:
        raise HamError(rc, load_library().ham_last_error().decode())


_check = check


def make_config(**kw) -> HamConfig:
    c = HamConfig()
    defaults = dict(embed_layers=1, max_group=4, stop_mode=HAM_STOP_FORCED, stop_id=0, stop_conf=0.5,
                    rope_theta=500000.0, norm_eps=1e-5, dtype=HAM_BF16, max_batch=1, max_prompt=1, max_steps=0,
                    ctx_layers=())
    defaults.update(kw)
    layers = [int(x) for x in defaults.pop("ctx_layers")]
    if len(layers) > 8:
        raise ValueError("at most 8 context layers")
    c.n_ctx_layers = len(layers)
    for i, l in enumerate(layers):
        c.ctx_layers[i] = l
    for k, v in defaults.items():
        setattr(c, k, v)
    return c


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def ham_weights_bytes(cfg: HamConfig) -> int:
    return load_library().ham_weights_bytes(ctypes.byref(cfg))


def ham_state_bytes(cfg: HamConfig) -> int:
    return load_library().ham_state_bytes(ctypes.byref(cfg))


def ham_workspace_bytes(cfg: HamConfig) -> int:
    return load_library().ham_workspace_bytes(ctypes.byref(cfg))


def ham_tensor_info(cfg: HamConfig, tensor_id: int) -> dict:
    off = ctypes.c_size_t()
    v = [ctypes.c_int32() for _ in range(6)]
    _check(load_library().ham_tensor_info(ctypes.byref(cfg), tensor_id, ctypes.byref(off),
                                          *[ctypes.byref(x) for x in v]))
    keys = ("rows", "cols", "row_off", "mat_rows", "interleave", "tiled")
    d = {k: x.value for k, x in zip(keys, v)}
    d["offset"] = off.value
    return d


def ham_init_weights(cfg: HamConfig, seed: int, weights, state, workspace, stream: int) -> int:
    h = ctypes.c_void_p()
    _check(load_library().ham_init_weights(
        ctypes.byref(cfg), seed, weights.data_ptr(), weights.numel() * weights.element_size(), state.data_ptr(),
        state.numel() * state.element_size(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        stream, ctypes.byref(h)))
    return h.value


def ham_prefill(model: int, batch: int, prompt, prompt_len: int, max_new: Sequence[int], forced=None,
                teacher=None, out_tokens=None, out_lens=None) -> None:
    arr = (ctypes.c_int32 * batch)(*[int(x) for x in max_new])
    _check(load_library().ham_prefill(model, batch, _ptr(prompt), prompt_len, arr, _ptr(forced), _ptr(teacher),
                                      _ptr(out_tokens), _ptr(out_lens)))


def ham_prefill_embeds(model: int, embeds, positions, max_new: Sequence[int], forced=None, teacher=None,
                       out_tokens=None, out_lens=None) -> None:
    """embeds: fp32 [batch][n][d_model], positions: int32 [batch][n] (device tensors)."""
    batch, n = int(embeds.shape[0]), int(embeds.shape[1])
    arr = (ctypes.c_int32 * batch)(*[int(x) for x in max_new])
    _check(load_library().ham_prefill_embeds(model, batch, _ptr(embeds), _ptr(positions), n, arr, _ptr(forced),
                                             _ptr(teacher), _ptr(out_tokens), _ptr(out_lens)))


def ham_state_info(cfg: HamConfig, layer: int) -> dict:
    k, v, s = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_int32()
    _check(load_library().ham_state_info(ctypes.byref(cfg), layer, ctypes.byref(k), ctypes.byref(v),
                                         ctypes.byref(s)))
    return {"k_offset": k.value, "v_offset": v.value, "slots": s.value}


def ham_macro_step(model: int, forced=None, teacher=None, out_tokens=None, out_lens=None) -> None:
    _check(load_library().ham_macro_step(model, _ptr(forced), _ptr(teacher), _ptr(out_tokens), _ptr(out_lens)))


def ham_kv_stats(model: int, batch: int) -> List[dict]:
    out = (HamKvStats * batch)()
    _check(load_library().ham_kv_stats(model, out))
    return [o.as_dict() for o in out]


def ham_set_debug(model: int, buf) -> None:
    _check(load_library().ham_set_debug(model, _ptr(buf), 0 if buf is None else buf.numel() * buf.element_size()))


def ham_op_decode_attention(dtype: int, q, k, vt, kv_len, enable, kv_max: int, out, workspace, stream: int,
                            n_heads: int, n_kv_heads: int, head_dim: int, slots_cap: int) -> None:
    """Decode attention of one act row per sequence (include/ham_ops.h)."""
    rows = kv_len.numel()
    check(load_library().ham_op_decode_attention(
        dtype, rows, n_heads, n_kv_heads, head_dim, slots_cap, q.data_ptr(), k.data_ptr(), vt.data_ptr(),
        kv_len.data_ptr(), enable.data_ptr(), kv_max, out.data_ptr(), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), stream))


def ham_op_attention_step(dtype: int, qkv, cos, sin, k, vt, kv_len, new_slot, enable, kv_cap: int, err, out,
                          workspace, stream: int, n_heads: int, n_kv_heads: int, head_dim: int,
                          slots_cap: int) -> None:
    """Fused decode-attention step of one base layer, one row per sequence (include/ham_ops.h)."""
    rows = kv_len.numel()
    check(load_library().ham_op_attention_step(
        dtype, rows, n_heads, n_kv_heads, head_dim, slots_cap, qkv.data_ptr(), cos.data_ptr(), sin.data_ptr(),
        k.data_ptr(), vt.data_ptr(), kv_len.data_ptr(), new_slot.data_ptr(), enable.data_ptr(), kv_cap,
        err.data_ptr(), out.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(), stream))


def ham_op_attention_step_noalloc(dtype: int, qkv, cos, sin, k, vt, kv_len, new_slot, enable, kv_cap: int, err,
                                  out, stream: int, n_heads: int, n_kv_heads: int, head_dim: int,
                                  slots_cap: int) -> None:
    """ham_op_attention_step with its split records in the library's own device array."""
    rows = kv_len.numel()
    check(load_library().ham_op_attention_step_noalloc(
        dtype, rows, n_heads, n_kv_heads, head_dim, slots_cap, qkv.data_ptr(), cos.data_ptr(), sin.data_ptr(),
        k.data_ptr(), vt.data_ptr(), kv_len.data_ptr(), new_slot.data_ptr(), enable.data_ptr(), kv_cap,
        err.data_ptr(), out.data_ptr(), stream))


def ham_op_attention_step_splits(dtype: int, rows: int, n_kv_heads: int, head_dim: int, kv_cap: int) -> int:
    return load_library().ham_op_attention_step_splits(dtype, rows, n_kv_heads, head_dim, kv_cap)


def ham_op_attention_workspace_bytes(rows: int, n_heads: int, n_kv_heads: int, head_dim: int) -> int:
    return load_library().ham_op_attention_workspace_bytes(rows, n_heads, n_kv_heads, head_dim)


def kv8_shape(dtype: int, rows: int, n_heads: int, n_kv_heads: int, head_dim: int, slots_cap: int) -> HamKv8Shape:
    """Shape of a layer's KV cache in 8 bits (include/ham_ops.h)."""
    return HamKv8Shape(dtype, rows, n_heads, n_kv_heads, head_dim, slots_cap)


def ham_op_kv8_cache_bytes(shape: HamKv8Shape) -> int:
    return load_library().ham_op_kv8_cache_bytes(ctypes.byref(shape))


def ham_op_kv8_workspace_bytes(shape: HamKv8Shape) -> int:
    return load_library().ham_op_kv8_workspace_bytes(ctypes.byref(shape))


def ham_op_kv8_info(shape: HamKv8Shape) -> dict:
    v = [ctypes.c_size_t() for _ in range(4)]
    _check(load_library().ham_op_kv8_info(ctypes.byref(shape), *[ctypes.byref(x) for x in v]))
    return {k: x.value for k, x in zip(("codes", "scales", "bounds", "open"), v)}


def _current_device() -> int:
    import torch
    return torch._C._cuda_getDevice()   # of a process that holds a tensor on a GPU


def _rows_as_read(t, rows: int, need: int) -> bool:
    """Whether a tensor of another size than the call's `need` bytes holds more rows of the same extent: a call reads row r
    at r * need / rows, which in a tensor of longer rows is another place."""
    return t.nbytes > need and t.dim() > 0 and t.nbytes * rows == need * t.shape[0]


def _fits(rows: int, tensors) -> bool:
    """Whether tensors hold what a call reads and writes of them: (tensor, bytes of `rows` rows or 0 for any number, bytes of a
    value or 0 for any), on the current device, packed, and rows where the call expects them."""
    device = tensors[0][0].get_device()
    for t, need, size in tensors:
        if (need and t.nbytes != need and not _rows_as_read(t, rows, need) or size and t.itemsize != size
                or t.get_device() != device or not t.is_contiguous()):
            return False
    return device >= 0 and device == _current_device()


def _refuse(rows: int, names: str, tensors) -> None:
    for name, (t, need, size) in zip(names.split(), tensors):
        if size and t.itemsize != size:
            raise HamError(HAM_EINVAL, f"{name} holds values of {t.itemsize} bytes, the call reads {size}")
        if need and t.nbytes != need and not _rows_as_read(t, rows, need):
            raise HamError(HAM_EINVAL, f"{name} holds {t.nbytes} bytes, the call needs {need} ({rows} rows, or more of the same extent)")
        if not t.is_contiguous():
            raise HamError(HAM_EINVAL, f"{name} must be contiguous")
    for name, (t, _, _) in zip(names.split(), tensors):
        if not t.is_cuda:
            raise HamError(HAM_EINVAL, f"{name} must be on a GPU")
        if t.get_device() != _current_device():
            raise HamError(HAM_EINVAL, f"{name} must be on the current device")


@functools.lru_cache(None)
def _types(dtype: int):
    """Types of fp32, int32 and stored values."""
    import torch
    return torch.float32, torch.int32, torch.bfloat16 if dtype == HAM_BF16 else torch.float32


def _fits_exactly(tensors) -> bool:
    """_fits of tensors that hold just what the call reads and writes: (tensor, bytes or 0 for any number, type or None for any)."""
    device = tensors[0][0].get_device()
    for t, need, kind in tensors:
        if need and t.nbytes != need or kind and t.dtype is not kind or t.get_device() != device or not t.is_contiguous():
            return False
    return device >= 0 and device == _current_device()


def _refuse_inexact(names: str, tensors) -> None:
    for name, (t, need, kind) in zip(names.split(), tensors):
        if need and t.nbytes != need:
            raise HamError(HAM_EINVAL, f"{name} holds {t.nbytes} bytes, the call needs {need}")
        if kind and t.dtype is not kind:
            raise HamError(HAM_EINVAL, f"{name} holds values of {t.dtype}, the call reads {kind}")
    _refuse(1, names, [(t, need, 0) for t, need, _ in tensors])


def ham_op_kv8_append(shape: HamKv8Shape, qkv, cos, sin, start, count, cache, q, err, stream: int, n_tokens=None) -> None:
    """RoPE and append of ``count[r]`` slots per row (include/ham_ops.h): qkv fp32 [rows][n_tokens][...], q act rows of
    the same tokens or None.  ``n_tokens`` is taken from qkv if not given: its first dimension is then ``rows``."""
    rows, hd, H = shape.rows, shape.head_dim, shape.n_heads
    width = (H + 2 * shape.n_kv_heads) * hd
    n = n_tokens
    if n is None:
        if qkv.dim() == 0 or qkv.shape[0] != rows:
            raise HamError(HAM_EINVAL, f"qkv's first dimension must be the {rows} rows, or n_tokens given")
        n = qkv.numel() // (rows * width or 1)
    rope, act, i4 = rows * n * hd * 2, rows * n * H * hd * 4, 4 * rows   # act rows: fp32, or a bf16 hi/lo pair
    es = 2 if shape.dtype == HAM_BF16 else 4
    args = ((qkv, rows * n * width * 4, 4), (cos, rope, 4), (sin, rope, 4), (start, i4, 4), (count, i4, 4), (cache, 0, 0), (err, i4, 4))
    if q is not None:
        args += ((q, act, es),)
    if not _fits(rows, args):
        _refuse(rows, "qkv cos sin start count cache err q", args)
    _check(load_library().ham_op_kv8_append(
        ctypes.byref(shape), n, qkv.data_ptr(), cos.data_ptr(), sin.data_ptr(), start.data_ptr(), count.data_ptr(),
        cache.data_ptr(), cache.nbytes, None if q is None else q.data_ptr(), err.data_ptr(), stream))


def ham_op_kv8_pack(shape: HamKv8Shape, k, vt, kv_len, kv_max: int, cache, err, stream: int, src_slots=None) -> None:
    """A filled cache of the storage type, k [rows][n_kv_heads][slots][head_dim] and vt its V tiles, into 8 bits.
    ``src_slots`` (slots of a row of k and vt) is taken from k's dimensions if not given; of a k without them (a flat view of
    a state buffer) it is the shape's slots_cap."""
    rows, Hk, hd = shape.rows, shape.n_kv_heads, shape.head_dim
    pairs, slots = rows * Hk, src_slots
    if slots is None:
        if k.dim() >= 4 and k.shape[1] == Hk:
            slots = k.numel() // (k.shape[0] * Hk * hd or 1)
        else:
            slots = k.shape[1] if k.dim() == 3 and k.shape[0] == pairs else shape.slots_cap
    es = 2 if shape.dtype == HAM_BF16 else 4
    need, i4 = pairs * slots * hd * es, 4 * rows
    args = ((k, need, es), (vt, need, es), (kv_len, i4, 4), (cache, 0, 0), (err, i4, 4))
    if not _fits(rows, args):
        _refuse(rows, "k vt kv_len cache err", args)
    _check(load_library().ham_op_kv8_pack(
        ctypes.byref(shape), k.data_ptr(), vt.data_ptr(), slots, kv_len.data_ptr(), kv_max, cache.data_ptr(), cache.nbytes,
        err.data_ptr(), stream))


def ham_op_kv8_select(shape: HamKv8Shape, q, cache, kv_len, enable, kv_max: int, n_blocks: int, keep_first: int,
                      keep_last: int, blocks, count, err, workspace, stream: int) -> None:
    """The ``n_blocks`` closed blocks of each (row, kv head) with the greatest bounds of q . k, ascending, into ``blocks``
    int32 [rows][n_kv_heads][n_blocks]; how many into ``count`` int32 [rows][n_kv_heads]."""
    i4, act = 4 * shape.rows, shape.rows * shape.n_heads * shape.head_dim * 4
    lists, counts = i4 * shape.n_kv_heads * n_blocks, i4 * shape.n_kv_heads
    es = 2 if shape.dtype == HAM_BF16 else 4
    args = ((q, act, es), (cache, 0, 0), (kv_len, i4, 4), (enable, i4, 4), (blocks, lists, 4), (count, counts, 4), (err, i4, 4),
            (workspace, 0, 0))
    if not _fits(shape.rows, args):
        _refuse(shape.rows, "q cache kv_len enable blocks count err workspace", args)
    _check(load_library().ham_op_kv8_select(
        ctypes.byref(shape), q.data_ptr(), cache.data_ptr(), cache.nbytes, kv_len.data_ptr(), enable.data_ptr(), kv_max,
        n_blocks, keep_first, keep_last, blocks.data_ptr(), count.data_ptr(), err.data_ptr(), workspace.data_ptr(),
        workspace.nbytes, stream))


def ham_op_kv8_attention(shape: HamKv8Shape, q, cache, kv_len, enable, kv_max: int, blocks, count, out, err, workspace,
                         stream: int) -> None:
    """Attention of one act row per sequence over an 8-bit cache: every block, or those of ``blocks`` [rows][n_kv_heads][most]
    and ``count`` (ham_op_kv8_select), and the open one."""
    i4, act, pairs = 4 * shape.rows, shape.rows * shape.n_heads * shape.head_dim * 4, shape.rows * shape.n_kv_heads
    es = 2 if shape.dtype == HAM_BF16 else 4
    args = ((q, act, es), (cache, 0, 0), (kv_len, i4, 4), (enable, i4, 4), (out, act, es), (err, i4, 4), (workspace, 0, 0))
    most = 0
    if blocks is not None:
        most = blocks.shape[-1] if blocks.dim() else 0
        args += ((blocks, 4 * pairs * most, 4),)
    if count is not None:
        args += ((count, 4 * pairs, 4),)
    if not _fits(shape.rows, args):
        _refuse(shape.rows, "q cache kv_len enable out err workspace" + ("" if blocks is None else " blocks") + " count", args)
    _check(load_library().ham_op_kv8_attention(
        ctypes.byref(shape), q.data_ptr(), cache.data_ptr(), cache.nbytes, kv_len.data_ptr(), enable.data_ptr(), kv_max,
        None if blocks is None else blocks.data_ptr(), None if count is None else count.data_ptr(), most, out.data_ptr(),
        err.data_ptr(), workspace.data_ptr(), workspace.nbytes, stream))


def paged_shape(dtype: int, rows: int, n_heads: int, n_kv_heads: int, head_dim: int, page_slots: int, n_pages: int,
                row_pages: int) -> HamPagedShape:
    """Shape of a paged KV cache (include/ham_ops.h): ``n_pages`` pages of the pool, tables of ``row_pages`` entries."""
    return HamPagedShape(dtype, rows, n_heads, n_kv_heads, head_dim, page_slots, n_pages, row_pages)


def ham_op_paged_pool_bytes(shape: HamPagedShape) -> int:
    """Bytes of one layer's pool."""
    return load_library().ham_op_paged_pool_bytes(ctypes.byref(shape))


def ham_op_paged_workspace_bytes(shape: HamPagedShape) -> int:
    return load_library().ham_op_paged_workspace_bytes(ctypes.byref(shape))


def _pool_bytes(shape: HamPagedShape, layers: int = 1) -> int:
    """Bytes that a call takes `pool` to hold: a pool of more pages would have its layers elsewhere."""
    return layers * shape.n_pages * shape.n_kv_heads * 2 * shape.page_slots * shape.head_dim * (2 if shape.dtype == HAM_BF16 else 4)


def ham_op_paged_append(shape: HamPagedShape, qkv, cos, sin, offsets, start, table, pool, q, err, stream: int) -> None:
    """RoPE of packed projection rows, fp32 [n_tokens][...], and the append of their K and V to a layer's pool
    (include/ham_ops.h): row r's tokens offsets[r] .. offsets[r + 1] - 1 become slots start[r] ..; q act rows of the same tokens or
    None."""
    rows, hd, H = shape.rows, shape.head_dim, shape.n_heads
    n = qkv.shape[0] if qkv.dim() else 0
    i4, (f32, i32, kind) = 4 * rows, _types(shape.dtype)
    args = ((qkv, n * (H + 2 * shape.n_kv_heads) * hd * 4, f32), (cos, n * hd * 2, f32), (sin, n * hd * 2, f32), (offsets, i4 + 4, i32),
            (start, i4, i32), (table, i4 * shape.row_pages, i32), (pool, _pool_bytes(shape), kind), (err, i4, i32))
    if q is not None:
        args += ((q, n * H * hd * 4, kind),)
    if not _fits_exactly(args):
        _refuse_inexact("qkv cos sin offsets start table pool err q", args)
    _check(load_library().ham_op_paged_append(
        ctypes.byref(shape), n, qkv.data_ptr(), cos.data_ptr(), sin.data_ptr(), offsets.data_ptr(), start.data_ptr(), table.data_ptr(),
        pool.data_ptr(), pool.nbytes, None if q is None else q.data_ptr(), err.data_ptr(), stream))


def ham_op_paged_attention(shape: HamPagedShape, q, pool, table, kv_len, enable, kv_max: int, out, err, workspace, stream: int) -> None:
    """Attention of one act row per sequence over its pages of a layer's pool."""
    i4, act, (_, i32, kind) = 4 * shape.rows, shape.rows * shape.n_heads * shape.head_dim * 4, _types(shape.dtype)
    args = ((q, act, kind), (pool, _pool_bytes(shape), kind), (table, i4 * shape.row_pages, i32), (kv_len, i4, i32), (enable, i4, i32),
            (out, act, kind), (err, i4, i32), (workspace, 0, None))
    if not _fits_exactly(args):
        _refuse_inexact("q pool table kv_len enable out err workspace", args)
    _check(load_library().ham_op_paged_attention(
        ctypes.byref(shape), q.data_ptr(), pool.data_ptr(), pool.nbytes, table.data_ptr(), kv_len.data_ptr(), enable.data_ptr(), kv_max,
        out.data_ptr(), err.data_ptr(), workspace.data_ptr(), workspace.nbytes, stream))


def ham_op_paged_prompt(shape: HamPagedShape, q, offsets, pool, table, kv_len, kv_max: int, out, err, workspace, stream: int) -> None:
    """Causal attention of packed act rows, the last offsets[r + 1] - offsets[r] of the kv_len[r] slots of each row, over their
    pages of a layer's pool."""
    i4, n = 4 * shape.rows, q.shape[0] if q.dim() else 0
    act, (_, i32, kind) = n * shape.n_heads * shape.head_dim * 4, _types(shape.dtype)
    args = ((q, act, kind), (offsets, i4 + 4, i32), (pool, _pool_bytes(shape), kind), (table, i4 * shape.row_pages, i32), (kv_len, i4, i32),
            (out, act, kind), (err, i4, i32), (workspace, 0, None))
    if not _fits_exactly(args):
        _refuse_inexact("q offsets pool table kv_len out err workspace", args)
    _check(load_library().ham_op_paged_prompt(
        ctypes.byref(shape), n, q.data_ptr(), offsets.data_ptr(), pool.data_ptr(), pool.nbytes, table.data_ptr(), kv_len.data_ptr(),
        kv_max, out.data_ptr(), err.data_ptr(), workspace.data_ptr(), workspace.nbytes, stream))


def ham_op_paged_advance(shape: HamPagedShape, n_layers: int, parent, count, kv_len, start, table, refs, pool, err, workspace,
                         stream: int) -> None:
    """Rows take over the pages of rows ``parent`` (or None: their own), then get ``count`` more slots, or fewer; in place.
    ``pool`` holds n_layers layers' pools."""
    i4, i32 = 4 * shape.rows, _types(shape.dtype)[1]
    args = ((count, i4, i32), (kv_len, i4, i32), (start, i4, i32), (table, i4 * shape.row_pages, i32), (refs, 4 * shape.n_pages, i32),
            (pool, _pool_bytes(shape, n_layers), None), (err, i4, i32), (workspace, 0, None))
    if parent is not None:
        args += ((parent, i4, i32),)
    if not _fits_exactly(args):
        _refuse_inexact("count kv_len start table refs pool err workspace parent", args)
    _check(load_library().ham_op_paged_advance(
        ctypes.byref(shape), n_layers, None if parent is None else parent.data_ptr(), count.data_ptr(), kv_len.data_ptr(),
        start.data_ptr(), table.data_ptr(), refs.data_ptr(), pool.data_ptr(), pool.nbytes, err.data_ptr(), workspace.data_ptr(),
        workspace.nbytes, stream))


def ham_op_paged_compact(shape: HamPagedShape, n_layers: int, kv_len, table, refs, pool, map, used, err, workspace, stream: int) -> None:
    """Pages in use to the front of the pool: ``map`` int32 [n_pages] their new places, ``used`` int32 [1] their number."""
    i4, i32 = 4 * shape.rows, _types(shape.dtype)[1]
    args = ((kv_len, i4, i32), (table, i4 * shape.row_pages, i32), (refs, 4 * shape.n_pages, i32),
            (pool, _pool_bytes(shape, n_layers), None), (map, 4 * shape.n_pages, i32), (used, 4, i32), (err, i4, i32), (workspace, 0, None))
    if not _fits_exactly(args):
        _refuse_inexact("kv_len table refs pool map used err workspace", args)
    _check(load_library().ham_op_paged_compact(
        ctypes.byref(shape), n_layers, kv_len.data_ptr(), table.data_ptr(), refs.data_ptr(), pool.data_ptr(), pool.nbytes, map.data_ptr(),
        used.data_ptr(), err.data_ptr(), workspace.data_ptr(), workspace.nbytes, stream))


def ham_steps_done(model: int) -> int:
    return load_library().ham_steps_done(model)


def ham_destroy(model: int) -> None:
    load_library().ham_destroy(model)


class HamRuntime:
    """Allocates the library's three buffers as torch tensors on one device and
    binds them (``ham_init_weights``).  Device memory and the stream are torch's;
    the computation is the library's."""

    def __init__(self, cfg: HamConfig, seed: int, device: str = "cuda:0", stream=None):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        self.stream = stream or torch.cuda.current_stream(self.device)
        nb = [ham_weights_bytes(cfg), ham_state_bytes(cfg), ham_workspace_bytes(cfg)]
        if 0 in nb:
            raise HamError(HAM_EINVAL, "invalid configuration")
        self.weights, self.state, self.workspace = (
            torch.empty(n, dtype=torch.uint8, device=self.device) for n in nb)
        self.handle = ham_init_weights(cfg, seed, self.weights, self.state, self.workspace,
                                       self.stream.cuda_stream)
        B = cfg.max_batch
        self.out_tokens = torch.full((B, 4), -1, dtype=torch.int32, device=self.device)
        self.out_lens = torch.zeros(B, dtype=torch.int32, device=self.device)
        self.batch = 0

    def prefill(self, prompt, max_new, forced=None, teacher=None):
        self.batch = prompt.shape[0]
        ham_prefill(self.handle, prompt.shape[0], prompt, prompt.shape[1], max_new, forced, teacher,
                    self.out_tokens, self.out_lens)

    def prefill_embeds(self, embeds, positions, max_new, forced=None, teacher=None):
        self.batch = embeds.shape[0]
        ham_prefill_embeds(self.handle, embeds, positions, max_new, forced, teacher, self.out_tokens, self.out_lens)

    def kv_cache(self, layer: int, n_slots: int):
        """K and V of base layer ``layer``, slots [0, n_slots) of the current batch, as
        float32 [batch][n_kv_heads][n_slots][head_dim] tensors (a copy)."""
        torch = self.torch
        info = ham_state_info(self.cfg, layer)
        c = self.cfg
        es = 2 if c.dtype == HAM_BF16 else 4
        B, Hk, S, hd = c.max_batch, c.n_kv_heads, info["slots"], c.head_dim
        n = B * Hk * S * hd

        def view(off):
            raw = self.state[off: off + n * es]
            if es == 2:  # bf16 bits -> float32
                return (raw.view(torch.int16).to(torch.int32) << 16).view(torch.float32)
            return raw.view(torch.float32)
        K = view(info["k_offset"]).view(B, Hk, S, hd)[: self.batch, :, :n_slots]
        V = view(info["v_offset"]).view(B, Hk, S // 32, hd, 32).permute(0, 1, 2, 4, 3).reshape(B, Hk, S, hd)
        return K.clone(), V[: self.batch, :, :n_slots].clone()

    def macro_step(self, forced=None, teacher=None):
        ham_macro_step(self.handle, forced, teacher, self.out_tokens, self.out_lens)

    def save_state(self, buf) -> None:
        """Copy the decode state (KV cache + counters) into ``buf`` (uint8, >= state bytes)."""
        _check(load_library().ham_state_save(self.handle, buf.data_ptr(), buf.numel() * buf.element_size()))

    def restore_state(self, buf) -> None:
        """Continue from the point of the last save_state (its copy in ``buf``)."""
        _check(load_library().ham_state_restore(self.handle, buf.data_ptr(), buf.numel() * buf.element_size()))

    def set_graph(self, enable: bool) -> None:
        _check(load_library().ham_set_graph(self.handle, 1 if enable else 0))

    def kv_stats(self):
        return ham_kv_stats(self.handle, self.batch)

    def tensor(self, tensor_id: int):
        """A generated tensor [rows][cols] in logical row-major order (bf16 as int16 bits)."""
        torch = self.torch
        t = ham_tensor_info(self.cfg, tensor_id)
        es = 2 if self.cfg.dtype == HAM_BF16 else 4
        dt = torch.int16 if es == 2 else torch.float32
        R, K = t["mat_rows"], t["cols"]
        flat = self.weights[t["offset"]: t["offset"] + R * K * es].view(dt)
        if t["tiled"]:   # undo the fragment tiling: [tile][frag][group][row][elem] -> [tile][row][frag][group][elem]
            epl = 16 // es
            flat = flat.view(R // 16, K // (4 * epl), 4, 16, epl).permute(0, 3, 1, 2, 4)
        mat = flat.reshape(R, K)
        r = torch.arange(t["rows"], device=mat.device)
        if t["interleave"]:
            idx = 16 * (r // 8) + r % 8 + (8 if t["interleave"] == 2 else 0)
        else:
            idx = r + t["row_off"]
        return mat[idx]

    def close(self):
        if self.handle:
            ham_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
