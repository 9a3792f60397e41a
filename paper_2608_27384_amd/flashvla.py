"""ctypes binding of libflashvla (the C ABI declared in include/flashvla.h).

Argument marshalling only: every step of the decode path runs in the HIP
library.  Device tensors are torch tensors (PyTorch provides device memory
and streams); the binding passes their data pointers and the current HIP
stream.  There is no fallback: if the library is missing the import of this
module's functions raises.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import (POINTER, byref, c_char_p, c_float, c_int32, c_int64, c_size_t, c_uint64,
                    c_void_p)
from typing import Dict, Optional, Sequence

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libflashvla.so")

FV_OK, FV_ERR_INVALID_ARG, FV_ERR_STATE, FV_ERR_OOM, FV_ERR_HIP, FV_ERR_INTERNAL = range(6)
FV_BF16, FV_FP32 = 0, 1
FV_QUERY_ATTN_SPLITS, FV_QUERY_DEVICE_BYTES, FV_QUERY_NOALLOC_SCRATCH_BYTES = 1, 2, 3
FV_QUERY_OUT_PROJ_SPLITS = 4
FV_NOALLOC_SCRATCH_BYTES = 24 << 20
FV_MASK_CHUNK_CAUSAL, FV_MASK_ISOLATED, FV_MASK_BIDIRECTIONAL = 0, 1, 2
MASK_MODES = {"causal": FV_MASK_CHUNK_CAUSAL, "isolated": FV_MASK_ISOLATED,
              "bidirectional": FV_MASK_BIDIRECTIONAL}

EXPORTED = (
    "fv_create", "fv_set_prefix", "fv_decode_step", "fv_velocity", "fv_euler_shift",
    "fv_sequential_decode", "fv_get_noise_state", "fv_set_noise_state", "fv_set_graph_mode",
    "fv_destroy", "fv_status_string", "fv_last_error", "fv_abi_version", "fv_debug_forward",
    "fv_debug_stage", "fv_query", "fv_set_mask_mode", "fv_set_schedule", "fv_cold_start",
    "fv_get_valid_slots", "fv_set_valid_slots", "fv_multibuffer_velocity", "fv_set_prefix_async",
    "fv_decode_step_noalloc",
    "fv_rope_append", "fv_prompt_attention", "fv_paged_attention_workspace", "fv_paged_attention",
    "fv_pages_workspace", "fv_pages_grow", "fv_pages_fork", "fv_pages_free", "fv_pages_compact",
    "fv_pages_gather", "fv_context_error",
    "fv_quant_append", "fv_quant_attention_workspace", "fv_quant_attention",
    "fv_quant_part_workspace", "fv_quant_part_attention", "fv_quant_workspace", "fv_quant_grow",
    "fv_quant_fork", "fv_quant_free", "fv_quant_compact", "fv_quant_gather",
)


class FvCfg(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in (
        "n_layers", "width", "n_q_heads", "n_kv_heads", "head_dim", "mlp_dim", "action_dim",
        "chunk_len", "n_chunks", "max_prefix", "max_batch", "dtype", "mlp_gated")] + [
        ("rms_eps", c_float), ("rope_theta", c_float), ("noise_seed", c_uint64)]


class FvWeights(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("w_in", "b_in", "w_t1", "b_t1", "w_t2", "b_t2")] + [
        (n, POINTER(c_void_p)) for n in ("w_mod", "b_mod", "wq", "wk", "wv", "wo", "wg", "wu",
                                         "wd")] + [("w_out", c_void_p), ("b_out", c_void_p)]


class FvPages(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("dtype", "n_layers", "n_kv_heads", "head_dim", "page_len",
                                       "n_pages", "max_seqs", "max_pages")] + [
        (n, c_void_p) for n in ("k", "v", "table", "len", "refs")]


class FvRopeArgs(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("q", "k", "v", "q_out", "k_out")] + [
        (n, c_int32) for n in ("ldq", "ldk", "ldv", "ldq_out", "ldk_out")] + [
        (n, c_void_p) for n in ("pos", "seqs", "at")] + [
        (n, c_int32) for n in ("n", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "layer",
                               "n_axes")] + [("sections", c_int32 * 4), ("theta", c_float)]


class FvPromptArgs(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("q", "k", "v", "out")] + [
        (n, c_int32) for n in ("ldq", "ldk", "ldv", "ldo")] + [
        (n, c_void_p) for n in ("cu_q", "cu_k")] + [
        (n, c_int32) for n in ("n_seqs", "n_q", "n_k", "n_q_heads", "n_kv_heads", "head_dim",
                               "dtype", "causal")] + [("scale", c_float)]


class FvPagedArgs(ctypes.Structure):
    _fields_ = [("q", c_void_p), ("out", c_void_p), ("ldq", c_int32), ("ldo", c_int32),
                ("seqs", c_void_p)] + [
        (n, c_int32) for n in ("n", "n_q_heads", "layer", "max_len")] + [
        ("scale", c_float), ("work", c_void_p), ("work_bytes", c_size_t)]


class FvQuantPages(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("dtype", "n_layers", "n_kv_heads", "head_dim", "page_len",
                                       "n_pages", "max_seqs", "max_pages")] + [
        (n, c_void_p) for n in ("k", "v", "k_scale", "v_scale", "table", "len", "refs")]


class FvPartArgs(ctypes.Structure):
    _fields_ = [("q", c_void_p), ("out", c_void_p), ("ldq", c_int32), ("ldo", c_int32),
                ("cu_q", c_void_p), ("seqs", c_void_p)] + [
        (n, c_int32) for n in ("n_seqs", "n_q", "n_q_heads", "layer", "max_len", "causal")] + [
        ("scale", c_float), ("work", c_void_p), ("work_bytes", c_size_t)]


FV_PAGES_OK, FV_PAGES_BAD, FV_PAGES_FULL = range(3)


class FlashVLAError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libflashvla.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"libflashvla.so not built at {LIB_PATH}; run "
                              "python -m paper_2608_27384_amd.build")
        L = ctypes.CDLL(LIB_PATH)
        H, S = c_void_p, c_int32
        sig = {
            "fv_create": ([POINTER(FvWeights), POINTER(FvCfg), POINTER(c_void_p)], S),
            "fv_set_prefix": ([H, c_void_p, c_void_p, POINTER(c_int32), c_int32, c_int32, c_void_p], S),
            "fv_decode_step": ([H, c_void_p, c_void_p, c_void_p, c_void_p], S),
            "fv_decode_step_noalloc": ([H, c_void_p, c_void_p, c_void_p, c_void_p], S),
            "fv_velocity": ([H, c_void_p, c_void_p, c_void_p, c_void_p], S),
            "fv_euler_shift": ([H, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p], S),
            "fv_sequential_decode": ([H, c_void_p, c_int32, c_void_p, c_void_p], S),
            "fv_get_noise_state": ([H, POINTER(c_uint64), POINTER(c_uint64)], S),
            "fv_set_noise_state": ([H, c_uint64, c_uint64], S),
            "fv_set_graph_mode": ([H, c_int32], S),
            "fv_destroy": ([H], S),
            "fv_status_string": ([S], c_char_p),
            "fv_last_error": ([H], c_char_p),
            "fv_abi_version": ([], c_int32),
            "fv_debug_forward": ([H, c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p], S),
            "fv_debug_stage": ([H, c_int32, c_int32, c_int32, c_void_p], S),
            "fv_query": ([H, c_int32, c_int32, POINTER(c_int64)], S),
            "fv_set_mask_mode": ([H, c_int32], S),
            "fv_set_schedule": ([H, c_void_p, c_void_p], S),
            "fv_cold_start": ([H, c_void_p, c_int32, c_int32, c_void_p], S),
            "fv_get_valid_slots": ([H, POINTER(c_int32), c_int32], S),
            "fv_set_valid_slots": ([H, POINTER(c_int32), c_int32], S),
            "fv_set_prefix_async": ([H, c_void_p, c_void_p, POINTER(c_int32), c_int32, c_int32,
                                     c_void_p], S),
            "fv_multibuffer_velocity": ([H, c_void_p, c_void_p, c_int32, c_int32, c_void_p,
                                         c_void_p, c_void_p, c_void_p], S),
            "fv_rope_append": ([POINTER(FvRopeArgs), POINTER(FvPages), c_void_p], S),
            "fv_prompt_attention": ([POINTER(FvPromptArgs), c_void_p], S),
            "fv_paged_attention_workspace": ([POINTER(FvPagedArgs), POINTER(FvPages),
                                              POINTER(c_size_t)], S),
            "fv_paged_attention": ([POINTER(FvPagedArgs), POINTER(FvPages), c_void_p], S),
            "fv_pages_workspace": ([POINTER(FvPages), POINTER(c_size_t)], S),
            "fv_pages_grow": ([POINTER(FvPages), c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                               c_void_p], S),
            "fv_pages_fork": ([POINTER(FvPages), c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                               c_void_p], S),
            "fv_pages_free": ([POINTER(FvPages), c_void_p, c_int32, c_void_p, c_void_p], S),
            "fv_pages_compact": ([POINTER(FvPages), c_void_p, c_void_p, c_void_p], S),
            "fv_pages_gather": ([POINTER(FvPages), c_void_p, c_int32, c_int32, c_void_p, c_void_p,
                                 c_void_p], S),
            "fv_context_error": ([], c_char_p),
            "fv_quant_append": ([POINTER(FvRopeArgs), POINTER(FvQuantPages), c_void_p], S),
            "fv_quant_attention_workspace": ([POINTER(FvPagedArgs), POINTER(FvQuantPages),
                                              POINTER(c_size_t)], S),
            "fv_quant_attention": ([POINTER(FvPagedArgs), POINTER(FvQuantPages), c_void_p], S),
            "fv_quant_part_workspace": ([POINTER(FvPartArgs), POINTER(FvQuantPages),
                                         POINTER(c_size_t)], S),
            "fv_quant_part_attention": ([POINTER(FvPartArgs), POINTER(FvQuantPages), c_void_p], S),
            "fv_quant_workspace": ([POINTER(FvQuantPages), POINTER(c_size_t)], S),
            "fv_quant_grow": ([POINTER(FvQuantPages), c_void_p, c_void_p, c_int32, c_void_p,
                               c_void_p, c_void_p], S),
            "fv_quant_fork": ([POINTER(FvQuantPages), c_void_p, c_void_p, c_int32, c_void_p,
                               c_void_p, c_void_p], S),
            "fv_quant_free": ([POINTER(FvQuantPages), c_void_p, c_int32, c_void_p, c_void_p], S),
            "fv_quant_compact": ([POINTER(FvQuantPages), c_void_p, c_void_p, c_void_p], S),
            "fv_quant_gather": ([POINTER(FvQuantPages), c_void_p, c_int32, c_int32, c_void_p,
                                 c_void_p, c_void_p], S),
        }
        for name, (args, res) in sig.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, res
        _lib = L
    return _lib


def _check(handle, status: int, what: str) -> None:
    if status != FV_OK:
        msg = lib().fv_last_error(handle) if handle else b""
        txt = lib().fv_status_string(status).decode()
        raise FlashVLAError(status, f"{what}: {txt}: {(msg or b'').decode()}")


def _ptr(x) -> Optional[int]:
    """Device pointer of a torch tensor (or None)."""
    if x is None:
        return None
    return x.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return int(getattr(stream, "cuda_stream", stream))
    import torch
    return int(torch.cuda.current_stream().cuda_stream)


def make_cfg(shape, max_batch: int, max_prefix: int, noise_seed: int = 0) -> FvCfg:
    """fv_cfg from a shape object (attributes named as in fv_cfg)."""
    return FvCfg(n_layers=shape.n_layers, width=shape.width, n_q_heads=shape.n_q_heads,
                 n_kv_heads=shape.n_kv_heads, head_dim=shape.head_dim, mlp_dim=shape.mlp_dim,
                 action_dim=shape.action_dim, chunk_len=shape.chunk_len,
                 n_chunks=shape.n_chunks, max_prefix=max_prefix, max_batch=max_batch,
                 dtype=FV_BF16 if shape.dtype == "bf16" else FV_FP32,
                 mlp_gated=1 if shape.mlp_gated else 0, rms_eps=shape.rms_eps,
                 rope_theta=shape.rope_theta, noise_seed=noise_seed)


class _HostWeights:
    """Keeps contiguous fp32 host arrays alive while fv_create copies them."""

    def __init__(self, w: Dict):
        self.keep = []
        self.s = FvWeights()

        def one(a):
            a = np.ascontiguousarray(a, dtype=np.float32)
            self.keep.append(a)
            return a.ctypes.data

        def many(lst):
            if lst is None:
                return None
            arr = (c_void_p * len(lst))(*[one(a) for a in lst])
            self.keep.append(arr)
            return ctypes.cast(arr, POINTER(c_void_p))

        for k in ("w_in", "b_in", "w_t1", "b_t1", "w_t2", "b_t2", "w_out", "b_out"):
            setattr(self.s, k, one(w[k]))
        for k in ("w_mod", "b_mod", "wq", "wk", "wv", "wo", "wg", "wu", "wd"):
            p = many(w.get(k))
            if p is not None:
                setattr(self.s, k, p)


# ------------------------------------------------------------- C-ABI names

def fv_create(weights: Dict, cfg: FvCfg) -> int:
    hw = _HostWeights(weights)
    h = c_void_p()
    st = lib().fv_create(ctypes.byref(hw.s), ctypes.byref(cfg), ctypes.byref(h))
    if st != FV_OK:
        raise FlashVLAError(st, "fv_create: " + lib().fv_status_string(st).decode())
    return h.value


def fv_set_prefix(h, k, v, lengths: Sequence[int], ld: int, stream=None) -> None:
    lens = (c_int32 * len(lengths))(*[int(x) for x in lengths])
    _check(h, lib().fv_set_prefix(h, _ptr(k), _ptr(v), lens, len(lengths), ld, _stream(stream)),
           "fv_set_prefix")


def fv_set_prefix_async(h, k, v, lengths: Sequence[int], ld: int, copy_stream) -> None:
    lens = (c_int32 * len(lengths))(*[int(x) for x in lengths])
    _check(h, lib().fv_set_prefix_async(h, _ptr(k), _ptr(v), lens, len(lengths), ld,
                                        _stream(copy_stream)), "fv_set_prefix_async")


def fv_decode_step(h, buffer, t, out_chunk, stream=None) -> None:
    _check(h, lib().fv_decode_step(h, _ptr(buffer), _ptr(t), _ptr(out_chunk), _stream(stream)),
           "fv_decode_step")


def fv_decode_step_noalloc(h, buffer, t, out_chunk, stream=None) -> None:
    _check(h, lib().fv_decode_step_noalloc(h, _ptr(buffer), _ptr(t), _ptr(out_chunk),
                                           _stream(stream)), "fv_decode_step_noalloc")


def fv_velocity(h, buffer, t, v_out, stream=None) -> None:
    _check(h, lib().fv_velocity(h, _ptr(buffer), _ptr(t), _ptr(v_out), _stream(stream)),
           "fv_velocity")


def fv_euler_shift(h, buffer, t, v, out_chunk, stream=None) -> None:
    _check(h, lib().fv_euler_shift(h, _ptr(buffer), _ptr(t), _ptr(v), _ptr(out_chunk),
                                   _stream(stream)), "fv_euler_shift")


def fv_sequential_decode(h, noise, n_steps: int, out_chunk, stream=None) -> None:
    _check(h, lib().fv_sequential_decode(h, _ptr(noise), n_steps, _ptr(out_chunk),
                                         _stream(stream)), "fv_sequential_decode")


def fv_get_noise_state(h):
    seed, step = c_uint64(), c_uint64()
    _check(h, lib().fv_get_noise_state(h, ctypes.byref(seed), ctypes.byref(step)),
           "fv_get_noise_state")
    return seed.value, step.value


def fv_set_noise_state(h, seed: int, step: int) -> None:
    _check(h, lib().fv_set_noise_state(h, seed, step), "fv_set_noise_state")


def fv_set_graph_mode(h, enabled: bool) -> None:
    _check(h, lib().fv_set_graph_mode(h, 1 if enabled else 0), "fv_set_graph_mode")


def fv_debug_forward(h, buffer, t, n_layers_run: int, h_out, mod_out=None, stream=None) -> None:
    _check(h, lib().fv_debug_forward(h, _ptr(buffer), _ptr(t), n_layers_run, _ptr(h_out),
                                     _ptr(mod_out), _stream(stream)), "fv_debug_forward")


def fv_set_mask_mode(h, mode: int) -> None:
    _check(h, lib().fv_set_mask_mode(h, mode), "fv_set_mask_mode")


def fv_set_schedule(h, t, stream=None) -> None:
    _check(h, lib().fv_set_schedule(h, _ptr(t), _stream(stream)), "fv_set_schedule")


def fv_cold_start(h, buffer, first_stream: int, n_streams: int, stream=None) -> None:
    _check(h, lib().fv_cold_start(h, _ptr(buffer), first_stream, n_streams, _stream(stream)),
           "fv_cold_start")


def fv_get_valid_slots(h, count: int):
    arr = (c_int32 * count)()
    _check(h, lib().fv_get_valid_slots(h, arr, count), "fv_get_valid_slots")
    return [int(x) for x in arr]


def fv_set_valid_slots(h, counts: Sequence[int]) -> None:
    arr = (c_int32 * len(counts))(*[int(c) for c in counts])
    _check(h, lib().fv_set_valid_slots(h, arr, len(counts)), "fv_set_valid_slots")


def fv_multibuffer_velocity(h, k, v, prefix_len: int, ld: int, buffers, t, v_out,
                            stream=None) -> None:
    _check(h, lib().fv_multibuffer_velocity(h, _ptr(k), _ptr(v), prefix_len, ld, _ptr(buffers),
                                            _ptr(t), _ptr(v_out), _stream(stream)),
           "fv_multibuffer_velocity")


def fv_query(h, what: int, batch: int = 1) -> int:
    val = c_int64(0)
    _check(h, lib().fv_query(h, what, batch, ctypes.byref(val)), "fv_query")
    return int(val.value)


def fv_debug_stage(h, stage: int, layer: int, reps: int, stream=None) -> None:
    _check(h, lib().fv_debug_stage(h, stage, layer, reps, _stream(stream)), "fv_debug_stage")


def fv_destroy(h) -> None:
    if h:
        lib().fv_destroy(h)


# ------------------------------------------------------------- convenience

class Expert:
    """One fv_handle: the action expert on one GPU plus its decode state."""

    def __init__(self, weights: Dict, shape, max_batch: int, max_prefix: int,
                 noise_seed: int = 0):
        self.shape = shape
        self.cfg = make_cfg(shape, max_batch, max_prefix, noise_seed)
        self.handle = fv_create(weights, self.cfg)
        self.batch = max_batch

    def set_prefix(self, k, v, lengths, stream=None):
        fv_set_prefix(self.handle, k, v, lengths, k.shape[2], stream)
        self.batch = len(lengths)

    def set_prefix_async(self, k, v, lengths, copy_stream):
        fv_set_prefix_async(self.handle, k, v, lengths, k.shape[2], copy_stream)

    def decode_step(self, buffer, t, out_chunk, stream=None):
        fv_decode_step(self.handle, buffer, t, out_chunk, stream)

    def decode_step_noalloc(self, buffer, t, out_chunk, stream=None):
        fv_decode_step_noalloc(self.handle, buffer, t, out_chunk, stream)

    def noalloc_scratch_bytes(self, batch=None) -> int:
        return fv_query(self.handle, FV_QUERY_NOALLOC_SCRATCH_BYTES,
                        self.batch if batch is None else batch)

    def velocity(self, buffer, t, v_out, stream=None):
        fv_velocity(self.handle, buffer, t, v_out, stream)

    def euler_shift(self, buffer, t, v, out_chunk, stream=None):
        fv_euler_shift(self.handle, buffer, t, v, out_chunk, stream)

    def sequential_decode(self, noise, n_steps, out_chunk, stream=None):
        fv_sequential_decode(self.handle, noise, n_steps, out_chunk, stream)

    @property
    def noise_state(self):
        return fv_get_noise_state(self.handle)

    def set_noise_state(self, seed: int, step: int):
        fv_set_noise_state(self.handle, seed, step)

    def set_graph_mode(self, enabled: bool):
        fv_set_graph_mode(self.handle, enabled)

    def debug_forward(self, buffer, t, n_layers_run, h_out, mod_out=None, stream=None):
        fv_debug_forward(self.handle, buffer, t, n_layers_run, h_out, mod_out, stream)

    def set_mask_mode(self, mode):
        fv_set_mask_mode(self.handle, MASK_MODES[mode] if isinstance(mode, str) else mode)

    def set_schedule(self, t, stream=None):
        fv_set_schedule(self.handle, t, stream)

    def cold_start(self, buffer, first_stream=0, n_streams=None, stream=None):
        n = self.batch - first_stream if n_streams is None else n_streams
        fv_cold_start(self.handle, buffer, first_stream, n, stream)

    def set_valid_slots(self, counts):
        fv_set_valid_slots(self.handle, counts)

    def multibuffer_velocity(self, k, v, prefix_len, buffers, t, v_out, stream=None):
        fv_multibuffer_velocity(self.handle, k, v, prefix_len, k.shape[1], buffers, t, v_out,
                                stream)
        self.batch = self.cfg.n_chunks

    def valid_slots(self, count=None):
        return fv_get_valid_slots(self.handle, self.batch if count is None else count)

    def attn_split(self, batch=None) -> int:
        return fv_query(self.handle, FV_QUERY_ATTN_SPLITS, self.batch if batch is None else batch)

    def out_proj_splits(self, batch=None) -> int:
        return fv_query(self.handle, FV_QUERY_OUT_PROJ_SPLITS,
                        self.batch if batch is None else batch)

    def device_bytes(self) -> int:
        return fv_query(self.handle, FV_QUERY_DEVICE_BYTES)

    def debug_stage(self, stage, layer, reps, stream=None):
        fv_debug_stage(self.handle, stage, layer, reps, stream)

    def close(self):
        if self.handle:
            fv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------- observation context

def _check_context(status: int, what: str) -> None:
    if status != FV_OK:
        txt = lib().fv_status_string(status).decode()
        raise FlashVLAError(status, f"{what}: {txt}: {lib().fv_context_error().decode()}")


def _refuse(message: str):
    raise FlashVLAError(FV_ERR_INVALID_ARG, message)


_torch = _new_version = None


def _tmod():
    global _torch, _new_version
    if _torch is None:
        import torch
        _new_version = torch._C._increment_version
        _torch = torch
    return _torch


def _dtype(t, what: str) -> int:
    torch = _tmod()
    if t.dtype is torch.bfloat16:
        return FV_BF16
    if t.dtype is not torch.float32:
        _refuse(f"{what} must be bfloat16 or float32, not {t.dtype}")
    return FV_FP32


def _rows(t, what: str, dtype, gpu: int, shape=None) -> int:
    """Leading dimension of a [tokens, heads, head_dim] tensor whose heads lie side by side.
    gpu: the number of the call's GPU (-1: none, which the call refuses)."""
    got = t.shape
    if t.dtype is not dtype or t.get_device() != gpu:
        _refuse(f"{what} must have dtype {dtype} on the call's GPU: {t.dtype} on {t.device}")
    if len(got) != 3 or (shape is not None and got != shape):
        _refuse(f"{what} has shape {tuple(got)}" + (f", not {tuple(shape)}" if shape else ""))
    n, h, d = got
    ld, sh, sd = t.stride()
    if (sd != 1 and d > 1) or (sh != d and h > 1):
        _refuse(f"the heads of {what} must lie side by side (strides {(ld, sh, sd)})")
    if n > 1 and ld > 1 << 20:
        _refuse(f"the rows of {what} lie {ld} elements apart, more than 2^20")
    return ld if n > 1 else h * d


def _int32(t, what: str, gpu: int, shape=None) -> int:
    """Pointer of a dense int32 tensor."""
    if t.dtype is not _torch.int32 or t.get_device() != gpu or not t.is_contiguous():
        _refuse(f"{what} must be contiguous int32 on the call's GPU: {t.dtype} on {t.device}")
    if shape is not None and t.shape != shape:
        _refuse(f"{what} has shape {tuple(t.shape)}, not {tuple(shape)}")
    return t.data_ptr()


def _no_gradient(*tensors) -> None:
    """Refuses, in grad mode, tensors that a gradient would have to pass: the calls form none."""
    if _torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                _refuse("a tensor requires a gradient, which the call does not form "
                        "(torch.no_grad() takes it)")


def _wrote(*tensors) -> None:
    """What autograd kept of these tensors for a backward pass is no longer there."""
    _new_version(tensors)


class _On:
    """The raw stream of a call, and for the call's duration the GPU and stream that
    it runs on as torch's current ones where they are others: the C calls take the
    NULL stream to be the current GPU's, and a workspace has to come from the
    allocator's pool of the stream that uses it."""

    __slots__ = ("raw", "scope")

    def __init__(self, device, stream):
        torch = _tmod()
        if device.type != "cuda":
            _refuse(f"tensors must be on a GPU, not {device}")
        self.scope = None
        if stream is None:
            self.raw = torch._C._cuda_getCurrentRawStream(device.index)
            if torch._C._cuda_getDevice() != device.index:
                self.scope = torch.cuda.device(device)
        else:
            if not isinstance(stream, torch.cuda.Stream):
                stream = torch.cuda.ExternalStream(int(stream), device=device)
            if stream.device != device:
                _refuse(f"the stream is of {stream.device}, the tensors of {device}")
            self.raw = int(stream.cuda_stream)
            self.scope = torch.cuda.stream(stream)

    def __enter__(self):
        if self.scope is not None:
            self.scope.__enter__()
        return self

    def __exit__(self, *exc):
        if self.scope is not None:
            self.scope.__exit__(*exc)
        return False


def _work(nbytes: int, device):
    return _tmod().empty(nbytes, dtype=_tmod().uint8, device=device)


def prompt_attention(q, k, v, cu_q, cu_k, out, causal: bool = True, scale: Optional[float] = None,
                     stream=None) -> None:
    """fv_prompt_attention on torch tensors: q and out [tokens, heads, head_dim], k and v
    [keys, kv heads, head_dim] (rows may be strided), cu_q and cu_k int32 [prompts + 1].
    `scale` defaults to 1/sqrt(head_dim).  As every call here it forms no gradient: in grad
    mode tensors that require one are refused, and what is written counts as modified."""
    dtype, t, gpu, shape = _dtype(q, "q"), q.dtype, q.get_device(), q.shape
    _no_gradient(q, k, v, out)
    ldq, ldo = _rows(q, "q", t, gpu), _rows(out, "out", t, gpu, shape)
    ldk = _rows(k, "k", t, gpu)
    ldv = _rows(v, "v", t, gpu, k.shape)
    n_q, heads, dh = shape
    n_k, kv_heads, dk = k.shape
    if dk != dh:
        _refuse(f"head_dim of q is {dh}, of k {dk}")
    prompts = cu_q.shape
    if len(prompts) != 1 or prompts[0] < 1:
        _refuse("cu_q must have prompts + 1 entries")
    args = FvPromptArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ldq, ldk, ldv, ldo,
                        _int32(cu_q, "cu_q", gpu), _int32(cu_k, "cu_k", gpu, prompts),
                        prompts[0] - 1, n_q, n_k, heads, kv_heads, dh, dtype, 1 if causal else 0,
                        dh ** -0.5 if scale is None else scale)
    with _On(q.device, stream) as on:
        _check_context(lib().fv_prompt_attention(byref(args), on.raw), "fv_prompt_attention")
    _wrote(out)


def rope(q, k, pos, sections: Sequence[int], q_out, k_out=None, theta: float = 10000.0,
         stream=None) -> None:
    """fv_rope_append without a cache: rotates q into q_out and, if given, k into k_out."""
    _rope("fv_rope_append", None, 0, q, k, None, pos, None, None, sections, theta, q_out, k_out, stream)


def _rope(name, cache, layer, q, k, v, pos, seqs, at, sections, theta, q_out, k_out, stream, *pools) -> None:
    dtype, t, gpu = _dtype(q, "q"), q.dtype, q.get_device()
    _no_gradient(q, k, v, q_out, k_out)
    ldq, ldk = _rows(q, "q", t, gpu), _rows(k, "k", t, gpu)
    n, heads, dh = q.shape
    nk, kv_heads, dk = k.shape
    if nk != n or dk != dh:
        _refuse(f"k has shape {tuple(k.shape)}, q {tuple(q.shape)}")
    axes = len(sections)
    if not 1 <= axes <= 4:
        _refuse("sections must have 1 to 4 entries")
    args = FvRopeArgs(q.data_ptr(), k.data_ptr(), _ptr(v), q_out.data_ptr(), _ptr(k_out), ldq, ldk,
                      _rows(v, "v", t, gpu, k.shape) if v is not None else 0,
                      _rows(q_out, "q_out", t, gpu, q.shape),
                      _rows(k_out, "k_out", t, gpu, k.shape) if k_out is not None else 0,
                      _int32(pos, "pos", gpu, (axes, n)),
                      _int32(seqs, "seqs", gpu, (n,)) if seqs is not None else None,
                      _int32(at, "at", gpu, (n,)) if at is not None else None, n, heads, kv_heads,
                      dh, dtype, layer, axes, tuple(sections), theta)
    with _On(q.device, stream) as on:
        _check_context(getattr(lib(), name)(byref(args), None if cache is None else byref(cache),
                                            on.raw), name)
    _wrote(q_out, *pools) if k_out is None else _wrote(q_out, k_out, *pools)


class PageCache:
    """A paged cache of keys and values (fv_pages) over torch tensors that the caller
    owns: k, v [layers, pages, kv heads, page_len, head_dim], table int32 [sequences,
    pages of a sequence], length int32 [sequences], refs int32 [pages].  The object
    holds the tensors and nothing else; every call is stream-ordered and may be
    captured into a HIP graph."""

    _APPEND, _ATTEND, _UPKEEP = "fv_rope_append", "fv_paged_attention", "fv_pages_"

    def __init__(self, k, v, table, length, refs):
        dtype = _dtype(k, "k")
        self.dtype = k.dtype
        self._hold(FvPages, dtype, k, v, (), table, length, refs)

    def _hold(self, struct, dtype, k, v, scales, table, length, refs):
        if k.dim() != 5 or not k.is_contiguous():
            _refuse("k must be contiguous [layers, pages, kv heads, page_len, head_dim]")
        if v.shape != k.shape or v.dtype != k.dtype or v.device != k.device or not v.is_contiguous():
            _refuse("v must be as k")
        if table.dim() != 2:
            _refuse("table must be [sequences, pages of a sequence]")
        layers, pages, heads, page_len, dh = k.shape
        gpu = k.get_device()
        self.pools = (k, v) + scales  # what an append writes
        _no_gradient(*self.pools)
        self.k, self.v, self.table, self.length, self.refs = k, v, table, length, refs
        self.c = struct(dtype, layers, heads, dh, page_len, pages, table.shape[0], table.shape[1],
                        *(t.data_ptr() for t in self.pools), _int32(table, "table", gpu),
                        _int32(length, "length", gpu, table.shape[:1]),
                        _int32(refs, "refs", gpu, (pages,)))
        need = c_size_t()
        name = self._UPKEEP + "workspace"
        _check_context(getattr(lib(), name)(byref(self.c), byref(need)), type(self).__name__)
        self.work_bytes = need.value  # of the upkeep's calls

    @classmethod
    def empty(cls, n_layers: int, n_kv_heads: int, head_dim: int, n_pages: int, max_seqs: int,
              max_pages: int, page_len: int = 16, dtype=None, device="cuda"):
        """A fresh cache: uninitialised pages, no sequences."""
        torch = _tmod()
        dtype = torch.bfloat16 if dtype is None else dtype
        shape = (n_layers, n_pages, n_kv_heads, page_len, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        i32 = dict(dtype=torch.int32, device=device)
        return cls(k, v, torch.full((max_seqs, max_pages), -1, **i32), torch.zeros(max_seqs, **i32),
                   torch.zeros(n_pages, **i32))

    def append(self, layer: int, q, k, v, pos, seqs, at, sections: Sequence[int],
               theta: float = 10000.0, q_out=None, k_out=None, stream=None) -> None:
        """fv_rope_append: rotates q into q_out (default: q itself) and k into the pages
        (and k_out, if given), and stores v."""
        if v is None or seqs is None or at is None:
            _refuse("append needs v, seqs and at")
        if q.device != self.k.device:
            _refuse(f"q is on {q.device}, the cache on {self.k.device}")
        self._layer(layer)
        _rope(self._APPEND, self.c, layer, q, k, v, pos, seqs, at, sections, theta,
              q if q_out is None else q_out, k_out, stream, *self.pools)

    def attend(self, layer: int, q, seqs, out, scale: Optional[float] = None, max_len: int = 0,
               stream=None) -> None:
        """fv_paged_attention: q and out [rows, heads, head_dim], seqs int32 [rows]."""
        ldq, ldo = self._queries(layer, q, out)
        n, heads, dh = q.shape
        args = FvPagedArgs(q.data_ptr(), out.data_ptr(), ldq, ldo,
                           _int32(seqs, "seqs", self.k.get_device(), (n,)), n, heads, layer, max_len,
                           dh ** -0.5 if scale is None else scale, None, 0)
        self._attend(self._ATTEND, self._ATTEND + "_workspace", args, out, stream)

    def _queries(self, layer: int, q, out):
        """Checks an attention's queries and results; their leading dimensions."""
        t, gpu = self.dtype, self.k.get_device()
        _no_gradient(q, out)
        ldq = _rows(q, "q", t, gpu)
        ldo = _rows(out, "out", t, gpu, q.shape)
        self._layer(layer)
        if q.shape[2] != self.c.head_dim:
            _refuse(f"head_dim of q is {q.shape[2]}, of the cache {self.c.head_dim}")
        return ldq, ldo

    def _attend(self, name: str, workspace: str, args, out, stream) -> None:
        dev, cache = self.k.device, byref(self.c)
        with _On(dev, stream) as on:
            need, L, a = c_size_t(), lib(), byref(args)
            _check_context(getattr(L, workspace)(a, cache, byref(need)), name)
            if need.value:
                work = _work(need.value, dev)
                args.work, args.work_bytes = work.data_ptr(), need.value
            _check_context(getattr(L, name)(a, cache, on.raw), name)
        _wrote(out)

    def _layer(self, layer: int) -> None:
        if not 0 <= layer < self.c.n_layers:
            _refuse(f"layer {layer} of {self.c.n_layers}")

    def _upkeep(self, name: str, stream, *lists, status=None, work=True, pages=False):
        name = self._UPKEEP + name
        dev, gpu = self.k.device, self.k.get_device()
        n = lists[0].shape[0] if lists else 0
        args = [byref(self.c), *[_int32(t, name + " list", gpu, (n,)) for t in lists]]
        if lists:
            args.append(n)
        with _On(dev, stream) as on:
            if status is None:
                status = _tmod().empty(1, dtype=_tmod().int32, device=dev)
            args.append(_int32(status, "status", gpu, (1,)))
            if work:
                buf = _work(self.work_bytes, dev)
                args.append(buf.data_ptr())
            _check_context(getattr(lib(), name)(*args, on.raw), name)
        if pages:
            _wrote(self.table, self.length, self.refs, status, *self.pools)
        else:
            _wrote(self.table, self.length, self.refs, status)
        return status

    def grow(self, seqs, add, status=None, stream=None):
        """fv_pages_grow; returns the status tensor (int32 [1]: FV_PAGES_*)."""
        return self._upkeep("grow", stream, seqs, add, status=status)

    def fork(self, parents, children, status=None, stream=None):
        """fv_pages_fork; returns the status tensor."""
        return self._upkeep("fork", stream, parents, children, status=status, pages=True)

    def free(self, seqs, status=None, stream=None):
        """fv_pages_free; returns the status tensor."""
        return self._upkeep("free", stream, seqs, status=status, work=False)

    def compact(self, used=None, stream=None):
        """fv_pages_compact; returns the number of pages in use (int32 [1])."""
        return self._upkeep("compact", stream, status=used, pages=True)

    def gather(self, seqs, k_out, v_out, stream=None) -> None:
        """fv_pages_gather: k_out and v_out [layers, entries, ld, kv heads, head_dim], as
        Expert.set_prefix takes them."""
        c, dev = self.c, self.k.device
        _no_gradient(k_out, v_out)
        for t, what in ((k_out, "k_out"), (v_out, "v_out")):
            if t.dim() != 5 or t.dtype != self.dtype or t.device != dev or not t.is_contiguous():
                _refuse(f"{what} must be contiguous [layers, entries, ld, kv heads, head_dim]")
            if t.shape[0] != c.n_layers or tuple(t.shape[3:]) != (c.n_kv_heads, c.head_dim):
                _refuse(f"{what} has shape {tuple(t.shape)}")
        if k_out.shape != v_out.shape:
            _refuse("k_out and v_out must have the same shape")
        with _On(dev, stream) as on:
            ids = _int32(seqs, "seqs", self.k.get_device(), k_out.shape[1:2])
            name = self._UPKEEP + "gather"
            _check_context(getattr(lib(), name)(byref(c), ids, k_out.shape[1], k_out.shape[2],
                                                k_out.data_ptr(), v_out.data_ptr(), on.raw), name)
        _wrote(k_out, v_out)


class QuantCache(PageCache):
    """A paged cache in 8 bits (fv_quant_pages): k, v float8_e4m3fn [layers, pages, kv heads,
    page_len, head_dim], which hold their blocks in the order that the header states, and
    k_scale, v_scale float8_e8m0fnu [layers, pages, kv heads, page_len / 16], a power of two for
    each block of 16 positions.  dtype: of the queries, keys, values and results of its calls
    (bfloat16 or float32).  The calls are PageCache's: append quantises as it writes, gather
    reads back exactly what the codes stand for, and attend_part takes several new tokens a
    sequence."""

    _APPEND, _ATTEND, _UPKEEP = "fv_quant_append", "fv_quant_attention", "fv_quant_"

    def __init__(self, k, v, k_scale, v_scale, table, length, refs, dtype=None):
        torch = _tmod()
        self.dtype = torch.bfloat16 if dtype is None else dtype
        if self.dtype not in (torch.bfloat16, torch.float32):
            _refuse(f"dtype must be bfloat16 or float32, not {self.dtype}")
        if k.dtype is not torch.float8_e4m3fn:
            _refuse(f"k must be float8_e4m3fn, not {k.dtype}")
        blocks = (*k.shape[:3], k.shape[3] // 16) if k.dim() == 5 else None
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.dtype is not torch.float8_e8m0fnu or t.device != k.device or not t.is_contiguous():
                _refuse(f"{what} must be contiguous float8_e8m0fnu on the pages' device: {t.dtype} on {t.device}")
            if blocks is not None and tuple(t.shape) != blocks:
                _refuse(f"{what} has shape {tuple(t.shape)}, not {blocks}")
        self.k_scale, self.v_scale = k_scale, v_scale
        self._hold(FvQuantPages, FV_BF16 if self.dtype is torch.bfloat16 else FV_FP32, k, v,
                   (k_scale, v_scale), table, length, refs)

    @classmethod
    def empty(cls, n_layers: int, n_kv_heads: int, head_dim: int, n_pages: int, max_seqs: int,
              max_pages: int, page_len: int = 16, dtype=None, device="cuda"):
        """A fresh cache: uninitialised pages, no sequences."""
        torch = _tmod()
        shape = (n_layers, n_pages, n_kv_heads, page_len, head_dim)
        k, v = (torch.empty(shape, dtype=torch.float8_e4m3fn, device=device) for _ in range(2))
        ks, vs = (torch.empty((*shape[:3], page_len // 16), dtype=torch.float8_e8m0fnu, device=device)
                  for _ in range(2))
        i32 = dict(dtype=torch.int32, device=device)
        return cls(k, v, ks, vs, torch.full((max_seqs, max_pages), -1, **i32),
                   torch.zeros(max_seqs, **i32), torch.zeros(n_pages, **i32), dtype=dtype)

    def attend_part(self, layer: int, q, cu_q, seqs, out, causal: bool = True,
                    scale: Optional[float] = None, max_len: int = 0, stream=None) -> None:
        """fv_quant_part_attention: q and out [rows, heads, head_dim], cu_q int32 [entries + 1],
        seqs int32 [entries]; entry i's rows are the last tokens of sequence seqs[i]."""
        ldq, ldo = self._queries(layer, q, out)
        n, heads, dh = q.shape
        gpu, entries = self.k.get_device(), cu_q.shape
        if len(entries) != 1 or entries[0] < 1:
            _refuse("cu_q must have entries + 1 entries")
        args = FvPartArgs(q.data_ptr(), out.data_ptr(), ldq, ldo, _int32(cu_q, "cu_q", gpu),
                          _int32(seqs, "seqs", gpu, (entries[0] - 1,)), entries[0] - 1, n, heads,
                          layer, max_len, 1 if causal else 0, dh ** -0.5 if scale is None else scale,
                          None, 0)
        self._attend("fv_quant_part_attention", "fv_quant_part_workspace", args, out, stream)
