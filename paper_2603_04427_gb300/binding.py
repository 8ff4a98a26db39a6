"""ctypes binding of ``libtk.so`` (include/tk.h), one Python function per entry point.

Argument marshalling only: each function checks that the torch tensors it
is given have the dtype, device and contiguity the C ABI expects, passes
their ``data_ptr()`` and the current CUDA stream, and raises ``TkError`` on
a non-OK status.  Every step of the computation runs in the library's
kernels; there is no CPU or PyTorch fallback, and a missing library raises.
"""

from __future__ import annotations

import contextlib
import ctypes
import math
import os
import struct
from dataclasses import dataclass

import torch

TK_OK, TK_ERR_INVALID_ARG, TK_ERR_UNSUPPORTED, TK_ERR_WORKSPACE, TK_ERR_CUDA, TK_ERR_DEVICE = range(6)
TK_BF16, TK_F32, TK_I8, TK_I4 = 0, 1, 2, 3
TK_ROPE_HALF, TK_ROPE_PAIR = 0, 1
TK_ROPE_MAX_PAIRS, TK_ROPE_MAX_AXES = 64, 4

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtk.so")

EXPORTED = ("tk_kv_append", "tk_attn_prefill", "tk_decode_workspace_size", "tk_attn_decode",
            "tk_attn_decode_append", "tk_attn_decode_noalloc", "tk_attn_prefill_cached",
            "tk_prefill_cached_workspace_size",
            "tk_attn_forward", "tk_backward_workspace_size", "tk_attn_backward", "tk_copy_async",
            "tk_qk_norm_rope", "tk_qk_norm_rope_append", "tk_qk_norm_rope_backward",
            "tk_qk_norm_rope_workspace_size", "tk_block_tables",
            "tk_block_bounds", "tk_block_select", "tk_attn_decode_blocks",
            "tk_decode_blocks_workspace_size", "tk_attn_weights", "tk_attn_weights_workspace_size",
            "tk_cache_evict", "tk_cache_evict_workspace_size",
            "tk_check_wait_timeout", "tk_get_device_error", "tk_status_string", "tk_last_error",
            "tk_abi_version", "tk_graph_begin", "tk_graph_end", "tk_graph_launch",
            "tk_graph_destroy")


class TkError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: {_status_name(status)}: {detail}")
        self.status = status


class tk_cache_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "h_q", "h_kv", "r", "d_v", "capacity", "page_size", "num_pages",
        "max_pages_per_seq", "k_dtype")]


class tk_rope_desc(ctypes.Structure):
    """What a model fixes about its queries and keys (include/tk.h); see rope_plan."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("r", "rot_dim", "layout", "n_axes", "norm")]
                + [("eps", ctypes.c_float), ("w_offset", ctypes.c_float),
                   ("inv_freq", ctypes.c_float * TK_ROPE_MAX_PAIRS),
                   ("pair_axis", ctypes.c_uint8 * TK_ROPE_MAX_PAIRS)])


class tk_heads(ctypes.Structure):
    _fields_ = ([("data", ctypes.c_void_p), ("n_heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]
                + [(n, ctypes.c_int64) for n in ("batch_stride", "token_stride", "head_stride")])


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libtk.so once and declare the C signatures; raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run `python -m paper_2603_04427_gb300.build` "
                           "(or __graft_entry__.build()) first")
    L = ctypes.CDLL(path)
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    i64 = ctypes.c_int64
    dp = ctypes.POINTER(tk_cache_desc)
    rp = hp = vp     # addresses or byref(): checking a pointer's type costs more than passing it
    sig = {
        "tk_kv_append": (i32, [dp, vp, vp, vp, vp, vp, vp, vp, i32, vp]),
        "tk_attn_prefill": (i32, [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, i32, vp]),
        "tk_decode_workspace_size": (sz, [dp, i32]),
        "tk_attn_forward": (i32, [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, i32,
                                  vp]),
        "tk_backward_workspace_size": (sz, [i32, i32, i32]),
        "tk_attn_backward": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, i32, i32, i32, i32,
                                   i32, i32, f32, i32, vp]),
        "tk_attn_prefill_cached": (i32, [dp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, i32,
                                         f32, i32, vp, sz, vp]),
        "tk_prefill_cached_workspace_size": (sz, [dp, i32]),
        "tk_attn_decode": (i32, [dp, vp, vp, vp, vp, vp, vp, i32, vp, i32, f32, vp, sz, vp]),
        "tk_attn_decode_append": (i32, [dp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, f32, vp,
                                        sz, vp]),
        "tk_attn_decode_noalloc": (i32, [dp, vp, vp, vp, vp, vp, vp, i32, vp, i32, f32, vp]),
        "tk_qk_norm_rope": (i32, [rp, i32, i32, i32, hp, hp, hp, vp, vp, i32, vp, i64, i64, hp, hp,
                                  hp, vp]),
        "tk_qk_norm_rope_append": (i32, [vp, rp, i32, i32, hp, hp, hp, vp, vp, i32, vp, i64, i64,
                                         vp, hp, vp, vp, vp, vp]),
        "tk_qk_norm_rope_workspace_size": (sz, [rp]),
        "tk_qk_norm_rope_backward": (i32, [rp, i32, i32, i32, hp, hp, vp, vp, i32, vp, i64, i64,
                                           hp, hp, hp, hp, hp, hp, vp, vp, vp, sz, vp]),
        "tk_block_tables": (i32, [i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp,
                                  vp, vp, vp, vp]),
        "tk_block_bounds": (i32, [dp, i32, vp, vp, vp, vp, vp, i32, vp, vp]),
        "tk_block_select": (i32, [dp, i32, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp]),
        "tk_decode_blocks_workspace_size": (sz, [dp, i32, i32]),
        "tk_attn_decode_blocks": (i32, [dp, i32, vp, vp, vp, vp, vp, vp, i32, vp, i32, f32, vp, sz, vp]),
        "tk_attn_weights_workspace_size": (sz, [dp, i32, i32]),
        "tk_attn_weights": (i32, [dp, vp, i32, vp, vp, vp, vp, vp, i32, f32, f32, vp, vp, sz, vp]),
        "tk_cache_evict_workspace_size": (sz, [dp, i32]),
        "tk_cache_evict": (i32, [dp, vp, vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "tk_get_device_error": (i32, [ctypes.POINTER(i32), vp]),
        "tk_check_wait_timeout": (i32, [i32, vp]),
        "tk_copy_async": (i32, [vp, vp, sz, vp]),
        "tk_graph_begin": (i32, [vp]),
        "tk_graph_end": (i32, [vp, ctypes.POINTER(vp)]),
        "tk_graph_launch": (i32, [vp, vp]),
        "tk_graph_destroy": (i32, [vp]),
        "tk_status_string": (ctypes.c_char_p, [i32]),
        "tk_last_error": (ctypes.c_char_p, []),
        "tk_abi_version": (i32, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    _lib = L
    return L


def _status_name(s: int) -> str:
    names = {0: "TK_OK", 1: "TK_ERR_INVALID_ARG", 2: "TK_ERR_UNSUPPORTED", 3: "TK_ERR_WORKSPACE",
             4: "TK_ERR_CUDA", 5: "TK_ERR_DEVICE"}
    return names.get(s, f"status {s}")


def _check(status: int, where: str):
    if status != TK_OK:
        raise TkError(status, where, load_library().tk_last_error().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _raw_stream(stream, device):
    # the device's current stream without building a torch.cuda.Stream (60 ns against 2.9 us)
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _stream(stream):
    return ctypes.c_void_p(_raw_stream(stream, torch.cuda.current_device()))


def _need_out(t, name, device):
    """An output: float32 or bfloat16, contiguous, on `device` or in page-locked host memory
    (the kernel then writes it zero-copy)."""
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"{name} must be float32 or bfloat16")
    if t.is_cuda:
        _need(t, t.dtype, name, device)
    elif not t.is_pinned() or not t.is_contiguous():
        raise ValueError(f"{name} must be a CUDA tensor or a contiguous page-locked host tensor")


def _need(t, dtype, name, device=None):
    if t is None:
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


# ------------------------------------------------------------------ cache helper

@dataclass
class ThinKeyCache:
    """Caller-owned thin-key / full-value cache tensors plus their descriptor.

    Contiguous: k [B, H_kv, cap, r] (bf16 or int8; uint8 [B, H_kv, cap, r/2] of
    packed int4 codes), k_scale [B, H_kv, cap] fp32, v [B, H_kv, cap, d_v] bf16.
    Paged: pools [P, H_kv, page_size, ...] and a page table [B, max_pages] int32.
    """
    desc: tk_cache_desc
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor | None = None
    page_table: torch.Tensor | None = None

    @staticmethod
    def allocate(batch, h_q, h_kv, r, d_v, capacity=0, page_size=0, num_pages=0,
                 page_table=None, k_int8=False, device="cuda", fill=0, k_int4=False):
        if page_size:
            if page_table is None:
                raise ValueError("a paged cache needs a page table")
            page_table = page_table.to(device=device, dtype=torch.int32).contiguous()
            lead = (num_pages, h_kv, page_size)
            max_pages = page_table.shape[1]
        else:
            lead = (batch, h_kv, capacity)
            max_pages = 0
        if k_int8 and k_int4:
            raise ValueError("k_int8 and k_int4 are exclusive")
        kd = torch.int8 if k_int8 else (torch.uint8 if k_int4 else torch.bfloat16)
        k = torch.full(lead + (r // 2 if k_int4 else r,), fill, dtype=kd, device=device)
        v = torch.full(lead + (d_v,), fill, dtype=torch.bfloat16, device=device)
        ks = torch.zeros(lead, dtype=torch.float32, device=device) if (k_int8 or k_int4) else None
        desc = tk_cache_desc(batch, h_q, h_kv, r, d_v, 0 if page_size else capacity, page_size,
                             num_pages if page_size else 0, max_pages,
                             TK_I8 if k_int8 else (TK_I4 if k_int4 else TK_BF16))
        return ThinKeyCache(desc, k, v, ks, page_table)


# ------------------------------------------------------------------ entry points

def tk_abi_version() -> int:
    return int(load_library().tk_abi_version())


def tk_status_string(status: int) -> str:
    return load_library().tk_status_string(status).decode()


def tk_last_error() -> str:
    return load_library().tk_last_error().decode()


def tk_kv_append(cache: ThinKeyCache, k_new, v_new, seq_lens, stream=None):
    """Append k_new [B, H_kv, T, r] / v_new [B, H_kv, T, d_v] (bf16) at seq_lens[b]."""
    d = cache.desc
    dev = cache.k.device
    _need(k_new, torch.bfloat16, "k_new", dev)
    _need(v_new, torch.bfloat16, "v_new", dev)
    _need(seq_lens, torch.int32, "seq_lens", dev)
    T = k_new.shape[2]
    if tuple(k_new.shape) != (d.batch, d.h_kv, T, d.r) or tuple(v_new.shape) != (d.batch, d.h_kv, T, d.d_v):
        raise ValueError(f"k_new {tuple(k_new.shape)} / v_new {tuple(v_new.shape)} do not match the cache")
    L = load_library()
    _check(L.tk_kv_append(ctypes.byref(d), _ptr(cache.k), _ptr(cache.v), _ptr(cache.k_scale),
                          _ptr(cache.page_table), _ptr(seq_lens), _ptr(k_new), _ptr(v_new), T,
                          _stream(stream)), "tk_kv_append")


def tk_decode_workspace_size(desc: tk_cache_desc, max_seq_len: int) -> int:
    n = int(load_library().tk_decode_workspace_size(ctypes.byref(desc), int(max_seq_len)))
    if n == 0:
        raise TkError(TK_ERR_INVALID_ARG, "tk_decode_workspace_size", tk_last_error())
    return n


def decode_workspace(desc: tk_cache_desc, max_seq_len: int, device="cuda") -> torch.Tensor:
    """A zero-filled workspace of the size tk_attn_decode needs (torch owns the memory)."""
    return torch.zeros(tk_decode_workspace_size(desc, max_seq_len), dtype=torch.uint8, device=device)


def tk_attn_decode(cache: ThinKeyCache, q, seq_lens, max_seq_len: int, out, workspace,
                   scale: float | None = None, stream=None):
    """One decode step: q [B, H_q, r] bf16 -> out [B, H_q, d_v] (fp32 or bf16, on the GPU or
    in page-locked host memory, which the kernel then writes directly)."""
    d = cache.desc
    dev = cache.k.device
    _need(q, torch.bfloat16, "q", dev)
    _need(seq_lens, torch.int32, "seq_lens", dev)
    _need(workspace, torch.uint8, "workspace", dev)
    _need_out(out, "out", dev)
    if tuple(q.shape) != (d.batch, d.h_q, d.r) or tuple(out.shape) != (d.batch, d.h_q, d.d_v):
        raise ValueError(f"q {tuple(q.shape)} / out {tuple(out.shape)} do not match the cache")
    scale = 1.0 / math.sqrt(d.r) if scale is None else float(scale)
    L = load_library()
    _check(L.tk_attn_decode(ctypes.byref(d), _ptr(q), _ptr(cache.k), _ptr(cache.v),
                            _ptr(cache.k_scale), _ptr(cache.page_table), _ptr(seq_lens),
                            int(max_seq_len), _ptr(out),
                            TK_F32 if out.dtype == torch.float32 else TK_BF16, scale,
                            _ptr(workspace), workspace.numel(), _stream(stream)), "tk_attn_decode")
    return out


def tk_attn_decode_append(cache: ThinKeyCache, q, k_new, v_new, seq_lens, max_seq_len: int, out,
                          workspace, scale: float | None = None, stream=None):
    """Append one token per sequence (k_new [B, H_kv, r], v_new [B, H_kv, d_v] bf16) at
    seq_lens[b] and decode q [B, H_q, r] over the seq_lens[b] + 1 tokens, in one launch."""
    d = cache.desc
    dev = cache.k.device
    _need(q, torch.bfloat16, "q", dev)
    _need(k_new, torch.bfloat16, "k_new", dev)
    _need(v_new, torch.bfloat16, "v_new", dev)
    _need(seq_lens, torch.int32, "seq_lens", dev)
    _need(workspace, torch.uint8, "workspace", dev)
    _need_out(out, "out", dev)
    if tuple(q.shape) != (d.batch, d.h_q, d.r) or tuple(out.shape) != (d.batch, d.h_q, d.d_v):
        raise ValueError(f"q {tuple(q.shape)} / out {tuple(out.shape)} do not match the cache")
    if tuple(k_new.shape) != (d.batch, d.h_kv, d.r) or tuple(v_new.shape) != (d.batch, d.h_kv, d.d_v):
        raise ValueError(f"k_new {tuple(k_new.shape)} / v_new {tuple(v_new.shape)} do not match the cache")
    scale = 1.0 / math.sqrt(d.r) if scale is None else float(scale)
    L = load_library()
    _check(L.tk_attn_decode_append(ctypes.byref(d), _ptr(q), _ptr(cache.k), _ptr(cache.v),
                                   _ptr(cache.k_scale), _ptr(cache.page_table), _ptr(seq_lens),
                                   _ptr(k_new), _ptr(v_new), int(max_seq_len), _ptr(out),
                                   TK_F32 if out.dtype == torch.float32 else TK_BF16, scale,
                                   _ptr(workspace), workspace.numel(), _stream(stream)),
           "tk_attn_decode_append")
    return out


def tk_attn_forward(q, k, v, out, lse, scale: float | None = None, causal: bool = True, stream=None):
    """tk_attn_prefill that also writes lse [B, H_q, S] (fp32), each row's logsumexp."""
    dev = q.device
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, n, dev)
    _need(lse, torch.float32, "lse", dev)
    if out.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("out must be float32 or bfloat16")
    _need(out, out.dtype, "out", dev)
    B, hq, S, r = q.shape
    hkv, dv = k.shape[1], v.shape[3]
    if tuple(k.shape) != (B, hkv, S, r) or tuple(v.shape) != (B, hkv, S, dv) or \
            tuple(out.shape) != (B, hq, S, dv) or tuple(lse.shape) != (B, hq, S):
        raise ValueError("q / k / v / out / lse shapes are inconsistent")
    scale = 1.0 / math.sqrt(r) if scale is None else float(scale)
    L = load_library()
    _check(L.tk_attn_forward(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
                             TK_F32 if out.dtype == torch.float32 else TK_BF16,
                             B, hq, hkv, S, r, dv, scale, 1 if causal else 0, _stream(stream)),
           "tk_attn_forward")
    return out, lse


def tk_attn_backward(q, k, v, out, d_out, lse, dq, dk, dv, workspace=None,
                     scale: float | None = None, causal: bool = True, stream=None):
    """Gradients dq [B, H_q, S, r], dk [B, H_kv, S, r], dv [B, H_kv, S, d_v] (fp32)
    of prefill attention for dL/d(out) = d_out (bf16), from the forward's lse."""
    dev = q.device
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (out, "out"), (d_out, "d_out")):
        _need(t, torch.bfloat16, n, dev)
    for t, n in ((lse, "lse"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        _need(t, torch.float32, n, dev)
    B, hq, S, r = q.shape
    hkv, d_v = k.shape[1], v.shape[3]
    if tuple(k.shape) != (B, hkv, S, r) or tuple(v.shape) != (B, hkv, S, d_v) or \
            tuple(out.shape) != (B, hq, S, d_v) or tuple(d_out.shape) != (B, hq, S, d_v) or \
            tuple(lse.shape) != (B, hq, S) or tuple(dq.shape) != tuple(q.shape) or \
            tuple(dk.shape) != tuple(k.shape) or tuple(dv.shape) != tuple(v.shape):
        raise ValueError("backward tensor shapes are inconsistent")
    L = load_library()
    if workspace is None:
        workspace = torch.empty(int(L.tk_backward_workspace_size(B, hq, S)), dtype=torch.uint8,
                                device=dev)
    _need(workspace, torch.uint8, "workspace", dev)
    scale = 1.0 / math.sqrt(r) if scale is None else float(scale)
    _check(L.tk_attn_backward(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(d_out), _ptr(lse),
                              _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace), workspace.numel(),
                              B, hq, hkv, S, r, d_v, scale, 1 if causal else 0, _stream(stream)),
           "tk_attn_backward")
    return dq, dk, dv


def prefill_cached_workspace(cache: ThinKeyCache, max_seq_len: int):
    """The device workspace tk_attn_prefill_cached needs for this cache and this
    bound of seq_lens[b] + S (int8 / int4 keys), or None (bf16 keys)."""
    n = int(load_library().tk_prefill_cached_workspace_size(ctypes.byref(cache.desc), int(max_seq_len)))
    return torch.empty(n, dtype=torch.uint8, device=cache.k.device) if n else None


def tk_attn_prefill_cached(cache: ThinKeyCache, q, k_new, v_new, seq_lens, max_seq_len: int, out,
                           scale: float | None = None, causal: bool = True, workspace=None,
                           stream=None):
    """Append a chunk (k_new [B, H_kv, S, r], v_new [B, H_kv, S, d_v] bf16) at seq_lens[b]
    and prefill its queries q [B, H_q, S, r] over the cache (query i at position
    seq_lens[b] + i) -> out [B, H_q, S, d_v] (fp32 or bf16).  bf16, int8 or int4 keys;
    quantised keys need a workspace (prefill_cached_workspace; allocated here if None)."""
    d = cache.desc
    dev = cache.k.device
    for t, n in ((q, "q"), (k_new, "k_new"), (v_new, "v_new")):
        _need(t, torch.bfloat16, n, dev)
    _need(seq_lens, torch.int32, "seq_lens", dev)
    if out.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("out must be float32 or bfloat16")
    _need(out, out.dtype, "out", dev)
    S = q.shape[2]
    if tuple(q.shape) != (d.batch, d.h_q, S, d.r) or tuple(out.shape) != (d.batch, d.h_q, S, d.d_v) \
            or tuple(k_new.shape) != (d.batch, d.h_kv, S, d.r) \
            or tuple(v_new.shape) != (d.batch, d.h_kv, S, d.d_v):
        raise ValueError("q / k_new / v_new / out shapes do not match the cache")
    scale = 1.0 / math.sqrt(d.r) if scale is None else float(scale)
    L = load_library()
    if workspace is None and d.k_dtype != TK_BF16:
        workspace = prefill_cached_workspace(cache, max_seq_len)
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace", dev)
    _check(L.tk_attn_prefill_cached(ctypes.byref(d), _ptr(q), _ptr(cache.k), _ptr(cache.v),
                                    _ptr(cache.k_scale), _ptr(cache.page_table), _ptr(seq_lens),
                                    _ptr(k_new), _ptr(v_new),
                                    S, int(max_seq_len), _ptr(out),
                                    TK_F32 if out.dtype == torch.float32 else TK_BF16, scale,
                                    1 if causal else 0, _ptr(workspace),
                                    0 if workspace is None else workspace.numel(),
                                    _stream(stream)), "tk_attn_prefill_cached")
    return out


def _marshalled(lib, name, args):
    """A handle of the entry point without argument types, and the arguments as C values: a call
    then converts nothing (1.0 us against 2.4 us for 17 arguments)."""
    typed = getattr(lib, name)
    fn = lib[name]
    fn.restype = typed.restype
    return fn, tuple(t(a) if isinstance(a, (int, float)) else a for t, a in zip(typed.argtypes, args, strict=True))


class PreparedCall:
    """Entry-point calls with their arguments checked and marshalled once.

    For serving loops whose buffers stay fixed between steps: calling the
    object re-issues the same C calls in order (same pointers, same stream)
    without the per-call Python checks, and raises TkError on a non-OK status.
    With graph=True (a non-default stream required) the calls are run once,
    then recorded once into a CUDA graph (tk_graph_begin / tk_graph_end), and
    each call of the object is one tk_graph_launch of that graph."""

    def __init__(self, name: str, args: tuple, keep: tuple, before: tuple = (), graph: bool = False,
                 stream=None):
        L = load_library()
        self._calls = tuple((*_marshalled(L, n, a), n) for n, a in (*before, (name, args)))
        self._keep = keep  # the tensors whose pointers are in args stay alive
        self._graph = None
        if graph:
            if stream is None:
                raise ValueError("graph=True needs a non-default stream")
            self._stream = _stream(stream)
            self._run_calls()                     # first run: checks and set-up outside capture
            _check(L.tk_graph_begin(self._stream), "tk_graph_begin")
            try:
                self._run_calls()
            finally:
                g = ctypes.c_void_p()
                st = L.tk_graph_end(self._stream, ctypes.byref(g))
            _check(st, "tk_graph_end")
            self._graph = g
            self._launch = L.tk_graph_launch
            self._destroy = L.tk_graph_destroy

    def _run_calls(self):
        for fn, args, name in self._calls:
            st = fn(*args)
            if st != TK_OK:
                _check(st, name)

    def __call__(self):
        if self._graph is not None:
            st = self._launch(self._graph, self._stream)
            if st != TK_OK:
                _check(st, "tk_graph_launch")
            return
        self._run_calls()

    def __del__(self):
        g = getattr(self, "_graph", None)
        if g is not None and g.value:
            self._destroy(g)
            self._graph = None


def tk_copy_async(dst, src, stream=None):
    """Stream-ordered copy between device memory and page-locked host memory (same byte size)."""
    for t, n in ((dst, "dst"), (src, "src")):
        if not t.is_contiguous() or not (t.is_cuda or t.is_pinned()):
            raise ValueError(f"{n} must be contiguous, on a GPU or page-locked")
    nb = dst.numel() * dst.element_size()
    if src.numel() * src.element_size() != nb:
        raise ValueError("dst and src differ in size")
    _check(load_library().tk_copy_async(_ptr(dst), _ptr(src), nb, _stream(stream)), "tk_copy_async")
    return dst


def prepare_decode_append(cache: ThinKeyCache, q, k_new, v_new, seq_lens, max_seq_len: int, out,
                          workspace, scale: float | None = None, stream=None,
                          copy_in=None, graph: bool = False) -> PreparedCall:
    """tk_attn_decode_append with every argument checked once (see that function).

    copy_in = (dst, src): a device tensor and a page-locked host tensor of the
    same byte size, copied (tk_copy_async) before each decode -- e.g. the
    step's q, k_new and v_new packed in one host buffer.  `out` may be a
    page-locked host tensor: the kernel then writes the result there directly.
    graph=True records the step (copy and decode) as one CUDA graph launched
    per call; preparing it runs the step twice (once eagerly, once recorded:
    the recorded run does not execute), so the cache gets the new token once."""
    d = cache.desc
    dev = cache.k.device
    for t, n in ((q, "q"), (k_new, "k_new"), (v_new, "v_new")):
        _need(t, torch.bfloat16, n, dev)
    _need(seq_lens, torch.int32, "seq_lens", dev)
    _need(workspace, torch.uint8, "workspace", dev)
    _need_out(out, "out", dev)
    before = ()
    keep_in = ()
    if copy_in is not None:
        dst, src = copy_in
        if not dst.is_cuda or dst.device != dev or not dst.is_contiguous():
            raise ValueError("copy_in: dst must be a contiguous tensor on the cache's device")
        if src.is_cuda or not src.is_pinned() or not src.is_contiguous():
            raise ValueError("copy_in: src must be a contiguous page-locked host tensor")
        nb = dst.numel() * dst.element_size()
        if src.numel() * src.element_size() != nb:
            raise ValueError("copy_in: dst and src differ in size")
        before = (("tk_copy_async", (_ptr(dst), _ptr(src), ctypes.c_size_t(nb), _stream(stream))),)
        keep_in = (dst, src)
    if tuple(q.shape) != (d.batch, d.h_q, d.r) or tuple(out.shape) != (d.batch, d.h_q, d.d_v):
        raise ValueError(f"q {tuple(q.shape)} / out {tuple(out.shape)} do not match the cache")
    if tuple(k_new.shape) != (d.batch, d.h_kv, d.r) or tuple(v_new.shape) != (d.batch, d.h_kv, d.d_v):
        raise ValueError(f"k_new {tuple(k_new.shape)} / v_new {tuple(v_new.shape)} do not match the cache")
    scale = 1.0 / math.sqrt(d.r) if scale is None else float(scale)
    args = (ctypes.byref(d), _ptr(q), _ptr(cache.k), _ptr(cache.v), _ptr(cache.k_scale),
            _ptr(cache.page_table), _ptr(seq_lens), _ptr(k_new), _ptr(v_new), int(max_seq_len),
            _ptr(out), TK_F32 if out.dtype == torch.float32 else TK_BF16, ctypes.c_float(scale),
            _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream(stream))
    return PreparedCall("tk_attn_decode_append", args,
                        (cache, q, k_new, v_new, seq_lens, out, workspace) + keep_in, before,
                        graph=graph, stream=stream)


# ------------------------------------------------- between a projection and the attention

def rope_plan(r: int, rot_dim: int | None = None, layout: str = "half", base: float = 10000.0,
              axes=None, inv_freq=None, pair_axis=None, norm: bool = True, eps: float = 1e-6,
              w_offset: float = 0.0) -> tk_rope_desc:
    """The rotation and norm of a model's queries and keys, built once.

    rot_dim leading elements of a head are rotated (default all r), as pairs (j, j + rot_dim/2)
    (layout "half") or (2j, 2j+1) ("pair").  Frequencies: one position axis and
    base^(-j/pairs) by default; axes=(n0, n1, ...) gives each position axis a run of so many
    pairs with frequencies base^(-i/n) of its own; inv_freq and pair_axis set both freely
    (one entry per pair), e.g. scaled frequencies or axes interleaved over the pairs."""
    rot = r if rot_dim is None else int(rot_dim)
    pairs = rot // 2
    if layout not in ("half", "pair"):
        raise ValueError(f"layout must be 'half' or 'pair', got {layout!r}")
    if axes is not None and inv_freq is not None:
        raise ValueError("axes and inv_freq are exclusive")
    if inv_freq is None:
        axes = None if axes is None else tuple(axes)
        runs = (pairs,) if axes is None else axes
        if any(n < 0 for n in runs) or sum(runs) != pairs:
            raise ValueError(f"axes {runs} do not add up to {pairs} pairs")
        inv_freq = [base ** (-i / n) for n in runs for i in range(n)]
        if pair_axis is None:
            pair_axis = [a for a, n in enumerate(runs) for _ in range(n)]
    inv_freq = [float(f) for f in inv_freq]
    pair_axis = [0] * pairs if pair_axis is None else [int(a) for a in pair_axis]
    if len(inv_freq) != pairs or len(pair_axis) != pairs or pairs > TK_ROPE_MAX_PAIRS:
        raise ValueError(f"{len(inv_freq)} frequencies and {len(pair_axis)} axes for {pairs} pairs "
                         f"(at most {TK_ROPE_MAX_PAIRS})")
    if any(not 0 <= a < TK_ROPE_MAX_AXES for a in pair_axis):
        raise ValueError(f"pair_axis entries must be in 0 .. {TK_ROPE_MAX_AXES - 1}")
    # an axis without pairs is an axis of the positions all the same
    n_axes = max(max(pair_axis, default=0) + 1, 0 if axes is None else len(axes))
    if n_axes > TK_ROPE_MAX_AXES:
        raise ValueError(f"{n_axes} axes (at most {TK_ROPE_MAX_AXES})")
    d = tk_rope_desc(r, rot, TK_ROPE_HALF if layout == "half" else TK_ROPE_PAIR, n_axes, 1 if norm else 0, eps,
                     w_offset)
    d.inv_freq[:pairs] = inv_freq
    d.pair_axis[:pairs] = pair_axis
    return d


_HEADS_DTYPE = {torch.bfloat16: TK_BF16, torch.float32: TK_F32}
_pack_heads = struct.Struct("Piiqqq").pack     # the layout of tk_heads


def _heads(t, name, shape, device):
    """A tk_heads, as bytes, for a tensor of logical shape [B, H, S, width] on the GPU of index
    `device`, any strides with the width contiguous; None for None."""
    if t is None:
        return None
    dt = _HEADS_DTYPE.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} must be float32 or bfloat16")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, expected CUDA device {device}")
    if t.shape != shape:
        raise ValueError(f"{name} is {tuple(t.shape)}, expected {shape}")
    sb, sh, st, sw = t.stride()
    if sw != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return _pack_heads(t.data_ptr(), shape[1], dt, sb, st, sh)


def _weight(t, r, device):
    """A norm weight's address and type, checked; None, None without one."""
    if t is None:
        return None, None
    dt = _HEADS_DTYPE.get(t.dtype)
    if dt is None:
        raise TypeError("norm weights must be float32 or bfloat16")
    if not t.is_cuda or t.device != device or t.numel() != r or not t.is_contiguous():
        raise ValueError(f"a norm weight must be {r} contiguous elements on {device} (CUDA)")
    return t.data_ptr(), dt


def _weights(plan, q_weight, k_weight, device):
    """The weights' addresses and type, checked."""
    if q_weight is None and k_weight is None:
        return None, None, TK_F32
    if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
        raise TypeError("norm weights must be of one dtype")
    q, q_type = _weight(q_weight, plan.r, device)
    k, k_type = _weight(k_weight, plan.r, device)
    return q, k, k_type if q_type is None else q_type


def _positions(plan, positions, B, S, device):
    """(address, axis stride, batch stride) of positions [B, S] or [n_axes, B, S] int32."""
    if positions is None:
        return None, 0, 0
    if positions.dtype is not torch.int32 or positions.device != device:
        raise TypeError(f"positions must be int32 on {device}")
    shape, stride = positions.shape, positions.stride()
    if len(shape) == 2:                       # shared by every axis
        shape, stride = (plan.n_axes, *shape), (0, *stride)
    if shape != (plan.n_axes, B, S):
        raise ValueError(f"positions are {tuple(positions.shape)}, expected {(plan.n_axes, B, S)} or {(B, S)}")
    if stride[2] != 1 and S > 1:
        raise ValueError("positions must be contiguous along the tokens")
    return positions.data_ptr(), stride[0], stride[1]


_current_device = torch._C._cuda_getDevice     # torch.cuda.current_device without its set-up check (0.25 us)


def _need_current(index):
    """The library launches on the current GPU, whatever the stream is of."""
    if index != _current_device():
        raise ValueError(f"the tensors are on CUDA device {index}, the current one is {_current_device()}")


def _first(*tensors):
    """(batch, tokens, device, its index) by the first tensor that is there."""
    for t in tensors:
        if t is not None:
            if t.dim() != 4:
                raise ValueError(f"expected [B, H, S, width] tensors, got {tuple(t.shape)}")
            if not t.is_cuda:
                raise ValueError("expected CUDA tensors")
            B, _, S, _ = t.shape
            at = t.get_device()
            _need_current(at)
            return B, S, t.device, at
    raise ValueError("q, k and v are all None")


def _shape(t, B, S, width):
    return None if t is None else (B, t.shape[1], S, width)


def tk_qk_norm_rope(plan: tk_rope_desc, q, k, v, positions, q_out, k_out, v_out, q_weight=None,
                    k_weight=None, stream=None):
    """Per-head RMS norm and rotation of q [B, H_q, S, r] and k [B, H_kv, S, r], and the layout
    change of v [B, H_kv, S, d_v], in one launch.  Tensors are [B, H, S, width] with any strides
    (a transposed slice of a packed projection, say); bf16 or fp32 in and out.  positions int32
    [B, S] or [n_axes, B, S].  Any of the three may be None together with its output."""
    B, S, dev, at = _first(q, k, v)
    r, dv = plan.r, 0 if v is None else v.shape[3]
    sq, sk, sv = _shape(q, B, S, r), _shape(k, B, S, r), _shape(v, B, S, dv)
    st = load_library().tk_qk_norm_rope(
        ctypes.byref(plan), B, S, dv, _heads(q, "q", sq, at), _heads(k, "k", sk, at), _heads(v, "v", sv, at),
        *_weights(plan, q_weight, k_weight, dev), *_positions(plan, positions, B, S, dev),
        _heads(q_out, "q_out", sq, at), _heads(k_out, "k_out", sk, at), _heads(v_out, "v_out", sv, at),
        _raw_stream(stream, at))
    if st != TK_OK:
        _check(st, "tk_qk_norm_rope")
    return q_out, k_out, v_out


def _append_args(cache, plan, q, k, v, positions, slots, q_out, q_weight, k_weight, stream):
    """Checked and marshalled arguments of tk_qk_norm_rope_append, and what they point into."""
    d = cache.desc
    B, S, dev, at = _first(k)
    if v is None or v.dim() != 4:
        raise ValueError("k and v are required")
    sq, sk = (B, d.h_q, S, plan.r), (B, d.h_kv, S, plan.r)
    _need(slots, torch.int32, "slots", dev)
    if slots.numel() != B * S:
        raise ValueError(f"slots has {slots.numel()} entries for {B * S} tokens")
    for t, n in ((cache.k, "cache.k"), (cache.v, "cache.v"), (cache.k_scale, "cache.k_scale")):
        if t is not None and t.device != dev:
            raise ValueError(f"{n} is on {t.device}, expected {dev}")
    args = (ctypes.byref(d), ctypes.byref(plan), B, S, _heads(q, "q", sq, at), _heads(k, "k", sk, at),
            _heads(v, "v", (B, d.h_kv, S, d.d_v), at), *_weights(plan, q_weight, k_weight, dev),
            *_positions(plan, positions, B, S, dev), _ptr(slots), _heads(q_out, "q_out", sq, at),
            _ptr(cache.k), _ptr(cache.v), _ptr(cache.k_scale), _stream(stream))
    return args, (cache, plan, q, k, v, positions, slots, q_out, q_weight, k_weight)


def tk_qk_norm_rope_append(cache: ThinKeyCache, plan: tk_rope_desc, q, k, v, positions, slots, q_out,
                           q_weight=None, k_weight=None, stream=None):
    """tk_qk_norm_rope with k and v written to the cache at slots [B, S] int32 (tk_block_tables
    makes them; negative = not cached) and q to q_out [B, H_q, S, r] bf16.  q and q_out may be None."""
    args, _keep = _append_args(cache, plan, q, k, v, positions, slots, q_out, q_weight, k_weight, stream)
    _check(load_library().tk_qk_norm_rope_append(*args), "tk_qk_norm_rope_append")
    return q_out


def prepare_qk_norm_rope_append(cache: ThinKeyCache, plan: tk_rope_desc, q, k, v, positions, slots, q_out,
                                q_weight=None, k_weight=None, stream=None,
                                graph: bool = False) -> PreparedCall:
    """tk_qk_norm_rope_append on fixed buffers, checked and marshalled once (see PreparedCall)."""
    args, keep = _append_args(cache, plan, q, k, v, positions, slots, q_out, q_weight, k_weight, stream)
    return PreparedCall("tk_qk_norm_rope_append", args, keep, graph=graph, stream=stream)


def qk_norm_rope_workspace(plan: tk_rope_desc, device="cuda") -> torch.Tensor:
    """A zero-filled workspace of the size tk_qk_norm_rope_backward needs for weight gradients."""
    device = torch.device(device)
    if device.index is not None:
        _need_current(device.index)      # the size goes by its SM count
    n = int(load_library().tk_qk_norm_rope_workspace_size(ctypes.byref(plan)))
    if n == 0:
        raise TkError(TK_ERR_INVALID_ARG, "tk_qk_norm_rope_workspace_size", tk_last_error())
    return torch.zeros(n, dtype=torch.uint8, device=device)


def tk_qk_norm_rope_backward(plan: tk_rope_desc, q, k, positions, dq_out, dk_out, dv_out, dq, dk, dv,
                             q_weight=None, k_weight=None, dq_weight=None, dk_weight=None,
                             workspace=None, stream=None):
    """Gradients of tk_qk_norm_rope: from dq_out, dk_out, dv_out (gradients of its outputs, fp32 as
    tk_attn_backward writes them, or bf16) to dq, dk, dv (the inputs' dtype, any strides: slices of
    a packed gradient, say) and the weights' dq_weight, dk_weight [r] fp32.  q and k (the
    forward's inputs) may be None for a plan without norm.  Weight gradients need a workspace
    (qk_norm_rope_workspace; allocated here if None)."""
    B, S, dev, at = _first(dq_out, dk_out, dv_out)
    r, width = plan.r, 0 if dv_out is None else dv_out.shape[3]
    sq, sk, sv = _shape(dq_out, B, S, r), _shape(dk_out, B, S, r), _shape(dv_out, B, S, width)
    if not plan.norm:
        q = k = None
    dwq, dwq_type = _weight(dq_weight, r, dev)
    dwk, dwk_type = _weight(dk_weight, r, dev)
    if TK_BF16 in (dwq_type, dwk_type):
        raise TypeError("weight gradients must be float32")
    if workspace is None:
        if dwq is not None or dwk is not None:
            with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
                workspace = qk_norm_rope_workspace(plan, dev)   # zeroed, and freed, in the call's stream
    elif workspace.dtype is not torch.uint8 or workspace.get_device() != at or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous uint8 on {dev}")
    st = load_library().tk_qk_norm_rope_backward(
        ctypes.byref(plan), B, S, width, _heads(q, "q", sq, at), _heads(k, "k", sk, at),
        *_weights(plan, q_weight, k_weight, dev), *_positions(plan, positions, B, S, dev),
        _heads(dq_out, "dq_out", sq, at), _heads(dk_out, "dk_out", sk, at), _heads(dv_out, "dv_out", sv, at),
        _heads(dq, "dq", sq, at), _heads(dk, "dk", sk, at), _heads(dv, "dv", sv, at), dwq, dwk,
        None if workspace is None else workspace.data_ptr(),
        0 if workspace is None else workspace.numel(), _raw_stream(stream, at))
    if st != TK_OK:
        _check(st, "tk_qk_norm_rope_backward")
    return dq, dk, dv


@dataclass
class PagePool:
    """The page tables of a batch and the free pages of a paged cache (all int32, on one device).

    page_table [B, max_pages], free_pages [num_pages] with its first free_count[0] entries in
    use, free_count [1], seq_lens [B] tokens cached per sequence, workspace [1] (zero)."""
    page_size: int
    page_table: torch.Tensor
    free_pages: torch.Tensor
    free_count: torch.Tensor
    seq_lens: torch.Tensor
    workspace: torch.Tensor

    @staticmethod
    def allocate(batch, max_pages, page_size, num_pages, device="cuda"):
        """An empty pool: every page free, every sequence empty."""
        i32 = dict(dtype=torch.int32, device=device)
        return PagePool(page_size, torch.full((batch, max_pages), -1, **i32),
                        torch.arange(num_pages - 1, -1, -1, **i32), torch.full((1,), num_pages, **i32),
                        torch.zeros(batch, **i32), torch.zeros(1, **i32))


def _table_args(pool, new_lens, slots, positions, tokens_per_seq, offsets, seq_lens_out, free_count_out,
                refused, stream):
    dev = pool.page_table.device
    if pool.page_table.dim() != 2:
        raise ValueError("page_table must be [B, max_pages]")
    B, max_pages = pool.page_table.shape
    seq_lens_out = pool.seq_lens if seq_lens_out is None else seq_lens_out
    free_count_out = pool.free_count if free_count_out is None else free_count_out
    num_pages, rows = pool.free_pages.numel(), slots.numel()
    for t, n, size in ((pool.page_table, "page_table", B * max_pages), (pool.free_pages, "free_pages", num_pages),
                       (pool.free_count, "free_count", 1), (pool.seq_lens, "seq_lens", B),
                       (pool.workspace, "workspace", 1), (new_lens, "new_lens", B), (slots, "slots", rows),
                       (positions, "positions", rows), (offsets, "offsets", B + 1),
                       (seq_lens_out, "seq_lens_out", B), (free_count_out, "free_count_out", 1),
                       (refused, "refused", 1)):
        _need(t, torch.int32, n, dev)
        if t is not None and t.numel() != size:
            raise ValueError(f"{n} has {t.numel()} elements, expected {size}")
    _need_current(dev.index)
    args = (B, pool.page_size, num_pages, max_pages, _ptr(pool.seq_lens), _ptr(new_lens), _ptr(pool.page_table),
            _ptr(pool.free_pages), _ptr(pool.free_count), int(tokens_per_seq), rows, _ptr(slots),
            _ptr(positions), _ptr(offsets), _ptr(seq_lens_out), _ptr(free_count_out), _ptr(refused),
            _ptr(pool.workspace), _stream(stream))
    return args, (pool, new_lens, slots, positions, offsets, seq_lens_out, free_count_out, refused)


def tk_block_tables(pool: PagePool, new_lens, slots, positions, tokens_per_seq: int = 0, offsets=None,
                    seq_lens_out=None, free_count_out=None, refused=None, stream=None):
    """Pages, slots and positions of a step's new tokens: new_lens [B] int32 per sequence (0 idle,
    -1 finished: its pages are freed) -> the pool's page table and free stack updated, slots
    and positions [rows] filled (padded [B, tokens_per_seq], or packed by offsets [B + 1] when
    tokens_per_seq is 0).  seq_lens and free_count are updated in place unless outputs are given;
    refused [1] counts requests that did not fit (their length stays).  See include/tk.h."""
    args, _keep = _table_args(pool, new_lens, slots, positions, tokens_per_seq, offsets, seq_lens_out,
                              free_count_out, refused, stream)
    _check(load_library().tk_block_tables(*args), "tk_block_tables")
    return slots, positions


def prepare_block_tables(pool: PagePool, new_lens, slots, positions, tokens_per_seq: int = 0, offsets=None,
                         seq_lens_out=None, free_count_out=None, refused=None, stream=None,
                         graph: bool = False) -> PreparedCall:
    """tk_block_tables on fixed buffers, checked and marshalled once (see PreparedCall).  With
    graph=True preparing runs the step once; every call is one more step."""
    args, keep = _table_args(pool, new_lens, slots, positions, tokens_per_seq, offsets, seq_lens_out,
                             free_count_out, refused, stream)
    return PreparedCall("tk_block_tables", args, keep, graph=graph, stream=stream)


# ------------------------------------------------------- a long context, read or kept in part

def _lead(cache):
    """The leading dimensions of a cache's tensors: [P, H_kv, page_size] or [B, H_kv, capacity]."""
    d = cache.desc
    return (d.num_pages, d.h_kv, d.page_size) if d.page_size else (d.batch, d.h_kv, d.capacity)


def _cache_tensors(cache, device, keys=False, values=False):
    """Checks the tensors of the cache that a call reads, and the current GPU."""
    d = cache.desc
    lead = _lead(cache)
    if keys or values:
        width = d.r // 2 if d.k_dtype == TK_I4 else d.r
        key = {TK_BF16: torch.bfloat16, TK_I8: torch.int8, TK_I4: torch.uint8}.get(d.k_dtype)
        want = [(cache.k, key, "cache.k", (*lead, width))]
        if d.k_dtype != TK_BF16:
            want.append((cache.k_scale, torch.float32, "cache.k_scale", lead))
        if values:
            want.append((cache.v, torch.bfloat16, "cache.v", (*lead, d.d_v)))
        for t, dt, n, shape in want:
            if t is None:
                raise ValueError(f"{n} is None")
            _need(t, dt, n, device)
            if tuple(t.shape) != shape:
                raise ValueError(f"{n} is {tuple(t.shape)}, expected {shape}")
    if d.page_size:
        if cache.page_table is None:
            raise ValueError("a paged cache needs a page table")
        _need(cache.page_table, torch.int32, "cache.page_table", device)
        if tuple(cache.page_table.shape) != (d.batch, d.max_pages_per_seq):
            raise ValueError(f"cache.page_table is {tuple(cache.page_table.shape)}, expected "
                             f"{(d.batch, d.max_pages_per_seq)}")
    _need_current(device.index)


def _need_shape(t, dtype, name, shape, device):
    if t is None:
        return
    _need(t, dtype, name, device)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} is {tuple(t.shape)}, expected {tuple(shape)}")


def _device(t, name):
    if t is None or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t.device


def _block(cache, block):
    """Tokens of a block: the page of a paged cache, 64 by default of a contiguous one."""
    d = cache.desc
    return int(block) if block else (d.page_size or 64)


def _check_block(cache, block):
    d = cache.desc
    if block < 16 or block > 256 or block & (block - 1):
        raise ValueError(f"block {block} must be a power of two of 16 .. 256")
    if (d.page_size or d.capacity) % block or (d.page_size and block != d.page_size):
        raise ValueError(f"block {block} does not fit a cache of page size {d.page_size}, capacity {d.capacity}")


def _bounds_shape(cache, block):
    d = cache.desc
    lead = (d.num_pages, d.h_kv) if d.page_size else (d.batch, d.h_kv, d.capacity // block)
    return (*lead, 2, d.r)


def block_bounds(cache: ThinKeyCache, block: int | None = None) -> torch.Tensor:
    """Zeroed bounds of every block of the cache for tk_block_bounds: bf16
    [P, H_kv, 2, r] (paged: a block is a page) or [B, H_kv, capacity / block, 2, r]."""
    block = _block(cache, block)
    _check_block(cache, block)
    return torch.zeros(_bounds_shape(cache, block), dtype=torch.bfloat16, device=cache.k.device)


def _bounds_args(cache, bounds, seq_lens, old_lens, max_new, block, stream):
    d = cache.desc
    dev = _device(bounds, "bounds")
    block = _block(cache, block)
    _check_block(cache, block)
    _cache_tensors(cache, dev, keys=True)
    _need_shape(bounds, torch.bfloat16, "bounds", _bounds_shape(cache, block), dev)
    _need_shape(seq_lens, torch.int32, "seq_lens", (d.batch,), dev)
    _need_shape(old_lens, torch.int32, "old_lens", (d.batch,), dev)
    if max_new is None:
        max_new = d.max_pages_per_seq * d.page_size if d.page_size else d.capacity
    args = (ctypes.byref(d), block, _ptr(cache.k), _ptr(cache.k_scale), _ptr(cache.page_table), _ptr(old_lens),
            _ptr(seq_lens), int(max_new), _ptr(bounds), _stream(stream))
    return args, (cache, bounds, seq_lens, old_lens)


def tk_block_bounds(cache: ThinKeyCache, bounds, seq_lens, old_lens=None, max_new: int | None = None,
                    block: int | None = None, stream=None):
    """Minimum and maximum of the keys of each block that holds a token at old_lens[b] ..
    seq_lens[b] - 1 (int32 [B]; old_lens None: of every block), into bounds (see block_bounds).
    max_new bounds seq_lens - old_lens (default: the whole cache)."""
    args, _keep = _bounds_args(cache, bounds, seq_lens, old_lens, max_new, block, stream)
    _check(load_library().tk_block_bounds(*args), "tk_block_bounds")
    return bounds


def prepare_block_bounds(cache: ThinKeyCache, bounds, seq_lens, old_lens=None, max_new: int | None = None,
                         block: int | None = None, stream=None, graph: bool = False) -> PreparedCall:
    """tk_block_bounds on fixed buffers, checked and marshalled once (see PreparedCall)."""
    args, keep = _bounds_args(cache, bounds, seq_lens, old_lens, max_new, block, stream)
    return PreparedCall("tk_block_bounds", args, keep, graph=graph, stream=stream)


@dataclass
class BlockSelection:
    """The blocks that a decode step reads, per sequence and kv head.

    block: tokens of a block.  table [B * H_kv, n_select] int32: each block's place in the cache
    (page * H_kv + g, or (b * H_kv + g) * (capacity / block) + block; -1: none), lens
    [B * H_kv] int32: tokens in them; ids [B, H_kv, n_select] int32 or None: the blocks' numbers
    in their sequence."""
    block: int
    table: torch.Tensor
    lens: torch.Tensor
    ids: torch.Tensor | None = None

    @staticmethod
    def allocate(cache: ThinKeyCache, n_select: int, block: int | None = None, ids: bool = False):
        """An empty selection (decoding over it gives zero rows)."""
        d = cache.desc
        i32 = dict(dtype=torch.int32, device=cache.k.device)
        pairs = d.batch * d.h_kv
        return BlockSelection(_block(cache, block), torch.full((pairs, n_select), -1, **i32),
                              torch.zeros(pairs, **i32),
                              torch.full((d.batch, d.h_kv, n_select), -1, **i32) if ids else None)


def _need_selection(cache, sel, dev):
    d = cache.desc
    _check_block(cache, sel.block)
    if sel.table.dim() != 2:
        raise ValueError("selection.table must be [B * H_kv, n_select]")
    n = sel.table.shape[1]
    _need_shape(sel.table, torch.int32, "selection.table", (d.batch * d.h_kv, n), dev)
    _need_shape(sel.lens, torch.int32, "selection.lens", (d.batch * d.h_kv,), dev)
    _need_shape(sel.ids, torch.int32, "selection.ids", (d.batch, d.h_kv, n), dev)
    return n


def _select_args(cache, q, bounds, seq_lens, max_seq_len, sel, n_first, n_last, stream):
    d = cache.desc
    dev = _device(q, "q")
    _cache_tensors(cache, dev)
    n = _need_selection(cache, sel, dev)
    _need_shape(q, torch.bfloat16, "q", (d.batch, d.h_q, d.r), dev)
    _need_shape(bounds, torch.bfloat16, "bounds", _bounds_shape(cache, sel.block), dev)
    _need_shape(seq_lens, torch.int32, "seq_lens", (d.batch,), dev)
    args = (ctypes.byref(d), sel.block, _ptr(q), _ptr(bounds), _ptr(cache.page_table), _ptr(seq_lens),
            int(max_seq_len), n, int(n_first), int(n_last), _ptr(sel.table), _ptr(sel.lens), _ptr(sel.ids),
            _stream(stream))
    return args, (cache, q, bounds, seq_lens, sel, sel.table, sel.lens, sel.ids)


def tk_block_select(cache: ThinKeyCache, q, bounds, seq_lens, max_seq_len: int, selection: BlockSelection,
                    n_first: int = 1, n_last: int = 1, stream=None):
    """For q [B, H_q, r] bf16: the n_select blocks of each kv head whose keys can score highest by
    their bounds, into `selection`; the first n_first and last n_last blocks of a context are
    always among them."""
    args, _keep = _select_args(cache, q, bounds, seq_lens, max_seq_len, selection, n_first, n_last, stream)
    _check(load_library().tk_block_select(*args), "tk_block_select")
    return selection


def prepare_block_select(cache: ThinKeyCache, q, bounds, seq_lens, max_seq_len: int, selection: BlockSelection,
                         n_first: int = 1, n_last: int = 1, stream=None, graph: bool = False) -> PreparedCall:
    """tk_block_select on fixed buffers, checked and marshalled once (see PreparedCall)."""
    args, keep = _select_args(cache, q, bounds, seq_lens, max_seq_len, selection, n_first, n_last, stream)
    return PreparedCall("tk_block_select", args, keep, graph=graph, stream=stream)


def decode_blocks_workspace(cache: ThinKeyCache, selection: BlockSelection) -> torch.Tensor:
    """A zero-filled workspace of the size tk_attn_decode_blocks needs."""
    dev = _device(selection.table, "selection.table")
    _need_current(dev.index)
    n = int(load_library().tk_decode_blocks_workspace_size(ctypes.byref(cache.desc), selection.block,
                                                           selection.table.shape[1]))
    if n == 0:
        raise TkError(TK_ERR_INVALID_ARG, "tk_decode_blocks_workspace_size", tk_last_error())
    return torch.zeros(n, dtype=torch.uint8, device=dev)


def _decode_blocks_args(cache, q, sel, out, workspace, scale, stream):
    d = cache.desc
    dev = _device(q, "q")
    _cache_tensors(cache, dev, values=True)
    n = _need_selection(cache, sel, dev)
    _need_shape(q, torch.bfloat16, "q", (d.batch, d.h_q, d.r), dev)
    _need_out(out, "out", dev)
    if tuple(out.shape) != (d.batch, d.h_q, d.d_v):
        raise ValueError(f"out is {tuple(out.shape)}, expected {(d.batch, d.h_q, d.d_v)}")
    _need(workspace, torch.uint8, "workspace", dev)
    scale = 1.0 / math.sqrt(d.r) if scale is None else float(scale)
    args = (ctypes.byref(d), sel.block, _ptr(q), _ptr(cache.k), _ptr(cache.v), _ptr(cache.k_scale),
            _ptr(sel.table), _ptr(sel.lens), n, _ptr(out), TK_F32 if out.dtype == torch.float32 else TK_BF16,
            ctypes.c_float(scale), _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream(stream))
    return args, (cache, q, sel, sel.table, sel.lens, out, workspace)


def tk_attn_decode_blocks(cache: ThinKeyCache, q, selection: BlockSelection, out, workspace,
                          scale: float | None = None, stream=None):
    """tk_attn_decode of q [B, H_q, r] over the blocks of `selection` alone."""
    args, _keep = _decode_blocks_args(cache, q, selection, out, workspace, scale, stream)
    _check(load_library().tk_attn_decode_blocks(*args), "tk_attn_decode_blocks")
    return out


def prepare_attn_decode_blocks(cache: ThinKeyCache, q, selection: BlockSelection, out, workspace,
                               scale: float | None = None, stream=None, graph: bool = False) -> PreparedCall:
    """tk_attn_decode_blocks on fixed buffers, checked and marshalled once (see PreparedCall)."""
    args, keep = _decode_blocks_args(cache, q, selection, out, workspace, scale, stream)
    return PreparedCall("tk_attn_decode_blocks", args, keep, graph=graph, stream=stream)


def slot_weights(cache: ThinKeyCache) -> torch.Tensor:
    """Zeroed accumulated weights of every slot of the cache: fp32, laid out as k_scale."""
    return torch.zeros(_lead(cache), dtype=torch.float32, device=cache.k.device)


def attn_weights_workspace(cache: ThinKeyCache, max_seq_len: int, n_queries: int = 1) -> torch.Tensor:
    """A workspace of the size tk_attn_weights needs for contexts of max_seq_len tokens or fewer."""
    dev = _device(cache.k, "cache.k")
    _need_current(dev.index)
    n = int(load_library().tk_attn_weights_workspace_size(ctypes.byref(cache.desc), int(n_queries), int(max_seq_len)))
    if n == 0:
        raise TkError(TK_ERR_INVALID_ARG, "tk_attn_weights_workspace_size", tk_last_error())
    return torch.empty(n, dtype=torch.uint8, device=dev)


def _weights_args(cache, q, seq_lens, max_seq_len, weights, workspace, old_lens, decay, scale, stream):
    d = cache.desc
    dev = _device(q, "q")
    _cache_tensors(cache, dev, keys=True)
    if q.dim() == 3:
        q = q.unsqueeze(2)
    if q.dim() != 4:
        raise ValueError(f"q is {tuple(q.shape)}, expected [B, H_q, r] or [B, H_q, n, r]")
    n = q.shape[2]
    _need_shape(q, torch.bfloat16, "q", (d.batch, d.h_q, n, d.r), dev)
    _need_shape(seq_lens, torch.int32, "seq_lens", (d.batch,), dev)
    _need_shape(old_lens, torch.int32, "old_lens", (d.batch,), dev)
    _need_shape(weights, torch.float32, "weights", _lead(cache), dev)
    _need(workspace, torch.uint8, "workspace", dev)
    scale = 1.0 / math.sqrt(d.r) if scale is None else float(scale)
    args = (ctypes.byref(d), _ptr(q), n, _ptr(cache.k), _ptr(cache.k_scale), _ptr(cache.page_table), _ptr(old_lens),
            _ptr(seq_lens), int(max_seq_len), ctypes.c_float(scale), ctypes.c_float(decay), _ptr(weights),
            _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream(stream))
    return args, (cache, q, seq_lens, weights, workspace, old_lens)


def tk_attn_weights(cache: ThinKeyCache, q, seq_lens, max_seq_len: int, weights, workspace, old_lens=None,
                    decay: float = 1.0, scale: float | None = None, stream=None):
    """Adds the attention weights of q [B, H_q, r] (or the last n queries, [B, H_q, n, r]) over the
    cached tokens, their own included, to weights (slot_weights), summed over the query heads
    of a kv head.  Tokens from old_lens[b] on (None: all) have no weight yet; the earlier ones'
    is multiplied by decay first."""
    args, _keep = _weights_args(cache, q, seq_lens, max_seq_len, weights, workspace, old_lens, decay, scale, stream)
    _check(load_library().tk_attn_weights(*args), "tk_attn_weights")
    return weights


def prepare_attn_weights(cache: ThinKeyCache, q, seq_lens, max_seq_len: int, weights, workspace, old_lens=None,
                         decay: float = 1.0, scale: float | None = None, stream=None,
                         graph: bool = False) -> PreparedCall:
    """tk_attn_weights on fixed buffers, checked and marshalled once (see PreparedCall).  With
    graph=True preparing adds the weights once."""
    args, keep = _weights_args(cache, q, seq_lens, max_seq_len, weights, workspace, old_lens, decay, scale, stream)
    return PreparedCall("tk_attn_weights", args, keep, graph=graph, stream=stream)


def cache_evict_workspace(cache: ThinKeyCache, n_keep: int) -> torch.Tensor:
    """A workspace of the size tk_cache_evict needs."""
    n = int(load_library().tk_cache_evict_workspace_size(ctypes.byref(cache.desc), int(n_keep)))
    if n == 0:
        raise TkError(TK_ERR_INVALID_ARG, "tk_cache_evict_workspace_size", tk_last_error())
    return torch.empty(n, dtype=torch.uint8, device=cache.k.device)


def _evict_args(cache, seq_lens, max_seq_len, weights, n_keep, n_recent, workspace, weights_out, seq_lens_out, kept,
                pool, stream):
    d = cache.desc
    dev = _device(weights, "weights")
    _cache_tensors(cache, dev, values=True)
    weights_out = weights if weights_out is None else weights_out
    seq_lens_out = seq_lens if seq_lens_out is None else seq_lens_out
    _need_shape(seq_lens, torch.int32, "seq_lens", (d.batch,), dev)
    _need_shape(seq_lens_out, torch.int32, "seq_lens_out", (d.batch,), dev)
    _need_shape(weights, torch.float32, "weights", _lead(cache), dev)
    _need_shape(weights_out, torch.float32, "weights_out", _lead(cache), dev)
    _need_shape(kept, torch.int32, "kept", (d.batch, d.h_kv, n_keep), dev)
    _need(workspace, torch.uint8, "workspace", dev)
    free = count = None
    if pool is not None:
        free, count = pool.free_pages, pool.free_count
        _need_shape(free, torch.int32, "free_pages", (d.num_pages,), dev)
        _need_shape(count, torch.int32, "free_count", (1,), dev)
        if cache.page_table is None or pool.page_table.data_ptr() != cache.page_table.data_ptr():
            raise ValueError("the pool's page table is not the cache's")
    args = (ctypes.byref(d), _ptr(cache.k), _ptr(cache.v), _ptr(cache.k_scale), _ptr(cache.page_table),
            _ptr(seq_lens), int(max_seq_len), _ptr(weights), int(n_keep), int(n_recent), _ptr(weights_out),
            _ptr(seq_lens_out), _ptr(kept), _ptr(free), _ptr(count), _ptr(workspace),
            ctypes.c_size_t(workspace.numel()), _stream(stream))
    return args, (cache, seq_lens, weights, workspace, weights_out, seq_lens_out, kept, pool, free, count)


def tk_cache_evict(cache: ThinKeyCache, seq_lens, max_seq_len: int, weights, n_keep: int, n_recent: int, workspace,
                   weights_out=None, seq_lens_out=None, kept=None, pool: PagePool | None = None, stream=None):
    """Cuts contexts of more than n_keep tokens to the last n_recent and the n_keep - n_recent others
    with the largest weights of each kv head, moved into slots 0 .. n_keep - 1 of the cache.
    weights and seq_lens are updated in place unless outputs are given; kept [B, H_kv, n_keep] int32
    tells where each token was; pool (a PagePool of this cache) gets the pages back that
    hold no token any more.  See include/tk.h."""
    args, _keep = _evict_args(cache, seq_lens, max_seq_len, weights, n_keep, n_recent, workspace, weights_out,
                              seq_lens_out, kept, pool, stream)
    _check(load_library().tk_cache_evict(*args), "tk_cache_evict")


def prepare_cache_evict(cache: ThinKeyCache, seq_lens, max_seq_len: int, weights, n_keep: int, n_recent: int,
                        workspace, weights_out=None, seq_lens_out=None, kept=None, pool: PagePool | None = None,
                        stream=None, graph: bool = False) -> PreparedCall:
    """tk_cache_evict on fixed buffers, checked and marshalled once (see PreparedCall).  With
    graph=True preparing evicts once, so contexts that are over n_keep by then are cut."""
    args, keep = _evict_args(cache, seq_lens, max_seq_len, weights, n_keep, n_recent, workspace, weights_out,
                             seq_lens_out, kept, pool, stream)
    return PreparedCall("tk_cache_evict", args, keep, graph=graph, stream=stream)


def tk_attn_prefill(q, k, v, out, scale: float | None = None, causal: bool = True, stream=None):
    """Prefill: q [B, H_q, S, r], k [B, H_kv, S, r], v [B, H_kv, S, d_v] bf16 -> out [B, H_q, S, d_v]."""
    dev = q.device
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, n, dev)
    if out.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("out must be float32 or bfloat16")
    _need(out, out.dtype, "out", dev)
    B, hq, S, r = q.shape
    hkv, dv = k.shape[1], v.shape[3]
    if tuple(k.shape) != (B, hkv, S, r) or tuple(v.shape) != (B, hkv, S, dv) or \
            tuple(out.shape) != (B, hq, S, dv):
        raise ValueError("q / k / v / out shapes are inconsistent")
    scale = 1.0 / math.sqrt(r) if scale is None else float(scale)
    L = load_library()
    _check(L.tk_attn_prefill(_ptr(q), _ptr(k), _ptr(v), _ptr(out),
                             TK_F32 if out.dtype == torch.float32 else TK_BF16,
                             B, hq, hkv, S, r, dv, scale, 1 if causal else 0, _stream(stream)),
           "tk_attn_prefill")
    return out


def tk_attn_decode_noalloc(cache: ThinKeyCache, q, seq_lens, max_seq_len: int, out,
                           scale: float | None = None, stream=None):
    """tk_attn_decode without a workspace: uses the library's fixed device scratch.

    For callers that cannot allocate device memory.  Calls that may overlap on
    the GPU share the scratch and race; see include/tk.h.
    """
    d = cache.desc
    dev = cache.k.device
    _need(q, torch.bfloat16, "q", dev)
    _need(seq_lens, torch.int32, "seq_lens", dev)
    _need_out(out, "out", dev)
    if tuple(q.shape) != (d.batch, d.h_q, d.r) or tuple(out.shape) != (d.batch, d.h_q, d.d_v):
        raise ValueError(f"q {tuple(q.shape)} / out {tuple(out.shape)} do not match the cache")
    scale = 1.0 / math.sqrt(d.r) if scale is None else float(scale)
    L = load_library()
    _check(L.tk_attn_decode_noalloc(ctypes.byref(d), _ptr(q), _ptr(cache.k), _ptr(cache.v),
                                    _ptr(cache.k_scale), _ptr(cache.page_table), _ptr(seq_lens),
                                    int(max_seq_len), _ptr(out),
                                    TK_F32 if out.dtype == torch.float32 else TK_BF16, scale,
                                    _stream(stream)), "tk_attn_decode_noalloc")
    return out


def tk_check_wait_timeout(limit_us: int, stream=None):
    """Run the failure-detection diagnostic: a bounded wait that must run out
    after limit_us microseconds and record code 2 (see include/tk.h)."""
    _check(load_library().tk_check_wait_timeout(int(limit_us), _stream(stream)),
           "tk_check_wait_timeout")


def tk_get_device_error(stream=None) -> int:
    """Synchronise the stream and return (and clear) the device error word (0 = none)."""
    code = ctypes.c_int32(0)
    st = load_library().tk_get_device_error(ctypes.byref(code), _stream(stream))
    if st not in (TK_OK, TK_ERR_DEVICE):
        _check(st, "tk_get_device_error")
    return int(code.value)
