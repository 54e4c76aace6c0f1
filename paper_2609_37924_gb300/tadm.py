"""Thin ctypes binding of libtadm (include/tadm.h).

Functions keep the C names and only marshal arguments: every step of the
sampling loop runs in the library's CUDA kernels.  PyTorch provides device
memory and streams.  Loading fails loudly when the library is missing; there
is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "_lib", "libtadm.so")

TADM_OK = 0
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "CUDA", 4: "OOM", 5: "TIMEOUT", 6: "STATE"}

ABI_FUNCTIONS = [
    "tadm_weight_count", "tadm_weight_info", "tadm_create", "tadm_destroy", "tadm_last_error",
    "tadm_status_string", "tadm_workspace_size", "tadm_bind_workspace", "tadm_cache_size", "tadm_reset",
    "tadm_prefill", "tadm_anchor_forward", "tadm_denoise_step", "tadm_commit_block", "tadm_generate",
    "tadm_sync_status", "tadm_get_counters", "tadm_plan", "tadm_layer_cost", "tadm_gemm", "tadm_confidence",
    "tadm_topk_unmask", "tadm_attention", "tadm_probe_enable", "tadm_probe_read", "tadm_head_scratch_size",
    "tadm_head_confidence", "tadm_head_confidence_static", "tadm_probe_breakdown",
    "tadm_remdm_schedule", "tadm_remdm_uniforms", "tadm_remdm_update", "tadm_generate_remdm",
    "tadm_eb_update", "tadm_eb_scratch_bytes", "tadm_generate_entropy_bound",
    "tadm_ragged_sync_status", "tadm_attention_packed", "tadm_page_write", "tadm_page_read", "tadm_page_attention_scratch_size",
    "tadm_page_attention", "tadm_pages_scratch_size", "tadm_pages_reserve", "tadm_pages_fork", "tadm_pages_free",
    "tadm_pages_compact", "tadm_pages_copy",
    "tadm_sample_scratch_size", "tadm_sample", "tadm_lora_scratch_size", "tadm_lora_project", "tadm_residual_norm",
]


class TadmError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class tadm_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "vocab", "d_model", "n_heads", "n_kv_heads", "head_dim", "ffn", "glu", "n_shared", "n_anchor",
        "n_denoise", "fusion", "fusion_rank", "fusion_heads", "dtype", "tied_lm_head")] + [
        ("norm_eps", ctypes.c_float), ("rope_theta", ctypes.c_float)] + [
        (n, ctypes.c_int32) for n in ("sliding_window", "global_every", "qk_norm", "sandwich_norm")] + [
        ("rope_theta_global", ctypes.c_float), ("qkv_split", ctypes.c_int32)]


class tadm_step_outputs(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("conf", ctypes.c_void_p), ("tok", ctypes.c_void_p),
                ("selected", ctypes.c_void_p), ("fused", ctypes.c_void_p)]


class tadm_counters(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "shared_layers", "anchor_layers", "denoise_layers", "anchor_calls", "denoise_steps", "commit_passes",
        "kernel_launches")]


class tadm_page_pool(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in (
                    "layers", "pages", "n_kv_heads", "head_dim")]


class tadm_plan_event(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("kind", "block", "n", "k")]


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libtadm.so (built in-tree by ``__graft_entry__.build()``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: build it with __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    P, I, I64, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    cfgp = ctypes.POINTER(tadm_config)
    sig = {
        "tadm_weight_count": (I, [cfgp]),
        "tadm_weight_info": (I, [cfgp, I, ctypes.c_char_p, I, ctypes.POINTER(I64), ctypes.POINTER(I64)]),
        "tadm_create": (I, [cfgp, ctypes.POINTER(P), I, I, I, I, ctypes.POINTER(P)]),
        "tadm_destroy": (None, [P]),
        "tadm_last_error": (ctypes.c_char_p, [P]),
        "tadm_status_string": (ctypes.c_char_p, [I]),
        "tadm_workspace_size": (I, [P, ctypes.POINTER(SZ)]),
        "tadm_bind_workspace": (I, [P, P, SZ]),
        "tadm_cache_size": (I, [P, I, I, ctypes.POINTER(SZ)]),
        "tadm_reset": (I, [P, I]),
        "tadm_prefill": (I, [P, P, I, I, P]),
        "tadm_anchor_forward": (I, [P, P, I, I, I, P, P]),
        "tadm_denoise_step": (I, [P, P, I, I, I, I, I, P, ctypes.POINTER(tadm_step_outputs), P]),
        "tadm_commit_block": (I, [P, P, I, I, P]),
        "tadm_generate": (I, [P, P, I, I, P, I, I, I, I, P]),
        "tadm_sync_status": (I, [P]),
        "tadm_get_counters": (I, [P, ctypes.POINTER(tadm_counters)]),
        "tadm_plan": (I, [I, I, I, I, I, ctypes.POINTER(tadm_plan_event), I, ctypes.POINTER(I)]),
        "tadm_layer_cost": (I, [I, I, I, I, I, ctypes.POINTER(I64), ctypes.POINTER(I64)]),
        "tadm_gemm": (I, [P, P, P, I, I, I, I, I, I, I, I, P]),
        "tadm_confidence": (I, [P, I, I, I, P, P, P]),
        "tadm_topk_unmask": (I, [P, I, P, P, I, I, I, I, P, P]),
        "tadm_attention": (I, [P, P, P, P, I, I, I, I, I, I, I, I, I, I, P]),
        "tadm_head_scratch_size": (I, [I, I, I, ctypes.POINTER(SZ)]),
        "tadm_head_confidence": (I, [P, P, I, I, I, I, I, P, SZ, P, P, P]),
        "tadm_head_confidence_static": (I, [P, P, I, I, I, I, I, P, P, P]),
        "tadm_probe_enable": (I, [P, I]),
        "tadm_remdm_schedule": (I, [I, I, I, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                    ctypes.POINTER(ctypes.c_double)]),
        "tadm_remdm_uniforms": (I, [ctypes.c_uint64, I, I, I, P, P]),
        "tadm_remdm_update": (I, [P, I, P, I, I, I, I, I, I, ctypes.c_double, ctypes.c_double, ctypes.c_float,
                                  ctypes.c_uint64, I, P, P]),
        "tadm_generate_remdm": (I, [P, P, I, I, P, I, I, I, I, ctypes.c_double, ctypes.c_float, ctypes.c_uint64, P,
                                    SZ, P]),
        "tadm_eb_update": (I, [P, I, P, I, I, I, I, I, I, ctypes.c_double, ctypes.c_double, I, ctypes.c_uint64, I,
                               P, P, I, I, P, P]),
        "tadm_eb_scratch_bytes": (I, [P, I, I, I, ctypes.POINTER(SZ)]),
        "tadm_generate_entropy_bound": (I, [P, P, I, I, P, I, I, I, ctypes.c_double, ctypes.c_double,
                                            ctypes.c_double, I, ctypes.c_uint64, P, SZ, P]),
        "tadm_ragged_sync_status": (I, [P]),
        "tadm_attention_packed": (I, [P] * 5 + [I] * 6 + [I64] * 4 + [I] * 3 + [P]),
        "tadm_page_write": (I, [P, I, P, P, P, P, I, I, I, I64, I64, P, I, I, P]),
        "tadm_page_read": (I, [P, I, P, P, P, P, I, I, I, I64, I64, P, I, I, P]),
        "tadm_page_attention_scratch_size": (I, [I] * 8 + [ctypes.POINTER(SZ)]),
        "tadm_page_attention": (I, [P, P, I, P, P, P, I, I, I, I, I, I64, I64, P, I, I, I, I, P, SZ, P]),
        "tadm_pages_scratch_size": (I, [I, I, ctypes.POINTER(SZ)]),
        "tadm_pages_reserve": (I, [P, P, I, I, I, P, P, I, P, P, P, P, SZ, P]),
        "tadm_pages_fork": (I, [P, P, P, P, I, I, P, P, I, P, P, P, P, P, SZ, P]),
        "tadm_pages_free": (I, [P, P, P, I, I, I, P, I, P, P, P, P, P, SZ, P]),
        "tadm_pages_compact": (I, [P, P, P, I, I, P, P, P, P, SZ, P]),
        "tadm_pages_copy": (I, [P, P, P, I, P]),
        "tadm_sample_scratch_size": (I, [I, I, ctypes.POINTER(SZ)]),
        "tadm_sample": (I, [P, I64, I, I, I] + [P] * 7 + [I, P, SZ, P]),
        "tadm_lora_scratch_size": (I, [I] * 7 + [ctypes.POINTER(SZ)]),
        "tadm_lora_project": (I, [P] * 5 + [I] * 4 + [I64] * 3 + [P] * 3 + [I] * 4 + [P, SZ, P]),
        "tadm_residual_norm": (I, [P] * 5 + [I] * 3 + [I64] * 4 + [P, P, I64, P, ctypes.c_float, ctypes.c_float] + [I] * 3 + [P]),
        "tadm_probe_breakdown": (I, [P, I, ctypes.POINTER(I64), ctypes.POINTER(ctypes.c_double),
                                     ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]),
        "tadm_probe_read": (I, [P, ctypes.POINTER(I64), ctypes.POINTER(ctypes.c_double),
                                ctypes.POINTER(ctypes.c_double)]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _check(status: int, handle=None):
    if status != TADM_OK:
        msg = load_library().tadm_last_error(handle).decode() if handle else ""
        raise TadmError(status, msg)


def make_config(model) -> tadm_config:
    """tadm_config from any object with the ModelConfig attributes."""
    return tadm_config(
        vocab=model.vocab, d_model=model.d_model, n_heads=model.n_heads, n_kv_heads=model.n_kv_heads,
        head_dim=model.head_dim, ffn=model.ffn, glu=1 if model.glu == "geglu" else 0, n_shared=model.n_shared,
        n_anchor=model.n_anchor, n_denoise=model.n_denoise, fusion={"gated_mlp": 0, "paired_attn": 1, "none": 2}[model.fusion],
        fusion_rank=model.fusion_rank, fusion_heads=model.fusion_heads, dtype=1 if model.dtype == "bf16" else 0,
        tied_lm_head=int(bool(model.tied_lm_head)), norm_eps=model.norm_eps, rope_theta=model.rope_theta,
        sliding_window=getattr(model, "sliding_window", 0), global_every=getattr(model, "global_every", 0),
        qk_norm=int(bool(getattr(model, "qk_norm", False))),
        sandwich_norm=int(bool(getattr(model, "sandwich_norm", False))),
        rope_theta_global=getattr(model, "rope_theta_global", 0.0),
        qkv_split=int(bool(getattr(model, "qkv_split", False))))


# ---------------------------------------------------------------------------- C-named wrappers
def tadm_weight_inventory(cfg: tadm_config):
    lib = load_library()
    n = lib.tadm_weight_count(ctypes.byref(cfg))
    if n < 0:
        raise TadmError(1, "invalid config")
    out = []
    buf = ctypes.create_string_buffer(128)
    r, c = ctypes.c_int64(), ctypes.c_int64()
    for i in range(n):
        _check(lib.tadm_weight_info(ctypes.byref(cfg), i, buf, 128, ctypes.byref(r), ctypes.byref(c)))
        out.append((buf.value.decode(), (r.value,) if c.value == 1 else (r.value, c.value)))
    return out


def tadm_plan(prompt_len: int, gen_len: int, steps_per_block: int, K: int, block_len: int):
    lib = load_library()
    n = ctypes.c_int()
    _check(lib.tadm_plan(prompt_len, gen_len, steps_per_block, K, block_len, None, 0, ctypes.byref(n)))
    ev = (tadm_plan_event * n.value)()
    _check(lib.tadm_plan(prompt_len, gen_len, steps_per_block, K, block_len, ev, n.value, ctypes.byref(n)))
    return [(e.kind, e.block, e.n, e.k) for e in ev]


def tadm_layer_cost(L_S: int, L_A: int, L_D: int, T: int, K: int):
    full, cache = ctypes.c_int64(), ctypes.c_int64()
    _check(load_library().tadm_layer_cost(L_S, L_A, L_D, T, K, ctypes.byref(full), ctypes.byref(cache)))
    return full.value, cache.value


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_raw_stream = None


def _stream(stream=None) -> Optional[int]:
    """The handle of `stream`, or of the current stream of the current device (0.2 us by torch's private lookups, where it
    has them; a torch.cuda.Stream object costs 3 us per call)."""
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        import torch
        torch.cuda.init()
        get, dev = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        _raw_stream = (lambda: get(dev())) if get and dev else lambda: torch.cuda.current_stream().cuda_stream
    return _raw_stream()


_current_device = None


def _device() -> int:
    """The current device, on which a call launches."""
    global _current_device
    if _current_device is None:
        import torch
        torch.cuda.init()
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _current_device()


def tadm_gemm(A, B, C, dtype: int, stream=None):
    M, K = A.shape
    N = B.shape[0]
    c_dtype = 1 if str(C.dtype) == "torch.bfloat16" else 0
    _check(load_library().tadm_gemm(_ptr(A), _ptr(B), _ptr(C), M, N, K, A.stride(0), B.stride(0), C.stride(0),
                                    dtype, c_dtype, _stream(stream)))


def tadm_confidence(logits, mask_id: int, conf, tok, stream=None):
    rows, vocab = logits.shape
    _check(load_library().tadm_confidence(_ptr(logits), rows, vocab, mask_id, _ptr(conf), _ptr(tok), _stream(stream)))


def tadm_topk_unmask(z, conf, tok, k: int, mask_id: int, selected=None, stream=None):
    batch, rows = conf.shape
    _check(load_library().tadm_topk_unmask(_ptr(z), z.stride(0), _ptr(conf), _ptr(tok), batch, rows, k, mask_id,
                                           _ptr(selected), _stream(stream)))


def tadm_head_scratch_size(rows: int, vocab: int, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().tadm_head_scratch_size(rows, vocab, dtype, ctypes.byref(n)))
    return n.value


def tadm_head_confidence(x, w, mask_id: int, conf, tok, scratch, dtype: int, stream=None):
    rows, d = x.shape
    vocab = w.shape[0]
    _check(load_library().tadm_head_confidence(_ptr(x), _ptr(w), rows, d, vocab, mask_id, dtype, _ptr(scratch),
                                               scratch.numel() * scratch.element_size(), _ptr(conf), _ptr(tok),
                                               _stream(stream)))


def tadm_head_confidence_static(x, w, mask_id: int, conf, tok, dtype: int, stream=None):
    """The same result as tadm_head_confidence, with the partials in the
    library's fixed device array instead of caller scratch (no allocation)."""
    rows, d = x.shape
    vocab = w.shape[0]
    _check(load_library().tadm_head_confidence_static(_ptr(x), _ptr(w), rows, d, vocab, mask_id, dtype, _ptr(conf),
                                                      _ptr(tok), _stream(stream)))


def tadm_attention(q, k, v, o, n_heads: int, n_kv_heads: int, rows: int, ctx: int, causal: bool, dtype: int,
                   stream=None, window: int = 0):
    batch, _, _, hd = q.shape
    kv_stride = k.shape[2]
    _check(load_library().tadm_attention(_ptr(q), _ptr(k), _ptr(v), _ptr(o), batch, n_heads, n_kv_heads, hd, rows,
                                         ctx, kv_stride, int(causal), window, dtype, _stream(stream)))


REMDM_KINDS = {"cap": 0, "loop": 1}


def tadm_remdm_schedule(kind: str, T: int, n: int, eta: float, t_on: float = 0.55, t_off: float = 0.05,
                        alpha_on: float = 0.9):
    """(alpha_t, alpha_s, sigma_t, p_unmask) of reverse step n (host only)."""
    out = (ctypes.c_double * 4)()
    _check(load_library().tadm_remdm_schedule(REMDM_KINDS[kind], T, n, eta, t_on, t_off, alpha_on, out))
    return tuple(out)


def tadm_remdm_uniforms(seed: int, step: int, batch: int, rows: int, out, stream=None):
    """The sampler's draws of a step into out (device float [batch, rows, 3])."""
    _check(load_library().tadm_remdm_uniforms(seed, step, batch, rows, _ptr(out), _stream(stream)))


def tadm_remdm_update(z, logits, first_gen: int, mask_id: int, sigma: float, p_unmask: float, top_p: float,
                      seed: int, step: int, action, stream=None):
    """One ReMDM reverse step on z [batch, rows] from logits [batch * rows, vocab]."""
    batch, rows = z.shape
    vocab = logits.shape[1]
    _check(load_library().tadm_remdm_update(_ptr(z), rows, _ptr(logits), vocab, batch, rows, first_gen, vocab,
                                            mask_id, sigma, p_unmask, top_p, seed, step, _ptr(action),
                                            _stream(stream)))



def tadm_eb_update(z, logits, first_gen: int, mask_id: int, tau: float, eta: float, last: bool, seed: int,
                   step: int, entropy, probs=None, z_sum=None, stream=None):
    """One entropy-bound step (Alg. 2) on z [batch, rows] from the logits of
    the generated positions [batch * (rows - first_gen), vocab]; entropy
    [batch * (rows - first_gen)] fp32; probs (optional, fp32 or bf16) gets
    q = exp((l - max) / tau) and z_sum (optional, fp32) Z = sum q."""
    batch, rows = z.shape
    vocab = logits.shape[1]
    p_dtype = 0
    if probs is not None:
        p_dtype = {"torch.float32": 0, "torch.bfloat16": 1}[str(probs.dtype)]
    _check(load_library().tadm_eb_update(_ptr(z), rows, _ptr(logits), vocab, batch, rows, first_gen, vocab, mask_id,
                                         tau, eta, int(bool(last)), seed, step, _ptr(entropy),
                                         _ptr(probs) if probs is not None else None, p_dtype,
                                         probs.shape[1] if probs is not None else 0, _ptr(z_sum), _stream(stream)))


# ------------------------------------------------ sequences of different lengths
PAGE_TOKENS = 64


class PagePool:
    """The 8-bit KV cache's pages: e4m3 bytes k [layers, pages, kv heads, 64, hd]
    and v [layers, pages, kv heads, hd, 64], fp32 scales [layers, pages, kv
    heads].  Holds references to the tensors that it is made of."""

    def __init__(self, k, v, k_scale, v_scale):
        layers, pages, n_kv, tokens, hd = k.shape
        if tokens != PAGE_TOKENS or tuple(v.shape) != (layers, pages, n_kv, hd, tokens):
            raise TadmError(1, f"pages have shapes {tuple(k.shape)} and {tuple(v.shape)}")
        for s in (k_scale, v_scale):
            if tuple(s.shape) != (layers, pages, n_kv) or str(s.dtype) != "torch.float32":
                raise TadmError(1, f"scales must be fp32 {(layers, pages, n_kv)}")
        for t in (k, v, k_scale, v_scale):
            if not t.is_contiguous() or not t.is_cuda or t.device != k.device:
                raise TadmError(1, "a pool's tensors must be contiguous CUDA tensors of one device")
        if k.element_size() != 1 or v.element_size() != 1:
            raise TadmError(1, "pages hold one byte per element")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.layers, self.pages, self.n_kv_heads, self.head_dim = layers, pages, n_kv, hd
        self.c = tadm_page_pool(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), layers, pages,
                                n_kv, hd)
        self.ref = ctypes.addressof(self.c)
        self.index = k.get_device()

    @classmethod
    def empty(cls, layers: int, pages: int, n_kv_heads: int, head_dim: int, device="cuda"):
        """Pages that hold zeros, with the least scale that tadm_page_write gives."""
        import torch
        z = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)  # noqa: E731
        s = lambda: torch.full((layers, pages, n_kv_heads), 2.0 ** -60, dtype=torch.float32, device=device)  # noqa: E731
        return cls(z(layers, pages, n_kv_heads, PAGE_TOKENS, head_dim), z(layers, pages, n_kv_heads, head_dim, PAGE_TOKENS),
                   s(), s())


_DTYPES = {}


def _torch_types():
    import torch
    _DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.int32: "int32"})
    return _DTYPES


def _rows_of(device, *tensors):
    """The dtype code of row operands [rows, heads, hd] (fp32 or bf16, each row's heads dense, on the device), and for each the
    elements from one row to the next.  The strides of a single row or head do not matter."""
    kind = tensors[0].dtype
    dtype = (_DTYPES or _torch_types()).get(kind)
    if dtype not in (0, 1):
        raise TadmError(1, f"rows must be fp32 or bf16, not {kind}")
    ld = []
    for t in tensors:
        s, n = t.stride(), t.shape
        if len(s) != 3 or s[2] != 1 or (s[1] != n[2] and n[1] != 1) or t.dtype is not kind or t.get_device() != device:
            raise TadmError(1, "rows must be tensors [rows, heads, head_dim] of one type with dense heads on the current device")
        ld.append(s[0] if n[0] != 1 else n[1] * n[2])
    return dtype, ld


def _ints_of(device, *tensors):
    types = _DTYPES or _torch_types()
    for t in tensors:
        if types.get(t.dtype) != "int32" or not t.is_contiguous() or t.get_device() != device:
            raise TadmError(1, "lengths, tables and lists must be contiguous int32 tensors on the current device")


def _pool_of(device, pool):
    if pool.index != device:
        raise TadmError(1, "the page pool is not on the current device")
    return pool.ref


def _scratch_of(device, t):
    """Address and size of scratch memory; none at all is no address."""
    if t is None:
        return None, 0
    if not t.is_contiguous() or t.get_device() != device:
        raise TadmError(1, "scratch must be a contiguous tensor on the current device")
    return t.data_ptr(), t.nbytes


def tadm_ragged_sync_status(stream=None):
    """Waits for the stream; an error if an attention call below gave up a bounded wait since the last such error."""
    _check(load_library().tadm_ragged_sync_status(_stream(stream)))


def tadm_attention_packed(q, k, v, o, cu_rows, max_rows: int, causal: bool = True, window: int = 0, stream=None):
    """Attention of whole prompts packed one after the other: q, o [rows,
    heads, hd], k, v [rows, kv heads, hd] (fp32 or bf16, rows may be strided),
    cu_rows int32 [batch + 1]."""
    device = _device()
    dtype, ld = _rows_of(device, q, k, v, o)
    _ints_of(device, cu_rows)
    shape, kv = q.shape, k.shape
    rows, heads, hd = shape
    if o.shape != shape or kv != v.shape or kv[0] != rows or kv[2] != hd:
        raise TadmError(1, "shapes of q, k, v and o do not agree")
    status = load_library().tadm_attention_packed(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), cu_rows.data_ptr(), cu_rows.shape[0] - 1, rows,
        max_rows, heads, kv[1], hd, *ld, 1 if causal else 0, window,
        dtype, _stream(stream))
    if status:
        _check(status)


def _page_rows(call, pool, layer, k, v, cu_rows, start, table, max_rows, stream):
    device = _device()
    dtype, ld = _rows_of(device, k, v)
    _ints_of(device, cu_rows, start, table)
    shape = k.shape
    rows, heads, hd = shape
    if shape != v.shape or heads != pool.n_kv_heads or hd != pool.head_dim:
        raise TadmError(1, "rows do not have the pool's heads")
    batch = cu_rows.shape[0] - 1
    seqs, width = table.shape
    if start.shape[0] != batch or seqs < batch:
        raise TadmError(1, "start and table need an entry per sequence")
    status = call(_pool_of(device, pool), layer, k.data_ptr(), v.data_ptr(), cu_rows.data_ptr(), start.data_ptr(), batch, rows, max_rows,
                  *ld, table.data_ptr(), width, dtype, _stream(stream))
    if status:
        _check(status)


def tadm_page_write(pool, layer: int, k, v, cu_rows, start, table, max_rows: int, stream=None):
    """Rows k, v [rows, kv heads, hd] become tokens start[b] .. of the cache (e4m3, a power-of-two scale per page and head)."""
    _page_rows(load_library().tadm_page_write, pool, layer, k, v, cu_rows, start, table, max_rows, stream)


def tadm_page_read(pool, layer: int, k, v, cu_rows, start, table, max_rows: int, stream=None):
    """Tokens start[b] .. of the cache into the rows k, v [rows, kv heads, hd]."""
    _page_rows(load_library().tadm_page_read, pool, layer, k, v, cu_rows, start, table, max_rows, stream)


def tadm_page_attention_scratch_size(batch: int, total_rows: int, max_rows: int, max_len: int, n_heads: int,
                                     n_kv_heads: int, head_dim: int, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().tadm_page_attention_scratch_size(batch, total_rows, max_rows, max_len, n_heads, n_kv_heads,
                                                           head_dim, dtype, ctypes.byref(n)))
    return n.value


def tadm_page_attention(q, pool, layer: int, o, cu_rows, lens, table, max_rows: int, max_len: int, scratch,
                        causal: bool = False, window: int = 0, stream=None):
    """Attention of packed rows q, o [rows, heads, hd] over the cache: sequence b
    sees its first lens[b] tokens, its rows are the last ones of them."""
    device = _device()
    dtype, ld = _rows_of(device, q, o)
    _ints_of(device, cu_rows, lens, table)
    shape = q.shape
    rows, heads, hd = shape
    batch = cu_rows.shape[0] - 1
    seqs, width = table.shape
    if o.shape != shape or hd != pool.head_dim or lens.shape[0] != batch or seqs < batch:
        raise TadmError(1, "shapes of q, o, lens, table and the pool do not agree")
    status = load_library().tadm_page_attention(
        q.data_ptr(), _pool_of(device, pool), layer, o.data_ptr(), cu_rows.data_ptr(), lens.data_ptr(), batch, rows, max_rows,
        max_len, heads, *ld, table.data_ptr(), width, 1 if causal else 0, window, dtype,
        *_scratch_of(device, scratch), _stream(stream))
    if status:
        _check(status)


def tadm_pages_scratch_size(pages: int, n_seqs: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().tadm_pages_scratch_size(pages, n_seqs, ctypes.byref(n)))
    return n.value


def _seqs_of(tables, tables_out, per_seq, refs, refs_out, lists, status):
    device = _device()
    _ints_of(device, tables, tables_out, refs, refs_out, status, *per_seq, *lists)
    if tables_out.shape != tables.shape or refs_out.shape != refs.shape or any(
            t.shape[0] != tables.shape[0] for t in per_seq) or any(t.shape != lists[0].shape for t in lists):
        raise TadmError(1, "shapes of tables, lens, refs and lists do not agree")
    if status.numel() < 1:
        raise TadmError(1, "the outcome needs an element")
    return device


def tadm_pages_reserve(tables, refs, seqs, new_len, tables_out, refs_out, status, scratch, stream=None):
    """The pages that sequences seqs lack for new_len tokens, lowest free ids first."""
    device = _seqs_of(tables, tables_out, (), refs, refs_out, (seqs, new_len), status)
    _check(load_library().tadm_pages_reserve(
        tables.data_ptr(), refs.data_ptr(), refs.shape[0], tables.shape[0], tables.shape[1], seqs.data_ptr(),
        new_len.data_ptr(), seqs.shape[0], tables_out.data_ptr(), refs_out.data_ptr(), status.data_ptr(),
        *_scratch_of(device, scratch), _stream(stream)))


def tadm_pages_fork(pool, tables, lens, refs, src, dst, tables_out, lens_out, refs_out, status, scratch, stream=None):
    """Sequences dst become copies of src: full pages shared, the last page copied."""
    device = _seqs_of(tables, tables_out, (lens, lens_out), refs, refs_out, (src, dst), status)
    if refs.shape[0] != pool.pages:
        raise TadmError(1, "refs needs an entry per page")
    _check(load_library().tadm_pages_fork(
        _pool_of(device, pool), tables.data_ptr(), lens.data_ptr(), refs.data_ptr(), tables.shape[0], tables.shape[1],
        src.data_ptr(), dst.data_ptr(), src.shape[0], tables_out.data_ptr(), lens_out.data_ptr(), refs_out.data_ptr(),
        status.data_ptr(), *_scratch_of(device, scratch), _stream(stream)))


def tadm_pages_free(tables, lens, refs, seqs, tables_out, lens_out, refs_out, status, scratch, stream=None):
    """Sequences seqs give their pages back."""
    device = _seqs_of(tables, tables_out, (lens, lens_out), refs, refs_out, (seqs,), status)
    _check(load_library().tadm_pages_free(
        tables.data_ptr(), lens.data_ptr(), refs.data_ptr(), refs.shape[0], tables.shape[0], tables.shape[1],
        seqs.data_ptr(), seqs.shape[0], tables_out.data_ptr(), lens_out.data_ptr(), refs_out.data_ptr(),
        status.data_ptr(), *_scratch_of(device, scratch), _stream(stream)))


def tadm_pages_compact(pool, tables, refs, tables_out, refs_out, n_live, scratch, stream=None):
    """Pages in use move to the lowest ids; n_live int32 [1] gets their number."""
    device = _seqs_of(tables, tables_out, (), refs, refs_out, (), n_live)
    if refs.shape[0] != pool.pages:
        raise TadmError(1, "refs needs an entry per page")
    _check(load_library().tadm_pages_compact(
        _pool_of(device, pool), tables.data_ptr(), refs.data_ptr(), tables.shape[0], tables.shape[1], tables_out.data_ptr(),
        refs_out.data_ptr(), n_live.data_ptr(), *_scratch_of(device, scratch), _stream(stream)))


def tadm_pages_copy(pool, src, dst, stream=None):
    """Page src[i] onto page dst[i] in every layer."""
    device = _device()
    _ints_of(device, src, dst)
    if src.shape != dst.shape:
        raise TadmError(1, "src and dst differ in length")
    _check(load_library().tadm_pages_copy(_pool_of(device, pool), src.data_ptr(), dst.data_ptr(), src.shape[0], _stream(stream)))


# ------------------------------------------------ requests with settings of their own
def _matrix_of(device, t, what, shape=None):
    """The dtype code (fp32 or bf16) of a matrix with dense rows on the device (of `shape`), and the elements from one row to
    the next."""
    code, s, n = (_DTYPES or _torch_types()).get(t.dtype), t.stride(), t.shape
    if code not in (0, 1) or len(s) != 2 or (s[1] != 1 and n[1] != 1) or t.get_device() != device or (shape is not None and n != shape):
        raise TadmError(1, f"{what} must be an fp32 or bf16 matrix with dense rows on the current device" +
                        ("" if shape is None else f", {tuple(shape)}"))
    return code, s[0] if n[0] != 1 else n[1]


def _vector_of(device, t, shape, kind, what):
    """Address of a dense vector (None: none); kind: its dtype code."""
    if t is None:
        return None
    if (_DTYPES or _torch_types()).get(t.dtype) != kind or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise TadmError(1, f"{what} must be a dense vector of {shape[0]} {('fp32', 'bf16').__getitem__(kind) if kind in (0, 1) else kind} "
                        "values on the current device")
    return t.data_ptr()


def tadm_sample_scratch_size(rows: int, vocab: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().tadm_sample_scratch_size(rows, vocab, ctypes.byref(n)))
    return n.value


_sample_scratch = {}


def _scratch_on(device, stream, nbytes: int):
    """Scratch memory for work on `stream` (None: the current one), from torch's allocator."""
    import torch
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def tadm_sample(logits, u, tok, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, mask_id: int = -1,
                scratch=None, stream=None):
    """One token per row of logits [rows, vocab] (fp32 or bf16, rows may be strided) into tok (int32 [rows]), drawn with the
    row's temperature, top_k (int32), top_p and min_p (fp32 [rows] each, None: off) from its random number u (fp32
    [rows], 0 <= u < 1); prob (fp32 [rows]) gets the token's probability among the ids kept.  scratch: a device buffer of
    at least tadm_sample_scratch_size(rows, vocab) bytes; None: torch's allocator gives it for the call."""
    device = _device()
    dtype, ld = _matrix_of(device, logits, "logits")
    shape = logits.shape
    rows, vocab = shape
    one = shape[:1]
    args = (_vector_of(device, temperature, one, 0, "temperature"), _vector_of(device, top_k, one, "int32", "top_k"),
            _vector_of(device, top_p, one, 0, "top_p"), _vector_of(device, min_p, one, 0, "min_p"),
            _vector_of(device, u, one, 0, "u"), _vector_of(device, tok, one, "int32", "tok"), _vector_of(device, prob, one, 0, "prob"))
    if scratch is None:
        need = _sample_scratch.get(shape)
        if need is None:
            if len(_sample_scratch) > 4096:
                _sample_scratch.clear()
            need = _sample_scratch[shape] = tadm_sample_scratch_size(rows, vocab)
        if need:
            scratch = _scratch_on(device, stream, need)
    status = load_library().tadm_sample(logits.data_ptr(), ld, rows, vocab, mask_id, *args, dtype, *_scratch_of(device, scratch),
                                        _stream(stream))
    if status:
        _check(status)


def tadm_lora_scratch_size(batch: int, total_rows: int, n_in: int, n_out: int, n_adapters: int, rank: int, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().tadm_lora_scratch_size(batch, total_rows, n_in, n_out, n_adapters, rank, dtype, ctypes.byref(n)))
    return n.value


def tadm_lora_project(x, w, y, cu_rows, adapter, lora_a, lora_b, lora_scale, scratch, stream=None):
    """y [rows, n_out] = x [rows, n_in] W^T (W [n_out, n_in]) plus, for the rows of sequence b, lora_scale[a] B_a (A_a x)
    with a = adapter[b] (int32 [batch]; -1: none); lora_a [adapters, rank, n_in], lora_b [adapters, n_out, rank]."""
    device = _device()
    dtype, ldx = _matrix_of(device, x, "x")
    w_dtype, ldw = _matrix_of(device, w, "w")
    (rows, n_in), (n_out, k) = x.shape, w.shape
    y_dtype, ldy = _matrix_of(device, y, "y", (rows, n_out))
    _ints_of(device, cu_rows, adapter)
    (n, rank, a_in), batch = lora_a.shape, cu_rows.shape[0] - 1
    if k != n_in or a_in != n_in or lora_b.shape != (n, n_out, rank) or adapter.shape[0] != batch:
        raise TadmError(1, "shapes of x, w, y, the adapters and the sequences do not agree")
    for t in (lora_a, lora_b):
        if t.dtype is not x.dtype or not t.is_contiguous() or t.get_device() != device:
            raise TadmError(1, "adapters must be contiguous, of x's type, on the current device")
    if w_dtype != dtype:
        raise TadmError(1, "w must have x's type")
    status = load_library().tadm_lora_project(
        x.data_ptr(), w.data_ptr(), y.data_ptr(), cu_rows.data_ptr(), adapter.data_ptr(), batch, rows, n_in, n_out, ldx, ldw,
        ldy, lora_a.data_ptr(), lora_b.data_ptr(), _vector_of(device, lora_scale, (n,), 0, "lora_scale"), n, rank, dtype, y_dtype,
        *_scratch_of(device, scratch), _stream(stream))
    if status:
        _check(status)


def tadm_residual_norm(x, y, x_out, n_out=None, cu_rows=None, post_gain=None, gate=None, pre_gain=None,
                       residual_scale: float = 1.0, eps: float = 1e-6, stream=None):
    """x_out = residual_scale x + gate[b] u with u = y or, with post_gain, its RMS norm times the gain, and n_out = the RMS
    norm of x_out times pre_gain, for rows [rows, d]; gate [batch, d] has a row per sequence of cu_rows (int32 [batch + 1])."""
    device = _device()
    shape = x.shape
    x_dtype, ldx = _matrix_of(device, x, "x")
    xo_dtype, ldxo = _matrix_of(device, x_out, "x_out", shape) if x_out is not x else (x_dtype, ldx)
    y_dtype, ldy = _matrix_of(device, y, "y", shape)
    rows, d = shape
    if xo_dtype != x_dtype:
        raise TadmError(1, "x and x_out must have one type")
    batch, cu = 1, None
    if cu_rows is not None:
        _ints_of(device, cu_rows)
        batch, cu = cu_rows.shape[0] - 1, cu_rows.data_ptr()
    dtype, ldn, ldg, n_ptr, g_ptr = None, d, d, None, None
    if n_out is not None:
        dtype, ldn = _matrix_of(device, n_out, "n_out", shape)
        n_ptr = n_out.data_ptr()
    if gate is not None:
        g_dtype, ldg = _matrix_of(device, gate, "gate", (batch, d))
        if dtype is None:
            dtype = g_dtype
        if dtype != g_dtype:
            raise TadmError(1, "gate must have n_out's type")
        g_ptr = gate.data_ptr()
    if dtype is None:
        first = post_gain if post_gain is not None else pre_gain
        dtype = (_DTYPES or _torch_types()).get(first.dtype) if first is not None else 0
        if dtype not in (0, 1):
            raise TadmError(1, "gains must be fp32 or bf16")
    one = shape[1:]
    status = load_library().tadm_residual_norm(
        x.data_ptr(), y.data_ptr(), x_out.data_ptr(), n_ptr, cu, batch, rows, d, ldx, ldy, ldxo, ldn,
        _vector_of(device, post_gain, one, dtype, "post_gain"), g_ptr, ldg, _vector_of(device, pre_gain, one, dtype, "pre_gain"),
        residual_scale, eps, x_dtype, y_dtype, dtype, _stream(stream))
    if status:
        _check(status)


# ---------------------------------------------------------------------------- model handle
class TadmModel:
    """A handle plus its torch-allocated workspace.

    ``weights`` maps inventory names to device tensors (fp32 or bf16,
    contiguous).  The handle keeps references so the memory outlives it.
    """

    def __init__(self, model, weights: Dict[str, "object"], max_batch: int, max_rows: int, max_ctx: int = 0):
        import torch
        lib = load_library()
        self.lib = lib
        self.model = model
        self.cfg = make_config(model)
        inv = tadm_weight_inventory(self.cfg)
        self.weights = []
        for name, shape in inv:
            t = weights[name]
            if tuple(t.shape) != tuple(shape) and not (len(shape) == 1 and t.numel() == shape[0]):
                raise TadmError(1, f"weight {name} has shape {tuple(t.shape)}, expected {shape}")
            if not t.is_contiguous() or not t.is_cuda:
                raise TadmError(1, f"weight {name} must be a contiguous CUDA tensor")
            self.weights.append(t)
        arr = (ctypes.c_void_p * len(self.weights))(*[t.data_ptr() for t in self.weights])
        h = ctypes.c_void_p()
        _check(lib.tadm_create(ctypes.byref(self.cfg), arr, len(self.weights), max_batch, max_rows, max_ctx,
                               ctypes.byref(h)))
        self.h = h
        n = ctypes.c_size_t()
        _check(lib.tadm_workspace_size(h, ctypes.byref(n)), h)
        self.workspace = torch.empty(max(n.value, 256), dtype=torch.uint8, device="cuda")
        _check(lib.tadm_bind_workspace(h, self.workspace.data_ptr(), n.value), h)
        self.max_batch, self.max_rows, self.max_ctx = max_batch, max_rows, max_ctx

    def close(self):
        if getattr(self, "h", None):
            self.lib.tadm_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- C-named calls ----------------------------------------------------
    def tadm_cache_size(self, batch: int, rows: int) -> int:
        n = ctypes.c_size_t()
        _check(self.lib.tadm_cache_size(self.h, batch, rows, ctypes.byref(n)), self.h)
        return n.value

    def new_cache(self, batch: int, rows: int):
        import torch
        return torch.empty(self.tadm_cache_size(batch, rows), dtype=torch.uint8, device="cuda")

    def tadm_reset(self, batch: int):
        _check(self.lib.tadm_reset(self.h, batch), self.h)

    def tadm_prefill(self, prompt, stream=None):
        B, P = prompt.shape
        _check(self.lib.tadm_prefill(self.h, _ptr(prompt), B, P, _stream(stream)), self.h)

    def tadm_anchor_forward(self, x_t, t: int, h_cache, stream=None):
        B, R = x_t.shape
        _check(self.lib.tadm_anchor_forward(self.h, _ptr(x_t), B, R, t, _ptr(h_cache), _stream(stream)), self.h)

    def tadm_denoise_step(self, x_t, t: int, T: int, n_masked_at_start: int, h_cache, logits=None, conf=None,
                          tok=None, selected=None, fused=None, stream=None):
        B, R = x_t.shape
        out = tadm_step_outputs(_ptr(logits), _ptr(conf), _ptr(tok), _ptr(selected), _ptr(fused))
        _check(self.lib.tadm_denoise_step(self.h, _ptr(x_t), B, R, t, T, n_masked_at_start, _ptr(h_cache),
                                          ctypes.byref(out), _stream(stream)), self.h)

    def tadm_commit_block(self, x_block, stream=None):
        B, R = x_block.shape
        _check(self.lib.tadm_commit_block(self.h, _ptr(x_block), B, R, _stream(stream)), self.h)

    def tadm_generate(self, prompt, out, gen_len: int, steps_per_block: int, K: int, block_len: int = 0,
                      stream=None):
        B, P = prompt.shape
        _check(self.lib.tadm_generate(self.h, _ptr(prompt), B, P, _ptr(out), gen_len, steps_per_block, K,
                                      block_len, _stream(stream)), self.h)

    def tadm_generate_remdm(self, prompt, out, gen_len: int, steps: int, K: int, kind: str, eta: float,
                            top_p: float, seed: int, logits_scratch, stream=None):
        B, P = prompt.shape
        _check(self.lib.tadm_generate_remdm(self.h, _ptr(prompt), B, P, _ptr(out), gen_len, steps, K,
                                            REMDM_KINDS[kind], eta, top_p, seed, _ptr(logits_scratch),
                                            logits_scratch.numel() * logits_scratch.element_size(),
                                            _stream(stream)), self.h)

    def tadm_eb_scratch_bytes(self, batch: int, gen_len: int, self_cond: bool = True) -> int:
        out = ctypes.c_size_t(0)
        _check(self.lib.tadm_eb_scratch_bytes(self.h, batch, gen_len, int(bool(self_cond)), ctypes.byref(out)), self.h)
        return out.value

    def tadm_generate_entropy_bound(self, prompt, out, gen_len: int, steps: int, K: int, eta: float,
                                    tau_max: float, tau_min: float, seed: int, scratch, self_cond: bool = True,
                                    stream=None):
        """Alg. 2 generation; scratch: a device buffer of at least
        tadm_eb_scratch_bytes(batch, gen_len, self_cond) bytes."""
        B, P = prompt.shape
        _check(self.lib.tadm_generate_entropy_bound(self.h, _ptr(prompt), B, P, _ptr(out), gen_len, steps, K, eta,
                                                    tau_max, tau_min, int(bool(self_cond)), seed, _ptr(scratch),
                                                    scratch.numel() * scratch.element_size(), _stream(stream)),
               self.h)

    def tadm_sync_status(self):
        _check(self.lib.tadm_sync_status(self.h), self.h)

    def tadm_probe_enable(self, max_launches: int):
        _check(self.lib.tadm_probe_enable(self.h, max_launches), self.h)

    EPI_NAMES = ["plain", "residual", "qkv_rope", "glu", "fusion_gate_hidden", "fusion_out", "output_head",
                 "pa_up", "pa_silu", "pa_add", "pa_gate", "attention", "norms", "attention_short_rows"]
    N_GEMM_KINDS = 11

    def tadm_probe_breakdown(self) -> dict:
        n = len(self.EPI_NAMES)
        L, ms, fl, by = (ctypes.c_int64 * n)(), (ctypes.c_double * n)(), (ctypes.c_double * n)(), (ctypes.c_double * n)()
        _check(self.lib.tadm_probe_breakdown(self.h, n, L, ms, fl, by), self.h)
        return {self.EPI_NAMES[k]: {"launches": L[k], "ms": ms[k], "flops": fl[k], "bytes": by[k],
                                    "tflops": fl[k] / (ms[k] / 1e3) / 1e12}
                for k in range(n) if L[k] > 0}

    def tadm_probe_read(self):
        n, ms, fl = ctypes.c_int64(), ctypes.c_double(), ctypes.c_double()
        _check(self.lib.tadm_probe_read(self.h, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(fl)), self.h)
        return n.value, ms.value, fl.value

    def tadm_get_counters(self) -> dict:
        c = tadm_counters()
        _check(self.lib.tadm_get_counters(self.h, ctypes.byref(c)), self.h)
        return {f: getattr(c, f) for f, _ in tadm_counters._fields_}

    # -- user-facing ------------------------------------------------------------
    def generate(self, prompt, gen_len: int, steps_per_block: int, K: int, block_len: int = 0, stream=None):
        """Whole generation.  ``prompt`` may live on the host or the device;
        host prompts are copied in and the result copied back (pinned)."""
        import torch
        host = not prompt.is_cuda
        p = prompt.to("cuda", non_blocking=True) if host else prompt
        out = torch.empty((p.shape[0], p.shape[1] + gen_len), dtype=torch.int32, device="cuda")
        self.tadm_generate(p, out, gen_len, steps_per_block, K, block_len, stream)
        if host:
            res = torch.empty(out.shape, dtype=torch.int32, pin_memory=True)
            res.copy_(out, non_blocking=True)
            self.tadm_sync_status()
            return res
        return out


def upload_weights(model, host_weights: Dict[str, "object"]):
    """Copy generated host weights (float32 or raw bf16 bits) to the device."""
    import numpy as np
    import torch
    out = {}
    for name, w in host_weights.items():
        if w.dtype == np.uint16:
            t = torch.from_numpy(w.view(np.int16)).view(torch.bfloat16)
        else:
            t = torch.from_numpy(np.ascontiguousarray(w, dtype=np.float32))
        out[name] = t.to("cuda").contiguous()
    return out
