"""Thin ctypes binding over libwar.so (the C ABI declared in include/war.h).

Argument marshalling only: every step of the verify path runs in the HIP
kernels behind the C ABI.  torch provides device memory and the stream; arrays
are passed as raw device pointers (``tensor.data_ptr()``).  Importing this
module fails loudly when the library has not been built -- there is no
fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import torch

from .synth import ModelConfig, weight_shapes

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwar.so")

WAR_OK = 0
_ERRORS = {-1: "WAR_ERR_INVALID_ARG", -2: "WAR_ERR_OUT_OF_PAGES", -3: "WAR_ERR_HIP",
           -4: "WAR_ERR_UNSUPPORTED", -5: "WAR_ERR_DEVICE"}

EXPORTS = ["war_weight_count", "war_model_create", "war_model_destroy", "war_kv_pool_create",
           "war_kv_pool_destroy", "war_kv_alloc", "war_kv_fork", "war_kv_free", "war_kv_load",
           "war_prefill_append", "war_verify_step", "war_verify_step_sampled", "war_verify_step_tree",
           "war_verify_step_noalloc",
           "war_kv_commit", "war_pool_state", "war_kv_pool_bytes", "war_kv_pool_create_format", "war_kv_write",
           "war_kv_read", "war_constrain_workspace", "war_constrain_logits", "war_counts_begin", "war_counts_add",
           "war_verify_step_constrained", "war_attend_create", "war_attend_destroy", "war_attend_update", "war_attend_run",
           "war_residual_norm", "war_quantize", "war_dequantize", "war_linear_create", "war_linear_destroy",
           "war_linear_run", "war_rope_write",
           "war_last_error", "war_debug_mfma16", "war_debug_workspace", "war_debug_sample",
           "war_debug_gemm", "war_debug_gemm_plan", "war_debug_pool_waits", "war_profile", "war_profile_read", "war_debug_linear",
           "war_debug_linear_shape"]


class WarError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_ERRORS.get(status, status)}: {msg}")
        self.status = status


class _Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn_dim", C.c_int32),
                ("vocab", C.c_int32), ("rms_eps", C.c_float), ("rope_base", C.c_float),
                ("page_size", C.c_int32), ("max_rows", C.c_int32)]


class _Constraints(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("counts", C.c_void_p), ("repetition", C.c_void_p), ("frequency", C.c_void_p),
                ("presence", C.c_void_p), ("n_bias", C.c_int32), ("bias_ids", C.c_void_p), ("bias_values", C.c_void_p),
                ("n_masks", C.c_int32), ("masks", C.c_void_p), ("mask_index", C.c_void_p)]


class _Mx(C.Structure):
    _fields_ = [("format", C.c_int32), ("rows", C.c_int32), ("cols", C.c_int32), ("codes", C.c_void_p),
                ("code_stride", C.c_int64), ("scales", C.c_void_p), ("scale_stride", C.c_int64)]


class _Rope(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("adjacent", C.c_int32), ("n_axes", C.c_int32), ("axes", C.c_void_p),
                ("freqs", C.c_void_p)]


def load_library(path: str = LIB_PATH) -> C.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2607_17299_amd.build`")
    lib = C.CDLL(path)
    vp, i32, pi32 = C.c_void_p, C.c_int32, C.POINTER(C.c_int32)
    sig = {
        "war_weight_count": (i32, [C.POINTER(_Config)]),
        "war_model_create": (i32, [C.POINTER(_Config), C.POINTER(vp), i32, C.POINTER(vp)]),
        "war_model_destroy": (None, [vp]),
        "war_kv_pool_create": (i32, [C.POINTER(_Config), vp, i32, vp, i32, i32, vp, C.POINTER(vp)]),
        "war_kv_pool_destroy": (None, [vp]),
        "war_kv_alloc": (i32, [vp, i32, pi32, pi32, vp]),
        "war_kv_fork": (i32, [vp, i32, i32, i32, vp]),
        "war_kv_free": (i32, [vp, i32, pi32, vp]),
        "war_kv_load": (i32, [vp, i32, i32, i32, i32, vp, vp]),
        "war_prefill_append": (i32, [vp, vp, i32, vp, vp, pi32, vp, vp, vp, vp]),
        "war_verify_step": (i32, [vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]),
        "war_verify_step_sampled": (i32, [vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, C.c_float, i32,
                                          vp, vp, vp, vp]),
        "war_verify_step_tree": (i32, [vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]),
        "war_verify_step_noalloc": (i32, [vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]),
        "war_kv_commit": (i32, [vp, i32, vp, vp, vp, vp]),
        "war_pool_state": (i32, [vp, pi32, pi32, pi32, pi32, pi32, vp]),
        "war_kv_pool_bytes": (C.c_int64, [C.POINTER(_Config), i32, i32]),
        "war_kv_pool_create_format": (i32, [C.POINTER(_Config), vp, i32, i32, vp, i32, i32, vp, C.POINTER(vp)]),
        "war_kv_write": (i32, [vp, i32, i32, vp, vp, i32, vp, vp, C.c_int64, vp, C.c_int64, vp]),
        "war_kv_read": (i32, [vp, i32, i32, vp, vp, i32, vp, vp, C.c_int64, vp, C.c_int64, vp]),
        "war_attend_create": (i32, [vp, i32, i32, C.POINTER(vp)]),
        "war_attend_destroy": (None, [vp]),
        "war_attend_update": (i32, [vp, i32, i32, vp, vp, vp, vp, vp]),
        "war_attend_run": (i32, [vp, i32, vp, C.c_int64, vp, C.c_int64, vp]),
        "war_residual_norm": (i32, [i32, i32, vp, C.c_int64, vp, C.c_int64, i32, vp, C.c_float, C.POINTER(_Mx), vp,
                                    C.c_int64, vp]),
        "war_quantize": (i32, [C.POINTER(_Mx), vp, C.c_int64, vp, C.c_int64, i32, vp]),
        "war_dequantize": (i32, [C.POINTER(_Mx), vp, C.c_int64, i32, vp]),
        "war_linear_create": (i32, [C.POINTER(_Mx), vp, vp, C.POINTER(vp)]),
        "war_linear_destroy": (None, [vp]),
        "war_linear_run": (i32, [vp, C.POINTER(_Mx), vp, C.c_int64, i32, vp]),
        "war_rope_write": (i32, [vp, i32, C.POINTER(_Rope), i32, vp, vp, i32, vp, vp, vp, C.c_int64, vp, C.c_int64, vp,
                                 C.c_int64, vp, C.c_int64, vp]),
        "war_constrain_workspace": (C.c_int64, [i32, i32]),
        "war_constrain_logits": (i32, [C.POINTER(_Constraints), i32, i32, vp, vp, vp, vp, vp, i32, vp, C.c_int64, vp,
                                       C.c_int64, vp, vp, vp]),
        "war_counts_begin": (i32, [vp, i32, i32, i32, vp, vp, i32, vp, vp]),
        "war_counts_add": (i32, [vp, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp]),
        "war_verify_step_constrained": (i32, [vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, C.POINTER(_Constraints), vp,
                                              C.c_float, i32, vp, vp, vp, vp, vp]),
        "war_last_error": (C.c_char_p, []),
        "war_debug_sample": (i32, [vp, i32, i32, i32, vp, vp, vp, C.c_float, i32, vp, vp, vp]),
        "war_debug_mfma16": (i32, [vp, vp, vp, vp]),
        "war_debug_workspace": (i32, [vp, C.c_char_p, C.POINTER(vp), C.POINTER(C.c_int64)]),
        "war_debug_gemm": (i32, [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp]),
        "war_debug_gemm_plan": (i32, [i32, i32, i32, i32, C.c_int64, pi32, pi32, pi32]),
        "war_debug_pool_waits": (i32, [vp, C.POINTER(C.c_int64)]),
        "war_debug_linear": (i32, [vp, C.POINTER(_Mx), vp, C.c_int64, i32, i32, vp]),
        "war_debug_linear_shape": (i32, [i32, i32, i32, i32, i32]),
        "war_profile": (i32, [vp, i32]),
        "war_profile_read": (i32, [vp, C.c_char_p, i32]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    return lib


_LIB: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    global _LIB
    if _LIB is None:
        _LIB = load_library()
    return _LIB


def _check(status: int) -> None:
    if status != WAR_OK:
        raise WarError(status, lib().war_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _host_i32(xs: Sequence[int]):
    arr = (C.c_int32 * len(xs))(*[int(x) for x in xs])
    return arr


def config_struct(cfg: ModelConfig, max_rows: int) -> _Config:
    return _Config(cfg.n_layers, cfg.d_model, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim,
                   cfg.ffn_dim, cfg.vocab, cfg.rms_eps, cfg.rope_base, cfg.page_size, max_rows)


class Model:
    """A decoder over bf16 device weights (canonical order).  The library copies
    (and repacks) them at creation; the tensors may be dropped afterwards."""

    def __init__(self, cfg: ModelConfig, weights: Dict[str, torch.Tensor], max_rows: int = 1024):
        self.cfg, self.max_rows = cfg, max_rows
        names = [n for n, _ in weight_shapes(cfg)]
        ws = [weights[n] for n in names]
        for t in ws:
            assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous()
        arr = (C.c_void_p * len(ws))(*[t.data_ptr() for t in ws])
        self._cfg = config_struct(cfg, max_rows)
        h = C.c_void_p()
        torch.cuda.synchronize()                    # the weights are complete before the copy
        _check(lib().war_model_create(C.byref(self._cfg), arr, len(ws), C.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().war_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


KV_FORMATS = {"bf16": 0, "e4m3": 1}


class Pool:
    """A paged KV pool: caller-owned KV storage and block tables (torch tensors).
    kv_format "e4m3" holds keys and values in 8 bits, with a power-of-two scale for
    each token and kv-head (war.h)."""

    def __init__(self, cfg: ModelConfig, num_pages: int, max_seqs: int, max_pages_per_seq: int,
                 device="cuda", stream=None, kv_format: str = "bf16"):
        self.cfg, self.kv_format = cfg, kv_format
        self.num_pages, self.max_seqs, self.max_pages = num_pages, max_seqs, max_pages_per_seq
        if kv_format not in KV_FORMATS:
            raise ValueError(f"kv_format must be one of {sorted(KV_FORMATS)}")
        n = cfg.n_layers * num_pages * cfg.n_kv_heads * 2 * cfg.page_size * cfg.head_dim
        self._cfg = config_struct(cfg, 1)
        if kv_format == "e4m3":
            n = max(lib().war_kv_pool_bytes(C.byref(self._cfg), num_pages, KV_FORMATS[kv_format]), 0)
        self.kv = torch.empty(n, dtype=torch.bfloat16 if kv_format == "bf16" else torch.uint8, device=device)
        self.block_tables = torch.empty((max_seqs, max_pages_per_seq), dtype=torch.int32, device=device)
        if stream is not None:  # memory that the current stream freed may be in use there still
            stream.wait_stream(torch.cuda.current_stream(self.kv.device))
        h = C.c_void_p()
        _check(lib().war_kv_pool_create_format(C.byref(self._cfg), _ptr(self.kv), num_pages, KV_FORMATS[kv_format],
                                               _ptr(self.block_tables), max_seqs, max_pages_per_seq,
                                               _stream(stream), C.byref(h)))
        self.handle = h

    # ---- layout helpers (views of the caller-owned storage)
    def kv_view(self) -> torch.Tensor:
        """The bf16 pages."""
        c = self.cfg
        assert self.kv_format == "bf16"
        return self.kv.view(c.n_layers, self.num_pages, c.n_kv_heads, 2, c.page_size, c.head_dim)

    def _key_order(self) -> torch.Tensor:
        """Element index, inside a page's K region, of key slot s and dim d
        ([P, D]): the fragment order of include/war.h (groups of eight slots
        by (s / 4) % 2, 32-dim k-steps, eight 64-byte rows per run)."""
        c = self.cfg
        s = torch.arange(c.page_size).view(-1, 1)
        d = torch.arange(c.head_dim).view(1, -1)
        t, s8 = (s // 4) % 2, (s // 8) * 4 + s % 4
        return ((t * (c.head_dim // 32) + d // 32) * 8 + s8) * 32 + d % 32

    def gather_kv(self, seq: int, n_tokens: int, layer: int) -> torch.Tensor:
        """[2, Hkv, n_tokens, D] keys/values of a sequence read back from its pages."""
        c = self.cfg
        if self.kv_format != "bf16":
            shape = (1, n_tokens, c.n_kv_heads, c.head_dim)
            k, v = (torch.empty(shape, dtype=torch.bfloat16, device=self.kv.device) for _ in range(2))
            ids = torch.tensor([seq, 0], dtype=torch.int32, device=self.kv.device)
            kv_read(self, layer, ids[:1], ids[1:], k, v)
            return torch.stack([k[0].transpose(0, 1), v[0].transpose(0, 1)])
        pages = self.block_tables[seq, : -(-n_tokens // c.page_size)].long()
        v = self.kv_view()[layer, pages]                       # [np, H, 2, P, D]
        kraw = v[:, :, 0].reshape(len(pages), c.n_kv_heads, c.page_size * c.head_dim)
        korder = self._key_order().to(kraw.device).reshape(-1)
        k = kraw[:, :, korder].reshape(len(pages), c.n_kv_heads, c.page_size, c.head_dim)
        k = k.permute(1, 0, 2, 3).reshape(c.n_kv_heads, -1, c.head_dim)
        vt = v[:, :, 1].reshape(len(pages), c.n_kv_heads, c.head_dim, c.page_size)
        vv = vt.permute(1, 0, 3, 2).reshape(c.n_kv_heads, -1, c.head_dim)
        return torch.stack([k[:, :n_tokens], vv[:, :n_tokens]])

    # ---- operations
    def alloc(self, seq_ids: Sequence[int], n_tokens: Sequence[int], stream=None):
        _check(lib().war_kv_alloc(self.handle, len(seq_ids), _host_i32(seq_ids), _host_i32(n_tokens),
                                  _stream(stream)))

    def fork(self, src: int, dst: int, n_tokens: int, stream=None):
        _check(lib().war_kv_fork(self.handle, src, dst, n_tokens, _stream(stream)))

    def free(self, seq_ids: Sequence[int], stream=None):
        _check(lib().war_kv_free(self.handle, len(seq_ids), _host_i32(seq_ids), _stream(stream)))

    def load(self, seq: int, layer: int, pos0: int, kv: torch.Tensor, stream=None):
        assert kv.dtype == torch.bfloat16 and kv.is_contiguous() and kv.dim() == 4
        _check(lib().war_kv_load(self.handle, seq, layer, pos0, kv.shape[2], _ptr(kv), _stream(stream)))

    def state(self, stream=None) -> Dict:
        fc = C.c_int32()
        stack = (C.c_int32 * self.num_pages)()
        ref = (C.c_int32 * self.num_pages)()
        held = (C.c_int32 * self.max_seqs)()
        base = (C.c_int32 * self.max_seqs)()
        st = lib().war_pool_state(self.handle, C.byref(fc), stack, ref, held, base, _stream(stream))
        import numpy as np
        out = {"stack": np.array(stack[: fc.value], dtype=np.int32), "refcount": np.array(ref[:], np.int32),
               "held": np.array(held[:], np.int32), "base": np.array(base[:], np.int32),
               "table": self.block_tables.cpu().numpy(), "status": st}
        return out

    def waits(self) -> int:
        """Verify steps that waited to read the exact free page count."""
        n = C.c_int64()
        _check(lib().war_debug_pool_waits(self.handle, C.byref(n)))
        return n.value

    def close(self):
        if getattr(self, "handle", None):
            lib().war_kv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def verify_step(model: Model, pool: Pool, seq_ids: torch.Tensor, ctx_lens: torch.Tensor,
                last_tokens: torch.Tensor, draft_tokens: Optional[torch.Tensor],
                draft_lens: Optional[torch.Tensor], k_max: int, accept_lens: torch.Tensor,
                next_tokens: torch.Tensor, logits: Optional[torch.Tensor] = None, stream=None) -> None:
    B = seq_ids.numel()
    _check(lib().war_verify_step(model.handle, pool.handle, B, _ptr(seq_ids), _ptr(ctx_lens),
                                 _ptr(last_tokens), _ptr(draft_tokens), _ptr(draft_lens), k_max,
                                 _ptr(accept_lens), _ptr(next_tokens), _ptr(logits), _stream(stream)))


def verify_step_noalloc(model: Model, pool: Pool, seq_ids: torch.Tensor, ctx_lens: torch.Tensor,
                        last_tokens: torch.Tensor, draft_tokens: Optional[torch.Tensor],
                        draft_lens: Optional[torch.Tensor], k_max: int, accept_lens: torch.Tensor,
                        next_tokens: torch.Tensor, logits: Optional[torch.Tensor] = None, stream=None) -> None:
    """war_verify_step over the library's static device scratch (allocates nothing)."""
    B = seq_ids.numel()
    _check(lib().war_verify_step_noalloc(model.handle, pool.handle, B, _ptr(seq_ids), _ptr(ctx_lens),
                                         _ptr(last_tokens), _ptr(draft_tokens), _ptr(draft_lens), k_max,
                                         _ptr(accept_lens), _ptr(next_tokens), _ptr(logits), _stream(stream)))


def verify_step_sampled(model: Model, pool: Pool, seq_ids: torch.Tensor, ctx_lens: torch.Tensor,
                        last_tokens: torch.Tensor, draft_tokens: Optional[torch.Tensor],
                        draft_lens: Optional[torch.Tensor], k_max: int, uniforms: torch.Tensor,
                        temperature: float, top_k: int, accept_lens: torch.Tensor, next_tokens: torch.Tensor,
                        logits: Optional[torch.Tensor] = None, stream=None) -> None:
    """Sampled verification; uniforms fp32 [B * (k_max + 1), 2] on the device."""
    assert uniforms.dtype == torch.float32 and uniforms.is_contiguous()
    B = seq_ids.numel()
    _check(lib().war_verify_step_sampled(model.handle, pool.handle, B, _ptr(seq_ids), _ptr(ctx_lens),
                                         _ptr(last_tokens), _ptr(draft_tokens), _ptr(draft_lens), k_max,
                                         _ptr(uniforms), float(temperature), int(top_k), _ptr(accept_lens),
                                         _ptr(next_tokens), _ptr(logits), _stream(stream)))


def verify_step_tree(model: Model, pool: Pool, seq_ids: torch.Tensor, ctx_lens: torch.Tensor,
                     last_tokens: torch.Tensor, draft_tokens: Optional[torch.Tensor],
                     draft_parents: Optional[torch.Tensor], draft_lens: Optional[torch.Tensor], k_max: int,
                     accept_lens: torch.Tensor, next_tokens: torch.Tensor,
                     accept_path: Optional[torch.Tensor] = None, logits: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """Tree drafts: draft_parents int32 [B, k_max], node i's parent in [0, i)."""
    B = seq_ids.numel()
    _check(lib().war_verify_step_tree(model.handle, pool.handle, B, _ptr(seq_ids), _ptr(ctx_lens),
                                      _ptr(last_tokens), _ptr(draft_tokens), _ptr(draft_parents),
                                      _ptr(draft_lens), k_max, _ptr(accept_lens), _ptr(next_tokens),
                                      _ptr(accept_path), _ptr(logits), _stream(stream)))


def kv_commit(pool: Pool, seq_ids: torch.Tensor, ctx_lens: torch.Tensor, accept_lens: torch.Tensor,
              stream=None) -> None:
    _check(lib().war_kv_commit(pool.handle, seq_ids.numel(), _ptr(seq_ids), _ptr(ctx_lens),
                               _ptr(accept_lens), _stream(stream)))


def prefill_append(model: Model, pool: Pool, seq_ids: torch.Tensor, ctx_lens: torch.Tensor,
                   n_new: Sequence[int], new_tokens: torch.Tensor, next_tokens: torch.Tensor,
                   last_logits: Optional[torch.Tensor] = None, stream=None) -> None:
    n = seq_ids.numel()
    _check(lib().war_prefill_append(model.handle, pool.handle, n, _ptr(seq_ids), _ptr(ctx_lens),
                                    _host_i32(n_new), _ptr(new_tokens), _ptr(next_tokens),
                                    _ptr(last_logits), _stream(stream)))


def _require(ok: bool, msg: str) -> None:
    if not ok:
        raise ValueError(msg)


def _addr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _checked(device, dtype, **arrays) -> None:
    """Arrays of a type without gaps on the device (None: absent)."""
    for name, t in arrays.items():
        if t is not None and not (t.dtype is dtype and t.device == device and t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous {dtype} tensor on {device}")


def _call(fn, device, stream, *args) -> None:
    """fn(*args, stream) with `device` current; its current stream by default (read raw:
    a Stream object is made in 2 us, a third of a small call)."""
    if device.index is None:
        raise ValueError(f"tensors must be on the GPU, not on {device}")
    raw = torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == device.index:
        status = fn(*args, raw)
    else:
        with torch.cuda.device(device):
            status = fn(*args, raw)
    if status:
        _check(status)


def _rows_of(name: str, t: torch.Tensor, device, B: int, n: int, heads: int, dim: int) -> int:
    """The row stride of bf16 [B, n, heads, dim] whose rows b * n + i lie at one stride."""
    if t.dtype is torch.bfloat16 and t.device == device and t.shape == (B, n, heads, dim):
        sb, sn, sh, sd = t.stride()
        if sd == 1 and sh == dim and sb == n * sn and B * n > 1:  # the usual case, in half the time
            return sn
    if not (t.dtype is torch.bfloat16 and t.device == device and t.shape == (B, n, heads, dim)):
        raise ValueError(f"{name} must be bf16 [{B}, {n}, {heads}, {dim}] on {device}")
    if t.is_contiguous():
        return heads * dim
    sb, sn, sh, sd = t.stride()
    row = sn if n > 1 else sb if B > 1 else heads * dim
    if not (sd == 1 and (heads == 1 or sh == dim) and (n < 2 or B < 2 or sb == n * row)):
        raise ValueError(f"{name}: heads must lie one after the other, rows at one stride")
    return row


def _kv_move(fn, pool: Pool, layer, seq_ids, pos0, k, v, n_lens, stream):
    B, n, dev, c = seq_ids.numel(), k.shape[1], pool.kv.device, pool.cfg
    _checked(dev, torch.int32, seq_ids=seq_ids, pos0=pos0, n_lens=n_lens)
    _require(pos0.numel() == B and (n_lens is None or n_lens.numel() == B), "pos0 and n_lens must hold one entry a request")
    ks, vs = _rows_of("k", k, dev, B, n, c.n_kv_heads, c.head_dim), _rows_of("v", v, dev, B, n, c.n_kv_heads, c.head_dim)
    _call(fn, dev, stream, pool.handle, layer, B, seq_ids.data_ptr(), pos0.data_ptr(), n, _addr(n_lens), k.data_ptr(), ks,
          v.data_ptr(), vs)


def kv_write(pool: Pool, layer: int, seq_ids: torch.Tensor, pos0: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
             n_lens: Optional[torch.Tensor] = None, stream=None) -> None:
    """Keys (after RoPE) and values bf16 [B, n, Hkv, D] of tokens pos0[b] + i into their
    pages; n_lens: live rows of each request."""
    _kv_move(lib().war_kv_write, pool, layer, seq_ids, pos0, k, v, n_lens, stream)


def kv_read(pool: Pool, layer: int, seq_ids: torch.Tensor, pos0: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
            n_lens: Optional[torch.Tensor] = None, stream=None) -> None:
    """The same tokens' keys and values from their pages into k and v (8 bits: the
    numbers the codes stand for); rows beyond n_lens stay as they are."""
    _kv_move(lib().war_kv_read, pool, layer, seq_ids, pos0, k, v, n_lens, stream)


class AttendPlan:
    """Attention of given rows over a pool: owns the workspace of one plan, which
    serves all layers of a step.  At most max_batch requests of max_rows rows."""

    def __init__(self, pool: Pool, max_batch: int, max_rows: int):
        self.pool, self.max_rows, self.shape = pool, max_rows, None
        h = C.c_void_p()
        with torch.cuda.device(pool.kv.device):
            _check(lib().war_attend_create(pool.handle, max_batch, max_rows, C.byref(h)))
        self.handle = h

    def update(self, seq_ids: torch.Tensor, ctx_lens: torch.Tensor, n_lens: Optional[torch.Tensor] = None,
               draft_parents: Optional[torch.Tensor] = None, n_rows: Optional[int] = None, stream=None) -> None:
        """Plan the rows of these requests: n_rows (default max_rows) each, of which
        n_lens are live; row 0 at position ctx_lens[b]."""
        _require(bool(self.pool.handle), "the pool is closed")
        B, n, dev = seq_ids.numel(), self.max_rows if n_rows is None else n_rows, self.pool.kv.device
        _checked(dev, torch.int32, seq_ids=seq_ids, ctx_lens=ctx_lens, n_lens=n_lens, draft_parents=draft_parents)
        _require(ctx_lens.numel() == B and (n_lens is None or n_lens.numel() == B),
                 "ctx_lens and n_lens must hold one entry a request")
        _require(draft_parents is None or draft_parents.numel() == B * (n - 1), "draft_parents must be [B, n_rows - 1]")
        self.shape = None
        _call(lib().war_attend_update, dev, stream, self.handle, B, n, seq_ids.data_ptr(), ctx_lens.data_ptr(),
              _addr(n_lens), _addr(draft_parents))
        self.shape = (B, n)

    def close(self):
        if getattr(self, "handle", None):
            lib().war_attend_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def attend(plan: AttendPlan, layer: int, q: torch.Tensor, out: torch.Tensor, stream=None) -> torch.Tensor:
    """Attention of the planned rows in one layer: q, out bf16 [B, n_rows, Hq, D]."""
    _require(plan.shape is not None and bool(plan.pool.handle), "no plan: call update first (the pool must be open)")
    pool, (B, n) = plan.pool, plan.shape
    dev, H, D = pool.kv.device, pool.cfg.n_q_heads, pool.cfg.head_dim
    qs, os_ = _rows_of("q", q, dev, B, n, H, D), _rows_of("out", out, dev, B, n, H, D)
    _call(lib().war_attend_run, dev, stream, plan.handle, layer, q.data_ptr(), qs, out.data_ptr(), os_)
    return out


MX_FORMATS = {"e4m3": 2, "e2m1": 3}
_TYPES = {torch.bfloat16: 0, torch.float32: 1}


def _matrix(name: str, t: torch.Tensor, device, rows: int, cols: int, types=_TYPES) -> int:
    """The row stride of a [rows, cols] matrix of one of these types."""
    if t.dtype in types and t.device == device and t.shape == (rows, cols):
        row, col = t.stride()
        if col == 1 and rows > 1:
            return row
    if not (t.dtype in types and t.device == device and t.shape == (rows, cols) and (cols == 1 or t.stride(1) == 1)):
        raise ValueError(f"{name} must be [{rows}, {cols}] of {' or '.join(str(x) for x in types)} on {device}, columns "
                         "one after the other")
    return t.stride(0) if rows > 1 else (cols + 7) // 8 * 8


class Mx:
    """A matrix of microscaled numbers (war.h): codes uint8 [rows, cols] ("e4m3") or
    [rows, cols / 2] ("e2m1": two a byte, the even column in the low bits) and scales
    uint8 [rows, cols / 32], 2^(byte - 127) for 32 columns; rows of scales at a multiple
    of 4 bytes.  Both stay the caller's."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, format: str):
        if format not in MX_FORMATS:
            raise ValueError(f"format must be one of {sorted(MX_FORMATS)}")
        _require(codes.dim() == 2 and codes.dtype == torch.uint8 and scales.dtype == torch.uint8, "codes and scales must be uint8 matrices")
        rows, cols = codes.shape[0], codes.shape[1] * (1 if format == "e4m3" else 2)
        _require(cols >= 32 and cols % 32 == 0, "a row must hold whole blocks of 32")
        cs = _matrix("codes", codes, codes.device, rows, codes.shape[1], (torch.uint8,))
        ss = _matrix("scales", scales, codes.device, rows, cols // 32, (torch.uint8,))
        self.codes, self.scales, self.format, self.device, self.shape = codes, scales, format, codes.device, (rows, cols)
        self._c = _Mx(MX_FORMATS[format], rows, cols, codes.data_ptr(), -(-cs // 16) * 16 if rows < 2 else cs, scales.data_ptr(), ss)
        self._ref = C.byref(self._c)

    @staticmethod
    def empty(rows: int, cols: int, format: str, device="cuda") -> "Mx":
        """Memory for rows x cols numbers."""
        if format not in MX_FORMATS:
            raise ValueError(f"format must be one of {sorted(MX_FORMATS)}")
        codes = torch.empty((rows, cols if format == "e4m3" else cols // 2), dtype=torch.uint8, device=device)
        scales = torch.empty((rows, -(-cols // 128) * 4), dtype=torch.uint8, device=device)
        return Mx(codes, scales[:, : cols // 32], format)

    def __getitem__(self, rows: slice) -> "Mx":
        """Some of the rows, in the same memory."""
        _require(isinstance(rows, slice), "rows must be a slice: other indices would copy")
        return Mx(self.codes[rows], self.scales[rows], self.format)


def residual_norm(x: Optional[torch.Tensor], h: torch.Tensor, gain: torch.Tensor, eps: float, out, stream=None):
    """h += x (None: h stays), then out = h / sqrt(mean(h^2) + eps) * gain: into an Mx, or a
    bf16 matrix.  h fp32 or bf16 [rows, cols], x and gain bf16."""
    dev, (rows, cols) = h.device, h.shape
    hs = _matrix("h", h, dev, rows, cols)
    xs = 0 if x is None else _matrix("x", x, dev, rows, cols, (torch.bfloat16,))
    _checked(dev, torch.bfloat16, gain=gain)
    _require(gain.numel() == cols, "gain must hold an entry a column")
    if isinstance(out, Mx):
        _require(out.shape == (rows, cols) and out.device == dev, f"out must hold [{rows}, {cols}] on {dev}")
        mx, y, ys = out._ref, None, 0
    else:
        mx, y, ys = None, out.data_ptr(), _matrix("out", out, dev, rows, cols, (torch.bfloat16,))
    _call(lib().war_residual_norm, dev, stream, rows, cols, _addr(x), xs, h.data_ptr(), hs, _TYPES[h.dtype], gain.data_ptr(),
          eps, mx, y, ys)
    return out


def quantize(x: torch.Tensor, out: Mx, gate: Optional[torch.Tensor] = None, stream=None) -> Mx:
    """x (bf16 or fp32 [rows, cols]), or x * silu(gate), into codes."""
    dev, (rows, cols) = out.device, out.shape
    xs = _matrix("x", x, dev, rows, cols)
    gs = 0 if gate is None else _matrix("gate", gate, dev, rows, cols, (x.dtype,))
    _call(lib().war_quantize, dev, stream, out._ref, x.data_ptr(), xs, _addr(gate), gs, _TYPES[x.dtype])
    return out


def dequantize(mx: Mx, out: torch.Tensor, stream=None) -> torch.Tensor:
    """The numbers that codes stand for, into bf16 or fp32 [rows, cols]."""
    s = _matrix("out", out, mx.device, *mx.shape)
    _call(lib().war_dequantize, mx.device, stream, mx._ref, out.data_ptr(), s, _TYPES[out.dtype])
    return out


class Linear:
    """Weights [N, K] in 4 bits for y = x w^T + bias: an Mx in "e2m1", or a bf16 or fp32
    matrix that is quantised here; bias bf16 [N].  Laid out in memory of its own, so the
    arguments may be dropped afterwards."""

    def __init__(self, weight, bias: Optional[torch.Tensor] = None, stream=None):
        dev = weight.device
        if not isinstance(weight, Mx):
            _require(weight.dim() == 2, "weight must be a matrix")
            make = lambda: quantize(weight, Mx.empty(*weight.shape, "e2m1", dev), stream=stream)
            if stream is None:
                weight = make()
            else:  # that stream's own memory
                with torch.cuda.stream(stream):
                    weight = make()
        self.device, (self.out_features, self.in_features) = dev, weight.shape
        _checked(dev, torch.bfloat16, bias=bias)
        _require(bias is None or bias.numel() == self.out_features, "bias must hold an entry a row of the weights")
        h = C.c_void_p()
        create = lambda mx, b, st: lib().war_linear_create(mx, b, st, C.byref(h))
        _call(create, dev, stream, weight._ref, _addr(bias))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().war_linear_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def linear(weights: Linear, x: Mx, out: torch.Tensor, stream=None) -> torch.Tensor:
    """out = x w^T + bias: x [rows, K] in codes, out bf16 or fp32 [rows, N] (sums of e4m3 rows
    are cut on their way to bf16, as war.h says; fp32 has all of them)."""
    _require(bool(weights.handle), "the weights are closed")
    dev, N = weights.device, weights.out_features
    _require(x.device == dev and x.shape[1] == weights.in_features, f"x must have {weights.in_features} columns on {dev}")
    s = _matrix("out", out, dev, x.shape[0], N)
    _call(lib().war_linear_run, dev, stream, weights.handle, x._ref, out.data_ptr(), s, _TYPES[out.dtype])
    return out


class Rope:
    """Rotary positions: pair j of a head's first rotary_dim numbers (default all) turns by
    its row's position on axis axes[j] (default one axis) times base^(-2 j / rotary_dim),
    or freqs[j].  Pair j is (j, j + rotary_dim / 2); adjacent: (2 j, 2 j + 1)."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, base: float = 10000.0,
                 axes: Optional[Sequence[int]] = None, adjacent: bool = False, freqs: Optional[Sequence[float]] = None):
        R = head_dim if rotary_dim is None else rotary_dim
        _require(head_dim in (64, 128) and 8 <= R <= head_dim and R % 8 == 0, "rotary_dim must be a multiple of 8 in [8, head_dim]")
        axes = [0] * (R // 2) if axes is None else [int(a) for a in axes]
        freqs = [float(base) ** (-2.0 * j / R) for j in range(R // 2)] if freqs is None else [float(f) for f in freqs]
        _require(len(axes) == R // 2 and len(freqs) == R // 2, "axes and freqs must hold an entry a pair")
        _require(all(0 <= a < 4 for a in axes), "at most four axes")
        self.head_dim, self.n_axes = head_dim, max(axes) + 1
        self._axes, self._freqs = (C.c_uint8 * len(axes))(*axes), (C.c_double * len(freqs))(*freqs)
        self._c = _Rope(R, int(adjacent), self.n_axes, C.addressof(self._axes), C.addressof(self._freqs))
        self._ref = C.byref(self._c)


def rope_write(pool: Pool, layer: int, rope: Rope, seq_ids: torch.Tensor, pos0: torch.Tensor, q: torch.Tensor,
               k: torch.Tensor, v: torch.Tensor, q_out: torch.Tensor, n_lens: Optional[torch.Tensor] = None,
               positions: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Tokens pos0[b] + i: queries bf16 [B, n, Hq, D] turned into q_out (may be q), keys
    bf16 [B, n, Hkv, D] turned and written into their pages with the values.  positions
    int32 [n_axes, B, n]: where each row is on each axis (default: its place in the cache
    on all of them)."""
    B, n, dev, c = seq_ids.numel(), k.shape[1], pool.kv.device, pool.cfg
    _checked(dev, torch.int32, seq_ids=seq_ids, pos0=pos0, n_lens=n_lens, positions=positions)
    _require(bool(pool.handle), "the pool is closed")
    _require(rope.head_dim == c.head_dim, "rope is made for another head_dim")
    _require(pos0.numel() == B and (n_lens is None or n_lens.numel() == B), "pos0 and n_lens must hold one entry a request")
    _require(positions is None or (positions.shape[0] >= rope.n_axes and positions.shape[1:] == (B, n)),
             f"positions must be [{rope.n_axes}, {B}, {n}]")
    Hq, Hkv, D = c.n_q_heads, c.n_kv_heads, c.head_dim
    qs, os_ = _rows_of("q", q, dev, B, n, Hq, D), _rows_of("q_out", q_out, dev, B, n, Hq, D)
    ks, vs = _rows_of("k", k, dev, B, n, Hkv, D), _rows_of("v", v, dev, B, n, Hkv, D)
    _call(lib().war_rope_write, dev, stream, pool.handle, layer, rope._ref, B, seq_ids.data_ptr(), pos0.data_ptr(), n,
          _addr(n_lens), _addr(positions), q.data_ptr(), qs, q_out.data_ptr(), os_, k.data_ptr(), ks, v.data_ptr(), vs)
    return q_out


class Constraints:
    """What requests' next tokens are held to (war.h); every array is optional and stays
    the caller's, to be changed in place as requests come and go.
    By sequence id: counts int16 [n_seqs, vocab] (16 bits a token: counts_begin,
    counts_add), repetition, frequency, presence fp32 [n_seqs], bias_ids int32 and
    bias_values fp32 [n_seqs, n_bias].  masks int32 [n_masks, ceil(vocab / 32)]: a bit a
    token; mask_index int32, the mask of each row (negative: none), default row r mask r."""

    def __init__(self, vocab: int, counts: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None,
                 frequency: Optional[torch.Tensor] = None, presence: Optional[torch.Tensor] = None,
                 bias_ids: Optional[torch.Tensor] = None, bias_values: Optional[torch.Tensor] = None,
                 masks: Optional[torch.Tensor] = None, mask_index: Optional[torch.Tensor] = None,
                 n_seqs: Optional[int] = None):
        by_seq = [t for t in (counts, repetition, frequency, presence, bias_ids, bias_values) if t is not None]
        arrays = by_seq + [t for t in (masks, mask_index) if t is not None]
        _require(bool(by_seq) or n_seqs is not None, "n_seqs is needed where no array is by sequence")
        _require(bool(arrays), "nothing constrains")
        n = n_seqs if n_seqs is not None else by_seq[0].shape[0]
        dev = arrays[0].device
        _checked(dev, torch.int16, counts=counts)
        _checked(dev, torch.float32, repetition=repetition, frequency=frequency, presence=presence, bias_values=bias_values)
        _checked(dev, torch.int32, bias_ids=bias_ids, masks=masks, mask_index=mask_index)
        _require(all(t.shape[0] == n for t in by_seq), "arrays by sequence must have the same number of rows")
        _require(counts is None or counts.shape == (n, vocab), "counts must be [n_seqs, vocab]")
        _require(all(t is None or t.shape == (n,) for t in (repetition, frequency, presence)), "penalties must be [n_seqs]")
        _require((bias_ids is None) == (bias_values is None) and
                 (bias_ids is None or (bias_ids.dim() == 2 and bias_ids.shape == bias_values.shape)),
                 "bias_ids and bias_values must both be [n_seqs, n_bias]")
        _require(masks is None or (masks.dim() == 2 and masks.shape[1] == (vocab + 31) // 32),
                 "masks must be [n_masks, ceil(vocab / 32)]")
        self.vocab, self.device, self.masks, self.mask_index = vocab, dev, masks, mask_index
        self._keep = arrays
        self._c = _Constraints(n, _addr(counts), _addr(repetition), _addr(frequency), _addr(presence),
                               0 if bias_ids is None else bias_ids.shape[1], _addr(bias_ids), _addr(bias_values),
                               0 if masks is None else masks.shape[0], _addr(masks), _addr(mask_index))
        self._ref = C.byref(self._c)

    def _rows(self, rows: int) -> None:
        """The masks of a call with this many rows."""
        _require(self.masks is None or (self.mask_index.numel() if self.mask_index is not None else self.masks.shape[0]) >= rows,
                 "a mask (mask_index) is needed for each row")


def constrain_logits(logits: torch.Tensor, constraints: Constraints, seq_ids: torch.Tensor, last_tokens: torch.Tensor,
                     draft_tokens: Optional[torch.Tensor], draft_lens: Optional[torch.Tensor], k_max: int,
                     out: Optional[torch.Tensor] = None, greedy: Optional[torch.Tensor] = None,
                     draft_parents: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """Constrained logits fp32 [B * (k_max + 1), vocab] of a step's rows into out (may be
    logits itself) and each row's greedy token into greedy int32 (-1: no token is
    allowed); at least one of the two.  A workspace (uint8) of war_constrain_workspace
    bytes is allocated where none is given."""
    B, V, dev = seq_ids.numel(), constraints.vocab, constraints.device
    rows = B * (k_max + 1)
    _checked(dev, torch.int32, seq_ids=seq_ids, last_tokens=last_tokens, draft_tokens=draft_tokens, draft_lens=draft_lens,
             draft_parents=draft_parents, greedy=greedy)
    _require(last_tokens.numel() == B and (draft_lens is None or draft_lens.numel() == B) and
             all(t is None or t.numel() == B * k_max for t in (draft_tokens, draft_parents)) and
             (greedy is None or greedy.numel() == rows), "token arrays do not fit B requests of k_max drafts")
    for name, t in (("logits", logits), ("out", out)):
        if t is not None and not (t.dtype == torch.float32 and t.device == dev and t.shape == (rows, V) and
                                  (V == 1 or t.stride(1) == 1)):
            raise ValueError(f"{name} must be fp32 [{rows}, {V}] on {dev}, ids one after the other")
    constraints._rows(rows)
    fn = lib()
    if greedy is not None:
        need = fn.war_constrain_workspace(rows, V)
        if workspace is None:
            make = lambda: torch.empty(max(need, 0), dtype=torch.uint8, device=dev)
            if stream is None:
                workspace = make()
            else:  # that stream's own memory: what another one freed may still be in use there
                with torch.cuda.stream(stream):
                    workspace = make()
        _require(workspace.device == dev and workspace.is_contiguous() and
                 workspace.numel() * workspace.element_size() >= need, f"workspace must hold {need} bytes on {dev}")
    ls = logits.stride(0) if rows > 1 else V
    os_ = V if out is None else out.stride(0) if rows > 1 else V
    _call(fn.war_constrain_logits, dev, stream, constraints._ref, V, B, seq_ids.data_ptr(), last_tokens.data_ptr(),
          _addr(draft_tokens) if k_max else None, _addr(draft_parents), _addr(draft_lens), k_max, logits.data_ptr(), ls,
          _addr(out), os_, _addr(greedy), _addr(workspace) if greedy is not None else None)


def _counts_of(counts: torch.Tensor):
    if not (counts.dtype == torch.int16 and counts.dim() == 2 and counts.is_contiguous() and counts.is_cuda):
        raise ValueError("counts must be a contiguous int16 [n_seqs, vocab] on the GPU")
    return counts.device, counts.data_ptr(), counts.shape[1], counts.shape[0]


def counts_begin(counts: torch.Tensor, seq_ids: torch.Tensor, tokens: torch.Tensor, offsets: torch.Tensor,
                 stream=None) -> None:
    """New requests' rows of counts: their prompts' tokens (packed; request i's at
    offsets[i] .. offsets[i + 1]) are marked, everything else is cleared."""
    dev, at, V, S = _counts_of(counts)
    _checked(dev, torch.int32, seq_ids=seq_ids, tokens=tokens, offsets=offsets)
    _require(offsets.numel() == seq_ids.numel() + 1, "offsets must hold one more entry than seq_ids")
    _call(lib().war_counts_begin, dev, stream, at, V, S, seq_ids.numel(), seq_ids.data_ptr(), tokens.data_ptr(),
          tokens.numel(), offsets.data_ptr())


def counts_add(counts: torch.Tensor, seq_ids: torch.Tensor, first: Optional[torch.Tensor],
               tokens: Optional[torch.Tensor], lens: Optional[torch.Tensor], path: Optional[torch.Tensor] = None,
               stream=None) -> None:
    """Count generated tokens: first[b], then lens[b] (a step's accept_lens; -1: nothing)
    of tokens[b]; path: a tree's accept_path."""
    dev, at, V, S = _counts_of(counts)
    B = seq_ids.numel()
    _checked(dev, torch.int32, seq_ids=seq_ids, first=first, tokens=tokens, lens=lens, path=path)
    n = 0 if tokens is None or B == 0 else tokens.numel() // B
    _require((tokens is None or tokens.numel() == B * n) and (path is None or path.numel() == B * n) and
             all(t is None or t.numel() == B for t in (first, lens)), "token arrays do not fit the requests")
    _call(lib().war_counts_add, dev, stream, at, V, S, B, seq_ids.data_ptr(), _addr(first), _addr(tokens), n, _addr(path),
          _addr(lens))


def verify_step_constrained(model: Model, pool: Pool, seq_ids: torch.Tensor, ctx_lens: torch.Tensor,
                            last_tokens: torch.Tensor, draft_tokens: Optional[torch.Tensor],
                            draft_lens: Optional[torch.Tensor], k_max: int, constraints: Constraints,
                            accept_lens: torch.Tensor, next_tokens: torch.Tensor,
                            logits: Optional[torch.Tensor] = None, draft_parents: Optional[torch.Tensor] = None,
                            accept_path: Optional[torch.Tensor] = None, uniforms: Optional[torch.Tensor] = None,
                            temperature: float = 1.0, top_k: int = 1, stream=None) -> None:
    """A verify step (draft_parents: of draft trees; uniforms: sampled, as
    verify_step_sampled) whose rows' logits are constrained before a token is chosen.
    Afterwards counts_add counts what was committed."""
    B, dev = seq_ids.numel(), pool.kv.device
    _checked(dev, torch.int32, seq_ids=seq_ids, ctx_lens=ctx_lens, last_tokens=last_tokens, draft_tokens=draft_tokens,
             draft_lens=draft_lens, accept_lens=accept_lens, next_tokens=next_tokens, draft_parents=draft_parents,
             accept_path=accept_path)
    _checked(dev, torch.float32, uniforms=uniforms, logits=logits)
    _require(constraints.vocab == model.cfg.vocab and constraints.device == dev, "constraints of another vocabulary or device")
    rows = B * (k_max + 1)
    constraints._rows(rows)
    _require(all(t.numel() == B for t in (ctx_lens, last_tokens, accept_lens, next_tokens)) and
             (draft_lens is None or draft_lens.numel() == B) and
             all(t is None or t.numel() >= B * k_max for t in (draft_tokens, draft_parents, accept_path)) and
             (uniforms is None or uniforms.numel() == 2 * rows) and
             (logits is None or logits.numel() == rows * model.cfg.vocab), "arrays do not fit B requests of k_max drafts")
    _call(lib().war_verify_step_constrained, dev, stream, model.handle, pool.handle, B, seq_ids.data_ptr(),
          ctx_lens.data_ptr(), last_tokens.data_ptr(), _addr(draft_tokens), _addr(draft_parents), _addr(draft_lens), k_max,
          constraints._ref, _addr(uniforms), float(temperature), int(top_k), accept_lens.data_ptr(),
          next_tokens.data_ptr(), _addr(accept_path), _addr(logits))


def debug_mfma16(A: torch.Tensor, B: torch.Tensor, stream=None) -> torch.Tensor:
    """C = A @ B (A bf16 [16, 32], B bf16 [32, 16]) through one matrix-core instruction."""
    out = torch.empty((16, 16), dtype=torch.float32, device=A.device)
    _check(lib().war_debug_mfma16(_ptr(A.contiguous()), _ptr(B.contiguous()), _ptr(out), _stream(stream)))
    return out


def debug_sample(logits: torch.Tensor, ntok: torch.Tensor, drafts: torch.Tensor, k_max: int,
                 uniforms: torch.Tensor, temperature: float, top_k: int, accept_lens: torch.Tensor,
                 next_tokens: torch.Tensor, stream=None) -> None:
    """The sampled-verification decisions alone on given logit rows (war_debug.h)."""
    B, V = ntok.numel(), logits.shape[-1]
    _check(lib().war_debug_sample(_ptr(logits), V, B, k_max, _ptr(ntok), _ptr(drafts), _ptr(uniforms),
                                  float(temperature), int(top_k), _ptr(accept_lens), _ptr(next_tokens),
                                  _stream(stream)))


def debug_linear(weights: Linear, x: Mx, out: torch.Tensor, shape: int, stream=None) -> torch.Tensor:
    """linear() through a chosen shape of workgroups (war_debug.h)."""
    s = _matrix("out", out, weights.device, x.shape[0], weights.out_features)
    _call(lib().war_debug_linear, weights.device, stream, weights.handle, x._ref, out.data_ptr(), s, _TYPES[out.dtype], shape)
    return out


def debug_gemm_plan(M: int, N: int, K: int, epi: int, cap_elems: int = 64 << 20) -> tuple:
    """(tile shape or -1, splits, k range of a split) of a product (war_debug.h)."""
    out = [C.c_int32() for _ in range(3)]
    _check(lib().war_debug_gemm_plan(M, N, K, epi, cap_elems, *[C.byref(x) for x in out]))
    return tuple(x.value for x in out)


def debug_gemm(A: torch.Tensor, W: torch.Tensor, epi: int, shape: int, splits: int = 1, kper: int = 0,
               W2: Optional[torch.Tensor] = None, a_rows: Optional[torch.Tensor] = None, stream=None):
    """One product through a chosen kernel (war_debug.h): partial sums [splits, M, N],
    (logits [M, N], block maxima, their columns) or the SwiGLU output [M, N / 2]."""
    M = A.shape[0] if a_rows is None else a_rows.numel()
    N, K = W.shape[0] * (2 if W2 is not None else 1), A.shape[1]
    dev = A.device
    best = (torch.zeros((M, N // 128), device=dev), torch.zeros((M, N // 128), dtype=torch.int32, device=dev))
    out = (torch.full((splits, M, N), float("nan"), device=dev) if epi == 0 else
           torch.full((M, N), float("nan"), device=dev) if epi == 1 else
           torch.full((M, N // 2), float("nan"), dtype=torch.bfloat16, device=dev))
    _check(lib().war_debug_gemm(_ptr(A), _ptr(W), _ptr(W2), M, N, K, epi, shape, splits, kper or K, _ptr(a_rows),
                                _ptr(out), _ptr(best[0]), _ptr(best[1]), _stream(stream)))
    return (out, *best) if epi == 1 else out


def debug_workspace(model: Model, name: str, dtype: torch.dtype, shape) -> torch.Tensor:
    """Copy of a model workspace buffer (see war_debug.h), reinterpreted."""
    p, n = C.c_void_p(), C.c_int64()
    _check(lib().war_debug_workspace(model.handle, name.encode(), C.byref(p), C.byref(n)))
    numel = 1
    for s in shape:
        numel *= s
    nbytes = numel * torch.tensor([], dtype=dtype).element_size()
    assert nbytes <= n.value, (nbytes, n.value)
    buf = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    import ctypes
    hip = ctypes.CDLL("libamdhip64.so")
    hip.hipMemcpy(C.c_void_p(buf.data_ptr()), p, C.c_size_t(nbytes), 3)   # device to device
    return buf.view(dtype).view(*shape).clone()


def profile(model: Model, enable: bool) -> None:
    _check(lib().war_profile(model.handle, 1 if enable else 0))


def profile_read(model: Model) -> Dict[str, tuple]:
    """{kernel name: (calls, total_ms)} since the last read; synchronises."""
    buf = C.create_string_buffer(1 << 16)
    _check(lib().war_profile_read(model.handle, buf, len(buf)))
    out = {}
    for line in buf.value.decode().splitlines():
        name, calls, ms = line.split()
        out[name] = (int(calls), float(ms))
    return out
