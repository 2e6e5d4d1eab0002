"""Python binding of the DPB C-ABI library (``include/dpb.h``).

Argument marshalling only: every step of encode, decode and backward runs in
the library's CUDA kernels. PyTorch supplies device memory and the current
stream; tensors are passed to the library as raw pointers. The functions keep
the C names (``dpb_encode`` -> ``encode`` ...). Loading fails loudly if the
library has not been built: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from typing import Optional, Sequence

import torch

from . import build as _build

MAX_LEVELS = 8
MAX_CHILDREN = 256
F32, BF16 = 0, 1
SELECT_GLOBAL, SELECT_PER_LEVEL = 0, 1
SCORING_CONTRACTION, SCORING_COSET_WHT = 0, 1
DEV_BAD_INDEX, DEV_BAD_SIGMA, DEV_SHORT_CODE, DEV_TIMEOUT = 0x1, 0x2, 0x4, 0x8
DEV_BAD_LENGTH = 0x10
STATE_BLOCK = 256  # values of an 8-bit optimiser state that share a scale

_STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported configuration", 3: "CUDA error",
           4: "device wait timed out", 5: "out of memory", 6: "device-side error flagged"}


class DPBError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [
        ("d", ctypes.c_int32),
        ("levels", ctypes.c_int32),
        ("m_bits", ctypes.c_int32),
        ("bits", ctypes.c_int32 * MAX_LEVELS),
        ("children", ctypes.c_int32 * MAX_LEVELS),
        ("beam", ctypes.c_int32),
        ("k", ctypes.c_int32),
        ("k_per_level", ctypes.c_int32 * MAX_LEVELS),
        ("select_mode", ctypes.c_int32),
        ("norm_match", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("field_t", ctypes.c_int32),
        ("field_poly", ctypes.c_uint32),
        ("generator_seed", ctypes.c_uint64),
        ("scoring", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]

    def as_dict(self) -> dict:
        L = self.levels
        return {"d": self.d, "levels": L, "m_bits": self.m_bits, "bits": list(self.bits[:L]),
                "children": list(self.children[:L]), "beam": self.beam, "k": self.k,
                "k_per_level": list(self.k_per_level[:L]), "select_mode": self.select_mode,
                "norm_match": self.norm_match, "dtype": self.dtype, "field_t": self.field_t,
                "field_poly": self.field_poly, "generator_seed": self.generator_seed, "scoring": self.scoring}


# dpb_rope_config, dpb_attention_config and up to eight dpb_heads, as they lie in memory
_ROPE = struct.Struct("=q8ifi")
_ATTENTION = struct.Struct("=qq8ifi")
_ROWS = {n: struct.Struct(f"={3 * n}q") for n in (4, 6, 8)}
# dpb_linear_loss_config, dpb_embedding_config, dpb_norm_config and two or four dpb_rows (16 bytes each)
_LOSS = struct.Struct("=qiiqiiii")
_EMBEDDING = struct.Struct("=qiiiifi")
_NORM = struct.Struct("=qiifi")
_PLAIN_ROWS = {n: struct.Struct(f"={2 * n}q") for n in (2, 4)}


class _Arguments(threading.local):
    """This thread's memory for a call's config (at `at`) and dpb_heads (at
    `rows`, 24 bytes each): written anew for every call, cheaper than new
    ctypes objects."""

    def __init__(self):
        self.buf = ctypes.create_string_buffer(64 + 24 * 8)
        self.at = ctypes.addressof(self.buf)
        self.rows = self.at + 64


_arguments = _Arguments()


class AdamWConfig(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64),
                ("seed", ctypes.c_uint64), ("grad_scale", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("state_bits", ctypes.c_int32)]


_lib = None
EXPORTS = ("dpb_plan_create", "dpb_plan_destroy", "dpb_plan_config", "dpb_plan_tables",
           "dpb_code_length", "dpb_workspace_size", "dpb_encode", "dpb_decode", "dpb_backward",
           "dpb_workspace_status", "dpb_status_string", "dpb_last_error", "dpb_encode_noalloc",
           "dpb_stats_accumulate", "dpb_stats_update", "dpb_forward", "dpb_debug_set_wait_limit", "dpb_status_word",
           "dpb_qk_norm_rope", "dpb_qk_norm_rope_backward", "dpb_rope_workspace_size",
           "dpb_attention_forward", "dpb_attention_backward", "dpb_attention_workspace_size", "dpb_adamw_step",
           "dpb_linear_cross_entropy_forward", "dpb_linear_cross_entropy_backward",
           "dpb_linear_cross_entropy_workspace_size", "dpb_embedding", "dpb_embedding_backward",
           "dpb_embedding_workspace_size", "dpb_add_norm", "dpb_add_norm_backward", "dpb_norm_workspace_size")


def library_path() -> str:
    return _build.LIB


def load(path: Optional[str] = None):
    """Load libdpb.so (built in-tree by ``build.build()``); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"DPB CUDA library not built ({path} missing); run "
                           "paper_2607_20652_gb300.build.build() first")
    lib = ctypes.CDLL(path)
    vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    st = ctypes.c_int
    lib.dpb_plan_create.argtypes = [ctypes.POINTER(Config), vp, ctypes.POINTER(vp)]
    lib.dpb_plan_destroy.argtypes = [vp]
    lib.dpb_plan_config.argtypes = [vp, ctypes.POINTER(Config)]
    lib.dpb_plan_tables.argtypes = [vp, vp, vp]
    lib.dpb_code_length.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
    lib.dpb_workspace_size.argtypes = [vp, i64, ctypes.POINTER(sz)]
    lib.dpb_encode.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.dpb_decode.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    lib.dpb_backward.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.dpb_workspace_status.argtypes = [vp, ctypes.c_int, ctypes.POINTER(ctypes.c_int32), vp]
    lib.dpb_encode_noalloc.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.dpb_debug_set_wait_limit.argtypes = [ctypes.c_int32]
    lib.dpb_status_word.argtypes = [ctypes.c_int32, ctypes.POINTER(vp)]
    lib.dpb_stats_accumulate.argtypes = [vp, vp, i64, vp, vp, vp, ctypes.c_int32, vp, vp, sz, vp]
    lib.dpb_stats_update.argtypes = [vp, vp, ctypes.c_float, vp, vp, vp]
    lib.dpb_forward.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    hp = rc = ac = vp  # addresses within _Arguments
    lib.dpb_qk_norm_rope.argtypes = [rc, hp, hp, vp, vp, vp, vp, vp, hp, hp, vp, sz, vp]
    lib.dpb_qk_norm_rope_backward.argtypes = [rc, hp, hp, hp, hp, vp, vp, vp, vp, vp, hp, hp, vp, vp, vp, sz, vp]
    lib.dpb_rope_workspace_size.argtypes = [rc, ctypes.POINTER(sz)]
    lib.dpb_attention_forward.argtypes = [ac, hp, hp, hp, vp, vp, hp, vp, vp, sz, vp]
    lib.dpb_attention_backward.argtypes = [ac, hp, hp, hp, hp, vp, hp, vp, vp, hp, hp, hp, vp, sz, vp]
    lib.dpb_attention_workspace_size.argtypes = [ac, ctypes.POINTER(sz)]
    lib.dpb_adamw_step.argtypes = [ctypes.POINTER(AdamWConfig), vp, ctypes.c_int32, vp]
    lib.dpb_linear_cross_entropy_forward.argtypes = [rc, hp, hp, vp, vp, vp, vp, vp, sz, vp]
    lib.dpb_linear_cross_entropy_backward.argtypes = [rc, hp, hp, vp, vp, vp, hp, hp, vp, sz, vp]
    lib.dpb_linear_cross_entropy_workspace_size.argtypes = [rc, ctypes.c_int32, ctypes.POINTER(sz)]
    lib.dpb_embedding.argtypes = [rc, hp, vp, hp, vp, sz, vp]
    lib.dpb_embedding_backward.argtypes = [rc, hp, vp, hp, vp, sz, vp]
    lib.dpb_embedding_workspace_size.argtypes = [rc, ctypes.POINTER(sz)]
    lib.dpb_add_norm.argtypes = [rc, hp, hp, vp, hp, hp, vp]
    lib.dpb_add_norm_backward.argtypes = [rc, hp, hp, hp, vp, hp, vp, vp, sz, vp]
    lib.dpb_norm_workspace_size.argtypes = [rc, ctypes.POINTER(sz)]
    lib.dpb_status_string.argtypes = [st]
    lib.dpb_status_string.restype = ctypes.c_char_p
    lib.dpb_last_error.argtypes = []
    lib.dpb_last_error.restype = ctypes.c_char_p
    for name in EXPORTS:
        f = getattr(lib, name)
        if f.restype is None or f.restype is ctypes.c_int:
            f.restype = st
    lib.dpb_status_string.restype = ctypes.c_char_p
    lib.dpb_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int):
    if status != 0:
        msg = load().dpb_last_error().decode(errors="replace")
        raise DPBError(status, msg)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


_DTYPES = {"f32": (F32, torch.float32), "fp32": (F32, torch.float32), "float32": (F32, torch.float32),
           "bf16": (BF16, torch.bfloat16), "bfloat16": (BF16, torch.bfloat16)}


class Plan:
    """A DPB plan (``dpb_plan_create``): resolved config, seed matrix M and
    the generators of every level, resident on the current device."""

    def __init__(self, d: int, levels: int, m_bits: int = 0, children: int | Sequence[int] = 16,
                 beam: int = 8, k: int = 64, dtype: str = "bf16", norm_match: int = 1,
                 seed: int = 0, field_t: int = 0, field_poly: int = 0,
                 bits: Optional[Sequence[int]] = None, generators=None,
                 select_mode: int = SELECT_GLOBAL, k_per_level: Optional[Sequence[int]] = None,
                 scoring: int = SCORING_CONTRACTION):
        lib = load()
        c = Config()
        c.d, c.levels, c.m_bits = d, levels, m_bits
        if bits is not None:
            for l, b in enumerate(bits):
                c.bits[l] = b
        if isinstance(children, int):
            children = [0] + [children] * (levels - 1)
        for l, ch in enumerate(children):
            c.children[l] = ch
        c.beam, c.k = beam, k
        if k_per_level is not None:
            for l, kk in enumerate(k_per_level):
                c.k_per_level[l] = kk
        c.select_mode, c.norm_match = select_mode, norm_match
        c.dtype = _DTYPES[dtype][0]
        c.field_t, c.field_poly, c.generator_seed = field_t, field_poly, seed & (2**64 - 1)
        c.scoring = scoring
        gen_buf = None
        if generators is not None:
            import numpy as np
            g = np.zeros((MAX_LEVELS, MAX_CHILDREN), dtype=np.uint32)
            src = np.asarray(generators, dtype=np.uint32)
            g[: src.shape[0], : min(src.shape[1], MAX_CHILDREN)] = src[:, :MAX_CHILDREN]
            gen_buf = g
        handle = ctypes.c_void_p()
        _check(lib.dpb_plan_create(ctypes.byref(c),
                                   None if gen_buf is None else gen_buf.ctypes.data_as(ctypes.c_void_p),
                                   ctypes.byref(handle)))
        self._h = handle
        self._lib = lib
        out = Config()
        _check(lib.dpb_plan_config(self._h, ctypes.byref(out)))
        self.config = out.as_dict()
        kk = ctypes.c_int32()
        _check(lib.dpb_code_length(self._h, ctypes.byref(kk)))
        self.code_len = kk.value
        self.n_features = 1 << self.config["bits"][self.config["levels"] - 1]  # 2^N
        self.d = d
        self.torch_dtype = _DTYPES[dtype][1]

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            try:
                self._lib.dpb_plan_destroy(h)
            except Exception:
                pass
            self._h = None

    @property
    def handle(self):
        return self._h

    def tables(self):
        """(M [d] uint32, G [MAX_LEVELS, MAX_CHILDREN] uint32) as numpy arrays."""
        import numpy as np
        M = np.zeros(self.d, dtype=np.uint32)
        G = np.zeros((MAX_LEVELS, MAX_CHILDREN), dtype=np.uint32)
        _check(self._lib.dpb_plan_tables(self._h, M.ctypes.data_as(ctypes.c_void_p),
                                         G.ctypes.data_as(ctypes.c_void_p)))
        return M, G

    def workspace_size(self, T: int) -> int:
        n = ctypes.c_size_t()
        _check(self._lib.dpb_workspace_size(self._h, T, ctypes.byref(n)))
        return n.value

    def workspace(self, T: int, device=None) -> torch.Tensor:
        """A zero-filled workspace tensor (uint8) for up to T tokens."""
        n = self.workspace_size(T)
        return torch.zeros(n, dtype=torch.uint8, device=device or "cuda")

    def _stream_workspace(self, T: int, device, stream) -> torch.Tensor:
        """The workspace of calls made without one: one per (device, stream),
        kept with the plan (calls on one stream run in order, so they may
        share it; its status bits accumulate until read and cleared)."""
        dev = torch.device(device)
        s = stream if stream is not None else torch.cuda.current_stream(dev)
        key = (dev.index if dev.index is not None else torch.cuda.current_device(), s.cuda_stream)
        cache = self.__dict__.setdefault("_ws_cache", {})
        ws = cache.get(key)
        if ws is None or ws.numel() < self.workspace_size(T):
            # allocated and zeroed on the stream the calls use, so the first
            # kernel cannot start before the fill ends
            with torch.cuda.stream(s):
                ws = cache[key] = self.workspace(T, dev)
        return ws

    def status(self, device=None, stream=None, clear: bool = True) -> int:
        """The DPB_DEV_* bits that calls made without a workspace left on
        ``stream`` (synchronises it); cleared by default."""
        dev = torch.device(device or "cuda")
        s = stream if stream is not None else torch.cuda.current_stream(dev)
        key = (dev.index if dev.index is not None else torch.cuda.current_device(), s.cuda_stream)
        ws = self.__dict__.get("_ws_cache", {}).get(key)
        return 0 if ws is None else workspace_status(ws, clear=clear, stream=s)


def _rows(t: torch.Tensor, plan: Plan, name: str):
    if t.dtype != plan.torch_dtype or not t.is_cuda or not t.is_contiguous() or t.dim() != 2 \
            or t.shape[1] != plan.d:
        raise ValueError(f"{name} must be a contiguous CUDA {plan.torch_dtype} tensor of shape [T, {plan.d}]")


def encode(plan: Plan, x: torch.Tensor, mu=None, sigma=None, idx=None, val=None, xnorm=None,
           workspace=None, stream=None, want_xnorm: bool = True):
    """dpb_encode. Returns (idx int32 [T,k], val fp32 [T,k], xnorm fp32 [T] or None)."""
    _rows(x, plan, "x")
    T, k = x.shape[0], plan.code_len
    dev = x.device
    idx = torch.empty((T, k), dtype=torch.int32, device=dev) if idx is None else idx
    val = torch.empty((T, k), dtype=torch.float32, device=dev) if val is None else val
    if xnorm is None and want_xnorm:
        xnorm = torch.empty((T,), dtype=torch.float32, device=dev)
    ws = plan._stream_workspace(T, dev, stream) if workspace is None else workspace
    _check(plan._lib.dpb_encode(plan.handle, _ptr(x), T, _ptr(mu), _ptr(sigma), _ptr(idx), _ptr(val),
                                _ptr(xnorm), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))
    return idx, val, xnorm


def decode(plan: Plan, idx: torch.Tensor, val: torch.Tensor, xnorm=None, y=None, workspace=None,
           stream=None, r_out: Optional[torch.Tensor] = None):
    """dpb_decode. Returns y [T, d] in the plan's dtype; with ``r_out`` (fp32
    [T, d]) also keeps r there for dpb_backward."""
    T = idx.shape[0]
    if idx.dtype != torch.int32 or val.dtype != torch.float32 or idx.shape != val.shape \
            or not idx.is_contiguous() or not val.is_contiguous():
        raise ValueError("idx must be int32 and val float32, contiguous, same shape [T, k]")
    if idx.shape[1] != plan.code_len:
        raise ValueError(f"code length {idx.shape[1]} != plan's {plan.code_len}")
    y = torch.empty((T, plan.d), dtype=plan.torch_dtype, device=idx.device) if y is None else y
    ws = plan._stream_workspace(T, idx.device, stream) if workspace is None else workspace
    if r_out is not None and (r_out.dtype != torch.float32 or not r_out.is_contiguous()
                              or tuple(r_out.shape) != (T, plan.d)):
        raise ValueError(f"r_out must be a contiguous float32 tensor of shape [T, {plan.d}]")
    _check(plan._lib.dpb_decode(plan.handle, _ptr(idx), _ptr(val), T, _ptr(xnorm), _ptr(y), _ptr(r_out),
                                _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))
    return y


def forward(plan: Plan, x: torch.Tensor, mu=None, sigma=None, workspace=None, stream=None,
            r_out: Optional[torch.Tensor] = None):
    """dpb_forward (encode then decode). Returns (idx, val, xnorm, y)."""
    _rows(x, plan, "x")
    T, k, dev = x.shape[0], plan.code_len, x.device
    idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    val = torch.empty((T, k), dtype=torch.float32, device=dev)
    xnorm = torch.empty((T,), dtype=torch.float32, device=dev)
    y = torch.empty_like(x)
    if r_out is not None and (r_out.dtype != torch.float32 or not r_out.is_contiguous()
                              or tuple(r_out.shape) != (T, plan.d)):
        raise ValueError(f"r_out must be a contiguous float32 tensor of shape [T, {plan.d}]")
    ws = plan._stream_workspace(T, dev, stream) if workspace is None else workspace
    _check(plan._lib.dpb_forward(plan.handle, _ptr(x), T, _ptr(mu), _ptr(sigma), _ptr(idx), _ptr(val),
                                 _ptr(xnorm), _ptr(y), _ptr(r_out), _ptr(ws), ws.numel() * ws.element_size(),
                                 _stream(stream)))
    return idx, val, xnorm, y


def backward(plan: Plan, x: torch.Tensor, idx: torch.Tensor, val: torch.Tensor, grad_y: torch.Tensor,
             sigma=None, grad_x=None, grad_val=None, workspace=None, stream=None,
             r: Optional[torch.Tensor] = None):
    """dpb_backward. Returns (grad_x [T, d] plan dtype, grad_val fp32 [T, k]);
    ``r`` is the r_out of the decode of this code (optional)."""
    _rows(x, plan, "x")
    _rows(grad_y, plan, "grad_y")
    T = x.shape[0]
    grad_x = torch.empty_like(x) if grad_x is None else grad_x
    grad_val = torch.empty(idx.shape, dtype=torch.float32, device=x.device) if grad_val is None else grad_val
    ws = plan._stream_workspace(T, x.device, stream) if workspace is None else workspace
    if r is not None and (r.dtype != torch.float32 or not r.is_contiguous() or tuple(r.shape) != (T, plan.d)):
        raise ValueError(f"r must be a contiguous float32 tensor of shape [T, {plan.d}]")
    _check(plan._lib.dpb_backward(plan.handle, _ptr(x), _ptr(idx), _ptr(val), T, _ptr(sigma), _ptr(r),
                                  _ptr(grad_y), _ptr(grad_x), _ptr(grad_val), _ptr(ws),
                                  ws.numel() * ws.element_size(), _stream(stream)))
    return grad_x, grad_val


def stats_buffer(plan: Plan, device=None) -> torch.Tensor:
    """A zeroed moment-sum buffer fp64 [3, 2^N] (count, sum s, sum s^2)."""
    return torch.zeros((3, plan.n_features), dtype=torch.float64, device=device or "cuda")


def stats_accumulate(plan: Plan, x: torch.Tensor, sample: torch.Tensor, acc: torch.Tensor, mu=None,
                     sigma=None, workspace=None, stream=None):
    """dpb_stats_accumulate: adds the batch's moment sums to ``acc`` (level 0
    over every row of x, levels >= 1 over the rows in ``sample``)."""
    _rows(x, plan, "x")
    if sample.dtype != torch.int32 or not sample.is_contiguous() or sample.dim() != 1:
        raise ValueError("sample must be a contiguous 1-D int32 tensor of row numbers")
    if acc.dtype != torch.float64 or not acc.is_contiguous() or acc.numel() != 3 * plan.n_features:
        raise ValueError("acc must be a contiguous float64 tensor of 3 * 2^N entries (stats_buffer)")
    T = x.shape[0]
    ws = plan._stream_workspace(T, x.device, stream) if workspace is None else workspace
    _check(plan._lib.dpb_stats_accumulate(plan.handle, _ptr(x), T, _ptr(mu), _ptr(sigma),
                                          _ptr(sample) if sample.numel() else None, sample.numel(),
                                          _ptr(acc), _ptr(ws), ws.numel() * ws.element_size(),
                                          _stream(stream)))
    return acc


def stats_update(plan: Plan, acc: torch.Tensor, alpha: float, mu: torch.Tensor, sigma: torch.Tensor,
                 stream=None):
    """dpb_stats_update: one EMA step of (mu, sigma) in place; zeroes ``acc``."""
    if acc.dtype != torch.float64 or not acc.is_contiguous():
        raise ValueError("acc must be a contiguous float64 tensor")
    for name, t in (("mu", mu), ("sigma", sigma)):
        if t.dtype != torch.float32 or not t.is_contiguous() or t.numel() * 3 != acc.numel():
            raise ValueError(f"{name} must be a contiguous float32 tensor of 2^N entries")
    _check(plan._lib.dpb_stats_update(plan.handle, _ptr(acc), float(alpha), _ptr(mu), _ptr(sigma),
                                      _stream(stream)))
    return mu, sigma


def ema_step(accumulate, update, acc, group=None):
    """One standardisation step under data parallelism: each rank adds its
    own moment sums (``accumulate(acc)``), the sums are added up across the
    ranks of ``group`` (one all-reduce; skipped when torch.distributed is not
    initialised or the group has one rank), and every rank makes the same EMA
    step (``update(acc)``), so the tables stay identical everywhere."""
    accumulate(acc)
    import torch.distributed as dist
    if dist.is_available() and dist.is_initialized() and dist.get_world_size(group) > 1:
        dist.all_reduce(acc, op=dist.ReduceOp.SUM, group=group)
    update(acc)


def sample_rows(T: int, n: int, generator: Optional[torch.Generator] = None, device=None) -> torch.Tensor:
    """n distinct row numbers of [0, T) (all of them when T <= n), drawn
    uniformly by ``generator``: the sub-sample of levels >= 1."""
    n = min(n, T)
    rows = torch.randperm(T, generator=generator)[:n].to(torch.int32)
    return rows.to(device) if device is not None else rows


def stats_step(plan: Plan, x: torch.Tensor, mu: torch.Tensor, sigma: torch.Tensor, alpha: float,
               sample: torch.Tensor, acc: Optional[torch.Tensor] = None, workspace=None, stream=None,
               group=None):
    """The whole EMA update of one batch (§2.2 "Score Standardization"):
    moment sums on this rank, summed across ``group``, then the EMA step of
    mu and sigma in place."""
    acc = stats_buffer(plan, x.device) if acc is None else acc
    ema_step(lambda a: stats_accumulate(plan, x, sample, a, mu=mu, sigma=sigma, workspace=workspace,
                                        stream=stream),
             lambda a: stats_update(plan, a, alpha, mu, sigma, stream=stream), acc, group)
    return mu, sigma


def set_wait_limit(tries: int = -1):
    """dpb_debug_set_wait_limit: bound of the per-level encoder's main-loop
    mbarrier waits, and of the loss gradient's waits for other blocks, for the
    launches that follow (-1 restores the default)."""
    _check(load().dpb_debug_set_wait_limit(int(tries)))


def workspace_status(workspace: torch.Tensor, clear: bool = False, stream=None) -> int:
    """dpb_workspace_status: the sticky device status bits (0 = none)."""
    v = ctypes.c_int32()
    load().dpb_workspace_status(_ptr(workspace), int(clear), ctypes.byref(v), _stream(stream))
    return v.value


# ---- the training step around the bottleneck -------------------------------

STATUS_SLOTS, _GRAPH_SLOT = 256, 1
_slots: dict = {}  # (device, stream): number of the library's status word
_slots_lock = threading.Lock()
_captured: set = set()  # devices with calls in graphs


def _elsewhere(call, stream, device, args, kw):
    """Makes `call` on another stream or device than the current ones: outputs
    and workspaces are then allocated there, and the allocator is told that
    the tensors given are read there."""
    if device.type != "cuda":
        raise ValueError("tensors must be on a CUDA device")
    s = torch.cuda.current_stream(device) if stream is None else stream
    with torch.cuda.stream(s):
        out = call(*args, **kw)
    if stream is not None:
        for t in (*args, *kw.values()):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(s)
    return out


def _away(device, stream) -> bool:
    return stream is not None or device.index != torch.cuda.current_device()


def _raw_stream(device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _status_slot(device, stream: int) -> int:
    """The library's status word for calls made without a workspace: one for
    each (device, stream), and one for all calls captured into graphs, whose
    replays may run anywhere. The words outlive streams and graphs."""
    if torch._C._cuda_isCurrentStreamCapturing():
        _captured.add(device.index)
        return _GRAPH_SLOT
    slot = _slots.get((device.index, stream))
    if slot is None:
        with _slots_lock:
            used = sum(d == device.index for d, _ in _slots)
            slot = _slots.setdefault((device.index, stream), min(_GRAPH_SLOT + 1 + used, STATUS_SLOTS))
    return slot


def status(device=None, stream=None, clear: bool = True) -> int:
    """The DPB_DEV_* bits that the calls below, made without a workspace, left
    on ``stream`` (synchronises it), and those of such calls in graphs
    replayed so far on the device; cleared by default."""
    dev = torch.device(device or "cuda")
    s = stream if stream is not None else torch.cuda.current_stream(dev)
    index = dev.index if dev.index is not None else torch.cuda.current_device()
    lib, bits = load(), 0
    with torch.cuda.device(index):
        for slot in (_slots.get((index, s.cuda_stream)), _GRAPH_SLOT if index in _captured else None):
            if slot is not None:
                word, v = ctypes.c_void_p(), ctypes.c_int32()
                _check(lib.dpb_status_word(slot, word))
                rc = lib.dpb_workspace_status(word, int(clear), v, _stream(s))
                _check(0 if rc == 6 else rc)  # 6: there are bits
                bits |= v.value
    return bits


def _head_rows(t: torch.Tensor, name: str, dtype, shape, device):
    """(address, token stride, head stride) of a [tokens, heads, dim] tensor whose last dimension is dense."""
    st = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {list(shape)} on {device}, "
                         f"got {t.dtype} {list(t.shape)} on {t.device}")
    if st[2] != 1 and shape[2] > 1:
        raise ValueError(f"the last dimension of {name} must be dense")
    return t.data_ptr(), st[0], st[1]


def _dense(t: Optional[torch.Tensor], name: str, dtype, numel: int, device):
    """Address of a contiguous tensor of `numel` values (None: None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device or not t.is_contiguous() or t.numel() != numel:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {numel} values on {device}")
    return t.data_ptr()


def _space(t: Optional[torch.Tensor], device):
    """(address, bytes) of a workspace (None: none): memory of the rows' own device, without gaps or repeats."""
    if t is None:
        return None, 0
    if t.device != device or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}, got one on {t.device} with strides {t.stride()}")
    return t.data_ptr(), t.nbytes


def rope_tables(positions: int, rot_dim: int, base: float = 10000.0, scaling: Optional[str] = None,
                factor: float = 1.0, original: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0,
                device=None):
    """(cos, sin) fp32 [positions, rot_dim / 2] for qk_norm_rope, from angles in
    64 bits: position x base^(-2 i / rot_dim). For contexts ``factor`` times
    longer than trained on, ``scaling``: "linear" (positions divided by factor),
    "ntk" (a larger base: base x factor^(R / (R - 2))), or "yarn" (pairs that
    turn fewer than beta_slow times in ``original`` positions are divided by
    factor, those above beta_fast turns are kept, a ramp between, and both
    tables are multiplied by 0.1 ln(factor) + 1)."""
    import math
    if rot_dim <= 0 or rot_dim % 2 or positions < 1:
        raise ValueError("rot_dim must be even and positive, positions at least 1")
    if scaling not in (None, "linear", "ntk", "yarn") or (scaling and factor < 1.0):
        raise ValueError("scaling must be None, 'linear', 'ntk' or 'yarn', with factor >= 1")
    if scaling == "ntk":
        if rot_dim == 2:
            raise ValueError("'ntk' needs rot_dim above 2")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    freq = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    gain = 1.0
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "yarn":
        if original < 1:
            raise ValueError("'yarn' needs original, the trained context")
        turns = original * freq / (2 * math.pi)
        keep = ((turns - beta_slow) / (beta_fast - beta_slow)).clamp(0.0, 1.0)
        freq = freq * keep + freq / factor * (1 - keep)
        gain = 0.1 * math.log(factor) + 1.0
    ang = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    cos, sin = (ang.cos() * gain).float(), (ang.sin() * gain).float()
    return cos.to(device or "cuda"), sin.to(device or "cuda")


def _rope_config(q, k, weight_q, weight_k, cos, sin, positions, eps, interleaved, normalise, slot):
    """Writes the config; addresses of the weights, tables and positions."""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q and k must be [tokens, heads, dim]")
    T, hq, D = q.shape
    dt, dev = q.dtype, q.device
    if k.shape[0] != T or k.shape[2] != D or k.dtype is not dt:
        raise ValueError("q and k must have the same tokens, dim and dtype")
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise ValueError(f"q and k must be float32 or bfloat16, got {dt}")
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin must both be given or both be None")
    rot, rows = 0, 0
    if cos is not None:
        if cos.dim() != 2 or cos.shape != sin.shape:
            raise ValueError("cos and sin must be [positions, rot_dim / 2] of the same shape")
        rows, rot = cos.shape[0], 2 * cos.shape[1]
    at = (_dense(weight_q, "weight_q", dt, D, dev), _dense(weight_k, "weight_k", dt, D, dev),
          _dense(cos, "cos", torch.float32, rows * rot // 2, dev), _dense(sin, "sin", torch.float32, rows * rot // 2, dev),
          _dense(positions, "positions", torch.int32, T, dev))
    _ROPE.pack_into(_arguments.buf, 0, T, hq, k.shape[1], D, rot, bool(interleaved), bool(normalise), rows,
                    BF16 if dt is torch.bfloat16 else F32, eps, slot)
    return at


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, weight_q=None, weight_k=None, cos=None, sin=None, positions=None,
                 eps: float = 1e-6, interleaved: bool = False, normalise: bool = True, q_out=None, k_out=None,
                 workspace=None, stream=None):
    """dpb_qk_norm_rope. q [T, Hq, D], k [T, Hk, D], fp32 or bf16 (views of one
    packed projection are fine); cos, sin from rope_tables() (None: no
    rotation); positions int32 [T] (None: 0, 1, ...). Returns (q, k) normalised
    and rotated."""
    dev = q.device
    if _away(dev, stream):
        return _elsewhere(qk_norm_rope, stream, dev, (q, k, weight_q, weight_k, cos, sin, positions, eps, interleaved,
                                                      normalise, q_out, k_out, workspace), {})
    s = _raw_stream(dev)
    at = _rope_config(q, k, weight_q, weight_k, cos, sin, positions, eps, interleaved, normalise,
                      _status_slot(dev, s) if workspace is None else 0)
    dt, sq, sk, a = q.dtype, q.shape, k.shape, _arguments
    q_out = torch.empty(sq, dtype=dt, device=dev) if q_out is None else q_out
    k_out = torch.empty(sk, dtype=dt, device=dev) if k_out is None else k_out
    ws, ws_bytes = _space(workspace, dev)
    _ROWS[4].pack_into(a.buf, 64, *_head_rows(q, "q", dt, sq, dev), *_head_rows(k, "k", dt, sk, dev),
                       *_head_rows(q_out, "q_out", dt, sq, dev), *_head_rows(k_out, "k_out", dt, sk, dev))
    h = a.rows
    _check(load().dpb_qk_norm_rope(a.at, h, h + 24, *at, h + 48, h + 72, ws, ws_bytes, s))
    return q_out, k_out


def qk_norm_rope_backward(q: torch.Tensor, k: torch.Tensor, grad_q_out: torch.Tensor, grad_k_out: torch.Tensor,
                          weight_q=None, weight_k=None, cos=None, sin=None, positions=None, eps: float = 1e-6,
                          interleaved: bool = False, normalise: bool = True, weight_grads: bool = True, grad_q=None,
                          grad_k=None, workspace=None, stream=None):
    """dpb_qk_norm_rope_backward. Returns (grad_q, grad_k, grad_weight_q,
    grad_weight_k): the last two fp32 [D], or None without ``normalise`` or
    ``weight_grads``."""
    dev = q.device
    if _away(dev, stream):
        return _elsewhere(qk_norm_rope_backward, stream, dev,
                          (q, k, grad_q_out, grad_k_out, weight_q, weight_k, cos, sin, positions, eps, interleaved,
                           normalise, weight_grads, grad_q, grad_k, workspace), {})
    s = _raw_stream(dev)
    at = _rope_config(q, k, weight_q, weight_k, cos, sin, positions, eps, interleaved, normalise,
                      _status_slot(dev, s) if workspace is None else 0)
    lib, dt, sq, sk, a = load(), q.dtype, q.shape, k.shape, _arguments
    grad_q = torch.empty(sq, dtype=dt, device=dev) if grad_q is None else grad_q
    grad_k = torch.empty(sk, dtype=dt, device=dev) if grad_k is None else grad_k
    D = sq[2]
    gw = torch.empty((2, D), dtype=torch.float32, device=dev) if normalise and weight_grads else None
    gp = None if gw is None else gw.data_ptr()
    if workspace is None:
        n = ctypes.c_size_t()
        _check(lib.dpb_rope_workspace_size(a.at, n))
        workspace = torch.empty(n.value, dtype=torch.uint8, device=dev)  # scratch of this call
    _ROWS[6].pack_into(a.buf, 64, *_head_rows(q, "q", dt, sq, dev), *_head_rows(k, "k", dt, sk, dev),
                       *_head_rows(grad_q_out, "grad_q_out", dt, sq, dev),
                       *_head_rows(grad_k_out, "grad_k_out", dt, sk, dev),
                       *_head_rows(grad_q, "grad_q", dt, sq, dev), *_head_rows(grad_k, "grad_k", dt, sk, dev))
    h = a.rows
    _check(lib.dpb_qk_norm_rope_backward(a.at, h, h + 24, h + 48, h + 72, *at, h + 96, h + 120, gp,
                                         None if gp is None else gp + 4 * D, *_space(workspace, dev), s))
    return (grad_q, grad_k) + ((None, None) if gw is None else (gw[0], gw[1]))


def _attention_config(q, k, v, cu_q, cu_k, max_q, max_k, causal, scale, slot):
    """Writes the config; addresses of the offsets."""
    if q.dim() != 3 or k.dim() != 3 or q.dtype is not torch.bfloat16:
        raise ValueError(f"q, k and v must be bfloat16 tensors [tokens, heads, dim], got {q.dtype} {list(q.shape)}")
    Tq, Hq, D = q.shape
    Tk, Hk, _ = k.shape
    if cu_k is None and cu_q is not None:
        if Tq != Tk:
            raise ValueError("cu_k is needed: q and k have different token counts")
        cu_k, max_k = cu_q, max_q
    if (cu_q is None) != (cu_k is None):
        raise ValueError("cu_q and cu_k must both be given or both be None")
    seqs = 1
    if cu_q is not None:
        seqs = cu_q.numel() - 1
        if seqs < 0:
            raise ValueError("cu_q must have one entry more than there are sequences")
    at = (_dense(cu_q, "cu_q", torch.int32, seqs + 1, q.device), _dense(cu_k, "cu_k", torch.int32, seqs + 1, q.device))
    _ATTENTION.pack_into(_arguments.buf, 0, Tq, Tk, seqs, Tq if max_q is None or max_q > Tq else max_q,
                         Tk if max_k is None or max_k > Tk else max_k, Hq, Hk, D, bool(causal), BF16,
                         D ** -0.5 if scale is None else scale, slot)
    return at


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q=None, cu_k=None,
                      max_q: Optional[int] = None, max_k: Optional[int] = None, causal: bool = True,
                      scale: Optional[float] = None, out=None, lse=None, workspace=None, stream=None):
    """dpb_attention_forward. q [Tq, Hq, D], k and v [Tk, Hkv, D] bf16 (views
    of one packed projection are fine); cu_q, cu_k int32 [sequences + 1] token
    offsets (None: one sequence; cu_k None: as cu_q), max_q, max_k the longest
    sequences' lengths (None: the token count, which only costs empty blocks);
    scale defaults to D^-1/2. Returns (o [Tq, Hq, D], lse fp32 [Hq, Tq]); rows
    that the offsets leave out (padding) have o = 0 and lse = -inf."""
    dev = q.device
    if _away(dev, stream):
        return _elsewhere(attention_forward, stream, dev,
                          (q, k, v, cu_q, cu_k, max_q, max_k, causal, scale, out, lse, workspace), {})
    s = _raw_stream(dev)
    at = _attention_config(q, k, v, cu_q, cu_k, max_q, max_k, causal, scale, _status_slot(dev, s) if workspace is None else 0)
    dt, sq, a = torch.bfloat16, q.shape, _arguments
    sk = k.shape if k.shape[2] == sq[2] else (*k.shape[:2], sq[2])
    if out is None:
        out = torch.empty(sq, dtype=dt, device=dev)
    if lse is None:
        lse = torch.empty((sq[1], sq[0]), dtype=torch.float32, device=dev)
    ws, ws_bytes = _space(workspace, dev)
    _ROWS[4].pack_into(a.buf, 64, *_head_rows(q, "q", dt, sq, dev), *_head_rows(k, "k", dt, sk, dev),
                       *_head_rows(v, "v", dt, sk, dev), *_head_rows(out, "out", dt, sq, dev))
    h = a.rows
    _check(load().dpb_attention_forward(a.at, h, h + 24, h + 48, *at, h + 72,
                                        _dense(lse, "lse", torch.float32, sq[0] * sq[1], dev), ws, ws_bytes, s))
    return out, lse


def attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       grad_o: torch.Tensor, cu_q=None, cu_k=None, max_q: Optional[int] = None,
                       max_k: Optional[int] = None, causal: bool = True, scale: Optional[float] = None, grad_q=None,
                       grad_k=None, grad_v=None, workspace=None, stream=None):
    """dpb_attention_backward with the forward's inputs, its o and lse, and the
    gradient of o. Returns (grad_q, grad_k, grad_v); 0 in rows that the offsets
    leave out."""
    dev = q.device
    if _away(dev, stream):
        return _elsewhere(attention_backward, stream, dev,
                          (q, k, v, o, lse, grad_o, cu_q, cu_k, max_q, max_k, causal, scale, grad_q, grad_k, grad_v,
                           workspace), {})
    s = _raw_stream(dev)
    at = _attention_config(q, k, v, cu_q, cu_k, max_q, max_k, causal, scale, _status_slot(dev, s) if workspace is None else 0)
    lib, dt, sq, a = load(), torch.bfloat16, q.shape, _arguments
    sk = k.shape if k.shape[2] == sq[2] else (*k.shape[:2], sq[2])
    grad_q = torch.empty(sq, dtype=dt, device=dev) if grad_q is None else grad_q
    grad_k = torch.empty(sk, dtype=dt, device=dev) if grad_k is None else grad_k
    grad_v = torch.empty(sk, dtype=dt, device=dev) if grad_v is None else grad_v
    if workspace is None:
        n = ctypes.c_size_t()
        _check(lib.dpb_attention_workspace_size(a.at, n))
        workspace = torch.empty(n.value, dtype=torch.uint8, device=dev)  # scratch of this call
    _ROWS[8].pack_into(a.buf, 64, *_head_rows(q, "q", dt, sq, dev), *_head_rows(k, "k", dt, sk, dev),
                       *_head_rows(v, "v", dt, sk, dev), *_head_rows(o, "o", dt, sq, dev),
                       *_head_rows(grad_o, "grad_o", dt, sq, dev), *_head_rows(grad_q, "grad_q", dt, sq, dev),
                       *_head_rows(grad_k, "grad_k", dt, sk, dev), *_head_rows(grad_v, "grad_v", dt, sk, dev))
    h = a.rows
    _check(lib.dpb_attention_backward(a.at, h, h + 24, h + 48, h + 72,
                                      _dense(lse, "lse", torch.float32, sq[0] * sq[1], dev), h + 96, *at, h + 120, h + 144,
                                      h + 168, *_space(workspace, dev), s))
    return grad_q, grad_k, grad_v


class AdamWGroup:
    """What dpb_adamw_step takes of a list of parameters and their states: the
    states are one flat tensor each of the parameter's size, float32, or
    float8_e4m3fn codes with a float32 scale for each STATE_BLOCK values
    (ceil(n / STATE_BLOCK) of them). The tensors are held; a parameter's
    ``data`` may be rebound (its address is read at every step), the states'
    may not."""

    def __init__(self, params, exp_avg, exp_avg_sq, exp_avg_scale=None, exp_avg_sq_scale=None):
        import numpy as np
        self.params, self.exp_avg, self.exp_avg_sq = list(params), list(exp_avg), list(exp_avg_sq)
        self.scales = (None if exp_avg_scale is None else list(exp_avg_scale),
                       None if exp_avg_sq_scale is None else list(exp_avg_sq_scale))
        if not self.params:
            raise ValueError("no parameters")
        p0 = self.params[0]
        if p0.dtype not in (torch.float32, torch.bfloat16) or not p0.is_cuda:
            raise ValueError("parameters must be float32 or bfloat16 CUDA tensors")
        self.dtype, self.device = p0.dtype, p0.device
        self.state_bits = 32 if exp_avg_scale is None and exp_avg_sq_scale is None else 8
        sd = torch.float32 if self.state_bits == 32 else torch.float8_e4m3fn
        kinds = [(self.exp_avg, "exp_avg"), (self.exp_avg_sq, "exp_avg_sq")]
        if self.state_bits == 8:
            if None in self.scales:
                raise ValueError("8-bit states need both scales")
            kinds += [(self.scales[0], "exp_avg_scale"), (self.scales[1], "exp_avg_sq_scale")]
        for ts, name in kinds:
            if len(ts) != len(self.params):
                raise ValueError(f"{len(ts)} tensors of {name} for {len(self.params)} parameters")
        for i, p in enumerate(self.params):
            if p.dtype != self.dtype or p.device != self.device or not p.is_contiguous():
                raise ValueError(f"parameter {i} must be a contiguous {self.dtype} tensor on {self.device}")
            for ts, name in kinds:
                scale = name.endswith("scale")
                n = -(-p.numel() // STATE_BLOCK) if scale else p.numel()
                _dense(ts[i], f"{name}[{i}]", torch.float32 if scale else sd, n, self.device)
        self._numel = [p.numel() for p in self.params]
        self._table = np.zeros((len(self.params), 7), dtype=np.int64)  # rows of dpb_adamw_tensor
        for col, ts in enumerate((self.params, None, self.exp_avg, self.exp_avg_sq, *self.scales)):
            if ts is not None:
                self._table[:, col] = [x.data_ptr() for x in ts]
        self._table[:, 6] = self._numel
        self._table_at, self._last = self._table.ctypes.data, (self._table[:, 0].tolist(), None)

    def __reduce__(self):
        # a copy is made from its own tensors: the table holds addresses
        return AdamWGroup, (self.params, self.exp_avg, self.exp_avg_sq, *self.scales)

    def step(self, grads, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0, step: int = 1,
             seed: int = 0, grad_scale: Optional[torch.Tensor] = None, stream=None):
        """dpb_adamw_step: one step of every parameter that has a gradient (None
        leaves it as it is). ``grad_scale``: a float32 tensor of one value that
        multiplies the gradients; where it is not finite nothing changes. All
        numbers are read now: a CUDA graph of this call repeats this step."""
        dt, dev = self.dtype, self.device
        if _away(dev, stream):
            _elsewhere(self.step, stream, dev, (grads, lr, betas, eps, weight_decay, step, seed, grad_scale), {})
            if stream is not None:
                for ts in (grads, self.params, self.exp_avg, self.exp_avg_sq, *(x or () for x in self.scales)):
                    for x in ts:
                        if x is not None:
                            x.record_stream(stream)
            return
        t = self._table
        if len(grads) != len(self.params):
            raise ValueError(f"{len(grads)} gradients for {len(self.params)} parameters")
        at, left = [], False
        for g, n in zip(grads, self._numel):
            if g is None:
                left = True
                at.append(0)
            elif g.dtype is not dt or g.numel() != n or not g.is_contiguous() or g.device != dev:
                raise ValueError(f"gradient {len(at)} must be a contiguous {dt} tensor of {n} values on {dev}")
            else:
                at.append(g.data_ptr())
        ps = [p.data_ptr() for p in self.params]
        if ps != self._last[0]:
            for i in (t[:, 0] != ps).nonzero()[0]:  # rebound since the last step
                p = self.params[i]
                if p.dtype is not dt or p.numel() != self._numel[i] or not p.is_contiguous() or p.device != dev:
                    raise ValueError(f"parameter {i} must be a contiguous {dt} tensor of {self._numel[i]} values on {dev}")
            t[:, 0] = ps
        if at != self._last[1]:
            t[:, 1] = at
            t[:, 6] = [n if g else 0 for g, n in zip(at, self._numel)] if left else self._numel
        self._last = (ps, at)
        c = AdamWConfig(lr, betas[0], betas[1], eps, weight_decay, step, seed & (2**64 - 1),
                        _dense(grad_scale, "grad_scale", torch.float32, 1, dev), F32 if dt is torch.float32 else BF16,
                        self.state_bits)
        _check(load().dpb_adamw_step(c, self._table_at, len(ps), _raw_stream(dev)))


# ---- both ends of the model, and the stream between them --------------------


def _plain_rows(t: torch.Tensor, name: str, dtype, shape, device):
    """(address, row stride) of a [rows, dim] tensor whose last dimension is dense."""
    st = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {list(shape)} on {device}, "
                         f"got {t.dtype} {list(t.shape)} on {t.device}")
    if st[1] != 1 and shape[1] > 1:
        raise ValueError(f"the last dimension of {name} must be dense")
    return t.data_ptr(), st[0]


def _indices(t: torch.Tensor, name: str, n: int, device):
    """(address, bytes of an index) of n int32 or int64 indices."""
    if t.dtype not in (torch.int64, torch.int32) or t.device != device or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{name} must be a contiguous int32 or int64 tensor of {n} values on {device}")
    return t.data_ptr(), t.element_size()


def _loss_config(hidden, weight, targets, ignore_index, grad_stride, slot):
    """Writes the config; the targets' address."""
    if hidden.dim() != 2 or weight.dim() != 2 or hidden.shape[1] != weight.shape[1]:
        raise ValueError(f"hidden must be [tokens, dim] and weight [vocab, dim], got {list(hidden.shape)} and "
                         f"{list(weight.shape)}")
    if hidden.dtype is not torch.bfloat16:
        raise ValueError(f"hidden and weight must be bfloat16, got {hidden.dtype}")
    T, d = hidden.shape
    at, size = _indices(targets, "targets", T, hidden.device)
    _LOSS.pack_into(_arguments.buf, 0, T, weight.shape[0], d, ignore_index, size, BF16, grad_stride, slot)
    return at


def _loss_workspace(backward: int, device):
    n = ctypes.c_size_t()
    _check(load().dpb_linear_cross_entropy_workspace_size(_arguments.at, backward, n))
    return torch.empty(n.value, dtype=torch.uint8, device=device)  # scratch of this call


def linear_cross_entropy_forward(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                                 ignore_index: int = -100, loss=None, lse=None, want_counted: bool = False,
                                 workspace=None, stream=None):
    """dpb_linear_cross_entropy_forward. hidden [T, d], weight [V, d] bf16,
    targets int32 or int64 [T]. Returns (loss, lse), fp32 [T]: the cross entropy
    of each token's scores hidden weight^T and the log of the sum of their
    exponentials, both 0 where the target is ``ignore_index``; with
    ``want_counted`` also the number of the other tokens, int32 [1]."""
    dev = hidden.device
    if _away(dev, stream):
        return _elsewhere(linear_cross_entropy_forward, stream, dev,
                          (hidden, weight, targets, ignore_index, loss, lse, want_counted, workspace), {})
    s = _raw_stream(dev)
    at = _loss_config(hidden, weight, targets, ignore_index, 0, _status_slot(dev, s) if workspace is None else 0)
    a, T, bf = _arguments, hidden.shape[0], torch.bfloat16
    loss = torch.empty(T, dtype=torch.float32, device=dev) if loss is None else loss
    lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else lse
    counted = torch.empty(1, dtype=torch.int32, device=dev) if want_counted else None
    if workspace is None:
        workspace = _loss_workspace(0, dev)
    _PLAIN_ROWS[2].pack_into(a.buf, 64, *_plain_rows(hidden, "hidden", bf, hidden.shape, dev),
                             *_plain_rows(weight, "weight", bf, weight.shape, dev))
    h = a.rows
    _check(load().dpb_linear_cross_entropy_forward(a.at, h, h + 16, at, _dense(loss, "loss", torch.float32, T, dev),
                                                   _dense(lse, "lse", torch.float32, T, dev),
                                                   None if counted is None else counted.data_ptr(), *_space(workspace, dev), s))
    return (loss, lse, counted) if want_counted else (loss, lse)


def linear_cross_entropy_backward(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                                  grad_loss: torch.Tensor, ignore_index: int = -100, want_hidden: bool = True,
                                  want_weight: bool = True, grad_hidden=None, grad_weight=None, workspace=None,
                                  stream=None):
    """dpb_linear_cross_entropy_backward with the forward's inputs and lse, and
    grad_loss = dL/dloss, fp32 [T] (one value expanded to [T] is read as one).
    Returns (grad_hidden [T, d], grad_weight [V, d]); None for one that is not
    wanted."""
    dev = hidden.device
    if _away(dev, stream):
        return _elsewhere(linear_cross_entropy_backward, stream, dev,
                          (hidden, weight, targets, lse, grad_loss, ignore_index, want_hidden, want_weight, grad_hidden,
                           grad_weight, workspace), {})
    s = _raw_stream(dev)
    T, bf = hidden.shape[0], torch.bfloat16
    if grad_loss.dtype is not torch.float32 or grad_loss.shape != (T,) or grad_loss.device != dev:
        raise ValueError(f"grad_loss must be a float32 tensor of shape [{T}] on {dev}")
    step = grad_loss.stride(0) if T > 1 else 0
    if step not in (0, 1):
        raise ValueError("grad_loss must be contiguous or one value expanded")
    at = _loss_config(hidden, weight, targets, ignore_index, step, _status_slot(dev, s) if workspace is None else 0)
    a = _arguments
    if workspace is None:
        workspace = _loss_workspace(1, dev)
    if want_hidden and grad_hidden is None:
        grad_hidden = torch.empty(hidden.shape, dtype=bf, device=dev)
    if want_weight and grad_weight is None:
        grad_weight = torch.empty(weight.shape, dtype=bf, device=dev)
    _PLAIN_ROWS[4].pack_into(a.buf, 64, *_plain_rows(hidden, "hidden", bf, hidden.shape, dev),
                             *_plain_rows(weight, "weight", bf, weight.shape, dev),
                             *(_plain_rows(grad_hidden, "grad_hidden", bf, hidden.shape, dev) if want_hidden else (0, 0)),
                             *(_plain_rows(grad_weight, "grad_weight", bf, weight.shape, dev) if want_weight else (0, 0)))
    h = a.rows
    _check(load().dpb_linear_cross_entropy_backward(a.at, h, h + 16, at, _dense(lse, "lse", torch.float32, T, dev),
                                                    grad_loss.data_ptr(), h + 32 if want_hidden else None,
                                                    h + 48 if want_weight else None, *_space(workspace, dev), s))
    return grad_hidden if want_hidden else None, grad_weight if want_weight else None


def _kind(dtype, name: str) -> int:
    if dtype is not torch.float32 and dtype is not torch.bfloat16:
        raise ValueError(f"{name} must be float32 or bfloat16, got {dtype}")
    return BF16 if dtype is torch.bfloat16 else F32


def embedding(weight: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out=None, workspace=None, stream=None):
    """dpb_embedding. weight [V, d] fp32 or bf16, ids int32 or int64 [T].
    Returns scale x weight[ids], [T, d]; an id outside [0, V) gives a row of 0
    and sets DEV_BAD_INDEX (see status())."""
    dev = weight.device
    if _away(dev, stream):
        return _elsewhere(embedding, stream, dev, (weight, ids, scale, out, workspace), {})
    s = _raw_stream(dev)
    if weight.dim() != 2 or ids.dim() != 1:
        raise ValueError(f"weight must be [vocab, dim] and ids [tokens], got {list(weight.shape)} and {list(ids.shape)}")
    dt, (V, d), T, a = weight.dtype, weight.shape, ids.shape[0], _arguments
    kind = _kind(dt, "weight")
    at, size = _indices(ids, "ids", T, dev)
    out = torch.empty((T, d), dtype=dt, device=dev) if out is None else out
    ws, ws_bytes = _space(workspace, dev)
    _EMBEDDING.pack_into(a.buf, 0, T, V, d, size, kind, scale, _status_slot(dev, s) if workspace is None else 0)
    _PLAIN_ROWS[2].pack_into(a.buf, 64, *_plain_rows(weight, "weight", dt, weight.shape, dev),
                             *_plain_rows(out, "out", dt, (T, d), dev))
    _check(load().dpb_embedding(a.at, a.rows, at, a.rows + 16, ws, ws_bytes, s))
    return out


def embedding_backward(grad_out: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0, grad_weight=None,
                       workspace=None, stream=None):
    """dpb_embedding_backward. grad_out [T, d], ids [T]. Returns the gradient of
    the weight [vocab, d] in full, of grad_out's type."""
    dev = grad_out.device
    if _away(dev, stream):
        return _elsewhere(embedding_backward, stream, dev, (grad_out, ids, vocab, scale, grad_weight, workspace), {})
    s = _raw_stream(dev)
    if grad_out.dim() != 2 or ids.dim() != 1:
        raise ValueError(f"grad_out must be [tokens, dim] and ids [tokens], got {list(grad_out.shape)} and {list(ids.shape)}")
    dt, (T, d), a, lib = grad_out.dtype, grad_out.shape, _arguments, load()
    kind = _kind(dt, "grad_out")
    at, size = _indices(ids, "ids", T, dev)
    _EMBEDDING.pack_into(a.buf, 0, T, vocab, d, size, kind, scale, _status_slot(dev, s) if workspace is None else 0)
    if workspace is None:
        n = ctypes.c_size_t()
        _check(lib.dpb_embedding_workspace_size(a.at, n))
        workspace = torch.empty(n.value, dtype=torch.uint8, device=dev)  # scratch of this call
    grad_weight = torch.empty((vocab, d), dtype=dt, device=dev) if grad_weight is None else grad_weight
    _PLAIN_ROWS[2].pack_into(a.buf, 64, *_plain_rows(grad_out, "grad_out", dt, (T, d), dev),
                             *_plain_rows(grad_weight, "grad_weight", dt, (vocab, d), dev))
    _check(lib.dpb_embedding_backward(a.at, a.rows, at, a.rows + 16, *_space(workspace, dev), s))
    return grad_weight


def add_norm(x: torch.Tensor, delta=None, weight=None, eps: float = 1e-6, out=None, total=None, stream=None):
    """dpb_add_norm. x and delta [T, d] fp32 or bf16, weight [d]. Returns
    (y, total): total = x + delta rounded to the rows' type (x itself without
    delta), y = weight x total / sqrt(mean total^2 + eps)."""
    dev = x.device
    if _away(dev, stream):
        return _elsewhere(add_norm, stream, dev, (x, delta, weight, eps, out, total), {})
    s = _raw_stream(dev)
    if x.dim() != 2:
        raise ValueError(f"x must be [tokens, dim], got {list(x.shape)}")
    dt, sh, a = x.dtype, x.shape, _arguments
    kind = _kind(dt, "x")
    out = torch.empty(sh, dtype=dt, device=dev) if out is None else out
    if delta is not None and total is None:
        total = torch.empty(sh, dtype=dt, device=dev)
    _NORM.pack_into(a.buf, 0, sh[0], sh[1], kind, eps, 0)
    _PLAIN_ROWS[4].pack_into(a.buf, 64, *_plain_rows(x, "x", dt, sh, dev),
                             *((0, 0) if delta is None else _plain_rows(delta, "delta", dt, sh, dev)),
                             *_plain_rows(out, "out", dt, sh, dev),
                             *((0, 0) if total is None else _plain_rows(total, "total", dt, sh, dev)))
    h = a.rows
    _check(load().dpb_add_norm(a.at, h, None if delta is None else h + 16, _dense(weight, "weight", dt, sh[1], dev), h + 32,
                               None if total is None else h + 48, s))
    return out, x if total is None else total


def add_norm_backward(total: torch.Tensor, grad_out: torch.Tensor, grad_total=None, weight=None, eps: float = 1e-6,
                      weight_grad: bool = True, grad_x=None, workspace=None, stream=None):
    """dpb_add_norm_backward with the forward's total, the gradient of y and that
    of total (None: none). Returns (grad_x [T, d], which is delta's gradient
    too, grad_weight fp32 [d] or None without ``weight_grad``)."""
    dev = total.device
    if _away(dev, stream):
        return _elsewhere(add_norm_backward, stream, dev,
                          (total, grad_out, grad_total, weight, eps, weight_grad, grad_x, workspace), {})
    s = _raw_stream(dev)
    if total.dim() != 2:
        raise ValueError(f"total must be [tokens, dim], got {list(total.shape)}")
    dt, sh, a, lib = total.dtype, total.shape, _arguments, load()
    kind = _kind(dt, "total")
    _NORM.pack_into(a.buf, 0, sh[0], sh[1], kind, eps, 0)
    grad_x = torch.empty(sh, dtype=dt, device=dev) if grad_x is None else grad_x
    gw = torch.empty(sh[1], dtype=torch.float32, device=dev) if weight_grad else None
    if weight_grad and workspace is None:
        n = ctypes.c_size_t()
        _check(lib.dpb_norm_workspace_size(a.at, n))
        workspace = torch.empty(n.value, dtype=torch.uint8, device=dev)  # scratch of this call
    ws, ws_bytes = _space(workspace, dev)
    _PLAIN_ROWS[4].pack_into(a.buf, 64, *_plain_rows(total, "total", dt, sh, dev),
                             *_plain_rows(grad_out, "grad_out", dt, sh, dev),
                             *((0, 0) if grad_total is None else _plain_rows(grad_total, "grad_total", dt, sh, dev)),
                             *_plain_rows(grad_x, "grad_x", dt, sh, dev))
    h = a.rows
    _check(lib.dpb_add_norm_backward(a.at, h, h + 16, None if grad_total is None else h + 32,
                                     _dense(weight, "weight", dt, sh[1], dev), h + 48,
                                     None if gw is None else gw.data_ptr(), ws, ws_bytes, s))
    return grad_x, gw
