"""ctypes binding of libwdc.so (include/wdc.h): argument marshalling only.

Every step of the rollout runs in the library's HIP kernels; PyTorch supplies
device memory (``torch.empty`` on the GPU) and the current stream. There is no
Python or CPU fallback: a missing library raises at load time.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libwdc.so")

WDC_F32, WDC_BF16 = 0, 1
MODE_RISK, MODE_FORCED, MODE_ALL_EXACT, MODE_PERIODIC = 0, 1, 2, 3
SURROGATE_LIFTED, SURROGATE_SECANT = 0, 1
OBS_KERNEL, OBS_LINEAR = 0, 1
PRE_DECISION, POST_EXACT, POST_SURROGATE = 0, 1, 2
MAX_BANK = 8
# kernel timing classes, in the order of the WDC_T_* constants
TIMING_CLASSES = ("attention", "gemm", "stats", "observe", "exact_post", "psi", "norm")
STATUS = {0: "OK", 1: "E_ARG", 2: "E_SHAPE", 3: "E_DTYPE", 4: "E_ALIGN", 5: "E_WORKSPACE", 6: "E_STATE",
          7: "E_HIP", 8: "E_NONFINITE", 9: "E_UNSUPPORTED"}


class ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "dtype", "hidden", "heads", "head_dim", "mlp_ratio", "n_seq", "n_dual", "n_single", "cond_dim", "cam_dim",
        "text_tokens", "text_dim", "lat_c", "lat_f", "lat_h", "lat_w", "patch_t", "patch_h", "patch_w",
        "rope_t", "rope_h", "rope_w", "qk_norm", "max_batch")]


def desc_from_config(cfg, max_batch: int = 1) -> ModelDesc:
    """Model descriptor from any object with the workload fields (name, dtype, hidden, ...)."""
    d = ModelDesc()
    d.dtype = WDC_BF16 if cfg.dtype == "bf16" else WDC_F32
    d.hidden, d.heads, d.head_dim, d.mlp_ratio = cfg.hidden, cfg.heads, cfg.head_dim, cfg.mlp_ratio
    d.n_seq, d.n_dual, d.n_single = cfg.n_seq, cfg.n_dual, cfg.n_single
    d.cond_dim, d.cam_dim, d.text_tokens, d.text_dim = cfg.cond_dim, cfg.cam_dim, cfg.text_tokens, cfg.text_dim
    d.lat_c, d.lat_f, d.lat_h, d.lat_w = cfg.latent
    d.patch_t, d.patch_h, d.patch_w = cfg.patch
    d.rope_t, d.rope_h, d.rope_w = cfg.rope
    d.qk_norm = int(cfg.qk_norm)
    d.max_batch = max_batch
    return d


class Params(C.Structure):
    _fields_ = [("bank_capacity", C.c_int32), ("age_max", C.c_int32), ("n_min", C.c_int32), ("k_init", C.c_int32),
                ("k_ref", C.c_int32)] + [(n, C.c_double) for n in (
                    "theta_sim", "theta_q", "tau_in", "tau_obs", "gamma_q", "alpha_min", "alpha_max", "eps", "eps_nu",
                    "w_z", "w_age", "w_phase", "w_cam", "w_depth", "eta0", "beta_d", "eta_min", "eta_max",
                    "a_cam", "a_depth", "a_phase", "lam", "r0", "tau_risk")] + [(n, C.c_int32) for n in (
                    "period", "surrogate", "observation", "lift_condition", "impact_weight", "calibrate",
                    "support_constraint", "pad_")]


class StepLog(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("k", "exact", "bank", "support", "finite", "available", "slot", "pad_")] + [
        ("t", C.c_double), ("alpha", C.c_double), ("pi", C.c_double * MAX_BANK), ("kappa", C.c_double * MAX_BANK),
        ("sims_in", C.c_double * MAX_BANK)] + [(n, C.c_double) for n in (
            "d_z", "d_age", "d_phase", "p", "d_hat", "w", "r_cand", "margin", "sim_margin", "d_cf", "eta", "R")]

    def as_dict(self) -> dict:
        # one unpack of the record: reading it field by field through ctypes took 9.5 us, more than a kernel
        v = _STEP_LOG.unpack_from(self)
        b, m = max(0, min(v[2], MAX_BANK)), MAX_BANK
        return dict(zip(_STEP_LOG_NAMES, (*v[:10], list(v[10:10 + b]), list(v[10 + m:10 + m + b]),
                                          list(v[10 + 2 * m:10 + 2 * m + b]), *v[10 + 3 * m:])))


# 8 int32, t and alpha, three arrays of MAX_BANK, 12 doubles
_STEP_LOG = struct.Struct(f"=8i{2 + 3 * MAX_BANK + 12}d")
assert _STEP_LOG.size == C.sizeof(StepLog)
_STEP_LOG_NAMES = tuple(n for n, _ in StepLog._fields_)


class CacheDesc(C.Structure):
    """wdc_paged_cache"""
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p)] + [(n, C.c_int32) for n in ("pages", "page", "kv_heads", "pad_")]


class ChunksDesc(C.Structure):
    """wdc_chunks"""
    _fields_ = [(n, C.c_void_p) for n in ("d_q_start", "d_kv_len", "d_table")] + [(n, C.c_int32) for n in (
        "batch", "table_ld", "rows", "max_q", "max_kv", "pad_")]


_lib = None


def load() -> C.CDLL:
    """Load libwdc.so (built in-tree by paper_2608_01845_amd.build); raise if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_01845_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz, dbl, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_double, C.c_float
    pc, pq = C.POINTER(CacheDesc), C.POINTER(ChunksDesc)
    sig = {
        "wdc_params_default": (None, [C.POINTER(Params)]),
        "wdc_create": (i32, [C.POINTER(ModelDesc), C.POINTER(Params), vp, C.POINTER(vp)]),
        "wdc_destroy": (i32, [vp]),
        "wdc_last_error": (C.c_char_p, [vp]),
        "wdc_weights_bytes": (sz, [vp]),
        "wdc_weight_count": (i32, [vp]),
        "wdc_weight_info": (i32, [vp, i32, C.POINTER(C.c_char_p), C.POINTER(i64), C.POINTER(i32), C.POINTER(sz)]),
        "wdc_bind_weights": (i32, [vp, vp, sz]),
        "wdc_init_weights_random": (i32, [vp, vp, sz, C.c_uint64, f32]),
        "wdc_workspace_bytes": (sz, [vp]),
        "wdc_bind_workspace": (i32, [vp, vp, sz]),
        "wdc_state_bytes": (sz, [vp]),
        "wdc_state_create": (i32, [vp, vp, sz, C.POINTER(vp)]),
        "wdc_state_reset": (i32, [vp, C.POINTER(f32)]),
        "wdc_state_destroy": (i32, [vp]),
        "wdc_state_bank_slot": (i32, [vp, i32, C.POINTER(vp), C.POINTER(i32)]),
        "wdc_cond_embed": (i32, [vp, dbl, vp, vp, vp]),
        "wdc_dit_block_forward": (i32, [vp, i32, vp, vp]),
        "wdc_dit_forward": (i32, [vp, vp, dbl, vp, vp, vp, vp]),
        "wdc_dit_forward_batch": (i32, [vp, i32, vp, dbl, vp, vp, vp, vp]),
        "wdc_scheduler_step": (i32, [vp, vp, vp, dbl, dbl, vp, i64]),
        "wdc_surrogate_step": (i32, [vp, vp, vp, i32, i32, vp, C.POINTER(StepLog)]),
        "wdc_surrogate_step_noalloc": (i32, [vp, vp, vp, i32, i32, vp, C.POINTER(StepLog)]),
        "wdc_risk_update": (i32, [vp, vp, i32, i32, i32, vp, vp, C.POINTER(StepLog)]),
        "wdc_rollout": (i32, [vp, vp, vp, i32, vp, vp, vp, i32, C.POINTER(C.c_uint8), vp, C.POINTER(C.c_uint8),
                              C.POINTER(StepLog)]),
        "wdc_rollout_batch": (i32, [vp, vp, i32, vp, i32, vp, vp, vp, i32, C.POINTER(C.c_uint8), vp,
                                    C.POINTER(C.c_uint8), C.POINTER(StepLog)]),
        "wdc_attn_pad": (i64, [i64]),
        "wdc_attention": (i32, [vp, vp, vp, vp, i64, vp, i64]),
        "wdc_attention_plan": (i32, [vp, i64, C.POINTER(i32), C.POINTER(i32)]),
        "wdc_linear": (i32, [vp, vp, i64, vp, vp, vp, i64, i64, i64, i64]),
        "wdc_cache_append": (i32, [vp, pc, pq, vp, i64, vp, vp, vp, vp, i64]),
        "wdc_cache_attention_scratch": (sz, [vp, pc, pq]),
        "wdc_cache_attention": (i32, [vp, pc, pq, vp, i64, i32, vp, i64, vp, vp, sz]),
        "wdc_cache_mass_scratch": (sz, [vp, pc, pq]),
        "wdc_cache_mass": (i32, [vp, pc, pq, vp, i64, i32, vp, f32, vp, vp, vp, sz]),
        "wdc_cache_evict_scratch": (sz, [vp, pc, pq, i32]),
        "wdc_cache_evict": (i32, [vp, pc, pq, vp, vp, i32, i32, i32, vp, vp, vp, sz]),
        "wdc_set_timing": (i32, [vp, i32]),
        "wdc_timing": (i32, [vp, C.POINTER(dbl), C.POINTER(i64), C.POINTER(dbl)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def exported_symbols() -> List[str]:
    return [
        "wdc_params_default", "wdc_create", "wdc_destroy", "wdc_last_error", "wdc_weights_bytes", "wdc_weight_count",
        "wdc_weight_info", "wdc_bind_weights", "wdc_init_weights_random", "wdc_workspace_bytes", "wdc_bind_workspace",
        "wdc_state_bytes", "wdc_state_create", "wdc_state_reset", "wdc_state_destroy", "wdc_state_bank_slot",
        "wdc_cond_embed", "wdc_dit_block_forward", "wdc_dit_forward", "wdc_dit_forward_batch", "wdc_scheduler_step",
        "wdc_surrogate_step", "wdc_surrogate_step_noalloc", "wdc_risk_update", "wdc_rollout", "wdc_rollout_batch", "wdc_attn_pad", "wdc_attention", "wdc_attention_plan", "wdc_linear",
        "wdc_cache_append", "wdc_cache_attention_scratch", "wdc_cache_attention", "wdc_cache_mass_scratch",
        "wdc_cache_mass", "wdc_cache_evict_scratch", "wdc_cache_evict",
        "wdc_set_timing", "wdc_timing"]


class WdcError(RuntimeError):
    pass


def default_params(**overrides) -> Params:
    p = Params()
    load().wdc_params_default(C.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    return t.data_ptr()


def _ld(t) -> int:
    """Row stride of a [rows, cols] tensor (one of at most one row: its columns)."""
    rows, cols = t.shape
    return t.stride(0) if rows > 1 else cols


def _ptrs(ts):
    """Host array of device pointers of a list of tensors (None entries -> NULL), or None."""
    if ts is None:
        return None
    return (C.c_void_p * len(ts))(*[None if t is None else t.data_ptr() for t in ts])


_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _int32(**values):
    """Refuse what a 32-bit argument would cut."""
    for name, x in values.items():
        if not 0 <= x <= 0x7fffffff:
            raise ValueError(f"{name} = {x}: need 0 <= {name} < 2^31")


class PagedCache:
    """Pages of one layer's keys and values: k, v [pages, kv_heads, page, head_dim]
    contiguous device tensors (wdc_paged_cache)."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device:
            raise ValueError(f"k {tuple(k.shape)} {k.dtype} and v {tuple(v.shape)} {v.dtype} must be alike, "
                             "[pages, kv_heads, page, head_dim]")
        if not (k.is_contiguous() and v.is_contiguous()):
            raise ValueError("k and v must be contiguous")
        self.k, self.v, self.kv_heads, self.device = k, v, k.shape[1], k.get_device()
        self.dtype, self.head_dim, self.slots = k.dtype, k.shape[3], tuple(k.shape[:3])
        self.desc = CacheDesc(k.data_ptr(), v.data_ptr(), k.shape[0], k.shape[2], k.shape[1], 0)
        self.ref = C.byref(self.desc)


class Chunks:
    """The chunks of one call (wdc_chunks): q_start [batch + 1], kv_len [batch] and table
    [batch, pages] int32 device tensors, read when the work runs; rows, max_q and max_kv
    bound them (max_q: all rows, max_kv: all pages of the table, if not given)."""

    def __init__(self, q_start, kv_len, table, rows: int, max_q: Optional[int] = None, max_kv: Optional[int] = None):
        torch = _torch()
        for name, t, dim in (("q_start", q_start, 1), ("kv_len", kv_len, 1), ("table", table, 2)):
            if t.dtype != torch.int32 or t.dim() != dim or not t.is_contiguous() or t.device != kv_len.device:
                raise ValueError(f"{name}: a contiguous int32 tensor of {dim} dimension(s) on one device is needed")
        if q_start.numel() != kv_len.numel() + 1 or table.shape[0] != kv_len.numel():
            raise ValueError("q_start [batch + 1], kv_len [batch] and table [batch, pages] disagree on the batch")
        max_q, max_kv = rows if max_q is None else max_q, 0x7fffffff if max_kv is None else max_kv
        _int32(rows=rows, max_q=max_q, max_kv=max_kv)
        self.q_start, self.kv_len, self.table = q_start, kv_len, table
        self.rows, self.batch, self.device = rows, kv_len.numel(), kv_len.get_device()
        self.desc = ChunksDesc(q_start.data_ptr(), kv_len.data_ptr(), table.data_ptr(), kv_len.numel(), table.shape[1],
                               rows, max_q, max_kv, 0)
        self.ref = C.byref(self.desc)


class Context:
    """One model on one GPU stream. Device memory for weights, workspace and
    rollout state comes from torch allocations."""

    def __init__(self, cfg, params: Optional[Params] = None, device: str = "cuda:0", stream=None,
                 allocate_weights: bool = True, max_batch: int = 1):
        torch = _torch()
        self.lib = load()
        self.cfg = cfg
        self.device = torch.device(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.device_index = self.stream.device_index if self.device.index is None else self.device.index
        self.max_batch = max_batch
        self.desc = desc_from_config(cfg, max_batch)
        self.params = params if params is not None else default_params()
        h = C.c_void_p()
        self._check(self.lib.wdc_create(C.byref(self.desc), C.byref(self.params), C.c_void_p(self.stream.cuda_stream),
                                        C.byref(h)), None)
        self.h = h
        self.bf16 = cfg.dtype == "bf16"
        self.tdtype = torch.bfloat16 if self.bf16 else torch.float32
        ws = self.lib.wdc_workspace_bytes(h)
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=self.device)
        self._check(self.lib.wdc_bind_workspace(h, C.c_void_p(self.workspace.data_ptr()), self.workspace.numel()))
        self.weights = None
        nbytes = self.lib.wdc_weights_bytes(h)
        if allocate_weights and nbytes:
            self.weights = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
            self._check(self.lib.wdc_bind_weights(h, C.c_void_p(self.weights.data_ptr()), nbytes))

    # ---------------------------------------------------------------- plumbing
    def _check(self, status: int, h=-1):
        if status != 0:
            hh = self.h if h == -1 else h
            msg = self.lib.wdc_last_error(hh)
            raise WdcError(f"{STATUS.get(status, status)}: {msg.decode() if msg else ''}")

    def close(self):
        if getattr(self, "h", None):
            self.lib.wdc_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def n_tokens(self) -> int:
        c = self.cfg
        return c.n_video + c.text_tokens

    def weight_table(self) -> List[Tuple[str, Tuple[int, ...], int]]:
        out = []
        for i in range(self.lib.wdc_weight_count(self.h)):
            name = C.c_char_p()
            shape = (C.c_int64 * 2)()
            nd = C.c_int32()
            off = C.c_size_t()
            self._check(self.lib.wdc_weight_info(self.h, i, C.byref(name), shape, C.byref(nd), C.byref(off)))
            shp = (shape[0], shape[1]) if nd.value == 2 else (shape[0],)
            out.append((name.value.decode(), shp, off.value))
        return out

    def to_device(self, arr, dtype=None):
        """numpy -> device tensor in the model dtype (or ``dtype``); bf16 rounding is round-to-nearest-even."""
        torch = _torch()
        t = torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32))
        return t.to(self.device).to(dtype or self.tdtype).contiguous()

    def load_weights(self, named: Dict[str, np.ndarray], strict: bool = True):
        """Copy named tensors into the weight blob (name/shape from weight_table)."""
        torch = _torch()
        table = self.weight_table()
        seen = 0
        esz = 2 if self.bf16 else 4
        for name, shape, off in table:
            if name not in named:
                if strict:
                    raise KeyError(f"missing weight {name}")
                continue
            a = np.asarray(named[name], dtype=np.float32)
            if tuple(a.shape) != tuple(shape):
                raise ValueError(f"{name}: shape {a.shape} != {shape}")
            dev = self.to_device(a).reshape(-1).view(torch.uint8)
            self.weights[off: off + a.size * esz].copy_(dev)
            seen += 1
        return seen

    def bind_weights(self, blob):
        """Bind an existing weight blob (a uint8 device tensor, e.g. another context's
        ``weights`` for the same model) instead of this context's own."""
        self._check(self.lib.wdc_bind_weights(self.h, C.c_void_p(blob.data_ptr()), blob.numel()))
        self.weights = blob

    def init_random_weights(self, seed: int = 0, std: float = 0.02):
        self._check(self.lib.wdc_init_weights_random(self.h, C.c_void_p(self.weights.data_ptr()),
                                                     self.weights.numel(), seed, std))

    # ---------------------------------------------------------------- denoiser
    def cond_embed(self, t: float, cond=None, cam=None, out=None):
        torch = _torch()
        out = out if out is not None else torch.empty(self.cfg.hidden, dtype=torch.float32, device=self.device)
        self._check(self.lib.wdc_cond_embed(self.h, t, _ptr(cond), _ptr(cam), _ptr(out)))
        return out

    def block_forward(self, block: int, x, cemb):
        """In place on x [N, D] float32."""
        self._check(self.lib.wdc_dit_block_forward(self.h, block, _ptr(x), _ptr(cemb)))
        return x

    def forward(self, z, t: float, cond=None, text=None, cam=None, out=None):
        torch = _torch()
        out = out if out is not None else torch.empty_like(z)
        self._check(self.lib.wdc_dit_forward(self.h, _ptr(z), t, _ptr(cond), _ptr(text), _ptr(cam), _ptr(out)))
        return out

    def forward_batch(self, zs, t: float, conds=None, texts=None, cams=None, outs=None):
        """F_theta of len(zs) samples at one t in one batched pass; lists of tensors."""
        torch = _torch()
        b = len(zs)
        outs = outs if outs is not None else [torch.empty_like(z) for z in zs]
        self._check(self.lib.wdc_dit_forward_batch(self.h, b, _ptrs(zs), t, _ptrs(conds), _ptrs(texts), _ptrs(cams),
                                                   _ptrs(outs)))
        return outs

    def scheduler_step(self, z, v, t_cur: float, t_next: float, out=None):
        torch = _torch()
        out = out if out is not None else torch.empty_like(z)
        self._check(self.lib.wdc_scheduler_step(self.h, _ptr(z), _ptr(v), t_cur, t_next, _ptr(out), z.numel()))
        return out

    def attention(self, q, k, vt, n: int, out, ldo: int):
        self._check(self.lib.wdc_attention(self.h, _ptr(q), _ptr(k), _ptr(vt), n, _ptr(out), ldo))
        return out

    def attn_pad(self, n: int) -> int:
        return self.lib.wdc_attn_pad(n)

    def attention_plan(self, n: int):
        """(query blocks per head over all keys, key ranges of each remaining block)."""
        qb, ks = C.c_int32(), C.c_int32()
        self._check(self.lib.wdc_attention_plan(self.h, n, C.byref(qb), C.byref(ks)))
        return qb.value, ks.value

    def linear(self, a, w, bias, out, m: int, n: int, k: int, lda: int = None, ldc: int = None):
        self._check(self.lib.wdc_linear(self.h, _ptr(a), lda or k, _ptr(w), _ptr(bias), _ptr(out), ldc or n, m, n, k))
        return out

    # ---------------------------------------------------------------- paged key/value cache
    def _cache_check(self, cache, chunks):
        if cache.dtype is not self.tdtype or cache.head_dim != self.cfg.head_dim:
            raise ValueError(f"cache of {cache.dtype}, head size {cache.head_dim}: the context has {self.tdtype}, "
                             f"{self.cfg.head_dim}")
        if cache.device != chunks.device or cache.device != self.device_index:
            raise ValueError(f"cache or chunks not on {self.device}")

    def _tensor(self, name, t, dtype, shape, device, strided=False):
        """Pointer of an argument of this type, shape and device (an index); strided: rows may be apart."""
        if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
            raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}, expected {shape} {dtype} on cuda:{device}")
        if not t.is_contiguous() and not (strided and t.stride(1) == 1):
            raise ValueError(f"{name}: unsupported strides {t.stride()}")
        return t.data_ptr()

    def _scratch(self, nbytes: int):
        """Device memory that lives as long as the work just enqueued on this context's stream."""
        torch = _torch()
        # (torch.cuda.current_stream() builds a Stream object: 1.9 us a call, this 0.1)
        if torch._C._cuda_getCurrentRawStream(self.device_index) == self.stream.cuda_stream:
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    def _launch(self, call, *args):
        """One call; the null stream is the current device's, so that device has to be this context's."""
        torch = _torch()
        if torch._C._cuda_getDevice() == self.device_index:
            status = call(self.h, *args)
        else:
            with torch.cuda.device(self.device_index):
                status = call(self.h, *args)
        if status:
            self._check(status)

    def cache_append(self, cache: PagedCache, chunks: Chunks, qkv, q, pos=None, q_weight=None, k_weight=None):
        """Normalise and rotate q and k of qkv [rows, (heads + 2 kv_heads) head_dim], store k and v in the
        cache and write q [rows, heads head_dim]. Rows may be strided."""
        torch = _torch()
        self._cache_check(cache, chunks)
        hd, rows, dev, ptr = self.cfg.head_dim, chunks.rows, cache.device, self._tensor
        qkv_p = ptr("qkv", qkv, self.tdtype, (rows, (self.cfg.heads + 2 * cache.kv_heads) * hd), dev, True)
        q_p = ptr("q", q, self.tdtype, (rows, self.cfg.heads * hd), dev, True)
        pos_p = pos if pos is None else ptr("pos", pos, torch.int32, (rows, 3), dev)
        qw_p = q_weight if q_weight is None else ptr("q_weight", q_weight, torch.float32, (hd,), dev)
        kw_p = k_weight if k_weight is None else ptr("k_weight", k_weight, torch.float32, (hd,), dev)
        self._launch(self.lib.wdc_cache_append, cache.ref, chunks.ref, qkv_p, _ld(qkv), pos_p, qw_p, kw_p, q_p, _ld(q))
        return q

    def cache_attention(self, cache: PagedCache, chunks: Chunks, q, out, frame: int = 0, lse=None):
        """Attention of the chunks' rows q [rows, heads head_dim] over the cache into out (same shape);
        lse [rows, heads] float32 takes the rows' log-sum-exp. frame: rows per frame (0: all see all).
        out may be q itself."""
        self._cache_check(cache, chunks)
        _int32(frame=frame)
        shape, dev, ptr = (chunks.rows, self.cfg.heads * self.cfg.head_dim), cache.device, self._tensor
        q_p, out_p = ptr("q", q, self.tdtype, shape, dev, True), ptr("out", out, self.tdtype, shape, dev, True)
        lse_p = lse if lse is None else ptr("lse", lse, _torch().float32, (chunks.rows, self.cfg.heads), dev)
        n = self.lib.wdc_cache_attention_scratch(self.h, cache.ref, chunks.ref)
        scratch = self._scratch(n) if n else None
        self._launch(self.lib.wdc_cache_attention, cache.ref, chunks.ref, q_p, _ld(q), frame, out_p, _ld(out), lse_p,
                     _ptr(scratch), n)
        return out

    def cache_mass(self, cache: PagedCache, chunks: Chunks, q, lse, mass, frame: int = 0, decay: float = 1.0, out=None):
        """out = decay * mass + the weight each cached key receives from the chunks' rows (out: mass itself
        if not given); mass [pages, kv_heads, page] float32, lse from cache_attention with the same frame."""
        f32, dev, ptr, shape = _torch().float32, cache.device, self._tensor, cache.slots
        self._cache_check(cache, chunks)
        _int32(frame=frame)
        q_p = ptr("q", q, self.tdtype, (chunks.rows, self.cfg.heads * self.cfg.head_dim), dev, True)
        lse_p = ptr("lse", lse, f32, (chunks.rows, self.cfg.heads), dev)
        mass_p = ptr("mass", mass, f32, shape, dev)
        out_p = mass_p if out is None else ptr("out", out, f32, shape, dev)
        n = self.lib.wdc_cache_mass_scratch(self.h, cache.ref, chunks.ref)
        scratch = self._scratch(n) if n else None
        self._launch(self.lib.wdc_cache_mass, cache.ref, chunks.ref, q_p, _ld(q), frame, lse_p, decay, mass_p, out_p,
                     _ptr(scratch), n)
        return mass if out is None else out

    def cache_evict(self, cache: PagedCache, chunks: Chunks, mass, keep: int, sink: int = 0, recent: int = 0,
                    kv_len_out=None, index=None, out=None):
        """Trim every sequence to `keep` keys in place: the first `sink` slots, the last `recent` and the others of
        largest mass. Kept keys fill holes, so slots are not in order of age afterwards: the last `recent` slots are the
        newest keys only while `recent` is at most the rows appended since the last eviction. kv_len_out takes the
        new lengths (chunks.kv_len itself if not given), out the masses (mass itself), index [batch, kv_heads, keep]
        int32 the former slots."""
        torch = _torch()
        self._cache_check(cache, chunks)
        _int32(keep=keep, sink=sink, recent=recent)
        dev, ptr, shape, batch = cache.device, self._tensor, cache.slots, chunks.batch
        kv_len_out = chunks.kv_len if kv_len_out is None else kv_len_out
        mass_p = ptr("mass", mass, torch.float32, shape, dev)
        out_p = mass_p if out is None else ptr("out", out, torch.float32, shape, dev)
        len_p = ptr("kv_len_out", kv_len_out, torch.int32, (batch,), dev)
        idx_p = index if index is None else ptr("index", index, torch.int32, (batch, cache.kv_heads, keep), dev)
        n = self.lib.wdc_cache_evict_scratch(self.h, cache.ref, chunks.ref, keep)
        scratch = self._scratch(n) if n else None
        self._launch(self.lib.wdc_cache_evict, cache.ref, chunks.ref, mass_p, out_p, keep, sink, recent, len_p, idx_p,
                     _ptr(scratch), n)
        return kv_len_out

    def set_timing(self, on: bool):
        self._check(self.lib.wdc_set_timing(self.h, int(on)))

    def timing(self):
        n = len(TIMING_CLASSES)
        ms, cnt, work = (C.c_double * n)(), (C.c_int64 * n)(), (C.c_double * n)()
        self._check(self.lib.wdc_timing(self.h, ms, cnt, work))
        return {name: (ms[i], cnt[i], work[i]) for i, name in enumerate(TIMING_CLASSES)}

    # ---------------------------------------------------------------- surrogate, risk, rollout
    def new_state(self) -> "State":
        return State(self)

    def rollout(self, state: "State", z, steps: int, cond=None, text=None, cam=None, mode: int = MODE_RISK,
                forced: Optional[Sequence[int]] = None, replay_v=None):
        sched = (C.c_uint8 * steps)()
        logs = (StepLog * steps)()
        fz = None
        if forced is not None:
            fz = (C.c_uint8 * steps)(*[int(x) for x in forced])
        self._check(self.lib.wdc_rollout(self.h, state.h, _ptr(z), steps, _ptr(cond), _ptr(text), _ptr(cam), mode,
                                         fz, _ptr(replay_v), sched, logs))
        return list(sched), [l.as_dict() for l in logs]

    def rollout_batch(self, states: Sequence["State"], zs, steps: int, conds=None, texts=None, cams=None,
                      mode: int = MODE_RISK, forced: Optional[Sequence[Sequence[int]]] = None, replay_vs=None):
        """len(zs) rollouts at once (each latent updated in place); per-sample
        schedules [B][S] and logs [B][S]."""
        b = len(zs)
        sched = (C.c_uint8 * (b * steps))()
        logs = (StepLog * (b * steps))()
        fz = None
        if forced is not None:
            fz = (C.c_uint8 * (b * steps))(*[int(x) for row in forced for x in row])
        st = (C.c_void_p * b)(*[s.h.value for s in states])
        self._check(self.lib.wdc_rollout_batch(self.h, st, b, _ptrs(zs), steps, _ptrs(conds), _ptrs(texts),
                                               _ptrs(cams), mode, fz, _ptrs(replay_vs), sched, logs))
        return ([list(sched[i * steps:(i + 1) * steps]) for i in range(b)],
                [[logs[i * steps + k].as_dict() for k in range(steps)] for i in range(b)])

    def surrogate_step(self, state: "State", z, k: int, steps: int, zhat) -> dict:
        log = StepLog()
        self._check(self.lib.wdc_surrogate_step(self.h, state.h, _ptr(z), k, steps, _ptr(zhat), C.byref(log)))
        return log.as_dict()

    def surrogate_step_noalloc(self, state: "State", z, k: int, steps: int, zhat) -> dict:
        """surrogate_step without any allocation or timing event."""
        log = StepLog()
        self._check(self.lib.wdc_surrogate_step_noalloc(self.h, state.h, _ptr(z), k, steps, _ptr(zhat),
                                                        C.byref(log)))
        return log.as_dict()

    def risk_update(self, state: "State", phase: int, k: int, steps: int, z_cur=None, z_next=None) -> dict:
        log = StepLog()
        self._check(self.lib.wdc_risk_update(self.h, state.h, phase, k, steps, _ptr(z_cur), _ptr(z_next),
                                             C.byref(log)))
        return log.as_dict()


class State:
    """Rollout state (bank, anchor, history, risk); device memory from torch."""

    def __init__(self, ctx: Context):
        torch = _torch()
        self.ctx = ctx
        n = ctx.lib.wdc_state_bytes(ctx.h)
        self.mem = torch.empty(n, dtype=torch.uint8, device=ctx.device)
        h = C.c_void_p()
        ctx._check(ctx.lib.wdc_state_create(ctx.h, C.c_void_p(self.mem.data_ptr()), n, C.byref(h)))
        self.h = h

    def reset(self, cam: Optional[np.ndarray] = None):
        arr = None
        if cam is not None:
            c = np.ascontiguousarray(cam, dtype=np.float32)
            arr = c.ctypes.data_as(C.POINTER(C.c_float))
        self.ctx._check(self.ctx.lib.wdc_state_reset(self.h, arr))

    def bank_slot(self, i: int):
        p = C.c_void_p()
        ins = C.c_int32()
        self.ctx._check(self.ctx.lib.wdc_state_bank_slot(self.h, i, C.byref(p), C.byref(ins)))
        return p.value, ins.value

    def close(self):
        if getattr(self, "h", None):
            self.ctx.lib.wdc_state_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
