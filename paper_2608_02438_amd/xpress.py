"""Python binding of libxpress.so (the C ABI in include/xpress.h).

Argument marshalling only: every step of the refine + verify path runs in the
HIP kernels of the library.  PyTorch is used for device memory and streams.
The library must have been built (``python -m paper_2608_02438_amd.build``);
there is no fallback implementation, and loading fails loudly without it.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Dict, Optional

import numpy as np

# the library this process loads; XPRESS_LIB names another build of it (the
# host-ASan one of build.py --asan)
LIB_PATH = os.environ.get("XPRESS_LIB") or os.path.join(
    os.path.dirname(os.path.abspath(__file__)), "libxpress.so")

XP_OK, XP_EINVAL, XP_EUNSUPPORTED, XP_EHIP, XP_ENOMEM = 0, -1, -2, -3, -4
XP_F32, XP_BF16, XP_E4M3 = 0, 1, 2
XP_EARLY_EXIT, XP_WRITE_LOGITS = 1, 2
XP_DEVERR_TOKEN, XP_DEVERR_TEMPERATURE, XP_DEVERR_FILTER = 1, 2, 4
XP_DEVERR_PAGE, XP_DEVERR_SLOT, XP_DEVERR_POOL, XP_DEVERR_LENGTH = 8, 16, 32, 64

EXPORTS = ("xp_create", "xp_destroy", "xp_last_error", "xp_status_string",
           "xp_refine_block", "xp_verify_block", "xp_device_errors", "xp_timing_enable",
           "xp_timing_read", "xp_probe_hbm_read", "xp_probe_mfma_bf16", "xp_toeplitz_mixer",
           "xp_layer_create", "xp_layer_forward", "xp_layer_destroy", "xp_layer_last_error",
           "xp_layer_forward_noalloc", "xp_kv_create", "xp_kv_destroy", "xp_kv_last_error",
           "xp_kv_map", "xp_kv_write", "xp_kv_attn", "xp_kv_attn_shared", "xp_kv_device_errors",
           "xp_layer_forward_paged")
LAYER_WEIGHT_NAMES = ("g_attn", "Wq", "Wk", "Wv", "g_q", "g_k", "Wo", "g_mlp", "Wg", "Wu", "Wd")
STAGES = ("prep", "lmhead", "select", "rspace", "read", "verify")


class XpError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_status_name(status)}: {msg}")
        self.status = status


class _Weights(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int32), ("r", ctypes.c_int32), ("V", ctypes.c_int32),
                ("B", ctypes.c_int32), ("dtype", ctypes.c_int32)] + [
        (n, ctypes.c_void_p) for n in ("W_lm", "W_h", "W_g", "W_e", "W_in", "L", "W_1", "W_2", "W_r")]


WEIGHT_NAMES = ("W_lm", "W_h", "W_g", "W_e", "W_in", "L", "W_1", "W_2", "W_r")

class _LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("H", "n_heads", "n_kv", "head_dim", "ffn")] + [
        ("eps", ctypes.c_float), ("rope_theta", ctypes.c_float)] + [
        (n, ctypes.c_void_p) for n in ("g_attn", "Wq", "Wk", "Wv", "g_q", "g_k", "Wo", "g_mlp",
                                       "Wg", "Wu", "Wd")]


class _KvShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_heads", "n_kv", "head_dim", "page_size",
                                              "n_pages", "dtype")]


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libxpress.so and declare its signatures (no GPU work)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2608_02438_amd.build`")
    L = ctypes.CDLL(path)
    vp, i32, u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32
    L.xp_create.argtypes = [ctypes.POINTER(_Weights), i32, ctypes.POINTER(vp)]
    L.xp_create.restype = i32
    L.xp_destroy.argtypes = [vp]
    L.xp_destroy.restype = None
    L.xp_last_error.argtypes = [vp]
    L.xp_last_error.restype = ctypes.c_char_p
    L.xp_status_string.argtypes = [i32]
    L.xp_status_string.restype = ctypes.c_char_p
    L.xp_refine_block.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, u32, vp, vp, vp,
                                  vp, vp]
    L.xp_refine_block.restype = i32
    L.xp_verify_block.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.xp_verify_block.restype = i32
    L.xp_device_errors.argtypes = [vp, ctypes.POINTER(u32), vp]
    L.xp_device_errors.restype = i32
    L.xp_timing_enable.argtypes = [vp, u32, i32]
    L.xp_timing_enable.restype = i32
    L.xp_timing_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    L.xp_timing_read.restype = i32
    L.xp_probe_hbm_read.argtypes = [vp, ctypes.c_size_t, vp, i32, vp]
    L.xp_probe_hbm_read.restype = i32
    L.xp_probe_mfma_bf16.argtypes = [vp, i32, i32, vp, vp]
    L.xp_probe_mfma_bf16.restype = i32
    L.xp_toeplitz_mixer.argtypes = [vp, i32, i32, i32, vp, vp]
    L.xp_toeplitz_mixer.restype = i32
    L.xp_layer_create.argtypes = [ctypes.POINTER(_LayerWeights), i32, i32, i32, ctypes.POINTER(vp)]
    L.xp_layer_create.restype = i32
    L.xp_layer_forward.argtypes = [vp, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp]
    L.xp_layer_forward.restype = i32
    L.xp_layer_destroy.argtypes = [vp]
    L.xp_layer_destroy.restype = None
    L.xp_layer_last_error.argtypes = [vp]
    L.xp_layer_last_error.restype = ctypes.c_char_p
    L.xp_layer_forward_noalloc.argtypes = [ctypes.POINTER(_LayerWeights), i32, i32, i32, vp, vp,
                                           vp, i32, vp, vp, vp, vp]
    L.xp_layer_forward_noalloc.restype = i32
    i64 = ctypes.c_int64
    L.xp_kv_create.argtypes = [ctypes.POINTER(_KvShape), i32, i32, i32, i32, ctypes.POINTER(vp)]
    L.xp_kv_create.restype = i32
    L.xp_kv_destroy.argtypes = [vp]
    L.xp_kv_destroy.restype = None
    L.xp_kv_last_error.argtypes = [vp]
    L.xp_kv_last_error.restype = ctypes.c_char_p
    L.xp_kv_map.argtypes = [vp, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, i32, vp]
    L.xp_kv_map.restype = i32
    L.xp_kv_write.argtypes = [vp, i32, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp]
    L.xp_kv_write.restype = i32
    attn = [vp, i64, vp, vp, vp, i64, vp, vp, vp, vp, i32, i32, i32, ctypes.c_float, vp, i64, vp,
            vp]
    L.xp_kv_attn.argtypes = [vp, i32, i32, i32] + attn
    L.xp_kv_attn.restype = i32
    L.xp_kv_attn_shared.argtypes = [vp, i32, i32, i32, i32, vp, vp] + attn
    L.xp_kv_attn_shared.restype = i32
    L.xp_layer_forward_paged.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp,
                                         i64, vp, vp, vp, vp]
    L.xp_layer_forward_paged.restype = i32
    L.xp_kv_device_errors.argtypes = [vp, ctypes.POINTER(u32), vp]
    L.xp_kv_device_errors.restype = i32
    _lib = L
    return L


def _status_name(s: int) -> str:
    try:
        return load_library().xp_status_string(s).decode()
    except Exception:  # pragma: no cover
        return str(s)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    return int(t.data_ptr())


def _stream(stream) -> Optional[int]:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def _empty_on(stream, shape, dtype, device):
    """An output that work on `stream` (None: the current one) fills: memory of that
    stream's, so that no earlier work on another one still uses it."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def bf16_tensor(bits: np.ndarray, device="cuda"):
    """Device bf16 tensor from bf16 bit patterns (uint16)."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).to(device)


def device_tensor(x: np.ndarray, device="cuda"):
    """Device tensor of a stored input: uint16 -> bf16, float32 -> float32, ints as is."""
    import torch
    if x.dtype == np.uint16:
        return bf16_tensor(x, device)
    return torch.from_numpy(np.ascontiguousarray(x)).to(device)


@dataclass
class RefineOut:
    ids: object
    iters: object
    logits: Optional[object]
    traj: Optional[object]


class Refiner:
    """One xp_handle: weights on the device plus the workspace for max_batch sequences."""

    def __init__(self, weights: Dict[str, object], H: int, r: int, V: int, B: int,
                 max_batch: int):
        import torch
        L = load_library()
        w0 = weights["W_lm"]
        self.dtype = XP_BF16 if w0.dtype == torch.bfloat16 else XP_F32
        tdt = torch.bfloat16 if self.dtype == XP_BF16 else torch.float32
        self.tdtype = tdt
        self.H, self.r, self.V, self.B, self.max_batch = H, r, V, B, max_batch
        self.device = w0.device
        self._keep = {}
        st = _Weights(H=H, r=r, V=V, B=B, dtype=self.dtype)
        for n in WEIGHT_NAMES:
            t = weights[n]
            if t.dtype != tdt or not t.is_contiguous() or t.device != self.device:
                raise ValueError(f"{n}: expected a contiguous {tdt} tensor on {self.device}")
            self._keep[n] = t
            setattr(st, n, t.data_ptr())
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            s = L.xp_create(ctypes.byref(st), max_batch, ctypes.byref(h))
        if s != XP_OK:
            raise XpError(s, L.xp_last_error(None).decode())
        self._h = h
        self._L = L

    # ------------------------------------------------------------------
    def _check(self, s: int):
        if s != XP_OK:
            raise XpError(s, self._L.xp_last_error(self._h).decode())

    def refine_block(self, hidden, anchor, seed_ids=None, temp=None, u_draft=None, K: int = 6,
                     early_exit: bool = False, write_logits: bool = False,
                     want_traj: bool = False, out: Optional[RefineOut] = None,
                     stream=None, temperature=None, top_k=None, top_p=None) -> RefineOut:
        import torch
        batch = hidden.shape[0]
        if (tuple(hidden.shape) != (batch, self.B, self.H) or hidden.dtype != self.tdtype
                or not hidden.is_contiguous() or hidden.device != self.device):
            raise ValueError(f"hidden must be a contiguous [{batch}][{self.B}][{self.H}] "
                             f"{self.tdtype} tensor on {self.device}")
        for name, t, dt in (("anchor", anchor, torch.int32), ("seed_ids", seed_ids, torch.int32),
                            ("temp", temp, torch.uint8), ("u_draft", u_draft, torch.float32),
                            ("temperature", temperature, torch.float32),
                            ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32)):
            if t is not None and (t.dtype != dt or not t.is_contiguous() or t.device != self.device):
                raise ValueError(f"{name}: expected a contiguous {dt} tensor on {self.device}")
        if out is None:
            dev = self.device
            out = RefineOut(
                ids=torch.empty((batch, self.B), dtype=torch.int32, device=dev),
                iters=torch.empty((batch,), dtype=torch.int32, device=dev),
                logits=(torch.empty((batch, self.B, self.V), dtype=torch.float32, device=dev)
                        if write_logits else None),
                traj=(torch.empty((K + 1, batch, self.B), dtype=torch.int32, device=dev)
                      if want_traj else None))
        flags = (XP_EARLY_EXIT if early_exit else 0) | (XP_WRITE_LOGITS if write_logits else 0)
        s = self._L.xp_refine_block(
            self._h, batch, _ptr(hidden), _ptr(anchor), _ptr(seed_ids), _ptr(temp),
            _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(u_draft), K, flags, _ptr(out.ids),
            _ptr(out.iters),
            _ptr(out.logits) if write_logits else None, _ptr(out.traj), _stream(stream))
        self._check(s)
        return out

    def verify_block(self, draft_ids, target_ids, temp=None, target_logits=None, r_accept=None,
                     u_resample=None, out=None, stream=None):
        import torch
        batch = draft_ids.shape[0]
        if out is None:
            out = (torch.empty((batch,), dtype=torch.int32, device=self.device),
                   torch.empty((batch,), dtype=torch.int32, device=self.device))
        s = self._L.xp_verify_block(
            self._h, batch, _ptr(draft_ids), _ptr(temp), _ptr(target_ids), _ptr(target_logits),
            _ptr(r_accept), _ptr(u_resample), _ptr(out[0]), _ptr(out[1]), _stream(stream))
        self._check(s)
        return out

    def device_errors(self, stream=None) -> int:
        v = ctypes.c_uint32(0)
        self._check(self._L.xp_device_errors(self._h, ctypes.byref(v), _stream(stream)))
        return int(v.value)

    def timing_enable(self, stages=("lmhead",), capacity: int = 4096):
        """Record HIP events around the named stages of every following call."""
        mask = 0
        for n in stages:
            mask |= 1 << STAGES.index(n)
        self._check(self._L.xp_timing_enable(self._h, mask, capacity))

    def timing_read(self):
        """{stage: (total ms, recorded launches)} since the last read; synchronizes."""
        ms = (ctypes.c_float * len(STAGES))()
        n = (ctypes.c_int32 * len(STAGES))()
        self._check(self._L.xp_timing_read(self._h, ms, n))
        return {s: (float(ms[i]), int(n[i])) for i, s in enumerate(STAGES)}

    def close(self):
        if getattr(self, "_h", None):
            self._L.xp_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


def refiner_from_arrays(weights: Dict[str, np.ndarray], H, r, V, B, max_batch, device="cuda"):
    """Upload stored weights (bf16 bits or float32) and create a Refiner."""
    return Refiner({n: device_tensor(weights[n], device) for n in WEIGHT_NAMES}, H, r, V, B,
                   max_batch)


def _check(st: int, what: str):
    if st != XP_OK:
        raise XpError(st, what)


def probe_hbm_read(buf, out_sum, workgroups: int, stream=None):
    """Launch the HBM read probe over the whole of `buf` (a contiguous device
    tensor); `out_sum` (a device int32/uint32 tensor of one element) receives
    the sum of its 32-bit words modulo 2^32."""
    L = load_library()
    nbytes = buf.numel() * buf.element_size()
    _check(L.xp_probe_hbm_read(_ptr(buf), nbytes, _ptr(out_sum), workgroups, _stream(stream)),
           "xp_probe_hbm_read")


def probe_mfma_bf16(operands, workgroups: int, iters: int, out, stream=None):
    """Launch the bf16 MFMA probe; `operands` holds 8 x 64 x 2 x 16 bytes
    (8 x 64 x 2 x 8 bf16), `out` workgroups x 4 x 64 x 16 floats."""
    L = load_library()
    assert operands.numel() * operands.element_size() == 8 * 64 * 2 * 16
    assert out.numel() >= workgroups * 4 * 64 * 16
    _check(L.xp_probe_mfma_bf16(_ptr(operands), workgroups, iters, _ptr(out), _stream(stream)),
           "xp_probe_mfma_bf16")


def toeplitz_mixer(kappa, out=None, stream=None):
    """The full mixer L [r][B][B] of the Toeplitz form of Mix from its kernel
    taps kappa [r][B] (a device tensor, bf16 or float32; kappa[:, 0] unused),
    written by the device into `out` (allocated when None) for use as the
    weight "L"."""
    import torch
    L = load_library()
    assert kappa.dim() == 2 and kappa.is_contiguous()
    r, B = kappa.shape
    dt = {torch.float32: XP_F32, torch.bfloat16: XP_BF16}[kappa.dtype]
    if out is None:
        out = torch.empty((r, B, B), dtype=kappa.dtype, device=kappa.device)
    assert out.shape == (r, B, B) and out.dtype == kappa.dtype and out.is_contiguous()
    _check(L.xp_toeplitz_mixer(_ptr(kappa), r, B, dt, _ptr(out), _stream(stream)),
           "xp_toeplitz_mixer")
    return out


def layer_weights_struct(weights: Dict[str, object], H: int, n_heads: int, n_kv: int, ffn: int,
                         eps: float = 1e-6, theta: float = 1e6, head_dim: int = 128):
    """The xp_layer_weights record of a weight dict (LAYER_WEIGHT_NAMES to bf16
    device tensors)."""
    w = _LayerWeights(H=H, n_heads=n_heads, n_kv=n_kv, head_dim=head_dim, ffn=ffn, eps=eps,
                      rope_theta=theta)
    for n in LAYER_WEIGHT_NAMES:
        setattr(w, n, _ptr(weights[n]))
    return w


def layer_forward_noalloc(w, x, k_cache, v_cache, ctx_len, h_f32, h_bf16, causal=True,
                          stream=None):
    """xp_layer_forward_noalloc: one forward with the library's static
    scratch; `w` from layer_weights_struct, outputs preallocated by the
    caller (no allocation happens here or in the library)."""
    L = load_library()
    batch, B, _ = x.shape
    for t in (x, k_cache, v_cache, ctx_len, h_f32, h_bf16):
        assert t.is_contiguous()
    st = L.xp_layer_forward_noalloc(ctypes.byref(w), batch, B, 1 if causal else 0, _ptr(x),
                                    _ptr(k_cache), _ptr(v_cache), k_cache.shape[1],
                                    _ptr(ctx_len), _ptr(h_f32), _ptr(h_bf16), _stream(stream))
    if st != XP_OK:
        raise XpError(st, "xp_layer_forward_noalloc: " + L.xp_layer_last_error(None).decode())


class Layer:
    """The context layer (xp_layer_*): `weights` maps LAYER_WEIGHT_NAMES to
    bf16 device tensors, which must outlive the layer."""

    def __init__(self, weights: Dict[str, object], H: int, n_heads: int, n_kv: int, ffn: int,
                 max_batch: int, max_B: int, max_ctx: int, eps: float = 1e-6,
                 theta: float = 1e6, head_dim: int = 128):
        L = load_library()
        self._keep = dict(weights)
        w = _LayerWeights(H=H, n_heads=n_heads, n_kv=n_kv, head_dim=head_dim, ffn=ffn, eps=eps,
                          rope_theta=theta)
        for n in LAYER_WEIGHT_NAMES:
            setattr(w, n, _ptr(weights[n]))
        h = ctypes.c_void_p(0)
        st = L.xp_layer_create(ctypes.byref(w), max_batch, max_B, max_ctx, ctypes.byref(h))
        if st != XP_OK:
            raise XpError(st, "xp_layer_create: " + L.xp_layer_last_error(None).decode())
        self._h = h
        self.H = H

    def forward(self, x, k_cache, v_cache, ctx_len, causal=True, h_f32=None, h_bf16=None,
                stream=None):
        """x [batch][B][H] bf16; k_cache, v_cache [batch][C_max][n_kv][128] bf16;
        ctx_len [batch] int32 (device tensors).  Returns (h_f32, h_bf16)."""
        import torch
        L = load_library()
        batch, B, H = x.shape
        C_max = k_cache.shape[1]
        if h_f32 is None:
            h_f32 = torch.empty((batch, B, H), dtype=torch.float32, device=x.device)
        if h_bf16 is None:
            h_bf16 = torch.empty((batch, B, H), dtype=torch.bfloat16, device=x.device)
        for t in (x, k_cache, v_cache, ctx_len, h_f32, h_bf16):
            assert t.is_contiguous()
        st = L.xp_layer_forward(self._h, batch, B, 1 if causal else 0, _ptr(x), _ptr(k_cache),
                                _ptr(v_cache), C_max, _ptr(ctx_len), _ptr(h_f32), _ptr(h_bf16),
                                _stream(stream))
        if st != XP_OK:
            raise XpError(st, "xp_layer_forward: " + L.xp_layer_last_error(self._h).decode())
        return h_f32, h_bf16

    def forward_paged(self, x, kv, k_cache, v_cache, table, ctx_len, causal=True, window=0,
                      sinks=0, k_scale=None, v_scale=None, h_f32=None, h_bf16=None, stream=None):
        """forward() over the pages of `kv` (a PagedKV of the layer's heads): the
        block's keys and values are written to positions ctx_len .. + B - 1 of
        their requests' tables, then attended to (xp_layer_forward_paged)."""
        import torch
        L = load_library()
        batch, B, H = x.shape
        c = kv._cache(k_cache, v_cache, k_scale, v_scale)
        tb = kv._table(table, batch)
        ctx = kv._flat("ctx_len", ctx_len, torch.int32, batch)
        if h_f32 is None:
            h_f32 = _empty_on(stream, (batch, B, H), torch.float32, x.device)
        if h_bf16 is None:
            h_bf16 = _empty_on(stream, (batch, B, H), torch.bfloat16, x.device)
        for name, t, dt in (("x", x, torch.bfloat16), ("h_f32", h_f32, torch.float32),
                            ("h_bf16", h_bf16, torch.bfloat16)):
            if (t.dtype != dt or t.shape != (batch, B, self.H) or not t.is_contiguous()
                    or t.get_device() != kv._index):
                raise ValueError(f"{name}: expected a contiguous {dt} tensor "
                                 f"{(batch, B, self.H)} on {kv.device}")
        with torch.cuda.device(kv.device):
            st = L.xp_layer_forward_paged(self._h, kv._h, batch, B, 1 if causal else 0, window,
                                          sinks, _ptr(x), *c, *tb, ctx, _ptr(h_f32),
                                          _ptr(h_bf16), _stream(stream))
        if st != XP_OK:
            raise XpError(st, "xp_layer_forward_paged: " + L.xp_layer_last_error(self._h).decode())
        return h_f32, h_bf16

    def close(self):
        if getattr(self, "_h", None):
            load_library().xp_layer_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


class PagedKV:
    """The paged context cache (xp_kv_*): pages and slots from lengths, writes of
    new keys and values, and attention over the pages.  The caches [n_pages]
    [n_kv][page_size][head_dim] (``cache_shape``; bf16 or torch.float8_e4m3fn)
    and the tables belong to the caller."""

    def __init__(self, n_heads: int, n_kv: int, page_size: int, n_pages: int, max_batch: int,
                 max_tokens: int, max_len: int, head_dim: int = 128, cache_dtype=None,
                 shared: bool = False, device="cuda"):
        import torch
        L = load_library()
        self.cache_dtype = torch.bfloat16 if cache_dtype is None else cache_dtype
        dt = {torch.bfloat16: XP_BF16, torch.float8_e4m3fn: XP_E4M3}.get(self.cache_dtype)
        if dt is None:
            raise ValueError(f"cache_dtype {cache_dtype}: torch.bfloat16 or torch.float8_e4m3fn")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.n_heads, self.n_kv, self.head_dim, self.page_size = n_heads, n_kv, head_dim, page_size
        self.n_pages = n_pages
        self.cache_shape = torch.Size((n_pages, n_kv, page_size, head_dim))
        self._torch, self._index = torch, self.device.index
        self._raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        st = _KvShape(n_heads=n_heads, n_kv=n_kv, head_dim=head_dim, page_size=page_size,
                      n_pages=n_pages, dtype=dt)
        h = ctypes.c_void_p(0)
        with torch.cuda.device(self.device):
            s = L.xp_kv_create(ctypes.byref(st), max_batch, max_tokens, max_len,
                               1 if shared else 0, ctypes.byref(h))
        if s != XP_OK:
            raise XpError(s, "xp_kv_create: " + L.xp_kv_last_error(None).decode())
        self._h = h
        self._L = L

    # ------------------------------------------------------------------
    def _call(self, name, *args, stream=None):
        torch = self._torch
        if torch.cuda.current_device() == self._index:
            # the current stream's handle without the Stream object, 2.7 of a call's 10 us
            st = self._raw(self._index) if stream is None and self._raw else _stream(stream)
            s = getattr(self._L, name)(self._h, *args, st)
        else:
            with torch.cuda.device(self._index):
                s = getattr(self._L, name)(self._h, *args, _stream(stream))
        if s != XP_OK:
            raise XpError(s, f"{name}: " + self._L.xp_kv_last_error(self._h).decode())

    def _flat(self, name, t, dtype, n, optional=False):
        """The address of a contiguous device vector of n (None: any number of)
        elements, None for an optional one that is not given."""
        if t is None and optional:
            return None
        if (t is None or t.dtype != dtype or t.dim() != 1 or not t.is_contiguous()
                or t.get_device() != self._index or (n is not None and t.shape[0] != n)):
            raise ValueError(f"{name}: expected a contiguous {dtype} tensor of "
                             f"{'any number of' if n is None else n} elements on {self.device}")
        return t.data_ptr()

    def _rows(self, name, t, heads, tokens=None):
        """The token rows' distance of [tokens][heads][head_dim] bf16, heads contiguous."""
        shape, hd = t.shape, self.head_dim
        if (t.dtype != self._torch.bfloat16 or len(shape) != 3 or shape[1] != heads
                or shape[2] != hd or (tokens is not None and shape[0] != tokens)
                or t.get_device() != self._index):
            raise ValueError(f"{name}: expected bf16 [{'tokens' if tokens is None else tokens}]"
                             f"[{heads}][{hd}] rows on {self.device}")
        if t.is_contiguous():
            return heads * hd
        if t.stride(2) != 1 or (heads > 1 and t.stride(1) != hd):
            raise ValueError(f"{name}: expected contiguous [{heads}][{hd}] rows")
        # the row distance of a single row is free
        return t.stride(0) if shape[0] > 1 else heads * hd

    def _cache(self, k_cache, v_cache, k_scale, v_scale):
        for t in (k_cache, v_cache):
            if (t.dtype != self.cache_dtype or t.shape != self.cache_shape
                    or not t.is_contiguous() or t.get_device() != self._index):
                raise ValueError(f"k_cache, v_cache: expected contiguous {self.cache_dtype} "
                                 f"tensors {tuple(self.cache_shape)} on {self.device}")
        f32 = self._torch.float32
        return (k_cache.data_ptr(), v_cache.data_ptr(),
                self._flat("k_scale", k_scale, f32, self.n_kv, optional=True),
                self._flat("v_scale", v_scale, f32, self.n_kv, optional=True))

    def _table(self, table, n):
        if (table.dtype != self._torch.int32 or table.dim() != 2 or table.shape[0] != n
                or table.shape[1] < 1 or not table.is_contiguous()
                or table.get_device() != self._index):
            raise ValueError(f"table: expected a contiguous int32 [{n}][pages] tensor on "
                             f"{self.device}")
        return table.data_ptr(), table.shape[1]

    def map(self, lens, add, table, held, pool, pool_n, cu=None, kv_len=None, slots=None,
            stream=None):
        """Pages and slots from lengths (xp_kv_map): table, held, pool and pool_n
        are updated, and cu, kv_len and slots written where given.  Every page of a
        table counts as its request's own: one that shares a prefix's f pages has them
        in front with held = f, and ends by lens = f * page_size, add = 0 and then
        held = 0; the pages go back with the request that holds them for all."""
        i32, flat = self._torch.int32, self._flat
        n = lens.shape[0]
        self._call("xp_kv_map", n, flat("lens", lens, i32, n), flat("add", add, i32, n),
                   *self._table(table, n), flat("held", held, i32, n),
                   flat("pool", pool, i32, self.n_pages), flat("pool_n", pool_n, i32, 1),
                   flat("cu", cu, i32, n + 1, True), flat("kv_len", kv_len, i32, n, True),
                   flat("slots", slots, i32, None, True), 0 if slots is None else slots.shape[0],
                   stream=stream)
        return cu, kv_len, slots

    def write(self, k, v, slots, k_cache, v_cache, k_scale=None, v_scale=None, stream=None):
        """K and V rows [tokens][n_kv][head_dim] to their slots (xp_kv_write)."""
        n = k.shape[0]
        k_ld, v_ld = self._rows("k", k, self.n_kv), self._rows("v", v, self.n_kv, n)
        sl = self._flat("slots", slots, self._torch.int32, n)
        c = self._cache(k_cache, v_cache, k_scale, v_scale)
        if n:
            self._call("xp_kv_write", n, k.data_ptr(), k_ld, v.data_ptr(), v_ld, sl, *c,
                       stream=stream)

    def _attend(self, name, groups, q, k_cache, v_cache, table, kv_len, cu_q, max_q, causal,
                window, sinks, scale, k_scale, v_scale, out, lse, stream):
        torch = self._torch
        if scale == 0:
            raise ValueError("scale: 2^-60 .. 2^60, or None for 1 / sqrt(head_dim)")
        n, tokens = kv_len.shape[0], q.shape[0]
        lens = self._flat("kv_len", kv_len, torch.int32, n)
        cu = self._flat("cu_q", cu_q, torch.int32, n + 1, optional=True)
        if max_q is None:
            if cu_q is not None:
                raise ValueError("max_q is required with cu_q")
            max_q = tokens // n if n else 0
        elif cu_q is not None:
            max_q = min(max_q, tokens)                        # no request has more
        if out is None:
            out = _empty_on(stream, (tokens, self.n_heads, self.head_dim), torch.bfloat16,
                            self.device)
        q_ld = self._rows("q", q, self.n_heads)
        out_ld = self._rows("out", out, self.n_heads, tokens)
        if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous()
                                or tuple(lse.shape) != (tokens, self.n_heads)
                                or lse.get_device() != self._index):
            raise ValueError(f"lse: expected contiguous float32 [{tokens}][{self.n_heads}]")
        tb = self._table(table, n)
        c = self._cache(k_cache, v_cache, k_scale, v_scale)
        if n and tokens:
            self._call(name, n, tokens, max_q, *groups, q.data_ptr(), q_ld, cu, lens, *tb, *c,
                       1 if causal else 0, window, sinks, 0.0 if scale is None else scale,
                       out.data_ptr(), out_ld, _ptr(lse), stream=stream)
        return out

    def attend(self, q, k_cache, v_cache, table, kv_len, cu_q=None, max_q=None, causal=True,
               window=0, sinks=0, scale=None, k_scale=None, v_scale=None, out=None, lse=None,
               stream=None):
        """Attention of the tokens q [tokens][n_heads][head_dim] over their
        requests' pages (xp_kv_attn); without cu_q every request has the same
        number of them, with it at most max_q (any upper bound).  Returns out (allocated when None)."""
        return self._attend("xp_kv_attn", (), q, k_cache, v_cache, table, kv_len, cu_q, max_q,
                            causal, window, sinks, scale, k_scale, v_scale, out, lse, stream)

    def attend_shared(self, q, k_cache, v_cache, table, kv_len, group_start, shared_len, cu_q=None,
                      max_q=None, causal=True, window=0, sinks=0, scale=None, k_scale=None,
                      v_scale=None, out=None, lse=None, stream=None):
        """attend() for groups of neighbouring requests whose first shared_len keys
        are the same pages, read once per group (xp_kv_attn_shared)."""
        i32, groups = self._torch.int32, shared_len.shape[0]
        return self._attend("xp_kv_attn_shared",
                            (groups, self._flat("group_start", group_start, i32, groups + 1),
                             self._flat("shared_len", shared_len, i32, groups)), q,
                            k_cache, v_cache, table, kv_len, cu_q, max_q, causal, window, sinks,
                            scale, k_scale, v_scale, out, lse, stream)

    def device_errors(self, stream=None) -> int:
        """The XP_DEVERR_* bits set since the last read; synchronizes."""
        v = ctypes.c_uint32(0)
        self._call("xp_kv_device_errors", ctypes.byref(v), stream=stream)
        return int(v.value)

    def close(self):
        if getattr(self, "_h", None):
            self._L.xp_kv_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass
