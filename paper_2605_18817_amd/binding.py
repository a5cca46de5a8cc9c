"""ctypes binding of include/mrp.h — same names, argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

from . import build as _build

EXPORTED_SYMBOLS = [
    "mrp_create", "mrp_destroy", "mrp_workspace_bytes", "mrp_last_error", "mrp_packed_bytes",
    "mrp_pack_weight", "mrp_pack_body_weight", "mrp_chain_step", "mrp_remask", "mrp_commit", "mrp_verify_accept", "mrp_verify_accept_joint", "mrp_kl_loss", "mrp_residual_rms", "mrp_tbody_create", "mrp_chain_step_tf",
    "mrp_profile_enable", "mrp_profile_read", "mrp_verify_accept_static", "mrp_verify_accept_static_scratch_bytes",
    "mrp_build_candidates", "mrp_poll_error", "mrp_probe_lm_traffic",
    "mrp_rope_table", "mrp_qk_norm_rope", "mrp_qk_norm_rope_grad", "mrp_qk_norm_rope_grad_scratch_bytes",
    "mrp_cache_append", "mrp_paged_attention", "mrp_paged_attention_scratch_bytes",
]

MRP_MAX_HEADS = 16


class MrpError(RuntimeError):
    pass


class _Dims(C.Structure):
    _fields_ = [("d", C.c_int), ("V", C.c_int), ("max_rows", C.c_int), ("block_len", C.c_int),
                ("rms_eps", C.c_float)]


class _Head(C.Structure):
    _fields_ = [("W1_packed", C.c_void_p), ("W2_packed", C.c_void_p), ("gamma", C.c_void_p)]


class _TBodyDims(C.Structure):
    _fields_ = [("D", C.c_int), ("n_heads", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int),
                ("d_ff", C.c_int), ("max_prefix", C.c_int), ("rope_theta", C.c_float)]


class _TLayer(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("Wqkv_packed", "Wo_packed", "Wgu_packed", "Wdown_packed", "g1", "g2",
                                          "k_cache", "v_cache")]


class _RevealCfg(C.Structure):
    _fields_ = [("tau", C.c_float), ("r_min", C.c_int), ("max_accept", C.c_int), ("carry_hidden", C.c_int),
                ("tau_remask", C.c_float), ("head_reveal", C.c_int), ("fresh_block", C.c_int),
                ("state_offset", C.c_int), ("run_state0", C.c_int), ("remask_mode", C.c_int)]


class _StepIO(C.Structure):
    _fields_ = [("tok", C.c_void_p), ("conf", C.c_void_p), ("lse", C.c_void_p), ("revealed_at", C.c_void_p),
                ("masked", C.c_void_p), ("cond_tok", C.c_void_p), ("protect_pos", C.c_void_p),
                ("draft_pos", C.c_void_p), ("draft_tok", C.c_void_p), ("remasked", C.c_void_p),
                ("x_tok", C.c_void_p)]


class _Qk(C.Structure):
    _fields_ = [("n_heads", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int), ("rotary_dim", C.c_int),
                ("x_dtype", C.c_int), ("y_dtype", C.c_int), ("gain_dtype", C.c_int), ("eps", C.c_float),
                ("q_gain", C.c_void_p), ("k_gain", C.c_void_p), ("rope", C.c_void_p), ("n_pos", C.c_int)]


class _NewRows(C.Structure):
    _fields_ = [("B", C.c_int), ("max_new", C.c_int), ("cu_rows", C.c_void_p), ("kv_len", C.c_void_p)]


class _PagedCache(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("dtype", C.c_int), ("n_kv_heads", C.c_int),
                ("head_dim", C.c_int), ("n_pages", C.c_int), ("page_size", C.c_int), ("page_table", C.c_void_p),
                ("max_pages", C.c_int), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class _Attn(C.Structure):
    _fields_ = [("n_heads", C.c_int), ("dtype", C.c_int), ("scale", C.c_float), ("causal", C.c_int),
                ("window", C.c_int), ("n_sink", C.c_int)]


_lib = None


def library_path() -> str:
    return _build.LIB


def load_library():
    """Load the built library (building it only if no library is present)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build(force=True)
    lib = C.CDLL(_build.LIB)
    lib.mrp_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(_Dims)]
    lib.mrp_destroy.argtypes = [C.c_void_p]
    lib.mrp_workspace_bytes.argtypes = [C.POINTER(_Dims)]
    lib.mrp_workspace_bytes.restype = C.c_size_t
    lib.mrp_last_error.argtypes = [C.c_void_p]
    lib.mrp_last_error.restype = C.c_char_p
    lib.mrp_packed_bytes.argtypes = [C.c_int, C.c_int]
    lib.mrp_packed_bytes.restype = C.c_size_t
    lib.mrp_pack_weight.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p]
    lib.mrp_pack_body_weight.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p]
    lib.mrp_chain_step.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.POINTER(_Head), C.c_void_p, C.POINTER(_RevealCfg),
                                   C.POINTER(_StepIO)]
    lib.mrp_remask.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_float, C.c_void_p,
                               C.c_void_p, C.c_void_p, C.c_void_p]
    lib.mrp_verify_accept_joint.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.mrp_kl_loss.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                C.c_void_p, C.c_void_p]
    lib.mrp_residual_rms.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_long, C.c_void_p, C.c_int,
                                     C.c_void_p, C.c_void_p]
    lib.mrp_tbody_create.argtypes = [C.c_void_p, C.POINTER(_TBodyDims)]
    lib.mrp_chain_step_tf.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.POINTER(_Head), C.POINTER(_TLayer), C.c_void_p, C.c_void_p,
                                      C.POINTER(_RevealCfg), C.POINTER(_StepIO)]
    lib.mrp_commit.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                               C.c_void_p]
    lib.mrp_verify_accept.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.mrp_verify_accept_static.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.mrp_verify_accept_static_scratch_bytes.restype = C.c_size_t
    lib.mrp_build_candidates.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_int, C.c_int32, C.c_void_p, C.c_void_p]
    lib.mrp_poll_error.argtypes = [C.c_void_p, C.c_void_p]
    lib.mrp_probe_lm_traffic.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p]
    lib.mrp_rope_table.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_float, C.c_void_p]
    lib.mrp_qk_norm_rope.argtypes = [C.c_void_p, C.c_void_p, C.c_long, C.POINTER(_Qk), C.c_void_p, C.c_void_p, C.c_long,
                                     C.c_void_p, C.c_long, C.c_void_p, C.c_void_p]
    lib.mrp_qk_norm_rope_grad_scratch_bytes.argtypes = [C.c_long, C.POINTER(_Qk)]
    lib.mrp_qk_norm_rope_grad_scratch_bytes.restype = C.c_size_t
    lib.mrp_qk_norm_rope_grad.argtypes = [C.c_void_p, C.c_void_p, C.c_long, C.POINTER(_Qk), C.c_void_p, C.c_void_p,
                                          C.c_long, C.c_void_p, C.c_long, C.c_void_p, C.c_void_p, C.c_void_p, C.c_long,
                                          C.c_void_p, C.c_long, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t]
    lib.mrp_cache_append.argtypes = [C.c_void_p, C.c_void_p, C.c_long, C.POINTER(_NewRows), C.POINTER(_Qk), C.c_void_p,
                                     C.c_long, C.c_void_p, C.c_long, C.c_void_p, C.c_long, C.POINTER(_PagedCache),
                                     C.c_void_p]
    lib.mrp_paged_attention_scratch_bytes.argtypes = [C.c_void_p, C.c_long, C.POINTER(_NewRows), C.POINTER(_PagedCache),
                                                      C.POINTER(_Attn)]
    lib.mrp_paged_attention_scratch_bytes.restype = C.c_size_t
    lib.mrp_paged_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_long, C.POINTER(_NewRows), C.POINTER(_PagedCache),
                                        C.POINTER(_Attn), C.c_void_p, C.c_long, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_size_t]
    lib.mrp_profile_enable.argtypes = [C.c_void_p, C.c_int]
    lib.mrp_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.c_int]
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    """Device address of a torch tensor (None stays NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise MrpError("tensor must be a contiguous device tensor")
    return t.data_ptr()


_DTYPES: dict = {}          # torch.dtype -> MRP_DTYPE_*, filled on first use


def _dtypes() -> dict:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.float8_e4m3fn: 3, torch.int32: -32})
    return _DTYPES


def _dtype(t, allowed) -> int:
    code = _dtypes().get(t.dtype)
    if code is None or code not in allowed:
        raise MrpError(f"no form for tensors of {t.dtype} here")
    return code


_FLOATS, _HALVES, _CACHES, _INT = (0, 1, 2), (1, 2), (1, 2, 3), -32


def _dense(t, name: str, dtype: int, shape, device: int) -> Optional[int]:
    """Address of a dense tensor of this type and shape on the device (None stays NULL)."""
    if t is None:
        return None
    if t.shape != shape:
        raise MrpError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if _DTYPES.get(t.dtype) != dtype:
        raise MrpError(f"{name}: {t.dtype} does not fit here")
    if t.get_device() != device or not t.is_contiguous():
        raise MrpError(f"{name}: a contiguous tensor on device {device} is needed")
    return t.data_ptr()


def _rows(t, name: str, shape, dtype: int, device: int):
    """(address, row stride) of a tensor [n_rows][heads][head_dim] on the device whose rows are dense in themselves."""
    if t is None:
        return None, 0
    if t.shape != shape:
        raise MrpError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if _DTYPES.get(t.dtype) != dtype:
        raise MrpError(f"{name}: {t.dtype} is not the type that the others have")
    row, head, one = t.stride()
    n, heads, head_dim = shape
    if t.get_device() != device or one != 1 or (heads > 1 and head != head_dim):
        raise MrpError(f"{name}: a tensor on device {device} whose heads lie side by side is needed")
    return t.data_ptr(), (row if n > 1 else heads * head_dim)


def _int(value: int, name: str) -> int:
    """A size as the library's ints hold it (ctypes would keep the low 32 bits of another)."""
    if not 0 <= value < 2 ** 31:
        raise MrpError(f"{name}={value} out of range")
    return value


def _device_of(*tensors) -> Optional[int]:
    """The one device that the tensors (None: not given) are on."""
    found = {t.get_device() for t in tensors if t is not None}
    if len(found) > 1 or -1 in found:
        raise MrpError("tensors on one GPU are needed")
    return found.pop() if found else None


def _scratch(t, device: int):
    """(address, bytes) of a caller's scratch tensor."""
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        raise MrpError(f"scratch: a contiguous tensor on device {device} is needed")
    return t.data_ptr(), t.numel() * t.element_size()


def _stream() -> int:
    import torch
    return torch.cuda.current_stream().cuda_stream


def packed_bytes(rows: int, cols: int) -> int:
    return load_library().mrp_packed_bytes(rows, cols)


def pack_weight(w, body: bool = False):
    """bf16 (or int16 bit pattern) device tensor [rows][cols] -> packed device tensor (uint8).
    body=True: a head-body weight (converted to fp16 while packing); False: the LM head."""
    import torch
    rows, cols = w.shape
    n = packed_bytes(rows, cols)
    if n == 0:
        raise MrpError(f"cannot pack a {rows}x{cols} matrix (cols must be a multiple of 16)")
    out = torch.empty(n, dtype=torch.uint8, device=w.device)
    fn = load_library().mrp_pack_body_weight if body else load_library().mrp_pack_weight
    rc = fn(_stream(), _ptr(w), rows, cols, _ptr(out))
    if rc != 0:
        raise MrpError(f"mrp_pack_weight failed: {rc}")
    return out


def verify_accept_static(B: int, L: int, V: int, K: int, verify, draft_pos, draft_tok, draft_stride: int, match,
                         accept_len, correction_tok) -> int:
    """mrp_verify_accept_static: no context, no allocation; returns the status code."""
    return load_library().mrp_verify_accept_static(_stream(), B, L, V, K, _ptr(verify), _ptr(draft_pos),
                                                   _ptr(draft_tok), draft_stride, _ptr(match), _ptr(accept_len),
                                                   _ptr(correction_tok))


@dataclass
class Head:
    W1_packed: object
    W2_packed: object
    gamma: object


@dataclass
class TLayer:
    """One transformer layer of a head body (device tensors; weights packed with pack_weight(body=True))."""
    Wqkv_packed: object
    Wo_packed: object
    Wgu_packed: object
    Wdown_packed: object
    g1: object
    g2: object
    k_cache: object
    v_cache: object


@dataclass
class RevealCfg:
    tau: float = 0.9
    r_min: int = 1
    max_accept: int = 0
    carry_hidden: int = 1
    tau_remask: float = -1.0
    head_reveal: int = 1
    fresh_block: int = 1
    state_offset: int = 0
    run_state0: int = 1
    remask_mode: int = 0


class QkNormRope:
    """Norm and rotation of the heads of q and k (mrp_qk): gains [head_dim] or None, ``rope`` the table
    [n_pos][rotary_dim / 2][2] of MrpContext.rope_table or None.  The types of the inputs and outputs come with the
    tensors of a call.  Keeps the tensors that it is given."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, rope=None, q_gain=None, k_gain=None,
                 eps: float = 1e-6):
        gain = q_gain if q_gain is not None else k_gain
        gain_dtype = 1 if gain is None else _dtype(gain, _FLOATS)
        rot, n_pos = 0, 0
        if rope is not None:
            n_pos, rot = rope.shape[0], 2 * rope.shape[1]
        _dtypes()
        self.n_heads, self.n_kv_heads, self.head_dim, self.rotary_dim = n_heads, n_kv_heads, head_dim, rot
        self.tensors = (rope, q_gain, k_gain)
        self.device = dev = _device_of(*self.tensors)
        self._args = (gain_dtype, eps, _dense(q_gain, "q_gain", gain_dtype, (head_dim,), dev),
                      _dense(k_gain, "k_gain", gain_dtype, (head_dim,), dev),
                      _dense(rope, "rope", 0, (n_pos, rot // 2, 2), dev), n_pos)
        self._typed: dict = {}

    def typed(self, x_dtype: int, y_dtype: int):
        """The description for inputs and outputs of these types, as a call takes it."""
        ref = self._typed.get((x_dtype, y_dtype))
        if ref is None:
            c = _Qk(self.n_heads, self.n_kv_heads, self.head_dim, self.rotary_dim, x_dtype, y_dtype, *self._args)
            ref = self._typed[(x_dtype, y_dtype)] = C.byref(c)
        return ref


class NewRows:
    """New rows of a batch (mrp_new_rows): ``kv_len`` int32 [B] positions with the new rows, at most ``max_new`` rows a
    sequence, ``cu_rows`` int32 [B + 1] or None where every sequence has max_new."""

    def __init__(self, kv_len, max_new: int, cu_rows=None):
        _dtypes()
        _int(max_new, "max_new")
        self.B = B = kv_len.shape[0]
        self.tensors = (kv_len, cu_rows)
        self.device = dev = _device_of(*self.tensors)
        self.shape = (B, max_new)
        self.ref = C.byref(_NewRows(B, max_new, _dense(cu_rows, "cu_rows", _INT, (B + 1,), dev),
                                    _dense(kv_len, "kv_len", _INT, (B,), dev)))


class PagedCache:
    """Keys and values in pages (mrp_paged_cache): k_pages, v_pages [n_pages][page_size][n_kv_heads][head_dim] of bf16,
    fp16 or float8_e4m3fn, page_table int32 [B][max_pages], scales fp32 [n_kv_heads] for 8 bits."""

    def __init__(self, k_pages, v_pages, page_table, k_scale=None, v_scale=None):
        if k_pages.dim() != 4 or page_table.dim() != 2:
            raise MrpError("pages [n_pages][page_size][n_kv_heads][head_dim] and a table [B][max_pages] are needed")
        n, ps, hkv, hd = k_pages.shape
        self.B, self.n_kv_heads, self.head_dim, self.dtype = page_table.shape[0], hkv, hd, _dtype(k_pages, _CACHES)
        self.tensors = (k_pages, v_pages, page_table, k_scale, v_scale)
        self.device = dev = _device_of(*self.tensors)
        self.shape = (self.B, hkv, hd, ps * page_table.shape[1])
        self.ref = C.byref(_PagedCache(
            _dense(k_pages, "k_pages", self.dtype, k_pages.shape, dev), _dense(v_pages, "v_pages", self.dtype, k_pages.shape, dev),
            self.dtype, hkv, hd, n, ps, _dense(page_table, "page_table", _INT, page_table.shape, dev), page_table.shape[1],
            _dense(k_scale, "k_scale", 0, (hkv,), dev), _dense(v_scale, "v_scale", 0, (hkv,), dev)))


@dataclass
class AttnCfg:
    """Attention over a paged cache (mrp_attn): the rows of a sequence see all its positions (causal False) or those up to
    their own, with ``window`` > 0 only the last ``window`` of them and the first ``n_sink``."""
    n_heads: int
    scale: float
    causal: bool = True
    window: int = 0
    n_sink: int = 0

    def __post_init__(self):
        _int(self.window, "window"), _int(self.n_sink, "n_sink")


class StepIO:
    """Device buffers of one chain step (allocated with torch)."""

    def __init__(self, B: int, L: int, K: int, device="cuda"):
        import torch
        M = B * L
        self.B, self.L, self.K = B, L, K
        self.tok = torch.full((K + 1, M), -1, dtype=torch.int32, device=device)
        self.conf = torch.zeros((K + 1, M), dtype=torch.float32, device=device)
        self.lse = torch.zeros((K + 1, M), dtype=torch.float32, device=device)
        self.revealed_at = torch.full((M,), -1, dtype=torch.int8, device=device)
        self.masked = torch.ones((M,), dtype=torch.uint8, device=device)
        self.cond_tok = torch.zeros((B,), dtype=torch.int32, device=device)
        self.protect_pos = torch.full((B,), -1, dtype=torch.int32, device=device)
        self.draft_pos = torch.full((B, K + 1), -1, dtype=torch.int32, device=device)
        self.draft_tok = torch.full((B, K + 1), -1, dtype=torch.int32, device=device)
        self.remasked = torch.zeros((K + 1, M), dtype=torch.uint8, device=device)
        self.x_tok = torch.full((M,), -1, dtype=torch.int32, device=device)

    def c_struct(self) -> _StepIO:
        return _StepIO(_ptr(self.tok), _ptr(self.conf), _ptr(self.lse), _ptr(self.revealed_at), _ptr(self.masked),
                       _ptr(self.cond_tok), _ptr(self.protect_pos), _ptr(self.draft_pos), _ptr(self.draft_tok),
                       _ptr(self.remasked), _ptr(self.x_tok))


class MrpContext:
    """Owns an ``mrp_ctx`` (workspace) for fixed (d, V, max_rows, block_len)."""

    def __init__(self, d: int, V: int, max_rows: int, block_len: int, rms_eps: float = 1e-6):
        import torch
        if not torch.cuda.is_available():
            raise MrpError("no GPU: the MRP chain has no CPU path")
        self.lib = load_library()
        self.d, self.V, self.max_rows, self.L = d, V, max_rows, block_len
        self._dims = _Dims(d, V, max_rows, block_len, rms_eps)
        h = C.c_void_p()
        rc = self.lib.mrp_create(C.byref(h), C.byref(self._dims))
        if rc != 0:
            raise MrpError(f"mrp_create failed: {rc}")
        self._h = h
        self.device = torch.cuda.current_device()
        self._get_stream = torch._C._cuda_getCurrentRawStream
        self._scratch_bytes: dict = {}

    def close(self):
        if getattr(self, "_h", None):
            self.lib.mrp_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self) -> int:
        return self.lib.mrp_workspace_bytes(C.byref(self._dims))

    def last_error(self) -> str:
        return self.lib.mrp_last_error(self._h).decode()

    def _check(self, rc: int, what: str):
        if rc < 0:
            raise MrpError(f"{what} failed ({rc}): {self.last_error()}")
        return rc

    def chain_step(self, B: int, K: int, h, h_run, E, W_lm_packed, heads: Sequence[Head], z, cfg: RevealCfg,
                   io: StepIO, check: bool = True) -> int:
        harr = (_Head * max(len(heads), 1))(*[_Head(_ptr(x.W1_packed), _ptr(x.W2_packed), _ptr(x.gamma))
                                              for x in heads])
        if len(heads) < K <= MRP_MAX_HEADS:
            raise MrpError("fewer heads than K")
        ccfg = _RevealCfg(cfg.tau, cfg.r_min, cfg.max_accept, cfg.carry_hidden, cfg.tau_remask, cfg.head_reveal,
                          cfg.fresh_block, cfg.state_offset, cfg.run_state0, cfg.remask_mode)
        cio = io.c_struct()
        rc = self.lib.mrp_chain_step(self._h, _stream(), B, K, _ptr(h), _ptr(h_run), _ptr(E), _ptr(W_lm_packed),
                                     harr, _ptr(z), C.byref(ccfg), C.byref(cio))
        return self._check(rc, "mrp_chain_step") if check else rc

    def tbody_create(self, D: int, n_heads: int, n_kv_heads: int, d_ff: int, max_prefix: int,
                     rope_theta: float = 1.0e6, head_dim: int = 128, check: bool = True) -> int:
        dims = _TBodyDims(D, n_heads, n_kv_heads, head_dim, d_ff, max_prefix, rope_theta)
        rc = self.lib.mrp_tbody_create(self._h, C.byref(dims))
        return self._check(rc, "mrp_tbody_create") if check else rc

    def chain_step_tf(self, B: int, K: int, h, h_run, E, W_lm_packed, heads: Sequence[Head],
                      layers: Sequence[TLayer], prefix_len, z, cfg: RevealCfg, io: StepIO, check: bool = True) -> int:
        """layers: K * D entries, head k's layer l at [k * D + l]."""
        harr = (_Head * max(len(heads), 1))(*[_Head(_ptr(x.W1_packed), _ptr(x.W2_packed), _ptr(x.gamma))
                                              for x in heads])
        larr = (_TLayer * max(len(layers), 1))(*[
            _TLayer(_ptr(l.Wqkv_packed), _ptr(l.Wo_packed), _ptr(l.Wgu_packed), _ptr(l.Wdown_packed), _ptr(l.g1),
                    _ptr(l.g2), _ptr(l.k_cache), _ptr(l.v_cache)) for l in layers])
        if len(heads) < K <= MRP_MAX_HEADS:
            raise MrpError("fewer heads than K")
        ccfg = _RevealCfg(cfg.tau, cfg.r_min, cfg.max_accept, cfg.carry_hidden, cfg.tau_remask, cfg.head_reveal,
                          cfg.fresh_block, cfg.state_offset, cfg.run_state0, cfg.remask_mode)
        cio = io.c_struct()
        rc = self.lib.mrp_chain_step_tf(self._h, _stream(), B, K, _ptr(h), _ptr(h_run), _ptr(E), _ptr(W_lm_packed),
                                        harr, larr if len(layers) else None, _ptr(prefix_len), _ptr(z),
                                        C.byref(ccfg), C.byref(cio))
        return self._check(rc, "mrp_chain_step_tf") if check else rc

    def remask(self, B: int, state: int, conf_new, tau_remask: float, protect_pos, revealed_at, masked,
               remasked_out, check: bool = True) -> int:
        rc = self.lib.mrp_remask(self._h, _stream(), B, state, _ptr(conf_new), tau_remask, _ptr(protect_pos),
                                 _ptr(revealed_at), _ptr(masked), _ptr(remasked_out))
        return self._check(rc, "mrp_remask") if check else rc

    def commit(self, B: int, x_tok, revealed_at, masked, x_out, n_masked, check: bool = True) -> int:
        rc = self.lib.mrp_commit(self._h, _stream(), B, _ptr(x_tok), _ptr(revealed_at), _ptr(masked), _ptr(x_out),
                                 _ptr(n_masked))
        return self._check(rc, "mrp_commit") if check else rc

    def decode_block(self, B: int, K: int, backbone, E, W_lm_packed, heads: Sequence[Head], cfg: RevealCfg,
                     max_steps: Optional[int] = None):
        """Decode one block per sequence to completion: each denoising step takes the prior logits
        ``z`` (fp32 [M][V], device) and hidden states ``h`` (bf16 [M][d], device) from
        ``backbone(step, x_out, masked)``, runs one chain step on the still-masked rows and commits
        what it revealed (mrp_commit).  Only the count of masked rows comes back to the host, once
        per step, to end the loop.  Returns (x_out [M] int32 device, steps, io)."""
        import torch
        L = self.L
        M = B * L
        io = StepIO(B, L, K)
        x_out = torch.full((M,), -1, dtype=torch.int32, device="cuda")
        n_masked = torch.empty((B,), dtype=torch.int32, device="cuda")
        h_run = torch.empty((M, self.d), dtype=torch.float32, device="cuda")
        step_cfg = RevealCfg(**{**cfg.__dict__, "fresh_block": 0})
        max_steps = L if max_steps is None else max_steps
        steps = 0
        while steps < max_steps:
            z, h = backbone(steps, x_out, io.masked)
            self.chain_step(B, K, h, h_run, E, W_lm_packed, heads, z, step_cfg, io)
            self.commit(B, io.x_tok, io.revealed_at, io.masked, x_out, n_masked)
            steps += 1
            if int(n_masked.sum().item()) == 0:
                break
        return x_out, steps, io

    def verify_accept(self, B: int, K: int, verify, draft_pos, draft_tok, draft_stride: int, match, accept_len,
                      correction_tok, check: bool = True) -> int:
        rc = self.lib.mrp_verify_accept(self._h, _stream(), B, K, _ptr(verify), _ptr(draft_pos), _ptr(draft_tok),
                                        draft_stride, _ptr(match), _ptr(accept_len), _ptr(correction_tok))
        return self._check(rc, "mrp_verify_accept") if check else rc

    def verify_accept_joint(self, B: int, K: int, verify, draft_pos, draft_tok, draft_stride: int, match,
                            accept_len, correction_tok, check: bool = True) -> int:
        rc = self.lib.mrp_verify_accept_joint(self._h, _stream(), B, K, _ptr(verify), _ptr(draft_pos),
                                              _ptr(draft_tok), draft_stride, _ptr(match), _ptr(accept_len),
                                              _ptr(correction_tok))
        return self._check(rc, "mrp_verify_accept_joint") if check else rc

    def build_candidates(self, B: int, K: int, x_t, masked_t, draft_pos, draft_tok, draft_stride: int,
                         mask_token: int, cand_tok, cand_masked, check: bool = True) -> int:
        rc = self.lib.mrp_build_candidates(self._h, _stream(), B, K, _ptr(x_t), _ptr(masked_t), _ptr(draft_pos),
                                           _ptr(draft_tok), draft_stride, mask_token, _ptr(cand_tok),
                                           _ptr(cand_masked))
        return self._check(rc, "mrp_build_candidates") if check else rc

    def probe_lm_traffic(self, mode: int, M: int, W_lm_packed, z, check: bool = True) -> int:
        rc = self.lib.mrp_probe_lm_traffic(self._h, _stream(), mode, M, _ptr(W_lm_packed), _ptr(z))
        return self._check(rc, "mrp_probe_lm_traffic") if check else rc

    def poll_error(self) -> int:
        """Wait for the current stream; bits of the device error word set since the last poll (cleared)."""
        return self._check(self.lib.mrp_poll_error(self._h, _stream()), "mrp_poll_error")

    def kl_loss(self, M: int, teacher, student, row_mask, scale: float, loss_rows, grad=None,
                check: bool = True) -> int:
        rc = self.lib.mrp_kl_loss(self._h, _stream(), M, _ptr(teacher), _ptr(student), _ptr(row_mask), scale,
                                  _ptr(loss_rows), _ptr(grad))
        return self._check(rc, "mrp_kl_loss") if check else rc

    def residual_rms(self, n_blocks: int, S: int, N: int, X, bf16: bool, rms_pair, rms_delta,
                     check: bool = True) -> int:
        rc = self.lib.mrp_residual_rms(self._h, _stream(), n_blocks, S, N, _ptr(X), 1 if bf16 else 0,
                                       _ptr(rms_pair), _ptr(rms_delta))
        return self._check(rc, "mrp_residual_rms") if check else rc

    def _here(self, *things):
        """The descriptions are of the context's device (the call itself refuses another current device)."""
        for x in things:
            if x.device is not None and x.device != self.device:
                raise MrpError(f"tensors on device {x.device}: the context is of device {self.device}")

    def _raw_stream(self) -> int:
        """The current stream of the context's device (the same as _stream() where that device is the current one)."""
        return self._get_stream(self.device)

    def rope_table(self, n_pos: int, rotary_dim: int, theta: float):
        """cos and sin of every position and pair: fp32 [n_pos][rotary_dim / 2][2]."""
        import torch
        _int(n_pos, "n_pos"), _int(rotary_dim, "rotary_dim")
        out = torch.empty((n_pos, rotary_dim // 2, 2), dtype=torch.float32, device=f"cuda:{self.device}")
        self._check(self.lib.mrp_rope_table(self._h, self._raw_stream(), n_pos, rotary_dim, theta, out.data_ptr()), "mrp_rope_table")
        return out

    def qk_norm_rope(self, qk: QkNormRope, pos, q, k, q_out, k_out, check: bool = True) -> int:
        """q [n][n_heads][head_dim], k [n][n_kv_heads][head_dim] -> q_out, k_out; pos int32 [n]."""
        self._here(qk)
        dev, n, hd = self.device, q.shape[0], qk.head_dim
        x, y = _dtype(q, _FLOATS), _dtype(q_out, _FLOATS)
        qs, ks = (n, qk.n_heads, hd), (n, qk.n_kv_heads, hd)
        rc = self.lib.mrp_qk_norm_rope(self._h, self._raw_stream(), n, qk.typed(x, y), _dense(pos, "pos", _INT, (n,), dev),
                                       *_rows(q, "q", qs, x, dev), *_rows(k, "k", ks, x, dev),
                                       _dense(q_out, "q_out", y, qs, dev), _dense(k_out, "k_out", y, ks, dev))
        return self._check(rc, "mrp_qk_norm_rope") if check else rc

    def qk_norm_rope_grad(self, qk: QkNormRope, pos, q, k, dq_out, dk_out, dq, dk, dq_gain=None, dk_gain=None, scratch=None,
                          check: bool = True) -> int:
        """Gradients of qk_norm_rope: dq, dk (like q, k) and the gains' (fp32 [head_dim]) from dq_out, dk_out.  scratch: a
        uint8 tensor of qk_norm_rope_grad_scratch_bytes, or None to take one from torch's allocator."""
        self._here(qk)
        dev, n, hd = self.device, q.shape[0], qk.head_dim
        x, y = _dtype(q, _FLOATS), _dtype(dq_out, _FLOATS)
        qs, ks, ref = (n, qk.n_heads, hd), (n, qk.n_kv_heads, hd), qk.typed(x, y)
        if scratch is None:
            import torch
            scratch = torch.empty(self.lib.mrp_qk_norm_rope_grad_scratch_bytes(n, ref), dtype=torch.uint8, device=q.device)
        rc = self.lib.mrp_qk_norm_rope_grad(self._h, self._raw_stream(), n, ref, _dense(pos, "pos", _INT, (n,), dev),
                                            *_rows(q, "q", qs, x, dev), *_rows(k, "k", ks, x, dev),
                                            _dense(dq_out, "dq_out", y, qs, dev), _dense(dk_out, "dk_out", y, ks, dev),
                                            *_rows(dq, "dq", qs, x, dev), *_rows(dk, "dk", ks, x, dev),
                                            _dense(dq_gain, "dq_gain", 0, (hd,), dev), _dense(dk_gain, "dk_gain", 0, (hd,), dev),
                                            *_scratch(scratch, dev))
        return self._check(rc, "mrp_qk_norm_rope_grad") if check else rc

    def qk_norm_rope_grad_scratch_bytes(self, qk: QkNormRope, n: int) -> int:
        return self.lib.mrp_qk_norm_rope_grad_scratch_bytes(n, qk.typed(1, 1))

    def cache_append(self, rows: NewRows, qk: QkNormRope, q, k, v, cache: PagedCache, q_out, check: bool = True) -> int:
        """Norm, rotate and append k, append v, and norm and rotate q into q_out (q and q_out None: keys and values only)."""
        self._here(rows, qk, cache)
        if rows.B != cache.B:
            raise MrpError(f"{rows.B} sequences, but a page table of {cache.B}")
        if (q is None) != (q_out is None):
            raise MrpError("q and q_out go together")
        dev, n, hd = self.device, k.shape[0], qk.head_dim
        x = _dtype(k, _FLOATS)
        y = x if q_out is None else _dtype(q_out, _FLOATS)
        qs, ks = (n, qk.n_heads, hd), (n, qk.n_kv_heads, hd)
        rc = self.lib.mrp_cache_append(self._h, self._raw_stream(), n, rows.ref, qk.typed(x, y), *_rows(q, "q", qs, x, dev),
                                       *_rows(k, "k", ks, x, dev), *_rows(v, "v", ks, x, dev), cache.ref,
                                       _dense(q_out, "q_out", y, qs, dev))
        return self._check(rc, "mrp_cache_append") if check else rc

    def paged_attention_scratch_bytes(self, rows: NewRows, cache: PagedCache, cfg: AttnCfg, q) -> int:
        a = _Attn(cfg.n_heads, _dtype(q, _HALVES), cfg.scale, 1 if cfg.causal else 0, cfg.window, cfg.n_sink)
        return self.lib.mrp_paged_attention_scratch_bytes(self._h, q.shape[0], rows.ref, cache.ref, C.byref(a))

    def paged_attention(self, rows: NewRows, cache: PagedCache, cfg: AttnCfg, q, out, lse=None, scratch=None,
                        check: bool = True) -> int:
        """out [n][n_heads][head_dim] (lse fp32 [n][n_heads], or None) of q over the cache.  scratch: a uint8 tensor of
        paged_attention_scratch_bytes, or None to take one from torch's allocator."""
        self._here(rows, cache)
        if rows.B != cache.B:
            raise MrpError(f"{rows.B} sequences, but a page table of {cache.B}")
        dev, n = self.device, q.shape[0]
        y = _dtype(q, _HALVES)
        shape = (n, cfg.n_heads, cache.head_dim)
        if scratch is None:
            key = (n, cfg.n_heads, rows.shape, cache.shape)      # (all that the size depends on)
            need = self._scratch_bytes.get(key)
            if need is None:
                if len(self._scratch_bytes) >= 4096:
                    self._scratch_bytes.clear()
                need = self._scratch_bytes[key] = self.paged_attention_scratch_bytes(rows, cache, cfg, q)
            if need:
                import torch
                scratch = torch.empty(need, dtype=torch.uint8, device=q.device)
        a = _Attn(cfg.n_heads, y, cfg.scale, 1 if cfg.causal else 0, cfg.window, cfg.n_sink)
        rc = self.lib.mrp_paged_attention(self._h, self._raw_stream(), n, rows.ref, cache.ref, C.byref(a),
                                          *_rows(q, "q", shape, y, dev), _dense(out, "out", y, shape, dev),
                                          _dense(lse, "lse", 0, shape[:2], dev), *_scratch(scratch, dev))
        return self._check(rc, "mrp_paged_attention") if check else rc

    def profile_enable(self, on: bool):
        self._check(self.lib.mrp_profile_enable(self._h, 1 if on else 0), "mrp_profile_enable")

    def profile_read(self, cap: int = 4096) -> List[float]:
        buf = (C.c_float * cap)()
        n = self._check(self.lib.mrp_profile_read(self._h, buf, cap), "mrp_profile_read")
        return [buf[i] for i in range(n)]
