"""ctypes binding of the C-ABI library (include/centrifuge.h).

Argument marshalling only: every step of the path runs inside the HIP
library.  torch supplies device memory and the current stream.  There is no
CPU fallback: if the library has not been built, `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcentrifuge.so")

CF_BF16, CF_F32 = 0, 1
CF_LOSS_NLL, CF_LOSS_POLICY = 0, 1
_STATUS = {0: "CF_OK", 1: "CF_ERR_NULL", 2: "CF_ERR_SHAPE", 3: "CF_ERR_DTYPE", 4: "CF_ERR_WORKSPACE",
           5: "CF_ERR_UNSUPPORTED", 6: "CF_ERR_HIP"}

EXPORTS = (
    "cf_status_str", "cf_version", "cf_index_workspace_bytes", "cf_build_keep_index",
    "cf_build_keep_index_static", "cf_gather_rows",
    "cf_linear_bwd_reduced", "cf_linear_workspace_bytes", "cf_linear_bwd_reduced_ws", "cf_attn_workspace_bytes", "cf_attn_bwd_filtered",
    "cf_layer_workspace_bytes", "cf_layer_bwd_filtered", "cf_layer_bwd_compact", "cf_layer_bwd_compact_dev",
    "cf_layer_bwd_dense",
    "cf_lora_workspace_bytes", "cf_layer_bwd_lora", "cf_probe_mfma_bf16", "cf_probe_mfma_lds_bf16",
    "cf_probe_copy",
    "cf_qk_norm_rope_fwd", "cf_qk_norm_workspace_bytes", "cf_qk_norm_rope_bwd", "cf_layer_qk_workspace_bytes",
    "cf_lora_qk_workspace_bytes", "cf_layer_bwd_filtered_qk", "cf_layer_bwd_compact_qk", "cf_layer_bwd_dense_qk", "cf_layer_bwd_lora_qk",
    "cf_token_loss_workspace_bytes", "cf_token_loss", "cf_adamw_step", "cf_grad_norm_workspace_bytes", "cf_grad_norm",
)


class CfError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (%d)" % (where, _STATUS.get(code, "?"), code))


class LayerDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("S", C.c_int32), ("H", C.c_int32), ("Hq", C.c_int32),
                ("Hkv", C.c_int32), ("d", C.c_int32), ("F", C.c_int32), ("dtype", C.c_int32),
                ("rms_eps", C.c_float), ("softmax_scale", C.c_float)]


class Saved(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("x", "q", "k", "v", "attn_out", "lse", "r", "gate", "up",
                                           "rope_cos", "rope_sin")]


class Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")]


GRAD_NAMES = ("dwq", "dwk", "dwv", "dwo", "dwg", "dwu", "dwd", "dg1", "dg2", "dx")


class Grads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in GRAD_NAMES] + [("main_grad", C.c_int32)]


_LORA_T = ("aq", "bq", "ak", "bk", "av", "bv", "ao", "bo")


class Lora(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _LORA_T] + [("rank", C.c_int32), ("scale", C.c_float)]


class LoraGrads(C.Structure):
    _fields_ = [("d" + n, C.c_void_p) for n in _LORA_T] + [("dx", C.c_void_p)]


class Qk(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64)]


class QkNorm(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("gq", "gk", "rope_cos", "rope_sin", "positions")]


class LayerQk(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q_pre", "k_pre", "gq", "gk")] + [("eps", C.c_float)] + \
               [(n, C.c_void_p) for n in ("dgq", "dgk")]


class LossDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("V", C.c_int32), ("dtype", C.c_int32)] + \
               [(n, C.c_float) for n in ("logit_scale", "clip_lo", "clip_hi", "kl_coef", "norm")]


class AdamwTensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("p", "master", "g", "m", "v", "m_scale", "v_scale")] + \
               [("n", C.c_int64), ("weight_decay", C.c_float)]


class AdamwDesc(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps")] + \
               [(n, C.c_int32) for n in ("step", "p_dtype", "g_dtype", "state_bits")] + [("seed", C.c_uint32)] + \
               [("grad_scale", C.c_float), ("max_norm", C.c_float)] + [(n, C.c_void_p) for n in ("norm_dev", "step_dev", "lr_dev")]


_lib = None


def lib() -> C.CDLL:
    """Load libcentrifuge.so (built by paper_2502_00340_amd.build).  Raises if missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("HIP library not built: %s is missing (run __graft_entry__.build())" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    L.cf_status_str.restype = C.c_char_p
    L.cf_status_str.argtypes = [C.c_int]
    L.cf_version.restype = C.c_char_p
    L.cf_version.argtypes = []
    L.cf_index_workspace_bytes.restype = sz
    L.cf_index_workspace_bytes.argtypes = [i64]
    L.cf_build_keep_index.restype = C.c_int
    L.cf_build_keep_index.argtypes = [vp, i32, i32, vp, vp, vp, C.POINTER(i32), vp, sz, vp]
    L.cf_build_keep_index_static.restype = C.c_int
    L.cf_build_keep_index_static.argtypes = [vp, i32, i32, vp, vp, vp, vp]
    L.cf_gather_rows.restype = C.c_int
    L.cf_gather_rows.argtypes = [vp, i64, i64, i32, vp, vp, i32, vp, vp]
    L.cf_linear_bwd_reduced.restype = C.c_int
    L.cf_linear_bwd_reduced.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp, f32, vp]
    L.cf_linear_workspace_bytes.restype = sz
    L.cf_linear_workspace_bytes.argtypes = [i32, i32, i32, i32]
    L.cf_linear_bwd_reduced_ws.restype = C.c_int
    L.cf_linear_bwd_reduced_ws.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp, f32, vp, sz, vp]
    L.cf_attn_workspace_bytes.restype = sz
    L.cf_attn_workspace_bytes.argtypes = [C.POINTER(LayerDesc), i32]
    L.cf_attn_bwd_filtered.restype = C.c_int
    L.cf_attn_bwd_filtered.argtypes = [C.POINTER(LayerDesc), vp, vp, vp, vp, vp, vp, vp, vp, i32,
                                       vp, vp, vp, vp, sz, vp]
    L.cf_layer_workspace_bytes.restype = sz
    L.cf_layer_workspace_bytes.argtypes = [C.POINTER(LayerDesc), i32]
    L.cf_layer_bwd_filtered.restype = C.c_int
    L.cf_layer_bwd_filtered.argtypes = [C.POINTER(LayerDesc), C.POINTER(Saved), C.POINTER(Weights), vp, vp, i32,
                                        C.POINTER(Grads), vp, vp, vp, C.POINTER(i32), vp, sz, vp]
    L.cf_layer_bwd_compact_dev.restype = C.c_int
    L.cf_layer_bwd_compact_dev.argtypes = [C.POINTER(LayerDesc), C.POINTER(Saved), C.POINTER(Weights), vp, vp, vp,
                                           vp, i32, C.POINTER(Grads), vp, sz, vp]
    L.cf_layer_bwd_compact.restype = C.c_int
    L.cf_layer_bwd_compact.argtypes = [C.POINTER(LayerDesc), C.POINTER(Saved), C.POINTER(Weights), vp, vp, vp,
                                       i32, C.POINTER(Grads), vp, sz, vp]
    L.cf_layer_bwd_dense.restype = C.c_int
    L.cf_layer_bwd_dense.argtypes = [C.POINTER(LayerDesc), C.POINTER(Saved), C.POINTER(Weights), vp,
                                     C.POINTER(Grads), vp, sz, vp]
    L.cf_lora_workspace_bytes.restype = sz
    L.cf_lora_workspace_bytes.argtypes = [C.POINTER(LayerDesc), i32, i32]
    L.cf_layer_bwd_lora.restype = C.c_int
    L.cf_layer_bwd_lora.argtypes = [C.POINTER(LayerDesc), C.POINTER(Saved), C.POINTER(Weights), C.POINTER(Lora), vp,
                                    vp, i32, C.POINTER(LoraGrads), vp, vp, vp, C.POINTER(i32), vp, sz, vp]
    L.cf_probe_mfma_bf16.restype = C.c_int
    L.cf_probe_mfma_bf16.argtypes = [i32, i32, vp, C.POINTER(C.c_double), vp]
    L.cf_probe_mfma_lds_bf16.restype = C.c_int
    L.cf_probe_mfma_lds_bf16.argtypes = [i32, i32, i32, vp, C.POINTER(C.c_double), vp]
    L.cf_probe_copy.restype = C.c_int
    L.cf_probe_copy.argtypes = [vp, vp, sz, vp]
    desc, qk, qkn = C.POINTER(LayerDesc), C.POINTER(Qk), C.POINTER(QkNorm)
    layer = [desc, C.POINTER(Saved), C.POINTER(Weights), C.POINTER(LayerQk)]
    for name, res, args in (
            ("cf_qk_norm_rope_fwd", C.c_int, [desc, qkn, qk, i32, qk, vp]),
            ("cf_qk_norm_workspace_bytes", sz, [desc, i32]),
            ("cf_qk_norm_rope_bwd", C.c_int, [desc, qkn, qk, qk, vp, vp, i32, qk, vp, vp, i32, vp, sz, vp]),
            ("cf_layer_qk_workspace_bytes", sz, [desc, i32]),
            ("cf_lora_qk_workspace_bytes", sz, [desc, i32, i32]),
            ("cf_layer_bwd_filtered_qk", C.c_int, layer + [vp, vp, i32, C.POINTER(Grads), vp, vp, vp, C.POINTER(i32), vp, sz, vp]),
            ("cf_layer_bwd_compact_qk", C.c_int, layer + [vp, vp, vp, vp, i32, C.POINTER(Grads), vp, sz, vp]),
            ("cf_layer_bwd_dense_qk", C.c_int, layer + [vp, C.POINTER(Grads), vp, sz, vp]),
            ("cf_layer_bwd_lora_qk", C.c_int, layer + [C.POINTER(Lora), vp, vp, i32, C.POINTER(LoraGrads), vp, vp, vp, C.POINTER(i32),
                                                       vp, sz, vp]),
            ("cf_token_loss_workspace_bytes", sz, [i32]),
            ("cf_token_loss", C.c_int, [C.POINTER(LossDesc), vp, i64, vp, vp, vp, vp, vp, vp, vp, i32, vp, i64, vp, vp, vp, sz, vp]),
            ("cf_adamw_step", C.c_int, [C.POINTER(AdamwDesc), C.POINTER(AdamwTensor), i32, vp]),
            ("cf_grad_norm_workspace_bytes", sz, [i32]),
            ("cf_grad_norm", C.c_int, [C.POINTER(vp), C.POINTER(i64), i32, i32, f32, vp, vp, sz, vp])):
        getattr(L, name).restype, getattr(L, name).argtypes = res, args
    _lib = L
    return L


def _check(code: int, where: str):
    if code != 0:
        raise CfError(code, where)


_dummy = {}


def _ptr(t):
    """Device address of a tensor as a plain int (the declared argument types make it a pointer; a ctypes object of its
    own would only cost time); an empty tensor (no storage) maps to a small dummy allocation so that "zero rows" is not
    mistaken for a NULL argument."""
    if t is None:
        return None
    if t.numel() == 0:
        key = str(t.device)
        if key not in _dummy:
            _dummy[key] = torch.zeros(256, dtype=torch.uint8, device=t.device)
        return _dummy[key].data_ptr()
    return t.data_ptr()


def _addr(t):
    return None if t is None else t.data_ptr()


# torch's raw query of a device's current stream, absent from torch's public interface
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: int | None = None):
    """Handle of the current device's current stream, read on every call; device: its number, where the caller has just asked
    for it.  The raw query costs 0.1 us where building a torch.cuda.Stream object for it costs 2.8 us, a fifth of the
    smallest calls; a torch without it builds the object."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device() if device is None else device)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return CF_BF16
    if t.dtype == torch.float32:
        return CF_F32
    raise TypeError("unsupported dtype %s" % t.dtype)


def make_desc(B, S, H, Hq, Hkv, d, F, dtype, rms_eps=1e-5, softmax_scale=0.0) -> LayerDesc:
    code = {"bf16": CF_BF16, "f32": CF_F32, torch.bfloat16: CF_BF16, torch.float32: CF_F32}[dtype]
    return LayerDesc(B, S, H, Hq, Hkv, d, F, code, rms_eps, softmax_scale)


def torch_dtype(desc: LayerDesc):
    return torch.bfloat16 if desc.dtype == CF_BF16 else torch.float32


# --------------------------------------------------------------------------
# entry points (same names as the C ABI, without the prefix)
# --------------------------------------------------------------------------

_INDEX_NO_SCRATCH = 32768       # CF_INDEX_NO_SCRATCH_TOKENS of the header


def build_keep_index(mask: torch.Tensor, sync: bool = True):
    """mask: uint8 [B,S] on the GPU.  Returns (idx [T] int32 - first N_k valid,
    cu_kept [B+1] int32, n_kept_dev [1] int32, N_k or None)."""
    assert mask.dtype == torch.uint8 and mask.is_cuda and mask.dim() == 2 and mask.is_contiguous()
    B, S = mask.shape
    dev = mask.device
    idx = torch.empty(B * S, dtype=torch.int32, device=dev)
    cu = torch.empty(B + 1, dtype=torch.int32, device=dev)
    n_dev = torch.empty(1, dtype=torch.int32, device=dev)
    if not sync and 0 < B * S <= _INDEX_NO_SCRATCH:
        # one launch that touches neither a workspace nor the library's array: nothing to allocate for it or to share
        # (a layer's mask 11.9 -> 9.9 us, of which three allocations are 4 and the launch 3)
        _check((_lib or lib()).cf_build_keep_index_static(mask.data_ptr(), B, S, idx.data_ptr(), cu.data_ptr(), n_dev.data_ptr(),
                                                          _stream()), "cf_build_keep_index_static")
        return idx, cu, n_dev, None
    wsb = lib().cf_index_workspace_bytes(B * S)
    ws = torch.empty(wsb, dtype=torch.uint8, device=dev)
    n_host = C.c_int32(-1) if sync else None
    _check(lib().cf_build_keep_index(_ptr(mask), B, S, _ptr(idx), _ptr(cu), _ptr(n_dev),
                                     C.byref(n_host) if sync else None, _ptr(ws), wsb, _stream()),
           "cf_build_keep_index")
    return idx, cu, n_dev, (int(n_host.value) if sync else None)


def build_keep_index_static(mask: torch.Tensor, idx: torch.Tensor, cu_kept: torch.Tensor, n_kept_dev: torch.Tensor):
    """cf_build_keep_index_static: every buffer is the caller's, nothing is allocated or read back."""
    assert mask.dtype == torch.uint8 and mask.is_cuda and mask.dim() == 2 and mask.is_contiguous()
    B, S = mask.shape
    assert idx.dtype == torch.int32 and idx.numel() >= B * S and cu_kept.numel() >= B + 1
    _check(lib().cf_build_keep_index_static(_ptr(mask), B, S, _ptr(idx), _ptr(cu_kept), _ptr(n_kept_dev),
                                            _stream()), "cf_build_keep_index_static")


def gather_rows(src: torch.Tensor, idx: torch.Tensor, n_rows: int, out: torch.Tensor | None = None,
                n_kept_dev: torch.Tensor | None = None):
    """n_kept_dev None: exactly n_rows rows.  Otherwise min(*n_kept_dev, n_rows) rows are copied (the
    count is read on the device) and `out` has room for n_rows."""
    assert src.is_cuda and src.dim() == 2 and src.is_contiguous() and idx.dtype == torch.int32
    rows, cols = src.shape
    if out is None:
        out = torch.empty((n_rows, cols), dtype=src.dtype, device=src.device)
    _check(lib().cf_gather_rows(_ptr(src), rows, cols, _dtype_code(src), _ptr(idx), _ptr(n_kept_dev), n_rows,
                                _ptr(out), _stream()), "cf_gather_rows")
    return out


@functools.lru_cache(maxsize=1024)
def _linear_ws_bytes(n_kept, in_f, out_f, code, device):
    """A function of the sizes and of the current device, whose compute units the library asks for."""
    return lib().cf_linear_workspace_bytes(n_kept, in_f, out_f, code)


def linear_bwd_reduced(x_kept, dy_kept, w, need_dx=True, need_dw=True, dw_accumulate_into=None):
    """Returns (dx_kept or None, dw or None)."""
    n_kept, out_f = dy_kept.shape
    in_f = w.shape[0] if w is not None else x_kept.shape[1]
    dev = dy_kept.device
    dx = torch.empty((n_kept, in_f), dtype=dy_kept.dtype, device=dev) if need_dx else None
    beta = 0.0
    dw = None
    if need_dw:
        if dw_accumulate_into is not None:
            dw, beta = dw_accumulate_into, 1.0
        else:
            dw = torch.empty((in_f, out_f), dtype=dy_kept.dtype, device=dev)
    code = _dtype_code(dy_kept)
    device = torch.cuda.current_device()
    wsb = _linear_ws_bytes(n_kept, in_f, out_f, code, device) if need_dx else 0
    ws = torch.empty(wsb, dtype=torch.uint8, device=dev) if wsb else None
    at = _addr if n_kept and in_f and out_f else _ptr          # with all sizes no tensor is empty
    _check((_lib or lib()).cf_linear_bwd_reduced_ws(at(x_kept), at(dy_kept), at(w), n_kept, in_f, out_f, code, at(dx), at(dw),
                                                    beta, _addr(ws), wsb, _stream(device)), "cf_linear_bwd_reduced")
    return dx, dw


def attn_bwd_filtered(desc: LayerDesc, q_kept, k_full, v_full, o_kept, lse_full, do_kept, idx, cu_kept,
                      n_kept: int):
    dev = q_kept.device
    Nq, Nkv = desc.Hq * desc.d, desc.Hkv * desc.d
    dt = torch_dtype(desc)
    dq = torch.empty((n_kept, Nq), dtype=dt, device=dev)
    dk = torch.empty((n_kept, Nkv), dtype=dt, device=dev)
    dv = torch.empty((n_kept, Nkv), dtype=dt, device=dev)
    wsb = lib().cf_attn_workspace_bytes(C.byref(desc), n_kept)
    ws = torch.empty(max(wsb, 256), dtype=torch.uint8, device=dev)
    _check(lib().cf_attn_bwd_filtered(C.byref(desc), _ptr(q_kept), _ptr(k_full), _ptr(v_full), _ptr(o_kept),
                                      _ptr(lse_full), _ptr(do_kept), _ptr(idx), _ptr(cu_kept), n_kept,
                                      _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), ws.numel(), _stream()),
           "cf_attn_bwd_filtered")
    return dq, dk, dv


_SAVED = ("x", "q", "k", "v", "attn_out", "lse", "r", "gate", "up")
_WEIGHTS = ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")


class LayerBackward:
    """Pre-allocated outputs + workspace for repeated calls on one layer shape."""

    def __init__(self, desc: LayerDesc, device="cuda:0", max_kept: int | None = None, main_grad: bool = False,
                 qk_norm_eps: float | None = None):
        """main_grad: the parameter gradients are fp32 buffers, zeroed here, that every call adds to.  qk_norm_eps: the layer normalises its
        query and key heads; saved then holds q_pre and k_pre as well, weights gq and gk, and the gradients dgq and dgk."""
        self.desc = desc
        self.device = torch.device(device)
        dt = torch_dtype(desc)
        T = desc.B * desc.S
        H, F, Nq, Nkv = desc.H, desc.F, desc.Hq * desc.d, desc.Hkv * desc.d
        self.max_kept = T if max_kept is None else max_kept
        e = lambda *s: torch.empty(s, dtype=dt, device=self.device)
        p = (lambda *s: torch.zeros(s, dtype=torch.float32, device=self.device)) if main_grad else e
        self.grads = dict(dwq=p(H, Nq), dwk=p(H, Nkv), dwv=p(H, Nkv), dwo=p(Nq, H), dwg=p(H, F), dwu=p(H, F),
                          dwd=p(F, H), dg1=p(H), dg2=p(H), dx=e(T, H))
        self.qk_norm_eps = qk_norm_eps
        if qk_norm_eps is not None:
            self.grads.update(dgq=p(desc.d), dgk=p(desc.d))
        # zeros, not empty: entries past N_k are never written, and must stay valid row numbers for a
        # caller that passes a wrong count to filtered_known
        self.idx = torch.zeros(T, dtype=torch.int32, device=self.device)
        self.cu_kept = torch.empty(desc.B + 1, dtype=torch.int32, device=self.device)
        size = lib().cf_layer_workspace_bytes if qk_norm_eps is None else lib().cf_layer_qk_workspace_bytes
        self.ws_bytes = size(C.byref(desc), self.max_kept)
        if self.ws_bytes == 0:
            raise CfError(2, "cf_layer_workspace_bytes")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self._g = Grads(*([self.grads[n].data_ptr() for n in GRAD_NAMES] + [1 if main_grad else 0]))
        self.n_kept_dev = torch.zeros(1, dtype=torch.int32, device=self.device)
        # N_k comes back through page-locked host memory: the copy is asynchronous
        self._n_host = torch.empty(1, dtype=torch.int32).pin_memory()

    def _pack(self, saved: dict, weights: dict):
        rope = [saved[n].data_ptr() if saved.get(n) is not None else None for n in ("rope_cos", "rope_sin")]
        sv = Saved(*([saved[n].data_ptr() for n in _SAVED] + rope))
        w = Weights(*[weights[n].data_ptr() for n in _WEIGHTS])
        return sv, w

    def _call(self, name: str, saved: dict, weights: dict, *args):
        """cf_<name>, or cf_<name>_qk for a layer with query/key norm, with the arguments behind the weights."""
        sv, w = self._pack(saved, weights)
        if self.qk_norm_eps is None:
            _check(getattr(lib(), "cf_" + name)(C.byref(self.desc), C.byref(sv), C.byref(w), *args), "cf_" + name)
            return
        name = {"layer_bwd_compact_dev": "layer_bwd_compact"}.get(name, name) + "_qk"
        D, dt = self.desc, torch_dtype(self.desc)
        ts = saved["q_pre"], saved["k_pre"], weights["gq"], weights["gk"]
        for t, n in zip(ts, (D.B * D.S * D.Hq * D.d, D.B * D.S * D.Hkv * D.d, D.d, D.d)):
            if t.dtype is not dt or t.numel() != n or not t.is_contiguous():
                raise ValueError("q_pre, k_pre, gq and gk have to be contiguous and %s, like what the layer's call reads beside them" % dt)
        qk = LayerQk(*[t.data_ptr() for t in ts], self.qk_norm_eps,
                     _addr(self.grads.get("dgq")), _addr(self.grads.get("dgk")))
        _check(getattr(lib(), "cf_" + name)(C.byref(self.desc), C.byref(sv), C.byref(w), C.byref(qk), *args), "cf_" + name)

    def filtered_async(self, saved: dict, weights: dict, dy: torch.Tensor, mask: torch.Tensor) -> None:
        """Enqueues cf_layer_bwd_filtered and returns at once: nothing is read back and the stream is
        not synchronised.  Results land in self.grads (dx: first N_k rows), self.idx, self.cu_kept,
        self.n_kept_dev; the page-locked word behind n_kept() holds N_k once the stream has run."""
        self._n_host[0] = -1
        self._call("layer_bwd_filtered", saved, weights, _ptr(dy), _ptr(mask), self.max_kept, C.byref(self._g), _ptr(self.idx),
                   _ptr(self.cu_kept), _ptr(self.n_kept_dev), C.cast(self._n_host.data_ptr(), C.POINTER(C.c_int32)), _ptr(self.ws),
                   self.ws_bytes, _stream())

    def n_kept(self) -> int:
        """N_k of the last filtered call (synchronises the current stream)."""
        torch.cuda.current_stream().synchronize()
        return int(self._n_host[0])

    def filtered(self, saved: dict, weights: dict, dy: torch.Tensor, mask: torch.Tensor) -> int:
        """filtered_async, then waits for the stream and returns N_k."""
        self.filtered_async(saved, weights, dy, mask)
        return self.n_kept()

    def filtered_known(self, saved: dict, weights: dict, dy: torch.Tensor, mask: torch.Tensor, n_kept: int) -> None:
        """The filtered backward composed from the single-purpose calls by a caller that knows N_k
        beforehand (a fixed keep ratio: top-k per sequence gives N_k = B*k): cf_build_keep_index
        without the host copy, cf_gather_rows of the upstream gradient, cf_layer_bwd_compact with the
        host count.  n_kept must be the number of non-zero mask bytes."""
        if not hasattr(self, "_index_ws"):
            wsb = lib().cf_index_workspace_bytes(self.desc.B * self.desc.S)
            self._index_ws = torch.empty(wsb, dtype=torch.uint8, device=self.device)
            self._dy_kept = torch.empty((self.desc.B * self.desc.S, self.desc.H), dtype=dy.dtype, device=self.device)
        _check(lib().cf_build_keep_index(_ptr(mask), self.desc.B, self.desc.S, _ptr(self.idx), _ptr(self.cu_kept),
                                         _ptr(self.n_kept_dev), None, _ptr(self._index_ws), self._index_ws.numel(),
                                         _stream()), "cf_build_keep_index")
        _check(lib().cf_gather_rows(_ptr(dy), dy.shape[0], dy.shape[1], _dtype_code(dy), _ptr(self.idx), None, n_kept,
                                    _ptr(self._dy_kept), _stream()), "cf_gather_rows")
        self.compact(saved, weights, self._dy_kept, self.idx, self.cu_kept, n_kept)

    def compact_dev(self, saved: dict, weights: dict, dy_kept: torch.Tensor, idx: torch.Tensor,
                    cu_kept: torch.Tensor, n_kept_dev: torch.Tensor) -> None:
        """cf_layer_bwd_compact_dev: a layer below the index-building one, with the count still on the
        device (no host read anywhere in the stack)."""
        self._call("layer_bwd_compact_dev", saved, weights, _ptr(dy_kept), _ptr(idx), _ptr(cu_kept), _ptr(n_kept_dev), self.max_kept,
                   C.byref(self._g), _ptr(self.ws), self.ws_bytes, _stream())

    def compact(self, saved: dict, weights: dict, dy_kept: torch.Tensor, idx: torch.Tensor,
                cu_kept: torch.Tensor, n_kept: int) -> None:
        """Runs cf_layer_bwd_compact for a layer below the one that built (idx, cu_kept); results
        land in self.grads (dx: first n_kept rows).  No host synchronisation."""
        count = (n_kept,) if self.qk_norm_eps is None else (None, n_kept)
        self._call("layer_bwd_compact", saved, weights, _ptr(dy_kept), _ptr(idx), _ptr(cu_kept), *count, C.byref(self._g), _ptr(self.ws),
                   self.ws_bytes, _stream())

    def dense(self, saved: dict, weights: dict, dy: torch.Tensor) -> None:
        self._call("layer_bwd_dense", saved, weights, _ptr(dy), C.byref(self._g), _ptr(self.ws), self.ws_bytes, _stream())


def layer_bwd_filtered(desc, saved, weights, dy, mask):
    plan = LayerBackward(desc, device=dy.device)
    n = plan.filtered(saved, weights, dy, mask)
    out = dict(plan.grads)
    out["dx"] = out["dx"][:n]
    return out, plan.idx[:n], plan.cu_kept, n


def layer_bwd_dense(desc, saved, weights, dy):
    plan = LayerBackward(desc, device=dy.device)
    plan.dense(saved, weights, dy)
    return dict(plan.grads)


class LoraBackward(LayerBackward):
    """Pre-allocated adapter gradients + workspace for cf_layer_bwd_lora (base weights frozen)."""

    def __init__(self, desc: LayerDesc, rank: int, device="cuda:0", qk_norm_eps: float | None = None):
        self.desc = desc
        self.qk_norm_eps = qk_norm_eps
        self.device = torch.device(device)
        self.rank = rank
        dt = torch_dtype(desc)
        T = desc.B * desc.S
        H, Nq, Nkv = desc.H, desc.Hq * desc.d, desc.Hkv * desc.d
        e = lambda *s: torch.empty(s, dtype=dt, device=self.device)
        self.grads = dict(daq=e(H, rank), dbq=e(rank, Nq), dak=e(H, rank), dbk=e(rank, Nkv), dav=e(H, rank),
                          dbv=e(rank, Nkv), dao=e(Nq, rank), dbo=e(rank, H), dx=e(T, H))
        # zeros, not empty: entries past N_k are never written, and must stay valid row numbers for a
        # caller that passes a wrong count to filtered_known
        self.idx = torch.zeros(T, dtype=torch.int32, device=self.device)
        self.cu_kept = torch.empty(desc.B + 1, dtype=torch.int32, device=self.device)
        size = lib().cf_lora_workspace_bytes if qk_norm_eps is None else lib().cf_lora_qk_workspace_bytes
        self.ws_bytes = size(C.byref(desc), rank, T)
        if self.ws_bytes == 0:
            raise CfError(2, "cf_lora_workspace_bytes")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self._g = LoraGrads(*[self.grads[n].data_ptr() for n, _ in LoraGrads._fields_])
        self.max_kept = T
        self.n_kept_dev = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._n_host = torch.empty(1, dtype=torch.int32).pin_memory()

    def run_async(self, saved: dict, weights: dict, lora: dict, dy: torch.Tensor, mask: torch.Tensor | None) -> None:
        """mask None: every token kept (the dense LoRA backward).  Nothing synchronises: the kept count is
        in self.n_kept_dev, and n_kept() reads the page-locked copy after waiting for the stream."""
        lo = Lora(*([lora[n].data_ptr() for n in _LORA_T] + [self.rank, float(lora["scale"])]))
        self._n_host[0] = -1
        self._call("layer_bwd_lora", saved, weights, C.byref(lo), _ptr(dy), _ptr(mask), self.max_kept, C.byref(self._g), _ptr(self.idx),
                   _ptr(self.cu_kept), _ptr(self.n_kept_dev), C.cast(self._n_host.data_ptr(), C.POINTER(C.c_int32)), _ptr(self.ws),
                   self.ws_bytes, _stream())

    def run(self, saved: dict, weights: dict, lora: dict, dy: torch.Tensor, mask: torch.Tensor | None) -> int:
        """run_async, then waits for the stream and returns N_k."""
        self.run_async(saved, weights, lora, dy, mask)
        torch.cuda.current_stream().synchronize()
        return int(self._n_host[0])


# --------------------------------------------------------------------------
# around the layer calls: query/key norm with rotation, losses, AdamW
# --------------------------------------------------------------------------

def _need(ok, what: str):
    if not ok:
        raise ValueError(what)


def _on(tensors):
    """Every tensor given (None apart) lies on the current GPU: the library launches on its current stream.  Returns its number."""
    now = torch.cuda.current_device() if torch.cuda.is_initialized() else -2
    for t in tensors:
        if t is not None and t.get_device() != now:
            raise ValueError("a tensor is on %s, not on the current GPU" % t.device)
    return now


def _qk_rows(desc: LayerDesc, q, k, what: str, dtype, Nq: int, Nkv: int):
    """A cf_qk of q [n, Nq] and k [n, Nkv]: dense columns, any stride from row to row."""
    if q.dim() == 2 and k.dim() == 2:
        (n, w), (m, x), a, b = q.shape, k.shape, q.stride(), k.stride()
        if w == Nq and x == Nkv and n == m and q.dtype is dtype and k.dtype is dtype:
            if n > 1 and a[1] == 1 and b[1] == 1 and a[0] >= w and b[0] >= x:
                return n, Qk(q.data_ptr(), k.data_ptr(), a[0], b[0])
            if n == 0 or n == 1 and a[1] == 1 and b[1] == 1:
                return n, Qk(_ptr(q), _ptr(k), 0, 0)           # the stride of a single row means nothing
    raise ValueError("%s: expected %s [rows, %d] and [rows, %d] with dense columns, got %s %s, strides %s, and %s %s, strides %s" %
                     (what, dtype, Nq, Nkv, q.dtype, tuple(q.shape), q.stride(), k.dtype, tuple(k.shape), k.stride()))


def _qk_norm(desc: LayerDesc, d: int, gq, gk, rope_cos, rope_sin, positions, rows: int, dtype):
    for g in (gq, gk):
        if g.dtype is not dtype or g.dim() != 1 or g.shape[0] != d or not g.is_contiguous():
            raise ValueError("gains have to be %s [%d]" % (dtype, d))
    if rope_cos is not None or rope_sin is not None:
        for t in (rope_cos, rope_sin):
            if t is None or t.dtype is not torch.float32 or t.shape != (desc.S, d // 2) or not t.is_contiguous():
                raise ValueError("rope_cos and rope_sin have to be fp32 [%d, %d], contiguous, both or neither" % (desc.S, d // 2))
    if positions is not None and (positions.dtype is not torch.int32 or not positions.is_contiguous() or positions.numel() < rows):
        raise ValueError("positions have to be int32, contiguous, one per row")
    return QkNorm(gq.data_ptr(), gk.data_ptr(), _addr(rope_cos), _addr(rope_sin), None if positions is None else _ptr(positions))


def qk_norm_rope_fwd(desc: LayerDesc, q, k, gq, gk, rope_cos=None, rope_sin=None, positions=None, out=None):
    """Norm of every query and key head and its rotation at positions[row] (row mod S without positions).  q [n, Hq*d] and k [n, Hkv*d] may be columns
    of a longer row (a fused projection).  out: a pair to write to, q and k themselves for a pass in place."""
    dt, d = torch_dtype(desc), desc.d
    Nq, Nkv = desc.Hq * d, desc.Hkv * d
    n, rows = _qk_rows(desc, q, k, "q, k", dt, Nq, Nkv)
    p = _qk_norm(desc, d, gq, gk, rope_cos, rope_sin, positions, n, dt)
    if out is None:
        out = torch.empty_like(q), torch.empty_like(k)
    m, to = _qk_rows(desc, out[0], out[1], "out", dt, Nq, Nkv)
    _need(m == n, "out has another number of rows")
    device = _on((q, k, gq, gk, rope_cos, rope_sin, positions, *out))
    _check((_lib or lib()).cf_qk_norm_rope_fwd(C.byref(desc), C.byref(p), C.byref(rows), n, C.byref(to), _stream(device)), "cf_qk_norm_rope_fwd")
    return out


def _kept_count(idx, n_kept_dev, rows: int, kept: int):
    _need(idx is None or (idx.dtype == torch.int32 and idx.is_contiguous() and idx.numel() >= kept), "idx has to be int32, one per kept row")
    _need(idx is not None or kept <= rows, "without idx there are at most %d rows" % rows)
    _need(kept == 0 or rows > 0, "kept rows of an empty tensor")
    _need(n_kept_dev is None or (n_kept_dev.dtype == torch.int32 and n_kept_dev.numel() == 1), "n_kept_dev has to be one int32")


@functools.lru_cache(maxsize=1024)
def _qk_ws_bytes(d, code, n):
    return lib().cf_qk_norm_workspace_bytes(C.byref(LayerDesc(1, 1, 8, 1, 1, d, 8, code, 0.0, 0.0)), n)


def _ranges_meet(a, b) -> bool:
    """Whether the addresses from the first to the last element of two tensors meet."""
    end = lambda t: t.data_ptr() + (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))) * t.element_size()
    return a.numel() > 0 and b.numel() > 0 and a.data_ptr() < end(b) and b.data_ptr() < end(a)


def qk_norm_rope_bwd(desc: LayerDesc, q, k, gq, gk, dq, dk, rope_cos=None, rope_sin=None, positions=None, idx=None, n_kept_dev=None,
                     need_gains: bool = True, main_grads=None, out=None):
    """Backward of qk_norm_rope_fwd for compact dq [n, Hq*d], dk [n, Hkv*d]; q and k are its inputs at full length.  Returns (dx of q, dx of k, dgq, dgk).
    n_kept_dev: only the first min(*n_kept_dev, n) rows.  main_grads: fp32 (dgq, dgk) that are added to.  out: a pair to write to, dq and dk themselves for a
    pass in place."""
    dt, d = torch_dtype(desc), desc.d
    Nq, Nkv = desc.Hq * d, desc.Hkv * d
    rows, x = _qk_rows(desc, q, k, "q, k", dt, Nq, Nkv)
    n, dy = _qk_rows(desc, dq, dk, "dq, dk", dt, Nq, Nkv)
    _kept_count(idx, n_kept_dev, rows, n)
    p = _qk_norm(desc, d, gq, gk, rope_cos, rope_sin, positions, rows, dt)
    if out is None:
        out = torch.empty_like(dq), torch.empty_like(dk)
    elif idx is not None:
        for t in out:
            _need(not any(_ranges_meet(t, x) for x in (q, k)), "with idx, out must not overlap q and k")
    m, dx = _qk_rows(desc, out[0], out[1], "out", dt, Nq, Nkv)
    _need(m == n, "out has another number of rows")
    dgq = dgk = ws = None
    wsb = 0
    if main_grads is not None:
        dgq, dgk = main_grads
        for t in main_grads:
            _need(t.dtype is torch.float32 and t.shape == (d,) and t.is_contiguous(), "main_grads have to be fp32 [%d]" % d)
    elif need_gains:
        dgq, dgk = torch.empty_like(gq), torch.empty_like(gk)
    if dgq is not None:
        wsb = _qk_ws_bytes(d, desc.dtype, n)
        ws = torch.empty(wsb, dtype=torch.uint8, device=dq.device)
    device = _on((q, k, gq, gk, dq, dk, rope_cos, rope_sin, positions, idx, n_kept_dev, dgq, dgk, *out))
    _check((_lib or lib()).cf_qk_norm_rope_bwd(C.byref(desc), C.byref(p), C.byref(x), C.byref(dy), None if idx is None else _ptr(idx),
                                               _addr(n_kept_dev), n, C.byref(dx), _addr(dgq), _addr(dgk), int(main_grads is not None),
                                               _addr(ws), wsb, _stream(device)), "cf_qk_norm_rope_bwd")
    return out[0], out[1], dgq, dgk


def token_loss(logits, targets, old_logp=None, advantages=None, ref_logp=None, weights=None, clip=(0.2, 0.2), kl_coef: float = 0.0,
               logit_scale: float = 1.0, norm: float = 0.0, idx=None, n_kept_dev=None, max_kept: int | None = None, need_grad: bool = True, out=None):
    """Loss of the kept rows of logits [rows, V] (dense columns, any stride) and its gradient: the mean NLL of targets [rows] int64, or with advantages
    the clipped policy loss.  Per-row tensors are fp32 [rows] and read, like logits, at idx[j] (row j without idx).  Returns (stats [4]: loss, its first term, KL, clipped share;
    logp [max_kept]; dlogits [max_kept, V] or None).  max_kept: by default all of idx, or all rows.  out: dlogits to write to,
    logits itself for a gradient in place (without idx).  n_kept_dev: only the first min(*n_kept_dev, max_kept) rows are written; the others hold what they
    held, so a product over all max_kept rows wants a cleared out."""
    _need(logits.dim() == 2, "logits have to be [rows, V]")
    (rows, V), (ls, dense) = logits.shape, logits.stride()
    _need((dense == 1 or V == 1) and (ls >= V or rows < 2), "logits have to have dense columns, and rows that do not overlap")
    n = max_kept if max_kept is not None else rows if idx is None else idx.numel()
    _kept_count(idx, n_kept_dev, rows, n)
    _need(targets.dtype is torch.int64 and targets.shape == (rows,) and targets.is_contiguous(), "targets have to be int64 [%d]" % rows)
    policy = advantages is not None
    _need(policy or (old_logp is None and ref_logp is None), "old_logp and ref_logp belong to a loss with advantages")
    for t in (old_logp, advantages, ref_logp, weights):
        if t is not None and not (t.dtype is torch.float32 and t.shape == (rows,) and t.is_contiguous()):
            raise ValueError("old_logp, advantages, ref_logp and weights have to be fp32 [%d]" % rows)
    code = _dtype_code(logits)
    ds, dev = 0, logits.device
    if out is not None:
        _need(out.dim() == 2 and out.dtype is logits.dtype and out.shape[0] >= n and out.shape[1] == V and (out.stride(1) == 1 or V == 1),
              "out has to be %s [%d, %d] with dense columns" % (logits.dtype, n, V))
        ds = out.stride(0) if out.shape[0] > 1 else 0
        _need(out.shape[0] < 2 or ds >= V, "rows of out must not overlap")
        if idx is not None and n:
            a, b, e = logits.data_ptr(), out.data_ptr(), logits.element_size()
            _need(a >= b + ((n - 1) * ds + V) * e or b >= a + ((rows - 1) * ls + V) * e, "with idx, out must not overlap logits")
    elif need_grad:
        out = torch.empty((n, V), dtype=logits.dtype, device=dev)
    device = _on((logits, targets, old_logp, advantages, ref_logp, weights, idx, n_kept_dev, out))
    logp = torch.empty(n, dtype=torch.float32, device=dev)
    stats = torch.empty(4, dtype=torch.float32, device=dev)
    ws = torch.empty((16 * n + 256) // 256 * 256, dtype=torch.uint8, device=dev)        # cf_token_loss_workspace_bytes(n) or more: the call compares
    d = LossDesc(CF_LOSS_POLICY if policy else CF_LOSS_NLL, V, code, logit_scale, clip[0], clip[1], kl_coef, norm)
    _check((_lib or lib()).cf_token_loss(C.byref(d), _ptr(logits), ls if rows > 1 else 0, _ptr(targets), _addr(old_logp), _addr(ref_logp),
                                         _addr(advantages), _addr(weights), None if idx is None else _ptr(idx), _addr(n_kept_dev), n,
                                         None if out is None else _ptr(out), ds, _ptr(logp), stats.data_ptr(), ws.data_ptr(), ws.numel(),
                                         _stream(device)), "cf_token_loss")
    return stats, logp, out


STATE_BLOCK = 256       # elements that share a scale of an 8-bit state


def adamw_state_values(q: torch.Tensor, scale: torch.Tensor):
    """The fp32 values that an 8-bit state stands for (of v: its square root)."""
    n = q.numel()
    return (q.reshape(-1).float() * scale.repeat_interleave(STATE_BLOCK)[:n]).view(q.shape)


class AdamW:
    """AdamW over a list of parameters and the list of their gradients (LayerBackward.grads, main gradients or not; contiguous, one dtype each).  The plan
    keeps the tensors' addresses: gradients are new values in the same buffers.  One call at a time: its norm and workspace are its own."""

    def __init__(self, params, grads, lr: float, betas=(0.9, 0.95), eps: float = 1e-8, weight_decay=0.0, max_norm: float | None = None,
                 grad_scale: float = 1.0, state_bits: int = 32, master=None, state=None, seed: int = 0, step_dev=None, lr_dev=None):
        """weight_decay: a number, or one per parameter.  max_norm: clip by the global norm, which step() leaves in grad_norm; a norm that is not
        finite leaves everything unchanged.  master: None, True (made here from bf16 parameters) or a list of fp32 copies.  state: lists (m, v) in
        fp32 or (m, v, m_scale, v_scale) in 8 bits; None: zeros of state_bits.  step_dev, lr_dev: int32 / fp32 tensors that replace step() 's own
        count and lr, for steps captured into a graph."""
        self.params, self.grads_list = list(params), list(grads)
        n = len(self.params)
        _need(n > 0 and n == len(self.grads_list), "one gradient per parameter, and at least one")
        self.device = dev = self.params[0].device
        p_dt, g_dt = self.params[0].dtype, self.grads_list[0].dtype
        size = [p.numel() for p in self.params]
        self.master = [p.float() for p in self.params] if master is True else list(master) if master else None
        if state is None:
            _need(state_bits in (8, 32), "state_bits has to be 8 or 32")
            z = lambda: [torch.zeros(p.shape, dtype=torch.float32 if state_bits == 32 else torch.float8_e4m3fn, device=dev) for p in self.params]
            sc = lambda: [torch.zeros(-(-k // STATE_BLOCK), dtype=torch.float32, device=dev) for k in size]
            state = (z(), z()) if state_bits == 32 else (z(), z(), sc(), sc())
        self.m, self.v = list(state[0]), list(state[1])
        self.m_scale, self.v_scale = (list(state[2]), list(state[3])) if len(state) == 4 else (None, None)
        bits = 32 if self.m_scale is None else 8
        wd = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(x) for x in weight_decay]
        _need(len(wd) == n, "one weight_decay per parameter")

        def check(ts, what, dtype, numel=lambda i: size[i]):
            _need(len(ts) == n, "%s: one tensor per parameter" % what)
            for i, t in enumerate(ts):
                _need(t.dtype == dtype and t.numel() == numel(i) and t.is_contiguous() and t.device == dev,
                      "%s[%d] has to be %s, contiguous, of %d elements on %s" % (what, i, dtype, numel(i), dev))
        check(self.params, "params", p_dt)
        check(self.grads_list, "grads", g_dt)
        if self.master is not None:
            check(self.master, "master", torch.float32)
        for ts, what in ((self.m, "m"), (self.v, "v")):
            check(ts, what, torch.float32 if bits == 32 else torch.float8_e4m3fn)
        if bits == 8:
            for ts, what in ((self.m_scale, "m_scale"), (self.v_scale, "v_scale")):
                check(ts, what, torch.float32, lambda i: -(-size[i] // STATE_BLOCK))
        for t, dt in ((step_dev, torch.int32), (lr_dev, torch.float32)):
            _need(t is None or (t.dtype == dt and t.numel() == 1 and t.device == dev), "step_dev: one int32, lr_dev: one fp32, on %s" % dev)
        # what a step writes overlaps nothing; what it reads may overlap what it reads
        written = (self.params, self.master, self.m, self.v, self.m_scale, self.v_scale)
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), w) for ts, w in
                       [(ts, True) for ts in written if ts is not None] + [(self.grads_list, False), ([t for t in (step_dev, lr_dev) if t is not None], False)]
                       for t in ts if t.numel())
        end = {True: 0, False: 0}           # of the ranges so far, written ones and read ones
        for a, b, w in spans:
            _need(a >= end[True] and not (w and a < end[False]), "a tensor that a step writes may be listed once only, and overlap no other")
            end[w] = max(end[w], b)
        self.step_dev, self.lr_dev = step_dev, lr_dev
        at = lambda ts, i: ts[i].data_ptr() if ts is not None else None
        self._t = (AdamwTensor * n)(*[AdamwTensor(at(self.params, i), at(self.master, i), at(self.grads_list, i), at(self.m, i), at(self.v, i),
                                                  at(self.m_scale, i), at(self.v_scale, i), size[i], wd[i]) for i in range(n)])
        self.grad_norm, self.t = None, 0
        if max_norm is not None:
            self.grad_norm = torch.zeros(1, dtype=torch.float32, device=dev)
            self._g = (C.c_void_p * n)(*[g.data_ptr() for g in self.grads_list])
            self._n = (C.c_int64 * n)(*size)
            self._ws = torch.empty(lib().cf_grad_norm_workspace_bytes(n), dtype=torch.uint8, device=dev)
        self._d = AdamwDesc(lr, betas[0], betas[1], eps, 0, _dtype_code(self.params[0]), _dtype_code(self.grads_list[0]), bits, seed & 0xFFFFFFFF,
                            grad_scale, 0.0 if max_norm is None else max_norm, _addr(self.grad_norm), _addr(step_dev), _addr(lr_dev))

    def step(self, lr: float | None = None, step: int | None = None) -> None:
        """One update.  step: its number, 1 for the first; by default one more than the last call's (one that the norm left out counts).
        lr: from this call on."""
        L, st, d = _lib or lib(), _stream(_on(self.params[:1])), self._d
        d.step = self.t + 1 if step is None else step
        if lr is not None:
            d.lr = lr
        if self.grad_norm is not None:
            _check(L.cf_grad_norm(self._g, self._n, len(self._t), d.g_dtype, d.grad_scale, d.norm_dev, self._ws.data_ptr(), self._ws.numel(), st),
                   "cf_grad_norm")
        _check(L.cf_adamw_step(C.byref(d), self._t, len(self._t), st), "cf_adamw_step")
        self.t = d.step
