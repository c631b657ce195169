"""Binding of libqeft.so: the same entry points as include/qeft.h.

Argument marshalling only.  `raw` exposes the C functions as they are (integers for
pointers), the functions below take torch tensors and pass `data_ptr()` and the current
HIP stream.  PyTorch is used for device memory and streams, nothing else; there is no
fallback path: if the library is missing the import fails.  The calls of training and decode loops
go through `_marshal` (csrc/marshal.cpp), which does the same natively for exact tensors on
the current GPU and returns None for anything else: ctypes then, as everywhere where `_marshal.so` is missing.
"""
from __future__ import annotations

import ctypes as C
import os
import types

import torch  # imported first on purpose: the library must bind to the HIP runtime torch loaded

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqeft.so")

QEFT_OK = 0
QEFT_ERR_NULL, QEFT_ERR_SHAPE, QEFT_ERR_BITS, QEFT_ERR_ALIGN = -1, -2, -3, -4
QEFT_ERR_WORKSPACE, QEFT_ERR_UNSUPPORTED, QEFT_ERR_HIP = -5, -6, -7
QEFT_OP_FWD, QEFT_OP_BWD_DX, QEFT_OP_WEAK_GRAD, QEFT_OP_FWD_IRREGULAR, QEFT_OP_BWD_DX_IRREGULAR, QEFT_OP_BWD = 0, 1, 2, 3, 4, 5
QEFT_DTYPE_F16, QEFT_DTYPE_F32 = 0, 1
QEFT_LAYOUT_CANONICAL, QEFT_LAYOUT_DENSE3 = 0, 1
QEFT_GATE_NONE, QEFT_GATE_CHANNEL, QEFT_GATE_TOKEN = 0, 1, 2
QEFT_MAX_TOP, QEFT_STATE_BLOCK = 64, 128
_DTYPES = {torch.float16: QEFT_DTYPE_F16, torch.float32: QEFT_DTYPE_F32}


class qeft_desc_t(C.Structure):
    _fields_ = [("out_features", C.c_int32), ("in_features", C.c_int32), ("n_weak", C.c_int32),
                ("bits", C.c_int32), ("group_size", C.c_int32), ("layout", C.c_int32)]


class qeft_layout_t(C.Structure):
    _fields_ = [("kq", C.c_int64), ("n_groups", C.c_int64), ("words_per_row", C.c_int64),
                ("row_stride_words", C.c_int64), ("group_stride", C.c_int64), ("qweight_bytes", C.c_size_t),
                ("scales_bytes", C.c_size_t),
                ("zeros_bytes", C.c_size_t), ("weak_bytes", C.c_size_t)]


class qeft_weight_t(C.Structure):
    _fields_ = [("qweight", C.c_void_p), ("scales", C.c_void_p), ("zeros", C.c_void_p), ("weak", C.c_void_p)]


class qeft_cache_desc_t(C.Structure):
    _fields_ = [("pages", C.c_int32), ("page_size", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("token_stride", C.c_int64)]


class qeft_cache_t(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)]


class qeft_table_t(C.Structure):
    _fields_ = [("table", C.c_void_p), ("ld_table", C.c_int64), ("table_pages", C.c_int32), ("seqs", C.c_int32)]


class qeft_append_t(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_out", C.c_void_p), ("ldq", C.c_int64), ("ldq_out", C.c_int64),
                ("ldk", C.c_int64), ("ldv", C.c_int64), ("seq", C.c_void_p), ("index", C.c_void_p), ("pos", C.c_void_p), ("rot", C.c_void_p),
                ("ld_rot", C.c_int64), ("positions", C.c_int32), ("rot_dim", C.c_int32), ("heads", C.c_int32), ("tokens", C.c_int64)]


class qeft_attn_t(C.Structure):
    _fields_ = [("lens", C.c_void_p), ("longest", C.c_int64), ("q", C.c_void_p), ("out", C.c_void_p), ("ldq", C.c_int64), ("ldo", C.c_int64),
                ("heads", C.c_int32), ("scale", C.c_float), ("score", C.c_void_p), ("ld_score", C.c_int64), ("accumulate", C.c_int32),
                ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


class qeft_evict_t(C.Structure):
    _fields_ = [("lens", C.c_void_p), ("seen", C.c_void_p), ("longest", C.c_int64), ("budget", C.c_int64), ("score", C.c_void_p),
                ("pos", C.c_void_p), ("ld", C.c_int64), ("keep_first", C.c_int32), ("keep_last", C.c_int32), ("score_out", C.c_void_p),
                ("pos_out", C.c_void_p), ("ld_out", C.c_int64), ("lens_out", C.c_void_p), ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


class qeft_norm_desc_t(C.Structure):
    _fields_ = [("n", C.c_int32), ("residual_dtype", C.c_int32), ("gate", C.c_int32), ("scale", C.c_float), ("eps", C.c_float)]


class qeft_norm_fwd_t(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("r", "y", "gate", "w_pre", "w_post", "h", "x")] + \
               [(f, C.c_int64) for f in ("ldr", "ldy", "ldg", "ldh", "ldx", "m")]


class qeft_norm_bwd_t(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("dx", "dh", "h", "y", "gate", "w_pre", "w_post", "dr", "dy", "dgate", "dw_pre", "dw_post")] + \
               [(f, C.c_int64) for f in ("lddx", "lddh", "ldh", "ldy", "ldg", "lddr", "lddy", "lddg", "m")] + \
               [("accumulate", C.c_int32), ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


class qeft_logprob_desc_t(C.Structure):
    _fields_ = [("n", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float)]


class qeft_logprob_fwd_t(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("z", "token", "logp", "lse", "entropy", "top_logp", "top_index")] + \
               [("ldz", C.c_int64), ("ld_top", C.c_int64), ("m", C.c_int64), ("top", C.c_int32), ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


class qeft_logprob_bwd_t(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("z", "token", "lse", "entropy", "dlogp", "dlse", "dentropy", "dz")] + \
               [(f, C.c_int64) for f in ("ldz", "lddz", "m")]


class qeft_qk_desc_t(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("rot_dim", C.c_int32), ("eps", C.c_float)]


class qeft_qk_fwd_t(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("q", "k", "w_q", "w_k", "q_out", "k_out", "pos", "rot")] + \
               [(f, C.c_int64) for f in ("ldq", "ldk", "ldq_out", "ldk_out", "ld_rot", "m")] + [("positions", C.c_int32)]


class qeft_qk_bwd_t(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("gq", "gk", "q", "k", "w_q", "w_k", "dq", "dk", "dw_q", "dw_k", "pos", "rot")] + \
               [(f, C.c_int64) for f in ("ldgq", "ldgk", "ldq", "ldk", "lddq", "lddk", "ld_rot", "m")] + \
               [("positions", C.c_int32), ("accumulate", C.c_int32), ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


class qeft_append_norm_t(C.Structure):
    _fields_ = [("w_q", C.c_void_p), ("w_k", C.c_void_p), ("eps", C.c_float)]


class qeft_tensor_t(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("weight", "master", "grad", "m", "v", "m_scale", "v_scale")] + [("n", C.c_int64), ("decay", C.c_float)]


class qeft_tensors_t(C.Structure):
    _fields_ = [("plan", C.c_void_p), ("work", C.c_int64), ("count", C.c_int32), ("grad_dtype", C.c_int32), ("state_bits", C.c_int32), ("has_weight", C.c_int32),
                ("has_master", C.c_int32)]


class qeft_adamw_t(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64), ("seed", C.c_uint64),
                ("lr_at", C.c_void_p), ("step_at", C.c_void_p), ("factor", C.c_void_p), ("stochastic", C.c_int32)]


class qeft_grad_norm_t(C.Structure):
    _fields_ = [("scale", C.c_float), ("max_norm", C.c_float), ("out", C.c_void_p), ("steps", C.c_void_p), ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


EXPORTS = {
    "qeft_layout": (C.c_int, [C.POINTER(qeft_desc_t), C.POINTER(qeft_layout_t)]),
    "qeft_pack": (C.c_int, [C.POINTER(qeft_desc_t), C.c_void_p, C.c_int64, C.POINTER(qeft_weight_t), C.c_void_p]),
    "qeft_pack_search": (C.c_int, [C.POINTER(qeft_desc_t), C.c_void_p, C.c_int64, C.c_int, C.c_float,
                                   C.POINTER(qeft_weight_t), C.c_void_p]),
    "qeft_pack_codes": (C.c_int, [C.POINTER(qeft_desc_t), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.POINTER(qeft_weight_t), C.c_void_p]),
    "qeft_unpack": (C.c_int, [C.POINTER(qeft_desc_t), C.POINTER(qeft_weight_t), C.c_void_p, C.c_void_p, C.c_void_p,
                              C.c_void_p, C.c_void_p]),
    "qeft_workspace_bytes": (C.c_size_t, [C.POINTER(qeft_desc_t), C.c_int, C.c_int64]),
    "qeft_linear_fwd": (C.c_int, [C.POINTER(qeft_desc_t), C.POINTER(qeft_weight_t), C.c_void_p, C.c_int64, C.c_int64,
                                  C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "qeft_linear_fwd_group": (C.c_int, [C.c_int, C.POINTER(qeft_desc_t), C.POINTER(qeft_weight_t), C.c_void_p, C.c_int64,
                                        C.c_int64, C.POINTER(C.c_void_p), C.POINTER(C.c_int64), C.c_void_p]),
    "qeft_linear_bwd_dx": (C.c_int, [C.POINTER(qeft_desc_t), C.POINTER(qeft_weight_t), C.c_void_p, C.c_int64,
                                     C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "qeft_linear_fwd_irregular": (C.c_int, [C.POINTER(qeft_desc_t), C.POINTER(qeft_weight_t), C.c_void_p, C.c_void_p,
                                            C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "qeft_linear_bwd_dx_irregular": (C.c_int, [C.POINTER(qeft_desc_t), C.POINTER(qeft_weight_t), C.c_void_p, C.c_void_p,
                                               C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "qeft_sensitivity_workspace": (C.c_size_t, [C.c_int32, C.c_int64]),
    "qeft_sensitivity": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                   C.c_size_t, C.c_void_p]),
    "qeft_vote": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "qeft_weak_order": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]),
    "qeft_reorder": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int, C.c_void_p, C.c_int64,
                               C.c_void_p]),
    "qeft_merge_weak": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32,
                                  C.c_void_p]),
    "qeft_weak_grad": (C.c_int, [C.POINTER(qeft_desc_t), C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64,
                                 C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "qeft_linear_bwd": (C.c_int, [C.POINTER(qeft_desc_t), C.POINTER(qeft_weight_t), C.c_void_p, C.c_int64, C.c_int64, C.c_void_p,
                                  C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "qeft_weak_grad_noalloc": (C.c_int, [C.POINTER(qeft_desc_t), C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64,
                                         C.c_void_p, C.c_int, C.c_int, C.c_void_p]),
    "qeft_cache_append": (C.c_int, [C.POINTER(qeft_cache_desc_t), C.POINTER(qeft_cache_t), C.POINTER(qeft_table_t), C.POINTER(qeft_append_t),
                                    C.c_void_p]),
    "qeft_attn_workspace": (C.c_size_t, [C.POINTER(qeft_cache_desc_t), C.c_int64, C.c_int32, C.c_int64, C.c_int]),
    "qeft_attn_decode": (C.c_int, [C.POINTER(qeft_cache_desc_t), C.POINTER(qeft_cache_t), C.POINTER(qeft_table_t), C.POINTER(qeft_attn_t),
                                   C.c_void_p]),
    "qeft_evict_workspace": (C.c_size_t, [C.POINTER(qeft_cache_desc_t), C.c_int64, C.c_int64, C.c_int64]),
    "qeft_cache_evict": (C.c_int, [C.POINTER(qeft_cache_desc_t), C.POINTER(qeft_cache_t), C.POINTER(qeft_table_t), C.POINTER(qeft_evict_t),
                                   C.c_void_p]),
    "qeft_norm_fwd": (C.c_int, [C.POINTER(qeft_norm_desc_t), C.POINTER(qeft_norm_fwd_t), C.c_void_p]),
    "qeft_norm_workspace": (C.c_size_t, [C.POINTER(qeft_norm_desc_t), C.c_int64]),
    "qeft_norm_bwd": (C.c_int, [C.POINTER(qeft_norm_desc_t), C.POINTER(qeft_norm_bwd_t), C.c_void_p]),
    "qeft_logprob_workspace": (C.c_size_t, [C.POINTER(qeft_logprob_desc_t), C.c_int64, C.c_int32]),
    "qeft_logprob_fwd": (C.c_int, [C.POINTER(qeft_logprob_desc_t), C.POINTER(qeft_logprob_fwd_t), C.c_void_p]),
    "qeft_logprob_bwd": (C.c_int, [C.POINTER(qeft_logprob_desc_t), C.POINTER(qeft_logprob_bwd_t), C.c_void_p]),
    "qeft_logprob_fwd_bwd": (C.c_int, [C.POINTER(qeft_logprob_desc_t), C.POINTER(qeft_logprob_fwd_t), C.POINTER(qeft_logprob_bwd_t), C.c_void_p]),
    "qeft_qk_norm_fwd": (C.c_int, [C.POINTER(qeft_qk_desc_t), C.POINTER(qeft_qk_fwd_t), C.c_void_p]),
    "qeft_qk_norm_workspace": (C.c_size_t, [C.POINTER(qeft_qk_desc_t), C.c_int64]),
    "qeft_qk_norm_bwd": (C.c_int, [C.POINTER(qeft_qk_desc_t), C.POINTER(qeft_qk_bwd_t), C.c_void_p]),
    "qeft_cache_append_norm": (C.c_int, [C.POINTER(qeft_cache_desc_t), C.POINTER(qeft_cache_t), C.POINTER(qeft_table_t), C.POINTER(qeft_append_t),
                                         C.POINTER(qeft_append_norm_t), C.c_void_p]),
    "qeft_tensors_plan_bytes": (C.c_size_t, [C.POINTER(qeft_tensor_t), C.c_int32]),
    "qeft_tensors_plan": (C.c_int, [C.POINTER(qeft_tensor_t), C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.POINTER(qeft_tensors_t)]),
    "qeft_adamw_step": (C.c_int, [C.POINTER(qeft_tensors_t), C.POINTER(qeft_adamw_t), C.c_void_p]),
    "qeft_grad_norm_workspace": (C.c_size_t, [C.POINTER(qeft_tensors_t)]),
    "qeft_grad_norm": (C.c_int, [C.POINTER(qeft_tensors_t), C.POINTER(qeft_grad_norm_t), C.c_void_p]),
    "qeft_status_string": (C.c_char_p, [C.c_int]),
}


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run `python -m paper_2410_08661_amd.build`")
    lib = C.CDLL(LIB_PATH)
    for name, (res, args) in EXPORTS.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


raw = _load()


class QeftError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {raw.qeft_status_string(status).decode()} ({status})")


def _check(status: int, where: str) -> None:
    if status != QEFT_OK:
        raise QeftError(status, where)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _stream() -> int:
    # the current stream's handle without the Stream object around it: 0.3 us against 2.8, of an 8 us call
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def make_desc(out_features, in_features, n_weak, bits=4, group_size=128, layout=0) -> qeft_desc_t:
    return qeft_desc_t(out_features, in_features, n_weak, bits, group_size, layout)


def qeft_layout(desc: qeft_desc_t) -> qeft_layout_t:
    out = qeft_layout_t()
    _check(raw.qeft_layout(C.byref(desc), C.byref(out)), "qeft_layout")
    return out


class Weight:
    """The four device buffers of one stored layer (torch tensors own the memory)."""

    def __init__(self, desc: qeft_desc_t, device="cuda"):
        lay = qeft_layout(desc)
        self.desc, self.lay = desc, lay
        oc = desc.out_features
        self.qweight = torch.zeros((oc, lay.row_stride_words), dtype=torch.int32, device=device)
        self.scales = torch.zeros((oc, lay.group_stride), dtype=torch.float16, device=device)
        self.zeros = torch.zeros((oc, lay.group_stride), dtype=torch.float16, device=device)
        self.weak = torch.zeros((oc, desc.n_weak), dtype=torch.float16, device=device)

    def c_struct(self) -> qeft_weight_t:
        lay, d = self.lay, self.desc
        return qeft_weight_t(self.qweight.data_ptr() if lay.kq else None, self.scales.data_ptr() if lay.kq else None,
                             self.zeros.data_ptr() if lay.kq else None, self.weak.data_ptr() if d.n_weak else None)

    def nbytes(self) -> int:
        lay = self.lay
        return lay.qweight_bytes + lay.scales_bytes + lay.zeros_bytes + lay.weak_bytes


_MARSHALLED = ("qeft_linear_fwd", "qeft_linear_fwd_group", "qeft_linear_bwd_dx", "qeft_linear_bwd", "qeft_linear_fwd_irregular",
               "qeft_linear_bwd_dx_irregular", "qeft_weak_grad", "qeft_cache_append", "qeft_attn_decode", "qeft_cache_evict", "qeft_norm_fwd",
               "qeft_norm_bwd", "qeft_logprob_fwd", "qeft_logprob_bwd", "qeft_logprob_fwd_bwd", "qeft_qk_norm_fwd", "qeft_qk_norm_bwd", "qeft_cache_append_norm", "qeft_adamw_step",
               "qeft_grad_norm")


def _load_marshal():
    try:
        from . import _marshal as m
    except ImportError:   # not built, or not for this torch: every call is ctypes'
        return types.SimpleNamespace(**{n.removeprefix("qeft_"): lambda *args: None for n in _MARSHALLED})
    m.init(tuple(C.cast(getattr(raw, n), C.c_void_p).value for n in _MARSHALLED), qeft_desc_t, Weight, qeft_cache_desc_t, qeft_norm_desc_t,
           qeft_logprob_desc_t, qeft_qk_desc_t, qeft_tensors_t)
    return m


_native = _load_marshal()


def qeft_pack(desc: qeft_desc_t, W: torch.Tensor, out: Weight | None = None) -> Weight:
    out = out or Weight(desc, W.device)
    ws = out.c_struct()
    _check(raw.qeft_pack(C.byref(desc), _ptr(W), W.stride(0), C.byref(ws), _stream()), "qeft_pack")
    return out


def qeft_pack_search(desc: qeft_desc_t, W: torch.Tensor, n_grid: int = 80, shrink_step: float = 0.01,
                     out: Weight | None = None) -> Weight:
    """qeft_pack with the group-wise grid search over truncated ranges."""
    out = out or Weight(desc, W.device)
    ws = out.c_struct()
    _check(raw.qeft_pack_search(C.byref(desc), _ptr(W), W.stride(0), int(n_grid), float(shrink_step), C.byref(ws),
                                _stream()), "qeft_pack_search")
    return out


def qeft_pack_codes(desc, codes, scales, zeros, weak, out: Weight | None = None) -> Weight:
    out = out or Weight(desc, weak.device if weak is not None else codes.device)
    ws = out.c_struct()
    _check(raw.qeft_pack_codes(C.byref(desc), _ptr(codes), _ptr(scales), _ptr(zeros), _ptr(weak), C.byref(ws),
                               _stream()), "qeft_pack_codes")
    return out


def qeft_unpack(desc, w: Weight):
    lay = w.lay
    dev = w.qweight.device
    codes = torch.empty((desc.out_features, lay.kq), dtype=torch.uint8, device=dev)
    scales = torch.empty((desc.out_features, lay.n_groups), dtype=torch.float16, device=dev)
    zeros, weak = torch.empty_like(scales), torch.empty_like(w.weak)
    ws = w.c_struct()
    _check(raw.qeft_unpack(C.byref(desc), C.byref(ws), _ptr(codes) if lay.kq else None,
                           _ptr(scales) if lay.kq else None, _ptr(zeros) if lay.kq else None,
                           _ptr(weak) if desc.n_weak else None, _stream()), "qeft_unpack")
    return codes, scales, zeros, weak


def _empty_rows(m: int, cols: int, dtype, device) -> torch.Tensor:
    """[m][cols] tensor whose leading dimension is padded to a multiple of 8 elements."""
    ld = (max(cols, 1) + 7) // 8 * 8
    return torch.empty((m, ld), dtype=dtype, device=device)[:, :cols]


def qeft_workspace_bytes(desc, op: int, M: int) -> int:
    return int(raw.qeft_workspace_bytes(C.byref(desc), op, M))


def _workspace(desc, op, M, device):
    n = qeft_workspace_bytes(desc, op, M)
    return (torch.empty(n, dtype=torch.uint8, device=device), n) if n else (None, 0)


def qeft_linear_fwd(desc, w: Weight, X: torch.Tensor, Y: torch.Tensor | None = None, ws=None) -> torch.Tensor:
    """ws: a uint8 device tensor of qeft_workspace_bytes(desc, QEFT_OP_FWD, M) bytes; None allocates one when the
    operation can use it (3-bit layers at M > 16), False passes none (the library then runs its general kernel)."""
    if Y is None:
        Y = _empty_rows(X.shape[0], desc.out_features, torch.float16, X.device)
    if ws is None:
        ws, _ = _workspace(desc, QEFT_OP_FWD, X.shape[0], X.device)
    elif ws is False:
        ws = None
    st = _native.linear_fwd(desc, w, X, Y, ws)
    if st is None:
        M, wst = X.shape[0], w.c_struct()
        st = raw.qeft_linear_fwd(C.byref(desc), C.byref(wst), _ptr(X), M, X.stride(0) if M else desc.in_features,
                                 _ptr(Y), Y.stride(0) if M else desc.out_features, _ptr(ws),
                                 ws.numel() if ws is not None else 0, _stream())
    _check(st, "qeft_linear_fwd")
    return Y


class Group:
    """The host-side argument arrays of qeft_linear_fwd_group for a fixed set of layers and outputs
    (built once; a decode loop then only passes X)."""

    def __init__(self, descs, ws, Ys):
        n = len(descs)
        assert n == len(ws) == len(Ys) and n >= 1
        self.n = n
        self.descs = (qeft_desc_t * n)(*descs)
        self.wst = (qeft_weight_t * n)(*[w.c_struct() for w in ws])
        self.ys = (C.c_void_p * n)(*[_ptr(y) for y in Ys])
        self.ldy = (C.c_int64 * n)(*[y.stride(0) for y in Ys])
        self.keep = (list(ws), list(Ys))   # the device buffers the arrays point into
        self.Ys = list(Ys)


def qeft_linear_fwd_group(descs, ws, X: torch.Tensor, Ys=None, group: Group | None = None):
    """Forward of several layers that share the input X; returns the list of outputs."""
    if group is None:
        if Ys is None:
            Ys = [_empty_rows(X.shape[0], d.out_features, torch.float16, X.device) for d in descs]
        group = Group(descs, ws, Ys)
    st = _native.linear_fwd_group(group.n, group.descs, group.wst, X, group.ys, group.ldy)
    if st is None:
        M = X.shape[0]
        st = raw.qeft_linear_fwd_group(group.n, group.descs, group.wst, _ptr(X), M,
                                       X.stride(0) if M else group.descs[0].in_features, group.ys, group.ldy, _stream())
    _check(st, "qeft_linear_fwd_group")
    return group.Ys


def qeft_linear_bwd_dx(desc, w: Weight, dY: torch.Tensor, dX: torch.Tensor | None = None, ws=None) -> torch.Tensor:
    if dX is None:
        dX = _empty_rows(dY.shape[0], desc.in_features, torch.float16, dY.device)
    if ws is None:
        ws, _ = _workspace(desc, QEFT_OP_BWD_DX, dY.shape[0], dY.device)
    elif ws is False:
        ws = None
    st = _native.linear_bwd_dx(desc, w, dY, dX, ws)
    if st is None:
        M, wst = dY.shape[0], w.c_struct()
        st = raw.qeft_linear_bwd_dx(C.byref(desc), C.byref(wst), _ptr(dY), M, dY.stride(0) if M else desc.out_features,
                                    _ptr(dX), dX.stride(0) if M else desc.in_features, _ptr(ws),
                                    ws.numel() if ws is not None else 0, _stream())
    _check(st, "qeft_linear_bwd_dx")
    return dX


def qeft_linear_fwd_irregular(desc, w: Weight, perm: torch.Tensor, X: torch.Tensor, Y: torch.Tensor | None = None,
                              ws=None) -> torch.Tensor:
    """Forward of a layer whose weak columns stay at arbitrary channels; perm int32 [IC] on the device."""
    if Y is None:
        Y = _empty_rows(X.shape[0], desc.out_features, torch.float16, X.device)
    if ws is None:
        ws, _ = _workspace(desc, QEFT_OP_FWD_IRREGULAR, X.shape[0], X.device)
    st = _native.linear_fwd_irregular(desc, w, perm, X, Y, ws)
    if st is None:
        M, wst = X.shape[0], w.c_struct()
        st = raw.qeft_linear_fwd_irregular(C.byref(desc), C.byref(wst), _ptr(perm), _ptr(X), M,
                                           X.stride(0) if M else desc.in_features, _ptr(Y),
                                           Y.stride(0) if M else desc.out_features, _ptr(ws),
                                           ws.numel() if ws is not None else 0, _stream())
    _check(st, "qeft_linear_fwd_irregular")
    return Y


def qeft_linear_bwd_dx_irregular(desc, w: Weight, perm: torch.Tensor, dY: torch.Tensor, dX: torch.Tensor | None = None,
                                 ws=None) -> torch.Tensor:
    if dX is None:
        dX = _empty_rows(dY.shape[0], desc.in_features, torch.float16, dY.device)
    if ws is None:
        ws, _ = _workspace(desc, QEFT_OP_BWD_DX_IRREGULAR, dY.shape[0], dY.device)
    st = _native.linear_bwd_dx_irregular(desc, w, perm, dY, dX, ws)
    if st is None:
        M, wst = dY.shape[0], w.c_struct()
        st = raw.qeft_linear_bwd_dx_irregular(C.byref(desc), C.byref(wst), _ptr(perm), _ptr(dY), M,
                                              dY.stride(0) if M else desc.out_features, _ptr(dX),
                                              dX.stride(0) if M else desc.in_features, _ptr(ws),
                                              ws.numel() if ws is not None else 0, _stream())
    _check(st, "qeft_linear_bwd_dx_irregular")
    return dX


def qeft_sensitivity(X: torch.Tensor, n_batch: int) -> torch.Tensor:
    """Diagonal of the layer input's Hessian, fp32 [d]."""
    tokens, d = X.shape
    out = torch.empty(d, dtype=torch.float32, device=X.device)
    n = int(raw.qeft_sensitivity_workspace(d, tokens))
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=X.device)
    _check(raw.qeft_sensitivity(_ptr(X), tokens, X.stride(0), d, int(n_batch), _ptr(out), _ptr(ws), ws.numel(), _stream()),
           "qeft_sensitivity")
    return out


def qeft_vote(s: torch.Tensor, k: int, s_global: torch.Tensor | None = None) -> torch.Tensor:
    """Top-k channels of s (int32 [k], largest first); with s_global their votes are added to it."""
    idx = torch.empty(k, dtype=torch.int32, device=s.device)
    _check(raw.qeft_vote(_ptr(s), s.numel(), int(k), _ptr(idx), _ptr(s_global), _stream()), "qeft_vote")
    return idx


def qeft_weak_order(idx: torch.Tensor, d: int) -> torch.Tensor:
    perm = torch.empty(d, dtype=torch.int32, device=idx.device)
    _check(raw.qeft_weak_order(_ptr(idx), idx.numel(), int(d), _ptr(perm), _stream()), "qeft_weak_order")
    return perm


def qeft_reorder(A: torch.Tensor, perm: torch.Tensor, axis: int) -> torch.Tensor:
    rows, cols = A.shape
    out = _empty_rows(rows, cols, torch.float16, A.device)
    _check(raw.qeft_reorder(_ptr(A), rows, cols, A.stride(0), _ptr(perm), int(axis), _ptr(out), out.stride(0), _stream()),
           "qeft_reorder")
    return out


def qeft_merge_weak(tuned: torch.Tensor, base: torch.Tensor, target: torch.Tensor, idx: torch.Tensor | None = None) -> torch.Tensor:
    """target[:, idx] (or target[:, :k]) += tuned - base, in place."""
    oc, k = tuned.shape
    _check(raw.qeft_merge_weak(_ptr(tuned), _ptr(base), oc, k, _ptr(idx), _ptr(target), target.stride(0), target.shape[1],
                               _stream()), "qeft_merge_weak")
    return target


def qeft_weak_grad(desc, dY: torch.Tensor, Xw: torch.Tensor, dW: torch.Tensor | None = None, accumulate=False,
                   out_dtype=torch.float32, ws=None) -> torch.Tensor:
    if dW is None:
        dW = torch.zeros((desc.out_features, desc.n_weak), dtype=out_dtype, device=dY.device)
    code = _DTYPES[dW.dtype]
    if ws is None:
        ws, _ = _workspace(desc, QEFT_OP_WEAK_GRAD, dY.shape[0], dY.device)
    accumulate = int(bool(accumulate))
    st = _native.weak_grad(desc, dY, Xw, dW, code, accumulate, ws)
    if st is None:
        M = dY.shape[0]
        st = raw.qeft_weak_grad(C.byref(desc), _ptr(dY), M, dY.stride(0) if M else desc.out_features, _ptr(Xw),
                                Xw.stride(0) if M else max(desc.n_weak, 8), _ptr(dW), code, accumulate,
                                _ptr(ws), ws.numel() if ws is not None else 0, _stream())
    _check(st, "qeft_weak_grad")
    return dW


def qeft_weak_grad_noalloc(desc, dY: torch.Tensor, Xw: torch.Tensor, dW: torch.Tensor, accumulate=False) -> torch.Tensor:
    """qeft_weak_grad without a workspace argument: the library's own per-GPU scratch array takes the partial sums.
    dW must be given (this call allocates nothing, here or in the library)."""
    M = dY.shape[0]
    code = _DTYPES[dW.dtype]
    _check(raw.qeft_weak_grad_noalloc(C.byref(desc), _ptr(dY), M, dY.stride(0) if M else desc.out_features, _ptr(Xw),
                                      Xw.stride(0) if M else max(desc.n_weak, 8), _ptr(dW), code, int(bool(accumulate)),
                                      _stream()), "qeft_weak_grad_noalloc")
    return dW


def qeft_linear_bwd(desc, w: Weight, dY: torch.Tensor, Xw: torch.Tensor, dX: torch.Tensor | None = None,
                    dW: torch.Tensor | None = None, accumulate=False, out_dtype=torch.float32, ws=None):
    """dX and dW_weak of one layer in one call; returns (dX, dW).  ws: None allocates the weak gradient's workspace;
    a tensor of qeft_workspace_bytes(desc, QEFT_OP_BWD, M) bytes also lets dX split its rows where that pays."""
    if dX is None:
        dX = _empty_rows(dY.shape[0], desc.in_features, torch.float16, dY.device)
    if dW is None:
        dW = torch.zeros((desc.out_features, desc.n_weak), dtype=out_dtype, device=dY.device)
    code = _DTYPES[dW.dtype]
    if ws is None:
        ws, _ = _workspace(desc, QEFT_OP_WEAK_GRAD, dY.shape[0], dY.device)
    accumulate = int(bool(accumulate))
    st = _native.linear_bwd(desc, w, dY, dX, Xw, dW, code, accumulate, ws)
    if st is None:
        M, wst = dY.shape[0], w.c_struct()
        st = raw.qeft_linear_bwd(C.byref(desc), C.byref(wst), _ptr(dY), M, dY.stride(0) if M else desc.out_features, _ptr(dX),
                                 dX.stride(0) if M else desc.in_features, _ptr(Xw), Xw.stride(0) if M else max(desc.n_weak, 8),
                                 _ptr(dW), code, accumulate, _ptr(ws), ws.numel() if ws is not None else 0, _stream())
    _check(st, "qeft_linear_bwd")
    return dX, dW



# ---- between the linear layers: paged cache, attention of one token, eviction, norms ---------------------------------------------------------
#
# These calls check what the C functions cannot see, the types and shapes of tensors, and raise QeftError for what does not fit.

def _fail(status: int, where: str, what: str):
    e = QeftError(status, where)
    e.args = (f"{e.args[0]}: {what}",)
    raise e


def _take(where, name, t, dtype, shape, optional=False, least=0):
    """Pointer and row pitch of tensor t of this type and shape (entries None: any; rows of `least` values or more), whose rows are contiguous and whose leading axes, if there are
    three, lie one behind the other."""
    if t is None:
        if not optional:
            _fail(QEFT_ERR_NULL, where, f"{name} is missing")
        return 0, 0
    if t.dtype != dtype or t.dim() != len(shape):
        _fail(QEFT_ERR_UNSUPPORTED, where, f"{name} is {t.dtype} of {t.dim()} axes, not {dtype} of {len(shape)}")
    if any(want is not None and have != want for have, want in zip(t.shape, shape)):
        _fail(QEFT_ERR_SHAPE, where, f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.shape[0] > 0 and t.shape[-1] < least:   # (a view's pitch can be wider than its rows are)
        _fail(QEFT_ERR_SHAPE, where, f"{name}'s rows hold {t.shape[-1]} tokens, not {least}")
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        _fail(QEFT_ERR_UNSUPPORTED, where, f"{name} is not on the current GPU")
    if t.numel() == 0:   # (an empty tensor's pitch says nothing)
        return t.data_ptr(), max(t.shape[-1], 1) + 7 & ~7
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        _fail(QEFT_ERR_UNSUPPORTED, where, f"{name}'s rows are not contiguous")
    ld = t.stride(-2) if t.dim() > 1 and t.shape[-2] > 1 else None
    if t.dim() == 3 and t.shape[0] > 1:
        if ld is None:
            ld = t.stride(0)
        elif t.stride(0) != ld * t.shape[1]:
            _fail(QEFT_ERR_UNSUPPORTED, where, f"{name}'s leading axes do not lie one behind the other")
    elif ld is None:   # one row: any pitch it may have
        ld = t.shape[-1] + 7 & ~7
    return t.data_ptr(), ld


def make_cache_desc(pages, page_size, kv_heads, head_dim, page_stride=None, head_stride=None, token_stride=None) -> qeft_cache_desc_t:
    """Strides in elements; by default a pool is [pages][kv_heads][page_size][head_dim], contiguous."""
    return qeft_cache_desc_t(pages, page_size, kv_heads, head_dim, kv_heads * page_size * head_dim if page_stride is None else page_stride,
                             page_size * head_dim if head_stride is None else head_stride, head_dim if token_stride is None else token_stride)


class Cache:
    """The two pools of a paged cache: fp16 tensors [pages][kv_heads][page_size][head_dim] with the description's strides (made here if not given)."""

    def __init__(self, desc: qeft_cache_desc_t, k: torch.Tensor | None = None, v: torch.Tensor | None = None, device="cuda"):
        self.desc = desc
        shape = (desc.pages, desc.kv_heads, desc.page_size, desc.head_dim)
        strides = (desc.page_stride, desc.head_stride, desc.token_stride, 1)
        self.k, self.v = (torch.empty_strided(shape, strides, dtype=torch.float16, device=device).zero_() if t is None else t for t in (k, v))
        for name, t in (("k", self.k), ("v", self.v)):
            self._pool(name, t)

    def _pool(self, name, t):
        d = self.desc
        shape = (d.pages, d.kv_heads, d.page_size, d.head_dim)
        if t.dtype != torch.float16 or tuple(t.shape) != shape:
            _fail(QEFT_ERR_SHAPE, "Cache", f"{name} is {t.dtype} {tuple(t.shape)}, not float16 {shape}")
        if any(n > 1 and have != want for n, have, want in zip(shape, t.stride(), (d.page_stride, d.head_stride, d.token_stride, 1))):
            _fail(QEFT_ERR_SHAPE, "Cache", f"{name}'s strides {t.stride()} are not the description's")
        return t.data_ptr()

    def c_struct(self) -> qeft_cache_t:
        for name, t in (("k", self.k), ("v", self.v)):
            if not t.is_cuda or t.device.index != torch.cuda.current_device():
                _fail(QEFT_ERR_UNSUPPORTED, "Cache", f"{name} is not on the current GPU")
        return qeft_cache_t(self._pool("k", self.k), self._pool("v", self.v))


def _c_table(where, table):
    p, ld = _take(where, "table", table, torch.int32, (None, None))
    return qeft_table_t(p, ld, table.shape[1], table.shape[0])   # (an expanded view's pitch is 0, which the host's checks refuse)


def _c_workspace(where, ws):
    if ws is None:
        return 0, 0
    p, _ = _take(where, "ws", ws, torch.uint8, (None,))
    return p, ws.numel()


def _c_append(at, cache, table, k, v, index, seq, q, q_out, rot, pos):
    """The structs of an append."""
    d = cache.desc
    pools, tab = cache.c_struct(), _c_table(at, table)
    n = k.shape[0] if k is not None and k.dim() == 2 else None
    width = d.kv_heads * d.head_dim
    pk, ldk = _take(at, "k", k, torch.float16, (n, width))
    pv, ldv = _take(at, "v", v, torch.float16, (n, width))
    pq, ldq = _take(at, "q", q, torch.float16, (n, None), True)
    heads = 0 if q is None else q.shape[1] // d.head_dim
    if q is not None and heads * d.head_dim != q.shape[1]:
        _fail(QEFT_ERR_SHAPE, at, "q's rows are not whole heads")
    po, ldo = _take(at, "q_out", q_out if q is not None else None, torch.float16, (n, heads * d.head_dim), q is None)
    pi, ps, pp = (_take(at, name, t, torch.int32, (n,), t is not index)[0] for name, t in (("index", index), ("seq", seq), ("pos", pos)))
    pr, ldr = _take(at, "rot", rot, torch.float32, (None, None), True)
    a = qeft_append_t(pq, pk, pv, po, ldq, ldo, ldk, ldv, ps, pi, pp, pr, ldr,
                      rot.shape[0] if rot is not None else 0, rot.shape[1] if rot is not None else 0, heads, n)
    return pools, tab, a


def qeft_cache_append(cache: Cache, table: torch.Tensor, k: torch.Tensor, v: torch.Tensor, index: torch.Tensor, seq: torch.Tensor | None = None,
                      q: torch.Tensor | None = None, q_out: torch.Tensor | None = None, rot: torch.Tensor | None = None,
                      pos: torch.Tensor | None = None) -> torch.Tensor | None:
    """k, v fp16 [tokens][kv_heads * head_dim] into the cache, k rotated; q fp16 [tokens][heads * head_dim] rotated into q_out, which is returned
    (None without q).  index, seq, pos int32 [tokens]; rot fp32 [positions][rot_dim]; table int32 [seqs][pages]."""
    if q is not None and q_out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    st = _native.cache_append(cache.desc, cache.k, cache.v, table, k, v, index, seq, q, q_out, rot, pos)
    if st is None:
        d = cache.desc
        pools, tab, a = _c_append("qeft_cache_append", cache, table, k, v, index, seq, q, q_out, rot, pos)
        st = raw.qeft_cache_append(C.byref(d), C.byref(pools), C.byref(tab), C.byref(a), _stream())
    _check(st, "qeft_cache_append")
    return q_out


def qeft_attn_workspace(desc: qeft_cache_desc_t, seqs: int, heads: int, longest: int, weights=False) -> int:
    return int(raw.qeft_attn_workspace(C.byref(desc), seqs, heads, longest, int(bool(weights))))


def qeft_attn_decode(cache: Cache, table: torch.Tensor, lens: torch.Tensor, longest: int, q: torch.Tensor, out: torch.Tensor | None = None,
                     score: torch.Tensor | None = None, accumulate=False, scale: float | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of one token per sequence: q, out fp16 [seqs][heads * head_dim], lens int32 [seqs] on the GPU, longest the host's bound of them.
    score fp32 [seqs][kv_heads][tokens]: every token's weight is written there (added with accumulate).  scale: head_dim ** -0.5 by default.
    ws: uint8, qeft_attn_workspace bytes; None allocates it."""
    d = cache.desc
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if scale is None:
        scale = d.head_dim ** -0.5
    if ws is None:
        n = qeft_attn_workspace(d, q.shape[0], q.shape[1] // d.head_dim, longest, score is not None)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    st = _native.attn_decode(d, cache.k, cache.v, table, lens, longest, q, out, score, accumulate, scale, ws)
    if st is None:
        at = "qeft_attn_decode"
        pools, tab = cache.c_struct(), _c_table(at, table)
        n = table.shape[0]
        pq, ldq = _take(at, "q", q, torch.float16, (n, None))
        heads = q.shape[1] // d.head_dim
        if heads * d.head_dim != q.shape[1]:
            _fail(QEFT_ERR_SHAPE, at, "q's rows are not whole heads")
        po, ldo = _take(at, "out", out, torch.float16, (n, q.shape[1]))
        pl, _ = _take(at, "lens", lens, torch.int32, (n,))
        ps, lds = _take(at, "score", score, torch.float32, (n, d.kv_heads, None), True, min(longest, table.shape[1] * d.page_size))
        pw, nw = _c_workspace(at, ws)
        a = qeft_attn_t(pl, int(longest), pq, po, ldq, ldo, heads, float(scale), ps, lds, int(bool(accumulate)), pw, nw)
        st = raw.qeft_attn_decode(C.byref(d), C.byref(pools), C.byref(tab), C.byref(a), _stream())
    _check(st, "qeft_attn_decode")
    return out


def qeft_evict_workspace(desc: qeft_cache_desc_t, seqs: int, longest: int, budget: int) -> int:
    return int(raw.qeft_evict_workspace(C.byref(desc), seqs, longest, budget))


def qeft_cache_evict(cache: Cache, table: torch.Tensor, lens: torch.Tensor, longest: int, budget: int, score: torch.Tensor, pos: torch.Tensor,
                     seen: torch.Tensor, keep_first=0, keep_last=0, score_out: torch.Tensor | None = None, pos_out: torch.Tensor | None = None,
                     lens_out: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Every head keeps `budget` tokens, moved into the first slots; returns (score_out, pos_out, lens_out).  score fp32 and pos int32
    [seqs][kv_heads][tokens]; by default they are updated in place, lens_out is new."""
    d = cache.desc
    score_out, pos_out = score if score_out is None else score_out, pos if pos_out is None else pos_out
    if lens_out is None:
        lens_out = torch.empty_like(lens)
    if ws is None:
        n = qeft_evict_workspace(d, table.shape[0], longest, budget)
        ws = torch.empty(n, dtype=torch.uint8, device=lens.device) if n else None
    st = _native.cache_evict(d, cache.k, cache.v, table, lens, longest, budget, score, pos, seen, keep_first, keep_last, score_out, pos_out, lens_out, ws)
    if st is None:
        at = "qeft_cache_evict"
        pools, tab = cache.c_struct(), _c_table(at, table)
        n = table.shape[0]
        pl, pn, po = (_take(at, name, t, torch.int32, (n,))[0] for name, t in (("lens", lens), ("seen", seen), ("lens_out", lens_out)))
        most = min(longest, table.shape[1] * d.page_size)
        kept = min(budget, most)
        (ps, lds), (pso, ldso) = (_take(at, name, t, torch.float32, (n, d.kv_heads, None), False, least)
                                  for name, t, least in (("score", score, most), ("score_out", score_out, kept)))
        (pp, ldp), (ppo, ldpo) = (_take(at, name, t, torch.int32, (n, d.kv_heads, None), False, least)
                                  for name, t, least in (("pos", pos, most), ("pos_out", pos_out, kept)))
        if score.shape != pos.shape or lds != ldp or score_out.shape != pos_out.shape or ldso != ldpo:
            _fail(QEFT_ERR_SHAPE, at, "score and pos differ in shape or pitch")
        one = n * d.kv_heads == 1   # (one row: its width is all there is)
        pw, nw = _c_workspace(at, ws)
        a = qeft_evict_t(pl, pn, int(longest), int(budget), ps, pp, score.shape[2] if one else lds, int(keep_first), int(keep_last), pso, ppo,
                         score_out.shape[2] if one else ldso, po, pw, nw)
        st = raw.qeft_cache_evict(C.byref(d), C.byref(pools), C.byref(tab), C.byref(a), _stream())
    _check(st, "qeft_cache_evict")
    return score_out, pos_out, lens_out


def make_norm_desc(n, residual_dtype=torch.float16, gate=QEFT_GATE_NONE, scale=1.0, eps=1e-5) -> qeft_norm_desc_t:
    return qeft_norm_desc_t(n, _DTYPES[residual_dtype], gate, scale, eps)


def _residual(desc):
    return torch.float32 if desc.residual_dtype == QEFT_DTYPE_F32 else torch.float16


def qeft_norm_fwd(desc: qeft_norm_desc_t, r: torch.Tensor, w_pre: torch.Tensor, y: torch.Tensor | None = None, w_post: torch.Tensor | None = None,
                  gate: torch.Tensor | None = None, h: torch.Tensor | None = None, x: torch.Tensor | None = None):
    """(h, x): h = r + scale * gate * (y, normed with w_post if given), x = unit(h) * w_pre.  Without y only x is computed, from r; h is r then."""
    if x is None:
        x = _empty_rows(r.shape[0], desc.n, torch.float16, r.device)
    if h is None and y is not None:
        h = _empty_rows(r.shape[0], desc.n, _residual(desc), r.device)
    st = _native.norm_fwd(desc, r, w_pre, y, w_post, gate, h, x)
    if st is None:
        at, m, n = "qeft_norm_fwd", r.shape[0], desc.n
        pr, ldr = _take(at, "r", r, _residual(desc), (m, n))
        px, ldx = _take(at, "x", x, torch.float16, (m, n))
        py, ldy = _take(at, "y", y, torch.float16, (m, n), True)
        ph, ldh = _take(at, "h", h, _residual(desc), (m, n), True)
        pg, ldg = _take(at, "gate", gate, torch.float16, (m, n) if desc.gate == QEFT_GATE_TOKEN else (n,), True)
        pw, po = _take(at, "w_pre", w_pre, torch.float16, (n,))[0], _take(at, "w_post", w_post, torch.float16, (n,), True)[0]
        a = qeft_norm_fwd_t(pr, py, pg, pw, po, ph, px, ldr, ldy, ldg, ldh, ldx, m)
        st = raw.qeft_norm_fwd(C.byref(desc), C.byref(a), _stream())
    _check(st, "qeft_norm_fwd")
    return (r if y is None else h), x


def qeft_norm_workspace(desc: qeft_norm_desc_t, m: int) -> int:
    return int(raw.qeft_norm_workspace(C.byref(desc), m))


def qeft_norm_bwd(desc: qeft_norm_desc_t, dx: torch.Tensor, h: torch.Tensor, w_pre: torch.Tensor, dh: torch.Tensor | None = None,
                  y: torch.Tensor | None = None, w_post: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                  dr: torch.Tensor | None = None, dy: torch.Tensor | None = None, dw_pre: torch.Tensor | None = None,
                  dw_post: torch.Tensor | None = None, dgate: torch.Tensor | None = None, accumulate=False, ws: torch.Tensor | None = None):
    """(dr, dy, dw_pre, dw_post, dgate) of qeft_norm_fwd's r, y, w_pre, w_post and gate, from the gradients of x and h and the stored h.
    Gradients of what the call does not have are None; those not given are allocated, False leaves one out.  accumulate: the sums over rows (dw_pre, dw_post, a
    channel gate's dgate) are added to what the given tensors hold."""
    m, n, dev = dx.shape[0], desc.n, dx.device
    sums = torch.zeros if accumulate else torch.empty

    def out(t, has, make):
        return None if t is False or not has else make() if t is None else t

    dr = out(dr, True, lambda: _empty_rows(m, n, _residual(desc), dev))
    dy = out(dy, y is not None, lambda: _empty_rows(m, n, torch.float16, dev))
    dw_pre = out(dw_pre, True, lambda: sums(n, dtype=torch.float32, device=dev))
    dw_post = out(dw_post, w_post is not None, lambda: sums(n, dtype=torch.float32, device=dev))
    token = desc.gate == QEFT_GATE_TOKEN
    dgate = out(dgate, gate is not None, lambda: _empty_rows(m, n, torch.float16, dev) if token else sums(n, dtype=torch.float32, device=dev))
    if ws is None:
        size = qeft_norm_workspace(desc, m)
        ws = torch.empty(size, dtype=torch.uint8, device=dev) if size else None
    st = _native.norm_bwd(desc, dx, h, w_pre, dh, y, w_post, gate, dr, dy, dw_pre, dw_post, dgate, accumulate, ws)
    if st is None:
        at, res = "qeft_norm_bwd", _residual(desc)
        half, f32 = torch.float16, torch.float32
        pdx, lddx = _take(at, "dx", dx, half, (m, n))
        ph, ldh = _take(at, "h", h, res, (m, n))
        pdh, lddh = _take(at, "dh", dh, res, (m, n), True)
        py, ldy = _take(at, "y", y, half, (m, n), True)
        pg, ldg = _take(at, "gate", gate, half, (m, n) if token else (n,), True)
        pw, po = _take(at, "w_pre", w_pre, half, (n,))[0], _take(at, "w_post", w_post, half, (n,), True)[0]
        pdr, lddr = _take(at, "dr", dr, res, (m, n), True)
        pdy, lddy = _take(at, "dy", dy, half, (m, n), True)
        pdg, lddg = _take(at, "dgate", dgate, half, (m, n), True) if token else _take(at, "dgate", dgate, f32, (n,), True)
        pdw, pdo = _take(at, "dw_pre", dw_pre, f32, (n,), True)[0], _take(at, "dw_post", dw_post, f32, (n,), True)[0]
        pws, nws = _c_workspace(at, ws)
        a = qeft_norm_bwd_t(pdx, pdh, ph, py, pg, pw, po, pdr, pdy, pdg, pdw, pdo, lddx, lddh, ldh, ldy, ldg, lddr, lddy, lddg, m,
                            int(bool(accumulate)), pws, nws)
        st = raw.qeft_norm_bwd(C.byref(desc), C.byref(a), _stream())
    _check(st, "qeft_norm_bwd")
    return dr, dy, dw_pre, dw_post, dgate


# ---- the ends of a step: log probabilities, norms of heads with rotation, the optimizer ----------------------------------------------------------

def make_logprob_desc(n, dtype=torch.float16, scale=1.0) -> qeft_logprob_desc_t:
    """n logits of dtype (float16 or float32) a row, scaled by `scale` (one over the temperature)."""
    return qeft_logprob_desc_t(n, _DTYPES[dtype], scale)


def _logits(desc):
    return torch.float32 if desc.dtype == QEFT_DTYPE_F32 else torch.float16


def qeft_logprob_workspace(desc: qeft_logprob_desc_t, m: int, top: int = 0) -> int:
    return int(raw.qeft_logprob_workspace(C.byref(desc), m, top))


def _logprob_outputs(desc, z, token, logp, lse, entropy, top, ws):
    m, dev = z.shape[0], z.device
    new = lambda t, has: None if t is False or not has else torch.empty(m, dtype=torch.float32, device=dev) if t is None else t  # noqa: E731
    logp, lse, entropy = new(logp, token is not None), new(lse, True), new(entropy, True)
    if ws is None:
        n = qeft_logprob_workspace(desc, m, top)
        ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    return logp, lse, entropy, ws


def _c_logprob_fwd(at, desc, z, token, logp, lse, entropy, top, top_logp, top_index, ws):
    m = z.shape[0]
    pz, ldz = _take(at, "z", z, _logits(desc), (m, desc.n))
    pt = _take(at, "token", token, torch.int32, (m,), True)[0]
    pl, ps, pe = (_take(at, name, t, torch.float32, (m,), True)[0] for name, t in (("logp", logp), ("lse", lse), ("entropy", entropy)))
    (pv, ldv), (pi, ldi) = _take(at, "top_logp", top_logp, torch.float32, (m, top), True), _take(at, "top_index", top_index, torch.int32, (m, top), True)
    if m > 1 and top_logp is not None and top_index is not None and ldv != ldi:
        _fail(QEFT_ERR_SHAPE, at, "top_logp and top_index differ in pitch")
    pw, nw = _c_workspace(at, ws)
    return qeft_logprob_fwd_t(pz, pt, pl, ps, pe, pv, pi, ldz, ldv if m > 1 else top, m, top, pw, nw)


def qeft_logprob_fwd(desc: qeft_logprob_desc_t, z: torch.Tensor, token: torch.Tensor | None = None, top: int = 0, logp: torch.Tensor | None = None,
                     lse: torch.Tensor | None = None, entropy: torch.Tensor | None = None, top_logp: torch.Tensor | None = None,
                     top_index: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """(logp, lse, entropy, top_logp, top_index) of rows of logits z [m][n] and tokens int32 [m]; rows whose token is not in 0 .. n - 1 are left out.  Outputs that are
    not given are allocated, False leaves one out; without tokens logp is None, with top = 0 the alternatives are."""
    logp, lse, entropy, ws = _logprob_outputs(desc, z, token, logp, lse, entropy, top, ws)
    if top > 0:
        top_logp = torch.empty((z.shape[0], top), dtype=torch.float32, device=z.device) if top_logp is None else top_logp
        top_index = torch.empty((z.shape[0], top), dtype=torch.int32, device=z.device) if top_index is None else top_index
    st = _native.logprob_fwd(desc, z, token, logp, lse, entropy, top, top_logp, top_index, ws)
    if st is None:
        a = _c_logprob_fwd("qeft_logprob_fwd", desc, z, token, logp, lse, entropy, top, top_logp, top_index, ws)
        st = raw.qeft_logprob_fwd(C.byref(desc), C.byref(a), _stream())
    _check(st, "qeft_logprob_fwd")
    return logp, lse, entropy, top_logp, top_index


def _c_logprob_bwd(at, desc, z, lse, token, dlogp, dlse, entropy, dentropy, dz):
    m = z.shape[0]
    pz, ldz = _take(at, "z", z, _logits(desc), (m, desc.n))
    pdz, lddz = _take(at, "dz", dz, _logits(desc), (m, desc.n))
    pt = _take(at, "token", token, torch.int32, (m,), True)[0]
    pl, pe, pdl, pds, pde = (_take(at, name, t, torch.float32, (m,), True)[0]
                             for name, t in (("lse", lse), ("entropy", entropy), ("dlogp", dlogp), ("dlse", dlse), ("dentropy", dentropy)))
    return qeft_logprob_bwd_t(pz, pt, pl, pe, pdl, pds, pde, pdz, ldz, lddz, m)


def qeft_logprob_bwd(desc: qeft_logprob_desc_t, z: torch.Tensor, lse: torch.Tensor, token: torch.Tensor | None = None, dlogp: torch.Tensor | None = None,
                     dlse: torch.Tensor | None = None, entropy: torch.Tensor | None = None, dentropy: torch.Tensor | None = None,
                     dz: torch.Tensor | None = None) -> torch.Tensor:
    """The logits' gradient (of their dtype; dz may be z) from those of logp, lse and entropy, fp32 [m]; lse, and with dentropy entropy, as the forward gave them."""
    if dz is None:
        dz = _empty_rows(z.shape[0], desc.n, z.dtype, z.device)
    st = _native.logprob_bwd(desc, z, lse, token, dlogp, dlse, entropy, dentropy, dz)
    if st is None:
        a = _c_logprob_bwd("qeft_logprob_bwd", desc, z, lse, token, dlogp, dlse, entropy, dentropy, dz)
        st = raw.qeft_logprob_bwd(C.byref(desc), C.byref(a), _stream())
    _check(st, "qeft_logprob_bwd")
    return dz


def qeft_logprob_fwd_bwd(desc: qeft_logprob_desc_t, z: torch.Tensor, token: torch.Tensor | None = None, dlogp: torch.Tensor | None = None,
                         dlse: torch.Tensor | None = None, dentropy: torch.Tensor | None = None, dz: torch.Tensor | None = None,
                         logp: torch.Tensor | None = None, lse: torch.Tensor | None = None, entropy: torch.Tensor | None = None,
                         ws: torch.Tensor | None = None):
    """(dz, logp, lse, entropy): qeft_logprob_fwd and qeft_logprob_bwd in one call, where the gradients are known before, as those of a mean loss are."""
    logp, lse, entropy, ws = _logprob_outputs(desc, z, token, logp, lse, entropy, 0, ws)
    if dz is None:
        dz = _empty_rows(z.shape[0], desc.n, z.dtype, z.device)
    st = _native.logprob_fwd_bwd(desc, z, token, dlogp, dlse, dentropy, dz, logp, lse, entropy, ws)
    if st is None:
        at = "qeft_logprob_fwd_bwd"
        a = _c_logprob_fwd(at, desc, z, token, logp, lse, entropy, 0, None, None, ws)
        b = _c_logprob_bwd(at, desc, z, None, token, dlogp, dlse, None, dentropy, dz)
        st = raw.qeft_logprob_fwd_bwd(C.byref(desc), C.byref(a), C.byref(b), _stream())
    _check(st, "qeft_logprob_fwd_bwd")
    return dz, logp, lse, entropy


def make_qk_desc(head_dim, heads, kv_heads, rot_dim=0, eps=1e-6) -> qeft_qk_desc_t:
    return qeft_qk_desc_t(head_dim, heads, kv_heads, rot_dim, eps)


def _c_turn(at, desc, m, rot, pos):
    """Pointers of positions and rotations, the table's pitch and length."""
    pr, ldr = _take(at, "rot", rot, torch.float32, (None, desc.rot_dim), True)
    return _take(at, "pos", pos, torch.int32, (m,), True)[0], pr, ldr, rot.shape[0] if rot is not None else 0


def qeft_qk_norm_fwd(desc: qeft_qk_desc_t, q: torch.Tensor | None, k: torch.Tensor | None, w_q: torch.Tensor | None = None, w_k: torch.Tensor | None = None,
                     rot: torch.Tensor | None = None, pos: torch.Tensor | None = None, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """(q_out, k_out): every head of q fp16 [m][heads * head_dim] and k [m][kv_heads * head_dim] normed (with w_q, w_k fp16 [head_dim]; None: not normed), then rotated by
    rot fp32 [positions][rot_dim] at pos int32 [m] (None: the row's number).  q or k may be None."""
    q_out, k_out = (None if x is None else torch.empty_like(x, memory_format=torch.contiguous_format) if y is None else y for x, y in ((q, q_out), (k, k_out)))
    st = _native.qk_norm_fwd(desc, q, k, w_q, w_k, rot, pos, q_out, k_out)
    if st is None:
        at, half, d = "qeft_qk_norm_fwd", torch.float16, desc.head_dim
        m = (k if q is None else q).shape[0] if q is not None or k is not None else 0
        (pq, ldq), (pqo, ldqo) = (_take(at, name, t, half, (m, desc.heads * d), q is None) for name, t in (("q", q), ("q_out", q_out)))
        (pk, ldk), (pko, ldko) = (_take(at, name, t, half, (m, desc.kv_heads * d), k is None) for name, t in (("k", k), ("k_out", k_out)))
        pwq, pwk = (_take(at, name, t, half, (d,), True)[0] for name, t in (("w_q", w_q), ("w_k", w_k)))
        pp, pr, ldr, positions = _c_turn(at, desc, m, rot, pos)
        a = qeft_qk_fwd_t(pq, pk, pwq, pwk, pqo, pko, pp, pr, ldq, ldk, ldqo, ldko, ldr, m, positions)
        st = raw.qeft_qk_norm_fwd(C.byref(desc), C.byref(a), _stream())
    _check(st, "qeft_qk_norm_fwd")
    return q_out, k_out


def qeft_qk_norm_workspace(desc: qeft_qk_desc_t, m: int) -> int:
    return int(raw.qeft_qk_norm_workspace(C.byref(desc), m))


def qeft_qk_norm_bwd(desc: qeft_qk_desc_t, gq: torch.Tensor | None, gk: torch.Tensor | None, q: torch.Tensor | None = None, k: torch.Tensor | None = None,
                     w_q: torch.Tensor | None = None, w_k: torch.Tensor | None = None, rot: torch.Tensor | None = None, pos: torch.Tensor | None = None,
                     dq: torch.Tensor | None = None, dk: torch.Tensor | None = None, dw_q: torch.Tensor | None = None, dw_k: torch.Tensor | None = None,
                     accumulate=False, ws: torch.Tensor | None = None):
    """(dq, dk, dw_q, dw_k) of qeft_qk_norm_fwd's q, k, w_q and w_k, from the gradients gq, gk of its outputs and q, k as it took them (needed where the heads are normed).
    Gradients of what the call does not have are None; those not given are allocated, False leaves one out.  accumulate: added to what dw_q, dw_k hold."""
    some = gk if gq is None else gq
    m, d = (some.shape[0] if some is not None else 0), desc.head_dim
    sums = torch.zeros if accumulate else torch.empty

    def out(t, has, make):
        return None if t is False or not has else make() if t is None else t

    dq = out(dq, gq is not None, lambda: torch.empty_like(gq, memory_format=torch.contiguous_format))
    dk = out(dk, gk is not None, lambda: torch.empty_like(gk, memory_format=torch.contiguous_format))
    dw_q = out(dw_q, gq is not None and w_q is not None, lambda: sums(d, dtype=torch.float32, device=gq.device))
    dw_k = out(dw_k, gk is not None and w_k is not None, lambda: sums(d, dtype=torch.float32, device=gk.device))
    if ws is None and (dw_q is not None or dw_k is not None):
        n = qeft_qk_norm_workspace(desc, m)
        ws = torch.empty(n, dtype=torch.uint8, device=some.device) if n else None
    st = _native.qk_norm_bwd(desc, gq, gk, q, k, w_q, w_k, rot, pos, dq, dk, dw_q, dw_k, accumulate, ws)
    if st is None:
        at, half, f32 = "qeft_qk_norm_bwd", torch.float16, torch.float32
        (pgq, ldgq), (pq, ldq), (pdq, lddq) = (_take(at, name, t, half, (m, desc.heads * d), True) for name, t in (("gq", gq), ("q", q), ("dq", dq)))
        (pgk, ldgk), (pk, ldk), (pdk, lddk) = (_take(at, name, t, half, (m, desc.kv_heads * d), True) for name, t in (("gk", gk), ("k", k), ("dk", dk)))
        pwq, pwk = (_take(at, name, t, half, (d,), True)[0] for name, t in (("w_q", w_q), ("w_k", w_k)))
        pdwq, pdwk = (_take(at, name, t, f32, (d,), True)[0] for name, t in (("dw_q", dw_q), ("dw_k", dw_k)))
        pp, pr, ldr, positions = _c_turn(at, desc, m, rot, pos)
        pws, nws = _c_workspace(at, ws)
        a = qeft_qk_bwd_t(pgq, pgk, pq, pk, pwq, pwk, pdq, pdk, pdwq, pdwk, pp, pr, ldgq, ldgk, ldq, ldk, lddq, lddk, ldr, m, positions, int(bool(accumulate)), pws, nws)
        st = raw.qeft_qk_norm_bwd(C.byref(desc), C.byref(a), _stream())
    _check(st, "qeft_qk_norm_bwd")
    return dq, dk, dw_q, dw_k


def qeft_cache_append_norm(cache: Cache, table: torch.Tensor, k: torch.Tensor, v: torch.Tensor, index: torch.Tensor, seq: torch.Tensor | None = None,
                           q: torch.Tensor | None = None, q_out: torch.Tensor | None = None, rot: torch.Tensor | None = None, pos: torch.Tensor | None = None,
                           w_q: torch.Tensor | None = None, w_k: torch.Tensor | None = None, eps: float = 1e-6) -> torch.Tensor | None:
    """qeft_cache_append with every head of q and k normed before its rotation (w_q, w_k fp16 [head_dim]; None: those heads are not)."""
    if q is not None and q_out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    st = _native.cache_append_norm(cache.desc, cache.k, cache.v, table, k, v, index, seq, q, q_out, rot, pos, w_q, w_k, eps)
    if st is None:
        at, d = "qeft_cache_append_norm", cache.desc
        pools, tab, a = _c_append(at, cache, table, k, v, index, seq, q, q_out, rot, pos)
        pwq, pwk = (_take(at, name, t, torch.float16, (d.head_dim,), True)[0] for name, t in (("w_q", w_q), ("w_k", w_k)))
        norm = qeft_append_norm_t(pwq, pwk, float(eps))
        st = raw.qeft_cache_append_norm(C.byref(d), C.byref(pools), C.byref(tab), C.byref(a), C.byref(norm), _stream())
    _check(st, "qeft_cache_append_norm")
    return q_out


def make_adamw_states(weights, bits=32) -> dict:
    """Zero states of an optimizer for these weights, as TensorList takes them: m, v and, with bits = 8, m_scales, v_scales."""
    if bits not in (8, 32):
        _fail(QEFT_ERR_UNSUPPORTED, "make_adamw_states", f"states of {bits} bits")
    blocks = lambda w: -(-w.numel() // QEFT_STATE_BLOCK)  # noqa: E731
    out = {name: [torch.zeros(w.shape, dtype=torch.uint8 if bits == 8 else torch.float32, device=w.device) for w in weights] for name in ("m", "v")}
    if bits == 8:
        out.update({name: [torch.zeros(blocks(w), dtype=torch.uint8, device=w.device) for w in weights] for name in ("m_scales", "v_scales")})
    return out


class TensorList:
    """What an optimizer's step goes over, and the plan of it on the GPU: lists of contiguous tensors, one entry for each trained tensor.  grads fp16 or fp32; weights
    fp16 and / or masters fp32; m, v fp32, or uint8 with m_scales, v_scales; decay a number or one for each.  Without weights and masters the list serves
    qeft_grad_norm alone.  The list keeps the tensors; their contents may change between calls, their addresses may not."""

    def __init__(self, grads, weights=None, masters=None, m=None, v=None, m_scales=None, v_scales=None, decay=0.0):
        at, n = "TensorList", len(grads)
        parts = dict(weight=weights, master=masters, grad=grads, m=m, v=v, m_scale=m_scales, v_scale=v_scales)
        self.tensors = {name: None if ts is None else list(ts) for name, ts in parts.items()}
        decays = [float(decay)] * n if not hasattr(decay, "__len__") else [float(x) for x in decay]
        grad = grads[0].dtype if n else torch.float32
        state = m[0].dtype if m is not None and n else torch.float32
        if grad not in _DTYPES or state not in (torch.uint8, torch.float32):
            _fail(QEFT_ERR_UNSUPPORTED, at, f"gradients of {grad}, states of {state}")
        types = dict(weight=torch.float16, master=torch.float32, grad=grad, m=state, v=state, m_scale=torch.uint8, v_scale=torch.uint8)
        self.device = grads[0].device if n else torch.device("cuda", torch.cuda.current_device())
        self.index = -1 if self.device.index is None else self.device.index
        if len(decays) != n or any(ts is not None and len(ts) != n for ts in self.tensors.values()):
            _fail(QEFT_ERR_SHAPE, at, "lists of different lengths")
        rows = (qeft_tensor_t * max(n, 1))()
        for i in range(n):
            rows[i].n, rows[i].decay = grads[i].numel(), decays[i]
            for name, ts in self.tensors.items():
                if ts is None:
                    continue
                t, size = ts[i], -(-rows[i].n // QEFT_STATE_BLOCK) if name.endswith("scale") else rows[i].n
                if t.dtype != types[name]:
                    _fail(QEFT_ERR_UNSUPPORTED, at, f"{name} {i} is {t.dtype}, not {types[name]}")
                if t.numel() != size:
                    _fail(QEFT_ERR_SHAPE, at, f"{name} {i} has {t.numel()} values, not {size}")
                if not t.is_contiguous() or not t.is_cuda or t.device != self.device or t.device.index != torch.cuda.current_device():
                    _fail(QEFT_ERR_UNSUPPORTED, at, f"{name} {i} is not contiguous on the current GPU")
                setattr(rows[i], name, t.data_ptr())
        size = int(raw.qeft_tensors_plan_bytes(rows, n))
        plan = torch.zeros(max(size, 16), dtype=torch.uint8)
        self.c = qeft_tensors_t()
        _check(raw.qeft_tensors_plan(rows, n, _DTYPES[grad], 8 if state == torch.uint8 else 32, plan.data_ptr(), size, C.byref(self.c)), "qeft_tensors_plan")
        self.plan = plan.to(self.device)
        self.c.plan = self.plan.data_ptr()

    def here(self, at):
        if self.index != torch.cuda.current_device():
            _fail(QEFT_ERR_UNSUPPORTED, at, "the list's tensors are not on the current GPU")
        return C.byref(self.c)


def _number_at(at, name, t, dtype):
    """Pointer of a number on the device, the first entry of t."""
    if t is None:
        return 0
    if t.dtype != dtype or t.numel() < 1:
        _fail(QEFT_ERR_UNSUPPORTED, at, f"{name} is {t.dtype} of {t.numel()} values, not {dtype}")
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        _fail(QEFT_ERR_UNSUPPORTED, at, f"{name} is not on the current GPU")
    return t.data_ptr()


def qeft_adamw_step(tensors: TensorList, lr: float | torch.Tensor, step: int | torch.Tensor, beta1=0.9, beta2=0.999, eps=1e-8, factor: torch.Tensor | None = None,
                    stochastic=False, seed=0) -> None:
    """One step of AdamW over the list, in place.  lr and step (1 for the first) are numbers, or tensors on the GPU (fp32, int32) that hold one; factor: fp32 on the
    GPU, multiplies the gradients, and the step is left out where it is not finite.  stochastic: fp16 weights without a master are rounded so, as 8-bit states always are, by
    seed, step and place."""
    st = _native.adamw_step(tensors.c, tensors.index, lr, step, beta1, beta2, eps, factor, stochastic, seed)
    if st is None:
        at = "qeft_adamw_step"
        lr_at, step_at = (_number_at(at, name, t, kind) if isinstance(t, torch.Tensor) else 0 for name, t, kind in (("lr", lr, torch.float32), ("step", step, torch.int32)))
        a = qeft_adamw_t(0.0 if lr_at else lr, beta1, beta2, eps, 0 if step_at else step, seed & 0xFFFFFFFFFFFFFFFF, lr_at, step_at,
                         _number_at(at, "factor", factor, torch.float32), int(bool(stochastic)))
        st = raw.qeft_adamw_step(tensors.here(at), C.byref(a), _stream())
    _check(st, "qeft_adamw_step")


def qeft_grad_norm_workspace(tensors: TensorList) -> int:
    return int(raw.qeft_grad_norm_workspace(C.byref(tensors.c)))


def qeft_grad_norm(tensors: TensorList, max_norm=float("inf"), scale=1.0, out: torch.Tensor | None = None, steps: torch.Tensor | None = None,
                   ws: torch.Tensor | None = None) -> torch.Tensor:
    """fp32 [2]: the norm of all gradients times scale, and the factor that brings them back by scale and to a norm of max_norm at most (not-a-number where the norm is
    not finite).  steps: int32 on the GPU, counted up by one where it is finite."""
    if out is None:
        out = torch.empty(2, dtype=torch.float32, device=tensors.device)
    if ws is None:
        n = qeft_grad_norm_workspace(tensors)
        ws = torch.empty(n, dtype=torch.uint8, device=tensors.device) if n else None
    st = _native.grad_norm(tensors.c, tensors.index, max_norm, scale, out, steps, ws)
    if st is None:
        at = "qeft_grad_norm"
        po, ps = _take(at, "out", out, torch.float32, (2,))[0], _number_at(at, "steps", steps, torch.int32)
        pw, nw = _c_workspace(at, ws)
        a = qeft_grad_norm_t(float(scale), float(max_norm), po, ps, pw, nw)
        st = raw.qeft_grad_norm(tensors.here(at), C.byref(a), _stream())
    _check(st, "qeft_grad_norm")
    return out
