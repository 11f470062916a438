"""Python binding of the HIP gradient-dropping library (``libgd.so``).

Argument marshalling only: torch supplies device memory and the current HIP
stream; every step of the compressor runs in the library's kernels.  There is
no CPU fallback: if ``libgd.so`` has not been built, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgd.so")

GD_GLOBAL, GD_PER_TENSOR = 0, 1
GD_QUANT_NONE, GD_QUANT_SIGN_MEAN, GD_QUANT_THRESHOLD, GD_QUANT_GLOBAL_MEAN, GD_QUANT_COLUMN_MEAN = 0, 1, 2, 3, 4

STATUS = {
    0: "GD_OK",
    1: "GD_ERR_ARG",
    2: "GD_ERR_LAYOUT",
    3: "GD_ERR_CAPACITY",
    4: "GD_ERR_ALIGN",
    5: "GD_ERR_OOM",
    6: "GD_ERR_HIP",
}

EXPORTS = [
    "gd_create",
    "gd_destroy",
    "gd_keep_count",
    "gd_keep_total",
    "gd_compress",
    "gd_compress_sampled",
    "gd_set_columns",
    "gd_compress_pull",
    "gd_apply_quantised",
    "gd_quant_centres",
    "gd_apply_sparse",
    "gd_status_string",
    "gd_profile_enable",
    "gd_profile_read",
    "gd_debug_force_bracket",
    "gd_debug_apply_form",
    "gd_debug_state",
    "gd_compress_static",
    "gd_norm_create",
    "gd_norm_destroy",
    "gd_norm_forward",
    "gd_norm_backward",
    "gd_layernorm_create",
    "gd_layernorm_destroy",
    "gd_layernorm_forward",
    "gd_layernorm_backward",
    "gd_embed_create",
    "gd_embed_destroy",
    "gd_embed_forward",
    "gd_embed_backward",
    "gd_gated_create",
    "gd_gated_destroy",
    "gd_gated_forward",
    "gd_gated_backward",
    "gd_logprob_create",
    "gd_logprob_destroy",
    "gd_logprob_forward",
    "gd_logprob_backward",
    "gd_distill_create",
    "gd_distill_destroy",
    "gd_distill_forward",
    "gd_distill_backward",
    "gd_adamw_create",
    "gd_adamw_destroy",
    "gd_adamw_blocks",
    "gd_adamw_step",
    "gd_adamw_decode",
    "gd_linear_create",
    "gd_linear_destroy",
    "gd_linear_forward",
    "gd_linear_backward",
    "gd_quantise_rows",
]


class GDError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {STATUS.get(status, status)} ({_lib().gd_status_string(status).decode()})")


class _Sparse(ctypes.Structure):
    _fields_ = [
        ("idx", ctypes.c_void_p),
        ("val", ctypes.c_void_p),
        ("sign_bits", ctypes.c_void_p),
        ("means", ctypes.c_void_p),
        ("tensor_counts", ctypes.c_void_p),
        ("capacity", ctypes.c_uint64),
    ]


def _struct(name, **fields):
    """A ctypes structure from (C type, space-separated field names) pairs in order."""
    return type(name, (ctypes.Structure,), {"_fields_": [(f, t) for t, names in fields["of"] for f in names.split()]})


_vp, _u64, _dbl, _int, _flt = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_double, ctypes.c_int, ctypes.c_float
_NormIO = _struct("_NormIO", of=[(_u64, "rows"), (_vp, "x residual weight sum y y_scale"),
                                 (_u64, "x_stride residual_stride sum_stride y_stride"), (_flt, "eps")])
_NormGrad = _struct("_NormGrad", of=[(_u64, "rows"), (_vp, "dy x weight dsum dx dweight"),
                                     (_u64, "dy_stride x_stride dsum_stride dx_stride"), (_flt, "eps"),
                                     (_int, "accumulate")])
_LayerNormIO = _struct("_LayerNormIO", of=[(_u64, "rows"), (_vp, "x residual weight bias sum y y_scale"),
                                           (_u64, "x_stride residual_stride sum_stride y_stride"), (_flt, "eps")])
_LayerNormGrad = _struct("_LayerNormGrad", of=[(_u64, "rows"), (_vp, "dy x weight dsum dx dweight dbias"),
                                               (_u64, "dy_stride x_stride dsum_stride dx_stride"), (_flt, "eps"),
                                               (_int, "accumulate")])
_EmbedIO = _struct("_EmbedIO", of=[(_u64, "rows"), (_vp, "tokens weight y"), (_u64, "weight_stride y_stride"),
                                   (_flt, "scale"), (_int, "index")])
_EmbedGrad = _struct("_EmbedGrad", of=[(_u64, "rows"), (_vp, "tokens dy dweight"), (_u64, "dy_stride dweight_stride"),
                                       (_flt, "scale"), (_int, "index accumulate")])
_GatedIO = _struct("_GatedIO", of=[(_u64, "rows"), (_vp, "x weight x_scale weight_scale bias y pre"),
                                   (_u64, "x_stride weight_stride y_stride pre_stride")])
_GatedGrad = _struct("_GatedGrad", of=[(_u64, "rows"), (_vp, "dy x weight pre dz dx dweight dbias"),
                                       (_u64, "dy_stride x_stride weight_stride pre_stride dz_stride dx_stride "
                                              "dweight_stride"), (_int, "accumulate")])
_LogProbIO = _struct("_LogProbIO", of=[(_u64, "rows"), (_vp, "logits tokens logp entropy stats top_logp top_id"),
                                       (_u64, "stride"), (_flt, "scale"), (_int, "index"), (ctypes.c_uint32, "top")])
_LogProbGrad = _struct("_LogProbGrad", of=[(_u64, "rows"), (_vp, "logits tokens dlogp dentropy stats entropy dlogits "
                                                                 "logp_out entropy_out"),
                                           (_u64, "stride dlogits_stride"), (_flt, "scale"), (_int, "index")])
_DistillIO = _struct("_DistillIO", of=[(_u64, "rows"), (_vp, "logits ids teacher loss stats"),
                                       (_u64, "stride ids_stride teacher_stride"), (_flt, "scale"),
                                       (ctypes.c_uint32, "top"), (_int, "index teacher_type")])
_DistillGrad = _struct("_DistillGrad", of=[(_u64, "rows"), (_vp, "logits ids teacher dloss stats dlogits loss_out"),
                                           (_u64, "stride ids_stride teacher_stride dlogits_stride"), (_flt, "scale"),
                                           (ctypes.c_uint32, "top"), (_int, "index teacher_type")])
_AdamWIO = _struct("_AdamWIO", of=[(_vp, "params grad m v m_unit v_unit copy norm"), (_int, "grad_type copy_type"),
                                   (_u64, "step"), (_dbl, "lr beta1 beta2 eps weight_decay max_norm grad_scale")])
_LinearIO = _struct("_LinearIO", of=[(_u64, "rows"), (_vp, "x weight x_scale weight_scale bias residual y pre"),
                                     (_u64, "x_stride weight_stride residual_stride y_stride pre_stride")])
_LinearGrad = _struct("_LinearGrad", of=[(_u64, "rows"), (_vp, "dy x weight pre dz dx dweight dbias"),
                                         (_u64, "dy_stride x_stride weight_stride pre_stride dz_stride dx_stride "
                                                "dweight_stride"), (_int, "accumulate")])

_LIB = None


def _lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build the HIP library first (python -c "
                          "'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(LIB_PATH)
    vp, u64, u32, dbl, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_double, ctypes.c_int
    lib.gd_create.argtypes = [ctypes.POINTER(vp), vp, u32]
    lib.gd_create.restype = i32
    lib.gd_destroy.argtypes = [vp]
    lib.gd_destroy.restype = None
    lib.gd_keep_count.argtypes = [u64, dbl]
    lib.gd_keep_count.restype = u64
    lib.gd_keep_total.argtypes = [vp, dbl, i32]
    lib.gd_keep_total.restype = u64
    lib.gd_compress.argtypes = [vp, vp, vp, vp, dbl, i32, i32, ctypes.POINTER(_Sparse), vp]
    lib.gd_compress.restype = i32
    lib.gd_compress_sampled.argtypes = [vp, vp, vp, vp, dbl, i32, u32, u64, i32, ctypes.POINTER(_Sparse), vp]
    lib.gd_compress_sampled.restype = i32
    lib.gd_apply_quantised.argtypes = [vp, vp, u32, vp, vp, vp, vp, i32, ctypes.c_float, vp]
    lib.gd_apply_quantised.restype = i32
    lib.gd_compress_pull.argtypes = [vp, vp, vp, dbl, i32, ctypes.POINTER(_Sparse), vp]
    lib.gd_compress_pull.restype = i32
    lib.gd_set_columns.argtypes = [vp, vp]
    lib.gd_set_columns.restype = i32
    lib.gd_quant_centres.argtypes = [vp, i32]
    lib.gd_quant_centres.restype = u64
    lib.gd_apply_sparse.argtypes = [vp, u64, u32, vp, vp, vp, ctypes.c_float, vp]
    lib.gd_apply_sparse.restype = i32
    lib.gd_status_string.argtypes = [i32]
    lib.gd_status_string.restype = ctypes.c_char_p
    lib.gd_profile_enable.argtypes = [vp, i32]
    lib.gd_profile_enable.restype = i32
    lib.gd_profile_read.argtypes = [vp, ctypes.POINTER(dbl), ctypes.POINTER(u64)]
    lib.gd_profile_read.restype = i32
    lib.gd_debug_force_bracket.argtypes = [vp, i32]
    lib.gd_debug_force_bracket.restype = i32
    lib.gd_debug_apply_form.argtypes = [i32]
    lib.gd_debug_apply_form.restype = i32
    lib.gd_debug_state.argtypes = [vp, vp, u32, vp]
    lib.gd_debug_state.restype = i32
    lib.gd_compress_static.argtypes = [vp, u32, vp, vp, vp, dbl, i32, i32, ctypes.POINTER(_Sparse), vp]
    lib.gd_compress_static.restype = i32
    for what, args in (("norm", [ctypes.POINTER(vp), u32, i32]), ("layernorm", [ctypes.POINTER(vp), u32, i32]),
                       ("embed", [ctypes.POINTER(vp), u32, u32, i32, u64]),
                       ("logprob", [ctypes.POINTER(vp), u32, i32, u64]), ("distill", [ctypes.POINTER(vp), u32, i32, u64]), ("linear", [ctypes.POINTER(vp), u32, u32, i32, i32, u64]),
                       ("gated", [ctypes.POINTER(vp), u32, u32, i32, i32, u64]),
                       ("adamw", [ctypes.POINTER(vp), vp, u32, i32, vp])):
        create, destroy = getattr(lib, f"gd_{what}_create"), getattr(lib, f"gd_{what}_destroy")
        create.argtypes, create.restype = args, i32
        destroy.argtypes, destroy.restype = [vp], None
    for name, io in (("gd_norm_forward", _NormIO), ("gd_norm_backward", _NormGrad), ("gd_adamw_step", _AdamWIO),
                     ("gd_layernorm_forward", _LayerNormIO), ("gd_layernorm_backward", _LayerNormGrad),
                     ("gd_embed_forward", _EmbedIO), ("gd_embed_backward", _EmbedGrad),
                     ("gd_gated_forward", _GatedIO), ("gd_gated_backward", _GatedGrad),
                     ("gd_logprob_forward", _LogProbIO), ("gd_logprob_backward", _LogProbGrad),
                     ("gd_distill_forward", _DistillIO), ("gd_distill_backward", _DistillGrad),
                     ("gd_linear_forward", _LinearIO), ("gd_linear_backward", _LinearGrad)):
        getattr(lib, name).argtypes, getattr(lib, name).restype = [vp, ctypes.POINTER(io), vp], i32
    lib.gd_adamw_blocks.argtypes, lib.gd_adamw_blocks.restype = [vp], u64
    lib.gd_adamw_decode.argtypes, lib.gd_adamw_decode.restype = [vp] * 8, i32
    lib.gd_quantise_rows.argtypes, lib.gd_quantise_rows.restype = [vp, i32, u64, u64, u64, vp, u64, vp, vp], i32
    _LIB = lib
    return lib


def load() -> ctypes.CDLL:
    """Load ``libgd.so`` (raises ImportError when it has not been built)."""
    return _lib()


def keep_count(n: int, drop_ratio: float) -> int:
    return int(_lib().gd_keep_count(n, float(drop_ratio)))


def _stream_handle(stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream or None


def _check_f32(t: torch.Tensor, name: str, n: int) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous float32 tensor on the GPU")
    if t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} elements, the layout has {n}")


@dataclass
class SparseOut:
    """Device buffers of one compressed gradient (views of length k)."""

    idx: torch.Tensor  # int32 storage holding uint32 indices
    val: torch.Tensor  # float32
    tensor_counts: torch.Tensor  # int32 storage holding uint32 counts
    sign_bits: Optional[torch.Tensor] = None  # int32 storage holding uint32 words
    means: Optional[torch.Tensor] = None  # float32 [2T]
    k: int = 0


class Compressor:
    """A gradient layout (tensor offsets) bound to the device scratch of ``gd_create``."""

    def __init__(self, offsets: Sequence[int], device: Optional[torch.device] = None):
        lib = _lib()
        off = (ctypes.c_uint64 * len(offsets))(*[int(o) for o in offsets])
        self.offsets = [int(o) for o in offsets]
        self.T = len(offsets) - 1
        self.N = self.offsets[-1]
        self.device = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            st = lib.gd_create(ctypes.byref(h), off, self.T)
        if st != 0:
            raise GDError(st, "gd_create")
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None):
            _lib().gd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def keep_total(self, drop_ratio: float, per_tensor: bool = False) -> int:
        return int(_lib().gd_keep_total(self._h, float(drop_ratio), GD_PER_TENSOR if per_tensor else GD_GLOBAL))

    def alloc_out(self, drop_ratio: float, per_tensor: bool = False, quant=False,
                  capacity: Optional[int] = None) -> SparseOut:
        k = self.keep_total(drop_ratio, per_tensor)
        cap = max(k if capacity is None else capacity, 1)
        dev = self.device
        out = SparseOut(
            idx=torch.empty(cap, dtype=torch.int32, device=dev),
            val=torch.empty(cap, dtype=torch.float32, device=dev),
            tensor_counts=torch.empty(max(self.T, 1), dtype=torch.int32, device=dev),
            k=k,
        )
        if quant:
            centres = int(_lib().gd_quant_centres(self._h, int(quant)))
            out.sign_bits = torch.empty(max((cap + 31) // 32, 1), dtype=torch.int32, device=dev)
            out.means = torch.empty(max(centres, 1), dtype=torch.float32, device=dev)
        return out

    def compress(self, grad: torch.Tensor, residual: torch.Tensor, drop_ratio: float = 0.99,
                 per_tensor: bool = False, quant=False, base: Optional[torch.Tensor] = None,
                 out: Optional[SparseOut] = None, stream: Optional[torch.cuda.Stream] = None) -> SparseOut:
        """One gd_compress call; ``residual`` is updated in place.

        quant: False/GD_QUANT_NONE, True/GD_QUANT_SIGN_MEAN, or another GD_QUANT_* form.
        """
        _check_f32(grad, "grad", self.N)
        _check_f32(residual, "residual", self.N)
        if base is not None:
            _check_f32(base, "base", self.N)
        if out is None:
            out = self.alloc_out(drop_ratio, per_tensor, quant)
        sp = _Sparse(
            out.idx.data_ptr(),
            out.val.data_ptr(),
            out.sign_bits.data_ptr() if (quant and out.sign_bits is not None) else None,
            out.means.data_ptr() if (quant and out.means is not None) else None,
            out.tensor_counts.data_ptr(),
            out.idx.numel(),
        )
        st = _lib().gd_compress(
            self._h, grad.data_ptr(), None if base is None else base.data_ptr(), residual.data_ptr(),
            float(drop_ratio), GD_PER_TENSOR if per_tensor else GD_GLOBAL,
            int(quant), ctypes.byref(sp), _stream_handle(stream))
        if st != 0:
            raise GDError(st, "gd_compress")
        out.k = self.keep_total(drop_ratio, per_tensor)
        return out

    def compress_pull(self, params: torch.Tensor, copy: torch.Tensor, drop_ratio: float = 0.99,
                      per_tensor: bool = False, out: Optional[SparseOut] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> SparseOut:
        """gd_compress_pull: send params - copy; ``copy`` takes the sent values in place."""
        _check_f32(params, "params", self.N)
        _check_f32(copy, "copy", self.N)
        if out is None:
            out = self.alloc_out(drop_ratio, per_tensor)
        sp = _Sparse(out.idx.data_ptr(), out.val.data_ptr(), None, None, out.tensor_counts.data_ptr(),
                     out.idx.numel())
        st = _lib().gd_compress_pull(self._h, params.data_ptr(), copy.data_ptr(), float(drop_ratio),
                                     GD_PER_TENSOR if per_tensor else GD_GLOBAL, ctypes.byref(sp),
                                     _stream_handle(stream))
        if st != 0:
            raise GDError(st, "gd_compress_pull")
        out.k = self.keep_total(drop_ratio, per_tensor)
        return out

    def apply_quantised(self, params: torch.Tensor, idx, sign_bits, means, quant: int, lr: float = 1.0,
                        stream: Optional[torch.cuda.Stream] = None, validate: bool = False) -> None:
        """gd_apply_quantised: decode quantised pushes of this layout and apply them to params.

        validate: as for ``apply_sparse``, check first that each push's indices are strictly ascending.
        """
        _check_f32(params, "params", self.N)
        C = len(idx)
        if not (len(sign_bits) == len(means) == C):
            raise ValueError("idx, sign_bits and means must have one entry per push")
        for a, b, m in zip(idx, sign_bits, means):
            if a.dtype != torch.int32 or b.dtype != torch.int32 or m.dtype != torch.float32:
                raise TypeError("a push is int32 (uint32 bits) indices and sign words and float32 centres")
            if not (a.is_cuda and b.is_cuda and m.is_cuda and a.is_contiguous() and b.is_contiguous()
                    and m.is_contiguous()):
                raise TypeError("push tensors must be contiguous GPU tensors")
        if validate:
            _check_pushes_ascending(idx)
        arr = lambda xs: (ctypes.c_void_p * max(C, 1))(*[x.data_ptr() for x in xs])
        ip, bp, mp = arr(idx), arr(sign_bits), arr(means)
        nz = (ctypes.c_uint64 * max(C, 1))(*[a.numel() for a in idx])
        st = _lib().gd_apply_quantised(self._h, params.data_ptr(), C, ctypes.cast(ip, ctypes.c_void_p),
                                       ctypes.cast(bp, ctypes.c_void_p), ctypes.cast(mp, ctypes.c_void_p),
                                       ctypes.cast(nz, ctypes.c_void_p), int(quant), float(lr), _stream_handle(stream))
        if st != 0:
            raise GDError(st, "gd_apply_quantised")

    def set_columns(self, columns) -> None:
        """Matrix view of every tensor for the column-wise centres (gd_set_columns)."""
        import numpy as np

        c = np.ascontiguousarray(columns, dtype=np.uint32)
        if c.size != self.T:
            raise ValueError(f"need {self.T} column counts, got {c.size}")
        st = _lib().gd_set_columns(self._h, c.ctypes.data)
        if st != 0:
            raise GDError(st, "gd_set_columns")

    def quant_centres(self, quant: int) -> int:
        return int(_lib().gd_quant_centres(self._h, int(quant)))

    def compress_sampled(self, grad: torch.Tensor, residual: torch.Tensor, drop_ratio: float = 0.99,
                         per_tensor: bool = False, sample_ppm: int = 1000, seed: int = 0,
                         base: Optional[torch.Tensor] = None, out: Optional[SparseOut] = None,
                         capacity: Optional[int] = None, quant=False,
                         stream: Optional[torch.cuda.Stream] = None) -> SparseOut:
        """One gd_compress_sampled call; ``residual`` is updated in place.

        The number sent is data dependent: it is ``out.tensor_counts.sum()``
        (read it after the stream has run).  ``out.k`` is left as None.
        quant: as ``compress``, over the entries sent.
        """
        _check_f32(grad, "grad", self.N)
        _check_f32(residual, "residual", self.N)
        if base is not None:
            _check_f32(base, "base", self.N)
        if out is None:
            out = self.alloc_out(1.0, per_tensor, quant, capacity=self.N if capacity is None else capacity)
        sp = _Sparse(out.idx.data_ptr(), out.val.data_ptr(),
                     out.sign_bits.data_ptr() if (quant and out.sign_bits is not None) else None,
                     out.means.data_ptr() if (quant and out.means is not None) else None,
                     out.tensor_counts.data_ptr(),
                     out.idx.numel() if capacity is None else min(int(capacity), out.idx.numel()))
        st = _lib().gd_compress_sampled(
            self._h, grad.data_ptr(), None if base is None else base.data_ptr(), residual.data_ptr(),
            float(drop_ratio), GD_PER_TENSOR if per_tensor else GD_GLOBAL, int(sample_ppm), int(seed),
            int(quant), ctypes.byref(sp), _stream_handle(stream))
        if st != 0:
            raise GDError(st, "gd_compress_sampled")
        out.k = None
        return out

    def debug_force_bracket(self, mode: int) -> None:
        st = _lib().gd_debug_force_bracket(self._h, int(mode))
        if st != 0:
            raise GDError(st, "gd_debug_force_bracket")

    SEG_FIELDS = ("lo", "hi", "clo", "miss", "d0", "r1", "p18", "r2", "thr", "need", "zero")

    def debug_state(self):
        """(per-segment state of the last call as a list of dicts, decomposition info dict)."""
        import numpy as np

        words = np.zeros((max(self.T, 1), 16), dtype=np.uint32)
        info = np.zeros(4, dtype=np.uint64)
        st = _lib().gd_debug_state(self._h, words.ctypes.data, self.T, info.ctypes.data)
        if st != 0:
            raise GDError(st, "gd_debug_state")
        segs = [dict(zip(self.SEG_FIELDS, (int(x) for x in row[:len(self.SEG_FIELDS)])), form=int(row[-1])) for row in words]
        keys = ("unit_len", "units", "tile", "max_tiles")
        return segs, dict(zip(keys, (int(x) for x in info)))

    def profile_enable(self, every: int = 1) -> None:
        """Time dense launches 0, every, 2 * every, ... from now on (0: off)."""
        st = _lib().gd_profile_enable(self._h, int(every))
        if st != 0:
            raise GDError(st, "gd_profile_enable")

    def profile_read(self):
        """(summed milliseconds of the dense pass, number of timed launches)."""
        ms = ctypes.c_double(0.0)
        n = ctypes.c_uint64(0)
        st = _lib().gd_profile_read(self._h, ctypes.byref(ms), ctypes.byref(n))
        if st != 0:
            raise GDError(st, "gd_profile_read")
        return ms.value, n.value


def _check_pushes_ascending(idx: List[torch.Tensor]) -> None:
    """Raises GDError(GD_ERR_ARG) unless every push's indices (uint32 bits in
    int32 storage) are strictly ascending: the precondition gd_apply_sparse
    relies on and does not check.  Synchronises with the device."""
    for c, a in enumerate(idx):
        if a.numel() > 1:
            u = a.to(torch.int64) & 0xFFFFFFFF
            if not bool(torch.all(u[1:] > u[:-1])):
                raise GDError(1, f"apply: push {c} is not strictly ascending")


def apply_sparse(params: torch.Tensor, idx: List[torch.Tensor], val: List[torch.Tensor], lr: float = 1.0,
                 stream: Optional[torch.cuda.Stream] = None, validate: bool = False) -> None:
    """gd_apply_sparse: params[i] -= lr * (sum of pushed values at i, in push order).

    validate: first check that each push's indices are strictly ascending
    (unique and sorted), which the library assumes and does not check, and
    raise GDError(GD_ERR_ARG) otherwise.  This synchronises with the device.
    """
    if params.dtype != torch.float32 or not params.is_cuda or not params.is_contiguous():
        raise TypeError("params must be a contiguous float32 tensor on the GPU")
    C = len(idx)
    if len(val) != C:
        raise ValueError("idx and val must have the same number of pushes")
    for a, b in zip(idx, val):
        if a.dtype != torch.int32 or b.dtype != torch.float32 or a.numel() != b.numel():
            raise TypeError("each push is an int32 (uint32 bits) index tensor and a float32 value tensor")
        if not (a.is_cuda and b.is_cuda and a.is_contiguous() and b.is_contiguous()):
            raise TypeError("push tensors must be contiguous GPU tensors")
    if validate:
        _check_pushes_ascending(idx)
    ip = (ctypes.c_void_p * max(C, 1))(*[a.data_ptr() for a in idx])
    vp = (ctypes.c_void_p * max(C, 1))(*[b.data_ptr() for b in val])
    nz = (ctypes.c_uint64 * max(C, 1))(*[a.numel() for a in idx])
    st = _lib().gd_apply_sparse(params.data_ptr(), params.numel(), C, ctypes.cast(ip, ctypes.c_void_p),
                                ctypes.cast(vp, ctypes.c_void_p), ctypes.cast(nz, ctypes.c_void_p), float(lr),
                                _stream_handle(stream))
    if st != 0:
        raise GDError(st, "gd_apply_sparse")


def debug_apply_form(form: int) -> None:
    """gd_debug_apply_form: the form of later applies in this process (0 chosen per call, 1 scattered,
    2 streaming wherever the parameters are 16-byte aligned).  A test hook; results do not change."""
    st = _lib().gd_debug_apply_form(int(form))
    if st != 0:
        raise GDError(st, "gd_debug_apply_form")


STATIC_MAX_ELEMENTS = 1 << 21
STATIC_MAX_TENSORS = 64


def compress_static(offsets: Sequence[int], grad: torch.Tensor, residual: torch.Tensor, out: SparseOut,
                    drop_ratio: float = 0.99, per_tensor: bool = False, quant=False,
                    base: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> SparseOut:
    """gd_compress_static: gd_compress without a context and without any allocation, for layouts of at
    most STATIC_MAX_TENSORS tensors and STATIC_MAX_ELEMENTS elements.  ``out`` must be preallocated (for
    example by ``Compressor.alloc_out`` of the same layout); its ``k`` is set to the kept count."""
    n = int(offsets[-1])
    _check_f32(grad, "grad", n)
    _check_f32(residual, "residual", n)
    if base is not None:
        _check_f32(base, "base", n)
    off = (ctypes.c_uint64 * len(offsets))(*[int(o) for o in offsets])
    sp = _Sparse(out.idx.data_ptr(), out.val.data_ptr(),
                 out.sign_bits.data_ptr() if (quant and out.sign_bits is not None) else None,
                 out.means.data_ptr() if (quant and out.means is not None) else None,
                 out.tensor_counts.data_ptr(), out.idx.numel())
    st = _lib().gd_compress_static(off, len(offsets) - 1, grad.data_ptr(),
                                   None if base is None else base.data_ptr(), residual.data_ptr(),
                                   float(drop_ratio), GD_PER_TENSOR if per_tensor else GD_GLOBAL, int(quant),
                                   ctypes.byref(sp), _stream_handle(stream))
    if st != 0:
        raise GDError(st, "gd_compress_static")
    if per_tensor:
        out.k = sum(keep_count(int(offsets[t + 1]) - int(offsets[t]), drop_ratio) for t in range(len(offsets) - 1))
    else:
        out.k = keep_count(n, drop_ratio)
    return out


# ---- operators around the compressor ----

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


def _dtype_code(dtype: torch.dtype) -> int:
    if dtype not in _DTYPES:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
    return _DTYPES[dtype]


def _flat_on(device: int, t: torch.Tensor, name: str, dtype: torch.dtype, n: int) -> int:
    """Address of a contiguous tensor of n elements on the device."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor on cuda:{device}")
    if t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} elements, not {n}")
    return t.data_ptr()


def _rows_on(device: int, t: torch.Tensor, name: str, dtype: torch.dtype, columns: int, rows: Optional[int] = None):
    """(rows, address, row stride) of a tensor [..., columns] on the device whose rows are contiguous and evenly
    spaced."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device:
        raise TypeError(f"{name} must be a {dtype} tensor on cuda:{device}")
    dim = t.dim()
    if dim == 0 or t.size(-1) != columns:
        raise ValueError(f"{name} must have rows of {columns} elements, not shape {tuple(t.shape)}")
    if dim != 2:
        t = t.view(-1, columns)
    n = t.size(0)
    if rows is not None and n != rows:
        raise ValueError(f"{name} has {n} rows, not {rows}")
    down, across = t.stride()
    if across != 1 and columns > 1 and n > 0:
        raise ValueError(f"{name} must be contiguous within its rows")
    return n, t.data_ptr(), down if n > 1 else columns


def _untracked() -> RuntimeError:
    """What a forward raises for tensors that autograd would have to follow: its results would come out cut off from
    them, without a word."""
    return RuntimeError("autograd does not follow the layers' calls: make them under torch.no_grad() or on detached "
                        "tensors, and take gradients by their backward()")


def _meet(a, b, size: int) -> bool:
    """Whether two matrices share memory: (address, rows, row stride, columns) in elements of ``size`` bytes."""
    (pa, na, sa, ca), (pb, nb, sb, cb) = a, b
    if not na or not nb or pa >= pb + ((nb - 1) * sb + cb) * size or pb >= pa + ((na - 1) * sa + ca) * size:
        return False
    if sa == ca:  # one run
        na, ca = 1, na * ca
    if sb == cb:
        nb, cb = 1, nb * cb
    if na == nb == 1 or (na > 1 and nb > 1 and sa != sb):  # rows at two distances: not told apart
        return True
    step = (sa if na > 1 else sb) * size
    at = (pa - pb) % step  # where a's rows lie between those of b
    return at < cb * size or at + ca * size > step


def _apart(size: int, name: str, span, others: dict, same=()) -> None:
    """Raises unless a given output lies apart from the others, matrices of its own type, or is exactly the one of
    those named in ``same``."""
    for other, o in others.items():
        if _meet(span, o, size) and not (other in same and span == o):
            raise ValueError(f"{name} overlaps {other}" + (f"; it may be the same rows as {' or '.join(same)}" if same else ""))


def _new(stream: Optional[torch.cuda.Stream], make, *args, **kwargs) -> torch.Tensor:
    """A tensor that a call on ``stream`` writes: memory of that stream, which no work queued on another one still uses,
    and which is not used again before the work that the current stream has by then is done."""
    if stream is None:
        return make(*args, **kwargs)
    with torch.cuda.stream(stream):
        t = make(*args, **kwargs)
    t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _fresh(stream: Optional[torch.cuda.Stream], like: torch.Tensor, shape, dtype: torch.dtype) -> torch.Tensor:
    """A contiguous tensor on the device of ``like`` that a call on ``stream`` writes."""
    return like.new_empty(shape, dtype=dtype) if stream is None else _new(stream, like.new_empty, shape, dtype=dtype)


def _stream_on(device: int, stream: Optional[torch.cuda.Stream], *tensors) -> Optional[int]:
    """The stream's handle.  Tensors used on a stream that is not the current one are kept from reuse until its work so
    far is done; that the work before them is done is the caller's to see to."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device) or None
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return stream.cuda_stream or None


class _Handle:
    """A library handle on one device, freed with the object.

    Outputs in the layer's type that the caller gives are checked to lie apart from the call's inputs and its other
    outputs in that type, but where a call says that they may be the same rows; gradients of parameters, which are in
    float32 whatever the type, are the caller's to keep apart.  Autograd does not follow the calls: a
    layer's forward refuses tensors that require gradients while autograd records, and its backward gives the gradients.
    """

    _what = ""

    def _create(self, device, *args) -> None:
        lib = _lib()
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        index = self.device.index
        self._tensor, self._matrix, self._stream = (functools.partial(f, index) for f in (_flat_on, _rows_on, _stream_on))
        self._h = None
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            st = getattr(lib, f"gd_{self._what}_create")(ctypes.byref(h), *args)
        if st != 0:
            raise GDError(st, f"gd_{self._what}_create")
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None):
            getattr(_lib(), f"gd_{self._what}_destroy")(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class RMSNorm(_Handle):
    """Root-mean-square norm of rows of ``dim`` elements with the residual's addition (gd_norm_*).

    y = h * weight / sqrt(mean(h^2) + eps), h = x + residual.  Tensors are [..., dim] in ``dtype``; one object
    serves every layer of its shape on a stream.
    """

    _what = "norm"

    def __init__(self, dim: int, dtype: torch.dtype = torch.bfloat16, eps: float = 1e-6, device=None):
        self.dim, self.dtype, self.eps = int(dim), dtype, float(eps)
        if not 0 < self.dim < 1 << 32:
            raise GDError(1, "RMSNorm")
        self._create(device, self.dim, _dtype_code(dtype))

    def forward(self, x, weight, residual=None, out=None, sum_out=None, stream=None):
        """(y, h); h is x itself without a residual.  ``sum_out`` and ``out`` may be x or residual."""
        y, _, h = self._run(x, weight, residual, out, None, False, sum_out, stream)
        return y, h

    def forward_int8(self, x, weight, residual=None, out=None, scale=None, sum_out=None, stream=None):
        """(q, scale, h): rows of y in 8 bits, y = q * scale[row], scale[row] = max|y| / 127."""
        return self._run(x, weight, residual, out, scale, True, sum_out, stream)

    def _run(self, x, weight, residual, out, scale, int8, sum_out, stream):
        io = _NormIO(eps=self.eps)
        rows, io.x, io.x_stride = self._matrix(x, "x", self.dtype, self.dim)
        io.rows = rows
        io.weight = self._tensor(weight, "weight", self.dtype, self.dim)
        y = out
        if y is None:
            y = (_new(stream, x.new_empty, x.shape, dtype=torch.int8) if int8
                 else _new(stream, torch.empty_like, x, memory_format=torch.contiguous_format))
        _, io.y, io.y_stride = self._matrix(y, "out", torch.int8 if int8 else self.dtype, self.dim, rows)
        if int8:
            if scale is None:
                scale = _new(stream, x.new_empty, x.shape[:-1], dtype=torch.float32)
            io.y_scale = self._tensor(scale, "scale", torch.float32, rows)
        h = x
        if residual is not None:
            _, io.residual, io.residual_stride = self._matrix(residual, "residual", self.dtype, self.dim, rows)
            h = _new(stream, torch.empty_like, x, memory_format=torch.contiguous_format) if sum_out is None else sum_out
        elif sum_out is not None:
            h = sum_out
        if h is not x or sum_out is not None:
            _, io.sum, io.sum_stride = self._matrix(h, "sum_out", self.dtype, self.dim, rows)
        if rows and (out is not None or sum_out is not None):
            self._outputs_apart(io, out is not None and not int8, sum_out is not None)
        if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                        (residual is not None and residual.requires_grad)):
            raise _untracked()
        st = _lib().gd_norm_forward(self._h, io, self._stream(stream, x, weight, residual, y, scale, h))
        if st != 0:
            raise GDError(st, "gd_norm_forward")
        return y, scale, h

    def _outputs_apart(self, io, out, sum_out) -> None:
        """A given out or sum_out lies apart from what the call reads, and from the other."""
        rows, dim, size = io.rows, self.dim, self.dtype.itemsize
        others = {"x": (io.x, rows, io.x_stride, dim), "weight": (io.weight, 1, dim, dim)}
        if io.residual:
            others["residual"] = (io.residual, rows, io.residual_stride, dim)
        if sum_out:
            _apart(size, "sum_out", (io.sum, rows, io.sum_stride, dim), others, ("x", "residual"))
        if io.sum:
            others["sum_out"] = (io.sum, rows, io.sum_stride, dim)
        if out:
            _apart(size, "out", (io.y, rows, io.y_stride, dim), others, ("x", "residual"))

    def backward(self, dy, h, weight, dsum=None, dx=None, dweight=None, accumulate=False, stream=None):
        """(dx, dweight): the gradient of x and of residual, and the weight's in float32 (a slice of a flat
        gradient, say).  ``h`` is what forward returned, ``dsum`` a further gradient of h; dx may be dy or dsum."""
        io = _NormGrad(eps=self.eps, accumulate=int(accumulate))
        rows, io.dy, io.dy_stride = self._matrix(dy, "dy", self.dtype, self.dim)
        io.rows = rows
        _, io.x, io.x_stride = self._matrix(h, "h", self.dtype, self.dim, rows)
        io.weight = self._tensor(weight, "weight", self.dtype, self.dim)
        if dsum is not None:
            _, io.dsum, io.dsum_stride = self._matrix(dsum, "dsum", self.dtype, self.dim, rows)
        given = dx is not None
        if not given:
            dx = _new(stream, torch.empty_like, dy, memory_format=torch.contiguous_format)
        _, io.dx, io.dx_stride = self._matrix(dx, "dx", self.dtype, self.dim, rows)
        dweight = _gradient(dweight, accumulate, (self.dim,), self.device, stream)
        io.dweight = self._tensor(dweight, "dweight", torch.float32, self.dim)
        if rows and given:
            dim = self.dim
            others = {"dy": (io.dy, rows, io.dy_stride, dim), "h": (io.x, rows, io.x_stride, dim),
                      "weight": (io.weight, 1, dim, dim)}
            if dsum is not None:
                others["dsum"] = (io.dsum, rows, io.dsum_stride, dim)
            _apart(self.dtype.itemsize, "dx", (io.dx, rows, io.dx_stride, dim), others, ("dy", "dsum"))
        st = _lib().gd_norm_backward(self._h, io, self._stream(stream, dy, h, weight, dsum, dx, dweight))
        if st != 0:
            raise GDError(st, "gd_norm_backward")
        return dx, dweight


def _gradient(given, accumulate, shape, device, stream):
    if given is not None:
        return given
    if accumulate:
        raise ValueError("accumulate needs the gradient to add to")
    return _new(stream, torch.empty, shape, dtype=torch.float32, device=device)


class LayerNorm(_Handle):
    """Layer norm of rows of ``dim`` elements with the residual's addition (gd_layernorm_*).

    y = (h - mean(h)) / sqrt(var(h) + eps) * weight + bias, h = x + residual.  Tensors are [..., dim] in ``dtype``; one
    object serves every layer of its shape on a stream.
    """

    _what = "layernorm"

    def __init__(self, dim: int, dtype: torch.dtype = torch.bfloat16, eps: float = 1e-5, device=None):
        self.dim, self.dtype, self.eps = int(dim), dtype, float(eps)
        if not 0 < self.dim < 1 << 32:
            raise GDError(1, "LayerNorm")
        self._create(device, self.dim, _dtype_code(dtype))

    def forward(self, x, weight, bias=None, residual=None, out=None, sum_out=None, stream=None):
        """(y, h); h is x itself without a residual.  ``sum_out`` and ``out`` may be x or residual."""
        y, _, h = self._run(x, weight, bias, residual, out, None, False, sum_out, stream)
        return y, h

    def forward_int8(self, x, weight, bias=None, residual=None, out=None, scale=None, sum_out=None, stream=None):
        """(q, scale, h): rows of y in 8 bits, y = q * scale[row], scale[row] = max|y| / 127."""
        return self._run(x, weight, bias, residual, out, scale, True, sum_out, stream)

    def _run(self, x, weight, bias, residual, out, scale, int8, sum_out, stream):
        io, dim = _LayerNormIO(eps=self.eps), self.dim
        rows, io.x, io.x_stride = self._matrix(x, "x", self.dtype, dim)
        io.rows = rows
        io.weight = self._tensor(weight, "weight", self.dtype, dim)
        if bias is not None:
            io.bias = self._tensor(bias, "bias", self.dtype, dim)
        if out is None:  # what is made here needs no check
            y = _fresh(stream, x, x.shape, torch.int8 if int8 else self.dtype)
            io.y, io.y_stride = y.data_ptr(), dim
        else:
            y = out
            _, io.y, io.y_stride = self._matrix(y, "out", torch.int8 if int8 else self.dtype, dim, rows)
        if int8:
            if scale is None:
                scale = _fresh(stream, x, x.shape[:-1], torch.float32)
                io.y_scale = scale.data_ptr()
            else:
                io.y_scale = self._tensor(scale, "scale", torch.float32, rows)
        h = x
        if residual is not None:
            _, io.residual, io.residual_stride = self._matrix(residual, "residual", self.dtype, dim, rows)
            if sum_out is None:
                h = _fresh(stream, x, x.shape, self.dtype)
                io.sum, io.sum_stride = h.data_ptr(), dim
        if sum_out is not None:
            h = sum_out
            _, io.sum, io.sum_stride = self._matrix(h, "sum_out", self.dtype, dim, rows)
        if rows and (out is not None or sum_out is not None):
            self._outputs_apart(io, out is not None and not int8, sum_out is not None)
        if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                        (bias is not None and bias.requires_grad) or
                                        (residual is not None and residual.requires_grad)):
            raise _untracked()
        st = _lib().gd_layernorm_forward(self._h, io, self._stream(stream, x, weight, bias, residual, y, scale, h))
        if st != 0:
            raise GDError(st, "gd_layernorm_forward")
        return y, scale, h

    def _outputs_apart(self, io, out, sum_out) -> None:
        """A given out or sum_out lies apart from what the call reads, and from the other."""
        rows, dim, size = io.rows, self.dim, self.dtype.itemsize
        others = {"x": (io.x, rows, io.x_stride, dim), "weight": (io.weight, 1, dim, dim)}
        if io.bias:
            others["bias"] = (io.bias, 1, dim, dim)
        if io.residual:
            others["residual"] = (io.residual, rows, io.residual_stride, dim)
        if sum_out:
            _apart(size, "sum_out", (io.sum, rows, io.sum_stride, dim), others, ("x", "residual"))
        if io.sum:
            others["sum_out"] = (io.sum, rows, io.sum_stride, dim)
        if out:
            _apart(size, "out", (io.y, rows, io.y_stride, dim), others, ("x", "residual"))

    def backward(self, dy, h, weight, dsum=None, dx=None, dweight=None, dbias=None, accumulate=False, stream=None):
        """(dx, dweight, dbias): the gradient of x and of residual, and the weight's and the bias's in float32 (slices
        of a flat gradient, say).  ``h`` is what forward returned, ``dsum`` a further gradient of h; dx may be dy or
        dsum.  dbias False: a layer without a bias."""
        io = _LayerNormGrad(eps=self.eps, accumulate=int(accumulate))
        rows, io.dy, io.dy_stride = self._matrix(dy, "dy", self.dtype, self.dim)
        io.rows = rows
        _, io.x, io.x_stride = self._matrix(h, "h", self.dtype, self.dim, rows)
        io.weight = self._tensor(weight, "weight", self.dtype, self.dim)
        if dsum is not None:
            _, io.dsum, io.dsum_stride = self._matrix(dsum, "dsum", self.dtype, self.dim, rows)
        given = dx is not None
        if given:
            _, io.dx, io.dx_stride = self._matrix(dx, "dx", self.dtype, self.dim, rows)
        else:
            dx = _fresh(stream, dy, dy.shape, self.dtype)
            io.dx, io.dx_stride = dx.data_ptr(), self.dim
        dweight = _gradient(dweight, accumulate, (self.dim,), self.device, stream)
        io.dweight = self._tensor(dweight, "dweight", torch.float32, self.dim)
        if dbias is not False:
            dbias = _gradient(dbias, accumulate, (self.dim,), self.device, stream)
            io.dbias = self._tensor(dbias, "dbias", torch.float32, self.dim)
        else:
            dbias = None
        if rows and given:
            dim = self.dim
            others = {"dy": (io.dy, rows, io.dy_stride, dim), "h": (io.x, rows, io.x_stride, dim),
                      "weight": (io.weight, 1, dim, dim)}
            if dsum is not None:
                others["dsum"] = (io.dsum, rows, io.dsum_stride, dim)
            _apart(self.dtype.itemsize, "dx", (io.dx, rows, io.dx_stride, dim), others, ("dy", "dsum"))
        st = _lib().gd_layernorm_backward(self._h, io, self._stream(stream, dy, h, weight, dsum, dx, dweight, dbias))
        if st != 0:
            raise GDError(st, "gd_layernorm_backward")
        return dx, dweight, dbias


_INDEX = {torch.int32: 0, torch.int64: 1}


def _ids_on(device: int, t: torch.Tensor, name: str, n: Optional[int] = None):
    """(address, type code) of a contiguous tensor of token ids on the device."""
    if not isinstance(t, torch.Tensor) or t.dtype not in _INDEX or t.get_device() != device or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous int32 or int64 tensor on cuda:{device}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} elements, not {n}")
    return t.data_ptr(), _INDEX[t.dtype]


class Embedding(_Handle):
    """Rows of a weight [vocab, dim] in ``dtype`` by token, times ``scale``, and the weight's gradient (gd_embed_*).

    Tokens are int32 or int64 of any shape; one outside [0, vocab) is padding, whose rows are zeros and pass no
    gradient.  ``max_rows``: the most tokens of a backward call.  The object holds no weights.
    """

    _what = "embed"

    def __init__(self, vocab: int, dim: int, dtype: torch.dtype = torch.bfloat16, scale: float = 1.0,
                 max_rows: int = 8192, device=None):
        self.vocab, self.dim, self.dtype, self.scale = int(vocab), int(dim), dtype, float(scale)
        if not (0 < self.vocab < 1 << 32 and 0 < self.dim < 1 << 32 and 0 <= int(max_rows) < 1 << 64):
            raise GDError(1, "Embedding")
        self._create(device, self.vocab, self.dim, _dtype_code(dtype), int(max_rows))

    def forward(self, tokens, weight, out=None, stream=None):
        """y [*tokens.shape, dim]."""
        io = _EmbedIO(scale=self.scale)
        io.tokens, io.index = _ids_on(self.device.index, tokens, "tokens")
        rows = io.rows = tokens.numel()
        _, io.weight, io.weight_stride = self._matrix(weight, "weight", self.dtype, self.dim, self.vocab)
        if out is None:
            out = _fresh(stream, weight, (*tokens.shape, self.dim), self.dtype)
            io.y, io.y_stride = out.data_ptr(), self.dim
        else:
            _, io.y, io.y_stride = self._matrix(out, "out", self.dtype, self.dim, rows)
            if rows:
                _apart(self.dtype.itemsize, "out", (io.y, rows, io.y_stride, self.dim),
                       {"weight": (io.weight, self.vocab, io.weight_stride, self.dim)})
        if weight.requires_grad and torch.is_grad_enabled():
            raise _untracked()
        st = _lib().gd_embed_forward(self._h, io, self._stream(stream, tokens, weight, out))
        if st != 0:
            raise GDError(st, "gd_embed_forward")
        return out

    def backward(self, dy, tokens, dweight=None, accumulate=False, stream=None):
        """dweight [vocab, dim] in float32 (a slice of a flat gradient, say), rows of tokens that do not occur zeros;
        with ``accumulate`` it is added to, and those rows stay."""
        io = _EmbedGrad(scale=self.scale, accumulate=int(accumulate))
        io.tokens, io.index = _ids_on(self.device.index, tokens, "tokens")
        rows = io.rows = tokens.numel()
        _, io.dy, io.dy_stride = self._matrix(dy, "dy", self.dtype, self.dim, rows)
        dweight = _gradient(dweight, accumulate, (self.vocab, self.dim), self.device, stream)
        _, io.dweight, io.dweight_stride = self._matrix(dweight, "dweight", torch.float32, self.dim, self.vocab)
        st = _lib().gd_embed_backward(self._h, io, self._stream(stream, dy, tokens, dweight))
        if st != 0:
            raise GDError(st, "gd_embed_backward")
        return dweight


class Linear(_Handle):
    """A layer y = act(x weight^T + bias) + residual (gd_linear_*), weight [out, in] in ``dtype``.

    act: "none", "relu", "gelu" (by erf) or "silu".  The object holds the plan and scratch of calls of at most
    ``max_rows`` rows, no weights; one object serves every layer of its shape on a stream.
    """

    _what = "linear"

    def __init__(self, in_features: int, out_features: int, dtype: torch.dtype = torch.bfloat16, act: str = "none",
                 max_rows: int = 8192, device=None):
        if act not in ACTIVATIONS:
            raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, not {act!r}")
        self.inf, self.outf, self.dtype, self.act = int(in_features), int(out_features), dtype, act
        if not (0 < self.inf < 1 << 32 and 0 < self.outf < 1 << 32 and 0 <= int(max_rows) < 1 << 64):
            raise GDError(1, "Linear")
        self._create(device, self.inf, self.outf, _dtype_code(dtype), ACTIVATIONS[act], int(max_rows))

    def forward(self, x, weight, bias=None, residual=None, out=None, keep_pre=False, stream=None):
        """y, or (y, pre) with ``keep_pre`` (True, or a tensor to write): x weight^T + bias for the backward.
        ``out`` may be residual."""
        return self._run(x, weight, None, None, bias, residual, out, keep_pre, stream)

    def forward_int8(self, q, scale, weight_q, weight_scale, bias=None, residual=None, out=None, stream=None):
        """y in ``dtype`` from 8-bit operands: rows of x are q * scale[row], rows of weight weight_q *
        weight_scale[row], codes in -127..127 (see quantise_rows and RMSNorm.forward_int8)."""
        return self._run(q, weight_q, scale, weight_scale, bias, residual, out, False, stream)

    def _run(self, x, weight, xs, ws, bias, residual, out, keep_pre, stream):
        kind = self.dtype if xs is None else torch.int8
        io = _LinearIO()
        rows, io.x, io.x_stride = self._matrix(x, "x", kind, self.inf)
        io.rows = rows
        _, io.weight, io.weight_stride = self._matrix(weight, "weight", kind, self.inf, self.outf)
        if xs is not None:
            io.x_scale = self._tensor(xs, "scale", torch.float32, rows)
            io.weight_scale = self._tensor(ws, "weight_scale", torch.float32, self.outf)
        if bias is not None:
            io.bias = self._tensor(bias, "bias", self.dtype, self.outf)
        if residual is not None:
            _, io.residual, io.residual_stride = self._matrix(residual, "residual", self.dtype, self.outf, rows)
        shape = (rows, self.outf) if x.dim() == 2 else (*x.shape[:-1], self.outf)
        given = out is not None
        if not given:
            out = _new(stream, x.new_empty, shape, dtype=self.dtype)
        _, io.y, io.y_stride = self._matrix(out, "out", self.dtype, self.outf, rows)
        pre = None
        if keep_pre is not False:
            pre = _new(stream, x.new_empty, shape, dtype=self.dtype) if keep_pre is True else keep_pre
            _, io.pre, io.pre_stride = self._matrix(pre, "pre", self.dtype, self.outf, rows)
        if rows and (given or (pre is not None and keep_pre is not True)):
            k, n, size, others = self.inf, self.outf, self.dtype.itemsize, {}
            if xs is None:
                others = {"x": (io.x, rows, io.x_stride, k), "weight": (io.weight, n, io.weight_stride, k)}
            if bias is not None:
                others["bias"] = (io.bias, 1, n, n)
            if residual is not None:
                others["residual"] = (io.residual, rows, io.residual_stride, n)
            span = (io.y, rows, io.y_stride, n)
            if given:
                _apart(size, "out", span, others, ("residual",))
            if pre is not None:
                _apart(size, "pre", (io.pre, rows, io.pre_stride, n), {**others, "out": span})
        if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                        (bias is not None and bias.requires_grad) or
                                        (residual is not None and residual.requires_grad)):
            raise _untracked()
        st = _lib().gd_linear_forward(self._h, io, self._stream(stream, x, weight, xs, ws, bias, residual, out, pre))
        if st != 0:
            raise GDError(st, "gd_linear_forward")
        return out if pre is None else (out, pre)

    def backward(self, dy, x, weight, pre=None, dx=None, dweight=None, dbias=None, dz=None, need_dx=True,
                 need_dweight=True, accumulate=False, stream=None):
        """(dx, dweight, dbias, dz); dweight and dbias in float32 (slices of a flat gradient, say).

        dbias: a tensor to write, True for a new one, or None for a layer without a bias.
        dz = dy act'(pre) in ``dtype`` is the gradient that the products take (dy itself without an
        activation).  None for what is not needed; the gradient of the residual is dy.  dz may be dy or pre.
        """
        given_dz, given_dx = dz is not None, dx is not None
        io = _LinearGrad(accumulate=int(accumulate))
        rows, io.dy, io.dy_stride = self._matrix(dy, "dy", self.dtype, self.outf)
        io.rows = rows
        if self.act != "none":
            if pre is None:
                raise ValueError(f"the backward of {self.act} needs pre")
            _, io.pre, io.pre_stride = self._matrix(pre, "pre", self.dtype, self.outf, rows)
            if dz is None:
                dz = _new(stream, torch.empty_like, dy, memory_format=torch.contiguous_format)
            _, io.dz, io.dz_stride = self._matrix(dz, "dz", self.dtype, self.outf, rows)
        else:
            pre, dz = None, dy
        if need_dx:
            _, io.weight, io.weight_stride = self._matrix(weight, "weight", self.dtype, self.inf, self.outf)
            if dx is None:
                dx = _new(stream, dy.new_empty, (*dy.shape[:-1], self.inf))
            _, io.dx, io.dx_stride = self._matrix(dx, "dx", self.dtype, self.inf, rows)
        else:
            dx = None
        if need_dweight:
            _, io.x, io.x_stride = self._matrix(x, "x", self.dtype, self.inf, rows)
            dweight = _gradient(dweight, accumulate, (self.outf, self.inf), self.device, stream)
            _, io.dweight, io.dweight_stride = self._matrix(dweight, "dweight", torch.float32, self.inf, self.outf)
        else:
            dweight = None
        if dbias is not None:
            dbias = _gradient(None if dbias is True else dbias, accumulate, (self.outf,), self.device, stream)
            io.dbias = self._tensor(dbias, "dbias", torch.float32, self.outf)
        if rows and (given_dz or given_dx):
            self._outputs_apart(io, given_dz, given_dx)
        st = _lib().gd_linear_backward(self._h, io, self._stream(stream, dy, x, weight, pre, dz, dx, dweight, dbias))
        if st != 0:
            raise GDError(st, "gd_linear_backward")
        return dx, dweight, dbias, dz

    def _outputs_apart(self, io, dz, dx) -> None:
        """A given dz or dx lies apart from what the call reads, and from the other."""
        rows, k, n, size = io.rows, self.inf, self.outf, self.dtype.itemsize
        others = {"dy": (io.dy, rows, io.dy_stride, n), "x": (io.x, rows, io.x_stride, k),
                  "weight": (io.weight, n, io.weight_stride, k), "pre": (io.pre, rows, io.pre_stride, n),
                  "dz": (io.dz, rows, io.dz_stride, n)}
        others = {name: span for name, span in others.items() if span[0]}  # what the call was given
        if dz and io.dz:
            span = others.pop("dz")
            _apart(size, "dz", span, others, ("dy", "pre"))
            others["dz"] = span
        if dx and io.dx:
            _apart(size, "dx", (io.dx, rows, io.dx_stride, k), others)


class GatedLinear(_Handle):
    """A gated layer y = act(x Wg^T + bg) * (x Wu^T + bu) (gd_gated_*), weight [2 out, in] in ``dtype``: Wg's rows, then
    Wu's; bias [2 out] likewise.

    act: "none", "relu", "gelu" (by erf) or "silu".  The object holds the plan and scratch of calls of at most
    ``max_rows`` rows, no weights; one object serves every layer of its shape on a stream.
    """

    _what = "gated"

    def __init__(self, in_features: int, out_features: int, dtype: torch.dtype = torch.bfloat16, act: str = "silu",
                 max_rows: int = 8192, device=None):
        if act not in ACTIVATIONS:
            raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, not {act!r}")
        self.inf, self.outf, self.dtype, self.act = int(in_features), int(out_features), dtype, act
        if not (0 < self.inf < 1 << 32 and 0 < self.outf < 1 << 32 and 0 <= int(max_rows) < 1 << 64):
            raise GDError(1, "GatedLinear")
        self._create(device, self.inf, self.outf, _dtype_code(dtype), ACTIVATIONS[act], int(max_rows))

    def forward(self, x, weight, bias=None, out=None, keep_pre=False, stream=None):
        """y, or (y, pre) with ``keep_pre`` (True, or a tensor [..., 2 out] to write): both sums for the backward."""
        return self._run(x, weight, None, None, bias, out, keep_pre, stream)

    def forward_int8(self, q, scale, weight_q, weight_scale, bias=None, out=None, stream=None):
        """y in ``dtype`` from 8-bit operands: rows of x are q * scale[row], rows of weight weight_q *
        weight_scale[row], codes in -127..127 (see quantise_rows and the norms' forward_int8)."""
        return self._run(q, weight_q, scale, weight_scale, bias, out, False, stream)

    def _run(self, x, weight, xs, ws, bias, out, keep_pre, stream):
        kind, both = self.dtype if xs is None else torch.int8, 2 * self.outf
        io = _GatedIO()
        rows, io.x, io.x_stride = self._matrix(x, "x", kind, self.inf)
        io.rows = rows
        _, io.weight, io.weight_stride = self._matrix(weight, "weight", kind, self.inf, both)
        if xs is not None:
            io.x_scale = self._tensor(xs, "scale", torch.float32, rows)
            io.weight_scale = self._tensor(ws, "weight_scale", torch.float32, both)
        if bias is not None:
            io.bias = self._tensor(bias, "bias", self.dtype, both)
        given = out is not None
        if given:
            _, io.y, io.y_stride = self._matrix(out, "out", self.dtype, self.outf, rows)
        else:
            out = _fresh(stream, x, (*x.shape[:-1], self.outf), self.dtype)
            io.y, io.y_stride = out.data_ptr(), self.outf
        pre = None
        if keep_pre is True:
            pre = _fresh(stream, x, (*x.shape[:-1], both), self.dtype)
            io.pre, io.pre_stride = pre.data_ptr(), both
        elif keep_pre is not False:
            pre = keep_pre
            _, io.pre, io.pre_stride = self._matrix(pre, "pre", self.dtype, both, rows)
        if rows and (given or (pre is not None and keep_pre is not True)):
            k, n, size, others = self.inf, self.outf, self.dtype.itemsize, {}
            if xs is None:
                others = {"x": (io.x, rows, io.x_stride, k), "weight": (io.weight, both, io.weight_stride, k)}
            if bias is not None:
                others["bias"] = (io.bias, 1, both, both)
            span = (io.y, rows, io.y_stride, n)
            if given:
                _apart(size, "out", span, others)
            if pre is not None:
                _apart(size, "pre", (io.pre, rows, io.pre_stride, both), {**others, "out": span})
        if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                        (bias is not None and bias.requires_grad)):
            raise _untracked()
        st = _lib().gd_gated_forward(self._h, io, self._stream(stream, x, weight, xs, ws, bias, out, pre))
        if st != 0:
            raise GDError(st, "gd_gated_forward")
        return out if pre is None else (out, pre)

    def backward(self, dy, x, weight, pre, dx=None, dweight=None, dbias=None, dz=None, need_dx=True, need_dweight=True,
                 accumulate=False, stream=None):
        """(dx, dweight, dbias, dz); dweight and dbias in float32 (slices of a flat gradient, say).

        dbias: a tensor to write, True for a new one, or None for a layer without a bias.
        dz [..., 2 out] in ``dtype`` is the gradient of both sums that the products take; it may be pre.  None for what
        is not needed.
        """
        given_dz, given_dx, both = dz is not None, dx is not None, 2 * self.outf
        io = _GatedGrad(accumulate=int(accumulate))
        rows, io.dy, io.dy_stride = self._matrix(dy, "dy", self.dtype, self.outf)
        io.rows = rows
        _, io.pre, io.pre_stride = self._matrix(pre, "pre", self.dtype, both, rows)
        if given_dz:
            _, io.dz, io.dz_stride = self._matrix(dz, "dz", self.dtype, both, rows)
        else:
            dz = _fresh(stream, pre, pre.shape, self.dtype)
            io.dz, io.dz_stride = dz.data_ptr(), both
        if need_dx:
            _, io.weight, io.weight_stride = self._matrix(weight, "weight", self.dtype, self.inf, both)
            if given_dx:
                _, io.dx, io.dx_stride = self._matrix(dx, "dx", self.dtype, self.inf, rows)
            else:
                dx = _fresh(stream, dy, (*dy.shape[:-1], self.inf), self.dtype)
                io.dx, io.dx_stride = dx.data_ptr(), self.inf
        else:
            dx = None
        if need_dweight:
            _, io.x, io.x_stride = self._matrix(x, "x", self.dtype, self.inf, rows)
            dweight = _gradient(dweight, accumulate, (both, self.inf), self.device, stream)
            _, io.dweight, io.dweight_stride = self._matrix(dweight, "dweight", torch.float32, self.inf, both)
        else:
            dweight = None
        if dbias is not None:
            dbias = _gradient(None if dbias is True else dbias, accumulate, (both,), self.device, stream)
            io.dbias = self._tensor(dbias, "dbias", torch.float32, both)
        if rows and (given_dz or given_dx):
            k, n, size = self.inf, self.outf, self.dtype.itemsize
            others = {"dy": (io.dy, rows, io.dy_stride, n), "x": (io.x, rows, io.x_stride, k),
                      "weight": (io.weight, both, io.weight_stride, k), "pre": (io.pre, rows, io.pre_stride, both)}
            others = {name: span for name, span in others.items() if span[0]}  # what the call was given
            span = (io.dz, rows, io.dz_stride, both)
            if given_dz:
                _apart(size, "dz", span, others, ("pre",))
            if given_dx and dx is not None:
                _apart(size, "dx", (io.dx, rows, io.dx_stride, k), {**others, "dz": span})
        st = _lib().gd_gated_backward(self._h, io, self._stream(stream, dy, x, weight, pre, dz, dx, dweight, dbias))
        if st != 0:
            raise GDError(st, "gd_gated_backward")
        return dx, dweight, dbias, dz


@dataclass
class LogProbs:
    """What TokenLogProbs.forward says of each row, in float32."""

    logp: torch.Tensor  # of the given token
    entropy: Optional[torch.Tensor] = None
    stats: Optional[torch.Tensor] = None  # [..., 2] for backward, their sum the log of the sum of exp (see gd.h)
    top_logp: Optional[torch.Tensor] = None  # [..., top], falling
    top_ids: Optional[torch.Tensor] = None  # [..., top] int64


class _Scores(_Handle):
    """Rows of ``vocab`` logits in ``dtype``, multiplied by ``scale`` (one over a temperature) before all else, for
    calls of at most ``max_rows`` rows."""

    def __init__(self, vocab: int, dtype: torch.dtype = torch.bfloat16, scale: float = 1.0, max_rows: int = 8192,
                 device=None):
        self.vocab, self.dtype, self.scale = int(vocab), dtype, float(scale)
        if not (0 < self.vocab < 1 << 32 and 0 <= int(max_rows) < 1 << 64):
            raise GDError(1, type(self).__name__)
        self._create(device, self.vocab, _dtype_code(dtype), int(max_rows))

    def _logits(self, io, logits) -> int:
        rows, io.logits, io.stride = self._matrix(logits, "logits", self.dtype, self.vocab)
        io.rows, io.scale = rows, self.scale
        return rows

    def _dlogits(self, io, logits, out, stream, apart):
        """The gradient's buffer: new, or a given one that is the logits themselves or lies apart from what is read."""
        if out is None:
            out = _fresh(stream, logits, logits.shape, self.dtype)
            io.dlogits, io.dlogits_stride = out.data_ptr(), self.vocab
            return out
        _, io.dlogits, io.dlogits_stride = self._matrix(out, "out", self.dtype, self.vocab, io.rows)
        if io.rows:
            _apart(self.dtype.itemsize, "out", (io.dlogits, io.rows, io.dlogits_stride, self.vocab),
                   {"logits": (io.logits, io.rows, io.stride, self.vocab), **apart}, ("logits",))
        return out


class TokenLogProbs(_Scores):
    """Log probabilities of given tokens under rows of logits, the rows' entropy and top alternatives, and the gradient
    (gd_logprob_*).

    Logits are [..., vocab], tokens int32 or int64 of the shape before; a token outside [0, vocab) is padding, whose log
    probability is 0 and passes no gradient.  A logit of minus infinity is masked.
    """

    _what = "logprob"

    def forward(self, logits, tokens, top: int = 0, entropy: bool = True, keep_stats: bool = False,
                out: Optional[LogProbs] = None, stream=None):
        """LogProbs; ``top`` up to 64 alternatives, of equal logits the lower id first; ``keep_stats`` for backward.
        ``out``: one of an earlier call of the same shape and wishes, to write again; what it holds beyond these wishes would
        stay that call's, and is refused."""
        if not 0 <= top < 1 << 32:
            raise GDError(1, "gd_logprob_forward")
        io = _LogProbIO()
        rows = self._logits(io, logits)
        io.tokens, io.index = _ids_on(self.device.index, tokens, "tokens", rows)
        io.top, shape = top, tokens.shape
        if out is None:
            f32 = torch.float32
            out = LogProbs(_fresh(stream, logits, shape, f32), _fresh(stream, logits, shape, f32) if entropy else None,
                           _fresh(stream, logits, (*shape, 2), f32) if keep_stats else None)
            if top:
                out.top_logp = _fresh(stream, logits, (*shape, top), f32)
                out.top_ids = _fresh(stream, logits, (*shape, top), torch.int64)
        else:
            spans = []
            for name, n, size in (("logp", rows, 4), ("entropy", rows * entropy, 4), ("stats", 2 * rows * keep_stats, 4),
                                  ("top_logp", rows * top, 4), ("top_ids", rows * top, 8)):
                t, name = getattr(out, name), "out." + name
                if n:
                    at = self._tensor(t, name, torch.float32 if size == 4 else torch.int64, n)
                    spans.append((at, at + n * size, name))
                elif rows and t is not None:
                    raise ValueError(f"{name} is of another call, and not asked for in this one")
            if rows:
                self._outputs_apart(io, tokens, spans)
        io.logp = out.logp.data_ptr()
        if entropy:
            io.entropy = out.entropy.data_ptr()
        if keep_stats:
            io.stats = out.stats.data_ptr()
        if top:
            io.top_logp, io.top_id = out.top_logp.data_ptr(), out.top_ids.data_ptr()
        if logits.requires_grad and torch.is_grad_enabled():
            raise _untracked()
        st = _lib().gd_logprob_forward(self._h, io, self._stream(stream, logits, tokens, out.logp, out.entropy, out.stats,
                                                                 out.top_logp, out.top_ids))
        if st != 0:
            raise GDError(st, "gd_logprob_forward")
        return out

    def _outputs_apart(self, io, tokens, spans) -> None:
        """Given outputs (first byte, past the last, name) lie apart from what the call reads, and from one another, of
        whatever types they are."""
        size, token_bytes = self.dtype.itemsize, tokens.nbytes
        past = 0
        for at, to, _ in sorted([*spans, (io.tokens, io.tokens + token_bytes, ""),
                                 (io.logits, io.logits + ((io.rows - 1) * io.stride + self.vocab) * size, "")]):
            if at < past:
                break
            past = to
        else:
            return
        others = {"logits": (io.logits, io.rows, io.stride * size, self.vocab * size),
                  "tokens": (io.tokens, 1, token_bytes, token_bytes)}
        for at, to, name in spans:  # an output may lie between the logits' rows
            span = (at, 1, to - at, to - at)
            _apart(1, name, span, others)
            others[name] = span

    def backward(self, logits, tokens, dlogp, dentropy=None, scores: Optional[LogProbs] = None, out=None, stream=None):
        """dlogits, from the gradients of the log probabilities and (or None) of the entropies, float32.  ``scores``:
        what forward returned for these logits, with its stats, to spare a pass over them; ``out`` may be the logits."""
        return self._back(logits, tokens, dlogp, dentropy, scores, out, stream, False)[1]

    def forward_backward(self, logits, tokens, dlogp, dentropy=None, out=None, stream=None):
        """(LogProbs, dlogits) in one call, where the gradients of the log probabilities are known before they are (a
        mean's are): without stats and alternatives, and with the entropy where ``dentropy`` is given."""
        return self._back(logits, tokens, dlogp, dentropy, None, out, stream, True)

    def _back(self, logits, tokens, dlogp, dentropy, scores, out, stream, forward):
        io = _LogProbGrad()
        rows = self._logits(io, logits)
        io.tokens, io.index = _ids_on(self.device.index, tokens, "tokens", rows)
        io.dlogp = self._tensor(dlogp, "dlogp", torch.float32, rows)
        result = None
        if dentropy is not None:
            io.dentropy = self._tensor(dentropy, "dentropy", torch.float32, rows)
        if scores is not None:
            io.stats = self._tensor(scores.stats, "scores.stats", torch.float32, 2 * rows)
            if dentropy is not None:
                io.entropy = self._tensor(scores.entropy, "scores.entropy", torch.float32, rows)
        if forward:
            result = LogProbs(_fresh(stream, logits, tokens.shape, torch.float32),
                              None if dentropy is None else _fresh(stream, logits, tokens.shape, torch.float32))
            io.logp_out = result.logp.data_ptr()
            if dentropy is not None:
                io.entropy_out = result.entropy.data_ptr()
        apart = {}
        if self.dtype == torch.float32 and out is not None and rows:
            apart = {name: (t.data_ptr(), 1, rows, rows) for name, t in (("dlogp", dlogp), ("dentropy", dentropy)) if t is not None}
            if scores is not None:
                apart["scores.stats"] = (io.stats, 1, 2 * rows, 2 * rows)
                if io.entropy:
                    apart["scores.entropy"] = (io.entropy, 1, rows, rows)
        out = self._dlogits(io, logits, out, stream, apart)
        if forward and logits.requires_grad and torch.is_grad_enabled():
            raise _untracked()
        st = _lib().gd_logprob_backward(self._h, io, self._stream(
            stream, logits, tokens, dlogp, dentropy, out, *(() if scores is None else (scores.stats, scores.entropy)),
            *((result.logp, result.entropy) if forward else ())))
        if st != 0:
            raise GDError(st, "gd_logprob_backward")
        return result, out


class Distill(_Scores):
    """The distance of rows of logits to a teacher's top logits, and its gradient (gd_distill_*).

    For every row the teacher names up to 256 ids, int32 or int64 [..., top], and its logits there [..., top] in float32,
    bfloat16 or float16; both softmaxes are taken of logits times ``scale``.  loss = sum w (log w - log q) over what is
    named.  An id outside [0, vocab) or a teacher's logit of minus infinity names nothing.
    """

    _what = "distill"

    def forward(self, logits, ids, teacher, keep_stats: bool = False, stream=None):
        """(loss, stats): float32 [...], and with ``keep_stats`` (else None) what backward takes to spare a pass over the
        logits."""
        io = _DistillIO()
        rows = self._logits(io, logits)
        self._named(io, ids, teacher, rows)
        loss, stats = _fresh(stream, logits, logits.shape[:-1], torch.float32), None
        io.loss = loss.data_ptr()
        if keep_stats:
            stats = _fresh(stream, logits, (*logits.shape[:-1], 2), torch.float32)
            io.stats = stats.data_ptr()
        if torch.is_grad_enabled() and (logits.requires_grad or teacher.requires_grad):
            raise _untracked()
        st = _lib().gd_distill_forward(self._h, io, self._stream(stream, logits, ids, teacher, loss, stats))
        if st != 0:
            raise GDError(st, "gd_distill_forward")
        return loss, stats

    def backward(self, logits, ids, teacher, dloss, stats=None, out=None, stream=None):
        """dlogits; ``stats``: what forward returned for these logits; ``out`` may be the logits."""
        return self._back(logits, ids, teacher, dloss, stats, out, stream, False)[1]

    def forward_backward(self, logits, ids, teacher, dloss, out=None, stream=None):
        """(loss, dlogits) in one call, where the gradients of the losses are known before they are (a mean's are)."""
        return self._back(logits, ids, teacher, dloss, None, out, stream, True)

    def _named(self, io, ids, teacher, rows) -> None:
        if not isinstance(ids, torch.Tensor) or ids.dtype not in _INDEX:
            raise TypeError("ids must be int32 or int64")
        if ids.dim() == 0 or ids.size(-1) == 0:
            raise ValueError("ids must have rows of at least one element")
        io.top, io.index = ids.size(-1), _INDEX[ids.dtype]
        _, io.ids, io.ids_stride = self._matrix(ids, "ids", ids.dtype, io.top, rows)
        io.teacher_type = _dtype_code(teacher.dtype)
        _, io.teacher, io.teacher_stride = self._matrix(teacher, "teacher", teacher.dtype, io.top, rows)

    def _back(self, logits, ids, teacher, dloss, stats, out, stream, forward):
        io = _DistillGrad()
        rows = self._logits(io, logits)
        self._named(io, ids, teacher, rows)
        io.dloss = self._tensor(dloss, "dloss", torch.float32, rows)
        if stats is not None:
            io.stats = self._tensor(stats, "stats", torch.float32, 2 * rows)
        loss = None
        if forward:
            loss = _fresh(stream, logits, logits.shape[:-1], torch.float32)
            io.loss_out = loss.data_ptr()
        apart = {}
        if out is not None and rows:
            if teacher.dtype == self.dtype:
                apart["teacher"] = (io.teacher, rows, io.teacher_stride, io.top)
            if self.dtype == torch.float32:
                apart["dloss"] = (io.dloss, 1, rows, rows)
                if stats is not None:
                    apart["stats"] = (io.stats, 1, 2 * rows, 2 * rows)
        out = self._dlogits(io, logits, out, stream, apart)
        if forward and torch.is_grad_enabled() and (logits.requires_grad or teacher.requires_grad):
            raise _untracked()
        st = _lib().gd_distill_backward(self._h, io, self._stream(stream, logits, ids, teacher, dloss, stats, out, loss))
        if st != 0:
            raise GDError(st, "gd_distill_backward")
        return loss, out


def quantise_rows(x: torch.Tensor, out=None, scale=None, stream: Optional[torch.cuda.Stream] = None):
    """(q, scale): rows of x in 8 bits, x = q * scale[row], scale[row] = max|x| / 127 (gd_quantise_rows).  Codes carry
    no gradient, so x may be one that requires it (a model's weight)."""
    code, index = _dtype_code(x.dtype), x.get_device()
    if index < 0 or x.dim() == 0 or x.size(-1) == 0:
        raise ValueError("x must be a GPU tensor of rows of at least one element")
    columns = x.size(-1)
    q = _new(stream, x.new_empty, x.shape, dtype=torch.int8) if out is None else out
    scale = _new(stream, x.new_empty, x.shape[:-1], dtype=torch.float32) if scale is None else scale
    rows, xp, xs = _rows_on(index, x, "x", x.dtype, columns)
    _, qp, qs = _rows_on(index, q, "out", torch.int8, columns, rows)
    sp = _flat_on(index, scale, "scale", torch.float32, rows)
    if torch.cuda.current_device() != index:
        with torch.cuda.device(index):
            st = _lib().gd_quantise_rows(xp, code, rows, columns, xs, qp, qs, sp, _stream_on(index, stream, x, q, scale))
    else:
        st = _lib().gd_quantise_rows(xp, code, rows, columns, xs, qp, qs, sp, _stream_on(index, stream, x, q, scale))
    if st != 0:
        raise GDError(st, "gd_quantise_rows")
    return q, scale


@dataclass
class AdamWState:
    """The moments of an AdamW, the caller's like every other state: in float32, or int8 and uint8 codes with a
    float32 unit per block of 256 elements of a tensor."""

    m: torch.Tensor
    v: torch.Tensor
    m_unit: Optional[torch.Tensor] = None
    v_unit: Optional[torch.Tensor] = None


class AdamW(_Handle):
    """An AdamW step over all tensors of a layout at once (gd_adamw_*), moments in ``bits`` = 32 or 8 bits.

    ``decay``: a factor per tensor on the step's weight decay (0 for biases and norms, say); all 1 by default.
    """

    _what = "adamw"

    def __init__(self, offsets: Sequence[int], bits: int = 32, decay: Optional[Sequence[float]] = None, device=None):
        if bits not in (32, 8):
            raise ValueError("bits must be 32 or 8")
        self.offsets = [int(o) for o in offsets]
        self.T, self.bits = len(self.offsets) - 1, bits
        if self.T < 1 or min(self.offsets) < 0:
            raise GDError(2, "AdamW")
        self.N = self.offsets[-1]
        if decay is not None and len(decay) != self.T:
            raise ValueError(f"need {self.T} decay factors, got {len(decay)}")
        d = None if decay is None else (ctypes.c_float * self.T)(*[float(x) for x in decay])
        self._create(device, (ctypes.c_uint64 * (self.T + 1))(*self.offsets), self.T, 1 if bits == 8 else 0, d)
        self.blocks = int(_lib().gd_adamw_blocks(self._h))

    def init_state(self) -> AdamWState:
        """Moments before the first step: zeros."""
        kinds = (torch.int8, torch.uint8) if self.bits == 8 else (torch.float32, torch.float32)
        m, v = (torch.zeros(self.N, dtype=k, device=self.device) for k in kinds)
        if self.bits == 32:
            return AdamWState(m, v)
        return AdamWState(m, v, *(torch.zeros(self.blocks, device=self.device) for _ in range(2)))

    def step(self, params, grad, state: AdamWState, step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
             weight_decay: float = 0.01, max_norm: Optional[float] = None, grad_scale: float = 1.0, copy=None,
             stream=None):
        """One step, numbered from 1: params (float32) and state change in place; ``copy`` (bfloat16 or float16)
        receives the new params rounded.  grad is float32, bfloat16 or float16.

        With ``max_norm`` the scaled gradient is clipped to that 2-norm over all tensors, and its norm is
        returned (one float32 on the device); when it is not finite, nothing else changes.
        """
        if not 1 <= int(step) < 1 << 63:
            raise ValueError("steps are numbered from 1")
        io = _AdamWIO(step=int(step), lr=lr, beta1=betas[0], beta2=betas[1], eps=eps, weight_decay=weight_decay,
                      grad_scale=grad_scale, max_norm=0.0, copy_type=1)
        io.params = self._tensor(params, "params", torch.float32, self.N)
        io.grad_type = _dtype_code(grad.dtype)
        io.grad = self._tensor(grad, "grad", grad.dtype, self.N)
        self._state(state, io)
        if copy is not None:
            if copy.dtype not in (torch.bfloat16, torch.float16):
                raise TypeError("copy must be bfloat16 or float16")
            io.copy_type = _DTYPES[copy.dtype]
            io.copy = self._tensor(copy, "copy", copy.dtype, self.N)
        norm = None
        if max_norm is not None:
            if not max_norm > 0:
                raise ValueError("max_norm must be above 0")
            norm = _new(stream, torch.empty, 1, dtype=torch.float32, device=self.device)
            io.max_norm, io.norm = max_norm, norm.data_ptr()
        st = _lib().gd_adamw_step(self._h, io, self._stream(stream, params, grad, state.m, state.v, state.m_unit,
                                                            state.v_unit, copy, norm))
        if st != 0:
            raise GDError(st, "gd_adamw_step")
        return norm

    def _state(self, state, io) -> None:
        if self.bits == 8:
            io.m = self._tensor(state.m, "state.m", torch.int8, self.N)
            io.v = self._tensor(state.v, "state.v", torch.uint8, self.N)
            io.m_unit = self._tensor(state.m_unit, "state.m_unit", torch.float32, self.blocks)
            io.v_unit = self._tensor(state.v_unit, "state.v_unit", torch.float32, self.blocks)
        else:
            io.m = self._tensor(state.m, "state.m", torch.float32, self.N)
            io.v = self._tensor(state.v, "state.v", torch.float32, self.N)

    def decode(self, state: AdamWState, stream=None):
        """(m, v) in float32 that an 8-bit state stands for."""
        if self.bits != 8:
            raise ValueError("the state is in 32 bits already")
        io = _AdamWIO()
        self._state(state, io)
        m, v = (_new(stream, torch.empty, self.N, dtype=torch.float32, device=self.device) for _ in range(2))
        st = _lib().gd_adamw_decode(self._h, io.m, io.v, io.m_unit, io.v_unit, m.data_ptr(), v.data_ptr(),
                                    self._stream(stream, state.m, state.v, state.m_unit, state.v_unit, m, v))
        if st != 0:
            raise GDError(st, "gd_adamw_decode")
        return m, v
