"""ctypes binding of include/orbit.h: argument marshalling only.

Every function named ``orbit_*`` here calls the C entry point of the same name
with raw device pointers taken from torch tensors and the current HIP stream;
no computation happens in Python. Missing libraries raise immediately — there
is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint8, c_void_p
from typing import Dict, Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "liborbit.so")

ORBIT_OK, ORBIT_E_ARG, ORBIT_E_UNSUPPORTED, ORBIT_E_DEVICE = 0, 1, 2, 3
ORBIT_F32, ORBIT_BF16 = 0, 1
ABI_VERSION = 2

BLOCK_PARAMS = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "qn_g", "qn_b", "kn_g", "kn_b",
                "w_proj", "b_proj", "ln2_g", "ln2_b", "w_fc1", "b_fc1", "w_fc2", "b_fc2")
AGG_PARAMS = ("q0", "w_q", "b_q", "w_k", "b_k", "w_v", "b_v", "w_o", "b_o", "pos")
BLOCK_EXT_PARAMS = ("post1_g", "post1_b", "gate1", "post2_g", "post2_b", "gate2")
GATED_NORM_PARAMS = ("gate", "post_g", "post_b", "pre_g", "pre_b")
QK_NORM_PARAMS = ("qn_g", "qn_b", "kn_g", "kn_b")
BLOCK_FP8_WEIGHTS = ("w_qkv", "w_proj", "w_fc1", "w_fc2")
BLOCK_FP8_STORES = tuple(w + t for w in BLOCK_FP8_WEIGHTS for t in ("", "_t"))
ROPE_PAIRS = 128
HEAD_PARAMS = ("lnf_g", "lnf_b", "w_h", "b_h", "w_hid", "b_hid")


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


_AxisArray = c_uint8 * ROPE_PAIRS


def _axis(axis):
    if len(axis) > ROPE_PAIRS:
        raise ValueError(f"an axis for each of at most {ROPE_PAIRS} pairs, not {len(axis)}")
    return _AxisArray.from_buffer_copy(bytes(axis).ljust(ROPE_PAIRS, b"\0"))


class BlockDesc(ctypes.Structure):
    _fields_ = [("B", c_int32), ("L", c_int32), ("d", c_int32), ("heads", c_int32),
                ("head_dim", c_int32), ("mlp", c_int32), ("qk_norm", c_int32), ("eps", c_float),
                ("dtype", c_int32)]


class BlockParams(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in BLOCK_PARAMS]


class BlockGrads(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in BLOCK_PARAMS]


class BlockExt(ctypes.Structure):
    _fields_ = [("act8", c_int32), ("post_norm", c_int32), ("gate_rows", c_int32), ("scale", c_float)]


class BlockExtParams(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in BLOCK_EXT_PARAMS]


class BlockExtGrads(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in BLOCK_EXT_PARAMS]


class EmbedDesc(ctypes.Structure):
    _fields_ = [("B", c_int32), ("V", c_int32), ("H", c_int32), ("W", c_int32), ("patch", c_int32),
                ("d", c_int32), ("dtype", c_int32)]


class AggDesc(ctypes.Structure):
    _fields_ = [("B", c_int32), ("L", c_int32), ("V", c_int32), ("d", c_int32), ("heads", c_int32),
                ("head_dim", c_int32), ("dtype", c_int32)]


class AggParams(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in AGG_PARAMS]


class AggGrads(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in AGG_PARAMS]


class HeadDesc(ctypes.Structure):
    _fields_ = [("B", c_int32), ("L", c_int32), ("d", c_int32), ("out", c_int32), ("final_ln", c_int32),
                ("eps", c_float), ("dtype", c_int32), ("hidden", c_int32)]


class WmseDesc(ctypes.Structure):
    _fields_ = [("B", c_int32), ("H", c_int32), ("W", c_int32), ("V", c_int32), ("patch", c_int32)]


class HeadParams(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in HEAD_PARAMS]


class HeadGrads(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in HEAD_PARAMS]


class GatedNormDesc(ctypes.Structure):
    _fields_ = [("rows", c_int32), ("n", c_int32), ("gate_rows", c_int32), ("post_norm", c_int32),
                ("pre_norm", c_int32), ("scale", c_float), ("eps", c_float), ("dtype", c_int32)]


class GatedNormParams(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in GATED_NORM_PARAMS]


class GatedNormGrads(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in GATED_NORM_PARAMS]


class Fp8LinearDesc(ctypes.Structure):
    _fields_ = [("rows", c_int32), ("n_in", c_int32), ("n_out", c_int32), ("dtype", c_int32)]


class QkRopeDesc(ctypes.Structure):
    _fields_ = [("tokens", c_int32), ("q_heads", c_int32), ("k_heads", c_int32), ("head_dim", c_int32),
                ("norm", c_int32), ("near", c_int32), ("axes", c_int32), ("pos_rows", c_int32), ("eps", c_float),
                ("dtype", c_int32), ("axis", _AxisArray)]

    @classmethod
    def of(cls, tokens, q_heads, k_heads, head_dim, dtype, axis, axes, pos_rows, norm=True, near=False, eps=1e-5):
        """axis: the axis of each of the head's head_dim / 2 pairs."""
        return cls(tokens, q_heads, k_heads, head_dim, int(norm), int(near), axes, pos_rows, eps, dtype, _axis(axis))


class BlockRope(ctypes.Structure):
    _fields_ = [("axes", c_int32), ("pos_rows", c_int32), ("near", c_int32), ("axis", _AxisArray),
                ("pos", c_void_p), ("freq", c_void_p)]

    @classmethod
    def of(cls, axis, axes, pos_rows, pos, freq, near=False):
        return cls(axes, pos_rows, int(near), _axis(axis), _ptr(pos), _ptr(freq))


class BlockFp8(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in BLOCK_FP8_STORES]


class BlockOpt(ctypes.Structure):
    _fields_ = [("rope", POINTER(BlockRope)), ("fp8", POINTER(BlockFp8))]

    @classmethod
    def of(cls, rope: Optional[BlockRope] = None, fp8: Optional[Dict[str, object]] = None):
        """fp8: the weights' stores by name (w_qkv, w_qkv_t, ...)."""
        f = None if fp8 is None else BlockFp8(*[_ptr(fp8.get(n)) for n in BLOCK_FP8_STORES])
        return cls(None if rope is None else ctypes.pointer(rope), None if f is None else ctypes.pointer(f))


class QkRopeParams(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in QK_NORM_PARAMS]


class QkRopeGrads(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in QK_NORM_PARAMS]


class OrbitError(RuntimeError):
    def __init__(self, fn: str, status: int, detail: str):
        super().__init__(f"{fn} failed with status {status}: {detail}")
        self.status = status
        self.detail = detail


# C prototypes: name -> (restype, argtypes)
P = c_void_p
_PROTOS = {
    "orbit_vit_block_saved_bytes": (c_size_t, [POINTER(BlockDesc)]),
    "orbit_vit_block_workspace_bytes": (c_size_t, [POINTER(BlockDesc)]),
    "orbit_vit_block_fwd": (c_int, [POINTER(BlockDesc), POINTER(BlockParams), P, P, P, P, c_size_t, P]),
    "orbit_vit_block_bwd": (c_int, [POINTER(BlockDesc), POINTER(BlockParams), P, P, P, P, POINTER(BlockGrads),
                                    c_int, P, c_size_t, P]),
    "orbit_vit_block_ext_saved_bytes": (c_size_t, [POINTER(BlockDesc), POINTER(BlockExt)]),
    "orbit_vit_block_ext_workspace_bytes": (c_size_t, [POINTER(BlockDesc), POINTER(BlockExt)]),
    "orbit_vit_block_ext_fwd": (c_int, [POINTER(BlockDesc), POINTER(BlockExt), POINTER(BlockParams),
                                        POINTER(BlockExtParams), P, P, P, P, c_size_t, P]),
    "orbit_vit_block_ext_bwd": (c_int, [POINTER(BlockDesc), POINTER(BlockExt), POINTER(BlockParams),
                                        POINTER(BlockExtParams), P, P, P, P, POINTER(BlockGrads),
                                        POINTER(BlockExtGrads), c_int, P, c_size_t, P]),
    "orbit_patch_embed": (c_int, [POINTER(EmbedDesc), P, P, P, P, P, P]),
    "orbit_patch_embed_workspace_bytes": (c_size_t, [POINTER(EmbedDesc)]),
    "orbit_patch_embed_bwd": (c_int, [POINTER(EmbedDesc), P, P, P, P, P, c_int, P, c_size_t, P]),
    "orbit_var_aggregate_saved_bytes": (c_size_t, [POINTER(AggDesc)]),
    "orbit_var_aggregate_workspace_bytes": (c_size_t, [POINTER(AggDesc)]),
    "orbit_var_aggregate": (c_int, [POINTER(AggDesc), P, POINTER(AggParams), P, P, P, c_size_t, P]),
    "orbit_var_aggregate_bwd": (c_int, [POINTER(AggDesc), P, POINTER(AggParams), P, P, P, POINTER(AggGrads),
                                        c_int, P, c_size_t, P]),
    "orbit_head_saved_bytes": (c_size_t, [POINTER(HeadDesc)]),
    "orbit_head_workspace_bytes": (c_size_t, [POINTER(HeadDesc)]),
    "orbit_head_fwd": (c_int, [POINTER(HeadDesc), P, POINTER(HeadParams), P, P, P, c_size_t, P]),
    "orbit_head_bwd": (c_int, [POINTER(HeadDesc), P, POINTER(HeadParams), P, P, P, POINTER(HeadGrads), c_int, P,
                               c_size_t, P]),
    "orbit_mse_workspace_bytes": (c_size_t, [c_int64]),
    "orbit_mse_loss": (c_int, [P, P, c_int64, c_float, P, P, P, c_size_t, P]),
    "orbit_wmse_workspace_bytes": (c_size_t, [POINTER(WmseDesc)]),
    "orbit_wmse_loss": (c_int, [POINTER(WmseDesc), P, P, c_float, P, P, P, c_size_t, P]),
    "orbit_gemm_workspace_bytes": (c_size_t, [c_int32] * 6),
    "orbit_gemm": (c_int, [c_int32, c_int32, c_int32, c_int32, P, c_int64, c_int32, P, c_int64, c_int32, P,
                           c_int64, c_int32, c_float, P, c_int32, P, c_size_t, P]),
    "orbit_attention_fwd": (c_int, [c_int32] * 5 + [P, c_int64, P, c_int64, P, c_int64, P, c_int64, P, P, c_int64,
                                                    P]),
    "orbit_attention_bwd_workspace_bytes": (c_size_t, [c_int32] * 4),
    "orbit_attention_bwd": (c_int, [c_int32] * 5 + [P, c_int64, P, c_int64, P, c_int64, P, c_int64, c_int32, P, P,
                                                    c_int64, P, P, P, c_int64, P, c_size_t, P]),
    "orbit_attention_bwd_noalloc": (c_int, [c_int32] * 5 + [P, c_int64, P, c_int64, P, c_int64, P, c_int64, c_int32,
                                                            P, P, c_int64, P, P, P, c_int64, P]),
    "orbit_layernorm_fwd": (c_int, [c_int32, c_int32, c_int32, P, P, P, c_float, P, P, P, P]),
    "orbit_act8_bytes": (c_size_t, [c_int64, c_int32]),
    "orbit_act8_pack": (c_int, [c_int32, c_int64, c_int32, P, c_int64, P, c_size_t, P]),
    "orbit_act8_unpack": (c_int, [c_int32, c_int64, c_int32, P, c_size_t, P, c_int64, P, c_int64, P]),
    "orbit_act8_weight_grad_workspace_bytes": (c_size_t, [c_int32] * 4),
    "orbit_act8_weight_grad": (c_int, [c_int32] * 4 + [P, c_size_t, P, c_int64, P, P, c_int32, P, c_size_t, P]),
    "orbit_gated_norm_fwd": (c_int, [POINTER(GatedNormDesc), POINTER(GatedNormParams), P, P, P, c_size_t, P, P, P, P]),
    "orbit_gated_norm_bwd_workspace_bytes": (c_size_t, [POINTER(GatedNormDesc)]),
    "orbit_gated_norm_bwd": (c_int, [POINTER(GatedNormDesc), POINTER(GatedNormParams), P, P, c_size_t, P, P, P, P, P,
                                     P, POINTER(GatedNormGrads), c_int, P, c_size_t, P]),
    "orbit_fp8_bytes": (c_size_t, [c_int64, c_int64]),
    "orbit_fp8_pack": (c_int, [c_int32, c_int64, c_int64, c_int32, P, c_int64, P, c_size_t, P, c_size_t, P]),
    "orbit_fp8_unpack": (c_int, [c_int32, c_int64, c_int64, P, c_size_t, P, c_int64, P]),
    "orbit_fp8_gemm_workspace_bytes": (c_size_t, [c_int32] * 3),
    "orbit_fp8_gemm": (c_int, [c_int32] * 4 + [P, c_size_t, P, c_size_t, P, c_int64, c_int32, P, c_int32, P, c_size_t, P]),
    "orbit_fp8_linear_saved_bytes": (c_size_t, [POINTER(Fp8LinearDesc)]),
    "orbit_fp8_linear_workspace_bytes": (c_size_t, [POINTER(Fp8LinearDesc)]),
    "orbit_fp8_linear_fwd": (c_int, [POINTER(Fp8LinearDesc), P, c_int64, P, c_size_t, P, P, c_int64, P, P, c_size_t, P]),
    "orbit_fp8_linear_bwd": (c_int, [POINTER(Fp8LinearDesc), P, P, c_size_t, P, c_int64, P, c_int64, P, P, c_int32, P,
                                     c_size_t, P]),
    "orbit_qk_rope_fwd": (c_int, [POINTER(QkRopeDesc), POINTER(QkRopeParams), P, P, P, c_int64, P, c_int64, P, P, P]),
    "orbit_qk_rope_bwd_workspace_bytes": (c_size_t, [POINTER(QkRopeDesc)]),
    "orbit_qk_rope_bwd": (c_int, [POINTER(QkRopeDesc), POINTER(QkRopeParams), P, P, P, c_int64, P, P, P, c_int64, P,
                                  c_int64, POINTER(QkRopeGrads), c_int32, P, c_size_t, P]),
    "orbit_vit_block_opt_saved_bytes": (c_size_t, [POINTER(BlockDesc), POINTER(BlockExt), POINTER(BlockOpt)]),
    "orbit_vit_block_opt_workspace_bytes": (c_size_t, [POINTER(BlockDesc), POINTER(BlockExt), POINTER(BlockOpt)]),
    "orbit_vit_block_opt_fwd": (c_int, [POINTER(BlockDesc), POINTER(BlockExt), POINTER(BlockOpt), POINTER(BlockParams),
                                        POINTER(BlockExtParams), P, P, P, P, c_size_t, P]),
    "orbit_vit_block_opt_bwd": (c_int, [POINTER(BlockDesc), POINTER(BlockExt), POINTER(BlockOpt), POINTER(BlockParams),
                                        POINTER(BlockExtParams), P, P, P, P, POINTER(BlockGrads),
                                        POINTER(BlockExtGrads), c_int, P, c_size_t, P]),
    "orbit_status_string": (c_char_p, [c_int]),
    "orbit_last_error": (c_char_p, []),
    "orbit_abi_version": (c_int, []),
    "orbit_timing_enable": (c_int, [c_int]),
    "orbit_timing_filter": (c_int, [c_char_p]),
    "orbit_timing_summary": (c_int, [c_char_p, POINTER(c_int64), POINTER(c_double), POINTER(c_double),
                                     POINTER(c_double)]),
    "orbit_timing_kernel_name": (c_char_p, [c_int]),
    "orbit_mfma_probe": (c_int, [c_int32, c_int32, ctypes.c_uint32, c_float, P, P]),
}

EXPORTS = tuple(_PROTOS)


def _stream(stream) -> Optional[int]:
    if stream is None:
        # the current stream's handle without a Stream object (0.4 us a call instead of 2.8), where this
        # torch has the private call for it
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


class OrbitLib:
    """The loaded library. Methods mirror the C entry points."""

    def __init__(self, path: str = LIB_PATH):
        if not os.path.exists(path):
            raise RuntimeError(f"HIP library {path} is missing: build it with "
                               "`python -m paper_2404_14712_amd.build` (no CPU fallback exists)")
        self.path = path
        self.lib = ctypes.CDLL(path)
        for name, (res, args) in _PROTOS.items():
            f = getattr(self.lib, name)
            f.restype = res
            f.argtypes = args
        v = self.lib.orbit_abi_version()
        if v != ABI_VERSION:
            raise RuntimeError(f"{path}: ABI version {v}, expected {ABI_VERSION}")

    # -- helpers --------------------------------------------------------
    def _check(self, fn: str, st: int):
        if st != ORBIT_OK:
            raise OrbitError(fn, st, self.lib.orbit_last_error().decode())

    @staticmethod
    def _struct(cls, tensors: Dict[str, object]):
        s = cls()
        for n, _ in cls._fields_:
            setattr(s, n, _ptr(tensors.get(n)))
        return s

    def last_error(self) -> str:
        return self.lib.orbit_last_error().decode()

    # -- block ---------------------------------------------------------------
    def orbit_vit_block_saved_bytes(self, desc: BlockDesc) -> int:
        return self.lib.orbit_vit_block_saved_bytes(ctypes.byref(desc))

    def orbit_vit_block_workspace_bytes(self, desc: BlockDesc) -> int:
        return self.lib.orbit_vit_block_workspace_bytes(ctypes.byref(desc))

    def orbit_vit_block_fwd(self, desc, params, x, y, saved, ws, stream=None):
        p = self._struct(BlockParams, params)
        self._check("orbit_vit_block_fwd", self.lib.orbit_vit_block_fwd(
            ctypes.byref(desc), ctypes.byref(p), _ptr(x), _ptr(y), _ptr(saved), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream)))

    def orbit_vit_block_bwd(self, desc, params, x, saved, dy, dx, grads, accumulate, ws, stream=None):
        p = self._struct(BlockParams, params)
        g = self._struct(BlockGrads, grads)
        self._check("orbit_vit_block_bwd", self.lib.orbit_vit_block_bwd(
            ctypes.byref(desc), ctypes.byref(p), _ptr(x), _ptr(saved), _ptr(dy), _ptr(dx), ctypes.byref(g),
            int(accumulate), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))

    # -- block with gated norms and / or saved tensors in 8 bits ------------------
    def orbit_vit_block_ext_saved_bytes(self, desc: BlockDesc, ext: BlockExt) -> int:
        return self.lib.orbit_vit_block_ext_saved_bytes(ctypes.byref(desc), ctypes.byref(ext))

    def orbit_vit_block_ext_workspace_bytes(self, desc: BlockDesc, ext: BlockExt) -> int:
        return self.lib.orbit_vit_block_ext_workspace_bytes(ctypes.byref(desc), ctypes.byref(ext))

    def orbit_vit_block_ext_fwd(self, desc, ext, params, x, y, saved, ws, stream=None):
        """params: the block's and the extension's, by name."""
        p, e = self._struct(BlockParams, params), self._struct(BlockExtParams, params)
        self._check("orbit_vit_block_ext_fwd", self.lib.orbit_vit_block_ext_fwd(
            ctypes.byref(desc), ctypes.byref(ext), ctypes.byref(p), ctypes.byref(e), _ptr(x), _ptr(y), _ptr(saved),
            _ptr(ws), _nbytes(ws), _stream(stream)))

    def orbit_vit_block_ext_bwd(self, desc, ext, params, x, saved, dy, dx, grads, accumulate, ws, stream=None):
        p, e = self._struct(BlockParams, params), self._struct(BlockExtParams, params)
        g, eg = self._struct(BlockGrads, grads), self._struct(BlockExtGrads, grads)
        self._check("orbit_vit_block_ext_bwd", self.lib.orbit_vit_block_ext_bwd(
            ctypes.byref(desc), ctypes.byref(ext), ctypes.byref(p), ctypes.byref(e), _ptr(x), _ptr(saved), _ptr(dy),
            _ptr(dx), ctypes.byref(g), ctypes.byref(eg), int(accumulate), _ptr(ws), _nbytes(ws), _stream(stream)))

    # -- patch embedding -------------------------------------------------------
    def orbit_patch_embed(self, desc, img, w_pe, b_pe, ve, tok, stream=None):
        self._check("orbit_patch_embed", self.lib.orbit_patch_embed(
            ctypes.byref(desc), _ptr(img), _ptr(w_pe), _ptr(b_pe), _ptr(ve), _ptr(tok), _stream(stream)))

    def orbit_patch_embed_workspace_bytes(self, desc) -> int:
        return self.lib.orbit_patch_embed_workspace_bytes(ctypes.byref(desc))

    def orbit_patch_embed_bwd(self, desc, img, dtok, dw_pe, db_pe, dve, accumulate, ws, stream=None):
        self._check("orbit_patch_embed_bwd", self.lib.orbit_patch_embed_bwd(
            ctypes.byref(desc), _ptr(img), _ptr(dtok), _ptr(dw_pe), _ptr(db_pe), _ptr(dve), int(accumulate),
            _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))

    # -- aggregation -----------------------------------------------------------
    def orbit_var_aggregate_saved_bytes(self, desc) -> int:
        return self.lib.orbit_var_aggregate_saved_bytes(ctypes.byref(desc))

    def orbit_var_aggregate_workspace_bytes(self, desc) -> int:
        return self.lib.orbit_var_aggregate_workspace_bytes(ctypes.byref(desc))

    def orbit_var_aggregate(self, desc, tok, params, z, saved, ws, stream=None):
        p = self._struct(AggParams, params)
        self._check("orbit_var_aggregate", self.lib.orbit_var_aggregate(
            ctypes.byref(desc), _ptr(tok), ctypes.byref(p), _ptr(z), _ptr(saved), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream)))

    def orbit_var_aggregate_bwd(self, desc, tok, params, saved, dz, dtok, grads, accumulate, ws, stream=None):
        p = self._struct(AggParams, params)
        g = self._struct(AggGrads, grads)
        self._check("orbit_var_aggregate_bwd", self.lib.orbit_var_aggregate_bwd(
            ctypes.byref(desc), _ptr(tok), ctypes.byref(p), _ptr(saved), _ptr(dz), _ptr(dtok), ctypes.byref(g),
            int(accumulate), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))

    # -- head ------------------------------------------------------------------
    def orbit_head_saved_bytes(self, desc) -> int:
        return self.lib.orbit_head_saved_bytes(ctypes.byref(desc))

    def orbit_head_workspace_bytes(self, desc) -> int:
        return self.lib.orbit_head_workspace_bytes(ctypes.byref(desc))

    def orbit_head_fwd(self, desc, x, params, pred, saved, ws, stream=None):
        p = self._struct(HeadParams, params)
        self._check("orbit_head_fwd", self.lib.orbit_head_fwd(
            ctypes.byref(desc), _ptr(x), ctypes.byref(p), _ptr(pred), _ptr(saved), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream)))

    def orbit_head_bwd(self, desc, x, params, saved, dpred, dx, grads, accumulate, ws, stream=None):
        p = self._struct(HeadParams, params)
        g = self._struct(HeadGrads, grads)
        self._check("orbit_head_bwd", self.lib.orbit_head_bwd(
            ctypes.byref(desc), _ptr(x), ctypes.byref(p), _ptr(saved), _ptr(dpred), _ptr(dx), ctypes.byref(g),
            int(accumulate), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))

    # -- loss ------------------------------------------------------------------
    def orbit_mse_workspace_bytes(self, n: int) -> int:
        return self.lib.orbit_mse_workspace_bytes(int(n))

    def orbit_mse_loss(self, pred, tgt, n, scale, loss, dpred, ws, stream=None):
        self._check("orbit_mse_loss", self.lib.orbit_mse_loss(
            _ptr(pred), _ptr(tgt), int(n), float(scale), _ptr(loss), _ptr(dpred), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream)))

    def orbit_wmse_workspace_bytes(self, desc) -> int:
        return self.lib.orbit_wmse_workspace_bytes(ctypes.byref(desc))

    def orbit_wmse_loss(self, desc, pred, tgt, scale, loss, dpred, ws, stream=None):
        self._check("orbit_wmse_loss", self.lib.orbit_wmse_loss(
            ctypes.byref(desc), _ptr(pred), _ptr(tgt), float(scale), _ptr(loss), _ptr(dpred), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream)))

    # -- building blocks -------------------------------------------------------
    def orbit_gemm_workspace_bytes(self, dtype, M, N, K, a_kmajor, b_kmajor) -> int:
        return self.lib.orbit_gemm_workspace_bytes(dtype, M, N, K, int(a_kmajor), int(b_kmajor))

    def orbit_gemm(self, dtype, M, N, K, A, lda, a_kmajor, B, ldb, b_kmajor, C, ldc, c_f32, alpha=1.0,
                   bias=None, accumulate=0, ws=None, stream=None):
        nb = 0 if ws is None else ws.numel() * ws.element_size()
        self._check("orbit_gemm", self.lib.orbit_gemm(
            dtype, M, N, K, _ptr(A), lda, int(a_kmajor), _ptr(B), ldb, int(b_kmajor), _ptr(C), ldc, int(c_f32),
            float(alpha), _ptr(bias), int(accumulate), _ptr(ws), nb, _stream(stream)))

    def orbit_attention_fwd(self, dtype, B, H, L, dh, q, ldq, k, ldk, v, ldv, o, ldo, lse, o32=None, ldo32=0,
                            stream=None):
        self._check("orbit_attention_fwd", self.lib.orbit_attention_fwd(
            dtype, B, H, L, dh, _ptr(q), ldq, _ptr(k), ldk, _ptr(v), ldv, _ptr(o), ldo, _ptr(lse), _ptr(o32),
            ldo32, _stream(stream)))

    def orbit_attention_bwd_workspace_bytes(self, B, H, L, dh) -> int:
        return self.lib.orbit_attention_bwd_workspace_bytes(B, H, L, dh)

    def orbit_attention_bwd(self, dtype, B, H, L, dh, q, ldq, k, ldk, v, ldv, o, ldo, o_f32, lse, dO, lddo, dq, dk,
                            dv, ldg, ws, stream=None):
        self._check("orbit_attention_bwd", self.lib.orbit_attention_bwd(
            dtype, B, H, L, dh, _ptr(q), ldq, _ptr(k), ldk, _ptr(v), ldv, _ptr(o), ldo, int(o_f32), _ptr(lse),
            _ptr(dO), lddo, _ptr(dq), _ptr(dk), _ptr(dv), ldg, _ptr(ws), ws.numel() * ws.element_size(),
            _stream(stream)))

    def orbit_attention_bwd_noalloc(self, dtype, B, H, L, dh, q, ldq, k, ldk, v, ldv, o, ldo, o_f32, lse, dO, lddo,
                                    dq, dk, dv, ldg, stream=None):
        self._check("orbit_attention_bwd_noalloc", self.lib.orbit_attention_bwd_noalloc(
            dtype, B, H, L, dh, _ptr(q), ldq, _ptr(k), ldk, _ptr(v), ldv, _ptr(o), ldo, int(o_f32), _ptr(lse),
            _ptr(dO), lddo, _ptr(dq), _ptr(dk), _ptr(dv), ldg, _stream(stream)))

    def orbit_layernorm_fwd(self, dtype, rows, n, x, g, b, eps, y, mean, rstd, stream=None):
        self._check("orbit_layernorm_fwd", self.lib.orbit_layernorm_fwd(
            dtype, rows, n, _ptr(x), _ptr(g), _ptr(b), float(eps), _ptr(y), _ptr(mean), _ptr(rstd),
            _stream(stream)))

    # -- 8-bit activation store ------------------------------------------------
    def orbit_act8_bytes(self, rows, n) -> int:
        return self.lib.orbit_act8_bytes(int(rows), int(n))

    def orbit_act8_pack(self, dtype, rows, n, x, ldx, store, stream=None):
        self._check("orbit_act8_pack", self.lib.orbit_act8_pack(
            dtype, rows, n, _ptr(x), ldx, _ptr(store), _nbytes(store), _stream(stream)))

    def orbit_act8_unpack(self, dtype, rows, n, store, x, ldx, gelu=None, ldgelu=0, stream=None):
        self._check("orbit_act8_unpack", self.lib.orbit_act8_unpack(
            dtype, rows, n, _ptr(store), _nbytes(store), _ptr(x), ldx, _ptr(gelu), ldgelu, _stream(stream)))

    def orbit_act8_weight_grad_workspace_bytes(self, dtype, rows, K, N) -> int:
        return self.lib.orbit_act8_weight_grad_workspace_bytes(dtype, rows, K, N)

    def orbit_act8_weight_grad(self, dtype, rows, K, N, store, dy, lddy, dw, db, accumulate, ws, stream=None):
        self._check("orbit_act8_weight_grad", self.lib.orbit_act8_weight_grad(
            dtype, rows, K, N, _ptr(store), _nbytes(store), _ptr(dy), lddy, _ptr(dw), _ptr(db), int(accumulate),
            _ptr(ws), _nbytes(ws), _stream(stream)))

    # -- gated norms -----------------------------------------------------------
    def orbit_gated_norm_fwd(self, desc, params, x, f, store, y, h, stats, stream=None):
        p = self._struct(GatedNormParams, params)
        self._check("orbit_gated_norm_fwd", self.lib.orbit_gated_norm_fwd(
            ctypes.byref(desc), ctypes.byref(p), _ptr(x), _ptr(f), _ptr(store), _nbytes(store), _ptr(y), _ptr(h),
            _ptr(stats), _stream(stream)))

    def orbit_gated_norm_bwd_workspace_bytes(self, desc) -> int:
        return self.lib.orbit_gated_norm_bwd_workspace_bytes(ctypes.byref(desc))

    def orbit_gated_norm_bwd(self, desc, params, f, store, y, stats, dh, dy, dx, df, grads, accumulate, ws,
                             stream=None):
        p = self._struct(GatedNormParams, params)
        g = self._struct(GatedNormGrads, grads)
        self._check("orbit_gated_norm_bwd", self.lib.orbit_gated_norm_bwd(
            ctypes.byref(desc), ctypes.byref(p), _ptr(f), _ptr(store), _nbytes(store), _ptr(y), _ptr(stats), _ptr(dh),
            _ptr(dy), _ptr(dx), _ptr(df), ctypes.byref(g), int(accumulate), _ptr(ws), _nbytes(ws), _stream(stream)))

    # -- 8-bit floating point --------------------------------------------------
    def orbit_fp8_bytes(self, rows, n) -> int:
        return self.lib.orbit_fp8_bytes(int(rows), int(n))

    def orbit_fp8_pack(self, dtype, rows, n, tile_rows, x, ldx, store, store_t=None, stream=None):
        self._check("orbit_fp8_pack", self.lib.orbit_fp8_pack(
            dtype, rows, n, tile_rows, _ptr(x), ldx, _ptr(store), _nbytes(store), _ptr(store_t), _nbytes(store_t),
            _stream(stream)))

    def orbit_fp8_unpack(self, dtype, rows, n, store, x, ldx, stream=None):
        self._check("orbit_fp8_unpack", self.lib.orbit_fp8_unpack(
            dtype, rows, n, _ptr(store), _nbytes(store), _ptr(x), ldx, _stream(stream)))

    def orbit_fp8_gemm_workspace_bytes(self, M, N, K) -> int:
        return self.lib.orbit_fp8_gemm_workspace_bytes(M, N, K)

    def orbit_fp8_gemm(self, dtype, M, N, K, A, B, C, ldc, c_f32=0, bias=None, accumulate=0, ws=None, stream=None):
        self._check("orbit_fp8_gemm", self.lib.orbit_fp8_gemm(
            dtype, M, N, K, _ptr(A), _nbytes(A), _ptr(B), _nbytes(B), _ptr(C), ldc, int(c_f32), _ptr(bias),
            int(accumulate), _ptr(ws), _nbytes(ws), _stream(stream)))

    def orbit_fp8_linear_saved_bytes(self, desc) -> int:
        return self.lib.orbit_fp8_linear_saved_bytes(ctypes.byref(desc))

    def orbit_fp8_linear_workspace_bytes(self, desc) -> int:
        return self.lib.orbit_fp8_linear_workspace_bytes(ctypes.byref(desc))

    def orbit_fp8_linear_fwd(self, desc, x, ldx, w_t, bias, y, ldy, saved, ws, stream=None):
        self._check("orbit_fp8_linear_fwd", self.lib.orbit_fp8_linear_fwd(
            ctypes.byref(desc), _ptr(x), ldx, _ptr(w_t), _nbytes(w_t), _ptr(bias), _ptr(y), ldy, _ptr(saved), _ptr(ws),
            _nbytes(ws), _stream(stream)))

    def orbit_fp8_linear_bwd(self, desc, saved, w, dy, lddy, dx, lddx, dw, db, accumulate, ws, stream=None):
        self._check("orbit_fp8_linear_bwd", self.lib.orbit_fp8_linear_bwd(
            ctypes.byref(desc), _ptr(saved), _ptr(w), _nbytes(w), _ptr(dy), lddy, _ptr(dx), lddx, _ptr(dw), _ptr(db),
            int(accumulate), _ptr(ws), _nbytes(ws), _stream(stream)))

    # -- rotary positions ------------------------------------------------------
    def orbit_qk_rope_fwd(self, desc, params, pos, freq, src, lds, dst, ldd, mean=None, rstd=None, stream=None):
        p = self._struct(QkRopeParams, params)
        self._check("orbit_qk_rope_fwd", self.lib.orbit_qk_rope_fwd(
            ctypes.byref(desc), ctypes.byref(p), _ptr(pos), _ptr(freq), _ptr(src), lds, _ptr(dst), ldd, _ptr(mean),
            _ptr(rstd), _stream(stream)))

    def orbit_qk_rope_bwd_workspace_bytes(self, desc) -> int:
        return self.lib.orbit_qk_rope_bwd_workspace_bytes(ctypes.byref(desc))

    def orbit_qk_rope_bwd(self, desc, params, pos, freq, src, lds, mean, rstd, dy, lddy, dx, lddx, grads, accumulate=0,
                          ws=None, stream=None):
        p, g = self._struct(QkRopeParams, params), self._struct(QkRopeGrads, grads)
        self._check("orbit_qk_rope_bwd", self.lib.orbit_qk_rope_bwd(
            ctypes.byref(desc), ctypes.byref(p), _ptr(pos), _ptr(freq), _ptr(src), lds, _ptr(mean), _ptr(rstd),
            _ptr(dy), lddy, _ptr(dx), lddx, ctypes.byref(g), int(accumulate), _ptr(ws), _nbytes(ws), _stream(stream)))

    # -- block with rotary positions and / or 8-bit products ---------------------
    def orbit_vit_block_opt_saved_bytes(self, desc, ext, opt) -> int:
        return self.lib.orbit_vit_block_opt_saved_bytes(ctypes.byref(desc), ctypes.byref(ext), ctypes.byref(opt))

    def orbit_vit_block_opt_workspace_bytes(self, desc, ext, opt) -> int:
        return self.lib.orbit_vit_block_opt_workspace_bytes(ctypes.byref(desc), ctypes.byref(ext), ctypes.byref(opt))

    def orbit_vit_block_opt_fwd(self, desc, ext, opt, params, x, y, saved, ws, stream=None):
        p, e = self._struct(BlockParams, params), self._struct(BlockExtParams, params)
        self._check("orbit_vit_block_opt_fwd", self.lib.orbit_vit_block_opt_fwd(
            ctypes.byref(desc), ctypes.byref(ext), ctypes.byref(opt), ctypes.byref(p), ctypes.byref(e), _ptr(x),
            _ptr(y), _ptr(saved), _ptr(ws), _nbytes(ws), _stream(stream)))

    def orbit_vit_block_opt_bwd(self, desc, ext, opt, params, x, saved, dy, dx, grads, accumulate, ws, stream=None):
        p, e = self._struct(BlockParams, params), self._struct(BlockExtParams, params)
        g, eg = self._struct(BlockGrads, grads), self._struct(BlockExtGrads, grads)
        self._check("orbit_vit_block_opt_bwd", self.lib.orbit_vit_block_opt_bwd(
            ctypes.byref(desc), ctypes.byref(ext), ctypes.byref(opt), ctypes.byref(p), ctypes.byref(e), _ptr(x),
            _ptr(saved), _ptr(dy), _ptr(dx), ctypes.byref(g), ctypes.byref(eg), int(accumulate), _ptr(ws), _nbytes(ws),
            _stream(stream)))

    # -- measurement aid -------------------------------------------------------
    def orbit_mfma_probe(self, blocks, iters, seed, x, out, stream=None):
        self._check("orbit_mfma_probe", self.lib.orbit_mfma_probe(int(blocks), int(iters), int(seed), float(x),
                                                                  _ptr(out), _stream(stream)))

    # -- timing ----------------------------------------------------------------
    def orbit_timing_enable(self, on: bool):
        self._check("orbit_timing_enable", self.lib.orbit_timing_enable(1 if on else 0))

    def orbit_timing_filter(self, prefix: Optional[str]):
        self._check("orbit_timing_filter", self.lib.orbit_timing_filter(prefix.encode() if prefix else None))

    def orbit_timing_summary(self, prefix: Optional[str] = None):
        n, ms, fl, by = c_int64(), c_double(), c_double(), c_double()
        self._check("orbit_timing_summary", self.lib.orbit_timing_summary(
            prefix.encode() if prefix else None, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(fl),
            ctypes.byref(by)))
        return {"launches": n.value, "ms": ms.value, "flops": fl.value, "bytes": by.value}

    def orbit_timing_kernel_names(self):
        out, i = [], 0
        while True:
            s = self.lib.orbit_timing_kernel_name(i)
            if s is None:
                return out
            out.append(s.decode())
            i += 1
