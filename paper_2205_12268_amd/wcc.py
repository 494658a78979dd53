"""ctypes binding of libwcc (argument marshalling only; every step runs in the HIP kernels).

torch is used for device memory and for the current HIP stream, nothing else.  There is no
CPU fallback: if ``csrc/libwcc.so`` is missing or does not load, importing the symbols below
raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "csrc", "libwcc.so")

F32, BF16, I8, I4 = 0, 1, 2, 3
STATIC_SCRATCH_BYTES = 64 << 20  # WCC_STATIC_SCRATCH_BYTES of wcc.h
NORM_L1, NORM_L2 = 0, 1
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3
KEPT_BLOCK = 32  # WCC_KEPT_BLOCK of wcc.h
TRAIN_FINE = 2  # WCC_TRAIN_FINE of wcc.h
STAGES = ("haar_fwd", "norm_select", "gather", "pointwise", "scatter_ihaar", "event_pair",
          "depthwise")

EXPORTS = ("wcc_create", "wcc_destroy", "wcc_workspace_bytes", "wcc_set_workspace", "wcc_k",
           "wcc_status_string", "wcc_set_profiling", "wcc_stage_times", "wcc_haar_fwd",
           "wcc_joint_topk", "wcc_gather_quant", "wcc_pointwise", "wcc_scatter_ihaar",
           "wcc_forward", "wcc_forward_static", "wcc_forward_fixed", "wcc_block_workspace_bytes", "wcc_depthwise3x3", "wcc_block_forward",
           "wcc_set_block_profile_layer", "wcc_block_is_chained",
           "wcc_adapter_workspace_bytes", "wcc_adapter_forward", "wcc_adapter_backward",
           "wcc_scores_workspace_bytes", "wcc_token_scores",
           "wcc_distill_workspace_bytes", "wcc_distill_forward", "wcc_distill_backward",
           "wcc_rows_keep", "wcc_rows_restore",
           "wcc_group_norm_workspace_bytes", "wcc_group_norm_forward", "wcc_group_norm_backward",
           "wcc_gated_workspace_bytes", "wcc_gated_forward", "wcc_gated_backward")


class Desc(C.Structure):
    """Mirror of ``wcc_desc``."""
    _fields_ = [("B", C.c_int32), ("C_in", C.c_int32), ("C_out", C.c_int32), ("H", C.c_int32),
                ("W", C.c_int32), ("levels", C.c_int32), ("keep_num", C.c_int64),
                ("keep_den", C.c_int64), ("w_dtype", C.c_int32), ("act_quant_bits", C.c_int32),
                ("act_dtype", C.c_int32), ("norm", C.c_int32)]


class BlockDesc(C.Structure):
    """Mirror of ``wcc_block_desc``."""
    _fields_ = [("B", C.c_int32), ("C", C.c_int32), ("expansion", C.c_int32), ("H", C.c_int32),
                ("W", C.c_int32), ("levels", C.c_int32), ("keep_num", C.c_int64),
                ("keep_den", C.c_int64), ("w_dtype", C.c_int32), ("act_quant_bits", C.c_int32),
                ("act_dtype", C.c_int32), ("norm", C.c_int32)]


class AdapterDesc(C.Structure):
    """Mirror of ``wcc_adapter_desc``."""
    _fields_ = [("rows", C.c_int64), ("C_in", C.c_int32), ("C_out", C.c_int32), ("adapters", C.c_int32),
                ("rank", C.c_int32), ("dtype", C.c_int32), ("ldx", C.c_int64), ("ldy", C.c_int64)]


class ScoresDesc(C.Structure):
    """Mirror of ``wcc_scores_desc``."""
    _fields_ = [("rows", C.c_int64), ("V", C.c_int32), ("top", C.c_int32), ("dtype", C.c_int32), ("ld", C.c_int64)]


class DistillDesc(C.Structure):
    """Mirror of ``wcc_distill_desc``."""
    _fields_ = [("rows", C.c_int64), ("V", C.c_int32), ("K", C.c_int32), ("dtype", C.c_int32), ("t_dtype", C.c_int32),
                ("temperature", C.c_float), ("ld", C.c_int64), ("ld_grad", C.c_int64)]


class RowsDesc(C.Structure):
    """Mirror of ``wcc_rows_desc``."""
    _fields_ = [("rows", C.c_int64), ("width", C.c_int32), ("dtype", C.c_int32), ("ld", C.c_int64)]


class GroupNormDesc(C.Structure):
    """Mirror of ``wcc_group_norm_desc``."""
    _fields_ = [("samples", C.c_int32), ("pixels", C.c_int64), ("C", C.c_int32), ("groups", C.c_int32), ("act", C.c_int32),
                ("dtype", C.c_int32), ("eps", C.c_float), ("ldx", C.c_int64), ("ldy", C.c_int64)]


class GatedDesc(C.Structure):
    """Mirror of ``wcc_gated_desc``."""
    _fields_ = [("rows", C.c_int64), ("C_in", C.c_int32), ("C_out", C.c_int32), ("act", C.c_int32), ("dtype", C.c_int32),
                ("train", C.c_int32), ("ldx", C.c_int64), ("ldy", C.c_int64)]


class WccError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib():
    """Loads libwcc.so (built by ``__graft_entry__.build()``); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
        L = C.CDLL(LIB_PATH)
        vp, dp = C.c_void_p, C.POINTER(Desc)
        L.wcc_create.argtypes = [C.POINTER(vp), C.c_int]
        L.wcc_destroy.argtypes = [vp]
        L.wcc_workspace_bytes.argtypes = [dp, C.POINTER(C.c_size_t)]
        L.wcc_set_workspace.argtypes = [vp, vp, C.c_size_t]
        L.wcc_k.argtypes = [dp]
        L.wcc_k.restype = C.c_int64
        L.wcc_status_string.argtypes = [C.c_int]
        L.wcc_status_string.restype = C.c_char_p
        L.wcc_set_profiling.argtypes = [vp, C.c_int]
        L.wcc_stage_times.argtypes = [vp, C.POINTER(C.c_float)]
        L.wcc_haar_fwd.argtypes = [vp, dp, vp, vp, vp, vp]
        L.wcc_joint_topk.argtypes = [vp, dp, vp, vp, vp, vp]
        L.wcc_gather_quant.argtypes = [vp, dp, vp, vp, C.c_float, vp, vp, vp]
        L.wcc_pointwise.argtypes = [vp, dp, vp, vp, vp, vp, vp, vp]
        L.wcc_scatter_ihaar.argtypes = [vp, dp, vp, vp, vp, vp]
        L.wcc_forward.argtypes = [vp, dp, vp, vp, vp, C.c_float, vp, vp, vp, vp]
        L.wcc_forward_static.argtypes = [vp, dp, vp, vp, vp, C.c_float, vp, vp, vp, vp]
        L.wcc_forward_fixed.argtypes = [vp, dp, vp, vp, vp, C.c_float, vp, vp, vp, vp]
        bp = C.POINTER(BlockDesc)
        L.wcc_block_workspace_bytes.argtypes = [bp, C.POINTER(C.c_size_t)]
        L.wcc_depthwise3x3.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp]
        L.wcc_block_forward.argtypes = [vp, bp] + [vp] * 12
        L.wcc_set_block_profile_layer.argtypes = [vp, C.c_int]
        L.wcc_block_is_chained.argtypes = [bp]
        sz = C.POINTER(C.c_size_t)
        L.wcc_adapter_workspace_bytes.argtypes = [C.POINTER(AdapterDesc), sz]
        L.wcc_adapter_forward.argtypes = [vp, C.POINTER(AdapterDesc)] + [vp] * 9
        L.wcc_adapter_backward.argtypes = [vp, C.POINTER(AdapterDesc)] + [vp] * 12
        L.wcc_scores_workspace_bytes.argtypes = [C.POINTER(ScoresDesc), sz]
        L.wcc_token_scores.argtypes = [vp, C.POINTER(ScoresDesc)] + [vp] * 7
        L.wcc_distill_workspace_bytes.argtypes = [C.POINTER(DistillDesc), sz]
        L.wcc_distill_forward.argtypes = [vp, C.POINTER(DistillDesc)] + [vp] * 8
        L.wcc_distill_backward.argtypes = [vp, C.POINTER(DistillDesc)] + [vp] * 7
        for call in ("wcc_rows_keep", "wcc_rows_restore"):
            getattr(L, call).argtypes = [vp, C.POINTER(RowsDesc)] + [vp] * 4
        L.wcc_group_norm_workspace_bytes.argtypes = [C.POINTER(GroupNormDesc), sz]
        L.wcc_group_norm_forward.argtypes = [vp, C.POINTER(GroupNormDesc)] + [vp] * 9
        L.wcc_group_norm_backward.argtypes = [vp, C.POINTER(GroupNormDesc)] + [vp] * 12
        L.wcc_gated_workspace_bytes.argtypes = [C.POINTER(GatedDesc), sz]
        L.wcc_gated_forward.argtypes = [vp, C.POINTER(GatedDesc)] + [vp] * 7
        L.wcc_gated_backward.argtypes = [vp, C.POINTER(GatedDesc)] + [vp] * 12
        for name in EXPORTS:
            if name not in ("wcc_k", "wcc_status_string"):
                getattr(L, name).restype = C.c_int
        L.wcc_block_is_chained.restype = C.c_int32
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().wcc_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise WccError(status, where)


def make_desc(B, C_in, C_out, H, W, levels, keep_num, keep_den, w_dtype, act_quant_bits,
              act_dtype=F32, norm=NORM_L1) -> Desc:
    return Desc(B, C_in, C_out, H, W, levels, keep_num, keep_den, w_dtype, act_quant_bits, act_dtype,
                norm)


def k_of(desc: Desc) -> int:
    return int(lib().wcc_k(C.byref(desc)))


def workspace_bytes(desc: Desc) -> int:
    out = C.c_size_t(0)
    _check(lib().wcc_workspace_bytes(C.byref(desc), C.byref(out)), "wcc_workspace_bytes")
    return int(out.value)


def make_block_desc(B, Cc, expansion, H, W, levels, keep_num, keep_den, w_dtype,
                    act_quant_bits, act_dtype=F32, norm=NORM_L1) -> BlockDesc:
    return BlockDesc(B, Cc, expansion, H, W, levels, keep_num, keep_den, w_dtype, act_quant_bits,
                     act_dtype, norm)


def block_is_chained(desc: BlockDesc) -> bool:
    """Whether wcc_block_forward without middle outputs chains the two layers of this block."""
    r = int(lib().wcc_block_is_chained(C.byref(desc)))
    if r < 0:
        raise ValueError("invalid block descriptor")
    return r == 1


def block_workspace_bytes(desc: BlockDesc) -> int:
    out = C.c_size_t(0)
    _check(lib().wcc_block_workspace_bytes(C.byref(desc), C.byref(out)), "wcc_block_workspace_bytes")
    return int(out.value)


def make_adapter_desc(rows, C_in, C_out, adapters, rank, dtype, ldx=None, ldy=None) -> AdapterDesc:
    return AdapterDesc(rows, C_in, C_out, adapters, rank, dtype, C_in if ldx is None else ldx, C_out if ldy is None else ldy)


def make_scores_desc(rows, V, top, dtype, ld=None) -> ScoresDesc:
    return ScoresDesc(rows, V, top, dtype, V if ld is None else ld)


def make_distill_desc(rows, V, K, dtype, t_dtype=F32, temperature=1.0, ld=None, ld_grad=None) -> DistillDesc:
    return DistillDesc(rows, V, K, dtype, t_dtype, temperature, V if ld is None else ld, V if ld_grad is None else ld_grad)


def make_rows_desc(rows, width, dtype, ld=None) -> RowsDesc:
    return RowsDesc(rows, width, dtype, width if ld is None else ld)


def make_group_norm_desc(samples, pixels, Cc, groups, dtype, act=ACT_NONE, eps=1e-5, ldx=None, ldy=None) -> GroupNormDesc:
    return GroupNormDesc(samples, pixels, Cc, groups, act, dtype, eps, Cc if ldx is None else ldx, Cc if ldy is None else ldy)


def make_gated_desc(rows, C_in, C_out, dtype, act=ACT_SILU, train=False, ldx=None, ldy=None) -> GatedDesc:
    """train: False, True, or TRAIN_FINE."""
    return GatedDesc(rows, C_in, C_out, act, dtype, int(train) if train == TRAIN_FINE else int(bool(train)), C_in if ldx is None else ldx, C_out if ldy is None else ldy)


def kept_room(width: int) -> int:
    """Codes of a row of `width` values: whole blocks."""
    return -(-width // KEPT_BLOCK) * KEPT_BLOCK


def _workspace_of(desc) -> int:
    if isinstance(desc, RowsDesc):  # (its calls need none)
        return 0
    call = {BlockDesc: "wcc_block_workspace_bytes", AdapterDesc: "wcc_adapter_workspace_bytes",
            ScoresDesc: "wcc_scores_workspace_bytes", DistillDesc: "wcc_distill_workspace_bytes",
            GroupNormDesc: "wcc_group_norm_workspace_bytes", GatedDesc: "wcc_gated_workspace_bytes"}.get(type(desc), "wcc_workspace_bytes")
    out = C.c_size_t(0)
    _check(getattr(lib(), call)(C.byref(desc), C.byref(out)), call)
    return int(out.value)


def adapter_workspace_bytes(desc: AdapterDesc) -> int:
    return _workspace_of(desc)


def scores_workspace_bytes(desc: ScoresDesc) -> int:
    return _workspace_of(desc)


def distill_workspace_bytes(desc: DistillDesc) -> int:
    return _workspace_of(desc)


def group_norm_workspace_bytes(desc: GroupNormDesc) -> int:
    return _workspace_of(desc)


def gated_workspace_bytes(desc: GatedDesc) -> int:
    return _workspace_of(desc)


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous"
    return C.c_void_p(t.data_ptr())


_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_TORCH = {F32: torch.float32, BF16: torch.bfloat16}


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _rows(t, rows, width, ld, dtype, device=None):
    """Address of a matrix of tokens: [rows, width] of the descriptor's type, rows `ld` elements apart."""
    if t is None:
        return None
    assert (t.is_cuda if device is None else t.get_device() == device), "not on the context's device"
    assert t.shape == (rows, width) and _DTYPES.get(t.dtype) == dtype, "not the descriptor's matrix"
    a, b = t.stride()
    assert (b == 1 or width <= 1) and (a == ld or rows <= 1), "not the descriptor's row stride"
    return t.data_ptr()


def _whole(t, shape, dtype, device=None):
    """Address of a contiguous tensor of this shape and torch type."""
    if t is None:
        return None
    assert (t.is_cuda if device is None else t.get_device() == device), "not on the context's device"
    assert t.is_contiguous() and t.dtype == dtype and t.shape == shape, "not the descriptor's tensor"
    return t.data_ptr()


def _kept(codes, steps, lead, width, device):
    """Addresses of rows in 8 bits: codes [*lead, whole blocks of width], steps [*lead, blocks]."""
    room = kept_room(width)
    return _whole(codes, (*lead, room), torch.int8, device), _whole(steps, (*lead, room // KEPT_BLOCK), torch.uint8, device)


# (the current stream's handle without an object around it, which costs 2.5 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


class Context:
    """Owns a ``wcc_ctx`` and the torch tensor that backs its workspace."""

    def __init__(self, device: int = 0):
        self._h = C.c_void_p()
        self.device = device
        _check(lib().wcc_create(C.byref(self._h), device), "wcc_create")
        self._ws = None

    def close(self):
        if self._h:
            lib().wcc_destroy(self._h)
            self._h = C.c_void_p()
            self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def ensure_workspace(self, desc) -> int:
        need = _workspace_of(desc)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=f"cuda:{self.device}")
            _check(lib().wcc_set_workspace(self._h, _ptr(self._ws), self._ws.numel()),
                   "wcc_set_workspace")
        return need

    def set_workspace(self, tensor) -> None:
        self._ws = tensor
        _check(lib().wcc_set_workspace(self._h, _ptr(tensor), 0 if tensor is None else tensor.numel()),
               "wcc_set_workspace")

    def set_profiling(self, on: bool) -> None:
        _check(lib().wcc_set_profiling(self._h, int(bool(on))), "wcc_set_profiling")

    def stage_times(self) -> dict:
        ms = (C.c_float * len(STAGES))()
        _check(lib().wcc_stage_times(self._h, ms), "wcc_stage_times")
        return {n: float(ms[i]) for i, n in enumerate(STAGES)}

    # ---- the five stages and the fused call: same names as the C entry points ----
    def wcc_haar_fwd(self, desc, x, coef, norm=None):
        _check(lib().wcc_haar_fwd(self._h, C.byref(desc), _ptr(x), _ptr(coef), _ptr(norm), _stream()),
               "wcc_haar_fwd")

    def wcc_joint_topk(self, desc, coef, norm, idx):
        _check(lib().wcc_joint_topk(self._h, C.byref(desc), _ptr(coef), _ptr(norm), _ptr(idx),
                                    _stream()), "wcc_joint_topk")

    def wcc_gather_quant(self, desc, coef, idx, alpha_in, xc, alpha_dev):
        _check(lib().wcc_gather_quant(self._h, C.byref(desc), _ptr(coef), _ptr(idx),
                                      C.c_float(alpha_in), _ptr(xc), _ptr(alpha_dev), _stream()),
               "wcc_gather_quant")

    def wcc_pointwise(self, desc, w, w_scale, xc, alpha_dev, yc):
        _check(lib().wcc_pointwise(self._h, C.byref(desc), _ptr(w), _ptr(w_scale), _ptr(xc),
                                   _ptr(alpha_dev), _ptr(yc), _stream()), "wcc_pointwise")

    def wcc_scatter_ihaar(self, desc, yc, idx, y):
        _check(lib().wcc_scatter_ihaar(self._h, C.byref(desc), _ptr(yc), _ptr(idx), _ptr(y),
                                       _stream()), "wcc_scatter_ihaar")

    def wcc_forward(self, desc, x, w, w_scale, alpha_in, y, idx_out=None, alpha_out=None):
        _check(lib().wcc_forward(self._h, C.byref(desc), _ptr(x), _ptr(w), _ptr(w_scale),
                                 C.c_float(alpha_in), _ptr(y), _ptr(idx_out), _ptr(alpha_out),
                                 _stream()), "wcc_forward")

    def wcc_forward_static(self, desc, x, w, w_scale, alpha_in, y, idx_out=None, alpha_out=None):
        _check(lib().wcc_forward_static(self._h, C.byref(desc), _ptr(x), _ptr(w), _ptr(w_scale),
                                        C.c_float(alpha_in), _ptr(y), _ptr(idx_out), _ptr(alpha_out),
                                        _stream()), "wcc_forward_static")

    def wcc_forward_fixed(self, desc, x, w, w_scale, alpha_in, idx, y, alpha_out=None):
        _check(lib().wcc_forward_fixed(self._h, C.byref(desc), _ptr(x), _ptr(w), _ptr(w_scale),
                                       C.c_float(alpha_in), _ptr(idx), _ptr(y), _ptr(alpha_out),
                                       _stream()), "wcc_forward_fixed")

    # ---- the inverted residual block (next row) ----
    def wcc_depthwise3x3(self, x, w, y):
        B, Cc, H, W = x.shape
        _check(lib().wcc_depthwise3x3(self._h, B, Cc, H, W, _ptr(x), _ptr(w), _ptr(y), _stream()),
               "wcc_depthwise3x3")

    def wcc_block_forward(self, desc, x, w1, w1_scale, w_dw, w3, w3_scale, y, t1_out=None,
                          t2_out=None, idx1_out=None, idx3_out=None):
        _check(lib().wcc_block_forward(self._h, C.byref(desc), _ptr(x), _ptr(w1), _ptr(w1_scale),
                                       _ptr(w_dw), _ptr(w3), _ptr(w3_scale), _ptr(y), _ptr(t1_out),
                                       _ptr(t2_out), _ptr(idx1_out), _ptr(idx3_out), _stream()),
               "wcc_block_forward")

    def set_block_profile_layer(self, layer: int) -> None:
        _check(lib().wcc_set_block_profile_layer(self._h, int(layer)), "wcc_set_block_profile_layer")

    # ---- the head of a model, on rows of tokens ----
    def wcc_adapter_forward(self, desc, x, w, adapter_of_row, a, b, ranks, scale, y):
        d, t = desc, _TORCH[desc.dtype]
        _check(lib().wcc_adapter_forward(
            self._h, C.byref(d), _rows(x, d.rows, d.C_in, d.ldx, d.dtype), _whole(w, (d.C_out, d.C_in), t),
            _whole(adapter_of_row, (d.rows,), torch.int32), _whole(a, (d.adapters, d.rank, d.C_in), t),
            _whole(b, (d.adapters, d.C_out, d.rank), t), _whole(ranks, (d.adapters,), torch.int32),
            _whole(scale, (d.adapters,), torch.float32), _rows(y, d.rows, d.C_out, d.ldy, d.dtype), _stream()), "wcc_adapter_forward")

    def wcc_adapter_backward(self, desc, x, w, adapter_of_row, a, b, ranks, scale, dy, dx=None, da=None, db=None):
        d, t = desc, _TORCH[desc.dtype]
        _check(lib().wcc_adapter_backward(
            self._h, C.byref(d), _rows(x, d.rows, d.C_in, d.ldx, d.dtype), _whole(w, (d.C_out, d.C_in), t),
            _whole(adapter_of_row, (d.rows,), torch.int32), _whole(a, (d.adapters, d.rank, d.C_in), t),
            _whole(b, (d.adapters, d.C_out, d.rank), t), _whole(ranks, (d.adapters,), torch.int32),
            _whole(scale, (d.adapters,), torch.float32), _rows(dy, d.rows, d.C_out, d.ldy, d.dtype),
            _rows(dx, d.rows, d.C_in, d.ldx, d.dtype), _whole(da, (d.adapters, d.rank, d.C_in), torch.float32),
            _whole(db, (d.adapters, d.C_out, d.rank), torch.float32), _stream()), "wcc_adapter_backward")

    def wcc_token_scores(self, desc, logits, tokens=None, logprob=None, entropy=None, top_idx=None, top_logprob=None):
        d, f = desc, torch.float32
        _check(lib().wcc_token_scores(
            self._h, C.byref(d), _rows(logits, d.rows, d.V, d.ld, d.dtype), _whole(tokens, (d.rows,), torch.int32),
            _whole(logprob, (d.rows,), f), _whole(entropy, (d.rows,), f), _whole(top_idx, (d.rows, d.top), torch.int32),
            _whole(top_logprob, (d.rows, d.top), f), _stream()), "wcc_token_scores")

    def wcc_distill_forward(self, desc, logits, t_idx, t_logit, loss, stats=None, weight=None, dlogits=None):
        d, f = desc, torch.float32
        _check(lib().wcc_distill_forward(
            self._h, C.byref(d), _rows(logits, d.rows, d.V, d.ld, d.dtype), _whole(t_idx, (d.rows, d.K), torch.int32),
            _whole(t_logit, (d.rows, d.K), _TORCH[d.t_dtype]), _whole(loss, (d.rows,), f), _whole(stats, (d.rows, 2), f),
            _whole(weight, (d.rows,), f), _rows(dlogits, d.rows, d.V, d.ld_grad, d.dtype), _stream()), "wcc_distill_forward")

    def wcc_distill_backward(self, desc, logits, t_idx, t_logit, stats, weight, dlogits):
        d, f = desc, torch.float32
        _check(lib().wcc_distill_backward(
            self._h, C.byref(d), _rows(logits, d.rows, d.V, d.ld, d.dtype), _whole(t_idx, (d.rows, d.K), torch.int32),
            _whole(t_logit, (d.rows, d.K), _TORCH[d.t_dtype]), _whole(stats, (d.rows, 2), f), _whole(weight, (d.rows,), f),
            _rows(dlogits, d.rows, d.V, d.ld_grad, d.dtype), _stream()), "wcc_distill_backward")

    # ---- a block on rows ----
    def _own_stream(self):
        device = _current_device()
        assert device == self.device, "the current device is not the context's"
        return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(device)

    def wcc_rows_keep(self, desc, x, codes, steps):
        d, dev = desc, self.device
        _check(lib().wcc_rows_keep(self._h, C.byref(d), _rows(x, d.rows, d.width, d.ld, d.dtype, dev),
                                   *_kept(codes, steps, (d.rows,), d.width, dev), self._own_stream()), "wcc_rows_keep")

    def wcc_rows_restore(self, desc, codes, steps, x):
        d, dev = desc, self.device
        _check(lib().wcc_rows_restore(self._h, C.byref(d), *_kept(codes, steps, (d.rows,), d.width, dev),
                                      _rows(x, d.rows, d.width, d.ld, d.dtype, dev), self._own_stream()), "wcc_rows_restore")

    def wcc_group_norm_forward(self, desc, x, gamma, beta, counts, y, stats=None, codes=None, steps=None):
        d, dev, f, rows = desc, self.device, torch.float32, desc.samples * desc.pixels
        _check(lib().wcc_group_norm_forward(
            self._h, C.byref(d), _rows(x, rows, d.C, d.ldx, d.dtype, dev), _whole(gamma, (d.C,), f, dev), _whole(beta, (d.C,), f, dev),
            _whole(counts, (d.samples,), torch.int32, dev), _rows(y, rows, d.C, d.ldy, d.dtype, dev),
            _whole(stats, (d.samples, d.groups, 2), f, dev), *_kept(codes, steps, (rows,), d.C, dev), self._own_stream()), "wcc_group_norm_forward")

    def wcc_group_norm_backward(self, desc, x, codes, steps, gamma, beta, counts, stats, dy, dx=None, dgamma=None, dbeta=None):
        d, dev, f, rows = desc, self.device, torch.float32, desc.samples * desc.pixels
        _check(lib().wcc_group_norm_backward(
            self._h, C.byref(d), _rows(x, rows, d.C, d.ldx, d.dtype, dev), *_kept(codes, steps, (rows,), d.C, dev), _whole(gamma, (d.C,), f, dev),
            _whole(beta, (d.C,), f, dev), _whole(counts, (d.samples,), torch.int32, dev), _whole(stats, (d.samples, d.groups, 2), f, dev),
            _rows(dy, rows, d.C, d.ldy, d.dtype, dev), _rows(dx, rows, d.C, d.ldx, d.dtype, dev), _whole(dgamma, (d.C,), f, dev),
            _whole(dbeta, (d.C,), f, dev), self._own_stream()), "wcc_group_norm_backward")

    def wcc_gated_forward(self, desc, x, w_gate, w_up, y, codes=None, steps=None):
        d, dev, t = desc, self.device, _TORCH[desc.dtype]
        _check(lib().wcc_gated_forward(
            self._h, C.byref(d), _rows(x, d.rows, d.C_in, d.ldx, d.dtype, dev), _whole(w_gate, (d.C_out, d.C_in), t, dev),
            _whole(w_up, (d.C_out, d.C_in), t, dev), _rows(y, d.rows, d.C_out, d.ldy, d.dtype, dev),
            *_kept(codes, steps, (2, d.rows), d.C_out, dev), self._own_stream()), "wcc_gated_forward")

    def wcc_gated_backward(self, desc, x, x_codes, x_steps, w_gate, w_up, codes, steps, dy, dx=None, dw_gate=None, dw_up=None):
        d, dev, t = desc, self.device, _TORCH[desc.dtype]
        _check(lib().wcc_gated_backward(
            self._h, C.byref(d), _rows(x, d.rows, d.C_in, d.ldx, d.dtype, dev), *_kept(x_codes, x_steps, (d.rows,), d.C_in, dev),
            _whole(w_gate, (d.C_out, d.C_in), t, dev), _whole(w_up, (d.C_out, d.C_in), t, dev), *_kept(codes, steps, (2, d.rows), d.C_out, dev),
            _rows(dy, d.rows, d.C_out, d.ldy, d.dtype, dev), _rows(dx, d.rows, d.C_in, d.ldx, d.dtype, dev),
            _whole(dw_gate, (d.C_out, d.C_in), t, dev), _whole(dw_up, (d.C_out, d.C_in), t, dev), self._own_stream()), "wcc_gated_backward")
