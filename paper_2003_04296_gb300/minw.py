"""ctypes binding of libminw.so (include/minw.h).

Argument marshalling only: every function passes device pointers, sizes and
the current CUDA stream to the C entry point of the same name and raises on a
non-OK status.  Every step of the computation runs in the library's CUDA
kernels; there is no fallback of any kind.  torch provides device memory and
streams.
"""
import ctypes
import math
import os

import torch

from . import build as _build

_LIB = None

MINW_OK, MINW_EINVAL, MINW_EUNSUPPORTED, MINW_ECUDA, MINW_ETIMEOUT, MINW_EDEVICE = range(6)
VARIANT_AUTO, VARIANT_POPC, VARIANT_TC, VARIANT_TC_E4M3, VARIANT_TC_E2M1, VARIANT_TC_E2M1_PAIRS = 0, 1, 2, 3, 4, 5
VARIANT_TC_E2M1_N128 = 6
CODES_E4M3, CODES_E2M1 = 0, 1
LAYER_CONV, LAYER_FC = 0, 1
F32, BF16 = 0, 1
ACT_NONE, ACT_HARDTANH, ACT_RELU, ACT_SILU = range(4)


class MinwError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class Quant(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("thr", ctypes.c_float * 3), ("scale", ctypes.c_float)]


class BlockExtra(ctypes.Structure):
    _fields_ = [("res_codes", ctypes.c_void_p), ("res_bits", ctypes.c_int32), ("res_f32", ctypes.c_void_p),
                ("y_nhwc", ctypes.c_void_p), ("in_format", ctypes.c_int32), ("out_format", ctypes.c_int32),
                ("res_format", ctypes.c_int32), ("acc_out", ctypes.c_void_p), ("e2m1_pairs", ctypes.c_int32)]


class PlanOptions(ctypes.Structure):
    _fields_ = [("cta_pairs", ctypes.c_int32), ("channel_major", ctypes.c_int32),
                ("channel_major_min_tiles_per_sm", ctypes.c_int32), ("dup_weights", ctypes.c_int32),
                ("kblocks_per_stage", ctypes.c_int32), ("first_tma", ctypes.c_int32), ("pdl", ctypes.c_int32),
                ("graph", ctypes.c_int32), ("tma_lanes", ctypes.c_int32),
                ("resident_weights", ctypes.c_int32), ("first_tensor_cores", ctypes.c_int32),
                ("wait_cycles", ctypes.c_int64)]


STALL_CONV_TC, STALL_CONV_FIRST = 1, 2


class PipeRates(ctypes.Structure):
    _fields_ = [("sm_clock_mhz", ctypes.c_double), ("popc_per_s", ctypes.c_double),
                ("bmma_b1_mac_per_s", ctypes.c_double), ("imma_s8_mac_per_s", ctypes.c_double),
                ("tc_e4m3_flop_per_s", ctypes.c_double * 2), ("tc_e2m1_flop_per_s", ctypes.c_double * 2),
                ("tc_bf16_flop_per_s", ctypes.c_double * 2), ("tma_box_cycles", ctypes.c_double)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("type", ctypes.c_int32), ("limit", ctypes.c_float)]


class Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("rows", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("type", ctypes.c_int32), ("limit", ctypes.c_float)]


class LayerDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("C", ctypes.c_int32), ("H", ctypes.c_int32),
                ("W", ctypes.c_int32), ("O", ctypes.c_int32), ("kh", ctypes.c_int32),
                ("kw", ctypes.c_int32), ("stride", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("pool", ctypes.c_int32), ("bits_in", ctypes.c_int32), ("bits_w", ctypes.c_int32),
                ("bits_out", ctypes.c_int32), ("thr_w", ctypes.c_float * 3),
                ("thr_out", ctypes.c_float * 3), ("w", ctypes.c_void_p), ("w_scale", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("shift", ctypes.c_void_p), ("variant", ctypes.c_int32)]


WRESNET_MAX_N = 18
_NB = 3 * WRESNET_MAX_N


class WResNetDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("bits_w", ctypes.c_int32), ("thr_w", ctypes.c_float * 3),
                ("image_hw", ctypes.c_int32), ("num_classes", ctypes.c_int32),
                ("stem_w", ctypes.c_void_p), ("stem_scale", ctypes.c_void_p), ("stem_shift", ctypes.c_void_p),
                ("c1_w", ctypes.c_void_p * _NB), ("c1_wscale", ctypes.c_void_p * _NB),
                ("c1_scale", ctypes.c_void_p * _NB), ("c1_shift", ctypes.c_void_p * _NB),
                ("c2_w", ctypes.c_void_p * _NB), ("c2_wscale", ctypes.c_void_p * _NB),
                ("c2_scale", ctypes.c_void_p * _NB), ("c2_shift", ctypes.c_void_p * _NB),
                ("down_w", ctypes.c_void_p * 2), ("down_wscale", ctypes.c_void_p * 2),
                ("down_scale", ctypes.c_void_p * 2), ("down_shift", ctypes.c_void_p * 2),
                ("fc_w", ctypes.c_void_p), ("fc_scale", ctypes.c_void_p), ("fc_shift", ctypes.c_void_p),
                ("keep_activations", ctypes.c_int32)]


WDENSE_MAX_LAYERS = 32
_NL = 3 * WDENSE_MAX_LAYERS


class WDenseDesc(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("growth", ctypes.c_int32), ("bits_w", ctypes.c_int32),
                ("thr_w", ctypes.c_float * 3), ("image_hw", ctypes.c_int32), ("num_classes", ctypes.c_int32),
                ("stem_w", ctypes.c_void_p), ("stem_scale", ctypes.c_void_p), ("stem_shift", ctypes.c_void_p),
                ("b_w", ctypes.c_void_p * _NL), ("b_wscale", ctypes.c_void_p * _NL),
                ("b_scale", ctypes.c_void_p * _NL), ("b_shift", ctypes.c_void_p * _NL),
                ("c_w", ctypes.c_void_p * _NL), ("c_wscale", ctypes.c_void_p * _NL),
                ("c_scale", ctypes.c_void_p * _NL), ("c_shift", ctypes.c_void_p * _NL),
                ("t_w", ctypes.c_void_p * 2), ("t_wscale", ctypes.c_void_p * 2),
                ("t_scale", ctypes.c_void_p * 2), ("t_shift", ctypes.c_void_p * 2),
                ("fc_w", ctypes.c_void_p), ("fc_scale", ctypes.c_void_p), ("fc_shift", ctypes.c_void_p)]


class ResNet18Desc(ctypes.Structure):
    _fields_ = [("bits_a", ctypes.c_int32), ("bits_w", ctypes.c_int32), ("thr_a", ctypes.c_float * 3),
                ("thr_w", ctypes.c_float * 3), ("image_hw", ctypes.c_int32), ("num_classes", ctypes.c_int32),
                ("stem_w", ctypes.c_void_p), ("stem_scale", ctypes.c_void_p), ("stem_shift", ctypes.c_void_p),
                ("conv_w", ctypes.c_void_p * 16), ("conv_wscale", ctypes.c_void_p * 16),
                ("conv_scale", ctypes.c_void_p * 16), ("conv_shift", ctypes.c_void_p * 16),
                ("down_w", ctypes.c_void_p * 3), ("down_wscale", ctypes.c_void_p * 3),
                ("down_scale", ctypes.c_void_p * 3), ("down_shift", ctypes.c_void_p * 3),
                ("fc_w", ctypes.c_void_p), ("fc_scale", ctypes.c_void_p), ("fc_shift", ctypes.c_void_p)]


# name -> (restype, argtypes)
_P, _I32, _I64, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_QP = ctypes.POINTER(Quant)
SIGNATURES = {
    "minw_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "minw_version": (_I32, []),
    "aqe_forward": (ctypes.c_int, [_P, _P, _I64, _F, _QP, _P]),
    "aqe_backward": (ctypes.c_int, [_P, _P, _P, _I64, _F, _P]),
    "aqe_forward_stochastic": (ctypes.c_int, [_P, _P, _I64, _F, ctypes.c_uint64, ctypes.c_uint64, _P]),
    "minw_to_bf16_nhwc": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _P, _P]),
    "minw_to_bf16_nhwc_pad": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _P, _P]),
    "minw_pack_weight_bf16_pad": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _QP, _P, _P, _P]),
    "minw_pack_weight_bf16": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _P, _P]),
    "minw_conv2d_bf16": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32, _I32, _I32,
                                        _I32, _P, _P, _P, _P]),
    "minw_conv2d_bf16_hardtanh": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32, _I32,
                                                 _I32, _P, _P, _P, _I32, _I32, _P, _P, _P]),
    "minw_bf16_matrix": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _P, _P]),
    "minw_sgd_clip": (ctypes.c_int, [_P, _P, _I64, _F, _P]),
    "minw_fc_train_workspace_bytes": (ctypes.c_size_t, [_I32, _I32, _I32]),
    "minw_conv_train_workspace_bytes": (ctypes.c_size_t, [_I32] * 9),
    "minw_conv_train_step": (ctypes.c_int, [_P, _P, _P] + [_I32] * 9 + [_F, _F, _QP, _QP, _P, _P, _P, _P,
                                            ctypes.c_size_t, _P]),
    "minw_fc_train_step": (ctypes.c_int, [_P, _P, _P, _I32, _I32, _I32, _F, _F, _QP, _QP, _P, _P, _P, _P,
                                          ctypes.c_size_t, _P]),
    "aqe_quantize_pack": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _F, _P, _P, _P]),
    "aqe_backward_masked": (ctypes.c_int, [_P, _P, _P, _I64, _F, _P]),
    "minw_pack_weights": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _P, _P]),
    "minw_conv2d": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32,
                                   _I32, _I32, _P, _P, _P, _P, _I32, _P]),
    "minw_conv_block": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32,
                                       _I32, _I32, _I32, _P, _P, _QP, _P, _P, _I32, _P]),
    "minw_conv_first": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32, _I32,
                                       _QP, _P, _I32, _P, _P, _QP, _P, _P, _P]),
    "aqe_quantize_codes": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _P]),
    "minw_pack_weight_codes": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _P, _P]),
    "aqe_quantize_codes_e2m1": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _P]),
    "minw_pack_weight_codes_e2m1": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _P, _P]),
    "minw_conv2d_codes": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32,
                                         _I32, _I32, _P, _P, _P, _P, _P]),
    "minw_conv_block_codes": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32,
                                             _I32, _I32, _I32, _P, _P, _QP, _P, _P, _P, _P]),
    "minw_conv_block_codes_ex": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _I32, _P, _I32, _I32, _I32, _I32,
                                                _I32, _I32, _I32, _P, _P, _QP, _P, _P, _P,
                                                ctypes.POINTER(BlockExtra), _P]),
    "minw_fc_workspace_bytes": (ctypes.c_size_t, [_I32, _I32, _I32]),
    "minw_fc_ksplit": (_I32, [_I32, _I32, _I32, ctypes.c_size_t]),
    "minw_get_plan_options": (ctypes.c_int, [ctypes.POINTER(PlanOptions)]),
    "minw_set_plan_options": (ctypes.c_int, [ctypes.POINTER(PlanOptions)]),
    "minw_test_stall_next_launch": (ctypes.c_int, [_I32]),
    "minw_measure_pipe_rates": (ctypes.c_int, [ctypes.POINTER(PipeRates), _P]),
    "minw_fc_codes": (ctypes.c_int, [_P, _I32, _I32, _I32, _P, _I32, _I32, _P, _P, _QP, _P, _P, _P, _P, _P,
                                     ctypes.c_size_t, _P]),
    "minw_fc_codes_noalloc": (ctypes.c_int, [_P, _I32, _I32, _I32, _P, _I32, _I32, _P, _P, _QP, _P, _P, _P, _P,
                                             _P]),
    "minw_group_norm_workspace_bytes": (ctypes.c_size_t, [_I32, _I64, _I32, _I32, _I32]),
    "minw_group_norm": (ctypes.c_int, [_P, _I32, _I64, _P, _P, _I32, _I64, _I32, _I32, _F, _I32, _P, _I32, _I64, _P, _P,
                                       _P, ctypes.c_size_t, _P]),
    "minw_group_norm_backward": (ctypes.c_int, [_P, _I32, _I64, _P, _I32, _I64, _P, _P, _P, _P, _I32, _I64, _I32, _I32,
                                                _I32, _P, _I64, _P, _P, _P, ctypes.c_size_t, _P]),
    "minw_grad_workspace_bytes": (ctypes.c_size_t, [_I32]),
    "minw_grad_norm": (ctypes.c_int, [_P, _I32, _P, _P, ctypes.c_size_t, _P]),
    "minw_grad_clip": (ctypes.c_int, [_P, _P, _I32, _F, _P, _P, ctypes.c_size_t, _P]),
    "minw_sgd_clip_norm": (ctypes.c_int, [_P, _P, _I32, _F, _F, _P, _P, ctypes.c_size_t, _P]),
    "minw_orthogonal_workspace_bytes": (ctypes.c_size_t, [_P, _I32]),
    "minw_orthogonalize": (ctypes.c_int, [_P, _P, _I32, _I32, _P, ctypes.c_size_t, _P]),
    "minw_sgd_orthogonal": (ctypes.c_int, [_P, _P, _P, _I32, _I32, _F, _I32, _F, _P, ctypes.c_size_t, _P]),
    "minw_adapters_workspace_bytes": (ctypes.c_size_t, [_I64, _I32, _I32, _I32, _I32, _I32]),
    "minw_adapters": (ctypes.c_int, [_P, _I32, _I64, _I64, _I32, _P, _P, _P, _I32, _I32, _I32, _P, _P, _I32, _I64, _I32,
                                     _P, _P, _I32, _P, _I32, _I64, _P, _P, ctypes.c_size_t, _P]),
    "minw_w4_adapters": (ctypes.c_int, [_P, _I32, _I64, _I64, _P, _P, _I32, _I32, _I32, _P, _P, _P, _I32, _I32, _I32, _P,
                                        _P, _P, _I32, _P, _I32, _I64, _P, ctypes.c_size_t, _P]),
    "minw_adapters_backward": (ctypes.c_int, [_P, _I32, _I64, _I64, _I32, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _I32,
                                              _I64, _I32, _P, _I64, _I32, _P, _P, _P, ctypes.c_size_t, _P]),
    "minw_pack_w4": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _QP, _P, _P, _P, _P]),
    "minw_w4_matvec": (ctypes.c_int, [_P, _I32, _I64, _I32, _P, _P, _I32, _I32, _I32, _P, _P, _I32, _P, _I32, _I64,
                                      _P]),
    "minw_net_create": (ctypes.c_int, [ctypes.POINTER(LayerDesc), _I32, _I32, _I32, _P,
                                       ctypes.POINTER(ctypes.c_void_p)]),
    "minw_resnet18_create": (ctypes.c_int, [ctypes.POINTER(ResNet18Desc), _I32, _P,
                                            ctypes.POINTER(ctypes.c_void_p)]),
    "minw_wresnet_create": (ctypes.c_int, [ctypes.POINTER(WResNetDesc), _I32, _P,
                                           ctypes.POINTER(ctypes.c_void_p)]),
    "minw_wresnet_activation": (ctypes.c_int, [_P, _I32, _P, ctypes.c_size_t, _P]),
    "minw_wdense_create": (ctypes.c_int, [ctypes.POINTER(WDenseDesc), _I32, _P, ctypes.POINTER(ctypes.c_void_p)]),
    "minw_wdense_features": (ctypes.c_int, [_P, _I32, _P, ctypes.c_size_t, ctypes.POINTER(ctypes.c_int32),
                                            ctypes.POINTER(ctypes.c_int32), _P]),
    "minw_forward": (ctypes.c_int, [_P, _P, _I32, _P, _P]),
    "minw_forward_host": (ctypes.c_int, [_P, _P, _I32, _P, _P]),
    "minw_net_enable_timing": (ctypes.c_int, [_P, _I32]),
    "minw_net_layer_times": (ctypes.c_int, [_P, _P]),
    "minw_net_layer_variants": (ctypes.c_int, [_P, _P]),
    "minw_net_layer_candidates": (ctypes.c_int, [_P, ctypes.c_int32, _P]),
    "minw_net_launches": (_I32, [_P]),
    "minw_net_kernels": (_I32, [_P]),
    "minw_net_destroy": (None, [_P]),
    "minw_get_last_device_error": (ctypes.c_int, [_P]),
}


def library_path():
    return _build.LIB


def lib(build_if_missing=False):
    """Load libminw.so.  Raises if it is missing: there is no other path."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            if not build_if_missing:
                raise RuntimeError(f"libminw.so not built ({path}); run __graft_entry__.build()")
            _build.build()
        L = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _LIB = L
    return _LIB


def status_string(s):
    return lib().minw_status_string(int(s)).decode()


def _check(status, where):
    if status != MINW_OK:
        raise MinwError(status, where)


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return ctypes.c_void_p(t.data_ptr())


def _host_ptr(a):
    if isinstance(a, torch.Tensor):
        if a.is_cuda or not a.is_contiguous():
            raise ValueError("contiguous host tensor expected")
        return a.data_ptr()
    if not a.flags["C_CONTIGUOUS"]:
        raise ValueError("contiguous host array expected")
    return a.ctypes.data


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    # the current stream's handle without a Stream object around it (3 us of a call's host time), where torch has these
    # functions: they are no part of its interface
    if torch.cuda.is_initialized():
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


_VALUE_TYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _value_type(t):
    try:
        return _VALUE_TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"float32 or bfloat16 expected, got {t.dtype}") from None


def _addr(t):
    """_ptr as a plain number (the calls on small tensors are bound by the host)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return t.data_ptr()


def _rows(t):
    """(address, row length) of a channels-last tensor [..., C] whose rows lie a fixed number of elements apart (the
    first C channels of a wider buffer, for instance)."""
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if t.is_contiguous():
        return t.data_ptr(), t.size(-1)
    size, stride = t.shape, t.stride()
    if size[-1] != 1 and stride[-1] != 1:
        raise ValueError("the last dimension has to be contiguous")
    ld, inner = None, 1                   # row length, rows inside the dimension
    for n, st in zip(reversed(size[:-1]), reversed(stride[:-1])):
        if n == 1:
            continue
        if ld is None:
            if st < size[-1]:
                raise ValueError("rows overlap")
            ld = st
        elif st != ld * inner:
            raise ValueError("rows a fixed number of elements apart expected")
        inner *= n
    return t.data_ptr(), size[-1] if ld is None else ld


_FLOAT = torch.float32


def _f32(t, n, what):
    """Address of a dense fp32 vector of n values (None passes)."""
    if t is None:
        return None
    if t.dtype is not _FLOAT or t.numel() != n:
        raise ValueError(f"{what}: {n} float32 values expected")
    return _addr(t)


def _scratch(workspace):
    return (None, 0) if workspace is None else (_addr(workspace), workspace.nbytes)


def quant(bits, thr=(0.0, 0.0, 0.0), scale=1.0):
    q = Quant()
    q.bits = int(bits)
    t = list(thr) + [0.0] * (3 - len(thr))
    for i in range(3):
        q.thr[i] = float(t[i])
    q.scale = float(scale)
    return q


def packed_words(N, C, H, W, bits):
    return N * H * W * bits * ((C + 31) // 32)


# ---------------------------------------------------------------------------
# entry points (same names as the C ABI)
# ---------------------------------------------------------------------------

def aqe_forward(x, y, alpha, q, stream=None):
    _check(lib().aqe_forward(_ptr(x), _ptr(y), x.numel(), float(alpha), ctypes.byref(q), _stream(stream)),
           "aqe_forward")


def aqe_forward_stochastic(x, y, alpha, seed, offset=0, stream=None):
    """Eq. our: alpha sign(x - z) + (1 - alpha) x, z ~ U[-1, 1) from
    Philox4x64-10 keyed by seed; offset advances the counter (ceil(n / 8) per
    call for fresh noise)."""
    _check(lib().aqe_forward_stochastic(_ptr(x), _ptr(y), x.numel(), float(alpha), int(seed) & (2**64 - 1),
                                        int(offset) & (2**64 - 1), _stream(stream)), "aqe_forward_stochastic")


def minw_to_bf16_nhwc(x, out, stream=None):
    """fp32 NCHW -> bf16 NHWC (out: a uint16 or bfloat16 tensor [B][H][W][C])."""
    B, C, H, W = x.shape
    _check(lib().minw_to_bf16_nhwc(_ptr(x), B, C, H, W, _ptr(out), _stream(stream)), "minw_to_bf16_nhwc")


def minw_pack_weight_bf16(w, q, out, channel_scale=None, stream=None):
    """Latent weights [O][C][kh][kw] -> bf16 level values [O][kh][kw][C]."""
    O, C, kh, kw = w.shape
    _check(lib().minw_pack_weight_bf16(_ptr(w), O, C, kh, kw, ctypes.byref(q), _ptr(channel_scale), _ptr(out),
                                       _stream(stream)), "minw_pack_weight_bf16")


def minw_to_bf16_nhwc_pad(x, Cp, out, stream=None):
    """fp32 NCHW -> bf16 NHWC with the channels padded to Cp (zeros) (out [B][H][W][Cp])."""
    B, C, H, W = x.shape
    _check(lib().minw_to_bf16_nhwc_pad(_ptr(x), B, C, H, W, int(Cp), _ptr(out), _stream(stream)),
           "minw_to_bf16_nhwc_pad")


def minw_pack_weight_bf16_pad(w, Cp, q, out, channel_scale=None, stream=None):
    """Latent weights [O][C][kh][kw] -> bf16 level values [O][kh][kw][Cp], channels past C zero."""
    O, C, kh, kw = w.shape
    _check(lib().minw_pack_weight_bf16_pad(_ptr(w), O, C, kh, kw, int(Cp), ctypes.byref(q), _ptr(channel_scale),
                                           _ptr(out), _stream(stream)), "minw_pack_weight_bf16_pad")


def minw_conv2d_bf16(act, B, C, H, W, wgt, O, kh, kw, bits_w, stride, pad, pool, scale, shift, y_out, stream=None):
    _check(lib().minw_conv2d_bf16(_ptr(act), B, C, H, W, _ptr(wgt), O, kh, kw, bits_w, stride, pad, int(pool),
                                  _ptr(scale), _ptr(shift), _ptr(y_out), _stream(stream)), "minw_conv2d_bf16")


def minw_conv2d_bf16_hardtanh(act, B, C, H, W, ldc, wgt, O, kh, kw, bits_w, stride, pad, scale, shift, out,
                              out_ld, out_off, residual=None, y_out=None, stream=None):
    _check(lib().minw_conv2d_bf16_hardtanh(_ptr(act), B, C, H, W, int(ldc), _ptr(wgt), O, kh, kw, bits_w, stride,
                                           pad, _ptr(scale), _ptr(shift), _ptr(out), int(out_ld), int(out_off),
                                           _ptr(residual), _ptr(y_out), _stream(stream)),
           "minw_conv2d_bf16_hardtanh")


def minw_bf16_matrix(x, out, transpose=False, stream=None):
    """fp32 matrix [rows][cols] -> bf16 (int16 bit patterns), transposed when asked,
    zero-padded to out's column count."""
    rows, cols = x.shape
    _check(lib().minw_bf16_matrix(_ptr(x), rows, cols, int(bool(transpose)), out.shape[1], _ptr(out),
                                  _stream(stream)), "minw_bf16_matrix")


def minw_sgd_clip(w, g, lr, stream=None):
    _check(lib().minw_sgd_clip(_ptr(w), _ptr(g), w.numel(), float(lr), _stream(stream)), "minw_sgd_clip")


def minw_fc_train_workspace_bytes(B, K, O):
    return int(lib().minw_fc_train_workspace_bytes(B, K, O))


def minw_fc_train_step(A, W, g_out, alpha, lr, q_w, q_a, a_out, g_in, workspace, a_pre=None, stream=None):
    """One Algorithm 1 step of a fully connected layer (W updated in place;
    a_pre, when given, receives the product before the activation AQE)."""
    B, K = A.shape
    O = W.shape[0]
    nbytes = workspace.numel() * workspace.element_size()
    _check(lib().minw_fc_train_step(_ptr(A), _ptr(W), _ptr(g_out), B, K, O, float(alpha), float(lr),
                                    ctypes.byref(q_w), ctypes.byref(q_a) if q_a is not None else None,
                                    _ptr(a_out), _ptr(g_in), _ptr(a_pre), _ptr(workspace), nbytes,
                                    _stream(stream)),
           "minw_fc_train_step")


def minw_conv_train_workspace_bytes(B, C, H, W, O, kh, kw, stride, pad):
    return int(lib().minw_conv_train_workspace_bytes(B, C, H, W, O, kh, kw, stride, pad))


def minw_conv_train_step(A, W, g_out, stride, pad, alpha, lr, q_w, q_a, a_out, g_in, workspace, a_pre=None,
                         stream=None):
    """One Algorithm 1 step of a convolutional layer: A [B][C][H][W], W
    [O][C][kh][kw] (updated in place), g_out [B][O][Ho][Wo]; a_pre, when
    given, receives the convolution before the activation AQE."""
    B, C, H, Wd = A.shape
    O, _, kh, kw = W.shape
    nbytes = workspace.numel() * workspace.element_size()
    _check(lib().minw_conv_train_step(_ptr(A), _ptr(W), _ptr(g_out), B, C, H, Wd, O, kh, kw, int(stride), int(pad),
                                      float(alpha), float(lr), ctypes.byref(q_w),
                                      ctypes.byref(q_a) if q_a is not None else None, _ptr(a_out), _ptr(g_in),
                                      _ptr(a_pre), _ptr(workspace), nbytes, _stream(stream)),
           "minw_conv_train_step")


def aqe_backward(x, gy, gx, alpha, stream=None):
    _check(lib().aqe_backward(_ptr(x), _ptr(gy), _ptr(gx), x.numel(), float(alpha), _stream(stream)),
           "aqe_backward")


def aqe_quantize_pack(x, q, planes, alpha=1.0, y=None, mask=None, stream=None):
    B, C, H, W = x.shape
    _check(lib().aqe_quantize_pack(_ptr(x), B, C, H, W, ctypes.byref(q), _ptr(planes), float(alpha),
                                   _ptr(y), _ptr(mask), _stream(stream)), "aqe_quantize_pack")


def aqe_backward_masked(mask, gy, gx, alpha, stream=None):
    _check(lib().aqe_backward_masked(_ptr(mask), _ptr(gy), _ptr(gx), gy.numel(), float(alpha),
                                     _stream(stream)), "aqe_backward_masked")


def minw_pack_weights(w, q, planes, channel_scale=None, stream=None):
    O, C, kh, kw = w.shape
    _check(lib().minw_pack_weights(_ptr(w), O, C, kh, kw, ctypes.byref(q), _ptr(channel_scale),
                                   _ptr(planes), _stream(stream)), "minw_pack_weights")


def minw_conv2d(act, B, C, H, W, bits_a, wgt, O, kh, kw, bits_w, stride, pad, acc_out=None,
                scale=None, shift=None, y_out=None, variant=VARIANT_AUTO, stream=None):
    _check(lib().minw_conv2d(_ptr(act), B, C, H, W, bits_a, _ptr(wgt), O, kh, kw, bits_w, stride, pad,
                             _ptr(acc_out), _ptr(scale), _ptr(shift), _ptr(y_out), int(variant),
                             _stream(stream)), "minw_conv2d")


def minw_conv_block(act, B, C, H, W, bits_a, wgt, O, kh, kw, bits_w, stride, pad, pool, scale, shift,
                    q_out=None, planes_out=None, y_out=None, variant=VARIANT_AUTO, stream=None):
    _check(lib().minw_conv_block(_ptr(act), B, C, H, W, bits_a, _ptr(wgt), O, kh, kw, bits_w, stride,
                                 pad, int(pool), _ptr(scale), _ptr(shift),
                                 ctypes.byref(q_out) if q_out is not None else None,
                                 _ptr(planes_out), _ptr(y_out), int(variant), _stream(stream)),
           "minw_conv_block")


def minw_conv_first(x, w, stride, pad, scale, shift, q_w=None, channel_scale=None, pool=0, q_out=None,
                    planes_out=None, y_out=None, stream=None):
    B, C, H, W = x.shape
    O, _, kh, kw = w.shape
    _check(lib().minw_conv_first(_ptr(x), B, C, H, W, _ptr(w), O, kh, kw, stride, pad,
                                 ctypes.byref(q_w) if q_w is not None else None, _ptr(channel_scale),
                                 int(pool), _ptr(scale), _ptr(shift),
                                 ctypes.byref(q_out) if q_out is not None else None,
                                 _ptr(planes_out), _ptr(y_out), _stream(stream)), "minw_conv_first")


def aqe_quantize_codes(x, q, codes, stream=None):
    B, C, H, W = x.shape
    _check(lib().aqe_quantize_codes(_ptr(x), B, C, H, W, ctypes.byref(q), _ptr(codes), _stream(stream)),
           "aqe_quantize_codes")


def minw_pack_weight_codes(w, q, codes, channel_scale=None, stream=None):
    O, C, kh, kw = w.shape
    _check(lib().minw_pack_weight_codes(_ptr(w), O, C, kh, kw, ctypes.byref(q), _ptr(channel_scale),
                                        _ptr(codes), _stream(stream)), "minw_pack_weight_codes")


def aqe_quantize_codes_e2m1(x, q, codes, stream=None):
    B, C, H, W = x.shape
    _check(lib().aqe_quantize_codes_e2m1(_ptr(x), B, C, H, W, ctypes.byref(q), _ptr(codes), _stream(stream)),
           "aqe_quantize_codes_e2m1")


def minw_pack_weight_codes_e2m1(w, q, codes, channel_scale=None, stream=None):
    O, C, kh, kw = w.shape
    _check(lib().minw_pack_weight_codes_e2m1(_ptr(w), O, C, kh, kw, ctypes.byref(q), _ptr(channel_scale),
                                             _ptr(codes), _stream(stream)), "minw_pack_weight_codes_e2m1")


def minw_conv2d_codes(act, B, C, H, W, bits_a, wgt, O, kh, kw, bits_w, stride, pad, acc_out=None,
                      scale=None, shift=None, y_out=None, stream=None):
    _check(lib().minw_conv2d_codes(_ptr(act), B, C, H, W, bits_a, _ptr(wgt), O, kh, kw, bits_w, stride, pad,
                                   _ptr(acc_out), _ptr(scale), _ptr(shift), _ptr(y_out), _stream(stream)),
           "minw_conv2d_codes")


def minw_conv_block_codes(act, B, C, H, W, bits_a, wgt, O, kh, kw, bits_w, stride, pad, pool, scale, shift,
                          q_out=None, codes_out=None, planes_out=None, y_out=None, stream=None):
    _check(lib().minw_conv_block_codes(_ptr(act), B, C, H, W, bits_a, _ptr(wgt), O, kh, kw, bits_w, stride,
                                       pad, int(pool), _ptr(scale), _ptr(shift),
                                       ctypes.byref(q_out) if q_out is not None else None,
                                       _ptr(codes_out), _ptr(planes_out), _ptr(y_out), _stream(stream)),
           "minw_conv_block_codes")


def minw_conv_block_codes_ex(act, B, C, H, W, bits_a, wgt, O, kh, kw, bits_w, stride, pad, pool, scale, shift,
                             q_out=None, codes_out=None, planes_out=None, y_out=None, res_codes=None, res_bits=0,
                             res_f32=None, y_nhwc=None, in_format=CODES_E4M3, out_format=CODES_E4M3,
                             res_format=CODES_E4M3, acc_out=None, e2m1_pairs=False, stream=None):
    ex = BlockExtra()
    ex.e2m1_pairs = int(bool(e2m1_pairs))
    ex.res_codes = res_codes.data_ptr() if res_codes is not None else None
    ex.res_bits = int(res_bits)
    ex.res_f32 = res_f32.data_ptr() if res_f32 is not None else None
    ex.y_nhwc = y_nhwc.data_ptr() if y_nhwc is not None else None
    ex.in_format, ex.out_format, ex.res_format = int(in_format), int(out_format), int(res_format)
    ex.acc_out = acc_out.data_ptr() if acc_out is not None else None
    _check(lib().minw_conv_block_codes_ex(_ptr(act), B, C, H, W, bits_a, _ptr(wgt), O, kh, kw, bits_w, stride, pad,
                                          int(pool), _ptr(scale), _ptr(shift),
                                          ctypes.byref(q_out) if q_out is not None else None, _ptr(codes_out),
                                          _ptr(planes_out), _ptr(y_out), ctypes.byref(ex), _stream(stream)),
           "minw_conv_block_codes_ex")


def minw_fc_workspace_bytes(B, K, O):
    return int(lib().minw_fc_workspace_bytes(B, K, O))


def minw_fc_ksplit(B, K, O, workspace_bytes):
    """K slices of minw_fc_codes for this shape and workspace size (host query)."""
    return lib().minw_fc_ksplit(int(B), int(K), int(O), int(workspace_bytes))


def minw_fc_codes(act, B, K, bits_a, wgt, O, bits_w, scale=None, shift=None, q_out=None, codes_out=None,
                  planes_out=None, y_out=None, acc_out=None, workspace=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().minw_fc_codes(_ptr(act), B, K, bits_a, _ptr(wgt), O, bits_w, _ptr(scale), _ptr(shift),
                               ctypes.byref(q_out) if q_out is not None else None, _ptr(codes_out),
                               _ptr(planes_out), _ptr(y_out), _ptr(acc_out), _ptr(workspace), nbytes,
                               _stream(stream)), "minw_fc_codes")


def minw_fc_codes_noalloc(act, B, K, bits_a, wgt, O, bits_w, scale=None, shift=None, q_out=None,
                          codes_out=None, planes_out=None, y_out=None, acc_out=None, stream=None):
    """minw_fc_codes with the library's fixed scratch array (allocates nothing)."""
    _check(lib().minw_fc_codes_noalloc(_ptr(act), B, K, bits_a, _ptr(wgt), O, bits_w, _ptr(scale), _ptr(shift),
                                       ctypes.byref(q_out) if q_out is not None else None, _ptr(codes_out),
                                       _ptr(planes_out), _ptr(y_out), _ptr(acc_out), _stream(stream)),
           "minw_fc_codes_noalloc")


def get_plan_options():
    o = PlanOptions()
    _check(lib().minw_get_plan_options(ctypes.byref(o)), "minw_get_plan_options")
    return {name: getattr(o, name) for name, _ in PlanOptions._fields_}


def set_plan_options(opts=None, **changes):
    """minw_set_plan_options: None and no changes restores the defaults;
    otherwise the current options (or opts) updated with changes."""
    if opts is None and not changes:
        _check(lib().minw_set_plan_options(None), "minw_set_plan_options")
        return
    cur = dict(opts if opts is not None else get_plan_options())
    cur.update(changes)
    o = PlanOptions(**cur)
    _check(lib().minw_set_plan_options(ctypes.byref(o)), "minw_set_plan_options")


def minw_measure_pipe_rates(stream=None):
    """minw_measure_pipe_rates as a dict (two-element lists for the N = 128 /
    N = 256 tensor-core rates)."""
    r = PipeRates()
    _check(lib().minw_measure_pipe_rates(ctypes.byref(r), _stream(stream)), "minw_measure_pipe_rates")
    out = {}
    for name, _ in PipeRates._fields_:
        v = getattr(r, name)
        out[name] = list(v) if hasattr(v, "__len__") else float(v)
    return out


def minw_test_stall_next_launch(kernel):
    _check(lib().minw_test_stall_next_launch(int(kernel)), "minw_test_stall_next_launch")


def minw_get_last_device_error(stream=None):
    return lib().minw_get_last_device_error(_stream(stream))


class Net:
    """Owner of a minw_net (minw_net_create / minw_forward / minw_net_destroy).

    ``layers`` is a list of dicts with the minw_layer_desc fields; ``w``,
    ``w_scale``, ``scale`` and ``shift`` are device tensors."""

    @classmethod
    def wresnet(cls, params, max_batch, device, stream=None, keep_activations=False):
        """minw_wresnet_create from a parameter dict shaped like
        ``inputs.wresnet_params`` (latent fp32 weights, BN maps); the tensors
        are copied to ``device`` for the call and released after it."""
        d = WResNetDesc()
        d.keep_activations = int(bool(keep_activations))
        d.n, d.bits_w = params["n"], params["bits_w"]
        for i in range(3):
            d.thr_w[i] = float(params["thr_w"][i])
        d.image_hw, d.num_classes = params["hw"], params["classes"]
        keep = []

        def dev(a):
            t = torch.from_numpy(a).to(device).contiguous()
            keep.append(t)
            return t.data_ptr()
        st = params["stem"]
        d.stem_w, d.stem_scale, d.stem_shift = dev(st["w"]), dev(st["scale"]), dev(st["shift"])
        nd = 0
        for b, blk in enumerate(params["blocks"]):
            c1, c2 = blk["c1"], blk["c2"]
            d.c1_w[b], d.c1_wscale[b], d.c1_scale[b], d.c1_shift[b] = (dev(c1["w"]), dev(c1["w_scale"]),
                                                                      dev(c1["scale"]), dev(c1["shift"]))
            d.c2_w[b], d.c2_wscale[b], d.c2_scale[b], d.c2_shift[b] = (dev(c2["w"]), dev(c2["w_scale"]),
                                                                      dev(c2["scale"]), dev(c2["shift"]))
            if blk["down"] is not None:
                c = blk["down"]
                d.down_w[nd], d.down_wscale[nd] = dev(c["w"]), dev(c["w_scale"])
                d.down_scale[nd], d.down_shift[nd] = dev(c["scale"]), dev(c["shift"])
                nd += 1
        fc = params["fc"]
        d.fc_w, d.fc_scale, d.fc_shift = dev(fc["w"]), dev(fc["scale"]), dev(fc["shift"])
        h = ctypes.c_void_p()
        _check(lib().minw_wresnet_create(ctypes.byref(d), int(max_batch), _stream(stream), ctypes.byref(h)),
               "minw_wresnet_create")
        net = cls.__new__(cls)
        net._h = h
        net.max_batch = max_batch
        net.out_features = params["classes"]
        return net

    def wresnet_activation(self, index, out, stream=None):
        """minw_wresnet_activation: the fp32 output of stage-step `index` of
        the most recent forward (0 the stem, b + 1 block b) into `out`."""
        _check(lib().minw_wresnet_activation(self._h, int(index), _ptr(out), out.numel(), _stream(stream)),
               "minw_wresnet_activation")

    @classmethod
    def wdense(cls, params, max_batch, device, stream=None):
        """minw_wdense_create from a parameter dict shaped like
        ``inputs.wdense_params`` (latent fp32 weights, BN maps); the tensors
        are copied to ``device`` for the call and released after it."""
        d = WDenseDesc()
        d.layers, d.growth, d.bits_w = params["layers"], params["growth"], params["bits_w"]
        for i in range(3):
            d.thr_w[i] = float(params["thr_w"][i])
        d.image_hw, d.num_classes = params["hw"], params["classes"]
        keep = []

        def dev(a):
            t = torch.from_numpy(a).to(device).contiguous()
            keep.append(t)
            return t.data_ptr()
        st = params["stem"]
        d.stem_w, d.stem_scale, d.stem_shift = dev(st["w"]), dev(st["scale"]), dev(st["shift"])
        j = 0
        for lay_list in params["blocks"]:
            for lay in lay_list:
                b, c = lay["b"], lay["c"]
                d.b_w[j], d.b_wscale[j], d.b_scale[j], d.b_shift[j] = (dev(b["w"]), dev(b["w_scale"]),
                                                                       dev(b["scale"]), dev(b["shift"]))
                d.c_w[j], d.c_wscale[j], d.c_scale[j], d.c_shift[j] = (dev(c["w"]), dev(c["w_scale"]),
                                                                       dev(c["scale"]), dev(c["shift"]))
                j += 1
        for i, t in enumerate(params["trans"]):
            d.t_w[i], d.t_wscale[i], d.t_scale[i], d.t_shift[i] = (dev(t["w"]), dev(t["w_scale"]),
                                                                   dev(t["scale"]), dev(t["shift"]))
        fc = params["fc"]
        d.fc_w, d.fc_scale, d.fc_shift = dev(fc["w"]), dev(fc["scale"]), dev(fc["shift"])
        h = ctypes.c_void_p()
        _check(lib().minw_wdense_create(ctypes.byref(d), int(max_batch), _stream(stream), ctypes.byref(h)),
               "minw_wdense_create")
        net = cls.__new__(cls)
        net._h = h
        net.max_batch = max_batch
        net.out_features = params["classes"]
        return net

    def wdense_features(self, block, out, stream=None):
        """minw_wdense_features: block `block`'s bf16 NHWC features after
        the most recent forward into the int16 device tensor `out`; returns
        (final channels, elements per pixel row)."""
        c, r = ctypes.c_int32(), ctypes.c_int32()
        _check(lib().minw_wdense_features(self._h, int(block), _ptr(out), out.numel(), ctypes.byref(c),
                                          ctypes.byref(r), _stream(stream)), "minw_wdense_features")
        return c.value, r.value

    @classmethod
    def resnet18(cls, params, max_batch, device, stream=None):
        """minw_resnet18_create from a parameter dict shaped like
        ``inputs.resnet18_params`` (latent fp32 weights, BN maps); the tensors
        are copied to ``device`` for the call and released after it."""
        d = ResNet18Desc()
        d.bits_a, d.bits_w = params["bits_a"], params["bits_w"]
        for i in range(3):
            d.thr_a[i] = float(params["thr_a"][i])
            d.thr_w[i] = float(params["thr_w"][i])
        d.image_hw, d.num_classes = params["hw"], params["classes"]
        keep = []

        def dev(a):
            t = torch.from_numpy(a).to(device).contiguous()
            keep.append(t)
            return t.data_ptr()
        st = params["stem"]
        d.stem_w, d.stem_scale, d.stem_shift = dev(st["w"]), dev(st["scale"]), dev(st["shift"])
        nd = 0
        for b, blk in enumerate(params["blocks"]):
            for j, c in enumerate((blk["c1"], blk["c2"])):
                d.conv_w[2 * b + j], d.conv_wscale[2 * b + j] = dev(c["w"]), dev(c["w_scale"])
                d.conv_scale[2 * b + j], d.conv_shift[2 * b + j] = dev(c["scale"]), dev(c["shift"])
            if blk["down"] is not None:
                c = blk["down"]
                d.down_w[nd], d.down_wscale[nd] = dev(c["w"]), dev(c["w_scale"])
                d.down_scale[nd], d.down_shift[nd] = dev(c["scale"]), dev(c["shift"])
                nd += 1
        fc = params["fc"]
        d.fc_w, d.fc_scale, d.fc_shift = dev(fc["w"]), dev(fc["scale"]), dev(fc["shift"])
        h = ctypes.c_void_p()
        _check(lib().minw_resnet18_create(ctypes.byref(d), int(max_batch), _stream(stream), ctypes.byref(h)),
               "minw_resnet18_create")
        net = cls.__new__(cls)
        net._h = h
        net.max_batch = max_batch
        net.out_features = params["classes"]
        return net

    def __init__(self, layers, max_batch, variant=VARIANT_AUTO, stream=None):
        arr = (LayerDesc * len(layers))()
        keep = []
        for d, L in zip(arr, layers):
            d.kind = L["kind"]
            d.C, d.H, d.W, d.O = L["C"], L["H"], L["W"], L["O"]
            d.kh, d.kw, d.stride, d.pad, d.pool = L.get("kh", 1), L.get("kw", 1), L.get("stride", 1), \
                L.get("pad", 0), int(L.get("pool", 0))
            d.bits_in, d.bits_w, d.bits_out = L["bits_in"], L["bits_w"], L["bits_out"]
            d.variant = int(L.get("variant", 0))
            for i in range(3):
                d.thr_w[i] = float(L["thr_w"][i])
                d.thr_out[i] = float(L["thr_out"][i])
            for k in ("w", "w_scale", "scale", "shift"):
                t = L.get(k)
                keep.append(t)
                setattr(d, k, t.data_ptr() if t is not None else None)
        h = ctypes.c_void_p()
        _check(lib().minw_net_create(arr, len(layers), int(max_batch), int(variant), _stream(stream),
                                     ctypes.byref(h)), "minw_net_create")
        self._h = h
        self.max_batch = max_batch
        self.out_features = layers[-1]["O"]

    def forward(self, x, logits, stream=None):
        _check(lib().minw_forward(self._h, _ptr(x), x.shape[0], _ptr(logits), _stream(stream)),
               "minw_forward")

    def forward_host(self, x_host, logits_host, stream=None):
        """Host-buffer forward (numpy or pinned CPU tensors): copies in, runs,
        copies the logits out and waits for them."""
        _check(lib().minw_forward_host(self._h, ctypes.c_void_p(_host_ptr(x_host)), x_host.shape[0],
                                       ctypes.c_void_p(_host_ptr(logits_host)), _stream(stream)),
               "minw_forward_host")

    def enable_timing(self, on=True):
        _check(lib().minw_net_enable_timing(self._h, int(on)), "minw_net_enable_timing")

    def layer_times(self):
        """Milliseconds of each layer's kernel in the most recent forward."""
        n = self.launches
        arr = (ctypes.c_float * n)()
        _check(lib().minw_net_layer_times(self._h, arr), "minw_net_layer_times")
        return list(arr)

    def layer_variants(self):
        """Kernel per layer: 0 fp32 first layer, VARIANT_POPC, VARIANT_TC (E4M3
        operands), VARIANT_TC_E2M1, VARIANT_TC_E2M1_PAIRS or VARIANT_TC_E2M1_N128."""
        n = self.launches
        arr = (ctypes.c_int32 * n)()
        _check(lib().minw_net_layer_variants(self._h, arr), "minw_net_layer_variants")
        return list(arr)

    def layer_candidates(self, layer):
        """Creation-time milliseconds of layer `layer`'s candidates under
        VARIANT_AUTO: [E4M3, E2M1, E2M1 pairs, popcount, E2M1 128-channel
        tiles], -1 where not one."""
        arr = (ctypes.c_float * 5)()
        _check(lib().minw_net_layer_candidates(self._h, int(layer), arr), "minw_net_layer_candidates")
        return list(arr)

    @property
    def kernels(self):
        """Kernels one forward launches."""
        return lib().minw_net_kernels(self._h)

    @property
    def launches(self):
        return lib().minw_net_launches(self._h)

    def close(self):
        if self._h:
            lib().minw_net_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def layer_descs(net_params, device):
    """minw_layer_desc dicts (device tensors) for a network described by
    ``inputs.convnet_params``: marshalling of the same fields, no compute."""
    out = []
    thr_a = net_params["thr_a"]
    c, h, w = net_params["in_shape"]
    for L in net_params["layers"]:
        d = dict(bits_in=L["bits_in"], bits_w=L["bits_w"], bits_out=L["bits_out"],
                 thr_w=list(net_params["thr_w"]), thr_out=list(thr_a) if L["bits_out"] else [0.0] * 3,
                 w=torch.from_numpy(L["w"]).to(device).contiguous(),
                 w_scale=torch.from_numpy(L["w_scale"]).to(device),
                 scale=torch.from_numpy(L["scale"]).to(device),
                 shift=torch.from_numpy(L["shift"]).to(device), O=L["O"])
        if L["kind"] == "conv":
            d.update(kind=LAYER_CONV, C=c, H=h, W=w, kh=L["kh"], kw=L["kw"], stride=L["stride"],
                     pad=L["pad"], pool=int(L["pool"]))
            h = (h + 2 * L["pad"] - L["kh"]) // L["stride"] + 1
            w = (w + 2 * L["pad"] - L["kw"]) // L["stride"] + 1
            if L["pool"]:
                h, w = h // 2, w // 2
            c = L["O"]
        else:
            d.update(kind=LAYER_FC, C=c, H=h, W=w)
            c, h, w = L["O"], 1, 1
        out.append(d)
    return out


# ---------------------------------------------------------------------------
# heads: group norm, clipped updates, 4-bit weights
# ---------------------------------------------------------------------------

def minw_group_norm_workspace_bytes(B, P, C, groups, backward=False):
    return lib().minw_group_norm_workspace_bytes(int(B), int(P), int(C), int(groups), int(bool(backward)))


def _image_rows(x, groups):
    shape = x.shape
    if len(shape) == 3:
        B, P, C = shape
    elif len(shape) >= 2:
        B, P, C = shape[0], math.prod(shape[1:-1]), shape[-1]
    else:
        raise ValueError("[B, ..., C] expected")
    return B, P, C, groups


def minw_group_norm(x, gamma, beta, groups, eps, y, act=ACT_NONE, mean=None, rstd=None, workspace=None, stream=None):
    """y = act(group norm of x) on channels-last tensors [B, ..., C] (fp32 or bf16, each; rows may be wider than C);
    gamma, beta fp32 [C] or None; mean, rstd fp32 [B, groups] or None receive the statistics."""
    B, P, C, G = _image_rows(x, groups)
    if y.shape != x.shape:
        raise ValueError("y: x's shape expected")
    px, ldx = _rows(x)
    py, ldy = _rows(y)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_group_norm(px, _value_type(x), ldx, _f32(gamma, C, "gamma"), _f32(beta, C, "beta"), B, P, C, G,
                                 float(eps), int(act), py, _value_type(y), ldy, _f32(mean, B * G, "mean"),
                                 _f32(rstd, B * G, "rstd"), ws, ws_bytes, _stream(stream)), "minw_group_norm")


def minw_group_norm_backward(x, dy, gamma, beta, mean, rstd, groups, dx, dgamma=None, dbeta=None, act=ACT_NONE,
                             workspace=None, stream=None):
    """dx (x's type), dgamma, dbeta from dy and the forward's mean and rstd."""
    B, P, C, G = _image_rows(x, groups)
    if dy.shape != x.shape or dx.shape != x.shape or dx.dtype != x.dtype:
        raise ValueError("dy, dx: x's shape expected, and dx its type")
    px, ldx = _rows(x)
    pd, ldd = _rows(dy)
    po, ldo = _rows(dx)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_group_norm_backward(px, _value_type(x), ldx, pd, _value_type(dy), ldd, _f32(gamma, C, "gamma"),
                                          _f32(beta, C, "beta"), _f32(mean, B * G, "mean"), _f32(rstd, B * G, "rstd"),
                                          B, P, C, G, int(act), po, ldo, _f32(dgamma, C, "dgamma"),
                                          _f32(dbeta, C, "dbeta"), ws, ws_bytes, _stream(stream)),
           "minw_group_norm_backward")


def _limits(limits, n):
    one = isinstance(limits, (int, float)) or getattr(limits, "ndim", None) == 0          # numpy's and torch's too
    limits = [float(limits)] * n if one else [float(v) for v in limits]
    if len(limits) != n:
        raise ValueError("a limit per tensor expected")
    return limits


class TensorList:
    """Dense device tensors (fp32 or bf16, any lengths and offsets) as the host array that the calls on lists take;
    made once for tensors that stay where they are: it holds the tensors and the addresses they had when it was made.
    Making one takes the host 0.7 us a tensor (232 us for 331; a call with two such lists 10 us), as does a call that is
    given plain lists of tensors.  limits: the clip of each weight tensor, or one for all (infinity for none)."""

    def __init__(self, tensors, limits=float("inf")):
        self.tensors = list(tensors)
        limits = _limits(limits, len(self.tensors))
        self.array = (Tensor * max(1, len(self.tensors)))()
        for e, t, limit in zip(self.array, self.tensors, limits):
            p = _ptr(t)
            e.data, e.n, e.type, e.limit = p.value, t.numel(), _value_type(t), limit

    def __len__(self):
        return len(self.tensors)


def _list(tensors):
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def _pair(a, b):
    a, b = _list(a), _list(b)
    if len(a) != len(b):
        raise ValueError("lists of the same length expected")
    return a, b


def minw_grad_workspace_bytes(count):
    return lib().minw_grad_workspace_bytes(int(count))


def minw_grad_norm(grads, norm, workspace, stream=None):
    """norm (one fp32 value on the device) = the 2-norm over all tensors of grads (a TensorList, or tensors)."""
    g = _list(grads)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_grad_norm(g.array, len(g), _f32(norm, 1, "norm"), ws, ws_bytes, _stream(stream)),
           "minw_grad_norm")


def minw_grad_clip(grads, out, max_norm, norm, workspace, stream=None):
    """out = grads scaled to the norm max_norm where theirs is larger (out may be grads)."""
    g, o = _pair(grads, out)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_grad_clip(g.array, o.array, len(g), float(max_norm), _f32(norm, 1, "norm"), ws, ws_bytes,
                                _stream(stream)), "minw_grad_clip")


def minw_sgd_clip_norm(weights, grads, max_norm, lr, norm, workspace, stream=None):
    """weights -= lr times the clipped grads, each kept within its limit (a TensorList's)."""
    w, g = _pair(weights, grads)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_sgd_clip_norm(w.array, g.array, len(g), float(max_norm), float(lr), _f32(norm, 1, "norm"), ws,
                                    ws_bytes, _stream(stream)), "minw_sgd_clip_norm")


class MatrixList:
    """Device matrices [rows][cols] (fp32 or bf16; rows may be wider apart) as the host array that the calls on
    matrices take; a tensor of more dimensions counts as [shape[0]][the rest] and has to be dense.  Made once for tensors that
    stay where they are, as a TensorList.  limits: the clip of each weight matrix, or one for all (infinity for none)."""

    def __init__(self, tensors, limits=float("inf")):
        self.tensors = list(tensors)
        limits = _limits(limits, len(self.tensors))
        self.array = (Matrix * max(1, len(self.tensors)))()
        for e, t, limit in zip(self.array, self.tensors, limits):
            if t.ndim < 2:
                raise ValueError("matrices expected")
            if t.ndim > 2 or t.numel() == 0:
                p, (e.rows, e.cols) = _ptr(t), (t.shape[0], math.prod(t.shape[1:]))
                e.data, e.ld = p.value, e.cols
            else:
                e.rows, e.cols = t.shape
                e.data, e.ld = _rows(t)
            e.type, e.limit = _value_type(t), limit

    def __len__(self):
        return len(self.tensors)


def _matrices(tensors):
    return tensors if isinstance(tensors, MatrixList) else MatrixList(tensors)


def minw_orthogonal_workspace_bytes(grads):
    """Workspace bytes of the calls on matrices of these sizes (a MatrixList, or tensors)."""
    g = _matrices(grads)
    return lib().minw_orthogonal_workspace_bytes(g.array, len(g))


def minw_orthogonalize(grads, out, workspace, steps=5, stream=None):
    """out = each matrix of grads orthogonalised by `steps` Newton-Schulz steps (out may be grads)."""
    g, o = _matrices(grads), _matrices(out)
    if len(g) != len(o):
        raise ValueError("lists of the same length expected")
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_orthogonalize(g.array, o.array, len(g), int(steps), ws, ws_bytes, _stream(stream)),
           "minw_orthogonalize")


def minw_sgd_orthogonal(weights, momenta, grads, lr, workspace, momentum=0.95, nesterov=True, steps=5, stream=None):
    """momenta = momentum momenta + grads (None: none), weights -= lr sqrt(max(1, rows / cols)) times the orthogonalised
    result, each kept within its limit (a MatrixList's)."""
    w, g = _matrices(weights), _matrices(grads)
    m = None if momenta is None else _matrices(momenta)
    if len(w) != len(g) or (m is not None and len(m) != len(g)):
        raise ValueError("lists of the same length expected")
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_sgd_orthogonal(w.array, None if m is None else m.array, g.array, len(g), int(steps), float(momentum),
                                     int(bool(nesterov)), float(lr), ws, ws_bytes, _stream(stream)),
           "minw_sgd_orthogonal")


def w4_shapes(O, K, group):
    """Shapes of the w4 layout of [O][K] weights: (codes uint8, scales bfloat16)."""
    return (O, (K + 127) // 128 * 64), (O, (K + group - 1) // group)


def _w4(codes, scales, O, K, group):
    if group < 1 or (tuple(codes.shape), tuple(scales.shape)) != w4_shapes(O, K, group):
        raise ValueError("codes and scales of w4_shapes(O, K, group) expected")
    if codes.dtype != torch.uint8 or scales.dtype != torch.bfloat16:
        raise ValueError("codes uint8 and scales bfloat16 expected")
    return _addr(codes), _addr(scales)


def minw_pack_w4(w, group, codes, scales, q=None, channel_scale=None, stream=None):
    """w [O][K] (fp32 or bf16) -> 4-bit codes and group scales; with q, the levels of that quantizer (1-3 bits) in
    integer units, scales 1."""
    O, K = w.shape
    pc, ps = _w4(codes, scales, O, K, int(group))
    _check(lib().minw_pack_w4(_ptr(w), _value_type(w), O, K, int(group), None if q is None else ctypes.byref(q),
                              _f32(channel_scale, O, "channel_scale"), pc, ps, _stream(stream)), "minw_pack_w4")


def minw_w4_matvec(x, codes, scales, group, y, scale=None, shift=None, act=ACT_NONE, stream=None):
    """y [T][O] = act(scale (x [T][K] times the w4 weights) + shift); x, y fp32 or bf16, rows may be wider."""
    (T, K), (Ty, O) = x.shape, y.shape
    if T != Ty:
        raise ValueError("x and y: the same number of rows expected")
    px, ldx = _rows(x)
    py, ldy = _rows(y)
    pc, ps = _w4(codes, scales, O, K, int(group))
    _check(lib().minw_w4_matvec(px, _value_type(x), ldx, T, pc, ps, O, K, int(group), _f32(scale, O, "scale"),
                                _f32(shift, O, "shift"), int(act), py, _value_type(y), ldy, _stream(stream)),
           "minw_w4_matvec")


def minw_adapters_workspace_bytes(T, K, O, n, r, backward=False):
    """Workspace bytes for T rows through n adapters of rank r, [K] -> [O]."""
    return lib().minw_adapters_workspace_bytes(int(T), int(K), int(O), int(n), int(r), int(bool(backward)))


def _pools(down, up, K, O):
    """(down, up, type, n, r) of adapters down [n][r][K], up [n][r][O]."""
    n, r = down.shape[0], down.shape[1]
    if tuple(down.shape) != (n, r, K) or tuple(up.shape) != (n, r, O) or down.dtype != up.dtype:
        raise ValueError("down [n][r][K] and up [n][r][O] of one type expected")
    return _addr(down), _addr(up), _value_type(down), n, r


def _ids(ids, T):
    if ids.dtype != torch.int32 or ids.numel() != T:
        raise ValueError(f"ids: {T} int32 values expected")
    return _addr(ids)


def minw_adapters(x, ids, down, up, y, alpha=None, base=None, scale=None, shift=None, act=ACT_NONE, h=None, workspace=None,
                  stream=None):
    """y [T][O] = act(scale (base + alpha[u] (x [T][K] down[u]^T) up[u]) + shift) with u = ids[t] of each row (no adapter
    where it is no index of the pools); h fp32 [T][r] or None receives x down[u]^T.  x, y, base: rows may be wider."""
    (T, K), (Ty, O) = x.shape, y.shape
    if T != Ty or (base is not None and base.shape != y.shape):
        raise ValueError("x, y and base: the same number of rows expected, y and base: the same columns")
    px, ldx = _rows(x)
    py, ldy = _rows(y)
    pb, ldb = (None, 0) if base is None else _rows(base)
    pd, pu, pt, n, r = _pools(down, up, K, O)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_adapters(px, _value_type(x), ldx, T, K, _ids(ids, T), pd, pu, pt, n, r, _f32(alpha, n, "alpha"), pb,
                               0 if base is None else _value_type(base), ldb, O, _f32(scale, O, "scale"),
                               _f32(shift, O, "shift"), int(act), py, _value_type(y), ldy, _f32(h, T * r, "h"), ws, ws_bytes,
                               _stream(stream)), "minw_adapters")


def minw_w4_adapters(x, codes, scales, group, ids, down, up, y, alpha=None, scale=None, shift=None, act=ACT_NONE,
                     workspace=None, stream=None):
    """minw_w4_matvec with each row's adapter: y = act(scale (x times the w4 weights + its adapter's term) + shift)."""
    (T, K), (Ty, O) = x.shape, y.shape
    if T != Ty:
        raise ValueError("x and y: the same number of rows expected")
    px, ldx = _rows(x)
    py, ldy = _rows(y)
    pc, ps = _w4(codes, scales, O, K, int(group))
    pd, pu, pt, n, r = _pools(down, up, K, O)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_w4_adapters(px, _value_type(x), ldx, T, pc, ps, O, K, int(group), _ids(ids, T), pd, pu, pt, n, r,
                                  _f32(alpha, n, "alpha"), _f32(scale, O, "scale"), _f32(shift, O, "shift"), int(act), py,
                                  _value_type(y), ldy, ws, ws_bytes, _stream(stream)), "minw_w4_adapters")


def minw_adapters_backward(x, ids, down, up, h, dy, ddown=None, dup=None, dx=None, alpha=None, accumulate=False,
                           workspace=None, stream=None):
    """Gradients of minw_adapters' term from dy [T][O] (that of base + the term) and the forward's h: dx (x's type; added
    to where accumulate is set), ddown and dup (fp32, of the pools' shapes); each may be None."""
    (T, K), (Ty, O) = x.shape, dy.shape
    if T != Ty or (dx is not None and (dx.shape != x.shape or dx.dtype != x.dtype)):
        raise ValueError("x and dy: the same number of rows expected, dx: x's shape and type")
    px, ldx = _rows(x)
    pg, ldg = _rows(dy)
    po, ldo = (None, 0) if dx is None else _rows(dx)
    pd, pu, pt, n, r = _pools(down, up, K, O)
    ws, ws_bytes = _scratch(workspace)
    _check(lib().minw_adapters_backward(px, _value_type(x), ldx, T, K, _ids(ids, T), pd, pu, pt, n, r,
                                        _f32(alpha, n, "alpha"), _f32(h, T * r, "h"), pg, _value_type(dy), ldg, O, po, ldo,
                                        int(bool(accumulate)), _f32(ddown, n * r * K, "ddown"), _f32(dup, n * r * O, "dup"),
                                        ws, ws_bytes, _stream(stream)), "minw_adapters_backward")
