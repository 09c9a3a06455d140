"""ctypes mirrors of the argument structures of include/qsr.h that the package fills in C++ (csrc/torch_calls.cpp)."""
import ctypes as C

from paper_2310_14423_amd.operators import AdamWConfig, Tensor  # noqa: F401


class RMSNormArgs(C.Structure):
    _fields_ = [("K", C.c_int32), ("type", C.c_int32), ("y_type", C.c_int32), ("rows", C.c_int64), ("d", C.c_int64),
                ("x", C.c_void_p), ("residual", C.c_void_p), ("weight", C.c_void_p), ("sum", C.c_void_p), ("y", C.c_void_p),
                ("scale", C.c_void_p), ("rstd", C.c_void_p), ("x_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("sum_stride", C.c_int64), ("y_stride", C.c_int64), ("weight_stride", C.c_int64), ("eps", C.c_double)]


class RMSNormBackwardArgs(C.Structure):
    _fields_ = [("K", C.c_int32), ("type", C.c_int32), ("rows", C.c_int64), ("d", C.c_int64), ("y_grad", C.c_void_p),
                ("sum", C.c_void_p), ("weight", C.c_void_p), ("rstd", C.c_void_p), ("residual_grad", C.c_void_p),
                ("x_grad", C.c_void_p), ("weight_grad", C.c_void_p), ("y_grad_stride", C.c_int64), ("sum_stride", C.c_int64),
                ("residual_grad_stride", C.c_int64), ("x_grad_stride", C.c_int64), ("weight_stride", C.c_int64)]


class TokenLogprobsArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int64), ("stride", C.c_int64), ("type", C.c_int32), ("top", C.c_int32),
                ("logits", C.c_void_p), ("tokens", C.c_void_p), ("temperature", C.c_double), ("logp", C.c_void_p),
                ("entropy", C.c_void_p), ("lse", C.c_void_p), ("stats", C.c_void_p), ("top_logp", C.c_void_p), ("top_id", C.c_void_p)]


class TokenLogprobsBackwardArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int64), ("stride", C.c_int64), ("grad_stride", C.c_int64), ("type", C.c_int32),
                ("reserved", C.c_int32), ("logits", C.c_void_p), ("tokens", C.c_void_p), ("temperature", C.c_double),
                ("stats", C.c_void_p), ("entropy", C.c_void_p), ("logp_grad", C.c_void_p), ("entropy_grad", C.c_void_p),
                ("grad", C.c_void_p)]
