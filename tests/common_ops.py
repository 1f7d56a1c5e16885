"""The argument structures of include/cada_ops.h that Python reaches through _ops.so, for tests of the C ABI itself."""
import ctypes as C

from paper_2012_15469_amd.binding import _lib


class cada_linear(C.Structure):
    _fields_ = [("rows", C.c_int64), ("in_", C.c_int64), ("out", C.c_int64), ("type", C.c_int32), ("act", C.c_int32),
                ("x", C.c_void_p), ("ldx", C.c_int64), ("w", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p),
                ("residual", C.c_void_p), ("ldr", C.c_int64), ("y", C.c_void_p), ("ldy", C.c_int64), ("pre", C.c_void_p), ("ldpre", C.c_int64),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class cada_linear_grad(C.Structure):
    _fields_ = [("rows", C.c_int64), ("in_", C.c_int64), ("out", C.c_int64), ("type", C.c_int32), ("act", C.c_int32),
                ("dy", C.c_void_p), ("lddy", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64), ("w", C.c_void_p), ("ldw", C.c_int64),
                ("pre", C.c_void_p), ("ldpre", C.c_int64), ("dx", C.c_void_p), ("lddx", C.c_int64), ("dw", C.c_void_p), ("lddw", C.c_int64),
                ("db", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class cada_xent(C.Structure):
    _fields_ = [("rows", C.c_int64), ("classes", C.c_int64), ("type", C.c_int32), ("label_bytes", C.c_int32), ("logits", C.c_void_p), ("ldz", C.c_int64),
                ("labels", C.c_void_p), ("ignore_index", C.c_int64), ("smoothing", C.c_double), ("scale", C.c_double), ("mean", C.c_void_p),
                ("loss", C.c_void_p), ("grad", C.c_void_p), ("ldg", C.c_int64), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("stream", C.c_void_p)]


for _name, _type in (("cada_linear_forward", cada_linear), ("cada_linear_backward", cada_linear_grad), ("cada_cross_entropy", cada_xent)):
    for _f in (getattr(_lib, _name), getattr(_lib, _name.replace("cross_entropy", "xent") + "_workspace")):
        _f.restype, _f.argtypes = C.c_int, [C.POINTER(_type)]
