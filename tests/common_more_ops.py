"""The argument structures of the embedding's, layer norm's and the last layer's loss in include/cada_ops.h, for tests of the C ABI itself."""
import ctypes as C

from paper_2012_15469_amd.binding import _lib

P, I64, I32, F64 = C.c_void_p, C.c_int64, C.c_int32, C.c_double
_END = [("workspace", P), ("workspace_bytes", C.c_size_t), ("stream", P)]


class cada_norm(C.Structure):
    _fields_ = [("rows", I64), ("width", I64), ("type", I32), ("eps", F64), ("x", P), ("ldx", I64), ("weight", P), ("bias", P), ("y", P), ("ldy", I64),
                ("mean", P), ("rstd", P), ("stream", P)]


class cada_norm_grad(C.Structure):
    _fields_ = [("rows", I64), ("width", I64), ("type", I32), ("dy", P), ("lddy", I64), ("x", P), ("ldx", I64), ("mean", P), ("rstd", P), ("weight", P),
                ("residual", P), ("ldr", I64), ("dx", P), ("lddx", I64), ("dw", P), ("db", P)] + _END


class cada_embedding(C.Structure):
    _fields_ = [("rows", I64), ("vocab", I64), ("width", I64), ("type", I32), ("token_bytes", I32), ("tokens", P), ("ignore_index", I64), ("w", P), ("ldw", I64),
                ("scale", F64), ("y", P), ("ldy", I64), ("stream", P)]


class cada_embedding_grad(C.Structure):
    _fields_ = [("rows", I64), ("vocab", I64), ("width", I64), ("type", I32), ("token_bytes", I32), ("tokens", P), ("ignore_index", I64), ("dy", P), ("lddy", I64),
                ("scale", F64), ("dw", P), ("lddw", I64)] + _END


class cada_linear_xent(C.Structure):
    _fields_ = [("rows", I64), ("in_", I64), ("classes", I64), ("type", I32), ("label_bytes", I32), ("x", P), ("ldx", I64), ("w", P), ("ldw", I64), ("bias", P), ("labels", P),
                ("ignore_index", I64), ("smoothing", F64), ("scale", F64), ("mean", P), ("loss", P), ("dx", P), ("lddx", I64), ("dw", P), ("lddw", I64), ("db", P)] + _END


for _name, _type in (("cada_linear_xent_workspace", cada_linear_xent), ("cada_linear_cross_entropy", cada_linear_xent),
                     ("cada_layer_norm_forward", cada_norm), ("cada_layer_norm_backward", cada_norm_grad), ("cada_layer_norm_backward_workspace", cada_norm_grad),
                     ("cada_embedding_forward", cada_embedding), ("cada_embedding_backward", cada_embedding_grad), ("cada_embedding_backward_workspace", cada_embedding_grad)):
    _f = getattr(_lib, _name)
    _f.restype, _f.argtypes = C.c_int, [C.POINTER(_type)]


def filled(kind, base, **kw):
    a = kind()
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a
