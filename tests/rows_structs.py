"""The argument structs of the embedding and norm calls as ctypes, for tests that call the library past the binding."""
import ctypes as C

I32, I64, PTR, F32, SIZE = C.c_int32, C.c_int64, C.c_void_p, C.c_float, C.c_size_t


class EmbedArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", I32), ("V", I32), ("Dh", I32), ("tokens", PTR), ("table", PTR), ("table_stride", I64), ("scale", F32),
                ("out", PTR), ("out_stride", I64), ("out_type", I32)]


class EmbedBwdArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", I32), ("V", I32), ("Dh", I32), ("tokens", PTR), ("d_out", PTR), ("d_out_stride", I64), ("d_out_type", I32),
                ("scale", F32), ("d_table", PTR), ("d_table_stride", I64), ("d_table_type", I32), ("accumulate", I32), ("workspace", PTR),
                ("workspace_bytes", SIZE)]


class RowNormArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", I32), ("D", I32), ("kind", I32), ("x", PTR), ("x_stride", I64), ("x_type", I32), ("residual", PTR),
                ("residual_stride", I64), ("sum_out", PTR), ("sum_stride", I64), ("weight", PTR), ("bias", PTR), ("eps", F32), ("out", PTR),
                ("out_stride", I64)]


class RowNormBwdArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", I32), ("D", I32), ("kind", I32), ("d_out", PTR), ("d_out_stride", I64), ("x", PTR), ("x_stride", I64),
                ("x_type", I32), ("d_sum", PTR), ("d_sum_stride", I64), ("weight", PTR), ("eps", F32), ("d_x", PTR), ("d_x_stride", I64), ("d_weight", PTR),
                ("d_bias", PTR), ("workspace", PTR), ("workspace_bytes", SIZE)]


class LmheadBwdArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("M", I32), ("Dh", I32), ("V", I32), ("hidden", PTR), ("hidden_stride_row", I64), ("row_idx", PTR), ("m_dev", PTR), ("w", PTR),
                ("w_stride_row", I64), ("inv_temperature", F32), ("forbid_token", I32), ("out_scatter", I32), ("lse", PTR), ("target", PTR), ("d_lse", PTR),
                ("d_ztarget", PTR), ("d_hidden", PTR), ("d_hidden_stride_row", I64), ("d_hidden_type", I32), ("d_w", PTR), ("d_w_stride_row", I64),
                ("d_w_type", I32), ("accumulate", I32), ("workspace", PTR), ("workspace_bytes", SIZE)]
