"""The argument structs of the paged-cache and head calls as ctypes, for tests that call the library past the binding."""
import ctypes as C


class PagedKv(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("stride_page", C.c_int64), ("stride_h", C.c_int64), ("stride_t", C.c_int64), ("type", C.c_int32),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class HeadMap(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("eps", C.c_float), ("rope", C.c_void_p),
                ("rope_len", C.c_int32), ("rot_dim", C.c_int32), ("rope_style", C.c_int32), ("positions", C.c_void_p)]


def _heads(name, stride):
    return [(name, C.c_void_p), (stride + "_stride_t", C.c_int64), (stride + "_stride_h", C.c_int64)]


class QkArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                *_heads("q", "q"), *_heads("k", "k"), *_heads("q_out", "qo"), *_heads("k_out", "ko"), ("map", HeadMap)]


class QkBwdArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                *_heads("d_q_out", "dqo"), *_heads("d_k_out", "dko"), *_heads("q", "q"), *_heads("k", "k"), *_heads("d_q", "dq"), *_heads("d_k", "dk"),
                ("d_q_weight", C.c_void_p), ("d_k_weight", C.c_void_p), ("map", HeadMap), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class AppendArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                *_heads("q", "q"), *_heads("k", "k"), *_heads("v", "v"), *_heads("q_out", "qo"), ("slots", C.c_void_p), ("cache", PagedKv),
                ("map", HeadMap)]


class PagedAttnArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("B", C.c_int32), ("Lq", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                ("q", C.c_void_p), ("q_stride_b", C.c_int64), ("q_stride_t", C.c_int64), ("q_stride_h", C.c_int64),
                ("out", C.c_void_p), ("o_stride_b", C.c_int64), ("o_stride_t", C.c_int64), ("o_stride_h", C.c_int64),
                ("lse", C.c_void_p), ("cache", PagedKv), ("block_table", C.c_void_p), ("table_stride", C.c_int64), ("kv_len", C.c_void_p),
                ("max_kv_len", C.c_int32), ("q_len", C.c_void_p), ("mask_mode", C.c_int32), ("block_size", C.c_int32), ("scale", C.c_float),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]
