"""How a call of svg_kv4_attn_fwd is cut, as the library's host function says it, for the tests of the choice and of the results."""
import ctypes as C

import paper_2502_01776_amd as S


class Cache(C.Structure):
    _fields_ = [("data", C.c_void_p), ("table", C.c_void_p), ("B", C.c_int), ("H", C.c_int), ("D", C.c_int), ("page_log2", C.c_int),
                ("pages", C.c_int), ("max_pages", C.c_int)]


class Plan(C.Structure):
    _fields_ = [("rows", C.c_int), ("tile", C.c_int), ("tiles", C.c_int), ("parts", C.c_int), ("reach", C.c_int)]


def plan(cache, attn, N, group):
    c = Cache(cache.data, cache.page_table, cache.B, cache.H, cache.D, cache.page_size.bit_length() - 1, cache.pages, cache.max_pages)
    f = S.lib()._ZN3svg8kv4_planERKNS_3Kv4ERK12svg_kv4_attnxi
    f.restype, f.argtypes = Plan, [C.POINTER(Cache), C.POINTER(S.SvgKv4Attn), C.c_longlong, C.c_int]
    return f(C.byref(c), C.byref(attn), N, group)
