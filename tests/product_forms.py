"""Products that reach every form of svg_fp4_linear, for the tests of the choice (host) and of the results (GPU)."""
import ctypes as C

import paper_2502_01776_amd as S

ROWS1, ROWS2_EIGHT, ROWS2, ROWS4, TILES64, TILES128, SQUARE = range(7)
TILE = {TILES64: (64, 128), TILES128: (128, 256), SQUARE: (256, 256)}       # tokens and columns of an output tile
PLACES = {TILES64: 512, TILES128: 512, SQUARE: 256}                         # workgroups of a launch: more tiles are a second turn

# (M, N, K, head dimension that divides N, a multiple of 8)
PRODUCTS = [
    (5, 248, 700, 248), (16, 1016, 1280, 8), (20, 248, 1280, 248), (20, 8184, 300, 88), (31, 8184, 1280, 88), (20, 10224, 300, 144),
    (31, 10224, 512, 144), (50, 504, 1100, 72), (200, 640, 1536, 64),
    *((700, 2552, K, 88) for K in (130, 512, 700, 1000, 1280, 1790)),       # 64 x 128
    *((1025, 4088, K, 56) for K in (130, 512, 700, 1000, 1280)),            # 128 x 256; 64 x 128 behind an activation, a second turn
    *((4100, 4088, K, 56) for K in (130, 512, 700, 1280)),                  # the same, a second turn of both
    *((2050, 4088, K, 56) for K in (130, 512, 700, 1280)),                  # 256 x 256; 64 x 128
    *((4100, 6136, K, 104) for K in (130, 512, 700, 1280)),                 # 256 x 256, a second turn
    (1025, 6136, 1536, 104), (8000, 2552, 1000, 88), (4100, 2552, 700, 88),
]


def column_tiles(K):
    return -(-K // 256) * 2


def form(M, N, K, activation, operand=False):
    f = S.lib()._ZN3svg15fp4_linear_formExxib
    f.restype, f.argtypes = C.c_int, [C.c_longlong, C.c_longlong, C.c_int, C.c_bool]
    return f(-(-M // 16), -(-N // 256) * 8 if operand else -(-N // 32), column_tiles(K), bool(activation))
