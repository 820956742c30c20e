"""Refusals of the operators around the attention, on the host: nothing is enqueued, so no GPU is needed."""
import ctypes as C

import pytest

import paper_2502_01776_amd as S
from paper_2502_01776_amd import binding

A, B_, X, Y, Z, W = (0x10000000 * k for k in range(1, 7))           # addresses that are never read


def desc(**kw):
    base = dict(rows=64, channels=256, groups=2, pre_norm=2, gate=A, scale=A, shift=A)
    base.update(kw)
    return S.gate_norm_desc(**base)


def fwd(d, x=X, y=Y, r=Z, h=W, codes=None, scales=None):
    return S.lib().svg_gate_norm_fwd(C.byref(d) if d else None, x, y, r, h, codes, scales, None)


def test_struct_sizes():
    assert C.sizeof(S.SvgGateNorm) == 8 + 9 * 4 + 4 + 5 * 8 + 8 * 8 and C.sizeof(S.SvgGateNormGrads) == 64 and C.sizeof(S.SvgTokens) == 56


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(channels=0), dict(groups=0), dict(stream_type=1), dict(branch_type=2), dict(post_norm=3),
                                 dict(pre_norm=-1), dict(eps=-1.0), dict(post_eps=float("nan")), dict(ld_x=255), dict(ld_h=8), dict(ld_mod=1),
                                 dict(groups=3), dict(gate=A + 2), dict(group_ptr=A + 1), dict(weight=A + 3), dict(ld_y=-4)])
def test_gate_norm_descriptors(bad):
    assert fwd(desc(**bad)) == -1
    assert S.svg_gate_norm_workspace_bytes(desc(**bad)) == 0
    with pytest.raises(S.SvgError):
        S.svg_gate_norm_fwd(desc(**bad), X, Y, Z, W, stream=0)


def test_gate_norm_arguments():
    d = desc()
    assert fwd(None) == -1
    assert fwd(d, x=None) == -1
    assert fwd(d, r=None, h=None) == -1
    assert fwd(d, x=X + 1) == -1 and fwd(d, y=Y + 1) == -1
    assert fwd(d, codes=A) == -1 and fwd(d, scales=A) == -1 and fwd(d, codes=A + 8, scales=B_) == -1
    assert fwd(desc(channels=16385)) == -2 and fwd(desc(rows=2 ** 31, groups=1)) == -2
    assert fwd(d, h=X) == -4 and fwd(d, r=Y) == -4 and fwd(d, h=Z) == -4 and fwd(d, r=X + 512) == -4
    assert fwd(desc(ld_r=264), r=X) == -4                                # in place with another stride
    assert fwd(d, codes=X, scales=A) == -4 and fwd(d, codes=A, scales=A + 16) == -4
    assert fwd(desc(channels=40), codes=A, scales=B_) == -2              # not whole blocks
    assert fwd(desc(ld_x=257), codes=A, scales=B_) == -2                 # unaligned rows
    assert fwd(desc(rows=0)) == 0
    d.reserved = 1
    assert fwd(d) == -1


def bwd(d, r=X, y=Y, dr=Z, dh=W, dx=7 * A, dy=8 * A, grads=None, ws=9 * A, n=None):
    n = S.svg_gate_norm_workspace_bytes(d) if n is None else n
    return S.lib().svg_gate_norm_bwd(C.byref(d), r, y, dr, dh, dx, dy, C.byref(grads) if grads else None, ws, n, None)


def test_gate_norm_gradient_arguments():
    d = desc()
    n = S.svg_gate_norm_workspace_bytes(d)
    assert n > 0
    assert bwd(d, ws=None) == -3 and bwd(d, n=n - 1) == -3 and bwd(d, ws=9 * A + 4) == -1
    assert bwd(d, dx=None, dy=None) == -1                                # nothing wanted
    assert bwd(d, dr=None, dh=None) == -1                                # nothing given
    assert bwd(d, r=None) == -1
    assert bwd(desc(post_norm=1), y=None) == -1
    assert bwd(d, y=None, grads=S.gate_norm_grads(gate=B_)) == -1
    assert bwd(d, grads=S.gate_norm_grads(gate=B_ + 1)) == -1
    assert bwd(d, grads=S.gate_norm_grads(gate=B_, ld_mod=10)) == -1
    assert bwd(d, dx=X) == -4 and bwd(d, dy=X) == -4 and bwd(d, dx=W) == -4 and bwd(d, dy=7 * A) == -4 and bwd(d, ws=Z) == -4
    assert bwd(desc(ld_x=264), dx=Z) == -4                               # in place with another stride


def tokens(**kw):
    t = dict(B=2, N=10, H=4, D=64, stride_b=2560, stride_n=64, stride_h=640, type=0, reserved=0)
    t.update(kw)
    return S.SvgTokens(*t.values())


def quant(t, x=X, act=0, codes=Y, scales=Z):
    return S.lib().svg_fp4_quantize(C.byref(t) if t else None, x, act, codes, scales, None)


def dequant(t, x=X, codes=Y, scales=Z):
    return S.lib().svg_fp4_dequantize(C.byref(t) if t else None, codes, scales, x, None)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(N=-2), dict(H=0), dict(D=0), dict(stride_b=-1), dict(stride_n=-64), dict(stride_h=-5),
                                 dict(type=3), dict(type=-1), dict(reserved=1), dict(stride_n=2 ** 41)])
def test_token_matrices(bad):
    assert quant(tokens(**bad)) == -1 and dequant(tokens(**bad)) == -1


def test_quantiser_arguments():
    t = tokens()
    assert quant(None) == -1 and dequant(None) == -1
    assert quant(t, x=None) == -1 and quant(t, codes=None) == -1 and quant(t, scales=None) == -1 and quant(t, act=3) == -1 and quant(t, act=-1) == -1
    assert quant(t, x=X + 1) == -1 and quant(t, codes=Y + 8) == -1 and quant(t, scales=Z + 4) == -1
    assert quant(t, codes=X) == -4 and quant(t, scales=X) == -4 and quant(t, scales=Y) == -4 and dequant(t, codes=X) == -4
    assert quant(tokens(B=2 ** 20, N=2 ** 20)) == -2 and quant(tokens(H=2 ** 12, D=2 ** 12)) == -2
    assert quant(tokens(stride_b=2 ** 40, B=2 ** 22, N=1)) == -2
    # an output whose elements share places
    for bad in (dict(stride_n=63), dict(stride_h=0), dict(stride_b=64), dict(stride_n=64, stride_h=64)):
        assert dequant(tokens(**bad)) == -4, bad
    assert quant(tokens(B=0)) == 0 and quant(tokens(N=0)) == 0 and dequant(tokens(N=0)) == 0
    assert [S.svg_fp4_buffer_bytes(*a) for a in ((16, 256, 0), (17, 257, 0), (16, 256, 1), (17, 600, 1), (0, 5, 0))] == [2048, 8192, 256, 1024, 0]
    assert [S.svg_fp4_buffer_bytes(*a) for a in ((-1, 5, 0), (1, 0, 0), (1, 2 ** 21, 0), (2 ** 31, 5, 0), (1, 5, 2))] == [0] * 5


def linear(M=10, N=256, K=512, a=X, as_=Y, w=Z, ws=W, bias=None, act=0, t=None, out=7 * A, workspace=None, n=0):
    t = t or tokens(B=1, N=10, stride_n=64, stride_h=640)
    return S.lib().svg_fp4_linear(M, N, K, a, as_, w, ws, bias, act, C.byref(t), out, workspace, n, None)


def linear_quantize(M=10, N=256, K=512, a=X, as_=Y, w=Z, ws=W, bias=None, act=0, codes=7 * A, scales=8 * A):
    return S.lib().svg_fp4_linear_quantize(M, N, K, a, as_, w, ws, bias, act, codes, scales, None, 0, None)


@pytest.mark.parametrize("call", [linear, linear_quantize])
def test_product_arguments(call):
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(a=None), dict(as_=None), dict(w=None), dict(ws=None), dict(a=X + 8), dict(ws=W + 4),
                dict(bias=A + 2), dict(act=7)):
        assert call(**bad) == -1, bad
    for bad in (dict(M=2 ** 31), dict(N=2 ** 21), dict(K=2 ** 21)):
        assert call(**bad) == -2, bad


def test_product_outputs():
    assert linear(out=None) == -1 and linear(out=7 * A + 1) == -1
    assert linear(M=11) == -1 and linear(N=128) == -1                    # not the token matrix's rows and columns
    assert linear(t=tokens(B=1, stride_n=32)) == -4
    assert linear(out=X) == -4 and linear(out=W) == -4
    assert linear_quantize(codes=None) == -1 and linear_quantize(scales=8 * A + 4) == -1
    assert linear_quantize(codes=X) == -4 and linear_quantize(scales=7 * A) == -4 and linear_quantize(scales=Z) == -4
    assert linear(M=0, t=tokens(B=1, N=0)) == 0 and linear_quantize(M=0) == 0
    assert S.svg_fp4_linear_workspace_bytes(0, 5, 5) == 0 and S.svg_fp4_linear_workspace_bytes(5, 0, 5) == 0


def test_tokens_of_tensors():
    import torch
    t = S.tokens_of(torch.zeros(2, 5, 7, 64, dtype=torch.bfloat16))
    assert [t.B, t.N, t.H, t.D, t.stride_b, t.stride_n, t.stride_h, t.type] == [2, 7, 5, 64, 2240, 64, 448, S.SVG_BF16]
    t = S.tokens_of(torch.zeros(6, 40)[:, 3:20])
    assert [t.B, t.N, t.H, t.D, t.stride_n, t.type] == [1, 6, 1, 17, 40, S.SVG_F32]
    for bad in (torch.zeros(4, 6).t(), torch.zeros(3), torch.zeros(2, 3, 4)):
        with pytest.raises(ValueError):
            S.tokens_of(bad)
    assert binding.EXPORTS.count("svg_fp4_linear") == 1


@pytest.mark.parametrize("strides", [dict(ld_x=2 ** 40), dict(ld_h=2 ** 39), dict(ld_mod=2 ** 40, groups=2 ** 20)])
def test_tensors_whose_extent_passes_64_bits_are_refused(strides):
    """2^30 rows of 2^40 elements each: their last byte has no address, and their overlaps could not be told."""
    d = desc(**{**dict(rows=2 ** 30, groups=1), **strides})
    assert fwd(d) == -2 and S.svg_gate_norm_workspace_bytes(d) == 0
    grads = S.gate_norm_grads(gate=A, ld_mod=2 ** 40)
    big = desc(rows=2 ** 20, groups=2 ** 20)
    assert S.lib().svg_gate_norm_bwd(C.byref(big), X, Y, Z, W, A, B_, C.byref(grads), None, 0, None) == -2


def test_overlaps_of_rows_of_one_stride():
    """Slices that reach one element into each other's columns, or around the end of a row into the next one's."""
    wide = dict(ld_x=600, ld_r=600, ld_y=600, ld_h=600)
    for columns in (-599, -255, -1, 1, 255, 345, 599, 600 * 63 + 255):
        assert fwd(desc(**wide), r=X + 2 * columns) == -4, columns
    assert fwd(desc(**{**wide, "ld_r": 602}), r=X + 2 * 300) == -4          # another stride: their rows meet somewhere
    assert fwd(desc(rows=1, groups=1, **wide), r=X + 2 * 255) == -4


TABLES = ("gate", "scale", "shift", "group_ptr", "post_weight", "post_bias", "weight", "bias")


@pytest.mark.parametrize("name", TABLES)
def test_results_over_the_parameters_are_refused(name):
    for out in (dict(r=Z), dict(h=W), dict(codes=Y, scales=B_), dict(codes=B_, scales=Y)):
        at = next(v for k, v in out.items() if v != B_)
        args = {**dict(x=X, y=None, r=7 * A, h=8 * A), **out}
        assert fwd(desc(**{name: at}), **args) == -4, out
        assert fwd(desc(**{name: at + 64}), **args) == -4, out
    assert fwd(desc(ld_mod=512, gate=Z + 4 * 200), r=None, h=Z) == -4        # the second group's row of a table, one stride apart


GRADS = ("gate", "scale", "shift", "post_weight", "post_bias", "weight", "bias")


@pytest.mark.parametrize("name", GRADS)
def test_gradients_over_other_tensors_are_refused(name):
    """Over the rows, the workspace, the descriptor's tables (a table is read again behind a gradient's write), and each other."""
    d = desc(gate=100 * A, scale=101 * A, shift=102 * A, post_weight=103 * A, post_bias=104 * A, weight=105 * A, bias=106 * A, group_ptr=107 * A,
             post_norm=2)
    free = 110 * A
    for at in (X, Y, Z, W, 7 * A, 8 * A, 9 * A, *(k * A for k in range(100, 108))):
        assert bwd(d, grads=S.gate_norm_grads(**{name: at})) == -4, hex(at)
        assert bwd(d, grads=S.gate_norm_grads(**{name: at + 8})) == -4, hex(at)
    for other in GRADS:
        if other != name:
            assert bwd(d, grads=S.gate_norm_grads(**{name: free, other: free + 4 * 255})) == -4, other
    table = name in GRADS[:3]
    if table:                                                            # slices of one tensor that reach into each other
        for columns in (-255, 255, 513, 600):
            assert bwd(d, grads=S.gate_norm_grads(**{n: free if n == name else free + 4 * columns for n in (name, "shift" if name != "shift" else "gate")},
                                                  ld_mod=600)) == -4, columns


@pytest.mark.parametrize("name", TABLES)
def test_row_gradients_and_workspace_over_the_parameters_are_refused(name):
    d = desc(**{"gate": 100 * A, "scale": 101 * A, "shift": 102 * A, name: 110 * A})
    for out in ("dx", "dy", "ws"):
        assert bwd(d, **{out: 110 * A}) == -4, out


def test_products_over_their_bias_are_refused():
    for at in (9 * A, 9 * A - 4 * 255, 9 * A + 64):
        assert linear(bias=at, out=9 * A) == -4 and linear_quantize(bias=at, codes=9 * A) == -4, hex(at)
        assert linear_quantize(bias=at, scales=9 * A) == -4, hex(at)


def test_token_matrices_of_other_types_are_refused():
    import torch
    for dtype in (torch.float64, torch.int32, torch.float8_e4m3fn):
        for shape in ((4, 6), (1, 2, 3, 4)):
            with pytest.raises(ValueError, match="element type"):
                S.tokens_of(torch.zeros(shape).to(dtype))
