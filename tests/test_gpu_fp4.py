"""Microscaled 4-bit operands and products against the 64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import block_oracle as O
from test_gpu_gate_norm import HALF, U, assert_four_bit, close, f64

pytestmark = pytest.mark.gpu

ACT = {S.SVG_ACT_NONE: lambda v: v, S.SVG_ACT_SILU: O.silu, S.SVG_ACT_GELU_TANH: O.gelu_tanh}


def buffers(rows, cols):
    return [torch.full((S.svg_fp4_buffer_bytes(rows, cols, w),), 0xAA, dtype=torch.uint8, device="cuda") for w in (0, 1)]


def quantise(x, act=S.SVG_ACT_NONE):
    t = S.tokens_of(x)
    codes, scales = buffers(t.B * t.N, t.H * t.D)
    S.svg_fp4_quantize(t, x, act, codes, scales)
    torch.cuda.synchronize()
    return codes, scales


def rows_of(x):
    """The token matrix of a tensor in 64 bits."""
    v = f64(x)
    return v if v.ndim == 2 else v.transpose(0, 2, 1, 3).reshape(v.shape[0] * v.shape[2], -1)


def data(rows, cols, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen) * torch.exp(2 * torch.randn(rows, 1, generator=gen))
    return x.to(dtype).cuda()


def check_exact(x):
    codes, scales = quantise(x)
    v = rows_of(x)
    ref_codes, ref_scales = O.mx_quantise(v)
    got, gs = O.from_operand(codes.cpu().numpy(), scales.cpu().numpy(), *v.shape)
    assert np.array_equal(gs, ref_scales)
    ok = np.repeat(ref_scales != 255, 32, axis=1)[:, :v.shape[1]]
    assert np.array_equal(got[ok] & 7, ref_codes[ok] & 7) and np.array_equal((got ^ ref_codes)[ok & (ref_codes & 7 > 0)] & 8, 0 * got[ok & (ref_codes & 7 > 0)])
    full = O.from_operand(codes.cpu().numpy(), scales.cpu().numpy(), -(-v.shape[0] // 16) * 16, -(-v.shape[1] // 256) * 256)[0]
    assert not full[v.shape[0]:].any() and not full[:, v.shape[1]:].any()
    values = O.mx_values(ref_codes, ref_scales)
    for t in (torch.float32, torch.bfloat16):
        back = torch.full((v.shape[0], v.shape[1]), 7.0, dtype=t, device="cuda")
        S.svg_fp4_dequantize(S.tokens_of(back), codes, scales, back)
        normal = np.where(np.abs(values) < 2.0 ** -126, 0.0, values)                 # a subnormal may be flushed
        b = np.where(np.abs(f64(back)) < 2.0 ** -126, 0.0, f64(back))
        assert np.array_equal(b, normal, equal_nan=True), t
    return codes, scales


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (1, 32), (3, 33), (15, 128), (16, 255), (17, 256), (33, 257), (5, 500), (2, 513),
                                       (130, 1000), (7, 4091), (64, 5120)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_quantise_is_exact(rows, cols, dtype):
    check_exact(data(rows, cols, dtype, rows + cols))


@pytest.mark.parametrize("B,H,N,D", [(1, 3, 21, 64), (2, 5, 19, 128), (2, 3, 17, 40), (1, 7, 33, 9), (3, 1, 16, 32)])
def test_quantise_heads_and_strides(B, H, N, D):
    x = data(B * H * N, D, torch.bfloat16, 3).view(B, H, N, D)
    check_exact(x)
    check_exact(x.transpose(1, 2).contiguous().transpose(1, 2))                       # heads between the tokens
    wide = data(B * H * N, D + 5, torch.float16, 4).view(B, H, N, D + 5)
    check_exact(wide[..., 3:3 + D])                                                   # no alignment
    check_exact(wide[:, :, :N - 2, :D])


def test_quantise_extremes():
    x = torch.zeros(8, 96)
    x[0, :9] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9])        # ties and saturation
    x[1, :3] = torch.tensor([3e38, -3.4e38, 1e38])
    x[2, 1], x[2, 40] = float("inf"), 1.0
    x[3, 33], x[3, 1] = float("nan"), -2.0
    x[4, :4] = torch.tensor([2.0 ** -126, 2.0 ** -127, 2.0 ** -130, -(2.0 ** -149)])  # subnormal blocks
    x[5, :2] = torch.tensor([2.0 ** -125, 2.0 ** -126 * 1.5])
    x[6, 32:64] = -1e-30
    x[7] = torch.arange(96) - 48.0
    check_exact(x.cuda())
    check_exact(x.to(torch.bfloat16).cuda())


@pytest.mark.parametrize("act", [S.SVG_ACT_SILU, S.SVG_ACT_GELU_TANH])
def test_quantise_behind_an_activation(act):
    x = data(40, 700, torch.float32, 5).clamp(-20, 20)
    codes, scales = quantise(x, act)
    v = ACT[act](f64(x))
    assert_four_bit(codes, scales, v, 16 * U * (np.abs(v) + np.abs(f64(x)) * np.exp(-np.abs(f64(x)))) + 1e-37)


# ---- products --------------------------------------------------------------------------------------

class Product:
    def __init__(self, M, N, K, seed=0, bias=True):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(M, K, generator=gen, device="cuda")
        w = torch.randn(N, K, generator=gen, device="cuda") / K ** 0.5
        self.a, self.w = quantise(x), quantise(w)
        self.bias = torch.randn(N, generator=gen, device="cuda") if bias else None
        values = lambda q, r: torch.from_numpy(O.mx_values(*O.from_operand(*(t.cpu().numpy() for t in q), r, K)))  # noqa: E731
        av, wv = values(self.a, M), values(self.w, N)
        self.sum = (av @ wv.t()).numpy() + (f64(self.bias) if bias else 0.0)
        # fp32 accumulation: at most one rounding or truncation (2^-23) of the running magnitude for each 32 columns, and a few at the end
        self.noise = (K / 32 + 16) * 2.0 ** -23 * ((av.abs() @ wv.abs().t()).numpy() + (np.abs(f64(self.bias)) if bias else 0.0))
        self.M, self.N, self.K = M, N, K
        n = S.svg_fp4_linear_workspace_bytes(M, N, K)
        self.ws, self.ws_bytes = (torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None), n

    def linear(self, out, act=S.SVG_ACT_NONE, stream=None):
        S.svg_fp4_linear(self.M, self.N, self.K, *self.a, *self.w, self.bias, act, S.tokens_of(out), out, self.ws, self.ws_bytes, stream)
        torch.cuda.synchronize()
        return out

    def expected(self, act):
        """(values, noise): the slopes of the activations are at most 1.13; their own arithmetic is 16 roundings of its terms."""
        v = ACT[act](self.sum)
        return v, 1.13 * self.noise + (16 * U * (np.abs(v) + np.abs(self.sum)) if act else 0.0)


SHAPES = [(1, 32, 32), (1, 1, 1), (2, 48, 300), (3, 1024, 512), (15, 96, 256), (16, 33, 1024), (17, 256, 640), (31, 130, 257), (32, 512, 2048),
          (33, 64, 1000), (48, 320, 768), (64, 256, 4096), (65, 100, 512), (100, 1000, 1100), (128, 128, 256), (129, 257, 512), (130, 384, 5120),
          (200, 640, 1536), (256, 256, 512), (300, 700, 900), (511, 520, 384), (513, 512, 512), (700, 1100, 130), (1000, 300, 2048), (1025, 2049, 256)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product_sizes(M, N, K):
    p = Product(M, N, K, M + N + K)
    out = p.linear(torch.full((M, N), float("nan"), device="cuda"))
    close(out, p.sum, U, p.noise, "out")
    codes, scales = buffers(M, N)
    S.svg_fp4_linear_quantize(M, N, K, *p.a, *p.w, p.bias, S.SVG_ACT_GELU_TANH, codes, scales, p.ws, p.ws_bytes)
    torch.cuda.synchronize()
    assert_four_bit(codes, scales, *p.expected(S.SVG_ACT_GELU_TANH))


@pytest.mark.parametrize("M,N,K", [(5, 192, 600), (70, 192, 600), (600, 192, 600)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("act", list(ACT))
def test_product_types_and_activations(M, N, K, dtype, act):
    p = Product(M, N, K, 11, bias=act != S.SVG_ACT_SILU)
    ref, noise = p.expected(act)
    close(p.linear(torch.full((M, N), float("nan"), dtype=dtype, device="cuda"), act), ref, HALF[dtype],
          noise + (2.0 ** -25 if dtype == torch.float16 else 0.0), "out")


@pytest.mark.parametrize("B,H,T,D", [(1, 3, 7, 64), (2, 4, 40, 128), (3, 5, 100, 24), (1, 2, 700, 64), (2, 3, 300, 10)])
def test_product_into_heads(B, H, T, D):
    p = Product(B * T, H * D, 300, 7)
    for t in (torch.bfloat16, torch.float32):
        out = p.linear(torch.full((B, H, T, D), float("nan"), dtype=t, device="cuda"))
        close(out.transpose(1, 2).reshape(B * T, H * D), p.sum, HALF[t], p.noise, "heads")
    rows = torch.full((B * T, H * D + 9), 7.0, device="cuda")                         # a row stride, no alignment
    p.linear(rows[:, 1:1 + H * D])
    close(rows[:, 1:1 + H * D], p.sum, U, p.noise, "rows")
    assert (rows[:, 0] == 7).all() and (rows[:, 1 + H * D:] == 7).all()


def test_product_of_bad_blocks():
    """A block that stands for NaNs reaches the outputs of its row, and no others."""
    x = torch.randn(40, 256, device="cuda")
    w = torch.randn(64, 256, device="cuda")
    x[7, 100], w[33, 5] = float("nan"), float("inf")
    for rows in (40, 8):
        a, q = quantise(x[:rows]), quantise(w)
        out = torch.zeros(rows, 64, device="cuda")
        S.svg_fp4_linear(rows, 64, 256, *a, *q, None, 0, S.tokens_of(out), out)
        torch.cuda.synchronize()
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[7], bad[:, 33] = True, True
        assert torch.equal(torch.isnan(out), bad)


@pytest.mark.parametrize("E", [-127, -100, 100, 125])
def test_product_at_the_ends_of_the_scale(E):
    """Powers of two far apart: the products' sizes cancel, and what underflows is zero."""
    x = torch.ones(3, 64, device="cuda") * 2.0 ** max(E, -126)
    w = torch.ones(32, 64, device="cuda") * 2.0 ** -max(min(E, 120), -120)
    out = torch.zeros(3, 32, device="cuda")
    S.svg_fp4_linear(3, 32, 64, *quantise(x), *quantise(w), None, 0, S.tokens_of(out), out)
    torch.cuda.synchronize()
    assert torch.equal(out, (x.double() @ w.double().t()).float())


def test_no_rows():
    p = Product(4, 32, 64)
    out = torch.full((4, 32), 7.0, device="cuda")
    S.svg_fp4_linear(0, 32, 64, *p.a, *p.w, None, 0, S.tokens_of(out[:0]), out)
    S.svg_fp4_linear_quantize(0, 32, 64, *p.a, *p.w, None, 0, *buffers(16, 32))
    S.svg_fp4_quantize(S.tokens_of(out[:0]), out, 0, *p.a)
    S.svg_fp4_dequantize(S.tokens_of(out[:0]), *p.a, out)
    torch.cuda.synchronize()
    assert (out == 7).all()


def test_products_repeat_and_run_on_other_streams_and_in_graphs():
    for M, N, K in ((2, 640, 2048), (90, 384, 1024), (700, 512, 768)):
        p = Product(M, N, K, 3)
        want = p.linear(torch.empty(M, N, device="cuda")).clone()
        assert torch.equal(p.linear(torch.empty(M, N, device="cuda")), want)
        side, out = torch.cuda.Stream(), torch.zeros(M, N, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        assert torch.equal(p.linear(out, stream=side), want)
        x, t = torch.randn(M, K, device="cuda"), None
        codes, scales = buffers(M, N)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            S.svg_fp4_quantize(S.tokens_of(x), x, S.SVG_ACT_SILU, *p.a)
            S.svg_fp4_linear(M, N, K, *p.a, *p.w, p.bias, 0, S.tokens_of(out), out, p.ws, p.ws_bytes)
            S.svg_fp4_linear_quantize(M, N, K, *p.a, *p.w, p.bias, 2, codes, scales, p.ws, p.ws_bytes)
        for k in range(3):
            x.copy_(torch.randn(M, K, device="cuda"))
            for t in (out, codes, scales):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            eager, ec, es = torch.empty_like(out), torch.zeros_like(codes), torch.zeros_like(scales)
            a = quantise(x, S.SVG_ACT_SILU)
            S.svg_fp4_linear(M, N, K, *a, *p.w, p.bias, 0, S.tokens_of(eager), eager, p.ws, p.ws_bytes)
            S.svg_fp4_linear_quantize(M, N, K, *a, *p.w, p.bias, 2, ec, es, p.ws, p.ws_bytes)
            torch.cuda.synchronize()
            assert torch.equal(out, eager) and torch.equal(codes, ec) and torch.equal(scales, es)


def test_matrices_past_32_bit_offsets():
    """130 000 x 20480 outputs: 2.7e9 elements; the attention's layout with 2.3e9 elements as the quantiser's input."""
    M, N, K = 130_000, 20_480, 256
    x = torch.zeros(M, K, device="cuda")
    w = torch.randn(N, K, device="cuda")
    sample = [0, 5, 52_428, 52_429, 104_857, 104_858, M - 2, M - 1]
    x[sample] = torch.randn(len(sample), K, device="cuda")
    a, q = quantise(x), quantise(w)
    out = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    S.svg_fp4_linear(M, N, K, *a, *q, None, 0, S.tokens_of(out), out)
    torch.cuda.synchronize()
    av = O.mx_values(*O.mx_quantise(f64(x[sample])))
    wv = O.mx_values(*O.mx_quantise(f64(w)))
    close(out[sample], av @ wv.T, 2.0 ** -8, 32 * 2.0 ** -23 * (np.abs(av) @ np.abs(wv).T), "out")
    assert not out[1].any() and not out[M - 3].any()
    codes, scales = buffers(M, N)
    S.svg_fp4_linear_quantize(M, N, K, *a, *q, None, 0, codes, scales)
    back = torch.full_like(out, 7.0)
    S.svg_fp4_dequantize(S.tokens_of(back), codes, scales, back)
    torch.cuda.synchronize()
    v, noise = av @ wv.T, 32 * 2.0 ** -23 * (np.abs(av) @ np.abs(wv).T)
    exact, low, high = (O.mx_values(*O.mx_quantise(t)) for t in (v, v - noise, v + noise))
    sure = (low == high) & (exact == low)                      # no border within the noise, and none of the block's scale
    assert sure.mean() > 0.99 and np.array_equal(f64(back[sample])[sure], exact[sure])
    assert not back[1].any() and not back[M - 3].any()
    del out, back, codes
    heads = torch.zeros(1, 40, 450_000, 128, dtype=torch.bfloat16, device="cuda")
    heads[0, :, [0, 449_999]] = torch.randn(40, 2, 128, device="cuda").to(torch.bfloat16)
    codes, scales = quantise(heads)
    back = torch.full((450_000, 5120), 7.0, dtype=torch.bfloat16, device="cuda")
    S.svg_fp4_dequantize(S.tokens_of(back), codes, scales, back)
    v = f64(heads[0, :, [0, 449_999]]).transpose(1, 0, 2).reshape(2, 5120)
    assert np.array_equal(f64(back[[0, 449_999]]), O.mx_values(*O.mx_quantise(v)))
    assert not back[1].any() and not back[449_998].any()


@pytest.mark.parametrize("rows", [1, 3, 4, 5, 13, 17])
@pytest.mark.parametrize("first", [0, 1, 2, 5])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantise_rows_that_begin_anywhere(rows, first, dtype):
    """Rows of an odd stride and width at every offset; what lies around a matrix that is read back stays."""
    wide = data(rows, 1049, dtype, rows + first)
    x = wide[:, first:first + 1031]
    codes, scales = check_exact(x)
    back = torch.full((rows + 2, 1049), 7.0, dtype=dtype, device="cuda")
    part = back[1:1 + rows, first:first + 1031]
    S.svg_fp4_dequantize(S.tokens_of(part), codes, scales, part)
    torch.cuda.synchronize()
    assert np.array_equal(f64(part), O.mx_values(*O.mx_quantise(f64(x))))
    part.fill_(7.0)
    assert (back == 7).all()


@pytest.mark.parametrize("M,N,K", [(500, 1280, 2560), (230, 2560, 5120), (1573, 1536, 1536), (600, 4100, 700)])
@pytest.mark.parametrize("act", [S.SVG_ACT_NONE, S.SVG_ACT_SILU, S.SVG_ACT_GELU_TANH])
def test_products_where_the_activation_decides_the_form(M, N, K, act):
    p = Product(M, N, K, M)
    ref, noise = p.expected(act)
    close(p.linear(torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda"), act), ref, HALF[torch.bfloat16], noise, "out")


def test_activations_far_from_zero():
    """Their exponentials overflow or vanish: silu and GELU are v on one side and zero on the other."""
    x = torch.tensor([[1e30, -1e30, 300.0, -300.0, 88.0, -88.0, 3e19, -3e19] * 4], device="cuda")
    w = torch.eye(32, device="cuda")
    for act in (S.SVG_ACT_SILU, S.SVG_ACT_GELU_TANH):
        for k in range(8):                                          # one magnitude at a time: a block of its own
            v = torch.zeros_like(x)
            v[0, k] = x[0, k]
            out = torch.full((1, 32), float("nan"), device="cuda")
            S.svg_fp4_linear(1, 32, 32, *quantise(v), *quantise(w), None, act, S.tokens_of(out), out)
            value = O.mx_values(*O.mx_quantise(f64(v)))[0, k]
            assert out[0, k].item() == (pytest.approx(value, rel=1e-6) if value > 0 else pytest.approx(0.0, abs=1e-30))


@pytest.mark.parametrize("act", [S.SVG_ACT_SILU, S.SVG_ACT_GELU_TANH])
@pytest.mark.parametrize("M", [1, 130])
def test_activations_relative_to_their_value(act, M):
    """The sum is zero, so an output is the activation of its bias, any fp32 number.  In units of 2^-24 of the value: the exponent is off by
    1.224 |v| (its constant 0.224, one product) and 7.23 |z| (constants 2.23 and 4.23, square 1, sum 1, product 1), which counts with the share
    1 - sigmoid; there also the exponential's unit in the last place (2); sum 1, reciprocal 2, product 1.  The reciprocal of what is above 2^126
    may be flushed: |v| 2^-126."""
    rng = np.random.default_rng(M)
    v = np.concatenate([np.linspace(-87, 87, 4096), rng.normal(size=3000) * 3, -np.geomspace(1e-30, 12, 1000), np.geomspace(1e-30, 12, 96)]).astype(np.float32)
    N, K = v.size, 64
    a, w = quantise(torch.zeros(M, K, device="cuda")), quantise(torch.randn(N, K, device="cuda"))
    out = torch.full((M, N), float("nan"), device="cuda")
    S.svg_fp4_linear(M, N, K, *a, *w, torch.from_numpy(v).cuda(), act, S.tokens_of(out), out)
    torch.cuda.synchronize()
    x = v.astype(np.longdouble)
    z = x if act == S.SVG_ACT_SILU else 2 * np.sqrt(np.longdouble(2) / np.longdouble(np.pi)) * (x + np.longdouble("0.044715") * x ** 3)
    near = np.exp(-np.abs(z))
    sigmoid, rest = np.where(z < 0, near, 1) / (1 + near), np.where(z < 0, 1, near) / (1 + near)
    ref = x * sigmoid
    units = ((1.224 if act == S.SVG_ACT_SILU else 7.23) * np.abs(z) + 2) * rest + 4
    allowed = units * U * np.abs(ref) * (1 + 1e-4) + np.abs(x) * 2.0 ** -126
    err = np.abs(f64(out).astype(np.longdouble) - ref)
    assert (err <= allowed).all(), (act, float((err / allowed).max()))
    assert torch.equal(out, out[:1].expand(M, N))


@pytest.mark.parametrize("rows,cols", [(1, 32), (17, 64), (33, 288), (70, 544), (500, 1312), (1030, 4128)])
def test_the_padding_of_every_writer_is_zero(rows, cols):
    """Codes and scale bytes behind the last row and column, in column tiles that exist: a product takes them as part of K."""
    x = torch.randn(rows, cols, device="cuda")
    w, a = quantise(torch.randn(cols, 64, device="cuda")), quantise(torch.randn(rows, 64, device="cuda"))
    bias = torch.full((cols,), 5.0, device="cuda")
    product, norm = buffers(rows, cols), buffers(rows, cols)
    S.svg_fp4_linear_quantize(rows, cols, 64, *a, *w, bias, S.SVG_ACT_NONE, *product)
    S.svg_gate_norm_fwd(S.gate_norm_desc(rows, cols, stream_type=S.SVG_F32, pre_norm=2, shift=bias), x, None, None, None, *norm)
    torch.cuda.synchronize()
    rt, ct = -(-rows // 16), -(-cols // 256) * 2
    for name, q in (("quantiser", quantise(x)), ("product", product), ("norm", norm)):
        codes, scales = O.from_operand(*(t.cpu().numpy() for t in q), rt * 16, ct * 128)
        assert not codes[rows:].any() and not codes[:, cols:].any(), name
        assert not scales[rows:].any() and not scales[:, -(-cols // 32):].any(), name
        assert scales[:rows, :cols // 32].all(), name
