"""Few rows times 4-bit weights against the 64-bit form over the same operand.

Tolerance: every product is exact, so what is off is the fp32 accumulation (2^-23 of the magnitude summed for each of ceil(K / 32) additions in at most
three sums, and 16), the activations' bound of the header and one rounding to the output's type."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import block_oracle as O
from test_gpu_gate_norm import HALF, close, f64

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACT = {S.SVG_ACT_NONE: lambda v: v, S.SVG_ACT_SILU: O.silu, S.SVG_ACT_GELU_TANH: O.gelu_tanh}
SLOPE = {S.SVG_ACT_NONE: 1.0, S.SVG_ACT_SILU: 1.1, S.SVG_ACT_GELU_TANH: 1.13}      # the largest slope of each


def weights(N, K, seed, spread=1.0):
    w = np.random.default_rng(seed).standard_normal((N, K)) * np.exp(spread * np.random.default_rng(seed + 1).standard_normal((N, 1))) / np.sqrt(K)
    codes, scales = O.mx_quantise(w)
    dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda().view(torch.uint8).flatten() for x in O.to_operand(codes, scales)]
    return dev, O.mx_values(codes, scales)


def act_noise(z, act):
    """The activations' own bound, for arguments z in 64 bits."""
    if act == S.SVG_ACT_NONE:
        return 0 * z
    size = np.abs(ACT[act](z))
    inner = np.abs(z) * 1.3 if act == S.SVG_ACT_SILU else 7.3 * np.abs(1.596 * (z + 0.0447 * z ** 3))
    return 2.0 ** -24 * size * (8 + np.where(z < 0, inner, 0)) + 2e-36


def check(x, N, act_in=0, act=0, bias=True, out=None, out_type=torch.float32, seed=0):
    xv = f64(x)
    xv = xv if xv.ndim == 2 else xv.transpose(0, 2, 1, 3).reshape(xv.shape[0] * xv.shape[2], -1)
    M, K = xv.shape
    (codes, scales), w = weights(N, K, seed)
    b = torch.randn(N, generator=torch.Generator().manual_seed(seed)).cuda() if bias else None
    out = torch.full((M, N), 7.0, dtype=out_type, device="cuda") if out is None else out
    S.svg_fp4_linear_rows(S.tokens_of(x), x, act_in, N, codes, scales, b, act, S.tokens_of(out), out)
    torch.cuda.synchronize()
    a = ACT[act_in](xv)
    z = a @ w.T + (f64(b) if bias else 0)
    size = np.abs(a) @ np.abs(w).T + (np.abs(f64(b)) if bias else 0)
    noise = size * (3 * -(-K // 32) + 16) * 2.0 ** -23 + act_noise(xv, act_in) @ np.abs(w).T
    noise = noise * SLOPE[act] + act_noise(z, act)
    got = f64(out)
    got = got if got.ndim == 2 else got.transpose(0, 2, 1, 3).reshape(M, N)
    close(torch.from_numpy(got), ACT[act](z), HALF[out.dtype], noise, (M, N, K))
    return out, codes, scales, b


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M, N, K", [(1, 1, 1), (1, 16, 32), (1, 17, 33), (2, 31, 127), (3, 100, 128), (5, 257, 129), (6, 64, 1000), (8, 1001, 1537),
                                     (11, 48, 256), (16, 33, 513), (17, 130, 300), (33, 20, 700), (1, 5000, 257), (100, 70, 64)])
def test_sizes_and_types(M, N, K, kind):
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M + N + K)).to(TYPES[kind]).cuda()
    for out_type in TYPES.values():
        check(x, N, out_type=out_type, seed=M)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("act_in", list(ACT))
@pytest.mark.parametrize("act", list(ACT))
def test_activations(act, act_in, kind):
    for M, scale in ((1, 1.0), (4, 8.0), (7, 30.0)):
        x = (scale * torch.randn(M, 700, generator=torch.Generator().manual_seed(M))).to(TYPES[kind]).cuda()
        check(x, 150, act_in, act, bias=M != 4, seed=M)


@pytest.mark.parametrize("M, N, K, kind", [(1, 9000, 64, "f32"), (2, 17000, 128, "bf16"), (16, 17000, 160, "f32"), (4, 300, 20000, "f32"),
                                           (16, 40, 9000, "f32"), (3, 16, 70000, "bf16"), (16, 8200, 40, "f16"), (8, 8190, 4001, "f32"), (16, 8190, 2600, "f32")])
def test_forms(M, N, K, kind):
    """Two and eight wavefronts to a column of tiles, one to three blocks of columns, activations in more pieces than LDS holds at a time."""
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(K)).to(TYPES[kind]).cuda()
    check(x, N, seed=M, out_type=torch.bfloat16)


@pytest.mark.parametrize("N", [8192, 12280, 20480, 30715])
@pytest.mark.parametrize("M", [1, 8, 16])
def test_row_tiles_to_a_workgroup(M, N):
    """Two, three, five and four of them, with one to three blocks of columns."""
    x = torch.randn(M, 640, generator=torch.Generator().manual_seed(N)).cuda()
    check(x, N, seed=M)


def test_layouts():
    """Heads, views with odd strides and rows that are not aligned, in and out."""
    gen = torch.Generator().manual_seed(1)
    heads = torch.randn(2, 4, 3, 64, generator=gen).to(torch.bfloat16).cuda()
    check(heads, 96, out=torch.zeros(2, 3, 2, 48, device="cuda", dtype=torch.float16).transpose(1, 2))
    narrow = torch.randn(1, 5, 3, 7, generator=gen).cuda()               # heads of seven columns
    check(narrow, 35, out=torch.zeros(1, 5, 3, 7, device="cuda"))
    for kind in TYPES.values():
        wide = torch.randn(5, 321, generator=gen).to(kind).cuda()
        for first in (0, 1, 3):
            target = torch.full((5, 99), 7.0, dtype=kind, device="cuda")
            check(wide[:, first:first + 301], 77, out=target[:, 11:88])
            assert (target[:, :11] == 7).all() and (target[:, 88:] == 7).all()


def test_values_far_apart_keep_their_bits():
    """fp32 activations over the whole range of exponents: sums as exact as fp32 allows."""
    gen = torch.Generator().manual_seed(2)
    x = (torch.randn(3, 512, generator=gen) * torch.exp2(torch.randint(-60, 60, (3, 512), generator=gen).float())).cuda()
    check(x, 64)
    check(torch.full((2, 256), 3.4028234e38, device="cuda") * torch.tensor([[1.0], [2.0 ** -120]], device="cuda") * 2.0 ** -4, 32, bias=False)


def test_rows_that_are_not_finite_spoil_themselves_only():
    x = torch.randn(4, 300, generator=torch.Generator().manual_seed(3)).cuda()
    want, codes, scales, b = check(x, 130)
    for value in (float("inf"), -float("inf"), float("nan")):
        y = x.clone()
        y[1, 77] = value
        got = torch.zeros_like(want)
        S.svg_fp4_linear_rows(S.tokens_of(y), y, 0, 130, codes, scales, b, 0, S.tokens_of(got), got)
        assert torch.equal(got[[0, 2, 3]], want[[0, 2, 3]]) and not torch.isfinite(got[1]).any()


def test_results_repeat_and_do_not_depend_on_the_other_rows():
    x = torch.randn(40, 900, generator=torch.Generator().manual_seed(4)).cuda()
    want, codes, scales, b = check(x, 300)
    again = torch.zeros_like(want)
    S.svg_fp4_linear_rows(S.tokens_of(x), x, 0, 300, codes, scales, b, 0, S.tokens_of(again), again)
    assert torch.equal(again, want)
    one = torch.zeros(1, 300, device="cuda")
    S.svg_fp4_linear_rows(S.tokens_of(x[21:22]), x[21:22], 0, 300, codes, scales, b, 0, S.tokens_of(one), one)
    assert torch.equal(one[0], want[21])


def test_the_same_operand_as_the_products_of_4_bit_activations():
    """Activations that 4 bits hold exactly: svg_fp4_linear of their operand computes the same sums."""
    K, N, M = 512, 200, 5
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -1.0, -3.0])
    x = grid[torch.randint(0, 10, (M, K), generator=torch.Generator().manual_seed(5))].cuda()
    x[:, ::32] = 6.0                                                     # every block's scale is one
    w = torch.randn(N, K, generator=torch.Generator().manual_seed(6)).cuda()
    bytes_ = lambda r, c: [torch.zeros(S.svg_fp4_buffer_bytes(r, c, p), dtype=torch.uint8, device="cuda") for p in (0, 1)]  # noqa: E731
    wq, xq = bytes_(N, K), bytes_(M, K)
    S.svg_fp4_quantize(S.tokens_of(w), w, 0, *wq)
    S.svg_fp4_quantize(S.tokens_of(x), x, 0, *xq)
    a, b = (torch.zeros(M, N, device="cuda") for _ in range(2))
    S.svg_fp4_linear(M, N, K, *xq, *wq, None, 0, S.tokens_of(a), a)
    S.svg_fp4_linear_rows(S.tokens_of(x), x, 0, N, *wq, None, 0, S.tokens_of(b), b)
    values = torch.zeros(N, K, device="cuda")
    S.svg_fp4_dequantize(S.tokens_of(values), *wq, values)
    size = f64(x.abs()) @ f64(values.abs()).T
    assert (np.abs(f64(a) - f64(b)) <= size * (2 * K / 32 + 32) * 2.0 ** -23).all()


@pytest.mark.parametrize("M, N", [(1, 40), (5, 40), (3, 400)])
def test_blocks_of_every_magnitude(M, N):
    """Scale bytes at both ends of their range, blocks of zeros, and blocks that are not finite, which spoil their own output only."""
    K = 384
    gen = torch.Generator().manual_seed(N + M)
    w = torch.randn(N, K, generator=gen)
    w[0, 32:64] = 0.0
    w[1] *= 2.0 ** -126                                                  # bytes around 0: powers of two that are no normal fp32 numbers
    w[2] *= 2.0 ** 124
    w[3] = 0.0
    w[3, 200] = 2.0 ** -125
    w[4, 100], w[5, 383], w[6, 0] = float("nan"), float("inf"), -float("inf")
    w = w.cuda()
    operand = [torch.zeros(S.svg_fp4_buffer_bytes(N, K, p), dtype=torch.uint8, device="cuda") for p in (0, 1)]
    S.svg_fp4_quantize(S.tokens_of(w), w, 0, *operand)
    values = torch.zeros(N, K, device="cuda")
    S.svg_fp4_dequantize(S.tokens_of(values), *operand, values)
    values = f64(values)
    spoilt = [4, 5, 6]
    assert np.isnan(values[spoilt]).any(1).all() and np.isfinite(np.delete(values, spoilt, 0)).all() and values[3, 200] != 0
    kept = np.setdiff1d(np.arange(N), spoilt)
    for kind, power in (("f32", 100), ("bf16", 100), ("f32", -5), ("f16", 3)):
        x = (torch.randn(M, K, generator=gen) * 2.0 ** power).to(TYPES[kind]).cuda()
        out = torch.zeros(M, N, device="cuda")
        S.svg_fp4_linear_rows(S.tokens_of(x), x, 0, N, *operand, None, 0, S.tokens_of(out), out)
        got, xv = f64(out), f64(x)
        assert np.isnan(got[:, spoilt]).all()
        want, size = xv @ values[kept].T, np.abs(xv) @ np.abs(values[kept]).T
        # sums beyond the largest number of fp32 may be infinite; parts of products below its smallest normal number may be lost
        fits = size < 2.0 ** 127
        noise = size * (3 * -(-K // 32) + 16) * 2.0 ** -23 + 3 * K * 2.0 ** -126
        assert fits[:, kept != 2].all() and (np.abs(got[:, kept] - want)[fits] <= noise[fits]).all(), (kind, power)
