"""Every form of a product, its loops, tails and second turns on dense random operands: fp32 rows against the 64-bit form, and all other
outputs, whose arithmetic is the same, bit for bit against those."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import block_oracle as O
from product_forms import PRODUCTS
from test_gpu_fp4 import buffers, quantise
from test_gpu_gate_norm import U

pytestmark = pytest.mark.gpu


def values(q, rows, cols):
    return torch.from_numpy(O.mx_values(*O.from_operand(*(t.cpu().numpy() for t in q), rows, cols))).cuda()


@pytest.mark.parametrize("M,N,K,D", PRODUCTS)
def test_every_form(M, N, K, D):
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    a = quantise(torch.randn(M, K, generator=gen, device="cuda") * torch.exp(torch.randn(M, 1, generator=gen, device="cuda")))
    w = quantise(torch.randn(N, K, generator=gen, device="cuda") / K ** 0.5)
    bias = torch.randn(N, generator=gen, device="cuda")

    def product(out, act):
        S.svg_fp4_linear(M, N, K, *a, *w, bias, act, S.tokens_of(out), out)
        return out
    full = lambda *shape, t=torch.float32: torch.full(shape, float("nan"), dtype=t, device="cuda")  # noqa: E731
    av, wv = values(a, M, K), values(w, N, K)
    total = av @ wv.t() + bias.double()
    # fp32 accumulation: at most one rounding or truncation (2^-23) of the running magnitude for each 32 columns, and a few at the end
    noise = (K / 32 + 16) * 2.0 ** -23 * (av.abs() @ wv.abs().t() + bias.double().abs())
    for act in (S.SVG_ACT_NONE, S.SVG_ACT_GELU_TANH):
        out = product(full(M, N), act)
        if act:
            # 16 roundings of the activation's own on top of its slope, at most 1.13
            ref = 0.5 * total * (1 + torch.tanh(np.sqrt(2 / np.pi) * (total + 0.044715 * total ** 3)))
            allowed = 1.13 * noise + 16 * U * (ref.abs() + total.abs())
        else:
            ref, allowed = total, noise
        err = (out.double() - ref).abs()
        assert (err <= U * ref.abs() + (1 + U) * allowed).all(), (act, (err / allowed).max().item())
        for t in (torch.bfloat16, torch.float16):
            assert torch.equal(product(full(M, N, t=t), act), out.to(t)), (act, t)
        for first, stride in ((1, N + 9), (8, N + 24)):                     # no alignment, and with it
            rows = torch.full((M, stride), 7.0, dtype=torch.bfloat16, device="cuda")
            product(rows[:, first:first + N], act)
            assert torch.equal(rows[:, first:first + N], out.to(torch.bfloat16)), (act, first)
            assert (rows[:, :first] == 7).all() and (rows[:, first + N:] == 7).all(), (act, first)
        B = 2 if M % 2 == 0 else 1
        heads = product(full(B, N // D, M // B, D, t=torch.bfloat16), act)
        assert torch.equal(heads.transpose(1, 2).reshape(M, N), out.to(torch.bfloat16)), act
        codes, scales = buffers(M, N)
        S.svg_fp4_linear_quantize(M, N, K, *a, *w, bias, act, codes, scales)
        want, want_scales = quantise(out)
        used = (-(-N // 256) * 2 - 1) % 4 + 1                                # column tiles of the last group that exist
        got, ref_scales = (t.view(-1, 64, 4) for t in (scales, want_scales))
        groups = -(-(-(-N // 256) * 2) // 4)
        last = torch.arange(got.shape[0], device="cuda") % groups == groups - 1
        keep = (torch.arange(4, device="cuda")[None, None, :] < used) | ~last[:, None, None]
        assert torch.equal(codes, want) and torch.equal(got * keep, ref_scales * keep), act
