"""A whole transformer layer on the operators of the library: every stage against the 64-bit form of what the stage in front of it
wrote, and the whole under graph capture."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import transformer_layer as T  # noqa: E402
from oracle import block_oracle as O  # noqa: E402
from test_gpu_gate_norm import HALF, U, assert_four_bit, close, f64  # noqa: E402
from workloads import get_config  # noqa: E402

pytestmark = pytest.mark.gpu

BF16 = HALF[torch.bfloat16]


def values(a):
    return O.mx_values(*O.from_operand(a.codes.cpu().numpy(), a.scales.cpu().numpy(), a.rows, a.cols))


def product(a, linear):
    """a W^T + b of the operands in 64 bits and the noise of fp32 accumulation: one rounding (or truncation) of the running magnitude
    for each 32 columns, and a few at the end."""
    av, wv, b = torch.from_numpy(values(a)), torch.from_numpy(values(linear.weight)), f64(linear.bias)
    noise = (linear.K / 32 + 16) * 2.0 ** -23 * ((av.abs() @ wv.abs().t()).numpy() + np.abs(b))
    return (av @ wv.t()).numpy() + b, noise


def rows_of(x):
    return f64(x.transpose(1, 2).reshape(-1, x.shape[1] * x.shape[3]))


def normed(r, noise, scale, shift):
    """norm(r) (1 + scale) + shift and its fp32 noise, with `noise` on r: 64 roundings of each term."""
    hat, rho = O.normalise(r, O.NORM_LAYER, float(np.float32(1e-6)))
    h = hat * (1 + scale) + shift
    far = np.abs(hat) + np.abs(r).mean(1, keepdims=True) * rho
    own = 64 * U * far + 3 * noise.max(1, keepdims=True) * rho * (1 + np.abs(hat))
    return h, own * np.abs(1 + scale) + 64 * U * (np.abs(shift) + np.abs(h))


def activations(layer, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(layer.rows, layer.C, generator=gen, device="cuda").to(torch.bfloat16)
    return x, torch.randn(layer.B, layer.C, generator=gen, device="cuda")


@pytest.mark.parametrize("name", ["tiny", "mid64"])
def test_every_stage_follows_from_the_one_before(name):
    layer = T.Layer(get_config(name), widening=2, seed=3)
    x, emb = activations(layer, 5)
    out = layer.forward(x, emb)
    torch.cuda.synchronize()
    v, xs = O.silu(f64(emb)), f64(x)
    assert_four_bit(layer.emb.codes, layer.emb.scales, v, 16 * U * (np.abs(v) + np.abs(f64(emb)) * np.exp(-np.abs(f64(emb)))))
    close(layer.mod, *_split(product(layer.emb, layer.modulation), U), "modulation")
    group = np.arange(layer.rows) // (layer.rows // layer.B)
    gate1, scale1, shift1, gate2, scale2, shift2 = (t[group] for t in np.split(f64(layer.mod), 6, axis=1))
    assert_four_bit(layer.h1.codes, layer.h1.scales, *normed(xs, 0 * xs, scale1, shift1))
    close(torch.from_numpy(rows_of(layer.v)), *_split(product(layer.h1, layer.v_proj), BF16), "v")
    codes, scales = O.mx_quantise(rows_of(layer.o))
    assert np.array_equal(values(layer.o4), O.mx_values(codes, scales))
    close(layer.y, *_split(product(layer.o4, layer.o_proj), BF16), "y")
    r = xs + gate1 * f64(layer.y)
    noise = 64 * U * (np.abs(xs) + np.abs(gate1 * f64(layer.y)))
    close(layer.r, r, BF16, noise, "r")
    assert_four_bit(layer.h2.codes, layer.h2.scales, *normed(r, noise, scale2, shift2))
    u, noise = product(layer.h2, layer.up)
    g = O.gelu_tanh(u)
    assert_four_bit(layer.u.codes, layer.u.scales, g, 1.13 * noise + 16 * U * (np.abs(g) + np.abs(u)))
    close(layer.z, *_split(product(layer.u, layer.down), BF16), "z")
    r, z = f64(layer.r), f64(layer.z)
    close(out, r + gate2 * z, BF16, 64 * U * (np.abs(r) + np.abs(gate2 * z)), "out")


def _split(pair, half):
    return pair[0], half, pair[1]


def test_layer_replays_from_a_graph():
    layer = T.Layer(get_config("mid128"), widening=2, seed=1)
    x, emb = activations(layer, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward(x, emb)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.forward(x, emb)
    for replay in range(3):
        for t, new in zip((x, emb), activations(layer, 10 + replay)):
            t.copy_(new)
        want = layer.forward(x, emb).clone()
        labels = layer.labels.clone()
        for t in (layer.out, layer.r, layer.y, layer.z, layer.o, layer.mod):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.out, want) and torch.equal(layer.labels, labels)
