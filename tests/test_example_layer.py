"""Refusals of the example's layer, on the host: what has another size than its buffers must not reach a kernel."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import transformer_layer as T  # noqa: E402


def operand(rows, cols):
    a = object.__new__(T.Operand)
    a.rows, a.cols, a.codes, a.scales = rows, cols, None, None
    return a


@pytest.mark.parametrize("shape", [(17, 64), (15, 64), (16, 65), (1, 2, 16, 64), (1, 2, 8, 64)])
def test_an_operand_takes_matrices_of_its_size_only(shape):
    with pytest.raises(ValueError, match="16 x 64"):
        operand(16, 64).write(torch.zeros(shape))


def test_a_layer_takes_inputs_of_its_shape_only():
    layer = object.__new__(T.Layer)
    layer.rows, layer.C, layer.B = 32, 64, 2
    x, emb = torch.zeros(32, 64, dtype=torch.bfloat16), torch.zeros(2, 64)
    for bad in (x[:31], x[:, :63], x.float(), x.t(), torch.zeros(64, 64, dtype=torch.bfloat16)[::2], torch.zeros(32, 128, dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError, match="x has to be"):
            layer.forward(bad, emb)


def test_a_projection_takes_operands_and_outputs_of_its_size_only():
    linear = object.__new__(T.Linear)
    linear.N, linear.K, linear.weight, linear.bias = 128, 64, operand(128, 64), None
    with pytest.raises(ValueError, match="64 columns"):
        linear(operand(16, 65), torch.zeros(16, 128))
    with pytest.raises(ValueError, match="64 columns"):
        linear.to_operand(operand(16, 32), operand(16, 128), 0)
    for rows, cols in ((15, 128), (16, 129)):
        with pytest.raises(ValueError, match="16 x 128"):
            linear.to_operand(operand(16, 64), operand(rows, cols), 0)
