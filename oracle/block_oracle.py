"""Plain 64-bit forms of the operators around the attention: gate + residual + norm + modulation with its gradients, and
microscaled 4-bit floating point.  numpy, one formula at a time; shares nothing with the kernels."""
from __future__ import annotations

import numpy as np

NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])      # E2M1 magnitudes, by code


# ---- gate, residual, norm, modulation ------------------------------------------------------------

def group_of_rows(rows, groups, group_ptr=None):
    """Group of every row; the first and the last entry of group_ptr are taken as 0 and rows."""
    if group_ptr is None:
        return np.arange(rows) // max(1, rows // groups)
    return np.searchsorted(np.asarray(group_ptr)[1:-1], np.arange(rows), side="right")


def normalise(v, norm, eps):
    """(normalised rows, 1 / deviation)."""
    if norm == NORM_NONE:
        return v, np.ones((len(v), 1))
    c = v - v.mean(1, keepdims=True) if norm == NORM_LAYER else v
    rho = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    return c * rho, rho


def affine(hat, norm, weight, bias):
    if norm == NORM_NONE:
        return hat
    out = hat if weight is None else hat * weight
    return out + bias if norm == NORM_LAYER and bias is not None else out


def gate_norm(x, y, group, gate, scale, shift, alpha, post, pre, post_eps, eps, post_weight=None, post_bias=None, weight=None, bias=None):
    """(r, h); gate, scale, shift [groups, C] or None."""
    r = alpha * x
    if y is not None:
        p = affine(normalise(y, post, post_eps)[0], post, post_weight, post_bias)
        r = r + (p if gate is None else gate[group] * p)
    n = affine(normalise(r, pre, eps)[0], pre, weight, bias)
    h = n * (1.0 if scale is None else 1.0 + scale[group]) + (0.0 if shift is None else shift[group])
    return r, h


def _norm_grad(g, hat, rho, norm):
    if norm == NORM_NONE:
        return g
    out = g - hat * (g * hat).mean(1, keepdims=True)
    if norm == NORM_LAYER:
        out = out - g.mean(1, keepdims=True)
    return rho * out


def gate_norm_grad(r, y, dr, dh, group, groups, gate, scale, alpha, post, pre, post_eps, eps, post_weight=None, post_bias=None,
                   weight=None, bias=None):
    """Gradients of sum(dr * r + dh * h) by name; r is the stream that the forward pass gave.
    A weight or bias that a norm does not have (bias: layer form only) takes no part in it: its gradient is zero."""
    rows, C = r.shape
    one = np.ones((groups, C))
    gate = one if gate is None else gate
    scale = 0 * one if scale is None else scale
    w = np.ones(C) if weight is None or pre == NORM_NONE else weight
    wp = np.ones(C) if post_weight is None or post == NORM_NONE else post_weight
    d = np.zeros_like(r) if dr is None else dr.copy()
    out = {}
    sums = lambda v: np.stack([v[group == g].sum(0) for g in range(groups)])  # noqa: E731
    dh = np.zeros_like(r) if dh is None else dh
    hat, rho = normalise(r, pre, eps)
    dn = dh * (1.0 + scale[group])
    out["shift"], out["scale"] = sums(dh), sums(dh * affine(hat, pre, weight, bias))
    out["weight"], out["bias"] = ((dn * hat).sum(0) if pre != NORM_NONE else np.zeros(C)), (dn.sum(0) if pre == NORM_LAYER else np.zeros(C))
    d = d + _norm_grad(dn * w, hat, rho, pre)
    out["dx"] = alpha * d
    if y is None:
        out["dy"] = d * gate[group]
        return out
    hat, rho = normalise(y, post, post_eps)
    out["gate"] = sums(d * affine(hat, post, post_weight, post_bias))
    f = d * gate[group]
    out["post_weight"] = (f * hat).sum(0) if post != NORM_NONE else np.zeros(C)
    out["post_bias"] = f.sum(0) if post == NORM_LAYER else np.zeros(C)
    out["dy"] = _norm_grad(f * wp, hat, rho, post)
    return out


# ---- microscaled 4-bit floating point ------------------------------------------------------------

def mx_quantise(v):
    """v [rows, cols] in 64 bits -> (codes [rows, cols] with the sign in bit 3, scale bytes [rows, ceil(cols / 32)])."""
    rows, cols = v.shape
    blocks = np.zeros((rows, -(-cols // 32) * 32))
    blocks[:, :cols] = v
    blocks = blocks.reshape(rows, -1, 32)
    bad = ~np.isfinite(blocks).all(-1)
    blocks = np.where(bad[..., None], 0.0, blocks)
    top = np.abs(blocks).max(-1)
    E = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)
    E = np.clip(E, -127, 127)
    t = np.abs(np.ldexp(blocks, -E[..., None]))
    code = np.zeros(t.shape, dtype=np.uint8)
    for i in range(7):                                   # past the midpoint of codes i and i + 1; a tie goes to the even one
        mid = (GRID[i] + GRID[i + 1]) / 2
        code += (t > mid) if i % 2 == 0 else (t >= mid)
    code += 8 * np.signbit(blocks).astype(np.uint8)
    code = np.where(bad[..., None], 0, code).astype(np.uint8)
    return code.reshape(rows, -1)[:, :cols], np.where(bad, 255, E + 127).astype(np.uint8)


def mx_values(codes, scales):
    """The values that codes and scale bytes stand for."""
    rows, cols = codes.shape
    value = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    size = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return value * np.repeat(size, 32, axis=1)[:, :cols]


def operand_shape(rows, cols):
    tiles = -(-cols // 256) * 2
    return -(-rows // 16), tiles, -(-tiles // 4)


def to_operand(codes, scales):
    """Operand order: (bytes of the codes, bytes of the scales); the scale bytes of column tiles that do not exist are zero."""
    rows, cols = codes.shape
    rt, ct, groups = operand_shape(rows, cols)
    full = np.zeros((rt * 16, ct * 128), dtype=np.uint8)
    full[:rows, :cols] = codes
    sc = np.zeros((rt * 16, groups * 16), dtype=np.uint8)
    sc[:rows, :scales.shape[1]] = scales
    out = np.zeros((rt, ct, 64, 16), dtype=np.uint8)
    osc = np.zeros((rt, groups, 64, 4), dtype=np.uint8)
    for g in range(4):
        for i in range(16):
            block = full[i::16].reshape(rt, ct, 4, 32)[:, :, g]
            out[:, :, 16 * g + i] = block[..., 0::2] | (block[..., 1::2] << 4)
            osc[:, :, 16 * g + i] = sc[i::16].reshape(rt, groups, 4, 4)[..., g]
    return out.reshape(-1), osc.reshape(-1)


def from_operand(codes, scales, rows, cols):
    rt, ct, groups = operand_shape(rows, cols)
    c = np.asarray(codes).reshape(rt, ct, 64, 16)
    s = np.asarray(scales).reshape(rt, groups, 64, 4)
    full = np.zeros((rt * 16, ct * 128), dtype=np.uint8)
    sc = np.zeros((rt * 16, groups * 16), dtype=np.uint8)
    for g in range(4):
        for i in range(16):
            piece = c[:, :, 16 * g + i]
            block = np.stack([piece & 15, piece >> 4], -1).reshape(rt, ct, 32)
            full[i::16].reshape(rt, ct, 4, 32)[:, :, g] = block
            sc[i::16].reshape(rt, groups, 4, 4)[..., g] = s[:, :, 16 * g + i]
    return full[:rows, :cols], sc[:rows, :-(-cols // 32)]


def silu(v):
    return v / (1.0 + np.exp(-v))


def gelu_tanh(v):
    return 0.5 * v * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (v + 0.044715 * v ** 3)))
