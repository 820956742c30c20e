"""Pins of the 64-bit forms that the operators around the attention are tested against (CPU)."""
import itertools

import numpy as np
import pytest
import torch

from oracle import block_oracle as O


def test_grid_codes_are_fixed_points_and_ties_go_to_even():
    v = np.zeros((1, 32))
    v[0, :8], v[0, 8:16] = O.GRID, -O.GRID
    codes, scales = O.mx_quantise(v)
    assert scales[0, 0] == 127 and codes[0, :8].tolist() == list(range(8)) and codes[0, 8:16].tolist() == list(range(8, 16))
    v = np.zeros((1, 32))
    v[0, :9] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9]
    codes, scales = O.mx_quantise(v)
    assert scales[0, 0] == 127                       # floor(log2 7.9) - 2 = 0
    assert O.GRID[codes[0, :9]].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]


def test_codes_are_nearest_by_search_and_scales_by_definition():
    rng = np.random.default_rng(1)
    v = rng.normal(size=(9, 160)) * np.exp(rng.normal(size=(9, 160)))
    codes, scales = O.mx_quantise(v)
    value = O.mx_values(codes, scales)
    for r, b in itertools.product(range(9), range(5)):
        block = v[r, 32 * b:32 * b + 32]
        E = int(np.floor(np.log2(np.abs(block).max()))) - 2
        assert scales[r, b] == E + 127
        for x, got in zip(block, value[r, 32 * b:32 * b + 32]):
            every = np.concatenate([O.GRID, -O.GRID]) * 2.0 ** E
            assert abs(got - x) <= np.abs(every - x).min() * (1 + 1e-12)


def test_scale_bytes_at_the_ends_and_bad_blocks():
    v = np.zeros((6, 32))
    v[1, 3] = 2.0 ** -140
    v[2, 3] = 3e38
    v[3, 3], v[3, 4] = np.inf, 1.0
    v[4, 3] = np.nan
    v[5, 3] = 2.0 ** -125
    codes, scales = O.mx_quantise(v)
    assert scales[:, 0].tolist() == [0, 0, 127 + 125, 255, 255, 0]
    assert not codes[0].any() and not codes[3].any() and O.GRID[codes[5, 3]] == 4.0


def test_operand_order_round_trip_and_one_piece():
    rng = np.random.default_rng(2)
    codes = rng.integers(0, 16, (37, 333)).astype(np.uint8)
    scales = rng.integers(0, 255, (37, 11)).astype(np.uint8)
    c, s = O.to_operand(codes, scales)
    assert c.size == 3 * 4 * 1024 and s.size == 3 * 1 * 256
    back = O.from_operand(c, s, 37, 333)
    assert np.array_equal(back[0], codes) and np.array_equal(back[1], scales)
    piece = c[((1 * 4 + 2) * 64 + 16 * 1 + 5) * 16:][:16]              # row 21, columns 2 * 128 + 32 ..
    assert np.array_equal(piece & 15, codes[21, 288:320:2]) and np.array_equal(piece >> 4, codes[21, 289:320:2])
    assert s[((1 * 1 + 0) * 64 + 16 * 1 + 5) * 4 + 2] == scales[21, 9]


def test_activations_are_torch_s():
    v = np.linspace(-9, 9, 301)
    t = torch.from_numpy(v)
    assert np.allclose(O.silu(v), torch.nn.functional.silu(t).numpy(), rtol=1e-13, atol=1e-15)
    assert np.allclose(O.gelu_tanh(v), torch.nn.functional.gelu(t, approximate="tanh").numpy(), rtol=1e-12, atol=1e-15)


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
def test_gradients_are_those_of_autograd_and_of_differences(post, pre):
    rng = np.random.default_rng(10 * post + pre)
    rows, C, G = 11, 24, 3
    ptr = [0, 4, 4, 11]                                                  # the middle group is empty
    group = O.group_of_rows(rows, G, ptr)
    assert group.tolist() == [0] * 4 + [2] * 7
    p = {k: rng.normal(size=(G, C)) for k in ("gate", "scale", "shift")}
    p.update({k: 1 + 0.3 * rng.normal(size=C) for k in ("post_weight", "post_bias", "weight", "bias")})
    x, y, dr, dh = (rng.normal(size=(rows, C)) + 0.3 for _ in range(4))
    kw = dict(alpha=0.8, post=post, pre=pre, post_eps=1e-3, eps=1e-2)

    def loss(x, y, p):
        r, h = O.gate_norm(x, y, group, p["gate"], p["scale"], p["shift"], kw["alpha"], post, pre, kw["post_eps"], kw["eps"],
                           p["post_weight"], p["post_bias"], p["weight"], p["bias"])
        return (dr * r + dh * h).sum(), r

    r = loss(x, y, p)[1]
    g = O.gate_norm_grad(r, y, dr, dh, group, G, p["gate"], p["scale"], post_weight=p["post_weight"], post_bias=p["post_bias"],
                         weight=p["weight"], bias=p["bias"], **kw)
    at = {"dx": x, "dy": y, **p}
    used = {"dx", "dy", "gate", "scale", "shift"} | ({"weight"} if pre else set()) | ({"bias"} if pre == 2 else set())
    used |= ({"post_weight"} if post else set()) | ({"post_bias"} if post == 2 else set())
    step = 1e-6
    for name in used:
        direction = rng.normal(size=at[name].shape)
        moved = []
        for s in (step, -step):
            q, xs, ys = dict(p), x, y
            if name == "dx":
                xs = x + s * direction
            elif name == "dy":
                ys = y + s * direction
            else:
                q[name] = p[name] + s * direction
            moved.append(loss(xs, ys, q)[0])
        slope = (moved[0] - moved[1]) / (2 * step)
        assert abs(slope - (g[name] * direction).sum()) <= 1e-6 * max(1.0, abs(slope)), name
    if post == 2 and pre == 2:                                           # and torch's own layer norm agrees
        t = {k: torch.from_numpy(v).requires_grad_() for k, v in at.items()}
        ln = lambda v, w, b, e: torch.nn.functional.layer_norm(v, (C,), w, b, e)  # noqa: E731
        gi = torch.from_numpy(group)
        rt = kw["alpha"] * t["dx"] + t["gate"][gi] * ln(t["dy"], t["post_weight"], t["post_bias"], kw["post_eps"])
        ht = ln(rt, t["weight"], t["bias"], kw["eps"]) * (1 + t["scale"][gi]) + t["shift"][gi]
        (torch.from_numpy(dr) * rt + torch.from_numpy(dh) * ht).sum().backward()
        for name in used:
            assert np.allclose(t[name].grad.numpy(), g[name], rtol=1e-9, atol=1e-10), name


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
def test_gradients_of_every_parameter_are_those_of_differences(post, pre):
    """Also of the weights and biases that a norm does not have: the forward pass takes no notice of them, so they have none.  Central
    differences in 64 bits: r and h are linear in what stands behind the second norm (a step of 1e-3 leaves 1e-13 of rounding); of what stands in
    front of it the third derivative's part is the square of a step of 1e-5.  1e-6 of the terms' size is allowed."""
    rng = np.random.default_rng(100 + 10 * post + pre)
    rows, C, G = 9, 16, 2
    group = O.group_of_rows(rows, G, [0, 5, 9])
    p = {k: rng.normal(size=(G, C)) for k in ("gate", "scale", "shift")}
    p.update({k: 1 + 0.3 * rng.normal(size=C) for k in ("post_weight", "post_bias", "weight", "bias")})
    x, y, dr, dh = (rng.normal(size=(rows, C)) + 0.3 for _ in range(4))

    def forward(**changed):
        q = {**p, **changed}
        return O.gate_norm(x, y, group, q["gate"], q["scale"], q["shift"], 0.8, post, pre, 1e-3, 1e-2, q["post_weight"], q["post_bias"],
                           q["weight"], q["bias"])
    g = O.gate_norm_grad(forward()[0], y, dr, dh, group, G, p["gate"], p["scale"], alpha=0.8, post=post, pre=pre, post_eps=1e-3, eps=1e-2,
                         post_weight=p["post_weight"], post_bias=p["post_bias"], weight=p["weight"], bias=p["bias"])
    there = {"weight": pre != 0, "bias": pre == 2, "post_weight": post != 0, "post_bias": post == 2}
    for name in ("weight", "bias", "post_weight", "post_bias", "gate", "scale", "shift"):
        direction = rng.normal(size=p[name].shape)
        step = 1e-3 if name in ("weight", "bias", "scale", "shift") else 1e-5
        (ra, ha), (rb, hb) = forward(**{name: p[name] + step * direction}), forward(**{name: p[name] - step * direction})
        slope = ((dr * (ra - rb)).sum() + (dh * (ha - hb)).sum()) / (2 * step)
        assert abs(slope - (g[name] * direction).sum()) <= 1e-6 * (np.abs(dr).sum() + np.abs(dh).sum()), name
        assert there.get(name, True) or (slope == 0 and not g[name].any()), name
