"""What stands around the attention of a video transformer's layer, as cases that can be timed.

Two families of operators and the path that joins them:
  norm      svg_gate_norm_fwd: a branch's output through its norm and gate onto the residual stream, and the norm and
            modulation in front of the next branch
  norm_bwd  svg_gate_norm_bwd: its gradients, for the stream, the branch, the modulation tables and the norms' weights
  quant     svg_fp4_quantize and svg_fp4_dequantize: a tensor to microscaled 4-bit floating point and read back
  linear    svg_fp4_quantize of the activations, svg_fp4_linear with weights kept in 4 bits
  ffn       svg_gate_norm_fwd with a 4-bit output, svg_fp4_linear_quantize (GELU), svg_fp4_linear, svg_gate_norm_fwd

Where `own` is false the same is computed from elementary torch operations in 32 bits.

Microscaled 4-bit floating point (OCP MX, E2M1 elements with one E8M0 scale for 32 neighbours of a row):
E = clamp(floor(log2 max|v|) - 2, -127, 127), code = the E2M1 value nearest to v / 2^E, ties to even, at most 6.
A matrix of R rows and K columns is held in operand order: rows in tiles of 16, columns in tiles of 128; a tile is
64 pieces of 16 bytes, piece 16 g + i holding row i's columns 32 g to 32 g + 31, the even column of two in the low half of a byte
(rows padded to 16, columns to 256).  Scale bytes (E + 127): four column tiles together, [row tile][group][piece][column tile].
"""
from __future__ import annotations

import math

import torch

own = False

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_EPS = 1e-6


# ---------------------------------------------------------------------------------------------- the cases

def _norm(name, **kw):
    case = {"name": name, "op": "norm", "rows": 0, "C": 0, "groups": 1, "packed": False, "stream": "bf16", "branch": "bf16",
            "post": "none", "pre": "layer", "affine": False, "alpha": 1.0}
    case.update(kw)
    return case


def _quant(name, **kw):
    case = {"name": name, "op": "quant", "rows": 0, "K": 0, "heads": 0, "type": "bf16"}
    case.update(kw)
    return case


def _linear(name, **kw):
    case = {"name": name, "op": "linear", "M": 0, "N": 0, "K": 0, "type": "bf16", "out": "bf16", "heads": 0, "silu": False,
            "gelu": False}
    case.update(kw)
    return case


def _ffn(name, **kw):
    case = {"name": name, "op": "ffn", "rows": 0, "C": 0, "hidden": 0, "groups": 1, "packed": False, "pre": "layer"}
    case.update(kw)
    return case


def listed():
    return [
        # the smallest layer of the library's workloads: 272 tokens of 4 heads of 64; launches and latency are what counts
        _norm("norm_tiny", rows=272, C=256),
        # videos of different lengths packed into one call, an odd width, the stream kept in 32 bits, norms on both sides
        _norm("norm_packed_odd", rows=7013, C=1001, groups=5, packed=True, stream="f32", branch="f16", post="rms", pre="rms",
              affine=True, alpha=0.5),
        # the Wan2.1 shape: 21 x 1560 tokens of 40 heads of 128, parameter-free LayerNorm, one timestep
        _norm("norm_wan21", rows=32760, C=5120),
        # fine-tuning: gradients of a short packed batch with norms on both sides ...
        _norm("norm_bwd_packed", op="norm_bwd", rows=2971, C=1536, groups=4, packed=True, stream="f32", post="rms", pre="rms",
              affine=True),
        # ... and of one long video
        _norm("norm_bwd_wan21", op="norm_bwd", rows=32760, C=5120, affine=True),
        # text embeddings in half precision, a width that fills no block
        _quant("quant_text_odd", rows=226, K=4091, type="f16"),
        # the attention's output, [40 heads, tokens, 128], as the operand of the out projection
        _quant("quant_heads_wan21", rows=32760, K=5120, heads=40),
        # the modulation projection of a timestep (two guidance branches): six tables of 5120 from silu(embedding)
        _linear("linear_modulation", M=2, N=30720, K=5120, type="f32", out="f32", silu=True),
        # text tokens into the model's width
        _linear("linear_text", M=226, N=5120, K=4096, gelu=True),
        # the q projection, written as [40 heads, tokens, 128] for the attention
        _linear("linear_heads_wan21", M=32760, N=5120, K=5120, heads=40),
        # the feed-forward half of a small packed layer ...
        _ffn("ffn_packed", rows=1573, C=1536, hidden=6144, groups=3, packed=True, pre="rms"),
        # ... and of the Wan2.1 shape at four times its width
        _ffn("ffn_wan21", rows=32760, C=5120, hidden=20480),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def _width(rng, lo, hi, step):
    v = max(step, _log_int(rng, lo, hi) // step * step)
    return v + step if v == 3072 else v


def draw(rng):
    """One more case of the same operators with sizes of its own."""
    op = rng.choice(["norm", "norm", "norm_bwd", "quant", "linear", "linear", "ffn"])
    if op in ("norm", "norm_bwd"):
        C = _width(rng, 64, 8192, rng.choice([1, 8, 64]))
        rows = _log_int(rng, 1, min(120000, int(32760 * 5120 / C)))
        groups = rng.randint(1, min(8, rows))
        stream = rng.choice(["bf16", "bf16", "f32"])
        case = _norm("", op=op, rows=rows, C=C, groups=groups, packed=groups > 1, stream=stream,
                     branch=rng.choice(["bf16", "bf16", "f16"]), post=rng.choice(["none", "rms", "layer"]),
                     pre=rng.choice(["rms", "layer"]), affine=rng.random() < 0.5, alpha=rng.choice([1.0, 1.0, 0.7]))
    elif op == "quant":
        heads = rng.choice([0, rng.randint(2, 40)])
        K = heads * rng.choice([64, 128]) if heads else _width(rng, 32, 20480, rng.choice([1, 8, 32]))
        K = K + 128 if K == 3072 else K
        heads = K // 128 if heads and K % 128 == 0 else heads
        rows = _log_int(rng, 1, min(120000, int(32760 * 5120 / K)))
        case = _quant("", rows=rows, K=K, heads=heads, type=rng.choice(["bf16", "f16", "f32"]))
    elif op == "linear":
        K = _width(rng, 256, 8192, rng.choice([1, 32, 256]))
        N = _width(rng, 64, 20480, rng.choice([1, 64, 128]))
        M = _log_int(rng, 1, min(60000, int(2.5e12 / (2.0 * N * K))))
        heads = N // 64 if N % 64 == 0 and rng.random() < 0.3 else 0
        case = _linear("", M=M, N=N, K=K, type=rng.choice(["bf16", "bf16", "f16", "f32"]), out=rng.choice(["bf16", "bf16", "f16", "f32"]),
                       heads=heads, silu=rng.random() < 0.2, gelu=rng.random() < 0.3)
    else:
        C = _width(rng, 256, 5120, 64)
        hidden = _width(rng, 2 * C, 4 * C, 32)
        rows = _log_int(rng, 16, min(60000, int(6e12 / (4.0 * C * hidden))))
        groups = rng.randint(1, 4)
        case = _ffn("", rows=rows, C=C, hidden=hidden, groups=groups, packed=groups > 1, pre=rng.choice(["rms", "layer"]))
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _group_ptr(rows, groups, seed):
    """Ends of `groups` sequences of unlike lengths that fill `rows` rows."""
    share = torch.rand(groups, generator=torch.Generator().manual_seed(int(seed) + 5)) + 0.1
    ends = (torch.cumsum(share, 0) / share.sum() * rows).round().to(torch.int32)
    ends[-1] = rows
    return torch.cat([torch.zeros(1, dtype=torch.int32), ends]).cuda()


def _stream_rows(gen, rows, C, dtype):
    """A residual stream: some channels much larger than others, no zero mean."""
    x = _randn(gen, rows, C)
    x.mul_(torch.exp(0.6 * _randn(gen, 1, C))).add_(0.2 * _randn(gen, 1, C))
    return x.to(dtype)


def _operand_shape(rows, cols):
    """Row tiles, column tiles, and groups of four column tiles of a matrix in operand order."""
    tiles = -(-cols // 256) * 2
    return -(-rows // 16), tiles, -(-tiles // 4)


def _operand_buffers(rows, cols):
    rt, ct, groups = _operand_shape(rows, cols)
    return (torch.empty(rt * ct * 1024, dtype=torch.uint8, device="cuda"),
            torch.empty(rt * groups * 256, dtype=torch.uint8, device="cuda"))


def _weights(gen, N, K):
    """Weights as a program keeps them: 4-bit codes and scales in operand order."""
    rt, ct, groups = _operand_shape(N, K)
    w = torch.zeros(rt * 16, groups * 512, device="cuda")
    w[:N, :K] = _randn(gen, N, K) / math.sqrt(K)
    mag, exponent = _to_grid(w)
    code = torch.zeros_like(mag, dtype=torch.uint8)
    for edge in _GRID[1:]:
        code += mag >= edge
    code += 8 * torch.signbit(w).to(torch.uint8)
    pairs = (code[:, 0::2] | (code[:, 1::2] << 4))[:, :ct * 64]
    codes = pairs.view(rt, 16, ct, 4, 16).permute(0, 2, 3, 1, 4).contiguous().view(-1)
    scales = (exponent + 127).to(torch.uint8).view(rt, 16, groups, 4, 4).permute(0, 2, 4, 1, 3).contiguous().view(-1)
    return codes, scales


def prepare(case, seed):
    """Activations, parameters and buffers of one call in HBM."""
    gen, op, st = _gen(seed), case["op"], {"case": case}
    if op in ("norm", "norm_bwd"):
        rows, C, G = case["rows"], case["C"], case["groups"]
        stream, branch = _TYPES[case["stream"]], _TYPES[case["branch"]]
        st["mod"] = 0.3 * _randn(gen, G, 3 * C)           # gate | scale | shift, one row for each sequence
        st["group_ptr"] = _group_ptr(rows, G, seed) if case["packed"] else None
        for name in ("post_weight", "post_bias", "weight", "bias"):
            st[name] = None
        if case["affine"]:
            st["weight"] = 1.0 + 0.2 * _randn(gen, C)
            st["bias"] = 0.1 * _randn(gen, C) if case["pre"] == "layer" else None
            if case["post"] != "none":
                st["post_weight"] = 1.0 + 0.2 * _randn(gen, C)
                st["post_bias"] = 0.1 * _randn(gen, C) if case["post"] == "layer" else None
        st["y"] = (0.7 * _randn(gen, rows, C) + 0.1).to(branch)
        if op == "norm":
            st["x"] = _stream_rows(gen, rows, C, stream)
            st["r"], st["h"] = torch.empty_like(st["x"]), torch.empty_like(st["y"])
        else:
            st["r"] = _stream_rows(gen, rows, C, stream)
            st["dr"], st["dh"] = _randn(gen, rows, C).to(stream), _randn(gen, rows, C).to(branch)
            st["dx"], st["dy"] = torch.empty_like(st["r"]), torch.empty_like(st["y"])
            st["dmod"] = torch.empty_like(st["mod"])
            for name in ("post_weight", "post_bias", "weight", "bias"):
                st["d" + name] = torch.empty_like(st[name]) if st[name] is not None else None
        return st
    if op == "quant":
        rows, K, heads, dtype = case["rows"], case["K"], case["heads"], _TYPES[case["type"]]
        shape = (1, heads, rows, K // heads) if heads else (rows, K)
        x = _randn(gen, *shape)
        x.mul_(torch.exp(0.5 * _randn(gen, *shape[:-1], 1)))
        st["x"] = x.to(dtype)
        st["out"] = torch.empty(rows, K, dtype=torch.float32 if case["type"] == "f32" else torch.bfloat16, device="cuda")
        st["codes"], st["scales"] = _operand_buffers(rows, K)
        return st
    if op == "linear":
        M, N, K, heads = case["M"], case["N"], case["K"], case["heads"]
        st["x"] = _randn(gen, M, K).to(_TYPES[case["type"]])
        st["w"], st["w_scales"] = _weights(gen, N, K)
        st["bias"] = 0.1 * _randn(gen, N)
        st["a"], st["a_scales"] = _operand_buffers(M, K)
        st["out"] = torch.empty((1, heads, M, N // heads) if heads else (M, N), dtype=_TYPES[case["out"]], device="cuda")
        return st
    rows, C, hidden, G = case["rows"], case["C"], case["hidden"], case["groups"]
    st["x"] = _stream_rows(gen, rows, C, torch.bfloat16)
    st["y"] = (0.7 * _randn(gen, rows, C)).to(torch.bfloat16)
    st["mod"] = 0.3 * _randn(gen, G, 4 * C)               # gate of the attention | scale | shift | gate of the feed-forward
    st["group_ptr"] = _group_ptr(rows, G, seed) if case["packed"] else None
    st["up"], st["up_scales"] = _weights(gen, hidden, C)
    st["down"], st["down_scales"] = _weights(gen, C, hidden)
    st["up_bias"], st["down_bias"] = 0.1 * _randn(gen, hidden), 0.1 * _randn(gen, C)
    st["h"], st["h_scales"] = _operand_buffers(rows, C)
    st["u"], st["u_scales"] = _operand_buffers(rows, hidden)
    for name in ("r1", "z", "r2"):
        st[name] = torch.empty_like(st["x"])
    return st


# ---------------------------------------------------------------------------------------------- the framework's operators

def _own_desc(S, st, mod, C, rows, pre, post, stream, branch, **kw):
    types = {"bf16": S.SVG_BF16, "f16": S.SVG_F16, "f32": S.SVG_F32}
    norms = {"none": S.SVG_NORM_NONE, "rms": S.SVG_NORM_RMS, "layer": S.SVG_NORM_LAYER}
    return S.gate_norm_desc(rows=rows, channels=C, groups=mod.shape[0], group_ptr=st["group_ptr"], stream_type=types[stream],
                            branch_type=types[branch], pre_norm=norms[pre], post_norm=norms[post], eps=_EPS, post_eps=_EPS,
                            ld_mod=mod.shape[1], **kw)


def _run_own(st):
    import paper_2502_01776_amd as S
    case, op = st["case"], st["case"]["op"]
    if op in ("norm", "norm_bwd"):
        C, mod = case["C"], st["mod"]
        desc = _own_desc(S, st, mod, C, case["rows"], case["pre"], case["post"], case["stream"], case["branch"],
                         residual_scale=case["alpha"], gate=mod[:, :C], scale=mod[:, C:2 * C], shift=mod[:, 2 * C:],
                         post_weight=st["post_weight"], post_bias=st["post_bias"], weight=st["weight"], bias=st["bias"])
        if op == "norm":
            S.svg_gate_norm_fwd(desc, st["x"], st["y"], st["r"], st["h"])
            return {"r": st["r"], "h": st["h"]}
        dmod, n = st["dmod"], S.svg_gate_norm_workspace_bytes(desc)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        grads = S.gate_norm_grads(gate=dmod[:, :C], scale=dmod[:, C:2 * C], shift=dmod[:, 2 * C:], ld_mod=3 * C,
                                  post_weight=st["dpost_weight"], post_bias=st["dpost_bias"], weight=st["dweight"],
                                  bias=st["dbias"])
        S.svg_gate_norm_bwd(desc, st["r"], st["y"], st["dr"], st["dh"], st["dx"], st["dy"], grads, ws, n)
        return {k: st[k] for k in ("dx", "dy", "dmod", "dpost_weight", "dpost_bias", "dweight", "dbias")}
    if op == "quant":
        S.svg_fp4_quantize(S.tokens_of(st["x"]), st["x"], S.SVG_ACT_NONE, st["codes"], st["scales"])
        S.svg_fp4_dequantize(S.tokens_of(st["out"]), st["codes"], st["scales"], st["out"])
        return {"values": st["out"]}
    if op == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        n = S.svg_fp4_linear_workspace_bytes(M, N, K)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        S.svg_fp4_quantize(S.tokens_of(st["x"]), st["x"], S.SVG_ACT_SILU if case["silu"] else S.SVG_ACT_NONE, st["a"], st["a_scales"])
        S.svg_fp4_linear(M, N, K, st["a"], st["a_scales"], st["w"], st["w_scales"], st["bias"],
                         S.SVG_ACT_GELU_TANH if case["gelu"] else S.SVG_ACT_NONE, S.tokens_of(st["out"]), st["out"], ws, n)
        return {"out": st["out"]}
    rows, C, hidden, mod = case["rows"], case["C"], case["hidden"], st["mod"]
    n = max(S.svg_fp4_linear_workspace_bytes(rows, hidden, C), S.svg_fp4_linear_workspace_bytes(rows, C, hidden))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    before = _own_desc(S, st, mod, C, rows, case["pre"], "none", "bf16", "bf16", gate=mod[:, :C], scale=mod[:, C:2 * C],
                       shift=mod[:, 2 * C:3 * C])
    after = _own_desc(S, st, mod, C, rows, "none", "none", "bf16", "bf16", gate=mod[:, 3 * C:])
    S.svg_gate_norm_fwd(before, st["x"], st["y"], st["r1"], None, st["h"], st["h_scales"])
    S.svg_fp4_linear_quantize(rows, hidden, C, st["h"], st["h_scales"], st["up"], st["up_scales"], st["up_bias"],
                              S.SVG_ACT_GELU_TANH, st["u"], st["u_scales"], ws, n)
    S.svg_fp4_linear(rows, C, hidden, st["u"], st["u_scales"], st["down"], st["down_scales"], st["down_bias"], S.SVG_ACT_NONE,
                     S.tokens_of(st["z"]), st["z"], ws, n)
    S.svg_gate_norm_fwd(after, st["r1"], st["z"], st["r2"], None)
    return {"r1": st["r1"], "r2": st["r2"]}


# ---------------------------------------------------------------------------------------------- the plain form

def _scaled(v, exponent):
    """v * 2^exponent, exactly (powers of two from their bits, in two steps so that both are normal numbers)."""
    half = exponent // 2
    for e in (half, exponent - half):
        v = v * ((e + 127) << 23).view(torch.float32)
    return v


def _to_grid(v):
    """Magnitudes on the E2M1 grid and exponents of v [rows, multiple of 32] (32 bits; every step but the rounding is exact)."""
    blocks = v.view(v.shape[0], -1, 32)
    top = blocks.abs().amax(-1)
    exponent = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(-127, 127).to(torch.int32)
    t = _scaled(blocks.abs(), -exponent[..., None])
    step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
    return (torch.round(t / step) * step).clamp(max=6.0).view_as(v), exponent


def _fake_quant(v):
    """v [rows, K] in 32 bits -> the values that its microscaled 4-bit form stands for."""
    K = v.shape[1]
    if K % 32:
        v = torch.nn.functional.pad(v, (0, 32 - K % 32))
    mag, exponent = _to_grid(v)
    scaled = _scaled(mag.view(v.shape[0], -1, 32), exponent[..., None]).view_as(v)
    return torch.where(v < 0, -scaled, scaled)[:, :K]


def _unpack(codes, scales, rows, cols):
    """A matrix in operand order -> its values [rows, cols] in 32 bits."""
    rt, ct, groups = _operand_shape(rows, cols)
    pairs = codes.view(rt, ct, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(rt * 16, ct * 64)
    code = torch.stack([pairs & 15, pairs >> 4], -1).view(rt * 16, ct * 4, 32)
    table = torch.tensor(_GRID + tuple(-g for g in _GRID), device=codes.device)
    exponent = scales.view(rt, groups, 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(rt * 16, groups * 16)[:, :ct * 4].to(torch.int32) - 127
    return _scaled(table[code.to(torch.int32)], exponent[..., None]).view(rt * 16, ct * 128)[:rows, :cols]


def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _gelu(v):
    return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))


def _hat(v, kind):
    """The normalised rows and 1 / their deviation."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    rho = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + _EPS)
    return v * rho, rho


def _affine(v, weight, bias):
    v = v if weight is None else v * weight
    return v if bias is None else v + bias


def _group_of(st, rows, groups):
    row = torch.arange(rows, device="cuda")
    if st["group_ptr"] is None:
        return row // (rows // groups)
    return (row[:, None] >= st["group_ptr"][None, 1:-1]).sum(-1) if groups > 1 else row * 0


def _group_sums(v, index, groups):
    """Sums of v's rows over each group, [groups, C]."""
    if groups == 1:
        return v.sum(0, keepdim=True)
    member = (index[None, :] == torch.arange(groups, device=v.device)[:, None]).to(v.dtype)
    return member @ v


def _plain_norm_bwd(st):
    case = st["case"]
    C, G, alpha = case["C"], case["groups"], case["alpha"]
    index = _group_of(st, case["rows"], G)
    gate, scale = st["mod"][index, :C], st["mod"][index, C:2 * C]
    weight = 1.0 if st["weight"] is None else st["weight"]
    post_weight = 1.0 if st["post_weight"] is None else st["post_weight"]
    rhat, rho = _hat(st["r"].float(), case["pre"])
    dh = st["dh"].float()
    dn = dh * (1.0 + scale)
    e = dn * weight
    inner = e - rhat * (e * rhat).mean(-1, keepdim=True)
    if case["pre"] == "layer":
        inner = inner - e.mean(-1, keepdim=True)
    dr = st["dr"].float() + rho * inner
    y = st["y"].float()
    f = dr * gate
    yhat = y
    if case["post"] != "none":
        yhat, prho = _hat(y, case["post"])
        e = f * post_weight
        inner = e - yhat * (e * yhat).mean(-1, keepdim=True)
        if case["post"] == "layer":
            inner = inner - e.mean(-1, keepdim=True)
        dy = prho * inner
    else:
        dy = f
    p = _affine(yhat, st["post_weight"], st["post_bias"])
    n = _affine(rhat, st["weight"], st["bias"])
    dmod = torch.cat([_group_sums(dr * p, index, G), _group_sums(dh * n, index, G), _group_sums(dh, index, G)], 1)
    total = lambda have, v: None if have is None else v.sum(0)  # noqa: E731
    return {"dx": (alpha * dr).to(st["r"].dtype), "dy": dy.to(st["y"].dtype), "dmod": dmod,
            "dpost_weight": total(st["post_weight"], f * yhat), "dpost_bias": total(st["post_bias"], f),
            "dweight": total(st["weight"], dn * rhat), "dbias": total(st["bias"], dn)}


def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "norm_bwd":
        return _plain_norm_bwd(st)
    if op == "norm":
        C, mod = case["C"], st["mod"]
        index = _group_of(st, case["rows"], case["groups"])
        y = st["y"].float()
        if case["post"] != "none":
            y = _affine(_hat(y, case["post"])[0], st["post_weight"], st["post_bias"])
        r = case["alpha"] * st["x"].float() + mod[index, :C] * y
        n = _affine(_hat(r, case["pre"])[0], st["weight"], st["bias"])
        h = n * (1.0 + mod[index, C:2 * C]) + mod[index, 2 * C:]
        return {"r": r.to(st["x"].dtype), "h": h.to(st["y"].dtype)}
    if op == "quant":
        x = st["x"].float()
        if case["heads"]:
            x = x[0].transpose(0, 1).reshape(case["rows"], case["K"])
        return {"values": _fake_quant(x).to(st["out"].dtype)}
    if op == "linear":
        x = st["x"].float()
        a = _fake_quant(_silu(x) if case["silu"] else x)
        out = a @ _unpack(st["w"], st["w_scales"], case["N"], case["K"]).t() + st["bias"]
        out = _gelu(out) if case["gelu"] else out
        if case["heads"]:
            out = out.view(case["M"], case["heads"], -1).transpose(0, 1)[None]
        return {"out": out.to(st["out"].dtype).contiguous()}
    C, mod = case["C"], st["mod"]
    index = _group_of(st, case["rows"], case["groups"])
    r1 = st["x"].float() + mod[index, :C] * st["y"].float()
    h = _hat(r1, case["pre"])[0] * (1.0 + mod[index, C:2 * C]) + mod[index, 2 * C:3 * C]
    u = _gelu(_fake_quant(h) @ _unpack(st["up"], st["up_scales"], case["hidden"], C).t() + st["up_bias"])
    z = _fake_quant(u) @ _unpack(st["down"], st["down_scales"], C, case["hidden"]).t() + st["down_bias"]
    r2 = r1 + mod[index, 3 * C:] * z
    return {"r1": r1.to(st["x"].dtype), "r2": r2.to(st["x"].dtype)}


def run(state):
    """One pass through a case's operators and its outputs."""
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------- the same in 64 bits

def _exact_power(e):
    """2^e in 64 bits for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_mx(v):
    """Microscaled 4-bit values of v [rows, K] in 64 bits: the scale by comparison with powers of two, the code by
    comparison with the midpoints of neighbouring grid values (a tie goes to the even code)."""
    rows, K = v.shape
    out = torch.empty_like(v)
    mids = [(a + b) / 2 for a, b in zip(_GRID[:-1], _GRID[1:])]
    for k in range(0, K, 32 * 64):
        part = v[:, k:k + 32 * 64]
        n = part.shape[1]
        block = torch.zeros(rows, -(-n // 32) * 32, dtype=torch.float64, device=v.device)
        block[:, :n] = part.abs()
        block = block.view(rows, -1, 32)
        top = block.amax(-1, keepdim=True)
        E = torch.floor(torch.log2(top.clamp(min=1e-300)))
        E = torch.where(_exact_power(E) > top, E - 1, E)
        E = torch.where(_exact_power(E + 1) <= top, E + 1, E)
        size = _exact_power((E - 2).clamp(-127, 127))
        t = block / size
        value = torch.zeros_like(t)
        for i, mid in enumerate(mids):
            value += (_GRID[i + 1] - _GRID[i]) * ((t > mid) if i % 2 == 0 else (t >= mid))
        out[:, k:k + n] = (value * size).view(rows, -1)[:, :n].copysign(part)
    return out


def _exact_weights(st, name, N, K):
    """Values of a weight matrix, read piece by piece from its operand order."""
    rt, ct, groups = _operand_shape(N, K)
    grid = torch.tensor([s * g for s in (1, -1) for g in _GRID], dtype=torch.float64, device="cuda")
    codes = st[name].view(rt, ct, 64, 16)
    scales = st[name + "_scales"].view(rt, groups, 64, 4)
    w = torch.empty(rt * 16, ct * 128, dtype=torch.float64, device="cuda").view(rt, 16, ct, 128)
    for j in range(ct):
        for g in range(4):
            piece = codes[:, j, 16 * g:16 * g + 16].long()
            size = _exact_power(scales[:, j // 4, 16 * g:16 * g + 16, j % 4].long() - 127)[..., None]
            w[:, :, j, 32 * g:32 * g + 32:2] = grid[piece % 16] * size
            w[:, :, j, 32 * g + 1:32 * g + 32:2] = grid[piece // 16] * size
    return w.view(rt * 16, ct * 128)[:N, :K]


def _exact_normed(v, kind, weight, bias):
    """(normalised, with its weight and bias, deviation) of rows v in 64 bits."""
    centre = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    spread = (((v - centre) ** 2).mean(1, keepdim=True) + _EPS).sqrt() if kind != "none" else torch.ones_like(v[:, :1])
    hat = (v - centre) / spread
    full = hat * (weight.double() if weight is not None else 1.0) + (bias.double() if bias is not None else 0.0)
    return hat, full, spread


def _exact_spans(st, rows, groups):
    if st["group_ptr"] is None:
        return [(g * (rows // groups), (g + 1) * (rows // groups)) for g in range(groups)]
    ends = [0] + st["group_ptr"].tolist()[1:-1] + [rows]
    return list(zip(ends[:-1], ends[1:]))


def _exact_norm(st, case):
    C, mod = case["C"], st["mod"].double()
    r, h = torch.empty_like(st["x"], dtype=torch.float64), torch.empty_like(st["x"], dtype=torch.float64)
    for (lo, hi), m in zip(_exact_spans(st, case["rows"], case["groups"]), mod):
        p = _exact_normed(st["y"][lo:hi].double(), case["post"], st["post_weight"], st["post_bias"])[1]
        r[lo:hi] = case["alpha"] * st["x"][lo:hi].double() + m[:C] * p
        h[lo:hi] = _exact_normed(r[lo:hi], case["pre"], st["weight"], st["bias"])[1] * (1 + m[C:2 * C]) + m[2 * C:]
    return {"r": r, "h": h}


def _exact_norm_grad(g, hat, spread, kind):
    """Gradient of the rows behind a normalisation whose output's gradient is g: the part along the row itself, and for
    the layer form the mean, drop out."""
    if kind == "none":
        return g
    C = g.shape[1]
    g = g - hat * ((g * hat).sum(1, keepdim=True) / C) - (g.sum(1, keepdim=True) / C if kind == "layer" else 0)
    return g / spread


def _exact_norm_bwd(st, case):
    C, mod = case["C"], st["mod"].double()
    out = {k: torch.zeros_like(st[k], dtype=torch.float64) if st[k] is not None else None
           for k in ("dx", "dy", "dmod", "dpost_weight", "dpost_bias", "dweight", "dbias")}
    one = torch.ones(C, dtype=torch.float64, device="cuda")
    w, wp = (one if st[k] is None else st[k].double() for k in ("weight", "post_weight"))
    for g, (lo, hi) in enumerate(_exact_spans(st, case["rows"], case["groups"])):
        gate, scale = mod[g, :C], mod[g, C:2 * C]
        rhat, n, spread = _exact_normed(st["r"][lo:hi].double(), case["pre"], st["weight"], st["bias"])
        yhat, p, pspread = _exact_normed(st["y"][lo:hi].double(), case["post"], st["post_weight"], st["post_bias"])
        dh = st["dh"][lo:hi].double()
        dr = st["dr"][lo:hi].double() + _exact_norm_grad(dh * ((1 + scale) * w), rhat, spread, case["pre"])
        out["dx"][lo:hi] = case["alpha"] * dr
        out["dy"][lo:hi] = _exact_norm_grad(dr * (gate * wp), yhat, pspread, case["post"])
        out["dmod"][g] = torch.cat([(dr * p).sum(0), (dh * n).sum(0), dh.sum(0)])
        for key, part in (("dpost_weight", dr * gate * yhat), ("dpost_bias", dr * gate), ("dweight", dh * (1 + scale) * rhat),
                          ("dbias", dh * (1 + scale))):
            if out[key] is not None:
                out[key] += part.sum(0)
    return out


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "norm":
        return _exact_norm(st, case)
    if op == "norm_bwd":
        return _exact_norm_bwd(st, case)
    tanh_gelu = lambda v: v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))  # noqa: E731
    if op == "quant":
        x = st["x"].double()
        return {"values": _exact_mx(torch.cat(list(x[0]), 1) if case["heads"] else x)}
    if op == "linear":
        x = st["x"].double()
        a = _exact_mx(x * torch.sigmoid(x) if case["silu"] else x)
        out = a @ _exact_weights(st, "w", case["N"], case["K"]).t().contiguous() + st["bias"].double()
        out = tanh_gelu(out) if case["gelu"] else out
        if case["heads"]:
            out = torch.stack(out.chunk(case["heads"], 1))[None]
        return {"out": out}
    C, mod = case["C"], st["mod"].double()
    up = _exact_weights(st, "up", case["hidden"], C).t().contiguous()
    down = _exact_weights(st, "down", C, case["hidden"]).t().contiguous()
    r1, r2 = (torch.empty(case["rows"], C, dtype=torch.float64, device="cuda") for _ in range(2))
    for (lo, hi), m in zip(_exact_spans(st, case["rows"], case["groups"]), mod):
        for a in range(lo, hi, 8192):
            b = min(hi, a + 8192)
            r1[a:b] = st["x"][a:b].double() + m[:C] * st["y"][a:b].double()
            h = _exact_normed(r1[a:b], case["pre"], None, None)[0] * (1 + m[C:2 * C]) + m[2 * C:3 * C]
            u = tanh_gelu(_exact_mx(h) @ up + st["up_bias"].double())
            r2[a:b] = r1[a:b] + m[3 * C:] * (_exact_mx(u) @ down + st["down_bias"].double())
    return {"r1": r1, "r2": r2}


# ---------------------------------------------------------------------------------------------- what cannot be avoided

def work(case):
    """Bytes: inputs read once, outputs written once, weights in their 4.25 bits an element; between the steps of the
    feed-forward path nothing is counted but the stream.  Operations: the products; for the others those of the formulas."""
    size = {"bf16": 2.0, "f16": 2.0, "f32": 4.0}
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        n, tables = float(case["rows"]) * case["C"], 12.0 * case["groups"] * case["C"]
        s, b = size[case["stream"]], size[case["branch"]]
        if op == "norm":
            return {"bytes": n * 2 * (s + b) + tables, "flops": 20.0 * n}
        return {"bytes": n * 3 * (s + b) + 2 * tables, "flops": 40.0 * n}
    if op == "quant":
        n = float(case["rows"]) * case["K"]
        return {"bytes": n * (size[case["type"]] + (4.0 if case["type"] == "f32" else 2.0)), "flops": 10.0 * n}
    if op == "linear":
        M, N, K = float(case["M"]), float(case["N"]), float(case["K"])
        return {"bytes": M * K * size[case["type"]] + N * K * 0.53125 + M * N * size[case["out"]] + 4 * N, "flops": 2.0 * M * N * K}
    rows, C, hidden = float(case["rows"]), float(case["C"]), float(case["hidden"])
    return {"bytes": rows * C * 8 + 2 * C * hidden * 0.53125, "flops": 4.0 * rows * C * hidden}
