"""One layer of a video diffusion transformer on this library's operators.

The residual stream stays in bf16 and attention runs in bf16 over the profiled heads' tile lists; the six projections'
weights are kept as microscaled 4-bit operands and their inputs are written in that form by the operator in front of them:

    mod      = silu(embedding) Wm^T + bm                           gate, scale, shift of both halves, a row for each video
    h        = norm(x) (1 + scale1) + shift1                       in 4 bits
    q, k, v  = h Wq^T, h Wk^T, h Wv^T                              as [B, H, N, D]; QK-norm and rotary embedding of q and k
    o        = sparse attention of q, k, v by each head's pattern
    r        = x + gate1 (o Wo^T + bo);  h = norm(r) (1 + scale2) + shift2      one pass, h in 4 bits
    u        = gelu(h Wu^T + bu)                                   in 4 bits
    out      = r + gate2 (u Wd^T + bd)

    python examples/transformer_layer.py --workload wan21_14b      # times a layer of that shape

Nothing is allocated and nothing waits for the host after construction, so `forward` can be captured into a graph.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2502_01776_amd as S  # noqa: E402
from workloads import CONFIGS, get_config, sample_rows  # noqa: E402


class Operand:
    """A matrix of `rows` x `cols` as a microscaled 4-bit operand."""

    def __init__(self, rows, cols):
        self.rows, self.cols = rows, cols
        self.codes, self.scales = (torch.empty(S.svg_fp4_buffer_bytes(rows, cols, part), dtype=torch.uint8, device="cuda")
                                   for part in (S.SVG_FP4_CODES, S.SVG_FP4_SCALES))

    def write(self, x, activation=S.SVG_ACT_NONE):
        tokens = S.tokens_of(x)
        if (tokens.B * tokens.N, tokens.H * tokens.D) != (self.rows, self.cols):
            raise ValueError(f"the operand is {self.rows} x {self.cols}, not {tokens.B * tokens.N} x {tokens.H * tokens.D}")
        S.svg_fp4_quantize(tokens, x, activation, self.codes, self.scales)
        return self


class Linear:
    """A projection whose weights are kept in 4 bits."""

    def __init__(self, weight, bias=None):
        self.N, self.K = weight.shape
        self.weight, self.bias = Operand(self.N, self.K).write(weight), bias

    def _operands(self, a):
        if a.cols != self.K:
            raise ValueError(f"the projection's operand has {self.K} columns, not {a.cols}")
        bytes_ = S.svg_fp4_linear_workspace_bytes(a.rows, self.N, self.K)
        workspace = torch.empty(bytes_, dtype=torch.uint8, device="cuda") if bytes_ else None
        return (a.rows, self.N, self.K, a.codes, a.scales, self.weight.codes, self.weight.scales, self.bias), (workspace, bytes_)

    def __call__(self, a, out, activation=S.SVG_ACT_NONE):
        product, workspace = self._operands(a)
        S.svg_fp4_linear(*product, activation, S.tokens_of(out), out, *workspace)
        return out

    def to_operand(self, a, out, activation):
        product, workspace = self._operands(a)
        if (out.rows, out.cols) != (a.rows, self.N):
            raise ValueError(f"the projection's result is {a.rows} x {self.N}, not {out.rows} x {out.cols}")
        S.svg_fp4_linear_quantize(*product, activation, out.codes, out.scales, *workspace)
        return out


class Layer:
    def __init__(self, cfg, widening=4, seed=0):
        self.cfg, self.shape = cfg, S.shape_from_config(cfg)
        B, H, N, D = (cfg[k] for k in ("B", "H", "N", "D"))
        C, hidden, rows = H * D, widening * H * D, B * N
        self.C, self.rows, self.B = C, rows, B
        gen = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        linear = lambda n, k: Linear((randn(n, k) / math.sqrt(k)).to(torch.bfloat16), 0.1 * randn(n))  # noqa: E731
        self.modulation = linear(6 * C, C)
        self.q_proj, self.k_proj, self.v_proj, self.o_proj = (linear(C, C) for _ in range(4))
        self.up, self.down = linear(hidden, C), linear(C, hidden)
        self.q_weight, self.k_weight = 1.0 + 0.1 * randn(D), 1.0 + 0.1 * randn(D)
        angle = torch.arange(cfg["F"] * cfg["P"], device="cuda")[:, None] / 10000.0 ** (torch.arange(D // 2, device="cuda") / (D // 2))
        self.cos, self.sin = torch.cos(angle).float().contiguous(), torch.sin(angle).float().contiguous()
        # what a shape needs: tile lists of both patterns, sampled rows, workspace
        sampled = sample_rows(cfg)
        self.sampled = torch.from_numpy(sampled).cuda()
        self.lists = [torch.from_numpy(a).cuda() for pattern in (S.SVG_HEAD_SPATIAL, S.SVG_HEAD_TEMPORAL)
                      for a in S.svg_tile_list_build(self.shape, pattern)]
        self.ws_bytes = S.svg_workspace_bytes(self.shape, len(sampled))
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device="cuda")
        self.labels = torch.zeros(B * H, dtype=torch.uint8, device="cuda")
        self.mse = torch.zeros(B * H, 2, device="cuda")
        # activations
        bf16 = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.emb, self.mod = Operand(B, C), torch.empty(B, 6 * C, device="cuda")
        self.h1, self.h2, self.u, self.o4 = Operand(rows, C), Operand(rows, C), Operand(rows, hidden), Operand(rows, C)
        self.q, self.k, self.v, self.kt, self.vt, self.o = (bf16(B, H, N, D) for _ in range(6))
        self.y, self.z, self.r, self.out = (bf16(rows, C) for _ in range(4))
        table = lambda i: self.mod[:, i * C:(i + 1) * C]  # noqa: E731
        desc = lambda **kw: S.gate_norm_desc(rows, C, B, ld_mod=6 * C, eps=1e-6, **kw)  # noqa: E731
        # [gate | scale | shift] of the attention's half, then of the feed-forward's
        self.before = desc(pre_norm=S.SVG_NORM_LAYER, scale=table(1), shift=table(2))
        self.between = desc(pre_norm=S.SVG_NORM_LAYER, gate=table(0), scale=table(4), shift=table(5))
        self.behind = desc(gate=table(3))

    def forward(self, x, embedding):
        """x: bf16 [B N, C]; embedding: [B, C] of any of the element types.  Returns the next layer's x."""
        if x.shape != (self.rows, self.C) or x.dtype != torch.bfloat16 or not x.is_contiguous():
            raise ValueError(f"x has to be [{self.rows}, {self.C}] in bfloat16, row behind row")
        self.modulation(self.emb.write(embedding, S.SVG_ACT_SILU), self.mod)
        S.svg_gate_norm_fwd(self.before, x, None, None, None, self.h1.codes, self.h1.scales)
        for proj, out in ((self.q_proj, self.q), (self.k_proj, self.k), (self.v_proj, self.v)):
            proj(self.h1, out)
        for t, weight in ((self.q, self.q_weight), (self.k, self.k_weight)):
            S.svg_qk_norm_rope(self.shape, t, t, S.SVG_NORM_RMS, weight, None, 1e-6, self.cos, self.sin, S.SVG_ROPE_INTERLEAVED)
        self.attend()
        self.o_proj(self.o4.write(self.o), self.y)
        S.svg_gate_norm_fwd(self.between, x, self.y, self.r, None, self.h2.codes, self.h2.scales)
        self.up.to_operand(self.h2, self.u, S.SVG_ACT_GELU_TANH)
        self.down(self.u, self.z)
        S.svg_gate_norm_fwd(self.behind, self.r, self.z, self.out, None)
        return self.out

    def attend(self):
        """The attention alone: profile the heads, move k and v of the temporal ones, attend."""
        sh, q, k, v = self.shape, self.q, self.k, self.v
        S.svg_profile_heads(sh, q, k, v, self.sampled, len(self.sampled), self.labels, self.mse, self.ws, self.ws_bytes)
        S.svg_layout_kv_temporal(sh, k, v, self.kt, self.vt, self.labels)
        S.svg_sparse_attn_fwd_kv2(sh, q, k, v, self.kt, self.vt, self.o, self.labels, *self.lists)


def _milliseconds(f, repeats):
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    f()
    start.record()
    for _ in range(repeats):
        f()
    end.record()
    end.synchronize()
    return start.elapsed_time(end) / repeats


def main():
    parser = argparse.ArgumentParser(description="Times one transformer layer of a named workload's shape.")
    parser.add_argument("--workload", default="wan21_14b", choices=sorted(CONFIGS))
    parser.add_argument("--widening", type=int, default=4, help="hidden width of the feed-forward half over the model's")
    parser.add_argument("--repeats", type=int, default=10)
    args = parser.parse_args()
    layer = Layer(get_config(args.workload), args.widening)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(layer.rows, layer.C, generator=gen, device="cuda").to(torch.bfloat16)
    embedding = torch.randn(layer.B, layer.C, generator=gen, device="cuda")
    whole = _milliseconds(lambda: layer.forward(x, embedding), args.repeats)
    attention = _milliseconds(layer.attend, args.repeats)
    print(f"{args.workload}: {layer.rows} tokens of {layer.C} channels: {whole:.3f} ms a layer, {attention:.3f} of them attention, "
          f"{int(layer.labels.sum())} of {layer.labels.numel()} heads temporal")


if __name__ == "__main__":
    main()
