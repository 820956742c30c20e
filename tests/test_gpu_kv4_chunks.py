"""Video generated chunk by chunk on the 4-bit cache: tables, rows, attention and the timestep's projection together, eagerly and from a captured
graph whose replays carry the state on."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import block_oracle as B
from oracle import kv4_oracle as O

pytestmark = pytest.mark.gpu


class Step:
    """One step of every sequence: `chunk` more tokens, which see their own frame and all earlier ones."""

    def __init__(self, sequences, heads, group, D, page_size, chunk, steps, frame):
        self.b, self.h, self.g, self.D, self.ps, self.chunk, self.frame = sequences, heads, group, D, page_size, chunk, frame
        longest = chunk * steps + page_size
        self.max_pages = -(-longest // page_size)
        self.pages = sequences * self.max_pages
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.data = i32(sequences, self.max_pages) - 1, torch.full((self.pages * heads * O.record_bytes(D, page_size),), 0xFF, dtype=torch.uint8, device="cuda")
        self.cache = S.kv4_cache(sequences, self.pages, self.max_pages, heads, D, page_size, data=self.data, page_table=self.table)
        self.lengths, self.wanted, self.status = i32(sequences), i32(sequences), i32(1)
        self.free = torch.randperm(self.pages, generator=torch.Generator().manual_seed(3)).int().cuda()
        self.count = torch.full((1,), self.pages, dtype=torch.int32, device="cuda")
        self.slots = torch.zeros(sequences, chunk, dtype=torch.int64, device="cuda")
        # q, k and v as slices of one projection's output
        self.qkv = torch.zeros(sequences, chunk, (group + 2) * heads * D, dtype=torch.bfloat16, device="cuda")
        cut = lambda first, n: self.qkv[..., first * D:(first + n) * D].view(sequences, chunk, n, D).transpose(1, 2)  # noqa: E731
        self.q, self.k, self.v = cut(0, group * heads), cut(group * heads, heads), cut((group + 1) * heads, heads)
        self.o = torch.zeros(sequences, chunk, group * heads, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        self.lse = torch.zeros(sequences, group * heads, chunk, device="cuda")
        self.attn = S.kv4_attn(kv_len=self.lengths, causal=True, block=frame)
        self.ws_bytes = S.svg_kv4_attn_workspace_bytes(self.cache, self.attn, S.tokens_of(self.q))
        self.ws = torch.empty(max(16, self.ws_bytes), dtype=torch.uint8, device="cuda")
        # a row of modulation for each sequence
        N, K = 192, 384
        w = np.random.default_rng(4).standard_normal((N, K)) / np.sqrt(K)
        self.w_values = B.mx_values(*B.mx_quantise(w))
        self.w = [torch.from_numpy(np.ascontiguousarray(x)).cuda().view(torch.uint8).flatten() for x in B.to_operand(*B.mx_quantise(w))]
        self.emb, self.mod = torch.zeros(sequences, K, device="cuda"), torch.zeros(sequences, N, device="cuda")

    def run(self):
        self.wanted.copy_(self.lengths).add_(self.chunk)
        S.svg_kv4_resize(self.cache, self.lengths, self.wanted, self.free, self.count, self.lengths, self.count, self.slots, self.chunk, self.status)
        S.svg_kv4_write(self.cache, S.tokens_of(self.k), self.k, S.tokens_of(self.v), self.v, self.slots)
        S.svg_kv4_attn_fwd(self.cache, self.attn, S.tokens_of(self.q), self.q, S.tokens_of(self.o), self.o, self.lse, self.ws, self.ws_bytes)
        S.svg_fp4_linear_rows(S.tokens_of(self.emb), self.emb, S.SVG_ACT_SILU, self.mod.shape[1], *self.w, None, S.SVG_ACT_NONE, S.tokens_of(self.mod), self.mod)

    def inputs(self, step):
        gen = torch.Generator().manual_seed(100 + step)
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=gen).to(torch.bfloat16))
        self.emb.copy_(torch.randn(self.emb.shape, generator=gen))

    def state(self):
        return [x.clone() for x in (self.table, self.data, self.lengths, self.free, self.count, self.slots, self.status, self.o, self.lse, self.mod)]


CASES = [dict(sequences=2, heads=2, group=1, D=64, page_size=16, chunk=1, steps=6, frame=1),
         dict(sequences=3, heads=1, group=4, D=128, page_size=32, chunk=21, steps=5, frame=7),
         dict(sequences=1, heads=4, group=1, D=64, page_size=64, chunk=192, steps=5, frame=64),
         dict(sequences=2, heads=2, group=2, D=128, page_size=16, chunk=150, steps=4, frame=50)]


def check_against_oracle(s, step, kept):
    """kept: keys and values of all steps so far, quantised."""
    b, h, g, D, n = s.b, s.h, s.g, s.D, s.chunk * (step + 1)
    assert s.status.item() == 0 and (s.lengths == n).all()
    for i in range(b):
        k, v = (np.concatenate([x[j][i] for x in kept]) for j in (0, 1))
        rows = sorted({0, s.frame - 1, s.chunk // 2, s.chunk - 1})
        for r in rows:
            see = O.seen(n, s.chunk, r, s.frame, True, -1, 0)
            own = np.repeat(np.arange(h), g)
            ref, ref_lse, size, slack = O.attention(s.q[i, :, r:r + 1].double().cpu().numpy(), k[see][:, own], v[see][:, own], np.ones(see.sum(), bool), D ** -0.5)
            e = (D + 10) * 2.0 ** -23 * slack + 2.0 ** -21
            err = np.abs(s.o[i, :, r].double().cpu().numpy() - ref[:, 0])
            assert (err <= 2.0 ** -8 * np.abs(ref[:, 0]) + (2.0 ** -8 + 2 * e + (n / 32 + 64) * 2.0 ** -23) * size[:, 0] * 1.01).all(), (step, i, r)
            assert (np.abs(s.lse[i, :, r].double().cpu().numpy() - ref_lse[:, 0]) <= e[:, 0] + (n / 32 + 64) * 2.0 ** -23 + 2.0 ** -22 * np.abs(ref_lse[:, 0])).all()
    x = s.emb.double().cpu().numpy()
    a = B.silu(x)
    noise = (np.abs(a) @ np.abs(s.w_values).T) * ((3 * 12 + 16) * 2.0 ** -23 + 2.0 ** -24 * (8 + 1.3 * np.abs(x).max()))
    assert (np.abs(s.mod.double().cpu().numpy() - a @ s.w_values.T) <= noise).all()


@pytest.mark.parametrize("case", CASES)
def test_steps_follow_each_other(case):
    s, kept = Step(**case), []
    for step in range(case["steps"]):
        s.inputs(step)
        s.run()
        torch.cuda.synchronize()
        quantised = []
        for x in (s.k, s.v):
            rows = x.double().cpu().numpy().transpose(0, 2, 1, 3)
            quantised.append(B.mx_values(*B.mx_quantise(rows.reshape(-1, s.D))).reshape(rows.shape))
        kept.append(quantised)
        check_against_oracle(s, step, kept)
    # the first sequence is finished: its pages come back and the others go on
    free = s.count.item()
    held = -(-int(s.lengths[0]) // s.ps)
    s.wanted.copy_(s.lengths)
    s.wanted[0] = 0
    S.svg_kv4_resize(s.cache, s.lengths, s.wanted, s.free, s.count, s.lengths, s.count, s.slots, s.chunk, s.status)
    assert s.count.item() == free + held and s.lengths[0].item() == 0 and s.status.item() == 0 and (s.slots == -1).all()


@pytest.mark.parametrize("case", CASES)
def test_a_captured_step_carries_the_state_on(case):
    eager, graphed = Step(**case), Step(**case)
    # one run on the capture stream in front, on a state that is put back
    before = [x.clone() for x in (graphed.table, graphed.data, graphed.lengths, graphed.free, graphed.count)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        graphed.run()
    for x, y in zip((graphed.table, graphed.data, graphed.lengths, graphed.free, graphed.count), before):
        x.copy_(y)
    for step in range(case["steps"]):
        eager.inputs(step)
        eager.run()
        graphed.inputs(step)
        torch.cuda.synchronize()
        graph.replay()
        scratch = torch.randn(1 << 20, device="cuda").sum()              # eager work of our own between the replays
        torch.cuda.synchronize()
        assert torch.isfinite(scratch)
        for name, x, y in zip(("table", "data", "lengths", "free", "count", "slots", "status", "o", "lse", "mod"), eager.state(), graphed.state()):
            assert torch.equal(x, y), (step, name)
