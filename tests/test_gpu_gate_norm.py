"""Gate, residual, norm and modulation, and its gradients, against the 64-bit forms."""
import itertools

import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import block_oracle as O
from workloads import CONFIGS

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                          # half a step of fp32
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
STREAM = {"bf16": (torch.bfloat16, S.SVG_BF16), "f32": (torch.float32, S.SVG_F32)}
BRANCH = {"bf16": (torch.bfloat16, S.SVG_BF16), "f16": (torch.float16, S.SVG_F16)}
EPS = 1e-5


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def close(got, ref, half, noise, what):
    """One rounding to the output's type on top of the noise of the fp32 arithmetic."""
    err, allowed = np.abs(f64(got) - ref), half * np.abs(ref) + (1 + half) * noise
    assert (err <= allowed).all(), (what, float((err / np.maximum(allowed, 1e-300)).max()))


class Case:
    def __init__(self, rows, C, groups=1, ptr=None, stream="bf16", branch="bf16", post=0, pre=2, affine=True, alpha=1.0, seed=0,
                 ld=0, ld_mod=0, offset=0.3):
        gen = torch.Generator().manual_seed(seed)
        ts, tb = STREAM[stream][0], BRANCH[branch][0]
        wide = lambda t: torch.randn(rows, ld or C, generator=gen).add_(offset).to(t).cuda()[:, :C]  # noqa: E731
        self.x, self.y, self.dr, self.dh = wide(ts), wide(tb), wide(ts), wide(tb)
        mod = (0.5 * torch.randn(3, groups, ld_mod or C, generator=gen)).cuda()
        self.gate, self.scale, self.shift = mod[0, :, :C], mod[1, :, :C], mod[2, :, :C]
        vec = lambda: (1 + 0.3 * torch.randn(C, generator=gen)).cuda() if affine else None  # noqa: E731
        self.post_weight, self.post_bias, self.weight, self.bias = vec(), vec(), vec(), vec()
        self.ptr = None if ptr is None else torch.tensor(ptr, dtype=torch.int32).cuda()
        self.group = O.group_of_rows(rows, groups, ptr)
        self.kw = dict(alpha=float(np.float32(alpha)), post=post, pre=pre, post_eps=float(np.float32(EPS)), eps=float(np.float32(EPS)))
        self.rows, self.C, self.groups, self.ts, self.tb, self.ld = rows, C, groups, ts, tb, ld or C
        self.desc = S.gate_norm_desc(rows, C, groups, self.ptr, STREAM[stream][1], BRANCH[branch][1], post, pre, alpha, EPS, EPS,
                                     ld, ld, ld, ld, ld_mod, self.gate, self.scale, self.shift, self.post_weight,
                                     self.post_bias, self.weight, self.bias)

    def empty(self, dtype):
        """An output with the row stride of the descriptor; what lies between the rows is checked to stay."""
        return torch.full((self.rows, self.ld), float("nan"), dtype=dtype, device="cuda")[:, :self.C]

    def params(self):
        return [f64(t) for t in (self.post_weight, self.post_bias, self.weight, self.bias)]

    def forward(self):
        return O.gate_norm(f64(self.x), f64(self.y), self.group, f64(self.gate), f64(self.scale), f64(self.shift),
                           self.kw["alpha"], self.kw["post"], self.kw["pre"], self.kw["post_eps"], self.kw["eps"], *self.params())

    def noise(self):
        """fp32 noise of r and h: about 16 + 6 + 8 additions behind a statistic and a dozen operations per element, each off by at
        most U relative to what it adds up; 64 of them are allowed."""
        one = np.ones((self.rows, 1))
        hat, rho = O.normalise(f64(self.y), self.kw["post"], self.kw["post_eps"])
        mean = np.abs(f64(self.y)).mean(1, keepdims=True) * rho if self.kw["post"] else 0 * one
        wp, bp, w, b = (1.0 if t is None else np.abs(t) for t in self.params())
        p = (np.abs(hat) + mean) * wp + bp
        r = 64 * U * (np.abs(self.kw["alpha"] * f64(self.x)) + np.abs(f64(self.gate)[self.group]) * p)
        ref = self.forward()[0]
        hat, rho = O.normalise(ref, self.kw["pre"], self.kw["eps"])
        mean = np.abs(ref).mean(1, keepdims=True) * rho if self.kw["pre"] else 0 * one
        spread = r.max(1, keepdims=True) * rho if self.kw["pre"] else r
        h = ((64 * U * (np.abs(hat) + mean) + 3 * spread * (1 + np.abs(hat))) * w + 64 * U * b) * np.abs(1 + f64(self.scale)[self.group])
        return r, h + 64 * U * (np.abs(f64(self.shift)[self.group]) + np.abs(self.forward()[1]))


def run_forward(c, **kw):
    r, h = c.empty(c.ts), c.empty(c.tb)
    S.svg_gate_norm_fwd(c.desc, c.x, c.y, r, h, **kw)
    torch.cuda.synchronize()
    for t in (r, h):
        assert t._base is None or torch.isnan(t._base[:, c.C:]).all()
    return r, h


def check_forward(c):
    r, h = run_forward(c)
    ref_r, ref_h = c.forward()
    noise_r, noise_h = c.noise()
    close(r, ref_r, HALF[c.ts], noise_r, "r")
    close(h, ref_h, HALF[c.tb], noise_h, "h")


SIZES = [(1, 1), (1, 8), (2, 7), (3, 64), (17, 255), (5, 256), (9, 512), (4, 520), (7, 1000), (6, 1001), (3, 2048), (5, 5120), (2, 8192),
         (2, 8200), (3, 16384), (2, 12345)]


@pytest.mark.parametrize("rows,C", SIZES)
@pytest.mark.parametrize("post,pre", [(0, 2), (1, 1), (2, 0), (2, 2)])
def test_forward_sizes(rows, C, post, pre):
    check_forward(Case(rows, C, post=post, pre=pre, seed=rows * 31 + C))


@pytest.mark.parametrize("stream,branch", list(itertools.product(STREAM, BRANCH)))
@pytest.mark.parametrize("post,pre", list(itertools.product(range(3), range(3))))
def test_forward_types_and_norms(stream, branch, post, pre):
    for C, affine in ((96, True), (333, False)):
        check_forward(Case(33, C, 3, [0, 5, 5, 33], stream, branch, post, pre, affine, alpha=0.7, seed=post * 3 + pre))


@pytest.mark.parametrize("groups,ptr", [(1, None), (4, None), (24, None), (3, [0, 0, 24, 24]), (3, [0, 1, 2, 24]), (5, [0, 7, 7, 7, 20, 24]),
                                        (2, [9, 11, 13])])      # the last table's ends are taken as 0 and rows
def test_groups(groups, ptr):
    check_forward(Case(24, 72, groups, ptr, seed=groups))
    check_backward(Case(24, 72, groups, ptr, post=1, pre=1, stream="f32", seed=groups))


@pytest.mark.parametrize("ld,ld_mod", [(104, 0), (101, 99), (0, 300), (97, 0), (112, 112)])
def test_strides_and_alignment(ld, ld_mod):
    for C in (96, 95):
        check_forward(Case(19, C, 3, [0, 6, 12, 19], ld=ld, ld_mod=ld_mod, post=1, seed=ld))
        check_backward(Case(19, C, 3, [0, 6, 12, 19], ld=ld, ld_mod=ld_mod, post=1, seed=ld))


def test_rows_far_from_zero_keep_their_statistics():
    """mean / deviation = 500: a one-pass variance in fp32 would lose 2^-24 * 500^2 = 1.5 % of it."""
    check_forward(Case(6, 1024, stream="f32", post=2, pre=2, affine=False, offset=500.0))


def test_missing_parts():
    c = Case(13, 264, post=0, pre=2, alpha=0.5)
    r, h = torch.empty_like(c.x), torch.empty_like(c.y)
    plain = S.gate_norm_desc(13, 264, pre_norm=2, eps=EPS, residual_scale=0.5)
    S.svg_gate_norm_fwd(plain, c.x, None, r, h)                              # no branch, no tables, no weights
    half = np.abs(f64(c.x)).max() * U * 64
    close(r, 0.5 * f64(c.x), HALF[c.ts], 0.0, "r")
    ref = O.normalise(0.5 * f64(c.x), 2, float(np.float32(EPS)))[0]
    close(h, ref, HALF[c.tb], half * 10, "h")
    only = torch.full_like(c.y, float("nan"))
    S.svg_gate_norm_fwd(c.desc, c.x, c.y, None, only)                        # the stream is not wanted
    r2, h2 = run_forward(c)
    assert torch.equal(only, h2)
    S.svg_gate_norm_fwd(c.desc, c.x, c.y, r, None)                           # the next branch's input is not wanted
    assert torch.equal(r, r2)
    x = c.x.clone()
    S.svg_gate_norm_fwd(c.desc, x, c.y, x, h)                                # in place
    assert torch.equal(x, r2) and torch.equal(h, h2)


def test_no_rows_and_infinities_stay_in_their_rows():
    c = Case(8, 136, post=1, pre=2)
    S.svg_gate_norm_fwd(S.gate_norm_desc(0, 136), c.x, c.y, c.x.clone(), None)
    clean = run_forward(c)
    c.x[3, 5], c.y[5, 7] = float("inf"), float("nan")
    r, h = run_forward(c)
    keep = [0, 1, 2, 4, 6, 7]
    assert torch.equal(r[keep], clean[0][keep]) and torch.equal(h[keep], clean[1][keep])
    assert torch.isinf(r[3, 5]) and torch.isnan(h[3]).any() and torch.isnan(r[5]).all()


@pytest.mark.parametrize("rows,C", [(1, 32), (15, 64), (16, 256), (33, 288), (50, 1024), (17, 2080), (18, 5120), (3, 16384)])
def test_four_bit_output_is_the_rounded_fp32_result(rows, C):
    """Codes and scales against the 64-bit h: a code may differ only where h is within the fp32 noise of a border."""
    c = Case(rows, C, post=1, pre=1, stream="f32", seed=C)
    codes = torch.full((S.svg_fp4_buffer_bytes(rows, C, 0),), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((S.svg_fp4_buffer_bytes(rows, C, 1),), 0xAA, dtype=torch.uint8, device="cuda")
    r, h = run_forward(c, codes=codes, scales=scales)
    ref_r, ref_h = c.forward()
    noise_r, noise = c.noise()
    close(r, ref_r, HALF[c.ts], noise_r, "r")
    close(h, ref_h, HALF[c.tb], noise, "h")
    assert_four_bit(codes, scales, ref_h, noise)


def assert_four_bit(codes, scales, v, noise):
    """codes, scales (device, operand order) hold v up to `noise`; the padding's codes are zero."""
    rows, cols = v.shape
    got, gs = O.from_operand(codes.cpu().numpy(), scales.cpu().numpy(), rows, cols)
    pad = np.zeros((rows, -(-cols // 32) * 32))
    pad[:, :cols] = v
    npad = np.zeros_like(pad)
    npad[:, :cols] = noise
    top = np.abs(pad).reshape(rows, -1, 32)
    slack = npad.reshape(rows, -1, 32)
    low, high = np.maximum(top - slack, 0).max(-1), (top + slack).max(-1)
    field = lambda m: np.where(m > 0, np.clip(np.frexp(m)[1] - 1 - 2, -127, 127), -127) + 127  # noqa: E731
    assert ((gs >= field(low)) & (gs <= field(high))).all()
    size = np.ldexp(1.0, gs.astype(np.int64) - 127)[..., None]
    value = O.mx_values(got, gs)

    def nearest(x):
        t = np.abs(x.reshape(rows, -1, 32) / size)
        code = sum(((t > (O.GRID[i] + O.GRID[i + 1]) / 2) if i % 2 == 0 else (t >= (O.GRID[i] + O.GRID[i + 1]) / 2)).astype(int)
                   for i in range(7))
        return (O.GRID[code] * size).reshape(rows, -1)[:, :cols] * np.sign(x[:, :cols])
    a, b = nearest(pad - npad), nearest(pad + npad)
    assert ((value >= np.minimum(a, b)) & (value <= np.maximum(a, b))).all()
    full = O.from_operand(codes.cpu().numpy(), scales.cpu().numpy(), -(-rows // 16) * 16, -(-cols // 256) * 256)[0]
    assert not full[rows:].any() and not full[:, cols:].any()


# ---- gradients ------------------------------------------------------------------------------------

NAMES = ("gate", "scale", "shift", "post_weight", "post_bias", "weight", "bias")


def run_backward(c, grads=NAMES, **given):
    dev = dict(dtype=torch.float32, device="cuda")
    out = {n: torch.full((c.groups, c.C) if n in NAMES[:3] else (c.C,), float("nan"), **dev) for n in grads}
    dx, dy = c.empty(c.ts), c.empty(c.tb)
    n = S.svg_gate_norm_workspace_bytes(c.desc)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    t = dict(r=c.x, y=c.y, dr=c.dr, dh=c.dh)
    t.update(given)
    S.svg_gate_norm_bwd(c.desc, t["r"], t["y"], t["dr"], t["dh"], dx, dy, S.gate_norm_grads(**out), ws, n)
    torch.cuda.synchronize()
    out.update(dx=dx, dy=dy)
    return out


def check_backward(c, got=None, **given):
    """c.x is taken as the stream r that a forward pass gave."""
    t = dict(r=c.x, y=c.y, dr=c.dr, dh=c.dh)
    t.update(given)
    r, y, dr, dh = (f64(t[k]) for k in ("r", "y", "dr", "dh"))
    wp, bp, w, b = c.params()
    ref = O.gate_norm_grad(r, y, dr, dh, c.group, c.groups, f64(c.gate), f64(c.scale), post_weight=wp, post_bias=bp, weight=w, bias=b, **c.kw)
    got = got or run_backward(c, [n for n in NAMES if y is not None or n not in ("gate", "post_weight", "post_bias")], **given)
    # fp32 noise: 128 roundings of the terms that a value is added up from, in magnitude
    N = 128 * U
    one = np.ones(c.C)
    dh = np.zeros_like(r) if dh is None else dh
    hat, rho = O.normalise(r, c.kw["pre"], c.kw["eps"])
    far = np.abs(hat) + (np.abs(r).mean(1, keepdims=True) * rho if c.kw["pre"] else 0)      # hat's own noise is N of this
    e = np.abs(dh * (1 + f64(c.scale)[c.group])) * (np.abs(w) if w is not None and c.kw["pre"] else one)
    term = e if not c.kw["pre"] else rho * (e + e.mean(1, keepdims=True) + far * (e * far).mean(1, keepdims=True))
    d = (np.abs(dr) if dr is not None else 0) + term
    close(got["dx"], ref["dx"], HALF[c.ts], N * abs(c.kw["alpha"]) * d, "dx")
    sums = lambda v: np.stack([v[c.group == g].sum(0) for g in range(c.groups)])  # noqa: E731
    aw, ab = (np.abs(w) if w is not None and c.kw["pre"] else one), (np.abs(b) if b is not None and c.kw["pre"] == 2 else 0 * one)
    bound = {"shift": sums(np.abs(dh)), "scale": sums(np.abs(dh) * (far * aw + ab)),
             "weight": (np.abs(dh * (1 + f64(c.scale)[c.group])) * far).sum(0), "bias": np.abs(dh * (1 + f64(c.scale)[c.group])).sum(0)}
    if y is not None:
        yhat, yrho = O.normalise(y, c.kw["post"], c.kw["post_eps"])
        yfar = np.abs(yhat) + (np.abs(y).mean(1, keepdims=True) * yrho if c.kw["post"] else 0)
        gate = np.abs(f64(c.gate)[c.group])
        awp, abp = (np.abs(wp) if wp is not None and c.kw["post"] else one), (np.abs(bp) if bp is not None and c.kw["post"] == 2 else 0 * one)
        f = d * gate * awp
        term = f if not c.kw["post"] else yrho * (f + f.mean(1, keepdims=True) + yfar * (f * yfar).mean(1, keepdims=True))
        close(got["dy"], ref["dy"], HALF[c.tb], 2 * N * term + (2.0 ** -25 if c.tb == torch.float16 else 0), "dy")
        bound.update(gate=sums(d * (yfar * awp + abp)), post_weight=(d * gate * yfar).sum(0), post_bias=(d * gate).sum(0))
    for name in bound:
        if name in got:
            close(got[name], ref[name], U, 2 * N * bound[name], name)
    return ref, got


@pytest.mark.parametrize("rows,C", SIZES + [(1500, 64), (2100, 40)])
@pytest.mark.parametrize("post,pre", [(0, 2), (1, 1), (2, 0), (2, 2)])
def test_backward_sizes(rows, C, post, pre):
    check_backward(Case(rows, C, post=post, pre=pre, seed=rows * 31 + C))


@pytest.mark.parametrize("stream,branch", list(itertools.product(STREAM, BRANCH)))
@pytest.mark.parametrize("post,pre", list(itertools.product(range(3), range(3))))
def test_backward_types_and_norms(stream, branch, post, pre):
    for C, affine in ((96, True), (333, False)):
        check_backward(Case(33, C, 3, [0, 5, 5, 33], stream, branch, post, pre, affine, alpha=0.7, seed=post * 3 + pre))


def test_backward_of_many_strips_and_groups():
    ends = sorted(np.random.default_rng(4).integers(0, 3001, 40).tolist())
    check_backward(Case(3000, 48, 41, [0] + ends + [3000], stream="f32", post=2, pre=2))


def test_backward_missing_parts():
    c = Case(21, 120, 2, [0, 8, 21], stream="f32", post=0, pre=2)
    check_backward(c, dr=None)
    check_backward(c, y=None)
    ref, got = check_backward(c)
    dx = torch.empty_like(c.x)
    n = S.svg_gate_norm_workspace_bytes(c.desc)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    S.svg_gate_norm_bwd(c.desc, c.x, c.y, c.dr, c.dh, dx, None, None, ws, n)               # the stream's gradient alone
    assert torch.equal(dx, got["dx"])
    dr, dh = c.dr.clone(), c.dh.clone()
    S.svg_gate_norm_bwd(c.desc, c.x, c.y, dr, dh, dr, dh, None, ws, n)                     # in place
    assert torch.equal(dr, got["dx"]) and torch.equal(dh, got["dy"])
    last = S.gate_norm_desc(21, 120, 2, c.ptr, S.SVG_F32, S.SVG_BF16, gate=c.gate)         # the end of a layer: no norm behind it
    gate = torch.empty(2, 120, device="cuda")
    dy = torch.empty_like(c.y)
    S.svg_gate_norm_bwd(last, None, c.y, c.dr, None, dx, dy, S.gate_norm_grads(gate=gate), ws, n)
    assert torch.equal(dx, c.dr)
    close(dy, f64(c.dr) * f64(c.gate)[c.group], HALF[c.tb], 2 * U * np.abs(f64(c.dr) * f64(c.gate)[c.group]), "dy")
    terms = f64(c.dr) * f64(c.y)
    close(gate, np.stack([terms[c.group == g].sum(0) for g in range(2)]), U,
          64 * U * np.stack([np.abs(terms[c.group == g]).sum(0) for g in range(2)]), "gate")


def test_gradients_of_no_rows_and_of_empty_groups_are_zero():
    c = Case(10, 64, 4, [0, 4, 4, 10, 10])
    got = run_backward(c)
    for n in ("gate", "scale", "shift"):
        assert not got[n][1].any() and not got[n][3].any()
    gate, weight = torch.ones(4, 64, device="cuda"), torch.ones(64, device="cuda")
    desc = S.gate_norm_desc(0, 64, 4, gate=c.gate, pre_norm=1, weight=c.weight)
    n = S.svg_gate_norm_workspace_bytes(desc)
    S.svg_gate_norm_bwd(desc, c.x, c.y, c.dr, c.dh, None, None, S.gate_norm_grads(gate=gate, weight=weight),
                        torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    torch.cuda.synchronize()
    assert not gate.any() and not weight.any()


def test_backward_repeats_bit_for_bit():
    c = Case(2500, 1000, 3, [0, 900, 901, 2500], post=1, pre=2)
    a, b = run_backward(c), run_backward(c)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_gradient_against_differences_of_the_kernel():
    """Central differences of the fp32 stream along the gradient's own direction.  h is fp16: its roundings, 2^-12 |h| / sqrt(3) in the root
    mean square, are the noise (five deviations allowed); the third derivative's part is step^2 of the slope, 2 % allowed for it."""
    c = Case(48, 96, stream="f32", branch="f16", pre=2, post=1, alpha=1.0, seed=9)
    step = 0.05
    r, h = run_forward(c)
    dx, n = torch.empty_like(c.x), S.svg_gate_norm_workspace_bytes(c.desc)
    S.svg_gate_norm_bwd(c.desc, r, c.y, None, c.dh, dx, None, None, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    direction = dx / dx.square().mean().sqrt()

    def loss(x):
        r, h = torch.empty_like(c.x), torch.empty_like(c.y)
        S.svg_gate_norm_fwd(c.desc, x, c.y, r, h)
        return (h.double() * c.dh.double()).sum().item()
    slope = (loss(c.x + step * direction) - loss(c.x - step * direction)) / (2 * step)
    expected = (dx.double() * direction.double()).sum().item()
    noise = 5 * np.sqrt(2 / 3) * 2.0 ** -12 * np.linalg.norm(f64(c.dh) * f64(h)) / (2 * step)
    assert abs(slope - expected) <= noise + 0.02 * abs(expected)


# ---- as part of a program -------------------------------------------------------------------------

def test_other_stream_and_graph():
    c = Case(100, 512, 2, [0, 30, 100], post=1, pre=2)
    want = run_forward(c)
    side = torch.cuda.Stream()
    r, h = torch.empty_like(c.x), torch.empty_like(c.y)
    side.wait_stream(torch.cuda.current_stream())
    S.svg_gate_norm_fwd(c.desc, c.x, c.y, r, h, stream=side)
    side.synchronize()
    assert torch.equal(r, want[0]) and torch.equal(h, want[1])
    n = S.svg_gate_norm_workspace_bytes(c.desc)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dx, dy, gate, weight = torch.empty_like(c.x), torch.empty_like(c.y), torch.empty(2, 512, device="cuda"), torch.empty(512, device="cuda")
    grads = S.gate_norm_grads(gate=gate, weight=weight)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.svg_gate_norm_fwd(c.desc, c.x, c.y, r, h)
        S.svg_gate_norm_bwd(c.desc, r, c.y, c.dr, c.dh, dx, dy, grads, ws, n)
    for k in range(3):
        c.x.copy_(torch.randn(100, 512, device="cuda"))
        for t in (r, h, dx, dy, gate, weight):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        wr, wh = run_forward(c)
        wb = run_backward(c, ("gate", "weight"), r=wr)
        assert torch.equal(r, wr) and torch.equal(h, wh)
        assert all(torch.equal(a, b) for a, b in ((dx, wb["dx"]), (dy, wb["dy"]), (gate, wb["gate"]), (weight, wb["weight"])))


def test_tensors_past_32_bit_offsets():
    """450 000 rows of 5120 channels: 2.3e9 elements, 4.6e9 bytes a tensor."""
    rows, C = 450_000, 5120
    x = torch.empty(rows, C, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    sample = [0, 1, 209_715, 209_716, 419_430, 419_431, rows - 2, rows - 1]          # around byte 2^31 and 2^32
    gen = torch.Generator(device="cuda").manual_seed(5)
    for t in (x, y):
        t.zero_()
        t[sample] = torch.randn(len(sample), C, generator=gen, device="cuda").to(torch.bfloat16)
    desc = S.gate_norm_desc(rows, C, pre_norm=2)
    r, h = torch.full_like(x, 7.0), torch.full_like(y, 7.0)
    S.svg_gate_norm_fwd(desc, x, y, r, h)
    ref_r, ref_h = O.gate_norm(f64(x[sample]), f64(y[sample]), np.zeros(len(sample), int), None, None, None, 1.0, 0, 2, 1e-6, 1e-6)
    close(r[sample], ref_r, 2.0 ** -8, 0.0, "r")
    close(h[sample], ref_h, 2.0 ** -8, 1e-5, "h")
    assert not r[2].any() and not h[rows - 3].any()
    n = S.svg_gate_norm_workspace_bytes(desc)
    gate = torch.empty(1, C, device="cuda")
    rs, xs, ys = f64(r[sample]), f64(x[sample]), f64(y[sample])
    S.svg_gate_norm_bwd(desc, r, y, x, y, x, h, S.gate_norm_grads(gate=gate), torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    ref = O.gate_norm_grad(rs, ys, xs, ys, np.zeros(len(sample), int), 1, None, None, 1.0, 0, 2, 1e-6, 1e-6)
    close(x[sample], ref["dx"], 2.0 ** -8, 1e-4, "dx")
    close(h[sample], ref["dy"], 2.0 ** -8, 1e-4, "dy")
    close(gate, ref["gate"], U, 1e-3, "gate")
    assert not x[2].any() and not h[rows - 3].any()


# ---- rows of any alignment, and sums over many strips ------------------------------------------------

@pytest.mark.parametrize("C", [503, 504, 505, 509, 511, 513, 1007, 1009, 8063, 8065, 16127, 16129, 16383])
@pytest.mark.parametrize("stream,branch", [("bf16", "f16"), ("f32", "bf16")])
def test_widths_at_the_edges_of_a_wavefront(C, stream, branch):
    c = Case(3, C, 2, [0, 1, 3], stream, branch, post=2, pre=1, seed=C)
    check_forward(c)
    check_backward(c)


@pytest.mark.parametrize("rows,C", [(4100, 37), (3100, 513), (3100, 333), (2600, 1001), (4100, 504)])
def test_long_strips_of_odd_rows(rows, C):
    """More rows of a workgroup than are on their way at a time; the rows begin at every offset in a granule."""
    c = Case(rows, C, 3, [0, rows // 5, rows // 2, rows], "f32" if C == 333 else "bf16", "f16", post=1, pre=2, seed=rows)
    check_forward(c)
    check_backward(c)


@pytest.mark.parametrize("C", [5, 513, 516, 1001, 1017])
@pytest.mark.parametrize("ld", [0, 1031])
def test_odd_rows_in_place(C, ld):
    """No norm, so wavefronts never wait for each other: none may read what another one has written."""
    for pre, post in ((0, 0), (2, 1)):
        c = Case(2500, C, post=post, pre=pre, ld=ld, seed=C)
        r, h = run_forward(c)
        got = run_backward(c)
        x, dr, dh = (t._base.clone()[:, :C] if t._base is not None else t.clone() for t in (c.x, c.dr, c.dh))
        h2 = c.empty(c.tb)
        S.svg_gate_norm_fwd(c.desc, x, c.y, x, h2)
        assert torch.equal(x, r) and torch.equal(h2, h)
        n = S.svg_gate_norm_workspace_bytes(c.desc)
        S.svg_gate_norm_bwd(c.desc, c.x, c.y, dr, dh, dr, dh, None, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
        assert torch.equal(dr, got["dx"]) and torch.equal(dh, got["dy"])


@pytest.mark.parametrize("groups", [1, 2, 7, 8, 9, 17])
@pytest.mark.parametrize("rows,C", [(65000, 16), (900, 24)])
def test_sums_of_few_and_of_many_groups(rows, C, groups):
    """Up to eight groups are summed in one launch; the sums of many strips are added up in parts first."""
    ends = sorted(np.random.default_rng(groups).integers(0, rows + 1, groups - 1).tolist())
    check_backward(Case(rows, C, groups, [0] + ends + [rows] if groups > 1 else None, stream="f32", post=2, pre=2, seed=groups))


@pytest.mark.parametrize("groups", [1, 3, 17])
@pytest.mark.parametrize("post,pre", list(itertools.product(range(3), range(3))))
def test_parameters_that_a_norm_does_not_have_get_zero_gradients(post, pre, groups):
    """The forward pass takes no notice of them, whether the descriptor holds them or not; NaNs in the rows change nothing."""
    ends = sorted(np.random.default_rng(groups).integers(0, 41, groups - 1).tolist())
    for affine in (True, False):
        c = Case(40, 72, groups, [0] + ends + [40], post=post, pre=pre, affine=affine)
        check_backward(c)
        c.dh[3, 5], c.dr[7, 9] = float("nan"), float("inf")
        got = run_backward(c)
        there = {"weight": pre != 0, "bias": pre == 2, "post_weight": post != 0, "post_bias": post == 2}
        for name, has in there.items():
            assert has or not got[name].any(), name


@pytest.mark.parametrize("C", [64, 37, 520])
def test_column_slices_of_one_tensor(C):
    """Results beside their inputs in one tensor, without and with alignment: nothing is written outside of their columns."""
    rows = 70
    c = Case(rows, C, 2, [0, 31, rows], post=1, pre=2, seed=C)
    r, h = run_forward(c)
    grads = run_backward(c, ())
    wide, wide_b = (torch.full((rows, 3 * C), 7.0, dtype=t, device="cuda") for t in (c.ts, c.tb))
    cut = lambda t, i: t[:, i * C:(i + 1) * C]  # noqa: E731
    cut(wide, 1).copy_(c.x)
    cut(wide_b, 1).copy_(c.y)
    desc = S.gate_norm_desc(rows, C, 2, c.ptr, post_norm=1, pre_norm=2, post_eps=EPS, eps=EPS, ld_x=3 * C, ld_y=3 * C, ld_r=3 * C, ld_h=3 * C,
                            gate=c.gate, scale=c.scale, shift=c.shift, post_weight=c.post_weight, post_bias=c.post_bias, weight=c.weight,
                            bias=c.bias)
    S.svg_gate_norm_fwd(desc, cut(wide, 1), cut(wide_b, 1), cut(wide, 2), cut(wide_b, 2))
    torch.cuda.synchronize()
    assert torch.equal(cut(wide, 2), r) and torch.equal(cut(wide_b, 2), h)
    assert torch.equal(cut(wide, 1), c.x) and torch.equal(cut(wide_b, 1), c.y) and (cut(wide, 0) == 7).all() and (cut(wide_b, 0) == 7).all()
    for t, i, v in ((wide, 2, c.dr), (wide_b, 2, c.dh)):
        cut(t, i).copy_(v)
    n = S.svg_gate_norm_workspace_bytes(desc)
    S.svg_gate_norm_bwd(desc, cut(wide, 1), cut(wide_b, 1), cut(wide, 2), cut(wide_b, 2), cut(wide, 0), cut(wide_b, 0), None,
                        torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    torch.cuda.synchronize()
    assert torch.equal(cut(wide, 0), grads["dx"]) and torch.equal(cut(wide_b, 0), grads["dy"])
    assert torch.equal(cut(wide, 1), c.x) and torch.equal(cut(wide, 2), c.dr) and torch.equal(cut(wide_b, 1), c.y) and torch.equal(cut(wide_b, 2), c.dh)


@pytest.mark.parametrize("C", sorted({c["H"] * c["D"] for c in CONFIGS.values()}))
def test_widths_of_the_workloads(C):
    """Rows, gradients and the 4-bit form at the width of every workload of the library."""
    for stream, post, pre in (("bf16", 0, 2), ("f32", 1, 1)):
        c = Case(70, C, 2, [0, 30, 70], stream, "bf16", post, pre, seed=C)
        codes, scales = (torch.full((S.svg_fp4_buffer_bytes(70, C, w),), 0xAA, dtype=torch.uint8, device="cuda") for w in (0, 1))
        r, h = run_forward(c, codes=codes, scales=scales)
        ref_r, ref_h = c.forward()
        noise_r, noise_h = c.noise()
        close(r, ref_r, HALF[c.ts], noise_r, "r")
        close(h, ref_h, HALF[c.tb], noise_h, "h")
        assert_four_bit(codes, scales, ref_h, noise_h)
        check_backward(c)
