"""Video generated chunk by chunk on a cache of keys and values in 4 bits, as cases that can be timed.

Four families of operators:
  pages  svg_kv4_resize: page tables and slot maps from the sequences' lengths
  write  svg_kv4_write and svg_kv4_read: keys and values of new tokens into the cache's pages, and read back
  attn   svg_kv4_attn_fwd: attention of new queries over the cache, with its log-sum-exp
  rows   svg_fp4_linear_rows: few rows of activations (a timestep's, a token's) times weights kept in 4 bits

Where `own` is false the same is computed from elementary torch operations in 32 bits.

Microscaled 4-bit floating point (OCP MX, E2M1 elements with one E8M0 scale for 32 neighbours of a row):
E = clamp(floor(log2 max|v|) - 2, -127, 127), code = the E2M1 value nearest to v / 2^E, ties to even, at most 6, scale byte
E + 127; the even one of two neighbouring elements in the low half of a byte.

The cache is a pool of pages of `page` tokens.  For each page and head there is one record: the keys' codes [page][D / 2], the
values' codes [page][D / 2], the keys' scale bytes [page][D / 32], the values' scale bytes [page][D / 32].  A table row names the
pages of a sequence in order, a slot is page * page size + place.  Weights are held in the operand order of the matrix
instructions: rows in tiles of 16, columns in tiles of 128; a tile is 64 pieces of 16 bytes, piece 16 g + i holding row i's columns
32 g to 32 g + 31 (rows padded to 16, columns to 256); scale bytes of four column tiles together, [row tile][group][piece][column tile].
"""
from __future__ import annotations

import math

import torch

own = False

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SCORES = 1 << 28           # scores held at a time by the plain form


# ---------------------------------------------------------------------------------------------- the cases

def _pages(name, **kw):
    case = {"name": name, "op": "pages", "B": 1, "page": 64, "longest": 0, "chunk": 0, "shrink": 0.0}
    case.update(kw)
    return case


def _write(name, **kw):
    case = {"name": name, "op": "write", "B": 1, "H": 1, "N": 1, "D": 128, "page": 64, "type": "bf16", "out": "bf16", "packed": False,
            "padded": False}
    case.update(kw)
    return case


def _attn(name, **kw):
    case = {"name": name, "op": "attn", "B": 1, "H": 1, "group": 1, "N": 1, "D": 128, "page": 64, "longest": 1, "ragged": False,
            "causal": False, "block": 1, "window": -1, "sink": 0, "packed": False}
    case.update(kw)
    return case


def _rows(name, **kw):
    case = {"name": name, "op": "rows", "M": 1, "N": 0, "K": 0, "type": "bf16", "out": "bf16", "silu": False, "gelu": False}
    case.update(kw)
    return case


def listed():
    return [
        # one video of the smallest workload (frames of 64 tokens) grows by a frame: a call's latency is what counts
        _pages("pages_tiny", B=1, page=16, longest=272, chunk=64),
        # a server's videos of all lengths, each growing by up to a frame of 1560 tokens, every eighth one finished and released
        _pages("pages_server", B=200, page=64, longest=32760, chunk=1560, shrink=0.125),
        # a token for each of eight sequences, from a packed projection in fp32
        _write("write_token", B=8, H=8, N=1, page=16, type="f32", packed=True),
        # text and video rows of unlike lengths in one padded call, half precision
        _write("write_padded_odd", B=3, H=12, N=1999, D=64, page=32, type="f16", out="f32", padded=True),
        # three frames of the Wan2.1 shape, k and v slices of one packed projection
        _write("write_chunk_wan21", H=40, N=4680, packed=True),
        # the smallest workload's next frame over what it has so far
        _attn("attn_tiny", H=4, N=64, D=64, page=16, longest=272),
        # one token for each of eight sequences over caches of up to 65536, four query heads to a head of the cache
        _attn("attn_token", B=8, H=32, group=4, N=1, longest=65536, ragged=True, causal=True),
        # text queries of three packed videos over caches of odd lengths
        _attn("attn_text_odd", B=3, H=48, N=226, D=64, page=32, longest=5003, ragged=True, packed=True),
        # three frames of the CogVideoX-v1 shape over a sliding window of six frames and the first one; what lies before has left
        _attn("attn_window", H=48, N=4050, D=64, longest=17550, causal=True, block=1350, window=6, sink=1350),
        # three frames of the Wan2.1 shape over the whole video, a frame seeing its own and all earlier ones
        _attn("attn_chunk_wan21", H=40, N=4680, longest=32760, causal=True, block=1560, packed=True),
        # a timestep's embedding through its first projection
        _rows("rows_timestep", M=1, N=5120, K=256, type="f32", out="f32", silu=False),
        # tokens of a few sequences into a wide feed-forward half, behind the activation of the embedding's second projection
        _rows("rows_wide", M=4, N=20480, K=5120, silu=True, gelu=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same operators with sizes of its own."""
    op = rng.choice(["pages", "write", "write", "attn", "attn", "attn", "rows", "rows"])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "pages":
        B = _log_int(rng, 1, 200)
        case = _pages("", B=B, page=page, longest=_log_int(rng, 16, 32760), chunk=_log_int(rng, 1, 1560),
                      shrink=rng.choice([0.0, 0.0, 0.2]))
    elif op == "write":
        D, B, H = rng.choice([64, 128]), rng.randint(1, 8), _log_int(rng, 1, 48)
        N = _log_int(rng, 1, max(1, min(32760, 23000000 // (B * H * D))))
        case = _write("", B=B, H=H, N=N, D=D, page=page, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                      out=rng.choice(["bf16", "f32"]), packed=rng.random() < 0.5, padded=B > 1 and rng.random() < 0.5)
    elif op == "attn":
        D, B, heads, group = rng.choice([64, 128]), _log_int(rng, 1, 8), _log_int(rng, 1, 24), rng.choice([1, 1, 2, 4, 7])
        longest = _log_int(rng, 1, 65536)
        N = _log_int(rng, 1, max(1, min(longest, 4680, int(3.0e12 / (4.0 * B * heads * group * D * longest)))))
        causal = rng.random() < 0.6
        block = rng.choice([1, 1, _log_int(rng, 2, 2000)])
        case = _attn("", B=B, H=heads * group, group=group, N=N, D=D, page=page, longest=longest, ragged=rng.random() < 0.5,
                     causal=causal, block=block, window=_log_int(rng, 1, 8) if causal and block > 1 and rng.random() < 0.5 else -1,
                     sink=rng.choice([0, block]), packed=rng.random() < 0.5)
    else:
        M = rng.choice([1, 1, 2, 4, rng.randint(1, 16)])
        N, K = (max(32, _log_int(rng, 64, hi) // step * step) for hi, step in ((20480, rng.choice([1, 16])), (8192, rng.choice([1, 32]))))
        case = _rows("", M=M, N=N, K=K, type=rng.choice(["bf16", "f16", "f32"]), out=rng.choice(["bf16", "f16", "f32"]),
                     silu=rng.random() < 0.4, gelu=rng.random() < 0.3)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 29)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _power(exponent):
    """2^exponent in 32 bits for whole exponents of normal numbers."""
    return ((exponent + 127) << 23).view(torch.float32)


def _scaled(v, exponent):
    """v 2^exponent, in two steps that are both normal numbers."""
    half = exponent // 2
    return v * _power(half) * _power(exponent - half)


def _to_grid(v):
    """E2M1 magnitudes of v [..., multiple of 32] in 32 bits, as blocks of 32, and the blocks' exponents."""
    blocks = v.unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    exponent = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(-127, 127).to(torch.int32)
    t = _scaled(blocks.abs(), -exponent[..., None])
    step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
    return (torch.round(t / step) * step).clamp(max=6.0), exponent


def _encode(v):
    """Packed codes [..., n / 2] and scale bytes [..., n / 32] of v [..., n]."""
    mag, exponent = _to_grid(v)
    code = torch.zeros_like(mag, dtype=torch.uint8)
    for edge in _GRID[1:]:
        code += mag >= edge
    code = code.flatten(-2) + 8 * torch.signbit(v).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), (exponent + 127).to(torch.uint8)


def _fake_quant(v):
    """The values that v's microscaled 4-bit form stands for."""
    mag, exponent = _to_grid(v)
    scaled = _scaled(mag, exponent[..., None]).flatten(-2)
    return torch.where(v < 0, -scaled, scaled)


def _decode(codes, scales):
    """Values of packed codes [..., n / 2] and scale bytes [..., n / 32] in 32 bits."""
    table = torch.tensor(_GRID + tuple(-g for g in _GRID), device=codes.device)
    v = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(torch.int32)]
    return _scaled(v.unflatten(-1, (-1, 32)), scales.to(torch.int32)[..., None] - 127).flatten(-2)


def _operand_shape(rows, cols):
    tiles = -(-cols // 256) * 2
    return -(-rows // 16), tiles, -(-tiles // 4)


def _weights(gen, N, K):
    """Weights as a program keeps them: 4-bit codes and scales in operand order."""
    rt, ct, groups = _operand_shape(N, K)
    w = torch.zeros(rt * 16, groups * 512, device="cuda")
    w[:N, :K] = _randn(gen, N, K) / math.sqrt(K)
    codes, scales = _encode(w)
    codes = codes[:, :ct * 64].reshape(rt, 16, ct, 4, 16).permute(0, 2, 3, 1, 4).contiguous().view(-1)
    scales = scales.view(rt, 16, groups, 4, 4).permute(0, 2, 4, 1, 3).contiguous().view(-1)
    return codes, scales


def _record(case):
    """Bytes of a page's record for one head."""
    return case["page"] * (case["D"] + case["D"] // 16)


def _lengths(case, seed):
    """What the sequences hold: the longest first, the others anywhere below it where lengths are ragged."""
    rnd = torch.Generator().manual_seed(int(seed) * 31 + 7)
    top = case["longest"]
    lens = [top] + [max(1, int(top * float(torch.rand(1, generator=rnd)))) if case["ragged"] else top for _ in range(case["B"] - 1)]
    return lens


def _prepare_pages(case, seed, st):
    B, ps, top, chunk = case["B"], case["page"], case["longest"], case["chunk"]
    rnd = torch.Generator().manual_seed(int(seed) * 31 + 7)
    held = (torch.rand(B, generator=rnd) * top).to(torch.int32)
    grow = 1 + (torch.rand(B, generator=rnd) * chunk).to(torch.int32).clamp(max=chunk - 1)
    wanted = held + grow
    done = torch.rand(B, generator=rnd) < case["shrink"]
    wanted[done] = (held[done].float() * torch.rand(int(done.sum()), generator=rnd)).to(torch.int32) // 2
    count = lambda n: -(-n // ps)  # noqa: E731
    max_pages = count(top + chunk)
    used, pages = int(count(held).sum()), B * max_pages + 8
    order = torch.randperm(pages, generator=rnd).to(torch.int32)
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    at = 0
    for b in range(B):
        n = int(count(held[b]))
        table[b, :n] = order[at:at + n]
        at += n
    free = torch.full((pages,), -1, dtype=torch.int32)
    free[:pages - used] = order[used:]
    one = lambda n: torch.tensor([n], dtype=torch.int32).cuda()  # noqa: E731
    st.update(pages=pages, table=table.cuda(), lengths=held.cuda(), wanted=wanted.cuda(), free=free.cuda(), count=one(pages - used),
              new_lengths=torch.empty(B, dtype=torch.int32, device="cuda"), new_count=one(0), status=one(0),
              slots=torch.empty(B, chunk, dtype=torch.int64, device="cuda"))
    return st


def _prepare_write(case, seed, st):
    gen = _gen(seed)
    B, H, N, D, ps, dtype = case["B"], case["H"], case["N"], case["D"], case["page"], _TYPES[case["type"]]
    if case["packed"]:                                     # [B, N, q | k | v] as a fused projection leaves it
        x = (_randn(gen, B, N, 3 * H * D) * torch.exp(0.5 * _randn(gen, B, N, 1))).to(dtype)
        st["k"], st["v"] = (x[..., i * H * D:(i + 1) * H * D].view(B, N, H, D).transpose(1, 2) for i in (1, 2))
    else:
        st["k"], st["v"] = ((_randn(gen, B, H, N, D) * torch.exp(0.5 * _randn(gen, B, H, N, 1))).to(dtype) for _ in range(2))
    rnd = torch.Generator().manual_seed(int(seed) * 31 + 7)
    per = -(-N // ps) + 1
    pages = B * per + 3
    order = torch.randperm(pages, generator=rnd)[:B * per].view(B, per)
    at = torch.arange(N)[None, :] + torch.randint(0, ps, (B, 1), generator=rnd)      # new tokens begin anywhere in a page
    slots = order.gather(1, at // ps) * ps + at % ps
    if case["padded"]:
        used = 1 + (torch.rand(B, 1, generator=rnd) * N).long().clamp(max=N - 1)
        slots = torch.where(torch.arange(N)[None, :] < used, slots, -1)
    st.update(pages=pages, slots=slots.contiguous().cuda(), data=torch.zeros(pages * H * _record(case), dtype=torch.uint8, device="cuda"))
    st["k_out"], st["v_out"] = (torch.zeros(B, H, N, D, dtype=_TYPES[case["out"]], device="cuda") for _ in range(2))
    return st


def _prepare_attn(case, seed, st):
    gen = _gen(seed)
    B, H, G, N, D, ps = (case[k] for k in ("B", "H", "group", "N", "D", "page"))
    heads, lens = H // G, _lengths(case, seed)
    need = [-(-n // ps) for n in lens]
    pages, max_pages = sum(need) + 2, max(need)
    rnd = torch.Generator().manual_seed(int(seed) * 31 + 11)
    order = torch.randperm(pages, generator=rnd).to(torch.int32)
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    data = torch.zeros(pages, heads, _record(case), dtype=torch.uint8, device="cuda")
    at = 0
    for b, n in enumerate(need):
        rows = n * ps
        # keys of a frame have a direction in common, which some queries look for
        common = _randn(gen, heads, -(-rows // 64), D).repeat_interleave(64, 1)[:, :rows]
        k = _randn(gen, heads, rows, D) + 0.7 * common
        v = _randn(gen, heads, rows, D) + 0.3 * common
        page = order[at:at + n].cuda().long()
        parts = []
        for x in (k, v):
            codes, scales = _encode(x)
            parts.append((codes.view(heads, n, -1).transpose(0, 1), scales.view(heads, n, -1).transpose(0, 1)))
        data[page] = torch.cat([parts[0][0], parts[1][0], parts[0][1], parts[1][1]], -1)
        table[b, :n] = order[at:at + n]
        at += n
    q_lens = [min(N, n) for n in lens]
    if case["window"] >= 0:                                # pages that no query of the chunk sees any more have been given back
        for b, n in enumerate(lens):
            first = ((n - q_lens[b]) // case["block"] - case["window"]) * case["block"]
            lo, hi = -(-case["sink"] // ps), max(0, first) // ps
            if lo < hi:
                table[b, lo:hi] = -1
    if case["packed"]:
        q = _randn(gen, B, N, 3 * H * D).to(torch.bfloat16)[..., :H * D].view(B, N, H, D).transpose(1, 2)
        o = torch.zeros(B, N, H, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    else:
        q = _randn(gen, B, H, N, D).to(torch.bfloat16)
        o = torch.zeros(B, H, N, D, dtype=torch.bfloat16, device="cuda")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()  # noqa: E731
    st.update(pages=pages, table=table.cuda(), data=data.view(-1), q=q, o=o, lse=torch.zeros(B, H, N, device="cuda"), kv_len=i32(lens),
              q_len=i32(q_lens) if min(q_lens) < N else None, lens=lens, q_lens=q_lens)
    return st


def prepare(case, seed):
    """Inputs, tables, the cache or the weights, and buffers of one call in HBM."""
    op, st = case["op"], {"case": case}
    if op == "pages":
        return _prepare_pages(case, seed, st)
    if op == "write":
        return _prepare_write(case, seed, st)
    if op == "attn":
        return _prepare_attn(case, seed, st)
    gen, M, N, K = _gen(seed), case["M"], case["N"], case["K"]
    st["x"] = _randn(gen, M, K).to(_TYPES[case["type"]])
    st["w"], st["w_scales"] = _weights(gen, N, K)
    st["bias"] = 0.1 * _randn(gen, N)
    st["out"] = torch.empty(M, N, dtype=_TYPES[case["out"]], device="cuda")
    return st


# ---------------------------------------------------------------------------------------------- the framework's operators

def _run_own(st):
    import paper_2502_01776_amd as S
    case, op = st["case"], st["case"]["op"]
    if op == "rows":
        S.svg_fp4_linear_rows(S.tokens_of(st["x"]), st["x"], S.SVG_ACT_SILU if case["silu"] else S.SVG_ACT_NONE, case["N"], st["w"],
                              st["w_scales"], st["bias"], S.SVG_ACT_GELU_TANH if case["gelu"] else S.SVG_ACT_NONE,
                              S.tokens_of(st["out"]), st["out"])
        return {"out": st["out"]}
    if op == "pages":
        table = st["table"]
        cache = S.kv4_cache(case["B"], st["pages"], table.shape[1], 1, 64, case["page"], page_table=table)
        S.svg_kv4_resize(cache, st["lengths"], st["wanted"], st["free"], st["count"], st["new_lengths"], st["new_count"], st["slots"],
                         case["chunk"], st["status"])
        return {k: st[k] for k in ("table", "new_lengths", "free", "new_count", "slots", "status")}
    if op == "write":
        cache = S.kv4_cache(case["B"], st["pages"], 0, case["H"], case["D"], case["page"], data=st["data"])
        S.svg_kv4_write(cache, S.tokens_of(st["k"]), st["k"], S.tokens_of(st["v"]), st["v"], st["slots"])
        S.svg_kv4_read(cache, st["slots"], S.tokens_of(st["k_out"]), st["k_out"], S.tokens_of(st["v_out"]), st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"]}
    cache = S.kv4_cache(case["B"], st["pages"], st["table"].shape[1], case["H"] // case["group"], case["D"], case["page"],
                        data=st["data"], page_table=st["table"])
    attn = S.kv4_attn(kv_len=st["kv_len"], q_len=st["q_len"], max_kv=case["longest"], causal=case["causal"], block=case["block"],
                      window=case["window"], sink=case["sink"])
    q_tokens, o_tokens = S.tokens_of(st["q"]), S.tokens_of(st["o"])
    n = S.svg_kv4_attn_workspace_bytes(cache, attn, q_tokens)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    S.svg_kv4_attn_fwd(cache, attn, q_tokens, st["q"], o_tokens, st["o"], st["lse"], ws, n)
    return {"o": st["o"], "lse": st["lse"]}


# ---------------------------------------------------------------------------------------------- the plain form

def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _gelu(v):
    return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))


def _unpack(codes, scales, rows, cols):
    """A matrix in operand order -> its values [rows, cols] in 32 bits."""
    rt, ct, groups = _operand_shape(rows, cols)
    codes = codes.view(rt, ct, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(rt * 16, ct * 64)
    scales = scales.view(rt, groups, 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(rt * 16, groups * 16)[:, :ct * 4]
    return _decode(codes, scales)[:rows, :cols]


def _plain_pages(st):
    case, lens, wanted = st["case"], st["lengths"].long(), st["wanted"].long()
    ps, B, N = case["page"], case["B"], case["chunk"]
    have, want = -(-lens // ps), -(-wanted // ps)
    table, free, count = st["table"].clone(), st["free"].clone(), st["count"].long()
    entry = torch.arange(table.shape[1], device="cuda")[None, :]
    back = (entry >= want[:, None]) & (entry < have[:, None])
    take = (entry >= have[:, None]) & (entry < want[:, None])
    released, granted = back.sum(), take.sum()
    rank = lambda mask: torch.cumsum(mask.flatten().long(), 0).view_as(mask) - 1  # noqa: E731
    place = torch.arange(free.shape[0], device="cuda")
    free[count + torch.arange(int(released), device="cuda")] = table[back]      # (row by row, entries ascending)
    stack = count + released - 1 - rank(take)
    bad = (wanted < 0) | (wanted > table.shape[1] * ps) | (wanted - lens > N)
    ok = (granted <= count + released) & ~bad.any()
    table = torch.where(take & ok, free[stack.clamp(0, place[-1])], table)
    i = torch.arange(N, device="cuda")[None, :]
    at = lens[:, None] + i
    slots = table.long().gather(1, (at // ps).clamp(max=table.shape[1] - 1)) * ps + at % ps
    slots = torch.where((at < wanted[:, None]) & ok, slots, -1)
    new_count = torch.where(ok, count + released - granted, count)
    return {"table": table, "new_lengths": torch.where(ok, wanted, lens).to(torch.int32), "free": free,
            "new_count": new_count.to(torch.int32), "slots": slots, "status": (~ok).to(torch.int32).view(1)}


def _held(st, b, n):
    """Codes and scale bytes of keys and of values of sequence b's first n tokens, [heads, n, ...], and which of them exist."""
    case = st["case"]
    ps, D, heads = case["page"], case["D"], case["H"] // case["group"]
    page = st["table"][b, :-(-n // ps)].long()
    rec = st["data"].view(st["pages"], heads, -1)[page.clamp(min=0)].transpose(0, 1)
    cuts = [0, ps * D // 2, ps * D, ps * (D + D // 32), ps * (D + D // 16)]
    parts = [rec[..., a:z].reshape(heads, page.shape[0] * ps, -1)[:, :n] for a, z in zip(cuts[:-1], cuts[1:])]
    return parts, (page >= 0).repeat_interleave(ps)[:n]


def _visible(case, n, q_n, rows, exists):
    """[rows, n]: may query row i (of q_n, the sequence's last ones) see key j?"""
    block = case["block"]
    j = torch.arange(n, device="cuda")[None, :]
    own_block = torch.div(n - q_n + rows, block, rounding_mode="floor")[:, None]
    seen = exists[None, :]
    if case["causal"]:
        seen = seen & (j // block <= own_block)
    if case["window"] >= 0:
        seen = seen & ((j // block >= own_block - case["window"]) | (j < case["sink"]))
    return seen.expand(rows.shape[0], n)


def _plain_attn(st):
    case = st["case"]
    H, G, D = case["H"], case["group"], case["D"]
    o, lse = torch.zeros_like(st["o"]), torch.zeros_like(st["lse"])
    for b, (n, q_n) in enumerate(zip(st["lens"], st["q_lens"])):
        (kc, vc, ks, vs), exists = _held(st, b, n)
        q = st["q"][b, :, :q_n].float() / math.sqrt(D)
        step = max(1, min(H // G, _SCORES // (n * G * min(q_n, 2048))))
        for h in range(0, H // G, step):
            k, v = _decode(kc[h:h + step], ks[h:h + step]), _decode(vc[h:h + step], vs[h:h + step])
            heads = slice(h * G, (h + k.shape[0]) * G)
            for a in range(0, q_n, 2048):
                z = min(q_n, a + 2048)
                seen = _visible(case, n, q_n, torch.arange(a, z, device="cuda"), exists)
                scores = torch.matmul(q[heads, a:z].reshape(k.shape[0], G * (z - a), D), k.transpose(1, 2).contiguous())
                scores = scores.view(k.shape[0], G, z - a, n).masked_fill(~seen, -math.inf)
                top = scores.amax(-1, keepdim=True)
                e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
                total = e.sum(-1, keepdim=True)
                out = torch.matmul(e.view(k.shape[0], G * (z - a), n), v).view(k.shape[0], G, z - a, D)
                out = torch.where(total > 0, out / total, 0.0)
                o[b, heads, a:z] = out.reshape(-1, z - a, D).to(o.dtype)
                lse[b, heads, a:z] = (top + torch.log(total)).reshape(-1, z - a)
    return {"o": o, "lse": lse}


def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "pages":
        return _plain_pages(st)
    if op == "write":
        there = (st["slots"] >= 0)[:, None, :, None]
        return {n: torch.where(there, _fake_quant(st[n].float()), st[n + "_out"].float()).to(st[n + "_out"].dtype) for n in ("k", "v")}
    if op == "attn":
        return _plain_attn(st)
    x = st["x"].float()
    out = (_silu(x) if case["silu"] else x) @ _unpack(st["w"], st["w_scales"], case["N"], case["K"]).t() + st["bias"]
    return {"out": (_gelu(out) if case["gelu"] else out).to(st["out"].dtype)}


def run(state):
    """One pass through a case's operators and its outputs."""
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------- the same in 64 bits

def _exact_power(e):
    """2^e in 64 bits for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_mx(v):
    """Microscaled 4-bit values of v [..., n] in 64 bits: the scale by comparison with powers of two, the value by
    comparison with the midpoints of neighbouring grid values (a tie goes to the even code)."""
    block = v.unflatten(-1, (-1, 32))
    size = block.abs()
    top = size.amax(-1, keepdim=True)
    E = torch.floor(torch.log2(top.clamp(min=1e-300)))
    E = torch.where(_exact_power(E) > top, E - 1, E)
    E = torch.where(_exact_power(E + 1) <= top, E + 1, E)
    unit = _exact_power((E - 2).clamp(-127, 127))
    t, value = size / unit, torch.zeros_like(size)
    for i in range(7):
        mid = (_GRID[i] + _GRID[i + 1]) / 2
        value += (_GRID[i + 1] - _GRID[i]) * ((t > mid) if i % 2 == 0 else (t >= mid))
    return (value * unit).copysign(block).flatten(-2)


def _exact_values(codes, scales):
    """Values of packed codes and scale bytes in 64 bits, one half of the bytes after the other."""
    grid = torch.tensor([s * g for s in (1, -1) for g in _GRID], dtype=torch.float64, device="cuda")
    unit = _exact_power(scales.long() - 127).repeat_interleave(16, -1)
    out = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device="cuda")
    out[..., 0::2] = grid[(codes % 16).long()] * unit
    out[..., 1::2] = grid[(codes // 16).long()] * unit
    return out


def _exact_pages(st):
    """The lists walked on the host, one page after the other."""
    case, ps, N = st["case"], st["case"]["page"], st["case"]["chunk"]
    table, lens, wanted = st["table"].tolist(), st["lengths"].tolist(), st["wanted"].tolist()
    free, count = st["free"].tolist(), int(st["count"])
    stack = free[:count]
    for row, have, want in zip(table, lens, wanted):
        for j in range(-(-want // ps), -(-have // ps)):
            stack.append(row[j])
    free[:len(stack)] = stack
    for row, have, want in zip(table, lens, wanted):
        for j in range(-(-have // ps), -(-want // ps)):
            row[j] = stack.pop()
    slots = [[row[(have + i) // ps] * ps + (have + i) % ps if have + i < want else -1 for i in range(N)]
             for row, have, want in zip(table, lens, wanted)]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()  # noqa: E731
    return {"table": i32(table), "new_lengths": i32(wanted), "free": i32(free), "new_count": i32([len(stack)]),
            "slots": torch.tensor(slots, dtype=torch.int64).cuda(), "status": i32([0])}


def _exact_attn(st):
    case = st["case"]
    B, H, G, N, D, block, ps = (case[k] for k in ("B", "H", "group", "N", "D", "block", "page"))
    o = torch.zeros(B, H, N, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, H, N, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, q_n = st["lens"][b], st["q_lens"][b]
        parts, exists = _held(st, b, n)
        key = torch.arange(n, device="cuda")
        for h in range(H // G):
            k, v = (_exact_values(c[h], s[h]) for c, s in ((parts[0], parts[2]), (parts[1], parts[3])))
            for a in range(0, q_n, 1024):
                z = min(a + 1024, q_n)
                place = torch.arange(n - q_n + a, n - q_n + z, device="cuda")
                # the first key of the first block and the end of the last block that a query sees
                begin = torch.zeros_like(place) if case["window"] < 0 else (place // block - case["window"]) * block
                end = (place // block + 1) * block if case["causal"] else torch.full_like(place, n)
                seen = (key >= begin[:, None]) & (key < end[:, None])
                if case["window"] >= 0:
                    seen |= (key < case["sink"]) & (key < end[:, None])
                seen &= exists
                for g in range(G):
                    s = (st["q"][b, h * G + g, a:z].double() @ k.t().contiguous()) * (D ** -0.5)
                    s[~seen] = -math.inf
                    lse[b, h * G + g, a:z] = torch.logsumexp(s, 1)
                    o[b, h * G + g, a:z] = torch.exp(s - lse[b, h * G + g, a:z, None]).nan_to_num(0.0) @ v
    return {"o": o, "lse": lse}


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "pages":
        return _exact_pages(st)
    if op == "write":
        out = {}
        for name in ("k", "v"):
            out[name] = torch.zeros(st[name].shape, dtype=torch.float64, device="cuda")
            for b in range(case["B"]):
                rows = (st["slots"][b] >= 0).nonzero()[:, 0]
                out[name][b, :, rows] = _exact_mx(st[name][b, :, rows].double())
        return out
    if op == "attn":
        return _exact_attn(st)
    x = st["x"].double()
    rt, ct, groups = _operand_shape(case["N"], case["K"])
    codes = st["w"].view(rt, ct, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(rt * 16, ct * 64)
    scales = st["w_scales"].view(rt, groups, 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(rt * 16, groups * 16)[:, :ct * 4]
    w = _exact_values(codes, scales)[:case["N"], :case["K"]]
    out = (x * torch.sigmoid(x) if case["silu"] else x) @ w.t().contiguous() + st["bias"].double()
    return {"out": out * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (out + 0.044715 * out ** 3)) if case["gelu"] else out}


# ---------------------------------------------------------------------------------------------- what cannot be avoided

def _visible_pairs(case, n, q_n):
    """(query, key) pairs that take part in a sequence of n tokens whose last q_n are queries."""
    block, pairs, place = case["block"], 0, n - q_n
    while place < n:
        same = min(n, (place // block + 1) * block) - place if case["causal"] or case["window"] >= 0 else q_n
        end = min(n, (place // block + 1) * block) if case["causal"] else n
        begin = max(0, (place // block - case["window"]) * block) if case["window"] >= 0 else 0
        seen = end - begin + (min(begin, case["sink"]) if case["window"] >= 0 else 0)
        pairs += same * seen
        place += same
    return pairs


def work(case):
    """Bytes: inputs read once, outputs written once, 4-bit elements in 4.25 bits; a cache is counted as far as some query sees it.
    Operations: the products, and for the others those of the formulas.  Ragged lengths count as half the longest."""
    size, op = {"bf16": 2.0, "f16": 2.0, "f32": 4.0}, case["op"]
    if op == "pages":
        slots = float(case["B"]) * case["chunk"]
        return {"bytes": 8 * slots + 12.0 * case["B"] + 4 * slots / case["page"], "flops": 4 * slots}
    if op == "write":
        n = 2.0 * case["B"] * case["H"] * case["N"] * case["D"]
        return {"bytes": n * (size[case["type"]] + size[case["out"]]) + 8.0 * case["B"] * case["N"], "flops": 6 * n}
    if op == "attn":
        flops = cached = 0.0
        for b in range(case["B"]):
            n = case["longest"] if b == 0 or not case["ragged"] else max(1, case["longest"] // 2)
            q_n = min(case["N"], n)
            flops += 4.0 * case["H"] * case["D"] * _visible_pairs(case, n, q_n)
            first = max(0, ((n - q_n) // case["block"] - case["window"]) * case["block"]) if case["window"] >= 0 else 0
            cached += n - first + min(first, case["sink"])
        rows = float(case["B"]) * case["H"] * case["N"]
        return {"bytes": rows * (4 * case["D"] + 4) + cached * (case["H"] // case["group"]) * case["D"] * 1.0625, "flops": flops}
    M, N, K = float(case["M"]), float(case["N"]), float(case["K"])
    return {"bytes": M * K * size[case["type"]] + N * K * 0.53125 + M * N * size[case["out"]] + 4 * N, "flops": 2.0 * M * N * K}
