"""Attention over the 4-bit cache against the 64-bit form over the same cache.

Tolerance.  A weight is 2^x with x from an fp32 sum of D exact products: its relative error is e = (D + 8) 2^-23 slack + 2^-21 (+ 2^-23 for each unit
of the exponent, at most slack log2 e of them), slack being the magnitude a score is added up from.  Rounding it to bf16 adds 2^-8, the
result's rounding 2^-8 of the result.  fp32 sums over n keys add (n / 32 + 64) 2^-23 of the magnitude summed.  The log-sum-exp has e, the sums' part and
its own rounding.  A weight below 2^-126 of the row's largest is zero: 2^-126 of the largest |v| for each key."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
import kv4_plan
from oracle import kv4_oracle as O

pytestmark = pytest.mark.gpu


class Cache:
    """Sequences of random keys and values in pages in any order; whatever no sequence holds is 0xFF bytes (NaN scales)."""

    def __init__(self, lens, H, D, page_size, seed=0, spread=1.0, spare=3, odd=None, capacity=0):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.D, self.page_size = list(lens), H, D, page_size
        need = [-(-n // page_size) for n in lens]
        self.pages, self.max_pages = sum(need) + spare, max(need + [1, -(-capacity // page_size)])
        order = rng.permutation(self.pages)
        self.table = np.full((len(lens), self.max_pages), -1)
        data = np.full((self.pages, H, O.record_bytes(D, page_size)), 0xFF, dtype=np.uint8)
        at = 0
        for b, n in enumerate(lens):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            k, v = (rng.standard_normal((n, H, D)) * spread for _ in range(2))
            if odd is not None:
                odd(b, k, v)
            O.write(data, k, v, self.slots(b), page_size)
        self.host = data
        self.data = torch.from_numpy(data).cuda()
        self.dev_table = torch.from_numpy(self.table.astype(np.int32)).cuda()

    def slots(self, b, n=None):
        j = np.arange(self.lens[b] if n is None else n)
        return self.table[b, j // self.page_size] * self.page_size + j % self.page_size

    def desc(self):
        return S.kv4_cache(len(self.lens), self.pages, self.max_pages, self.H, self.D, self.page_size, data=self.data, page_table=self.dev_table)


def i32(a):
    return torch.tensor(list(a), dtype=torch.int32, device="cuda")


def queries(B, H, N, D, layout, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(B, H, N, D, generator=gen) * scale).to(torch.bfloat16)
    if layout == "heads":
        return x.cuda()
    wide = torch.zeros(B, N, 3 * H * D + (5 if layout == "odd" else 0), dtype=torch.bfloat16, device="cuda")
    first = 5 if layout == "odd" else 0
    view = wide[..., first:first + H * D].view(B, N, H, D).transpose(1, 2)
    view.copy_(x)
    return view


def run(cache, q, kv_len=None, q_len=None, max_kv=0, scale=0.0, out=None, fill=7.0, **mask):
    B, H, N, D = q.shape
    o = torch.full((B, H, N, D), fill, dtype=torch.bfloat16, device="cuda") if out is None else out
    lse = torch.full((B, H, N), fill, device="cuda")
    c = cache.desc()
    kv = i32(cache.lens if kv_len is None else kv_len)
    attn = S.kv4_attn(kv_len=kv, q_len=None if q_len is None else (ql := i32(q_len)), max_kv=max_kv, softmax_scale=scale, **mask)
    n = S.svg_kv4_attn_workspace_bytes(c, attn, S.tokens_of(q))
    ws = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    S.svg_kv4_attn_fwd(c, attn, S.tokens_of(q), q, S.tokens_of(o), o, lse, ws, n)
    torch.cuda.synchronize()
    return o, lse


def check(cache, q, kv_len=None, q_len=None, max_kv=0, scale=0.0, rows=None, heads=None, **mask):
    """rows, heads: the queries and their heads that the oracle computes (all where None)."""
    o, lse = run(cache, q, kv_len, q_len, max_kv, scale, **mask)
    B, H, N, D = q.shape
    heads = list(range(H)) if heads is None else heads
    for b in range(B):
        n = cache.lens[b] if kv_len is None else kv_len[b]
        n = max(0, min(n, cache.max_pages * cache.page_size))
        q_n = N if q_len is None else max(0, min(q_len[b], N))
        j = np.arange(n)
        page = cache.table[b, j // cache.page_size]
        exists = (page >= 0) & (page < cache.pages)
        k, v = O.read(cache.host, np.where(exists, page * cache.page_size + j % cache.page_size, -1), D, cache.page_size)
        wanted = range(q_n) if rows is None else [i for i in rows if i < q_n]
        for i in wanted:
            see = np.nonzero(O.seen(n, q_n, i, mask.get("block", 1), mask.get("causal", False), mask.get("window", -1), mask.get("sink", 0)) & exists)[0]
            got, got_lse = o[b, heads, i].double().cpu().numpy(), lse[b, heads, i].double().cpu().numpy()
            if not len(see):
                assert (got == 0).all() and np.isneginf(got_lse).all(), (b, i)
                continue
            one = np.ones(len(see), dtype=bool)
            group = H // cache.H
            own = [h // group for h in heads]                            # a head of the cache for each: the oracle's heads are not shared
            ref, ref_lse, size, slack = O.attention(q[b, heads, i:i + 1].double().cpu().numpy(), k[see][:, own], v[see][:, own], one, scale or D ** -0.5)
            e = (D + 8 + 1.4427) * 2.0 ** -23 * slack + 2.0 ** -21
            sums = (len(see) / 32 + 64) * 2.0 ** -23
            tol = 2.0 ** -8 * np.abs(ref[:, 0]) + (2.0 ** -8 + 2 * e + sums) * size[:, 0] * (1 + 2.0 ** -7) + len(see) * 2.0 ** -126 * np.abs(v[see][:, own]).max()
            bad = np.abs(got - ref[:, 0]) > tol
            assert not bad.any(), (b, i, float((np.abs(got - ref[:, 0]) / tol).max()))
            tol = e[:, 0] + sums + 2.0 ** -22 * np.abs(ref_lse[:, 0])
            assert (np.abs(got_lse - ref_lse[:, 0]) <= tol).all(), (b, i, float((np.abs(got_lse - ref_lse[:, 0]) / tol).max()))
        assert (o[b, :, q_n:] == 7).all() and (lse[b, :, q_n:] == 7).all(), "rows behind the last query"
    return o, lse


# The same rows take another form where the page table could hold more keys: its parts are then many and short, some of them empty.
def room(form, lens, H, D, page_size, N, group=1):
    """A capacity of the page table with which N rows of `group` heads take the form with `form` rows."""
    pages = [max(-(-max(lens) // page_size), -(-n // page_size)) for n in (0,) + tuple(1 << i for i in range(9, 25))]
    for n in pages:
        cache = S.kv4_cache(len(lens), 1, n, H, D, page_size)
        if n * page_size <= 1 << 23 and kv4_plan.plan(cache, S.kv4_attn(kv_len=None), N, group).tile == form:
            return n * page_size
    raise AssertionError("no capacity makes this form the best")


def plan(cache, q, **kw):
    return kv4_plan.plan(cache.desc(), S.kv4_attn(kv_len=i32(cache.lens), **kw), q.shape[2], q.shape[1] // cache.H)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N, form", [(n, f) for n in (1, 3, 16, 17, 31, 33, 129, 200) for f in (16, 32, 128) if f == 16 or n > f // 2])
def test_lengths_of_queries_and_keys(form, N, D):
    lens = [1, 15, 16, 17, 63, 64, 65, 200, 517]
    cache = Cache(lens, 2, D, 16, seed=N, capacity=room(form, lens, 2, D, 16, N))
    q = queries(len(lens), 2, N, D, "heads", N)
    assert plan(cache, q).tile == form
    check(cache, q, rows=range(0, N, 1 if N < 20 else 13))                # queries without a token of their own among them
    check(cache, q, rows=range(0, N, 1 if N < 20 else 13), causal=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B, group", [(1, 1), (3, 1), (70, 1), (1, 3)])
def test_form_with_128_rows_in_one_part(B, group, D):
    """So many heads that no sequence is cut: results straight from the registers."""
    H = 384 // group // min(B, 24)
    rng = np.random.default_rng(B)
    lens = [960] + [int(x) for x in rng.integers(1, 961, B - 1)]
    cache = Cache(lens, H, D, 32, seed=B)
    N = 210
    q = queries(B, H * group, N, D, "packed", B)
    q_len = [N] + [int(x) for x in rng.integers(0, N + 1, B - 1)]
    for mask in (dict(causal=True), dict(causal=True, block=100, window=2, sink=70), dict()):
        p = plan(cache, q, **mask)
        assert p.tile == 128 and p.parts == B
        check(cache, q, q_len=q_len, rows=range(0, N, 41), heads=[0, H * group // 2, H * group - 1], **mask)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form, B, heads, N", [(16, 3, 9, 70), (32, 1, 100, 210), (32, 70, 2, 130)])
def test_forms_with_fewer_rows_in_one_part(form, B, heads, N, D):
    """Results straight from the sums of the workgroup."""
    lens = [960] + [int(x) for x in np.random.default_rng(B).integers(1, 961, B - 1)]
    cache = Cache(lens, heads, D, 32, seed=B)
    q = queries(B, heads, N, D, "packed", B)
    for mask in (dict(causal=True, block=100, window=5, sink=70), dict(causal=True, window=800), dict(causal=True, block=230, window=3)):
        p = plan(cache, q, **mask)
        assert p.tile == form and p.parts == B
        check(cache, q, rows=range(0, N, 31), heads=[0, heads // 2, heads - 1], **mask)


@pytest.mark.parametrize("N, form", [(1, 16), (40, 32), (71, 128)])
@pytest.mark.parametrize("layout", ["packed", "odd"])
@pytest.mark.parametrize("group, D, page_size", [(1, 64, 32), (3, 128, 64), (4, 64, 16), (7, 128, 16), (16, 64, 256)])
def test_shared_heads_and_layouts(group, D, page_size, layout, N, form):
    cache = Cache([300, 77], 2, D, page_size, seed=group, capacity=room(form, [300, 77], 2, D, page_size, N, group))
    q = queries(2, 2 * group, N, D, layout, group)
    check(cache, q, rows=range(0, N, 7), causal=True)
    check(cache, q, rows=range(0, N, 13), scale=0.31)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block, window, sink, causal", [(1, -1, 0, True), (1, 0, 0, True), (1, 20, 3, True), (10, 1, 10, True), (64, 1, 0, True),
                                                        (50, 2, 64, True), (37, 0, 5, False), (37, 3, 0, False), (1000, 1, 70, True), (7, 0, 0, True)])
def test_masks(block, window, sink, causal, D):
    lens = [400, 131, 9]
    for N, form in ((1, 16), (9, 16), (24, 16), (24, 32), (150, 16), (150, 32), (150, 128)):
        cache = Cache(lens, 1, D, 16, seed=block, capacity=room(form, lens, 1, D, 16, N))
        q = queries(3, 1, N, D, "heads", N)
        check(cache, q, rows=range(0, N, 1 if N < 10 else 7), block=block, window=window, sink=sink, causal=causal)
    q = queries(3, 1, 150, D, "heads", 3)
    check(cache, q, q_len=[150, 20, 0], rows=range(0, 150, 7), block=block, window=window, sink=sink, causal=causal)


@pytest.mark.parametrize("N, form", [(1, 16), (2, 16), (100, 16), (100, 32), (100, 128)])
def test_pages_that_are_not_there(N, form):
    cache = Cache([500, 300, 64], 2, 64, 16, seed=9, capacity=room(form, [500, 300, 64], 2, 64, 16, N))
    cache.table[0, [0, 3, 4, 5, 6, 20]] = [-1, -1, -1, cache.pages, 2 ** 30, -1]
    cache.table[1, :] = -1                                                # nothing at all
    cache.table[2, 3] = -5
    cache.dev_table.copy_(torch.from_numpy(cache.table.astype(np.int32)))
    q = queries(3, 2, N, 64, "heads", 1)
    check(cache, q, rows=range(0, N, 9))
    check(cache, q, rows=range(0, N, 9), causal=True, block=16, window=3, sink=16)


@pytest.mark.parametrize("N, form", [(1, 16), (20, 16), (20, 32), (300, 16), (300, 32), (300, 128)])
def test_lengths_of_the_call(N, form):
    """Empty sequences and query lists, lengths out of range (cut off), no more keys than the hint says."""
    lens = [200, 90, 40, 130]
    cache = Cache(lens, 2, 128, 32, seed=2, capacity=room(form, lens, 2, 128, 32, N))
    q = queries(4, 2, N, 128, "heads", 2)
    check(cache, q, kv_len=[0, 90, -5, 129], q_len=[N, 0, N, -1], rows=range(0, N, 17))
    check(cache, q, kv_len=[0, 1, 40, 2], q_len=[N, N + 100, 1, 2], rows=range(0, N, 17), causal=True)
    check(cache, q, kv_len=[33, 20, 31, 64], max_kv=64, rows=range(0, N, 17))
    full = Cache([224, 224, 224, 224], 2, 128, 32, seed=2)
    o, _ = run(full, q, kv_len=[224] * 4)
    assert torch.equal(run(full, q, kv_len=[2 ** 31 - 1, 225, 2 ** 20, 224])[0], o)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N, form", [(1, 16), (32, 16), (32, 32), (128, 16), (128, 32), (128, 128)])
def test_sharp_rows(N, form, D):
    """Scores of +-60 and more: the reference maximum moves again and again, most weights are zero."""
    def grow(b, k, v):
        k *= np.linspace(0.1, 3, len(k))[:, None, None]
    capacity = room(form, [700], 1, D, 64, N)
    cache = Cache([700], 1, D, 64, seed=4, spread=2.0, odd=grow, capacity=capacity)
    q = queries(1, 1, N, D, "heads", 4, scale=6.0)
    check(cache, q, rows=range(0, N, 5))
    down = Cache([700], 1, D, 64, seed=4, spread=2.0, odd=lambda b, k, v: k.__imul__(np.linspace(3, 0.01, len(k))[:, None, None]), capacity=capacity)
    check(down, q, rows=range(0, N, 5), causal=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N, form", [(1, 16), (30, 16), (30, 32), (140, 32), (140, 128)])
def test_scores_far_below_and_above(N, form, D):
    """Scores of -D 2^109 and of D 2^109 beside lower ones: exact sums of powers of two, far outside of what an exponential can take."""
    def equal(b, k, v):
        k[:] = -2.0 ** 55 if b == 0 else 2.0 ** 55
        if b == 1:
            k[100:] *= 0.5
    lens = [333, 200]
    cache = Cache(lens, 1, D, 16, seed=9, odd=equal, capacity=room(form, lens, 1, D, 16, N))
    q = torch.full((2, 1, N, D), 2.0 ** 54, dtype=torch.bfloat16, device="cuda")
    assert plan(cache, q).tile == form
    o, lse = run(cache, q)
    for b, seen in ((0, 333), (1, 100)):
        _, v = O.read(cache.host, cache.slots(b)[:seen], D, 16)
        # weights of one: exact; sums of n keys, and the result's rounding
        mean, size = v[:, 0].mean(0), np.abs(v[:, 0]).mean(0)
        assert (np.abs(o[b, 0].double().cpu().numpy() - mean) <= 2.0 ** -8 * np.abs(mean) + (seen / 32 + 64) * 2.0 ** -23 * size).all()
        score = (-1.0 if b == 0 else 1.0) * D ** 0.5 * 2.0 ** 109
        assert (np.abs(lse[b, 0].double().cpu().numpy() - score) <= 2.0 ** -20 * abs(score)).all()


@pytest.mark.parametrize("N, form", [(1, 16), (3, 16), (60, 16), (60, 32), (140, 32), (140, 128)])
@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite(N, form, D):
    """They spoil the results of the queries that see them, in their 32 channels (values) or whole (keys), and nothing else, bit for bit."""
    capacity = room(form, [333, 200], 2, D, 16, N)
    plain = Cache([333, 200], 2, D, 16, seed=6, capacity=capacity)
    at = 333 - N // 2 - 1                                                # the queries behind it see it, those in front do not

    def odd(b, k, v):
        if b == 0:
            v[at, 1, 33], v[at, 0, 5] = np.inf, np.nan
        else:
            k[150, 0, 7] = np.nan
    spoilt = Cache([333, 200], 2, D, 16, seed=6, odd=odd, capacity=capacity)
    q = queries(2, 2, N, D, "heads", 6)
    for mask in (dict(), dict(causal=True), dict(causal=True, window=100, sink=2)):
        want, want_lse = run(plain, q, **mask)
        got, got_lse = run(spoilt, q, **mask)
        for i in range(N):
            for b, key in ((0, at), (1, 150)):
                sees = O.seen(plain.lens[b], N, i, 1, mask.get("causal", False), mask.get("window", -1), mask.get("sink", 0))[key]
                nan = torch.zeros(2, D, dtype=torch.bool, device="cuda")
                if sees and b == 0:
                    nan[1, 32:64] = True
                    nan[0, 0:32] = True
                elif sees:
                    nan[0] = True
                assert torch.equal(torch.isnan(got[b, :, i]), nan), (mask, i, b)
                assert torch.equal(got[b, :, i][~nan], want[b, :, i][~nan]), (mask, i, b)
                assert torch.equal(torch.isnan(got_lse[b, :, i]), torch.tensor([bool(sees and b == 1), False], device="cuda"))
        assert torch.equal(got_lse[0], want_lse[0])


@pytest.mark.parametrize("N, H, D", [(1, 2, 128), (1, 1, 64), (30, 1, 128), (130, 1, 64), (130, 2, 128), (2100, 2, 64), (2100, 2, 128)])
def test_long_caches_in_parts(N, H, D):
    """Few workgroups: the keys are cut into parts; the hint changes the cut, and with it the rounding only."""
    lens = [9001, 70]
    cache = Cache(lens, H, D, 64, seed=8)
    q = queries(2, H, N, D, "heads", 8)
    assert S.svg_kv4_attn_workspace_bytes(cache.desc(), S.kv4_attn(kv_len=i32(lens)), S.tokens_of(q)) > 0
    rows = range(0, N, 43 if N < 1000 else 517)
    a, _ = check(cache, q, rows=rows, causal=True)
    b, _ = check(cache, q, rows=rows, causal=True, max_kv=9001)
    c, _ = check(cache, q, rows=rows, causal=True, max_kv=64)               # a hint that is too low costs time, nothing else
    assert torch.equal(a, b)
    check(cache, q, rows=rows, causal=True, block=300, window=2, sink=300)
    assert torch.equal(run(cache, q, causal=True)[0], a)


def test_results_into_views_and_in_front_of_the_last_query():
    cache = Cache([100, 60], 2, 128, 16, seed=3)
    for N in (1, 5, 40):
        q = queries(2, 4, N, 128, "packed", 3)
        want, _ = run(cache, q, q_len=[N, N // 2], causal=True)
        for extra in (0, 3):
            wide = torch.full((2, N, 4 * 128 + 200 + extra), 7.0, dtype=torch.bfloat16, device="cuda")
            view = wide[..., extra:extra + 512].view(2, N, 4, 128).transpose(1, 2)
            got, _ = run(cache, q, q_len=[N, N // 2], causal=True, out=view)
            assert torch.equal(got, want) and (wide[..., :extra] == 7).all() and (wide[..., extra + 512:] == 7).all()


def test_pages_behind_32_bits():
    """A pool of more than 4 GB whose last pages hold the sequence."""
    H, D, page_size = 32, 128, 4096
    small = Cache([9000], H, D, page_size, seed=12, spare=0)
    pages = 2 ** 32 // (H * O.record_bytes(D, page_size)) + 6
    data = torch.empty(pages, H, O.record_bytes(D, page_size), dtype=torch.uint8, device="cuda")
    data[pages - 3:] = small.data
    for N in (1, 40):
        q = queries(1, H, N, D, "heads", 12)
        want = run(small, q, causal=True)
        big = Cache.__new__(Cache)
        big.__dict__.update(small.__dict__, pages=pages, data=data, dev_table=small.dev_table + (pages - 3))
        got = run(big, q, causal=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_calls_on_two_streams_and_another_stream_than_the_tensors():
    cache = Cache([900, 500], 2, 64, 32, seed=13)
    qs = [queries(2, 2, n, 64, "heads", n) for n in (1, 200)]
    want = [run(cache, q, causal=True) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = []
    kv = i32(cache.lens)
    for q, s in zip(qs, streams):
        o, lse = torch.zeros_like(want[len(got)][0]), torch.zeros_like(want[len(got)][1])
        c, attn = cache.desc(), S.kv4_attn(kv_len=kv, causal=True)
        n = S.svg_kv4_attn_workspace_bytes(c, attn, S.tokens_of(q))
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        S.svg_kv4_attn_fwd(c, attn, S.tokens_of(q), q, S.tokens_of(o), o, lse, ws, n, stream=s)
        got.append((o, lse, ws))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
