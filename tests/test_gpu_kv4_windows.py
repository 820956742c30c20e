"""Attention over the 4-bit cache under windows in every form, whole and in parts: the sizes are looked for on the host until the call is cut as the test wants it,
and the launch's own plan is compared before every check."""
import numpy as np
import pytest
import torch

import kv4_plan
import paper_2502_01776_amd as S
from oracle import kv4_oracle as O
from test_gpu_kv4_attn import Cache, check, plan, queries, run

pytestmark = pytest.mark.gpu

# (block, window, sink): windows of tokens, blocks that begin inside tiles, and sinks that end inside a tile, far in front of the window or beside it
SHORT = [(1, 0, 0), (1, 20, 3), (10, 1, 10), (64, 1, 0), (50, 2, 70), (100, 2, 130), (16, 3, 16)]
LONG = [(100, 2, 1500), (16, 3, 2000), (1, 20, 1790), (64, 10, 1700), (600, 2, 70), (500, 1, 700)]
# many rows are worth parts over thousands of keys only
LONGER = [(100, 2, 4500), (16, 3, 5200), (1, 20, 4800), (64, 10, 4300), (1900, 2, 70), (1350, 2, 1350)]
PAGE = 16


def lengths(form, parts):
    return [500, 330] if not parts else [6500, 1500] if form == 128 else [2900, 1000]


def masks(form, parts):
    return SHORT if not parts else LONGER if form == 128 else LONG


def sizes(form, parts, lens, D, N, causal, block, window, sink):
    """Heads and a capacity with which N rows are cut that way."""
    for capacity in (0, 4096, 16384, 1 << 18):
        for H in (1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256):
            max_pages = -(-max(*lens, capacity) // PAGE)
            p = kv4_plan.plan(S.kv4_cache(len(lens), 1, max_pages, H, D, PAGE), S.kv4_attn(kv_len=None, causal=causal, block=block, window=window, sink=sink), N, 1)
            if p.tile == form and (p.parts > len(lens)) == parts:
                return H, capacity
    raise AssertionError("no size is cut that way")


def cut(cache, q, form, parts, mask):
    p = plan(cache, q, **mask)
    assert p.tile == form and (p.parts > len(cache.lens)) == parts, (p.tile, p.parts)


FORMS = [(f, p, n) for f, n in ((16, 40), (32, 300), (128, 300)) for p in (False, True)]


@pytest.mark.parametrize("form, parts, N", FORMS)
@pytest.mark.parametrize("D", [64, 128])
def test_windows(D, form, parts, N):
    lens, kept = lengths(form, parts), {}
    for block, window, sink in masks(form, parts):
        mask = dict(causal=True, block=block, window=window, sink=sink)
        size = H, capacity = sizes(form, parts, lens, D, N, **mask)
        if size not in kept:
            kept[size] = Cache(lens, H, D, PAGE, seed=form, capacity=capacity)
        cache = kept[size]
        q = queries(2, H, N, D, "packed", block)
        cut(cache, q, form, parts, mask)
        rows, heads = sorted({0, 1, 31, N // 2, N - 2, N - 1} | set(range(0, N, 61))), sorted({0, H - 1})
        check(cache, q, rows=rows, heads=heads, **mask)
        check(cache, q, q_len=[N, N // 3], rows=rows, heads=heads, **mask)


@pytest.mark.parametrize("form, parts, N", FORMS)
@pytest.mark.parametrize("D", [64, 128])
def test_windows_over_pages_that_are_not_there(D, form, parts, N):
    """Pages between sink and window have left, others inside of both are gone too."""
    lens = lengths(form, parts)
    for block, window, sink in masks(form, parts)[4:]:
        mask = dict(causal=True, block=block, window=window, sink=sink)
        H, capacity = sizes(form, parts, lens, D, N, **mask)
        cache = Cache(lens, H, D, PAGE, seed=block + 1, capacity=capacity)
        rng = np.random.default_rng(block)
        for b, n in enumerate(lens):
            first = max(0, ((n - N) // block - window) * block) // PAGE
            if first > -(-sink // PAGE):
                cache.table[b, -(-sink // PAGE):first] = -1
            some = rng.random(-(-n // PAGE)) < 0.2
            cache.table[b, :len(some)][some] = rng.choice([-1, cache.pages, 2 ** 30, -2 ** 31], some.sum())
        cache.dev_table.copy_(torch.from_numpy(cache.table.astype(np.int32)))
        q = queries(2, H, N, D, "heads", block)
        cut(cache, q, form, parts, mask)
        check(cache, q, rows=sorted({0, N - 1} | set(range(0, N, 37))), heads=sorted({0, H - 1}), **mask)


@pytest.mark.parametrize("form, parts, N", FORMS)
@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite_under_windows(D, form, parts, N):
    """They spoil the queries whose window or sink holds them, in their 32 channels (values) or whole (keys), and nothing else, bit for bit."""
    lens = lengths(form, parts)
    block, window, sink = (50, 2, 70) if not parts else (1350, 2, 1350) if form == 128 else (500, 1, 700)
    mask = dict(causal=True, block=block, window=window, sink=sink)
    H, capacity = sizes(form, parts, lens, D, N, **mask)
    # a value in the sink, values in the window of some queries, a key in the window of some, a key that nobody sees any more
    spots = [(0, "v", 3, 0, 33), (0, "v", lens[0] - N // 2, H - 1, 5), (0, "k", lens[0] - N - block // 2, 0, 7), (1, "v", lens[1] - 3, 0, D - 1), (1, "k", sink - 1, H - 1, 0)]
    first = ((lens[0] - N) // block - window) * block
    if first > sink:
        spots.append((0, "k", (first + sink) // 2, 0, 1))

    def odd(b, k, v):
        for seq, what, token, head, channel in spots:
            if seq == b:
                (k if what == "k" else v)[token, head, channel] = np.inf if what == "v" and head else np.nan
    plain, spoilt = (Cache(lens, H, D, PAGE, seed=6, odd=o, capacity=capacity) for o in (None, odd))
    q = queries(2, H, N, D, "heads", 6)
    cut(plain, q, form, parts, mask)
    want, want_lse = run(plain, q, **mask)
    got, got_lse = run(spoilt, q, **mask)
    for b, n in enumerate(lens):
        nan = torch.zeros(H, N, D, dtype=torch.bool)
        nan_lse = torch.zeros(H, N, dtype=torch.bool)
        for i in range(N):
            see = O.seen(n, N, i, block, True, window, sink)
            for seq, what, token, head, channel in spots:
                if seq == b and see[token]:
                    nan[head, i, slice(None) if what == "k" else slice(channel // 32 * 32, channel // 32 * 32 + 32)] = True
                    nan_lse[head, i] |= what == "k"
        nan, nan_lse = nan.cuda(), nan_lse.cuda()
        assert nan.any()                                                  # (with a single head, all of a sequence may be)
        assert torch.equal(torch.isnan(got[b]), nan) and torch.equal(got[b][~nan], want[b][~nan])
        assert torch.equal(torch.isnan(got_lse[b]), nan_lse) and torch.equal(got_lse[b][~nan_lse], want_lse[b][~nan_lse])
