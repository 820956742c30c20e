"""Attention over the 4-bit cache with scores of any finite size that are no powers of two: far beyond what an exponential or a rounded reference can hold.

Keys of one row are m 2^a throughout, with m one of 1, 1.5, 2, 3, 4, 6, and queries 1.25 2^b: a score is D 1.25 m 2^(a+b), exact in fp32.  The largest is at least 1.3
times the next one in size, so where scores pass 1000 only the rows with the largest count, all with the same weight: o is the mean of their values."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import kv4_oracle as O
from test_gpu_kv4_attn import Cache, plan, room, run

pytestmark = pytest.mark.gpu

SIZES = np.array([1, 1.5, 2, 3, 4, 6])


def sized(lens, D, a, sign, order, seed, capacity):
    rng = np.random.default_rng(seed)
    sizes = [rng.choice(SIZES, n) for n in lens]
    sizes = [np.sort(x) if order == "up" else np.sort(x)[::-1] if order == "down" else x for x in sizes]

    def odd(b, k, v):
        k[:] = sign * sizes[b][:, None, None] * 2.0 ** a
    return Cache(lens, 1, D, 16, seed=seed, odd=odd, capacity=capacity), sizes


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N, form", [(1, 16), (30, 16), (30, 32), (140, 32), (140, 128)])
@pytest.mark.parametrize("order", ["up", "down", "any"])
def test_scores_of_any_size(order, N, form, D):
    lens = [333, 200, 70]
    capacity = room(form, lens, 1, D, 16, N)
    for a, b, sign in ((5, 3, 1), (10, 9, -1), (12, 12, 1), (13, 12, -1), (14, 13, 1), (15, 13, -1), (17, 17, 1), (30, 20, -1), (40, 37, 1), (55, 54, -1), (55, 54, 1)):
        cache, sizes = sized(lens, D, a, sign, order, a + N, capacity)
        q = torch.full((3, 1, N, D), 1.25 * 2.0 ** b, dtype=torch.bfloat16, device="cuda")
        assert plan(cache, q).tile == form
        o, lse = run(cache, q)
        for i, size in enumerate(sizes):
            best = size.max() if sign > 0 else size.min()
            top = np.nonzero(size == best)[0]
            _, v = O.read(cache.host, cache.slots(i)[top], D, 16)
            mean, magnitude = v[:, 0].mean(0), np.abs(v[:, 0]).mean(0)
            # weights of one and none, with a common factor that bf16 rounds once: sums of n keys, the factor's and the result's rounding
            tol = 2.0 ** -8 * np.abs(mean) + (2.0 ** -8 + (len(size) / 32 + 64) * 2.0 ** -23) * magnitude
            assert (np.abs(o[i, 0].double().cpu().numpy() - mean) <= tol).all(), (a, b, sign, i)
            score = sign * D ** 0.5 * 1.25 * best * 2.0 ** (a + b)
            # scale log2 e rounded twice, the score, the sum's logarithm and its way back: fewer than eight roundings
            assert (np.abs(lse[i, 0].double().cpu().numpy() - score - np.log(len(top))) <= 2.0 ** -21 * abs(score) + 1e-4).all(), (a, b, sign, i)


@pytest.mark.parametrize("N, form", [(1, 16), (40, 32), (140, 128)])
def test_rows_with_far_scores_leave_the_others_alone(N, form):
    """Queries of ordinary size in one tile with far ones: bit for bit what they are without them."""
    lens, D = [500, 90], 128
    cache = Cache(lens, 2, D, 16, seed=5, capacity=room(form, lens, 2, D, 16, N))
    gen = torch.Generator().manual_seed(N)
    q = torch.randn(2, 2, N, D, generator=gen).to(torch.bfloat16).cuda()
    want, want_lse = run(cache, q, causal=True)
    far = q.clone()
    far[:, :, ::3] *= 2.0 ** 40
    assert plan(cache, far).tile == form
    got, got_lse = run(cache, far, causal=True)
    rest = [i for i in range(N) if i % 3]
    assert torch.equal(got[:, :, rest], want[:, :, rest]) and torch.equal(got_lse[:, :, rest], want_lse[:, :, rest])
    assert torch.isfinite(got.float()).all() and torch.isfinite(got_lse[:, :, ::3][want_lse[:, :, ::3].isfinite()]).all()


def test_far_scores_in_parts():
    """The largest score lies in one part of many."""
    lens, D = [9001], 64
    for at in (0, 4000, 9000):
        def odd(b, k, v):
            k[:] = 3 * 2.0 ** 20
            k[at] = 4 * 2.0 ** 20
        cache = Cache(lens, 1, D, 64, seed=at, odd=odd)
        for N in (1, 130):
            q = torch.full((1, 1, N, D), 1.25 * 2.0 ** 20, dtype=torch.bfloat16, device="cuda")
            assert plan(cache, q).parts > 1
            o, lse = run(cache, q)
            _, v = O.read(cache.host, cache.slots(0)[[at]], D, 64)
            assert (np.abs(o[0, 0].double().cpu().numpy() - v[0, 0]) <= 2.0 ** -7 * np.abs(v[0, 0])).all()
            score = D ** 0.5 * 5 * 2.0 ** 40
            assert (np.abs(lse[0, 0].double().cpu().numpy() - score) <= 2.0 ** -21 * score).all()
