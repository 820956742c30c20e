"""Page tables of sequences some of whose pages are not there: what a window has left behind, and a stack with numbers that are no pages."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import kv4_oracle as O
from test_gpu_kv4 import check_resize, dev, state

pytestmark = pytest.mark.gpu


def punch(rng, table, held, free, count, page_size, share):
    """Pages here and there leave the sequences for the stack; their entries become numbers outside of the pool."""
    pages = len(free)
    for b, n in enumerate(held):
        for j in np.nonzero(rng.random(-(-n // page_size)) < share)[0]:
            if rng.random() < 0.8:                                        # (the others are in use elsewhere)
                free[count] = table[b, j]
                count += 1
            table[b, j] = rng.choice([-1, -1, -7, pages, 2 ** 30, 2 ** 31 - 1, -2 ** 31])
    return count


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sequences, page_size, longest, chunk, shrinking, spare, share", [
    (1, 16, 272, 64, 1.0, 3, 0.5), (1, 16, 200000, 1, 1.0, 0, 0.3), (2, 16, 400, 200, 0.5, 9, 1.0), (7, 32, 1000, 200, 0.5, 0, 0.4),
    (64, 16, 63, 17, 0.5, 0, 0.3), (255, 64, 700, 64, 0.5, 0, 0.5), (256, 16, 40, 16, 0.9, 0, 0.2), (257, 16, 140, 16, 0.6, 0, 0.5),
    (600, 16, 90, 40, 0.6, 0, 0.4), (3, 16, 60000, 30000, 0.7, 0, 0.4), (900, 16, 300, 5, 0.5, 0, 0.1)])
def test_tables_with_holes(sequences, page_size, longest, chunk, shrinking, spare, share, in_place):
    rng = np.random.default_rng(sequences * 1000 + page_size + longest)
    seen = set()
    for _ in range(4):
        table, held, wanted, free, count = state(rng, sequences, page_size, longest, chunk, shrinking, spare)
        wanted[rng.random(sequences) < 0.2] = 0
        count = punch(rng, table, held, free, count, page_size, share)
        seen.add(check_resize(table, held, wanted, free, count, page_size, chunk, in_place)[5])
    assert O.LENGTHS not in seen and O.PAGES not in seen


@pytest.mark.parametrize("n", [2, 40, 300, 700])
def test_pages_given_back_beside_holes_are_granted_in_the_same_call(n):
    """An empty stack: the sequences with even numbers give back, the others take all of it."""
    rng = np.random.default_rng(n)
    table = rng.permutation(n * 8).reshape(n, 8)
    table[::2][rng.random((-(-n // 2), 8)) < 0.4] = -1
    table[1::2] = -1
    held, wanted = np.where(np.arange(n) % 2 == 0, 128, 0), np.zeros(n, int)
    left = int((table[::2] >= 0).sum())
    for b in range(1, n, 2):
        take = min(left, int(rng.integers(1, 8)))
        wanted[b], left = 16 * take, left - take
    free = np.full(n * 8, -3)
    for in_place in (False, True):
        ref = check_resize(table, held, wanted, free, 0, 16, 128, in_place, expect=O.OK)
        assert ref[3] == left
    wanted[n // 2 * 2 - 1] += 16 * (left + 1)
    check_resize(table, held, wanted, free, 0, 16, 128 + 16 * (left + 1), expect=O.FULL if wanted.max() <= 128 else O.LENGTHS)


def test_room_on_the_stack_is_for_pages_that_are_there():
    """Six pages, three of them already on the stack: finishing takes three places, not six."""
    table, free = np.array([[0, -1, -1, 9, 4, 5]]), np.array([1, 2, 3, 6, 7, 8, -1, -1, -1])
    for in_place in (False, True):
        ref = check_resize(table, np.array([96]), np.array([0]), free, 6, 16, 0, in_place, expect=O.OK)
        assert ref[3] == 9 and sorted(ref[1].tolist()) == list(range(9))
        check_resize(table, np.array([96]), np.array([0]), free, 7, 16, 0, in_place, expect=O.LENGTHS)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sequences", [1, 3, 300])
def test_numbers_that_are_no_pages_are_never_granted(sequences, in_place):
    rng = np.random.default_rng(sequences)
    for bad in (-1, -2 ** 31, None, 2 ** 31 - 1):
        table, held, wanted, free, count = state(rng, sequences, 16, 100, 40, 0.0, 4 * sequences + 6)
        wanted = held + 17                                                # one page or two each
        taken = int((-(-wanted // 16) - -(-held // 16)).sum())
        bad = len(free) if bad is None else bad
        for at in {count - 1, count - taken, count - 1 - taken // 2}:     # the first, the last and one between
            wrong = free.copy()
            wrong[at] = bad
            check_resize(table, held, wanted, wrong, count, 16, 40, in_place, expect=O.PAGES)
        wrong = free.copy()
        wrong[:count - taken], wrong[count:] = bad, bad                   # not taken in this call
        check_resize(table, held, wanted, wrong, count, 16, 40, in_place, expect=O.OK)


def test_tokens_in_the_rest_of_a_page_that_is_not_there_have_no_slot():
    table = np.array([[3, -1, 5, -1]])
    ref = check_resize(table, np.array([20]), np.array([60]), np.array([0, 1, 2, 4, 6, 7, -1, -1]), 6, 16, 40, expect=O.OK)
    assert (ref[4][0, :12] == -1).all() and (ref[4][0, 12:] >= 0).all()


def test_a_window_moves_and_its_pages_come_back():
    """Three sequences grow by a frame a step, the pages behind their windows are given back, the last frames are attended to; then they finish one after the
    other.  The pool is smaller than what they would hold without a window, and at the end all of it is free."""
    n, H, D, ps, frame, window, sink, steps = 3, 2, 64, 16, 40, 1, 24, 9
    max_pages, pages = -(-frame * steps // ps), 36
    rng = np.random.default_rng(1)
    table, free = np.full((n, max_pages), -1), rng.permutation(pages)
    t, f, lengths, c = dev(table), dev(free), dev(np.zeros(n)), dev([pages])
    wanted, status = torch.zeros_like(lengths), dev([0])
    slots = torch.zeros(n, frame, dtype=torch.int64, device="cuda")
    data = torch.full((pages, H, O.record_bytes(D, ps)), 0xFF, dtype=torch.uint8, device="cuda")
    cache = S.kv4_cache(n, pages, max_pages, H, D, ps, data=data, page_table=t)
    host = data.cpu().numpy()
    for step in range(steps):
        wanted.copy_(lengths + frame)
        S.svg_kv4_resize(cache, lengths, wanted, f, c, lengths, c, slots, frame, status)
        assert status.item() == S.SVG_KV4_OK and (slots >= 0).all() and len(set(slots.flatten().tolist())) == n * frame
        q, k, v = (torch.randn(n, H, frame, D, generator=torch.Generator().manual_seed(10 * step + i)).to(torch.bfloat16).cuda() for i in range(3))
        S.svg_kv4_write(cache, S.tokens_of(k), k, S.tokens_of(v), v, slots)
        rows = lambda x: x.double().cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, H, D)  # noqa: E731
        O.write(host, rows(k), rows(v), slots.flatten().tolist(), ps)
        attn = S.kv4_attn(kv_len=lengths, causal=True, block=frame, window=window, sink=sink)
        need = S.svg_kv4_attn_workspace_bytes(cache, attn, S.tokens_of(q))
        o, ws = torch.zeros_like(q), torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
        S.svg_kv4_attn_fwd(cache, attn, S.tokens_of(q), q, S.tokens_of(o), o, None, ws, need)
        place, now = frame * (step + 1), t.cpu().numpy()
        for b in range(n):
            j = np.arange(place)
            kk, vv = O.read(host, now[b, j // ps] * ps + j % ps, D, ps)
            see = O.seen(place, frame, 0, frame, True, window, sink)
            assert (now[b, j[see] // ps] >= 0).all()
            ref, _, size, slack = O.attention(q[b, :, :1].double().cpu().numpy(), kk[see], vv[see], np.ones(see.sum(), bool), D ** -0.5)
            e = (D + 10) * 2.0 ** -23 * slack + 2.0 ** -21
            tol = 2.0 ** -8 * np.abs(ref[:, 0]) + (2.0 ** -8 + 2 * e + (place / 32 + 64) * 2.0 ** -23) * size[:, 0] * 1.01
            assert (np.abs(o[b, :, 0].double().cpu().numpy() - ref[:, 0]) <= tol).all(), (step, b)
        # whole pages between the sink and the next frame's window go back
        behind = max(0, (step + 1 - window) * frame) // ps
        count = c.item()
        for b in range(n):
            for e in range(-(-sink // ps), behind):
                if now[b, e] >= 0:
                    f[count], t[b, e] = int(now[b, e]), -1
                    count += 1
        c.fill_(count)
    assert n * max_pages > pages
    for b in range(n):
        wanted.copy_(lengths)
        wanted[b] = 0 if b != 1 else 50                                   # (the second one is cut off behind its sink first)
        S.svg_kv4_resize(cache, lengths, wanted, f, c, lengths, c, slots, frame, status)
        assert status.item() == S.SVG_KV4_OK
    wanted.zero_()
    S.svg_kv4_resize(cache, lengths, wanted, f, c, lengths, c, slots, frame, status)
    assert status.item() == S.SVG_KV4_OK and c.item() == pages and sorted(f.tolist()) == list(range(pages))


def test_a_captured_call_on_tables_with_holes():
    """Replayed with the caller's own edits between the replays, every one against the lists walked by hand."""
    rng, n, ps, chunk = np.random.default_rng(8), 40, 16, 90
    table, held, wanted, free, count = state(rng, n, ps, 300, chunk, 0.4, 400)
    count = punch(rng, table, held, free, count, ps, 0.3)
    t, f, lengths, c, w, status = dev(table), dev(free), dev(held), dev([count]), dev(wanted), dev([-9])
    slots = torch.zeros(n, chunk, dtype=torch.int64, device="cuda")
    cache = S.kv4_cache(n, len(free), table.shape[1], 1, 64, ps, page_table=t)
    before = [x.clone() for x in (t, f, lengths, c)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    call = lambda: S.svg_kv4_resize(cache, lengths, w, f, c, lengths, c, slots, chunk, status)  # noqa: E731
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for x, y in zip((t, f, lengths, c), before):
        x.copy_(y)
    seen = set()
    for _ in range(8):
        graph.replay()
        scratch = torch.randn(1 << 18, device="cuda").sum()               # eager work of our own between the replays
        torch.cuda.synchronize()
        assert torch.isfinite(scratch)
        ref = O.resize(table, held, wanted, free, count, ps, chunk)
        seen.add(ref[5])
        for name, got, want in zip(("table", "free", "lengths", "count", "slots", "status"), (t, f, lengths, c, slots, status), ref):
            assert np.array_equal(got.cpu().numpy().reshape(np.shape(want)), want), name
        table, free, held, count = ref[:4]
        count = punch(rng, table, held, free, count, ps, 0.1)
        wanted = np.clip(held + rng.integers(-200, chunk + 1, n), 0, table.shape[1] * ps)
        for x, y in ((t, table), (f, free), (w, wanted), (c, [count])):
            x.copy_(dev(y))
    assert O.OK in seen
