"""Page tables from lengths, and rows into a 4-bit cache's pages and out of them, against the oracle: all exact."""
import numpy as np
import pytest
import torch

import paper_2502_01776_amd as S
from oracle import block_oracle as B
from oracle import kv4_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


# ---- page tables ---------------------------------------------------------------------------------------------------

def state(rng, sequences, page_size, longest, chunk, shrinking, spare):
    """A pool of which some sequences hold pages, and what they want next."""
    held = rng.integers(0, longest + 1, sequences)
    wanted = held + rng.integers(0, chunk + 1, sequences)
    less = rng.random(sequences) < shrinking
    wanted[less] = rng.integers(0, held[less] + 1) if less.any() else 0
    max_pages = -(-(longest + chunk) // page_size) + 1
    used = -(-held // page_size)
    pages = int(used.sum()) + spare
    order = rng.permutation(pages)
    table = np.full((sequences, max_pages), -7)
    at = 0
    for b in range(sequences):
        table[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
    free = np.full(pages, -3)
    free[:pages - at] = order[at:]
    return table, held, wanted, free, pages - at


def check_resize(table, held, wanted, free, count, page_size, tokens, in_place=False, slots=True, expect=None):
    ref = O.resize(table, held, wanted, free, count, page_size, tokens, slots)
    if expect is not None:
        assert ref[5] == expect
    n = len(held)
    t, f, h, w, c = dev(table), dev(free), dev(held), dev(wanted), dev([count])
    nh, nc = (h, c) if in_place else (torch.full((n,), -9, dtype=torch.int32, device="cuda"), torch.full((1,), -9, dtype=torch.int32, device="cuda"))
    sl = torch.full((n, tokens), -9, dtype=torch.int64, device="cuda") if slots else None
    status = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    cache = S.kv4_cache(n, len(free), table.shape[1], 1, 64, page_size, page_table=t)
    S.svg_kv4_resize(cache, h, w, f, c, nh, nc, sl, tokens, status)
    torch.cuda.synchronize()
    names = ("table", "free", "lengths", "count", "slots", "status")
    for name, got, want in zip(names, (t, f, nh, nc, sl, status), ref):
        if got is not None:
            assert np.array_equal(got.cpu().numpy().reshape(np.shape(want)), want), name
    if not in_place:
        assert np.array_equal(h.cpu().numpy(), held) and c.item() == count
    return ref


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sequences, page_size, longest, chunk, shrinking, spare", [
    (1, 16, 0, 1, 0.0, 3), (1, 16, 272, 64, 0.0, 40), (1, 64, 500, 1, 0.0, 3), (2, 16, 100, 33, 0.5, 40), (7, 32, 1000, 200, 0.3, 90),
    (64, 16, 63, 17, 0.5, 200), (255, 64, 700, 64, 0.2, 600), (256, 16, 40, 16, 0.9, 0), (257, 16, 40, 16, 0.6, 300), (600, 16, 90, 40, 0.4, 900),
    (3, 256, 30000, 2049, 0.0, 40), (2, 16, 5000, 6000, 0.0, 800), (1500, 16, 20, 5, 0.5, 1600),
    (300, 64, 9000, 4200, 0.5, 20000)])
def test_page_tables(sequences, page_size, longest, chunk, shrinking, spare, in_place):
    rng = np.random.default_rng(sequences * 1000 + page_size + longest)
    for _ in range(3):
        check_resize(*state(rng, sequences, page_size, longest, chunk, shrinking, spare), page_size, chunk, in_place)


def test_pages_given_back_are_granted_in_the_same_call():
    """No free page at all: what the first sequences give back is what the last ones take, in the stack's order."""
    rng = np.random.default_rng(5)
    for n in (2, 40, 300, 700):
        table = rng.permutation(n * 4).reshape(n, 4)
        held = np.full(n, 64)
        wanted = np.where(np.arange(n) % 2 == 0, rng.integers(0, 49, n), 64)
        held[1::2] = 16
        table[1::2, 1:] = -1
        free = np.full(n * 4, -3)
        spare = int((-(-wanted // 16) - -(-held // 16)).clip(min=0).sum() - (-(-held // 16) - -(-wanted // 16)).clip(min=0).sum())
        count = max(0, spare)
        free[:count] = np.arange(count) + 100000 % (n * 4)
        check_resize(table, held, wanted, free, count, 16, 48, expect=O.OK)


def test_page_tables_that_cannot_be_made_change_nothing():
    rng = np.random.default_rng(6)
    for in_place in (False, True):
        table, held, wanted, free, count = state(rng, 9, 16, 100, 40, 0.0, 2)
        wanted[:] = held + 40
        check_resize(table, held, wanted, free, count, 16, 40, in_place, expect=O.FULL)
        table, held, wanted, free, count = state(rng, 9, 16, 100, 40, 0.3, 400)
        for b, value in ((4, -1), (8, 10 ** 6), (0, 2 ** 31 - 1), (0, -2 ** 31)):
            bad = wanted.copy()
            bad[b] = value
            check_resize(table, held, bad, free, count, 16, 40, in_place, expect=O.LENGTHS)
            bad = held.copy()
            bad[b] = value
            check_resize(table, bad, wanted, free, count, 16, 40, in_place, expect=O.LENGTHS)
        check_resize(table, held, wanted, free, -1, 16, 40, in_place, expect=O.LENGTHS)
        check_resize(table, held, wanted, free, len(free) + 1, 16, 40, in_place, expect=O.LENGTHS)
        check_resize(table, held, held + 40, free, count, 16, 39, in_place, expect=O.LENGTHS)
        # nothing to take, and no room for what is given back
        check_resize(table, held, 0 * held, free, len(free) - 1, 16, 40, in_place, expect=O.LENGTHS)


def test_page_tables_without_slots_and_without_sequences():
    rng = np.random.default_rng(7)
    for n in (1, 30):
        check_resize(*state(rng, n, 16, 3000, 9000, 0.2, 30 * 600), 16, 0, slots=False)
        table, held, wanted, free, count = state(rng, n, 16, 300, 40, 1.0, 5)
        check_resize(table, held, wanted, free, count, 16, 0)             # slots asked for, of no tokens
    check_resize(np.zeros((0, 4)), np.zeros(0, int), np.zeros(0, int), np.arange(5), 5, 16, 4)


def test_entries_outside_of_the_pool_give_no_slot():
    table, held, wanted = np.full((1, 4), -1), np.array([20]), np.array([60])
    table[0, 1] = 9
    check_resize(table, held, wanted, np.array([1, 2, -5, 7, 0, 0, 0, 0]), 4, 16, 40)


# ---- rows into pages and out of them ---------------------------------------------------------------------------------

def tensors(B_, N, H, D, dtype, layout, seed, offset=0):
    gen = torch.Generator().manual_seed(seed)
    if layout == "heads":
        make = lambda: torch.randn(B_, H, N, D, generator=gen)  # noqa: E731
        k, v = make(), make()
    else:
        wide = torch.randn(B_, N, 3 * H * D + offset, generator=gen)
        k, v = (wide[..., offset + i * H * D:offset + (i + 1) * H * D].view(B_, N, H, D).transpose(1, 2) for i in (1, 2))
    scale = torch.exp(2 * torch.randn(B_, 1, N, 1, generator=gen))
    return [(x * scale).to(dtype) for x in (k, v)] if layout == "heads" else list(_in_wide(k, v, scale, dtype, offset))


def _in_wide(k, v, scale, dtype, offset):
    B_, H, N, D = k.shape
    wide = torch.zeros(B_, N, 3 * H * D + offset, dtype=dtype, device="cuda")
    for i, x in ((1, k), (2, v)):
        view = wide[..., offset + i * H * D:offset + (i + 1) * H * D].view(B_, N, H, D).transpose(1, 2)
        view.copy_((x * scale).to(dtype))
        yield view


def rows_64(x):
    """[B,H,N,D] -> [B N, H, D] in 64 bits."""
    return x.detach().cpu().double().numpy().transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])


def nibbles_equal(a, b):
    """Codes are compared as values: a zero may have either sign."""
    for shift in (0, 4):
        x, y = (a >> shift) & 15, (b >> shift) & 15
        if not ((x == y) | ((x & 7 == 0) & (y & 7 == 0))).all():
            return False
    return True


def check_rows(k, v, slots, pages, page_size, out_type=torch.float32):
    B_, H, N, D = k.shape
    k, v = k.cuda() if not k.is_cuda else k, v.cuda() if not v.is_cuda else v
    data = torch.full((pages, H, O.record_bytes(D, page_size)), 0xA7, dtype=torch.uint8, device="cuda")
    ref = data.cpu().numpy()
    O.write(ref, rows_64(k), rows_64(v), slots.reshape(-1), page_size)
    cache = S.kv4_cache(B_, pages, 0, H, D, page_size, data=data)
    assert S.svg_kv4_bytes(cache) == data.numel()
    sl = dev(slots, np.int64)
    S.svg_kv4_write(cache, S.tokens_of(k), k, S.tokens_of(v), v, sl)
    torch.cuda.synchronize()
    got, codes = data.cpu().numpy(), page_size * D
    assert np.array_equal(got[..., codes:], ref[..., codes:]), "scale bytes"
    assert nibbles_equal(got[..., :codes], ref[..., :codes]), "codes"
    back = [torch.full((B_, H, N, D), 3.0, dtype=out_type, device="cuda") for _ in range(2)]
    S.svg_kv4_read(cache, sl, S.tokens_of(back[0]), back[0], S.tokens_of(back[1]), back[1])
    there = (slots.reshape(-1) >= 0) & (slots.reshape(-1) < pages * page_size)
    for x, want in zip(back, O.read(ref, slots.reshape(-1), D, page_size)):
        x, want = rows_64(x), np.where(there[:, None, None], want, 3.0)
        tiny = np.abs(want) < (2.0 ** -126 if out_type != torch.float16 else 2.0 ** -14)
        if out_type == torch.float16:                                     # fewer bits of exponent
            with np.errstate(over="ignore"):
                want = np.where(tiny, want, want.astype(np.float16).astype(np.float64))
            assert np.array_equal(x[~tiny], want[~tiny], equal_nan=True) and (np.abs(x - want)[tiny] <= 2.0 ** -25).all()
        else:
            assert np.array_equal(np.where(tiny, 0, x), np.where(tiny, 0, want), equal_nan=True)
    return data


def some_slots(rng, B_, N, page_size, skipped=0.0):
    per = -(-N // page_size) + 1
    pages = B_ * per + 2
    order = rng.permutation(pages)[:B_ * per].reshape(B_, per)
    at = np.arange(N)[None, :] + rng.integers(0, page_size, (B_, 1))
    slots = np.take_along_axis(order, at // page_size, 1) * page_size + at % page_size
    slots[rng.random(slots.shape) < skipped] = -1
    return slots.astype(np.int64), pages


@pytest.mark.parametrize("layout", ["heads", "packed"])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B_, N, H, D, page_size", [(1, 1, 1, 64, 16), (1, 1, 1, 128, 16), (8, 1, 3, 128, 64), (2, 33, 4, 64, 32), (1, 300, 5, 128, 128),
                                                  (3, 17, 2, 64, 16), (1, 65, 1, 128, 1024)])
def test_rows_into_pages(B_, N, H, D, page_size, kind, layout):
    rng = np.random.default_rng(N * 10 + H)
    k, v = tensors(B_, N, H, D, TYPES[kind], layout, seed=N + H)
    slots, pages = some_slots(rng, B_, N, page_size, 0.1 if N > 1 else 0.0)
    check_rows(k, v, slots, pages, page_size, TYPES[kind])


def test_rows_of_odd_alignment_and_unlike_types():
    rng = np.random.default_rng(3)
    slots, pages = some_slots(rng, 2, 19, 16)
    for kind in TYPES.values():
        k, v = tensors(2, 19, 3, 64, kind, "packed", 4, offset=1)
        check_rows(k, v, slots, pages, 16)
    k, _ = tensors(2, 19, 3, 128, torch.float32, "heads", 5)
    _, v = tensors(2, 19, 3, 128, torch.float16, "packed", 6, offset=3)
    check_rows(k, v, slots, pages, 16, torch.bfloat16)


def test_rows_of_one_run_of_columns():
    """[rows, H*D] as the token matrix of a projection's output gives the same bytes as [1, H, rows, D]."""
    rng = np.random.default_rng(4)
    slots, pages = some_slots(rng, 1, 21, 16)
    k, v = tensors(1, 21, 4, 128, torch.bfloat16, "heads", 7)
    data = check_rows(k, v, slots, pages, 16)
    flat = [x.cuda().transpose(1, 2).reshape(21, 4 * 128).contiguous() for x in (k, v)]
    again = torch.full_like(data, 0xA7)
    cache = S.kv4_cache(1, pages, 0, 4, 128, 16, data=again)
    S.svg_kv4_write(cache, S.tokens_of(flat[0]), flat[0], S.tokens_of(flat[1]), flat[1], dev(slots, np.int64))
    assert torch.equal(again, data)


def test_slots_outside_of_the_pool_are_skipped():
    k, v = tensors(1, 8, 2, 64, torch.bfloat16, "heads", 8)
    slots = np.array([[-1, 3, 16 * 5, 16 * 5 - 1, -2 ** 62, 2 ** 62, 2 ** 33, 0]], dtype=np.int64)
    check_rows(k, v, slots, 5, 16)


def test_values_that_are_special():
    k, v = (x.float() for x in tensors(1, 12, 2, 128, torch.float32, "heads", 9))
    k[0, 0, 0, :] = 0.0
    k[0, 0, 1, 5], k[0, 1, 1, 40] = float("inf"), float("nan")
    v[0, 0, 2, 127], v[0, 1, 3, 0] = -float("inf"), float("nan")
    k[0, 0, 4, :32] = 2.0 ** -133 * torch.arange(32)                      # below the smallest scale
    k[0, 0, 5, :] = 3.4e38
    v[0, 0, 6, :32] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4)      # ties
    v[0, 0, 7, :32] = -torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0] * 4)
    v[0, 1, 8, :] = 1.0
    slots = np.arange(12, dtype=np.int64)[None] + 4
    check_rows(k, v, slots, 2, 16)
    check_rows(k[..., :64].contiguous(), v[..., 64:].contiguous(), slots, 2, 16)


def test_places_beyond_32_bits():
    """A pool of more than 4 GB: the last page's record lies behind 2^32 bytes."""
    H, D, page_size = 64, 128, 4096
    pages = 2 ** 32 // (H * O.record_bytes(D, page_size)) + 2
    data = torch.empty(pages * H * O.record_bytes(D, page_size), dtype=torch.uint8, device="cuda")
    k, v = (x.cuda() for x in tensors(1, 5, H, D, torch.bfloat16, "heads", 10))
    slots = np.array([[0, pages * page_size - 1, (pages - 1) * page_size, pages * page_size // 2, 77]])
    cache = S.kv4_cache(1, pages, 0, H, D, page_size, data=data)
    S.svg_kv4_write(cache, S.tokens_of(k), k, S.tokens_of(v), v, dev(slots, np.int64))
    back = [torch.zeros_like(k) for _ in range(2)]
    S.svg_kv4_read(cache, dev(slots, np.int64), S.tokens_of(back[0]), back[0], S.tokens_of(back[1]), back[1])
    for x, y in zip((k, v), back):
        want = B.mx_values(*B.mx_quantise(rows_64(x).reshape(-1, D))).reshape(5, H, D)
        assert np.array_equal(rows_64(y), want)
    record = data.view(pages, H, -1)[pages - 1, H - 1].cpu().numpy()
    assert np.array_equal(record[O.parts(D, page_size)[2][0]:][:4], B.mx_quantise(rows_64(k)[2, H - 1][None])[1][0])
