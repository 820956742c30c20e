"""Page tables with pages that are not there, in the 64-bit form (no GPU): pages are neither lost nor made."""
import numpy as np
import pytest

from oracle import kv4_oracle as O


def real(table, lengths, page_size, pages):
    """The pages that the sequences hold."""
    return [int(table[b, j]) for b, n in enumerate(lengths) for j in range(-(-n // page_size)) if 0 <= table[b, j] < pages]


def test_a_finished_sequence_gives_back_the_pages_that_are_there():
    table, free = np.array([[0, -1, -1, 11, 4, 5], [-1] * 6]), np.full(11, -3)
    free[:5] = [6, 7, 8, 9, 10]
    table, free, lengths, count, _, status = O.resize(table, np.array([96, 0]), np.array([0, 0]), free, 5, 16, 96)
    assert status == O.OK and count == 8 and free[:8].tolist() == [6, 7, 8, 9, 10, 0, 4, 5]
    table, free, lengths, count, slots, status = O.resize(table, lengths, np.array([0, 96]), free, count, 16, 96)
    assert status == O.OK and count == 2 and table[1].tolist() == [5, 4, 0, 10, 9, 8] and (slots[1] >= 0).all()


def test_numbers_that_are_no_pages_are_never_granted():
    table, lengths = np.full((1, 4), -1), np.array([0])
    for bad in (-1, -5, 4, 2 ** 30):
        free = np.array([1, bad, 3, 0])
        for wanted, status in ((16, O.OK), (32, O.OK), (33, O.PAGES), (64, O.PAGES)):
            got = O.resize(table, lengths, np.array([wanted]), free, 4, 16, 64)
            assert got[5] == status
            if status != O.OK:
                assert (got[0] == table).all() and (got[1] == free).all() and got[2] == 0 and got[3] == 4 and (got[4] == -1).all()


@pytest.mark.parametrize("seed", range(4))
def test_pages_are_conserved(seed):
    """Sequences grow, shrink and finish while windows leave pages behind."""
    rng = np.random.default_rng(seed)
    n, page_size, max_pages, pages = 5, 16, 12, 40
    table, lengths = np.full((n, max_pages), -1), np.zeros(n, int)
    free, count = rng.permutation(pages), pages
    for _ in range(60):
        wanted = np.clip(lengths + rng.integers(-60, 61, n), 0, max_pages * page_size)
        wanted[rng.random(n) < 0.1] = 0
        table, free, lengths, count, _, status = O.resize(table, lengths, wanted, free, count, page_size, 60)
        assert status in (O.OK, O.FULL)
        for b in range(n):                                                # what lies far behind is given back by hand
            for j in range(1, max(1, lengths[b] // page_size - 3)):
                if table[b, j] >= 0:
                    free[count], table[b, j] = table[b, j], -1
                    count += 1
        assert sorted(free[:count].tolist() + real(table, lengths, page_size, pages)) == list(range(pages))
