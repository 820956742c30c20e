"""Which form of a product a call takes (host side, no GPU), and that the products the forms are tested with reach all of them."""
import itertools

import pytest

from product_forms import PLACES, PRODUCTS, ROWS1, ROWS2, ROWS2_EIGHT, ROWS4, SQUARE, TILE, TILES128, TILES64, column_tiles, form


def turns(M, N, f):
    m, n = TILE[f]
    return 2 if -(-M // m) * -(-N // n) > PLACES[f] else 1


def test_the_tested_products_reach_every_form_loop_and_tail():
    straight, loops = set(), set()
    for (M, N, K, D), act in itertools.product(PRODUCTS, (False, True)):
        assert N % D == 0 and D % 8 == 0
        f = form(M, N, K, act)
        assert f == form(M, N, K, act, operand=True)         # results of one arithmetic: compared bit for bit
        kt = column_tiles(K)
        if f in TILE:
            loops.add((f, act, turns(M, N, f), kt // 4 if f == TILES64 else min(kt // 4, 1), kt % 4))
        else:
            straight.add((f, kt % 4))
    assert {f for f, _ in straight} == {ROWS1, ROWS2_EIGHT, ROWS2, ROWS4} and {rest for f, rest in straight} == {0, 2}
    # groups of four steps: none, an even and an odd number (the 64 x 128 form takes them in pairs), each without and with half of one behind
    for groups, rest in ((0, 2), (1, 0), (1, 2), (2, 0), (2, 2), (3, 2)):
        assert (TILES64, False, 1, groups, rest) in loops, (groups, rest)
    for groups, rest in ((0, 2), (1, 0), (1, 2), (2, 0), (2, 2)):
        assert (TILES64, True, 2, groups, rest) in loops, (groups, rest)
    for f, turn, (groups, rest) in itertools.product((TILES128, SQUARE), (1, 2), ((0, 2), (1, 0), (1, 2))):
        assert (f, False, turn, groups, rest) in loops, (f, turn, groups, rest)
    assert {f for f, act, *_ in loops if act} == set(TILE)


def test_the_activation_decides_the_form_of_some_of_them():
    flips = {(form(M, N, K, False), form(M, N, K, True)) for M, N, K, _ in PRODUCTS}
    assert flips >= {(TILES128, TILES64), (SQUARE, TILES64)}


@pytest.mark.parametrize("M,N,K,act,expected", [
    (1, 5120, 5120, False, ROWS1), (16, 30720, 5120, False, ROWS1), (17, 8160, 512, False, ROWS2_EIGHT), (17, 8161, 512, False, ROWS2),
    (32, 20480, 5120, False, ROWS2), (33, 20480, 5120, False, ROWS4), (64, 20480, 5120, False, ROWS4), (65, 6400, 512, False, ROWS4),
    (65, 6401, 512, False, TILES64), (226, 5120, 4096, False, TILES64), (2048, 5120, 5120, False, SQUARE), (4096, 5120, 5120, False, TILES128),
    (32760, 5120, 20480, False, SQUARE), (17776, 512, 8192, False, SQUARE), (8000, 4096, 1024, True, SQUARE), (1573, 6144, 1536, True, TILES64)])
def test_the_choice(M, N, K, act, expected):
    assert form(M, N, K, act) == expected
