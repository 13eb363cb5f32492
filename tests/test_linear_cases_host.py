"""That the sizes of tests/linear_cases.py reach what they are there for, by the library's own choice."""
from paper_2403_16863_amd import linear
from tests import linear_cases as cases


def layout(rows_of_n):
    return linear.ROWS_N if rows_of_n else linear.ROWS


def test_every_tile_is_reached_uncut():
    for tile, M, K, N, rows_of_n in cases.ON_TILES:
        assert linear.linear_choice(M, N, K, layout(rows_of_n)) == (tile, 1), (M, K, N)
    for state in (False, True):
        assert {c[0] for c in cases.ON_TILES if c[4] == state} == set(range(linear.linear_num_tiles()))
    assert {c[0] for c in cases.ON_TILES if c[3] % 64 == 0} == set(range(linear.linear_num_tiles()))


def test_sums_are_split():
    for M, K, N, rows_of_n in cases.IN_RANGES:
        assert linear.linear_choice(M, N, K, layout(rows_of_n))[1] > 1, (M, K, N)
    longer = set()
    for M, N, K, w_rows, dw_rows in cases.BACKWARD_IN_RANGES:
        x = linear.linear_choice(M, K, N, linear.ROWS if w_rows else linear.ROWS_N)[1]
        w = linear.linear_choice(*((N, K) if dw_rows else (K, N)), M, linear.TOKENS)[1]
        assert x > 1 and w > 1, (M, N, K)
        longer.add(x * M * K > w * N * K)
    assert longer == {False, True}


def test_the_tests_that_go_through_tiles_go_through_all():
    assert linear.linear_num_tiles() <= 16
