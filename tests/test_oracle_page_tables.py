"""Pins of the page-table oracle: what it does on cases worked out by hand, and what has to hold on any."""
import random

from oracle.page_tables import LEN_CLAMPED, NO_PAGES, page_tables


def test_rows_take_share_and_give_back():
    held, tables, refs, slots, status = page_tables([40, 0, 33], [0, 0, 0], [[-1] * 3 for _ in range(3)], [0] * 5, 32, ctx_len=[31, 0, 0],
                                                    n_new=[3, 0, 1], kmax=3)
    assert (held, refs, status) == ([2, 0, 2], [1, 1, 1, 1, 0], 0)
    assert tables == [[0, 1, -1], [-1] * 3, [2, 3, -1]]
    assert slots == [[31, 32, 33], [-1] * 3, [64, -1, -1]]
    # row 0 ends, row 1 begins with one page of it, row 2 needs one more: row 0's second page is free again and is the lowest
    held, tables, refs, _, status = page_tables([0, 20, 70], held, tables, refs, 32, share_from=[-1, 0, -1], share_len=[0, 45, 0])
    assert (held, refs, status) == ([0, 1, 3], [1, 1, 1, 1, 0], 0)
    assert tables == [[-1] * 3, [0, -1, -1], [2, 3, 1]]


def test_too_few_pages_stop_the_rows_behind():
    held, tables, refs, slots, status = page_tables([64, 32, 96, 32, 0], [0] * 5, [[-1] * 3 for _ in range(5)], [0] * 4, 32, ctx_len=[0] * 5,
                                                    n_new=[1] * 5, kmax=1)
    assert status == NO_PAGES and held == [2, 1, 0, 0, 0] and refs == [1, 1, 1, 0]
    assert slots == [[0], [64], [-1], [-1], [-1]]


def test_lengths_are_clamped():
    assert page_tables([-1, 1000], [0, 0], [[-1] * 2] * 2, [0] * 8, 32)[4] == LEN_CLAMPED


def test_counts_agree_with_the_tables_whatever_happens():
    rng = random.Random(3)
    for _ in range(50):
        rows, most, pages, P = rng.randint(1, 9), rng.randint(1, 6), rng.randint(4, 40), 32 * rng.randint(1, 3)
        held, tables, refs = [0] * rows, [[-1] * most for _ in range(rows)], [0] * pages
        for _ in range(8):
            length = [rng.choice((0, rng.randint(0, most * P))) for _ in range(rows)]
            held, tables, refs, _, status = page_tables(length, held, tables, refs, P, share_from=[rng.randint(-1, rows - 1) for _ in range(rows)],
                                                        share_len=[rng.randint(0, most * P) for _ in range(rows)])
            count = [0] * pages
            for r in range(rows):
                assert tables[r][held[r]:] == [-1] * (most - held[r]) and len(set(tables[r][:held[r]])) == held[r]
                assert held[r] == -(-length[r] // P) or (status & NO_PAGES and held[r] < -(-length[r] // P))
                for page in tables[r][:held[r]]:
                    count[page] += 1
            assert count == refs
