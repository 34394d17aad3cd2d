"""bass_page_tables against the oracle, entry by entry, over sequences of calls."""
import random

import pytest

from oracle.page_tables import NO_PAGES, page_tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hip():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2404_15778_amd import harness
    return harness


class Both:
    """The same calls on the device and in the oracle."""

    def __init__(self, hip, rows, most, P, pages):
        self.dev = hip.DeviceTables(rows, most, P, pages)
        self.P, self.held, self.tables, self.refs = P, [0] * rows, [[-1] * most for _ in range(rows)], [0] * pages

    def update(self, length, sf=None, sl=None, ctx=None, n=None, kmax=0):
        self.dev.status.zero_()
        got = self.dev.update(length, sf, sl, ctx, n, kmax)
        self.held, self.tables, self.refs, slots, status = page_tables(length, self.held, self.tables, self.refs, self.P, sf, sl, ctx, n, kmax)
        assert self.dev.held.tolist() == self.held
        assert self.dev.tables.tolist() == self.tables
        assert self.dev.refs.tolist() == self.refs
        assert slots is None or got.tolist() == slots
        assert int(self.dev.status.item()) == status
        return status


# rows, table entries, page tokens, pages: one of everything; odd counts; a tile of pages and a bit more; several tiles; more rows than a scan's width
SHAPES = [(1, 1, 32, 1), (3, 7, 96, 20), (16, 40, 64, 4097), (61, 300, 32, 12301), (700, 9, 256, 4096)]


@pytest.mark.parametrize("rows,most,P,pages", SHAPES)
@pytest.mark.parametrize("kmax", [1, 7, 100])
def test_random_calls(hip, rows, most, P, pages, kmax):
    rng = random.Random(rows * 1000 + kmax)
    both, ctx = Both(hip, rows, most, P, pages), [0] * rows
    seen = 0
    for step in range(6):
        length, n, sf, sl = [], [], [], []
        for r in range(rows):
            if rng.random() < 0.2:
                ctx[r] = 0
                length.append(0)
                n.append(0)
            else:
                ctx[r] = rng.choice((ctx[r], rng.randint(0, most * P - 1)))
                n.append(rng.randint(0, kmax))
                length.append(min(ctx[r] + n[-1], most * P))
            sf.append(rng.randint(-2, rows - 1))
            sf[-1] = -1 if sf[-1] == r else sf[-1]
            sl.append(rng.randint(0, most * P))
        seen |= both.update(length, sf if step % 2 else None, sl if step % 2 else None, ctx, n, kmax)
    assert not seen & ~(NO_PAGES | 1)


def test_more_rows_than_are_kept_in_lds(hip):
    """5000 rows, three calls; some share, some end, and some find no pages."""
    rng = random.Random(5)
    rows, most, P, pages = 5000, 3, 32, 4501
    both, seen = Both(hip, rows, most, P, pages), 0
    for _ in range(3):
        length = [rng.choice((0, rng.randint(1, most * P))) for _ in range(rows)]
        sf = [rng.choice((-1, rng.randrange(rows))) for _ in range(rows)]
        sf = [-1 if x == r else x for r, x in enumerate(sf)]
        seen |= both.update(length, sf, [rng.randint(0, most * P) for _ in range(rows)], [max(n - 2, 0) for n in length], [min(n, 2) for n in length], 3)
    assert seen == NO_PAGES


def test_slots_far_beyond_two_to_the_thirty(hip):
    """Page numbers whose slots need all 31 bits."""
    P, pages = 1 << 20, 2047
    both = Both(hip, 2, 2047, P, pages)
    both.update([2000 * P, 0])
    both.update([2000 * P, 46 * P], ctx=[2000 * P - 2, 46 * P - 1], n=[2, 1], kmax=2)


def test_rows_that_find_too_few_keep_what_they_hold(hip):
    both = Both(hip, 4, 8, 32, 10)
    assert both.update([100, 60, 0, 32]) == 0
    assert both.update([256, 96, 33, 64], ctx=[100, 60, 0, 32], n=[4, 4, 4, 4], kmax=4) & NO_PAGES
    assert both.update([0, 96, 33, 64], ctx=[0, 60, 0, 32], n=[0, 4, 4, 4], kmax=4) == 0


def test_a_source_that_ends_in_the_same_call(hip):
    both = Both(hip, 5, 6, 32, 12)
    both.update([150, 0, 0, 0, 0])
    both.update([0, 150, 40, 64, 0], sf=[-1, 0, 0, 0, 0], sl=[0, 150, 100, 33, 150])
    both.update([0, 0, 40, 64, 150], sf=[-1, -1, -1, -1, 1], sl=[0, 0, 0, 0, 96])
    both.update([0] * 5)
    assert both.refs == [0] * 12


def test_bad_values_are_clamped_and_reported(hip):
    both = Both(hip, 4, 4, 32, 16)
    both.update([-5, 1000, 40, 10], sf=[0, 9, 1, -1], sl=[32, 32, -4, 7], ctx=[0, 100, -3, 0], n=[1, 9, 2, -1], kmax=2)
    both.tables[1][0], both.tables[2][0] = 99, -4  # entries that are no page
    both.dev.tables.copy_(__import__("torch").tensor(both.tables, dtype=both.dev.tables.dtype))
    both.update([40, 0, 0, 10], sf=[1, -1, -1, -1], sl=[64, 0, 0, 0], ctx=[0, 0, 0, 0], n=[2, 0, 0, 2], kmax=2)


def test_replayed_graph(hip):
    """A captured call, replayed on changing lengths with eager work between, as the oracle has it every time."""
    import torch
    import paper_2404_15778_amd as bass
    rows, most, P, pages, kmax = 9, 12, 32, 80, 5
    both = Both(hip, rows, most, P, pages)
    d = both.dev
    length, ctx, n = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(3))
    slots = torch.zeros((rows, kmax), dtype=torch.int32, device="cuda")
    call = lambda: bass.bass_page_tables(length, d.held, d.tables, d.refs, P, d.ws, None, None, ctx, n, slots, d.status)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    rng = random.Random(5)
    held, tables, refs = both.held, both.tables, both.refs
    for _ in range(5):
        c = [rng.randint(0, most * P - kmax) for _ in range(rows)]
        k = [rng.randint(0, kmax) for _ in range(rows)]
        want = [a + b for a, b in zip(c, k)]
        for t, v in ((length, want), (ctx, c), (n, k)):
            t.copy_(torch.tensor(v, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        held, tables, refs, s, _ = page_tables(want, held, tables, refs, P, None, None, c, k, kmax)
        assert d.held.tolist() == held and d.tables.tolist() == tables and d.refs.tolist() == refs and slots.tolist() == s
