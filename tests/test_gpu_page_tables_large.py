"""bass_page_tables with a table that ends less than a page before 2^31 tokens: pages whose size is no power of two."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_full_table_of_2_to_the_31_tokens():
    import torch
    from paper_2404_15778_amd import harness as hip
    P = 96
    pages = (2 ** 31 - 1) // P
    dt = hip.DeviceTables(2, pages, P, pages)
    top = pages * P
    slots = dt.update([top, 0], ctx_len=[top - 3, 0], n_new=[5, 0], kmax=5)
    assert dt.held.tolist() == [pages, 0] and int(dt.status.item()) == 0
    numbers = torch.arange(pages, dtype=torch.int32, device="cuda")
    assert torch.equal(dt.tables[0], numbers) and bool((dt.tables[1] == -1).all()) and bool((dt.refs == 1).all())
    assert slots.tolist() == [[top - 3, top - 2, top - 1, -1, -1], [-1] * 5]
    dt.update([2 ** 31 - 1, 0])  # more than the table has: clamped to what it holds
    assert dt.held.tolist() == [pages, 0] and int(dt.status.item()) == 1
    dt.update([0, top], [-1, 0], [0, top])  # handed over whole in one call
    assert dt.held.tolist() == [0, pages] and torch.equal(dt.tables[1], numbers) and bool((dt.tables[0] == -1).all()) and bool((dt.refs == 1).all())
    dt.update([0, 0])
    assert dt.held.tolist() == [0, 0] and not dt.refs.any() and bool((dt.tables == -1).all())
