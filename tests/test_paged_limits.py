"""Limits of the paged operators, without a GPU: both sides of each, and what a caller is told beyond them."""
import ctypes
import os

import pytest

import paper_2404_15778_amd as bass

ONE = ctypes.c_void_p(16)  # never dereferenced: every call here is refused


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(bass.LIB_PATH):
        from paper_2404_15778_amd import build
        build.build()


def desc(**kw):
    return bass.make_paged_desc(4, 3, 8, 2, 128, 64, 50, 10, "bf16", 0.1).replace(**kw)


@pytest.mark.parametrize("kw,attention_only", [(dict(D=96), False), (dict(n_pages=0), False), (dict(page_tokens=48), False), (dict(kmax=17), True),
                                               (dict(B=4097), True)])
def test_buffers_of_refused_shapes_are_refused(kw, attention_only):
    """An empty buffer would only say so at the first call, if at all."""
    d = desc(**kw)
    if attention_only:
        assert bass.alloc_page_pool(d, "cpu").numel() == bass.bass_page_pool_bytes(d)
    else:
        with pytest.raises(ValueError, match="alloc_page_pool"):
            bass.alloc_page_pool(d, "cpu")
    with pytest.raises(ValueError, match="alloc_paged_plan"):
        bass.alloc_paged_plan(d, "cpu")
    with pytest.raises(ValueError, match="alloc_paged_workspace"):
        bass.alloc_paged_workspace(d, "cpu")


def test_buffers_of_good_shapes():
    d = desc()
    assert bass.alloc_page_pool(d, "cpu", 7).tolist() == [7] * bass.bass_page_pool_bytes(d)
    assert bass.alloc_paged_plan(d, "cpu").numel() == bass.bass_paged_attention_plan_bytes(d)
    assert bass.alloc_paged_workspace(d, "cpu").numel() == bass.bass_paged_attention_workspace_bytes(d)
    assert bass.alloc_page_tables_workspace(4, 50, "cpu").numel() == bass.bass_page_tables_workspace_bytes(4, 50)
    with pytest.raises(ValueError, match="alloc_page_tables_workspace"):
        bass.alloc_page_tables_workspace(0, 50, "cpu")
