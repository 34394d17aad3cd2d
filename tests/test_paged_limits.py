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


# sequences, heads, kv heads, tokens of a page, entries of a table; the list has B Hkv (8 blocks + 256) entries at most
@pytest.mark.parametrize("B,Hq,Hkv,P,most", [(1000, 32, 32, 32, 2048), (4096, 8, 8, 32, 8159), (1, 4, 4, 64, 33554399), (1, 1, 1, 32, 67108863), (64, 64, 8, 256, 65520)])
def test_the_list_of_the_attention(B, Hq, Hkv, P, most):
    """As documented: shapes up to the limit have sizes, and the first beyond it is refused with a size of 0."""
    d = desc(B=B, kmax=1, Hq=Hq, Hkv=Hkv, page_tokens=P, n_pages=100)
    entries = lambda n: B * Hkv * (8 * n * (P // 32) + 256)  # noqa: E731
    largest = min((2 ** 31 - 1) // P, max(n for n in (((2 ** 31 - 1) // (B * Hkv) - 256) // (8 * (P // 32)) + i for i in (-1, 0, 1)) if entries(n) < 2 ** 31))
    assert most <= largest
    for n in (most, largest):
        assert bass.bass_paged_attention_plan_bytes(d.replace(max_pages=n)) > 0 and bass.bass_paged_attention_workspace_bytes(d.replace(max_pages=n)) > 0
    beyond = d.replace(max_pages=largest + 1)
    assert bass.bass_paged_attention_plan_bytes(beyond) == 0 == bass.bass_paged_attention_workspace_bytes(beyond)
    assert bass.lib().bass_paged_attention_plan(ctypes.byref(beyond), ONE, ONE, None, None, 0, ONE, 1 << 40, None, None) == bass.ERR_UNSUPPORTED


def test_products_beyond_64_bits():
    """Sizes whose products overflow are refused like any others beyond the limits."""
    for hkv in (1 << 20, 1 << 30):
        d = desc(B=4096, kmax=64, Hq=hkv, Hkv=hkv, page_tokens=32, n_pages=1, max_pages=(1 << 26) - 1)
        assert bass.bass_paged_attention_plan_bytes(d) == 0 == bass.bass_paged_attention_workspace_bytes(d)


def test_launches_of_more_threads_than_are_counted():
    """A launch counts its threads in 32 bits; what would need more is refused before anything is enqueued.  Just below, everything else has to be in order."""
    L, U = bass.lib(), bass.ERR_UNSUPPORTED

    def rows(append, **kw):
        d = desc(**kw)
        if append:
            return L.bass_paged_append(ctypes.byref(d), ONE, ONE, ONE, ONE, ONE, None, None)
        return L.bass_paged_gather(ctypes.byref(d), ONE, ONE, ONE, ONE, ONE, ONE, ONE, None, None)

    for append in (True, False):
        assert rows(append, B=1 << 19, kmax=2, Hq=16, Hkv=16) == U         # 2 windows of 32 tokens
        assert rows(append, B=1 << 20, kmax=1, Hq=16, Hkv=16) == U
        assert rows(append, B=16, kmax=(1 << 20) + 1, Hq=32, Hkv=32) == U

        # numbers of workgroups beyond 64 bits, which come out as 0 or a few there
        for kw in (dict(B=1 << 30, kmax=(1 << 31) - 31, Hq=1 << 30, Hkv=1 << 30), dict(B=(1 << 31) - 1, kmax=(1 << 31) - 1, Hq=1 << 26, Hkv=1 << 26)):
            assert rows(append, page_tokens=32, n_pages=1, **kw) == U

    def tables(rows, max_pages, kmax):
        slots = ONE if kmax else None
        return L.bass_page_tables(rows, max_pages, 32, 50, ONE, None, None, ONE, ONE, ONE, kmax, slots, slots, slots, ONE, 1 << 40, None, None)

    assert tables(1 << 26, 1, 0) == U
    assert tables(65538, 1, 65535) == U
    d = desc(B=4096, kmax=64, Hq=1024, Hkv=1024, D=128, page_tokens=32, n_pages=100, max_pages=1)
    assert bass.bass_paged_attention_plan_bytes(d) == 0 == bass.bass_paged_attention_workspace_bytes(d)
    assert L.bass_paged_verify_attention(ctypes.byref(d), *[ONE] * 6, None, ONE, 1 << 60, None, None) == U
    assert bass.bass_paged_attention_plan_bytes(d.replace(B=4095, Hq=512, Hkv=512)) > 0
