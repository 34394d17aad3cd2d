"""CPU-only checks of the paged operators: sizes on the host, and refusals before anything is launched."""
import ctypes
import os

import pytest

import paper_2404_15778_amd as bass

ONE = ctypes.c_void_p(16)  # never dereferenced: every call here is refused
ODD = ctypes.c_void_p(8)   # not aligned to 16 bytes
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(bass.LIB_PATH):
        from paper_2404_15778_amd import build
        build.build()


def desc(**kw):
    return bass.make_paged_desc(4, 3, 8, 2, 128, 64, 50, 10, "bf16", 0.1).replace(**kw)


def plan(d, *a, plan=ONE, size=BIG):
    a = a or (ONE, ONE, None, None, 0)
    return bass.lib().bass_paged_attention_plan(ctypes.byref(d), *a, plan, size, None, None)


def attend(d, args=None, ws=ONE, size=BIG):
    args = args or [ONE] * 6
    return bass.lib().bass_paged_verify_attention(ctypes.byref(d), *args, None, ws, size, None, None)


def tables(rows=4, max_pages=10, P=64, pages=50, length=ONE, sf=None, sl=None, held=ONE, tab=ONE, refs=ONE, kmax=0, ctx=None, n=None, slots=None,
           ws=ONE, size=BIG):
    return bass.lib().bass_page_tables(rows, max_pages, P, pages, length, sf, sl, held, tab, refs, kmax, ctx, n, slots, ws, size, None, None)


def test_sizes():
    assert bass.bass_page_pool_bytes(desc()) == 50 * 2 * 64 * 128 * 2
    assert bass.bass_page_pool_bytes(desc(dtype=bass.DTYPE_INT8KV)) == 50 * 2 * 64 * (128 + 4)
    assert bass.bass_paged_attention_plan_bytes(desc()) > 0 and bass.bass_paged_attention_workspace_bytes(desc()) > 0
    assert bass.bass_page_tables_workspace_bytes(4, 50) > 0
    assert bass.bass_page_tables_workspace_bytes(0, 50) == 0 == bass.bass_page_tables_workspace_bytes(4, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), bass.ERR_INVALID_ARG), (dict(kmax=0), bass.ERR_INVALID_ARG), (dict(Hkv=3), bass.ERR_INVALID_ARG), (dict(n_pages=0), bass.ERR_INVALID_ARG),
    (dict(max_pages=-1), bass.ERR_INVALID_ARG), (dict(page_tokens=0), bass.ERR_INVALID_ARG), (dict(page_tokens=48), bass.ERR_UNSUPPORTED),
    (dict(D=96), bass.ERR_UNSUPPORTED), (dict(dtype=bass.DTYPE_FP32), bass.ERR_UNSUPPORTED), (dict(dtype=9), bass.ERR_UNSUPPORTED),
    (dict(n_pages=1 << 25), bass.ERR_UNSUPPORTED), (dict(max_pages=1 << 25), bass.ERR_UNSUPPORTED)])
def test_bad_shapes(kw, code):
    d = desc(**kw)
    assert bass.bass_page_pool_bytes(d) == bass.bass_paged_attention_plan_bytes(d) == bass.bass_paged_attention_workspace_bytes(d) == 0
    assert plan(d) == attend(d) == code
    L = bass.lib()
    assert L.bass_paged_append(ctypes.byref(d), ONE, ONE, ONE, ONE, ONE, None, None) == code
    assert L.bass_paged_gather(ctypes.byref(d), ONE, ONE, ONE, ONE, ONE, ONE, ONE, None, None) == code


def test_limits_of_the_attention():
    assert plan(desc(kmax=17)) == attend(desc(kmax=17)) == bass.ERR_UNSUPPORTED                  # 68 query rows per kv head
    assert plan(desc(B=4097)) == bass.ERR_UNSUPPORTED
    assert plan(desc(B=4096, max_pages=1 << 20, Hkv=8)) == bass.ERR_UNSUPPORTED                  # the work list counts in 32 bits
    assert plan(desc(), ONE, ONE, ONE, ONE, 4097) == bass.ERR_UNSUPPORTED
    assert bass.bass_page_pool_bytes(desc(kmax=17)) > 0                                          # writing long prompts is fine


def test_missing_pointers_alignment_and_small_buffers():
    d = desc()
    for i in range(6):
        args = [ONE] * 6
        args[i] = None
        assert attend(d, args) == bass.ERR_INVALID_ARG
        if i != 3:  # tables are words
            args[i] = ODD
            assert attend(d, args) == bass.ERR_INVALID_ARG
    assert attend(d, ws=None) == attend(d, ws=ODD) == bass.ERR_INVALID_ARG
    assert attend(d, size=bass.bass_paged_attention_workspace_bytes(d) - 1) == bass.ERR_WORKSPACE_TOO_SMALL
    assert plan(d, size=bass.bass_paged_attention_plan_bytes(d) - 1) == bass.ERR_WORKSPACE_TOO_SMALL
    assert plan(d, plan=ODD) == plan(d, plan=None) == plan(d, None, ONE, None, None, 0) == bass.ERR_INVALID_ARG
    # a prefix number without lengths, lengths without numbers, a negative count
    assert plan(d, ONE, ONE, ONE, None, 1) == plan(d, ONE, ONE, None, ONE, 1) == plan(d, ONE, ONE, ONE, ONE, 0) == bass.ERR_INVALID_ARG
    assert plan(d, ONE, ONE, ONE, ONE, -1) == bass.ERR_INVALID_ARG
    L = bass.lib()
    assert L.bass_paged_append(ctypes.byref(d), ONE, ONE, ONE, ONE, None, None, None) == bass.ERR_INVALID_ARG
    assert L.bass_paged_append(ctypes.byref(d), ONE, ONE, ODD, ONE, ONE, None, None) == bass.ERR_INVALID_ARG
    assert L.bass_paged_gather(ctypes.byref(d), ONE, ONE, ONE, ONE, ONE, None, ONE, None, None) == bass.ERR_INVALID_ARG
    i8 = desc(dtype=bass.DTYPE_INT8KV)
    assert L.bass_paged_gather(ctypes.byref(i8), *[ONE] * 7, None, None) == bass.ERR_UNSUPPORTED
    assert L.bass_paged_gather_int8(ctypes.byref(d), *[ONE] * 9, None, None) == bass.ERR_UNSUPPORTED
    assert L.bass_paged_gather_int8(ctypes.byref(i8), ONE, ONE, ONE, ONE, None, ONE, ONE, ONE, ONE, None, None) == bass.ERR_INVALID_ARG


def test_page_tables_refusals():
    I, U = bass.ERR_INVALID_ARG, bass.ERR_UNSUPPORTED
    for kw in (dict(rows=0), dict(max_pages=0), dict(P=0), dict(pages=0), dict(kmax=-1), dict(length=None), dict(held=None), dict(tab=None),
               dict(refs=None), dict(ws=None), dict(ws=ODD), dict(sf=ONE), dict(sl=ONE), dict(slots=ONE, kmax=4), dict(slots=ONE, ctx=ONE, n=ONE)):
        assert tables(**kw) == I, kw
    for kw in (dict(P=33), dict(kmax=65536), dict(rows=1 << 20, max_pages=1 << 12), dict(pages=1 << 26), dict(max_pages=1 << 26)):
        assert tables(**kw) == U, kw
    assert tables(size=bass.bass_page_tables_workspace_bytes(4, 50) - 1) == bass.ERR_WORKSPACE_TOO_SMALL


def test_the_binding_refuses_tensors_on_the_host():
    torch = pytest.importorskip("torch")
    d = desc()
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        bass.bass_paged_attention_plan(d, t, t, None, None, torch.zeros(1 << 16, dtype=torch.uint8))
    with pytest.raises(ValueError):
        bass.bass_paged_attention_plan(d, t, t, t, None, None)
    with pytest.raises(ValueError):
        bass.bass_page_tables(t, t, None, t, 64, t)
    with pytest.raises(ValueError):
        bass.bass_paged_append(d, t, t, t, t, t)
