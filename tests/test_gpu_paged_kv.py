"""Rows into pages by slot and back through tables: every byte, INT8 codes and scales by the quantizer oracle."""
import numpy as np
import pytest

import workloads as wl
from oracle.kv_int8 import quantize_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hip():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2404_15778_amd import harness
    return harness


def block_offsets(D, int8):
    """Element offsets of [token][d] in a K and a V block, from the header's description."""
    t, d = np.arange(32)[:, None], np.arange(D)[None, :]
    if int8:
        k = ((((t // 16) * (D // 64) + d // 64) * 4 + d // 16 % 4) * 16 + t % 16) * 16 + d % 16
        v = ((((d // 32) * 4 + t // 4 % 4) * 16 + d % 16) * 2 + d // 16 % 2) * 8 + t // 16 * 4 + t % 4
    else:
        k = ((((t // 16) * (D // 32) + d // 32) * 4 + d // 8 % 4) * 16 + t % 16) * 8 + d % 8
        v = ((((d // 16) * 4 + t // 4 % 4) * 16 + d % 16) * 2 + t // 16) * 4 + t % 4
    return k, v


def expected_pools(rowsK, rowsV, slots, H, D, P, n_pages, int8):
    """Pools filled with 0xFF and then with the rows, as bytes."""
    nb = 32 * (D + 4) if int8 else 32 * D * 2
    pools = [np.full((n_pages, H, P // 32, nb), 0xFF, np.uint8) for _ in range(2)]
    for rows, pool, place in zip((rowsK, rowsV), pools, block_offsets(D, int8)):
        codes, scales = quantize_rows(wl.bf16_bits_to_f32(rows)) if int8 else (rows, None)
        for b, i in zip(*np.nonzero((slots >= 0) & (slots < n_pages * P))):
            page, t = divmod(int(slots[b, i]), P)
            block = pool[page, :, t // 32]
            if int8:
                block[:, place[t % 32]] = codes[b, i].view(np.uint8)
                block[:, 32 * D:].view(np.float32)[:, t % 32] = scales[b, i]
            else:
                block.view(np.uint16)[:, place[t % 32]] = rows[b, i]
    return pools


# B, kmax, Hkv, D, page tokens, pages, how the slots lie
CASES = [(1, 1, 1, 64, 32, 1, "run"), (3, 6, 2, 128, 64, 9, "run"), (2, 33, 3, 64, 96, 7, "run"), (4, 130, 2, 128, 32, 40, "run"),
         (2, 64, 1, 128, 64, 6, "aligned"), (2, 50, 2, 64, 32, 20, "scattered"), (3, 70, 2, 128, 64, 20, "scattered"), (2, 40, 1, 128, 256, 5, "holes")]


def make_slots(rng, B, kmax, P, n_pages, how):
    """run: consecutive tokens of random pages from an odd place on; holes: the same with rows left out; scattered: any places."""
    if how == "scattered":
        return rng.permutation(n_pages * P)[: B * kmax].reshape(B, kmax).astype(np.int32)
    per = n_pages // B
    pages = rng.permutation(n_pages)
    out = np.empty((B, kmax), np.int32)
    for b in range(B):
        first = 0 if how == "aligned" else int(rng.integers(0, max(1, min(P * per - kmax, 61))))
        t = first + np.arange(kmax)
        out[b] = np.where(t < per * P, pages[b * per + np.minimum(t // P, per - 1)] * P + t % P, -1)
    if how == "holes":
        out[rng.random((B, kmax)) < 0.3] = -1
        out[0, 0] = -1
        out[-1, -2:] = n_pages * P + 5  # beyond the pool
    return out


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("B,kmax,H,D,P,n_pages,how", CASES)
def test_append_writes_the_rows_and_nothing_else(hip, dtype, B, kmax, H, D, P, n_pages, how):
    rng = np.random.default_rng([B, kmax, D, P])
    K, V = (wl.to_bf16_bits(rng.standard_normal((B, kmax, H, D), dtype=np.float32) * rng.choice([1e-3, 1.0, 50.0], size=(B, kmax, H, 1)).astype(np.float32))
            for _ in range(2))
    K[0, 0, 0] = 0  # a row of zeros has scale 0
    slots = make_slots(rng, B, kmax, P, n_pages, how)
    pages = hip.DevicePages(B, kmax, H, H, D, P, n_pages, n_pages, dtype, 1.0, poison=True) if kmax <= 64 else \
        hip.DevicePages(B, 1, H, H, D, P, n_pages, n_pages, dtype, 1.0, poison=True)
    pages.append(hip.to_device(K), hip.to_device(V), hip.i32(slots))
    want = expected_pools(K, V, slots, H, D, P, n_pages, dtype == "int8kv")
    assert np.array_equal(pages.K.cpu().numpy(), want[0].reshape(-1))
    assert np.array_equal(pages.V.cpu().numpy(), want[1].reshape(-1))
    assert int(pages.status.item()) == (16 if (slots >= n_pages * P).any() else 0)


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("H,D,P", [(1, 64, 32), (3, 128, 96), (2, 128, 64)])
def test_gather_reads_what_append_wrote(hip, dtype, H, D, P):
    import torch
    rng = np.random.default_rng([H, D, P])
    B, T, most = 4, 210, -(-210 // P) + 1
    n_pages = B * most
    tables = rng.permutation(n_pages).reshape(B, most).astype(np.int32)
    K, V = (wl.to_bf16_bits(rng.standard_normal((B, T, H, D), dtype=np.float32)) for _ in range(2))
    t = np.arange(T)
    slots = np.ascontiguousarray(tables[:, t // P] * P + t % P)
    pages = hip.DevicePages(B, 1, H, H, D, P, n_pages, most, dtype, 1.0, poison=True)
    pages.append(hip.to_device(K), hip.to_device(V), hip.i32(slots))
    start, count, n = [0, 37, 205, 96], [70, 1, 5, 0], 70
    out = [x.cpu() for x in pages.gather(hip.i32(tables), hip.i32(start), hip.i32(count), n)]
    if dtype == "int8kv":
        (Kc, Ks), (Vc, Vs) = (quantize_rows(wl.bf16_bits_to_f32(x)) for x in (K, V))
        want = (Kc, Vc, Ks, Vs)
    else:
        out = [x.view(torch.int16) for x in out]
        want = (K.view(np.int16), V.view(np.int16))
    for got, all_rows in zip(out, want):
        expect = np.zeros((B, n) + all_rows.shape[2:], all_rows.dtype)
        for b in range(B):
            expect[b, :count[b]] = all_rows[b, start[b]:start[b] + count[b]]
        assert np.array_equal(got.numpy(), expect)
    assert int(pages.status.item()) == 0


def test_gather_of_what_is_not_there(hip):
    """Counts and tokens beyond the table, entries that are no page: left untouched and reported."""
    rng = np.random.default_rng(1)
    tables = np.array([[2, 0], [1, -1], [3, 77]], np.int32)
    pages = hip.DevicePages(3, 1, 2, 2, 64, 32, 4, 2, "bf16", 1.0)
    K, V = (wl.to_bf16_bits(rng.standard_normal((1, 128, 2, 64), dtype=np.float32)) for _ in range(2))
    pages.append(hip.to_device(K), hip.to_device(V), hip.i32(np.arange(128)[None]))
    Ko, Vo = (hip.to_host(x) for x in pages.gather(hip.i32(tables), hip.i32([60, 0, 30]), hip.i32([20, 40, 9]), 16))
    assert int(pages.status.item()) == 1 | 16
    for got, rows in ((Ko, K[0]), (Vo, V[0])):
        want = np.zeros((3, 16, 2, 64), np.uint16)
        want[0, :4] = rows[28:32]       # tokens 60 .. 63 of the table's 64, in page 0
        want[1, :16] = rows[32:48]      # 40 asked for, 16 places
        want[2, :2] = rows[126:128]     # tokens 30, 31 in page 3, the rest in no page
        assert np.array_equal(got, want)


def test_places_beyond_four_gigabytes(hip):
    """Pools of more than 2^32 bytes: the first and the last page."""
    import torch
    H, D, P, n_pages = 8, 128, 256, 8200
    pages = hip.DevicePages(1, 2, H, H, D, P, n_pages, 2, "bf16", 1.0)
    assert pages.K.numel() > 1 << 32
    K, V = (torch.randn((1, 2, H, D), device="cuda").to(torch.bfloat16) for _ in range(2))
    pages.append(K, V, hip.i32([[n_pages * P - 1, 0]]))
    tables = hip.i32([[n_pages - 1, 0]])
    Ko, Vo = pages.gather(tables, hip.i32([P - 1]), hip.i32([2]), 2)
    assert torch.equal(Ko, K) and torch.equal(Vo, V) and int(pages.status.item()) == 0
