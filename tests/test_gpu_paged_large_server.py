"""Attention over the tables of a large server: 1000 sequences of up to 65 536 tokens, 32 kv heads."""
import numpy as np
import pytest

import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
def test_a_thousand_sequences_of_up_to_65536_tokens(dtype):
    """Keys are zero, so every token counts alike: lse is the logarithm of their number; a page's values are one whole number, so O is their mean (rounded to bf16,
    2^-8; over INT8 pages the probabilities times the scale are too)."""
    from paper_2404_15778_amd import harness as hip
    rng = np.random.default_rng(3)
    B, H, D, P, most, pages = 1000, 32, 64, 32, 2048, 60
    pg = hip.DevicePages(B, 1, H, H, D, P, pages, most, dtype, 0.125)
    value = rng.integers(-8, 9, size=pages)
    V = np.repeat(value, P).astype(np.float32)[None, :, None, None] * np.ones((1, 1, H, D), np.float32)
    pg.append(hip.to_device(np.zeros(V.shape, np.uint16)), hip.to_device(wl.to_bf16_bits(V)), hip.i32(np.arange(pages * P)[None]))
    tables = rng.integers(0, pages, size=(B, most))
    tables[::2, :100] = tables[0, :100]  # half of them begin with the same 3200 tokens
    ctx = 3200 + rng.integers(0, 300, size=B)
    ctx[7], ctx[500] = most * P - 1, 60001
    nq = (rng.random(B) < 0.9).astype(int)
    nq[7] = nq[500] = 1
    Q = wl.to_bf16_bits(rng.standard_normal((B, 1, H, D), dtype=np.float32))
    O, lse = pg.verify(hip.to_device(Q), hip.i32(tables), hip.i32(ctx), hip.i32(nq), hip.i32(np.where(np.arange(B) % 2, -1, 0)), hip.i32([3200]))
    O, lse = wl.bf16_bits_to_f32(hip.to_host(O)), hip.to_host(lse)
    assert int(pg.status.item()) == 0 and int(pg.plan[:8].cpu().numpy().view(np.int32)[1]) == nq.sum() + 1
    for b in range(B):
        if nq[b] == 0:
            assert (O[b] == 0).all() and (lse[b] == 0).all()
            continue
        v = np.repeat(value[tables[b]], P)[:ctx[b] + 1].astype(np.float64)
        assert np.abs(lse[b] - np.log(len(v))).max() <= 2e-6
        assert np.abs(O[b] - v.mean()).max() <= 2 ** -8 * abs(v.mean()) + (2 ** -8 * np.abs(v).mean() if dtype == "int8kv" else 1e-5)
