"""ctx_len outside the cache, up to the ends of the 32-bit range: clamped and reported, and the other sequences' results are as if it had not been."""
import numpy as np
import pytest

import oracle
import workloads as wl
from test_gpu_paged_attention import Batch

pytestmark = pytest.mark.gpu
TOP = 2 ** 31 - 1
BAD = [TOP, TOP - 1, TOP - 3, TOP - 4, 10 ** 9, -1, -TOP - 1]


@pytest.fixture(scope="module")
def hip():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2404_15778_amd import harness
    return harness


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("n,prefix", [(5, 96), (16, 2048)])  # apart, and with a shared run of tiles
def test_paged(hip, n, prefix, bad):
    """The clamped sequence reaches entries of its table that are no page: page 0 is read in their place, and that is reported too.  With a negative length
    it has no common blocks with the others, so the prefix of all of them is computed apart."""
    import paper_2404_15778_amd as bass
    rng = np.random.default_rng(n)
    batch = Batch(n, 32, 8, 128, 32, prefix + rng.integers(0, 50, size=n), [4] * n, 4, np.zeros(n, int), [prefix])
    pg = batch.pages(hip, layers_poison=False)
    ctx = batch.ctx.copy()
    ctx[1] = bad
    O, lse = pg.verify(hip.to_device(batch.Q), hip.i32(batch.tables), hip.i32(ctx), hip.i32(batch.nq), hip.i32(batch.of), hip.i32(batch.plen))
    O, lse = wl.bf16_bits_to_f32(hip.to_host(O)), hip.to_host(lse)
    assert batch.shared_runs(pg) == (1 if n == 16 and bad > 0 else 0)
    assert int(pg.status.item()) == bass.STATUS_LEN_CLAMPED | (bass.STATUS_PAGE_CLAMPED if bad > 0 else 0)
    want, want_lse, A = batch.reference()
    assert np.isfinite(O).all() and np.isfinite(lse).all()
    off = (np.abs(O - want) <= (2 ** -8 * (1 + 2 ** -8) + 2 ** -10) * A + 2 ** -8 * np.abs(want) + 1e-30).all(axis=(1, 2, 3))
    off_lse = (np.abs(lse - want_lse) <= 2 ** -11 + 2 ** -20 * np.abs(want_lse)).all(axis=(1, 2))
    assert off[np.arange(n) != 1].all() and off_lse[np.arange(n) != 1].all()


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("Hq,Hkv", [(8, 8), (32, 4)])  # few query rows, and the kernels for many
def test_caches_of_their_own(hip, Hq, Hkv, bad):
    import paper_2404_15778_amd as bass
    n = 5
    w = wl.make_attention("clamp", n, Hq, Hkv, 128, "bf16", [50, 20, 300, 0, 111], [4] * n, 8, kmax=4, Lcap=320)
    _, _, _, da = hip.run_attention_workload(w, poison=False)
    ctx = np.array(w.ctx_len, np.int32)
    ctx[1] = bad
    da.status.zero_()
    O, _ = da.verify(hip.to_device(w.Q), hip.i32(ctx), hip.i32(w.draft_len))
    O = hip.to_host(O)
    want, _ = oracle.verify_attention(w.Q, w.K, w.V, w.ctx_len, w.draft_len, w.scale)
    assert int(da.status.item()) == bass.STATUS_LEN_CLAMPED and np.isfinite(O).all()
    assert np.abs(O - want)[np.arange(n) != 1].max() <= 2e-2
