"""Eviction of a sequence whose length does not fit its table (GPU): recorded, and nothing of the sequence
changes, its length included; the others are cut as ever."""
import numpy as np
import pytest
import torch

import cache_ref as R
from test_gpu_cache_store import BF

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [-1, -(2 ** 31), 10 ** 7, 2 ** 31 - 1, "table"])
def test_a_length_that_does_not_fit_stays(cuda_lib, bad):
    estp = cuda_lib
    rng = np.random.default_rng(7)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, [50, 40, 64], 2, 64, 16, BF)
    if bad == "table":  # one slot past it
        bad = cache.page_table.shape[1] * 16 + 1
    cache.length[1] = 0
    k, v, w, pos, length = R.evict(cache, 30, 4, 2)  # the other two
    cache.length[1] = bad
    ctx.cache_evict(cache, 30, recent=4, sinks=2)
    with pytest.raises(estp.EstpError) as e:
        ctx.sync_status()
    assert e.value.status == estp.ESTP_ERR_INVALID_ARG
    assert cache.length.tolist() == [30, bad, 30] and length.tolist() == [30, 0, 30]
    for t, a in zip((cache.k, cache.v, cache.weight, cache.position), (k, v, w, pos)):
        assert np.array_equal(R.host(t), a, equal_nan=True) if t.is_floating_point() else np.array_equal(R.host(t), a)
    # into another array of lengths too
    length_out = torch.full((3,), -9, dtype=torch.int32, device="cuda")
    cache.length[0] = 50
    ctx._lib.estp_cache_evict(ctx._h, cache._struct(), cache.length.data_ptr(), cache.seen.data_ptr(), length_out.data_ptr(), 3, 60, 0, 0, None)
    with pytest.raises(estp.EstpError):
        ctx.sync_status()
    assert length_out.tolist() == [50, bad, 30]
    ctx.close()
