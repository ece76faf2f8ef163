"""A cache whose pool or page table is empty (GPU).  A table that is not there is refused by the host; a
length that claims slots of a pool without pages is recorded on the device, as a page that is none."""
import numpy as np
import pytest
import torch

import cache_ref as R
from test_gpu_cache_attention import BF, F32, _rows

pytestmark = pytest.mark.gpu


def _cache(estp, dtype, n_pages, per, table=True):
    i32 = dict(dtype=torch.int32, device="cuda")
    k = torch.zeros(n_pages, 16, 2, 64, dtype=dtype, device="cuda")
    w = torch.zeros(n_pages, 2, 16, device="cuda")
    cache = estp.KVCache(k, k.clone(), torch.zeros(2, per, **i32), torch.zeros(2, **i32), torch.zeros(2, **i32), w, w.int())
    cache._struct()
    # an empty array has no address of its own: any aligned one stands for it
    if n_pages == 0:
        cache._c.k = cache._c.v = cache._c.weight = cache._c.position = cache.length.new_zeros(64).data_ptr()
    if not table:
        cache._c.page_table = None
    return cache


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_pages", [0, 4])
def test_a_page_table_that_is_not_there(cuda_lib, dtype, n_pages):
    estp = cuda_lib
    rng = np.random.default_rng(0)
    ctx = estp.Context(0)
    cache = _cache(estp, dtype, n_pages, 3, table=False)
    Q, kn = _rows(rng, 2, 4, 64, dtype), _rows(rng, 2, 2, 64, dtype)
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    for call in (lambda: ctx.cache_attention(cache, Q, kn, kn, cu, 1), lambda: ctx.cache_append(cache, kn, kn, cu),
                 lambda: ctx.cache_evict(cache, 4)):
        with pytest.raises(estp.EstpError) as e:
            call()
        assert e.value.status == estp.ESTP_ERR_INVALID_ARG and "page_table" in str(e.value)
    ctx.sync_status()
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_pages,per", [(0, 3), (4, 0), (0, 0)])
@pytest.mark.parametrize("n", [1, 20])
def test_no_slots_at_all(cuda_lib, dtype, n_pages, per, n):
    """Rows that have only themselves, against the definition."""
    estp = cuda_lib
    rng = np.random.default_rng(n)
    ctx = estp.Context(0)
    cache = _cache(estp, dtype, n_pages, per)
    Q, kn, vn = (_rows(rng, 2 * n, h, 64, dtype) for h in (4, 2, 2))
    cu = np.array([0, n, 2 * n], np.int32)
    sees = [np.tril(np.ones((n, n), bool))] * 2
    want, lse, wn, _ = R.attention(cache, Q, kn, vn, cu, 0.125, sees)
    out, l, w = ctx.cache_attention(cache, Q, kn, vn, torch.from_numpy(cu).cuda(), n, accumulate=n_pages > 0, details=True)
    ctx.cache_evict(cache, 4) if n_pages else None
    ctx.sync_status()
    # bf16: half an ulp of the result; scores, probabilities and sums in fp32 (see the attention tests)
    assert np.all(np.abs(R.host(out) - want) <= 2e-4 * float(vn.abs().max()) + (2.0 ** -8 * np.abs(want) if dtype == BF else 0))
    assert np.all(np.abs(R.host(l) - lse) <= 2e-5 + 2e-6 * np.abs(lse))
    assert np.all(np.abs(R.host(w) - wn) <= 2e-4 * wn + 1e-9)
    assert cache.length.tolist() == [0, 0]
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_slots_of_a_pool_without_pages(cuda_lib, dtype):
    estp = cuda_lib
    rng = np.random.default_rng(1)
    ctx = estp.Context(0)
    cache = _cache(estp, dtype, 0, 3)
    cache.max_slots = 48
    cache.length.fill_(20)
    Q, kn = _rows(rng, 2, 4, 64, dtype), _rows(rng, 2, 2, 64, dtype)
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    for call in (lambda: ctx.cache_attention(cache, Q, kn, kn, cu, 1), lambda: ctx.cache_append(cache, kn, kn, cu),
                 lambda: ctx.cache_evict(cache, 4)):
        call()
        with pytest.raises(estp.EstpError) as e:
            ctx.sync_status()
        assert e.value.status == estp.ESTP_ERR_INVALID_ARG
    ctx.close()
