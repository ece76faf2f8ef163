"""Cache attention whose waits run out with accumulation on (GPU, no fault and no hang): the weights, which
no later call could form again, stay as they were until the status has been read."""
import numpy as np
import pytest
import torch

import cache_ref as R
from test_gpu_cache_attention import BF, F32, _check, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 7, 9, 60])
def test_weights_outlive_a_wait_that_runs_out(cuda_lib, n):
    """4 and 28 rows a KV head: kept scores, added by the finish launch; 36 and 240: by the weight kernel."""
    estp = cuda_lib
    rng = np.random.default_rng(n)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, [700, 90, 0, 2000], 2, 128, 16, BF)
    Q, kn, vn = _rows(rng, 4 * n, 8, 128, BF), _rows(rng, 4 * n, 2, 128, BF), _rows(rng, 4 * n, 2, 128, BF)
    cu = torch.arange(0, 4 * n + 1, n, dtype=torch.int32, device="cuda")
    # what the workspace holds before: a step's partials and scores of other rows
    ctx.cache_attention(cache, Q.flip(0), kn, vn, cu, n, accumulate=True)
    ctx.sync_status()
    w0 = cache.weight.clone()
    ctx.set_wait_limit(2)
    ctx.cache_attention(cache, Q, kn, vn, cu, n, accumulate=True, details=True)
    ctx.set_wait_limit(0)
    torch.cuda.synchronize()
    assert torch.equal(cache.weight.nan_to_num(), w0.nan_to_num())
    # nor is anything added by later calls, of either type, before the error is known
    ctx.cache_attention(cache, Q, kn, vn, cu, n, accumulate=True)
    other = R.make_cache(estp, rng, [40, 300, 5, 1], 2, 128, 16, F32)
    u0 = other.weight.clone()
    ctx.cache_attention(other, Q.float(), kn.float(), vn.float(), cu, n, accumulate=True)
    with pytest.raises(estp.EstpError) as e:
        ctx.sync_status()
    assert e.value.status == estp.ESTP_ERR_TIMEOUT
    assert torch.equal(cache.weight.nan_to_num(), w0.nan_to_num()) and torch.equal(other.weight.nan_to_num(), u0.nan_to_num())
    # made again, the step is right
    sees = [R.tree(rng, n) for _ in range(4)]
    _check(estp, ctx, cache, Q, kn, vn, [n] * 4, sees)
    _check(estp, ctx, other, Q.float(), kn.float(), vn.float(), [n] * 4, sees)
    ctx.close()


def test_a_timeout_after_another_error(cuda_lib):
    """The status holds the first error; a wait that runs out behind it leaves the weights alone all the same."""
    estp = cuda_lib
    rng = np.random.default_rng(3)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, [700, 90], 2, 128, 16, BF)
    Q, kn, vn = _rows(rng, 2, 8, 128, BF), _rows(rng, 2, 2, 128, BF), _rows(rng, 2, 2, 128, BF)
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    w0 = cache.weight.clone()
    cache.length[1] = -1
    ctx.cache_attention(cache, Q, kn, vn, cu, 1, accumulate=True)  # refused on the device
    cache.length[1] = 90
    ctx.set_wait_limit(2)
    ctx.cache_attention(cache, Q, kn, vn, cu, 1, accumulate=True)
    ctx.set_wait_limit(0)
    with pytest.raises(estp.EstpError) as e:
        ctx.sync_status()
    assert e.value.status == estp.ESTP_ERR_INVALID_ARG
    assert torch.equal(cache.weight.nan_to_num(), w0.nan_to_num())
    _check(estp, ctx, cache, Q, kn, vn, [1, 1], [np.ones((1, 1), bool)] * 2)
    ctx.close()
