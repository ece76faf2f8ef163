"""The cache's kernels in the bounds-checked build (GPU): on valid inputs no check fires, and every output
equals the release build's bit for bit."""
import numpy as np
import pytest
import torch

import cache_ref as R
from test_gpu_cache_attention import BF, F32, _rows

pytestmark = pytest.mark.gpu


def _run(estp, library, dtype, d, n):
    rng = np.random.default_rng(n + d)
    ctx = estp.Context(0, library=library)
    lens, counts = [900, 0, 64, 333, 2100], [n, n, 1, 0, max(n // 2, 1)]
    cache = R.make_cache(estp, rng, lens, 2, d, 16, dtype, spare=2 * n + 2)
    m = sum(counts)
    Q, kn, vn = (_rows(rng, m, h, d, dtype) for h in (14, 2, 2))
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    tree = R.bits_of([R.tree(rng, c) for c in counts], 1)
    res = []
    for own in (True, False):  # with the rows' own keys, and the cache alone
        out = ctx.cache_attention(cache, Q, *((kn, vn) if own else (None, None)), cu, n, tree_mask=tree if own else None,
                                  accumulate=True, details=True)
        ctx.sync_status()
        res += [x for x in out if x is not None] + [cache.weight.clone()]
    ctx.cache_append(cache, kn, vn, cu, weight=res[2])
    ctx.sync_status()
    ctx.cache_append(cache, kn, vn, cu, rows=torch.arange(m, dtype=torch.int32, device="cuda").flip(0))
    ctx.sync_status()
    ctx.cache_evict(cache, 300, recent=20, sinks=4)
    ctx.sync_status()
    ctx.close()
    return [x.nan_to_num() for x in (*res, cache.k, cache.v, cache.weight, cache.position, cache.length, cache.seen)]


# 7 query heads a KV head: 7, 14, 28, 63 and 210 rows, every form of the forward and of the weights
@pytest.mark.parametrize("n", [1, 2, 4, 9, 30])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_checked_build_matches_release_bitwise(cuda_lib, dtype, d, n):
    estp = cuda_lib
    ref = _run(estp, estp.lib, dtype, d, n)
    got = _run(estp, estp.load_library(estp.CHECKS_LIB_PATH), dtype, d, n)
    assert len(ref) == len(got) == 13 and all(torch.equal(a, b) for a, b in zip(ref, got))
