"""Cache attention where a CTA's share holds segments of one tile (GPU): empty sequences in the batch,
calls without the rows' own K and V, blocks of rows of both sizes side by side.  Such a segment has no tile
for the second epilogue group, and the products of the segment after it need that segment's own Q.
Tolerances are those of the attention tests, whose checks these calls go through."""
import numpy as np
import pytest
import torch

import cache_ref as R
from test_gpu_cache_attention import BF, _check, _rows

pytestmark = pytest.mark.gpu


def _try(estp, lens, counts, Hq, Hkv, d, own, row_weight=False):
    rng = np.random.default_rng(sum(lens) + sum(counts) + d)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, lens, Hkv, d, 16, BF)
    n = sum(counts)
    Q = _rows(rng, n, Hq, d, BF)
    kn, vn = (_rows(rng, n, Hkv, d, BF), _rows(rng, n, Hkv, d, BF)) if own else (None, None)
    sees = [R.tree(rng, c) for c in counts]
    c = torch.from_numpy(rng.uniform(0, 1, n).astype(np.float32)).cuda() if row_weight else None
    out = _check(estp, ctx, cache, Q, kn, vn, counts, sees, use_tree=own, row_weight=c)
    # the same bits again: nothing depends on who comes first
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    for _ in range(3):
        again = ctx.cache_attention(cache, Q, kn, vn, cu, max(counts), tree_mask=R.bits_of(sees, -(-max(counts) // 64)) if own else None,
                                    row_weight=c, accumulate=True, details=True)
        ctx.sync_status()
        assert all(x is None and y is None or torch.equal(x, y) for x, y in zip(out, again))
    ctx.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("own", [False, True], ids=["cache_alone", "own_rows"])
def test_shares_that_begin_at_a_last_tile(cuda_lib, d, own):
    _try(cuda_lib, [1000] * 32, [20] * 32, 32, 8, d, own)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("own", [False, True], ids=["cache_alone", "own_rows"])
@pytest.mark.parametrize("n", [1, 5, 20, 40])
def test_empty_sequences_between_others(cuda_lib, d, own, n):
    """4, 20, 80 and 160 rows a KV head: each of the block sizes of a bf16 cache's kernels."""
    _try(cuda_lib, [0 if b % 4 == 1 else 300 for b in range(64)], [n] * 64, 32, 8, d, own)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("own", [False, True], ids=["cache_alone", "own_rows"])
def test_blocks_of_both_sizes(cuda_lib, d, own):
    """Sequences of more than 128 rows a KV head, whose blocks go to both groups, beside smaller ones."""
    lens = [(0, 700, 130, 1, 1025, 0, 260)[b % 7] for b in range(42)]
    counts = [(20, 40, 3, 33, 17, 50, 32, 64, 8)[b % 9] for b in range(42)]
    _try(cuda_lib, lens, counts, 32, 8, d, own, row_weight=True)
