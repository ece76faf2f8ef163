"""What a context was asked before changes no later result (GPU)."""
import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _call(ctx, rows, V, K, tail, dtype):
    g = torch.Generator().manual_seed(V)
    x = R.padded((torch.randn(rows, V, generator=g) * 3).to(dtype), fill=0.0)
    ids = torch.randint(0, V // K, (rows, K), generator=g).int() * K + torch.arange(K, dtype=torch.int32)
    tl = torch.log_softmax(torch.randn(rows, K, generator=g), 1) - 0.3
    loss, grad = ctx.distill_loss(x, ids.cuda(), tl.cuda(), tail=tail)
    ctx.sync_status()
    return loss, grad


# A row of 33700 bf16 tokens takes just under a third of an SM's shared memory, one of 50000 just under a half, and of
# 2 x 50000 just under a half in two CTAs.
@pytest.mark.parametrize("rows,V,K,tail,dtype,before", [(456, 50000, 8, False, BF, (33600, 33650, 33700, 33728, 33800)),
                                                        (456, 25000, 8, False, F32, (16800, 16850, 16864, 16900)),
                                                        (300, 50000, 40, True, BF, (32000, 32500, 33000, 33500)),
                                                        (228, 100000, 20, True, BF, (67000, 67200, 67456))], ids=str)
def test_lengths_asked_for_before(cuda_lib, rows, V, K, tail, dtype, before):
    want = _call(cuda_lib.Context(0), rows, V, K, tail, dtype)
    ctx = cuda_lib.Context(0)
    for other in before:
        _call(ctx, 3, other, K, tail, dtype)
    got = _call(ctx, rows, V, K, tail, dtype)
    for a, b in zip(want, got):
        assert not int((a != b).sum())
