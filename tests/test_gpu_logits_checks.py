"""The calls on rows of logits in the bounds-checked build, in every form of their kernels (GPU): no check fires, and every
output equals the release build's bit for bit."""
import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _outputs(estp, library, rows, V, dtype, K, top):
    g = torch.Generator(device="cuda").manual_seed(V + K)
    ctx = estp.Context(0, library=library)
    z = R.padded((torch.randn(rows, V, generator=g, device="cuda") * 2).to(dtype), extra=1, fill=3.0)
    step = V // K
    ids = torch.randint(0, step, (rows, K), generator=g, device="cuda") + step * torch.arange(K, device="cuda")
    ids = torch.where(torch.rand(rows, K, generator=g, device="cuda") < 0.1, -1, ids).int()
    x = torch.log_softmax(torch.randn(rows, K, generator=g, device="cuda"), 1) - 0.3
    w = torch.rand(rows, generator=g, device="cuda") - 0.5
    t = torch.randint(-1, V, (rows,), generator=g, device="cuda").int()
    out = []
    for tail in (False, True):
        out += [*ctx.distill_loss(z, ids, x, temperature=0.8, tail=tail, row_weight=w),
                ctx.distill_loss(z, ids, x, temperature=0.8, tail=tail, grads=False)]
    lp = ctx.token_logprobs(z, t, top_k=top)
    out += [lp.logprob, lp.entropy, lp.norm]
    if top:
        out += [lp.top_ids, lp.top_logprobs, ctx.token_logprobs_grad(z, t, lp, grad_logprob=w, grad_top=lp.top_logprobs)]
    out.append(ctx.token_logprobs_grad(z, t, lp, grad_logprob=w, grad_entropy=w, out=z))
    out.append(z._base)
    ctx.sync_status()  # raises EstpError(ESTP_ERR_BOUNDS) if any check fired
    ctx.close()
    return out


# one row and few by blocks; rows cut between warps, by whole and by equal pieces; many short rows by a warp each; clusters of
# one and of several CTAs with several rows each; rows that are read twice
@pytest.mark.parametrize("K,top", [(16, 20), (100, 0), (33, 64), (7, 128)], ids=str)
@pytest.mark.parametrize("rows,V,dtype", [(1, 152064, BF), (5, 40001, F32), (300, 9001, BF), (1500, 9001, F32), (700, 300, F32),
                                          (4001, 1003, BF), (500, 120003, BF), (3, 819300, BF), (2, 409900, F32), (310, 409999, F32)], ids=str)
def test_checked_build_gives_the_same_bits(cuda_lib, rows, V, dtype, K, top):
    estp = cuda_lib
    a = _outputs(estp, estp.lib, rows, V, dtype, K, top)
    b = _outputs(estp, estp.load_library(estp.CHECKS_LIB_PATH), rows, V, dtype, K, top)
    assert len(a) == len(b)
    for i, (p, q) in enumerate(zip(a, b)):
        assert not int((p != q).sum()), i
