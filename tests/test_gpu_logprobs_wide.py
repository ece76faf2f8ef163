"""Log probabilities of logits further apart than the type goes (GPU)."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,V", [(3, 1001), (400, 300), (2, 40001)])
@pytest.mark.parametrize("T", [1.0, 4.0, 1e6])
def test_a_token_that_far_below(cuda_lib, dtype, rows, V, T):
    """The greatest logit is 3e38 and the target's the type's lowest: z - max overflows, ln p is finite for T > 2."""
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", rows, V, dtype, seed=V)
    low = torch.finfo(dtype).min
    z[:, 5] = 3e38
    z[:, 7:] = low
    t = torch.full((rows,), 9, dtype=torch.int32)
    lp = ctx.token_logprobs(R.padded(z), t.cuda(), top_k=12, temperature=T)
    ctx.sync_status()
    want = R.softmax(z, T)[0]
    allowed = lambda y: R.SUM(V) + 2.0 ** -22 * torch.nan_to_num(y, neginf=0.0).abs()  # noqa: E731
    ids = R.order(z, 12)
    assert torch.equal(lp.top_ids.cpu().long(), ids)
    top = torch.take_along_dim(want, ids, 1)
    R.close(lp.top_logprobs, top, allowed(top), "alternatives")
    R.close(lp.logprob, want[:, 9], allowed(want[:, 9]), "target")
    assert (T > 2) == bool(torch.isfinite(lp.logprob).all()) and not math.isnan(float(lp.logprob.sum()))
