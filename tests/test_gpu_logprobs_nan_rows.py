"""The gradient of a row that holds NaN or +inf, where what reaches the row as a whole cancels (GPU)."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("V", [77, 20000])
def test_upstream_gradients_that_cancel(cuda_lib, dtype, bad, V):
    """l = g: T dz is g at the target and p_v (l - g) = 0 elsewhere, in a row whose p is NaN NaN everywhere; zeros where
    nothing is asked of the row."""
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", 6, V, dtype)
    z[1, 3] = z[2, V - 1] = z[4, 0] = bad
    t = torch.tensor([3, 5, -1, 0, 2, 7], dtype=torch.int32, device="cuda")
    g = torch.tensor([1.0, 1.0, 0.0, 2.0, 0.0, 0.0], device="cuda")
    x = R.padded(z)
    lp = ctx.token_logprobs(x, t)
    out = ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, grad_lse=g)
    ctx.sync_status()
    assert torch.isnan(out[1]).all()
    assert not out[2].any() and not out[4].any() and not out[5].any()
    want = torch.zeros(2, V)
    want[0, 3], want[1, 0] = 1.0, 2.0
    assert torch.equal(out[[0, 3]].float().cpu(), want)
