"""Alternatives that all lie in one warp's part of a row, and named tokens that stand side by side (GPU)."""
import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,V,k", [(300, 30011, 64), (300, 30011, 128), (1100, 9001, 20), (231, 40961, 33)])
@pytest.mark.parametrize("kind", ["ascending", "descending", "ties", "lump", "few"])
def test_alternatives_of_rows_cut_between_warps(cuda_lib, dtype, rows, V, k, kind):
    """What the warps of a row tell each other leaves nothing out, whichever of them holds the greatest logits."""
    if kind == "lump":  # more than k great ones, in one place that differs from row to row
        z = R.logits("normal", rows, V, dtype, seed=5)
        for r in range(rows):
            at = (r * 997) % (V - 150)
            z[r, at:at + 150] += 30
    elif kind == "few":  # fewer than k that are not masked
        z = torch.full((rows, V), -float("inf"), dtype=dtype)
        z[:, V - k // 2:] = torch.randn(rows, k // 2, generator=torch.Generator().manual_seed(1)).to(dtype)
    else:
        z = R.logits(kind, rows, V, dtype, seed=6)
    ctx = cuda_lib.Context(0)
    x = R.padded(z)
    lp = ctx.token_logprobs(x, top_k=k)
    ctx.sync_status()
    want = R.order(z, k)
    assert torch.equal(lp.top_ids.cpu().long(), want)
    m = z.double().amax(1, keepdim=True)
    lse = m + torch.log(torch.exp(z.double() - m).sum(1, keepdim=True))
    top = torch.take_along_dim(z.double(), want, 1) - lse
    R.close(lp.top_logprobs, top, R.SUM(V) + 2.0 ** -22 * torch.nan_to_num(top, neginf=0.0).abs())
    again = ctx.token_logprobs(x, top_k=k)
    for a, b in zip((lp.entropy, lp.norm, lp.top_ids, lp.top_logprobs), (again.entropy, again.norm, again.top_ids, again.top_logprobs)):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,V,K", [(6, 40001, 100), (6, 40001, 128), (5, 9001, 33), (5, 9001, 32), (620, 1003, 40), (620, 1003, 128),
                                      (3, 900, 128)])
def test_named_tokens_side_by_side(cuda_lib, dtype, rows, V, K):
    """Whole units of named tokens, across the ends of warps, of blocks and of 1024 units; and the two ends of a row."""
    z = R.logits("normal", rows, V, dtype, seed=7)
    ids = torch.zeros(rows, K, dtype=torch.int32)
    for r in range(rows):
        start = [0, V - K, 8192 - K // 2, 4096 - 3, V // 2, V // 5 - K // 2][r % 6] % (V - K + 1)
        ids[r] = torch.arange(start, start + K)[torch.randperm(K, generator=torch.Generator().manual_seed(r))]
    ids[rows - 1, ::2] = torch.arange(0, V, V // K)[: len(ids[0, ::2])] if V >= 4 * K else ids[rows - 1, ::2]
    x = torch.log_softmax(torch.randn(rows, K, generator=torch.Generator().manual_seed(2)), 1) - 0.5
    last = set()
    for j in range(K):  # (distinct ones only)
        if int(ids[rows - 1, j]) in last:
            ids[rows - 1, j] = -1
        last.add(int(ids[rows - 1, j]))
    ctx = cuda_lib.Context(0)
    view = R.padded(z)
    loss, grad = ctx.distill_loss(view, ids.cuda(), x.cuda(), tail=True)
    alone = ctx.distill_loss(view, ids.cuda(), x.cuda(), tail=True, grads=False)
    ctx.sync_status()
    want, gwant, size, gsize = R.distill(z, 1.0, ids, x, True)
    tol = 2 * R.SUM(V) + 2.0 ** -21
    R.close(loss, want, tol * (size + 1), "loss")
    R.close(alone, want, tol * (size + 1), "loss alone")
    R.close(grad, gwant, tol * gsize + R.HALF[dtype] * gwant.abs() + 1e-37, "gradient")
