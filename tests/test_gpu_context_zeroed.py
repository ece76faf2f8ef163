"""A context made while the default stream is busy: its arrival counters are zero when the first call on another stream
reads them, and stay what the calls made them (GPU)."""
import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _dirty():
    """Memory that the driver hands out next is likely not zero."""
    junk = [torch.full((4 << 20,), -1, dtype=torch.int32, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    del junk
    torch.cuda.empty_cache()


def _same(a, b):
    assert len(a) == len(b)
    for i, (p, q) in enumerate(zip(a, b)):
        assert torch.equal(p.view(torch.int32), q.view(torch.int32)), i


# blocks that share a row; rows cut between warps; both with lists
@pytest.mark.parametrize("rows,V,dtype", [(3, 152064, BF), (301, 9001, BF), (500, 9001, F32)], ids=str)
def test_first_calls_on_another_stream(cuda_lib, rows, V, dtype):
    x = R.padded(R.logits("normal", rows, V, dtype, seed=1), fill=0.0)
    g = torch.Generator().manual_seed(2)
    t = torch.randint(0, V, (rows,), generator=g).int().cuda()
    ids = torch.stack([torch.randperm(V, generator=g)[:9] for _ in range(rows)]).int().cuda()
    tl = (torch.log_softmax(torch.randn(rows, 9, generator=g), 1) - 0.3).cuda()

    def calls(ctx, stream):
        lp = ctx.token_logprobs(x, t, top_k=20, stream=stream)
        loss = ctx.distill_loss(x, ids, tl, tail=True, grads=False, stream=stream)
        plain = ctx.token_logprobs(x, t, stream=stream)
        return [lp.logprob, lp.entropy, lp.norm, lp.top_ids, lp.top_logprobs, loss, plain.logprob, plain.entropy, plain.norm]

    usual = cuda_lib.Context(0)
    want = calls(usual, None)
    usual.sync_status()
    side = torch.cuda.Stream()
    for _ in range(3):
        _dirty()
        torch.cuda._sleep(200_000_000)  # about a tenth of a second
        ctx = cuda_lib.Context(0)
        got = calls(ctx, side)
        side.synchronize()
        _same(want, got)
        torch.cuda.synchronize()  # what the default stream held is done: the counters are as the calls left them
        again = calls(ctx, side)
        ctx.sync_status(stream=side)
        _same(want, again)
        ctx.close()
