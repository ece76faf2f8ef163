"""The length head's counters on another stream than a busy default one (GPU)."""
import pytest
import torch

from test_gpu_context_zeroed import _dirty, _same

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_first_prediction_on_another_stream(cuda_lib):
    """The length head's counters, made by its first call and again by one of more prompts."""
    g = torch.Generator().manual_seed(3)
    D, K, lens = 1000, 32, [40, 1, 300, 7, 64]
    cu = torch.tensor([0] + lens).cumsum(0).int().cuda()
    n = sum(lens)
    hidden = torch.randn(n, D, generator=g).to(BF).cuda()
    H, S = torch.rand(n, generator=g).cuda(), (torch.rand(n, generator=g) / 100).cuda()
    head = cuda_lib.Head(torch.randn(K, D, generator=g).cuda(), torch.randn(K, generator=g).cuda(), (torch.arange(K) * 256.0).cuda())
    many = torch.cat([cu[:1], cu[1:2].expand(60), cu[1:]]).contiguous()  # empty prompts in front

    def calls(ctx, stream):
        out = []
        for c in (cu, many):
            pooled, pred = torch.empty(len(c) - 1, D, device="cuda"), torch.empty(len(c) - 1, device="cuda")
            torch.cuda.synchronize()
            torch.cuda._sleep(100_000_000 if stream is not None else 1)
            out += ctx.pool(hidden, H, S, c, 0.7, 0.3, 1.0, head=head, pooled=pooled, pred=pred, stream=stream)
            if stream is not None:
                stream.synchronize()
        return out

    usual = cuda_lib.Context(0)
    want = calls(usual, None)
    usual.sync_status()
    side = torch.cuda.Stream()
    for _ in range(3):
        _dirty()
        ctx = cuda_lib.Context(0)
        got = calls(ctx, side)
        _same(want, got)
        ctx.sync_status(stream=side)
        ctx.close()
