"""README's lines on log probabilities and distillation, run as they stand (GPU)."""
import os
import re

import pytest
import torch

import paper_2608_15592_gb300 as estp
import vocab_ref as R

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_lines_run(cuda_lib):
    blocks = re.findall(r"```python\n(.*?)```", open(README).read(), flags=re.S)
    code, = [b for b in blocks if "token_logprobs(" in b]
    rows, V, T, F32 = 9, 500, 2.0, torch.float32
    z, zt, zs = (R.logits("normal", rows, V, F32, seed=s) for s in (1, 2, 3))
    targets = torch.arange(rows).int()
    lp, p = R.softmax(z, 1.0)
    ref = lp[torch.arange(rows), targets.long()]
    old = (ref - 0.1).float()
    advantage = torch.linspace(-1, 1, rows)
    ctx = cuda_lib.Context(0)
    have = dict(estp=estp, ctx=ctx, logits=R.padded(z), targets=targets.cuda(), old_logprob=old.cuda(), rows=rows,
                advantage=advantage.cuda(), entropy_cost=torch.full((rows,), -0.01, device="cuda"), T=T,
                teacher_logits=R.padded(zt), student_logits=R.padded(zs), row_weight=torch.full((rows,), T * T / rows, device="cuda"))
    exec(code, have)
    ctx.sync_status()
    # the gradient of sum of advantage ratio / rows less the entropy's share, in the logits' place
    y = z.double().clone().requires_grad_(True)
    ly = torch.log_softmax(y, 1)
    ratio = torch.exp(ly[torch.arange(rows), targets.long()] - old.double())
    (-(advantage.double() * ratio).sum() / rows + 0.01 * (ly.exp() * ly).sum()).backward()
    got = have["logits"].cpu().double()
    # an element's terms are below 1 and each off by the sum's and the exponential's error
    assert float((got - y.grad).abs().max()) < 4 * (R.SUM(V) + 2.0 ** -20)
    # distillation, with the other tokens as one bucket
    lt, pt = R.softmax(zt, T)
    y = zs.double().clone().requires_grad_(True)
    ls = torch.log_softmax(y / T, 1)
    ids = R.order(zt, 64)
    q, s = pt.gather(1, ids), ls.gather(1, ids)
    rest = 1 - q.sum(1)
    other = torch.log(1 - s.exp().sum(1))
    loss = (q * (lt.gather(1, ids) - s)).sum(1) + rest * (torch.log(rest) - other)
    (loss.sum() * T * T / rows).backward()
    assert torch.equal(have["teacher"].top_ids.cpu().long(), ids)
    # the teacher's log probabilities are fp32, off by SUM + half a step of 16: the loss is stationary in none of them
    assert float((have["loss"].cpu().double() - loss.detach()).abs().max()) < 64 * (R.SUM(V) + 2.0 ** -20)
    assert float((have["g"].cpu().double() - y.grad).abs().max()) < 4 * (R.SUM(V) + 2.0 ** -20)
    ctx.close()
