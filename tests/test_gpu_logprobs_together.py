"""Log probabilities, their gradient and distillation as a program uses them: a teacher's alternatives taught
to a student, steps captured in graphs, other streams, the bounds-checked build (GPU)."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def test_a_teacher_teaches_a_student(cuda_lib):
    """The teacher's own alternatives: with all tokens named the loss is the full divergence, a student equal
    to its teacher has loss 0 and no gradient, and steps along the gradient lower the loss."""
    ctx, rows, V, T = cuda_lib.Context(0), 12, 96, 1.5
    teacher, student = R.logits("normal", rows, V, F32, seed=1), R.logits("normal", rows, V, F32, seed=2)
    said = ctx.token_logprobs(R.padded(teacher), top_k=V, temperature=T)
    lt, p = R.softmax(teacher, T)
    ls, _ = R.softmax(student, T)
    full = (p * (lt - ls)).sum(1)
    loss = ctx.distill_loss(R.padded(student), said.top_ids, said.top_logprobs, temperature=T, tail=True, grads=False)
    R.close(loss, full, 1e-5 * (1 + full))
    few = ctx.token_logprobs(R.padded(teacher), top_k=8, temperature=T)
    same, grad = ctx.distill_loss(R.padded(teacher), few.top_ids, few.top_logprobs, temperature=T, tail=True)
    assert float(same.abs().max()) < 2e-6 and float(grad.abs().max()) < 2e-6
    x = R.padded(student)
    first = None
    for _ in range(4):
        loss, grad = ctx.distill_loss(x, few.top_ids, few.top_logprobs, temperature=T, tail=True)
        assert first is None or bool((loss < first).all())
        first = loss
        x = R.padded(x.cpu() - 0.5 * grad.cpu())
    ctx.sync_status()


def test_policy_gradient_step(cuda_lib):
    """Entropy as the framework gives it elsewhere, a surrogate's gradient from the ratio of two policies."""
    ctx, rows, V = cuda_lib.Context(0), 20, 1000
    z, old = R.logits("normal", rows, V, BF, seed=3), R.logits("normal", rows, V, BF, seed=3) * 0.98
    t = torch.randint(0, V, (rows,)).int()
    x = R.padded(z)
    now, before = ctx.token_logprobs(x, t.cuda()), ctx.token_logprobs(R.padded(old), t.cuda())
    H = ctx.token_entropy(x._base, V=V) if x._base is not None and torch.isfinite(x._base).all() else ctx.token_entropy(R.padded(z, fill=0.0), V=V)
    assert float((H - now.entropy).abs().max()) < 1e-4
    advantage = torch.randn(rows, device="cuda")
    ratio = torch.exp(now.logprob - before.logprob)
    grad = ctx.token_logprobs_grad(x, t.cuda(), now, grad_logprob=-advantage * ratio / rows,
                                   grad_entropy=torch.full((rows,), -0.01 / rows, device="cuda"))
    ctx.sync_status()
    y = z.double().clone().requires_grad_(True)
    lp = torch.log_softmax(y, 1)
    picked = lp[torch.arange(rows), t.long()]
    ref = torch.log_softmax(old.double(), 1)[torch.arange(rows), t.long()]
    value = -(advantage.cpu().double() * torch.exp(picked - ref)).mean() + 0.01 * (lp.exp() * lp).sum(1).mean()
    value.backward()
    assert float((grad.cpu().double() - y.grad).norm() / y.grad.norm()) < 4e-3  # bf16 results


def _step(ctx, x, t, ids, tl, adv):
    lp = ctx.token_logprobs(x, t, top_k=7)
    g = ctx.token_logprobs_grad(x, t, lp, grad_logprob=adv, grad_top=lp.top_logprobs)
    loss, d = ctx.distill_loss(x, ids, tl, tail=True, row_weight=adv)
    return [lp.logprob, lp.entropy, lp.norm, lp.top_ids, lp.top_logprobs, g, loss, d]


def _inputs(rows, V, seed, dtype=BF):
    x = R.padded(R.logits("normal", rows, V, dtype, seed=seed), fill=0.0)
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (rows,), generator=g).int().cuda()
    ids = torch.stack([torch.randperm(V, generator=g)[:9] for _ in range(rows)]).int().cuda()
    tl = (torch.log_softmax(torch.randn(rows, 9, generator=g), 1) - 0.3).cuda()
    return [x, t, ids, tl, torch.randn(rows, generator=g).cuda()]


def test_first_call_in_a_graph(cuda_lib):
    """A new context's first calls are captured; larger eager calls follow; replays on new inputs give what the
    calls give, and two graphs of one context in turn."""
    ctx, other = cuda_lib.Context(0), cuda_lib.Context(0)
    a, b = _inputs(5, 30001, 1), _inputs(300, 2003, 2, F32)
    graphs = []
    for inp in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _step(ctx, *inp)
        graphs.append((g, inp, out))
    big = _inputs(2000, 9001, 3)
    _step(ctx, *big)
    for seed in (4, 5):
        for (g, inp, out), shape in zip(graphs, ((5, 30001, BF), (300, 2003, F32))):
            for dst, src in zip(inp, _inputs(shape[0], shape[1], seed, shape[2])):
                dst.copy_(src)
            for o in out:
                o.zero_()
            g.replay()
            want = _step(other, *inp)
            torch.cuda.synchronize()
            for i, (p, q) in enumerate(zip(out, want)):
                assert torch.equal(p, q), i
    ctx.sync_status()


def test_another_stream(cuda_lib):
    ctx, side = cuda_lib.Context(0), torch.cuda.Stream()
    x, t, ids, tl, adv = _inputs(40, 20000, 6)
    want = _step(ctx, x, t, ids, tl, adv)
    torch.cuda.synchronize()
    lp = ctx.token_logprobs(x, t, top_k=7, stream=side)
    g = ctx.token_logprobs_grad(x, t, lp, grad_logprob=adv, grad_top=lp.top_logprobs, stream=side)
    loss, d = ctx.distill_loss(x, ids, tl, tail=True, row_weight=adv, stream=side)
    ctx.sync_status(stream=side)
    for p, q in zip(want, [lp.logprob, lp.entropy, lp.norm, lp.top_ids, lp.top_logprobs, g, loss, d]):
        assert torch.equal(p, q)


@pytest.mark.parametrize("rows,V,dtype", [(1, 152064, BF), (37, 4001, BF), (600, 515, F32), (3, 100003, F32)])
def test_checked_build_gives_the_same_bits(cuda_lib, rows, V, dtype):
    release, checked = cuda_lib.Context(0), cuda_lib.Context(0, library=cuda_lib.load_library(cuda_lib.CHECKS_LIB_PATH))
    inp = _inputs(rows, V, 7, dtype)
    a, b = _step(release, *inp), _step(checked, *inp)
    release.sync_status()
    checked.sync_status()
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_overlapping_gradient_is_refused(cuda_lib):
    ctx = cuda_lib.Context(0)
    wide = torch.zeros(9, 64, dtype=BF, device="cuda")
    x, later = wide[:8], wide[1:]
    t = torch.zeros(8, dtype=torch.int32, device="cuda")
    lp = ctx.token_logprobs(x, t)
    g = torch.ones(8, device="cuda")
    for call in (lambda: ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, out=later),
                 lambda: ctx.distill_loss(x, t[:, None].contiguous(), g[:, None].contiguous(), out=later)):
        with pytest.raises(cuda_lib.EstpError) as e:
            call()
        assert e.value.status == cuda_lib.ESTP_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        ctx.token_logprobs(x.cpu(), t)
    with pytest.raises(ValueError):
        ctx.token_logprobs(x, t.cpu())
    ctx.sync_status()
    assert not math.isnan(float(lp.entropy.sum()))
