"""Distillation where every cluster, warp or block takes row after row: the copies of the next row into the place of the
present one, the statistics of every other row, the teachers' places used again, marks of named tokens made and
cleared, named tokens written a row late (GPU).  Every element is compared with 64 bits, formed on the GPU."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _teacher(rows, V, K, T, tail, seed):
    """Distinct tokens of each row (its own, a stretch of neighbours in some rows), entries that are none, of -inf, rows
    without entries, weights of 0."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    step = V // K
    ids = torch.randint(0, step, (rows, K), generator=g, device="cuda") + step * torch.arange(K, device="cuda")
    near = torch.randint(0, V - K + 1, (rows, 1), generator=g, device="cuda") + torch.arange(K, device="cuda")
    ids = torch.where((torch.arange(rows, device="cuda") % 5 == 3)[:, None], near, ids)
    ids = ids.gather(1, torch.rand(rows, K, generator=g, device="cuda").argsort(1))
    x = torch.randn(rows, K, generator=g, device="cuda") * 2 + 3
    if tail:
        x = torch.log_softmax(x / T, 1) + torch.log(0.05 + 0.9 * torch.rand(rows, 1, generator=g, device="cuda"))
    some = torch.rand(rows, K, generator=g, device="cuda") > 0.1
    some[7::11] = False
    x = torch.where(torch.rand(rows, K, generator=g, device="cuda") < 0.05, -math.inf, x)
    ids = torch.where(some, ids, -1 - ids)
    w = torch.rand(rows, generator=g, device="cuda")
    w[4::9] = 0
    return ids.int(), x, w


def _reference(z, T, ids, x, tail):
    """Loss and gradient of rows without repeated tokens, and the sizes of their terms."""
    rows, V = z.shape
    z = z.double()
    m = z.amax(1, keepdim=True)
    lp = torch.log_softmax((z - m) / T, 1)
    some, at = ids >= 0, ids.long().clamp(min=0)
    x = torch.where(some, x.double(), -math.inf)
    any_ = (some if tail else x > -math.inf).any(1, keepdim=True)
    lq = x if tail else torch.where(any_, torch.log_softmax(x / T, 1), -math.inf)
    q = torch.exp(lq)
    rest = torch.where(any_, (1 - q.sum(1, keepdim=True)).clamp(min=0), 0.0) if tail else torch.zeros_like(m)
    here = lp.gather(1, at)
    there = q > 0
    loss = torch.where(there, q * (lq - here), 0.0).sum(1)
    size = torch.where(there, q * (lq.abs() + here.abs()), 0.0).sum(1)
    total = q.sum(1, keepdim=True) + rest
    p = torch.exp(lp)
    grad, gsize = total * p, total * p
    far = 1 + ((z - m) / T).abs()
    if tail:
        spot = torch.where(some, at, V)
        named = torch.zeros(rows, V + 1, dtype=torch.bool, device=z.device).scatter_(1, spot, True)[:, :V]
        y = torch.where(named, -math.inf, lp)
        lt = torch.logsumexp(y, 1, keepdim=True)
        within = torch.exp(y - lt)
        lr = torch.log(torch.where(rest > 0, rest, 1.0))
        loss += (rest * (lr - lt))[:, 0]
        # (the rest is 1 less a sum of q that are each off by two units of their last place, 2^-22 relative)
        size += (rest * (lr.abs() + lt.abs()) + any_ * (2.0 ** -22 / 2.0 ** -21) * (lt.abs() + lr.abs() + 1))[:, 0]
        grad = grad - rest * within
        gsize = gsize + rest * within + within * any_ * (2.0 ** -22 / 2.0 ** -21)
    else:
        spot = torch.where(some, at, V)
    wide = lambda y, s: torch.cat([y, torch.zeros_like(m)], 1).scatter_add_(1, spot, s)[:, :V]  # noqa: E731
    return loss, wide(grad, -q) / T, size, wide(gsize, q) * far / T


def _check(ctx, z, T, K, tail, seed, lanes, place=False, alone=True):
    """`lanes`: threads that share a row at least.  Each adds V / lanes exponentials in four sums, half a step each, some 40
    sums and rescalings follow, and an exponential is off by two steps (vocab_ref): that is the error of ln s.  A
    term of the loss is off by 2^-21 of its size (the exponent of q is rounded, |ln q| half steps, and so is ln q).  In the
    gradient each element's own exponential is off by two steps and |d| roundings of its argument."""
    rows, V = z.shape
    ids, x, w = _teacher(rows, V, K, T, tail, seed)
    ls = 2.0 ** -21 + (V / (4 * lanes) + 40) * 2.0 ** -24
    view = R.padded(z, extra=1, fill=5.0)
    kept = view.clone()
    if alone:
        only = ctx.distill_loss(view, ids, x, temperature=T, tail=tail, row_weight=w, grads=False)
    loss, grad = ctx.distill_loss(view, ids, x, temperature=T, tail=tail, row_weight=w, out=view if place else None)
    ctx.sync_status()
    if place:
        assert grad is view and bool((view._base[:, V:] == 5).all())
    for r in range(0, rows, 64):
        s = slice(r, r + 64)
        want, gwant, size, gsize = _reference(kept[s], T, ids[s], x[s], tail)
        f = w[s].double()[:, None]
        allowed = ls * 2 + 2.0 ** -21 * size + 2.0 ** -24 * want.abs()
        for got in (loss[s], only[s]) if alone else (loss[s],):
            assert bool(torch.isfinite(got).all())
            over = (got.double() - want).abs() - allowed
            assert float(over.max()) <= 0, (r, int(over.argmax()), float(over.max()))
        off = (grad[s].double() - gwant * f).abs()
        off -= (2 * ls + 2.0 ** -21) * gsize * f + R.HALF[z.dtype] * (gwant * f).abs() + 2.0 ** -126 / T
        assert float(off.max()) <= 0, (r, int(off.argmax()) // V, int(off.argmax()) % V, float(off.max()))


def _logits(rows, V, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, V, generator=g, device="cuda") * 0.7).to(dtype)


# No tail; named tokens looked through (K up to 32); marked
FORMS = [(20, False), (17, True), (100, True)]


# 152 SMs hold at most 456 CTAs, so at most 456 / C clusters of C (and fewer of long rows).  9001 tokens: 5 rows a cluster
# where C = 1, more where C is greater.  A row of 128256 bf16 or 70001 fp32 takes more than the 200 KB of one CTA:
# C is 2 or more and clusters 228 at most, 4 rows or more each.  150001 fp32 needs 3 CTAs or more: 152 clusters, 4 rows.
@pytest.mark.parametrize("K,tail", FORMS, ids=str)
@pytest.mark.parametrize("rows,V,dtype", [(2000, 9001, BF), (2000, 9001, F32), (930, 128256, BF), (925, 70001, F32), (610, 150001, F32),
                                          (1830, 15003, F32)], ids=str)
def test_rows_of_a_cluster(cuda_lib, rows, V, dtype, K, tail):
    _check(cuda_lib.Context(0), _logits(rows, V, dtype, V), 1.0, K, tail, K, 256)


@pytest.mark.parametrize("K,tail", FORMS, ids=str)
@pytest.mark.parametrize("rows,V,dtype", [(1900, 9003, BF), (500, 128255, BF), (480, 70001, F32)], ids=str)
def test_rows_of_a_cluster_in_place(cuda_lib, rows, V, dtype, K, tail):
    _check(cuda_lib.Context(0), _logits(rows, V, dtype, V + 1), 0.8, K, tail, K + 1, 256, place=True)


# a warp a row: 3648 warps
@pytest.mark.parametrize("K,tail", FORMS + [(128, True), (128, False)], ids=str)
@pytest.mark.parametrize("rows,V,dtype", [(15001, 203, BF), (14700, 505, F32), (14603, 4003, BF)], ids=str)
@pytest.mark.parametrize("place", [False, True], ids=["apart", "in_place"])
def test_rows_of_a_warp(cuda_lib, rows, V, dtype, K, tail, place):
    _check(cuda_lib.Context(0), _logits(rows, V, dtype, V + 2), 1.3, K, tail, K + 2, 32, place=place)


# rows that are read twice: 304 blocks
@pytest.mark.parametrize("K,tail", [(20, False), (100, True)], ids=str)
@pytest.mark.parametrize("place", [False, True], ids=["apart", "in_place"])
def test_rows_of_a_block(cuda_lib, K, tail, place):
    _check(cuda_lib.Context(0), _logits(620, 819209, BF, 3), 1.0, K, tail, 5, 512, place=place)


# the loss alone: 3648 warps, rows whole, cut, and several a piece
@pytest.mark.parametrize("K,tail", FORMS, ids=str)
@pytest.mark.parametrize("rows,V,dtype", [(30001, 700, BF), (9000, 5003, F32), (4000, 20001, BF), (300, 40001, BF)], ids=str)
def test_the_loss_alone(cuda_lib, rows, V, dtype, K, tail):
    ctx, z, T = cuda_lib.Context(0), _logits(rows, V, dtype, V + 4), 0.9
    ids, x, _ = _teacher(rows, V, K, T, tail, K + 4)
    got = ctx.distill_loss(R.padded(z, fill=5.0), ids, x, temperature=T, tail=tail, grads=False)
    ctx.sync_status()
    ls = 2.0 ** -21 + (V / 128 + 40) * 2.0 ** -24
    for r in range(0, rows, 500):
        s = slice(r, r + 500)
        want, _, size, _ = _reference(z[s], T, ids[s], x[s], tail)
        over = (got[s].double() - want).abs() - (ls * 2 + 2.0 ** -21 * size + 2.0 ** -24 * want.abs())
        assert float(over.max()) <= 0, (r, int(over.argmax()), float(over.max()))


def test_the_calls_between_two_graphs(cuda_lib):
    """The sizes of the large eager step that a test of graphs makes and leaves unread."""
    for K, tail in FORMS:
        _check(cuda_lib.Context(0), _logits(2000, 9001, BF, 3), 1.0, K, tail, 3, 256)
