"""Distillation from a teacher's top logits: the loss and its gradient against 64 bits (GPU)."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _teacher(rows, V, K, T, tail, seed, repeat=False):
    """Distinct tokens (with `repeat` some twice) with holes, and logits or log probabilities of them."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(rows)]).int()
    x = torch.randn(rows, K, generator=g) * 2 + 3
    if tail:  # log probabilities that leave a rest, none of it in some rows
        x = torch.log_softmax(x / T, 1) + torch.log(0.05 + 0.95 * torch.rand(rows, 1, generator=g))
        x[1::4] = torch.log_softmax(x[1::4], 1)
    if K > 2:
        ids[::3, K // 2] = -1
        x[::3, K // 2] = math.nan  # not read
        x[::5, 1] = -math.inf
    ids[2::6] = -7
    if repeat:
        ids[:, K - 1] = ids[:, 0]
    return ids, x


def _check(ctx, z, T, K, tail, seed=3, weight=True, repeat=False):
    rows, V = z.shape
    ids, x = _teacher(rows, V, K, T, tail, seed, repeat)
    g = torch.Generator().manual_seed(seed)
    w = torch.rand(rows, generator=g) if weight else None
    if weight and rows > 3:
        w[3] = 0
    view = R.padded(z)
    loss, grad = ctx.distill_loss(view, ids.cuda(), x.cuda(), temperature=T, tail=tail, row_weight=None if w is None else w.cuda())
    alone = ctx.distill_loss(view, ids.cuda(), x.cuda(), temperature=T, tail=tail, grads=False)
    ctx.sync_status()
    want, gwant, size, gsize = R.distill(z, T, ids, x, tail)
    tol = 2 * R.SUM(V) + 2.0 ** -21
    R.close(loss, want, tol * (size + 1), "loss")
    R.close(alone, want, tol * (size + 1), "loss alone")
    f = torch.ones(rows, 1, dtype=torch.float64) if w is None else w.double()[:, None]
    R.close(grad, gwant * f, tol * gsize * f + R.HALF[z.dtype] * (gwant * f).abs() + 1e-37, "gradient")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("rows,V,K", [(1, 1, 1), (7, 3, 3), (5, 9, 4), (13, 100, 33), (400, 130, 20), (9, 8200, 128), (4, 32001, 64),
                                      (1, 152064, 32), (3, 128256, 100)])
def test_shapes(cuda_lib, dtype, tail, rows, V, K):
    _check(cuda_lib.Context(0), R.logits("normal", rows, V, dtype, seed=V), 1.0, K, tail)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("kind", ["ties", "equal", "masked", "lowest", "sharp", "far"])
@pytest.mark.parametrize("T", [0.7, 2.5])
def test_kinds(cuda_lib, dtype, tail, kind, T):
    _check(cuda_lib.Context(0), R.logits(kind, 14, 1003, dtype), T, 16, tail, weight=False)


@pytest.mark.parametrize("V,dtype", [(300007, F32), (500001, F32), (900001, BF)], ids=str)
def test_long_rows(cuda_lib, V, dtype):
    """The longest that a cluster keeps, and some of more units than a block marks at a time."""
    for tail in (False, True):
        _check(cuda_lib.Context(0), R.logits("normal", 2, V, dtype, seed=4), 1.0, 24, tail)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("rows,V,K", [(700, 1, 1), (1300, 33, 8), (4000, 40, 33), (650, 1001, 128), (611, 4095, 20), (3700, 1200, 9)])
def test_many_short_rows(cuda_lib, dtype, tail, rows, V, K):
    """A warp a row; some warps take several."""
    _check(cuda_lib.Context(0), R.logits("normal", rows, V, dtype, seed=rows), 0.8, K, tail, repeat=not tail and K > 2)


@pytest.mark.parametrize("rows,V", [(700, 60), (5, 5000)])
def test_kinds_of_rows_by_either_way(cuda_lib, rows, V):
    for kind in ("masked", "lowest", "sharp", "ties"):
        for tail in (False, True):
            _check(cuda_lib.Context(0), R.logits(kind, rows, V, BF), 1.3, 12, tail)


def test_repeated_tokens(cuda_lib):
    """Renormalised they count each time; with the tail they are left out and recorded."""
    z = R.logits("normal", 7, 500, F32)
    _check(cuda_lib.Context(0), z, 1.0, 12, False, repeat=True)
    ctx = cuda_lib.Context(0)
    with pytest.raises(cuda_lib.EstpError) as e:
        _check(ctx, z, 1.0, 12, True, repeat=True)
    assert e.value.status == cuda_lib.ESTP_ERR_INVALID_ARG
    ids, x = _teacher(7, 500, 12, 1.0, True, 3, True)
    loss = ctx.distill_loss(R.padded(z), ids.cuda(), x.cuda(), tail=True, grads=False)
    want, _, size, _ = R.distill(z, 1.0, ids, x, True)
    R.close(loss, want, (2 * R.SUM(500) + 2.0 ** -21) * (size + 1), "loss")


def test_tokens_past_the_vocabulary_are_left_out(cuda_lib):
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", 3, 50, F32)
    ids = torch.tensor([[1, 50, 4], [2 ** 30, 51, 99], [0, 1, 2]], dtype=torch.int32)
    x = torch.randn(3, 3)
    loss, grad = ctx.distill_loss(R.padded(z), ids.cuda(), x.cuda())
    with pytest.raises(cuda_lib.EstpError) as e:
        ctx.sync_status()
    assert e.value.status == cuda_lib.ESTP_ERR_INVALID_ARG
    want, gwant, size, gsize = R.distill(z, 1.0, ids, x, False)
    tol = 2 * R.SUM(50) + 2.0 ** -21
    R.close(loss, want, tol * (size + 1))
    R.close(grad, gwant, tol * gsize + 2.0 ** -24 * gwant.abs())
    assert loss[1] == 0 and not grad[1].any()


def test_rows_without_teacher_or_weight(cuda_lib):
    """NaN in such rows reaches nothing; in another one it shows."""
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", 6, 700, BF)
    z[0], z[1, 5], z[2], z[3, 9] = math.nan, math.inf, math.nan, math.nan
    ids = torch.arange(4, dtype=torch.int32).repeat(6, 1)
    ids[0], ids[1] = -1, -3
    w = torch.tensor([1.0, 1.0, 0.0, 1.0, 1.0, 0.0])
    for tail in (False, True):
        x = torch.full((6, 4), -2.0)
        loss, grad = ctx.distill_loss(R.padded(z), ids.cuda(), x.cuda(), tail=tail, row_weight=w.cuda())
        ctx.sync_status()
        assert loss[0] == 0 and loss[1] == 0 and torch.isnan(loss[2:4]).all() and torch.isfinite(loss[4:]).all()
        assert not grad[0].any() and not grad[1].any() and not grad[2].any() and not grad[5].any()
        assert torch.isnan(grad[3]).all() and torch.isfinite(grad[4]).all()


def test_a_tail_that_is_far_below(cuda_lib):
    """Named tokens hold all but 1e-40 of the student's mass: the rest has a loss and a gradient all the same."""
    ctx = cuda_lib.Context(0)
    z = torch.zeros(2, 4096)
    z[:, 10] = 100.0
    z[:, 11] = 99.0
    ids = torch.tensor([[10, 11], [10, 11]], dtype=torch.int32)
    x = torch.log(torch.tensor([[0.5, 0.25], [0.7, 0.3]]))
    loss, grad = ctx.distill_loss(R.padded(z), ids.cuda(), x.cuda(), tail=True)
    ctx.sync_status()
    want, gwant, size, gsize = R.distill(z, 1.0, ids, x, True)
    R.close(loss, want, (2 * R.SUM(4096) + 2.0 ** -21) * (size + 1))
    R.close(grad, gwant, (2 * R.SUM(4096) + 2.0 ** -21) * (gsize + gwant.abs()))
    assert bool((grad[0, 12:] < 0).all())


@pytest.mark.parametrize("V,K,T", [(4001, 8, 3.0), (32000, 20, 2.0), (300, 4, 1.0), (9000, 1, 2.0)])
def test_a_small_loss_keeps_its_digits(cuda_lib, V, K, T):
    """A student near its teacher, most of whose mass lies in the rest: the loss is far below its terms.  What is off: the
    named tokens' share of the sums (SUM(V) and two roundings of an exponent of some 20, 2^-19, relative), q by two steps,
    and the result's rounding; the logarithms' errors would be 2^-20 of 1."""
    ctx, rows = cuda_lib.Context(0), 6
    z = R.logits("normal", rows, V, F32, seed=V) / 3
    g = torch.Generator().manual_seed(K)
    teacher = z.double() + 0.02 * torch.randn(rows, V, generator=g, dtype=torch.float64)
    lt = torch.log_softmax(teacher / T, 1)
    ids = torch.topk(lt, K, dim=1).indices
    x = lt.gather(1, ids).float()
    loss, grad = ctx.distill_loss(R.padded(z), ids.int().cuda(), x.cuda(), temperature=T, tail=True)
    ctx.sync_status()
    want, gwant, _, gsize = R.distill(z, T, ids.int(), x, True)
    named = R.softmax(z, T)[1].gather(1, ids).sum(1) + x.double().exp().sum(1)
    allowed = (R.SUM(V) + 2.0 ** -19) * named + 2.0 ** -22 * want
    assert float(named.max()) < 1.5 and float((want / named).max()) < 0.05  # the case that is meant
    R.close(loss, want, allowed, "loss")
    R.close(grad, gwant, (2 * R.SUM(V) + 2.0 ** -21) * gsize, "gradient")


def test_gradient_agrees_with_differences(cuda_lib):
    ctx, rows, V, K = cuda_lib.Context(0), 3, 41, 5
    z = R.logits("normal", rows, V, F32, seed=2)
    for tail in (False, True):
        for T in (1.0, 1.7):
            ids, x = _teacher(rows, V, K, T, tail, 9)
            _, grad = ctx.distill_loss(R.padded(z), ids.cuda(), x.cuda(), temperature=T, tail=tail)
            grad = grad.cpu().double()
            for v in range(V):
                step = torch.zeros(rows, V, dtype=torch.float64)
                step[:, v] = 1e-5
                up, down = (R.distill(z.double() + sign * step, T, ids, x, tail)[0] for sign in (1, -1))
                assert torch.allclose(grad[:, v], (up - down) / 2e-5, rtol=1e-5, atol=2e-6)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,V", [(9, 5003), (400, 1001), (2, 60000)])
def test_in_place_and_padding(cuda_lib, dtype, rows, V):
    ctx = cuda_lib.Context(0)
    ids, x = _teacher(rows, V, 10, 1.0, True, 1)
    ids, x = ids.cuda(), x.cuda()
    view = R.padded(R.logits("normal", rows, V, dtype), extra=2, fill=7.0)
    loss, want = ctx.distill_loss(view, ids, x, tail=True)
    wide = torch.full((rows, V + -V % 8 + 8), 3.0, dtype=dtype, device="cuda")
    again, _ = ctx.distill_loss(view, ids, x, tail=True, out=wide)
    assert torch.equal(again, loss) and torch.equal(wide[:, :V], want) and bool((wide[:, V:] == 3).all())
    placed, got = ctx.distill_loss(view, ids, x, tail=True, out=view)
    ctx.sync_status()
    assert torch.equal(placed, loss) and got is view and torch.equal(view, want)
    assert bool((view._base[:, V:] == 7).all())
