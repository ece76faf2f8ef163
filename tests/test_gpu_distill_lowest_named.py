"""Distillation where a named token's logit is the type's lowest value and the teacher gives it next to nothing: the
loss is finite although the token's ln p is beyond fp32 or near its end (GPU)."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# ln q of the named token: about 1e-36, 6e-39 and 1e-42 (fp32's denormals), its least value
FAINT = [-82.9, -88.0, -96.7, -103.0]


def _near(T):
    """The fp32 number that the kernels take for T."""
    return torch.tensor(T, dtype=F32).item()


def _gradient(z, T, ids, x, tail):
    """The gradient and the sizes of its terms.  (vocab_ref's takes the other tokens relative to the greatest of all, from
    which 64 bits cannot tell them apart where that is 3e38.)"""
    rows, V = z.shape
    named = torch.zeros(rows, V, dtype=torch.bool).scatter_(1, ids.long(), True)
    p = R.softmax(z, T)[1]
    q = torch.exp(x.double() if tail else torch.log_softmax(x.double() / T, 1))
    rest = (1 - q.sum(1, keepdim=True)).clamp(min=0) if tail else torch.zeros(rows, 1, dtype=torch.float64)
    out = (q.sum(1, keepdim=True) + rest) * p
    steps = lambda y: 1 + torch.nan_to_num(y - y.amax(1, keepdim=True), nan=0.0, neginf=0.0).abs().clamp(max=200)  # noqa: E731
    y = z.double() / T
    size = out * steps(y)
    if tail:
        y = torch.where(named, -math.inf, y)
        within = torch.softmax(y, 1)
        out = out - rest * within
        # (the rest is 1 less a sum: off by a few steps of 1)
        size = size + rest * within * steps(y) + within * 4 * 2.0 ** -24 / R.SUM(V)
    return out.scatter_add(1, ids.long(), -q) / T, size.scatter_add(1, ids.long(), q) / T


def _check(ctx, z, T, ids, x, tail, faint):
    """`faint`: the named token whose term this is about.  Its q is off by the rounding of its exponent (|ln q| 2^-23), two
    steps of the exponential and one each of the sum and the quotient (2^-21), and among denormals by two steps and a
    half of 2^-149; all of that times |ln p|.  The other terms as in every case (vocab_ref)."""
    V = z.shape[1]
    view = R.padded(z)
    loss, grad = ctx.distill_loss(view, ids.cuda(), x.cuda(), temperature=T, tail=tail)
    alone = ctx.distill_loss(view, ids.cuda(), x.cuda(), temperature=T, tail=tail, grads=False)
    ctx.sync_status()
    want, _, size, _ = R.distill(z, T, ids, x, tail)
    gwant, gsize = _gradient(z, T, ids, x, tail)
    xs = x.double()
    lq = xs if tail else torch.log_softmax(xs / T, 1)
    lq = lq[:, faint]
    away = (R.softmax(z, T)[0][torch.arange(len(z)), ids[:, faint].long()]).abs()
    tol = 2 * R.SUM(V) + 2.0 ** -21
    allowed = tol * (size + 1) + away * (torch.exp(lq) * lq.abs() * 2.0 ** -23 + 3 * 2.0 ** -149)
    assert bool(torch.isfinite(want).all())
    R.close(loss, want, allowed, "loss")
    R.close(alone, want, allowed, "loss alone")
    # (an exponential below 2^-126 is flushed to 0, which p / T takes over as at most 2^-126 / T: s >= 1; and a gradient
    # that is itself below 2^-126 is rounded to a denormal)
    R.close(grad, gwant, tol * gsize + R.HALF[z.dtype] * gwant.abs() + 2.0 ** -126 / T + 1e-37, "gradient")


def _inputs(rows, V, T, tail, dtype, top=None):
    z = R.logits("normal", rows, V, dtype, seed=V)
    if top is not None:
        z[:, 0] = top
    ids = torch.tensor([V - 2, V // 2, V // 3], dtype=torch.int32).repeat(rows, 1)
    z[:, V // 3] = torch.finfo(dtype).min
    faint = torch.tensor([FAINT[r % len(FAINT)] for r in range(rows)])
    x = torch.stack([torch.full((rows,), math.log(0.5)), torch.full((rows,), math.log(0.2)), faint], 1)
    return z, ids, x if tail else x * T


# by clusters, a warp a row, two reads a row
@pytest.mark.parametrize("rows,V,dtype", [(9, 5003, BF), (9, 5003, F32), (700, 61, BF), (700, 61, F32), (2, 900001, BF), (2, 500001, F32)],
                         ids=str)
@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("T", [0.7, 1.0, 1e-3])
def test_the_lowest_value_named_faintly(cuda_lib, rows, V, dtype, tail, T):
    T = _near(T)
    z, ids, x = _inputs(rows, V, T, tail, dtype)
    _check(cuda_lib.Context(0), z, T, ids, x, tail, 2)


@pytest.mark.parametrize("rows,V,dtype", [(9, 5003, BF), (9, 5003, F32), (700, 61, BF), (700, 61, F32)], ids=str)
@pytest.mark.parametrize("T", [1.0, 4.0, 1024.0])
def test_logits_further_apart_than_the_type_goes(cuda_lib, rows, V, dtype, T):
    """The greatest logit is 3e38, so that its distance from the lowest overflows, while (z - max) / T or q times it does
    not.  Where the tokens of q = 0.5 and 0.2 lie that far below it too, the loss is some 1e38 / T; an entry of -inf
    leaves the faint token alone."""
    z, ids, x = _inputs(rows, V, T, True, dtype, top=3e38)
    ctx = cuda_lib.Context(0)
    near = ids.clone()
    near[:, 0] = 0  # the token with everything
    x[:, 0] = math.log(0.99)
    x[:, 1] = -math.inf
    for tail in (False, True):
        # (renormalised, the entries are logits: x T)
        _check(ctx, z, T, near, x if tail else x * T, tail, 2)
