"""Plain 64-bit definitions of the calls on rows of logits (CPU), logits to try them on, and how far the
kernels' fp32 arithmetic may be from them.

Error of a sum of V exponentials held in fp32: a lane adds V / 128 of them one after another in each of
its four sums (half a step, 2^-24, each), then some 20 sums and rescalings follow; the exponential itself and
its argument are off by about two steps (2^-22), the argument's rounding weighted by 2^d |d| <= 0.54.
So ln s is within SUM(V) = 2^-21 + (V / 128 + 32) 2^-24."""
import math

import torch


def SUM(V):
    return 2.0 ** -21 + (V / 128 + 32) * 2.0 ** -24


HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def padded(x, extra=0, fill=float("nan"), device="cuda"):
    """[rows, V] of x on the GPU whose rows start on 16 bytes; what lies between them is `fill`."""
    per = 16 // x.element_size()
    wide = torch.full((x.shape[0], x.shape[1] + -x.shape[1] % per + extra * per), fill, dtype=x.dtype, device=device)
    wide[:, : x.shape[1]] = x.to(device)
    return wide[:, : x.shape[1]]


def logits(kind, rows, V, dtype, seed=0):
    """Logits of one kind on the CPU."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, V, generator=g, dtype=torch.float64) * 3
    if kind == "ties":  # a handful of values: almost every comparison is one between equals
        x = torch.randint(-3, 3, (rows, V), generator=g).double()
        x[torch.rand(rows, V, generator=g) < 0.1] = -0.0
    elif kind == "equal":
        x = torch.full((rows, V), -1.25, dtype=torch.float64)
    elif kind == "ascending":
        x = torch.linspace(-40, 40, V, dtype=torch.float64).expand(rows, V).clone()
    elif kind == "descending":
        x = torch.linspace(40, -40, V, dtype=torch.float64).expand(rows, V).clone()
    elif kind == "masked":  # few tokens left, in some rows none
        x[torch.rand(rows, V, generator=g) < 0.97] = -math.inf
        x[::3] = -math.inf
        x[::3, V // 2] = 1.5
        x[::5] = -math.inf
    elif kind == "lowest":  # masks of the type's lowest value, some rows of nothing else
        x[torch.rand(rows, V, generator=g) < 0.9] = torch.finfo(dtype).min
        x[::2] = torch.finfo(dtype).min
    elif kind == "sharp":
        x = x * 0.1
        x[torch.arange(rows), torch.randint(0, V, (rows,), generator=g)] += 60
    elif kind == "far":  # large values beside each other
        x = x + 20000
    else:
        assert kind == "normal"
    return x.to(dtype)


def softmax(z, T):
    """ln p and p in 64 bits; a row of -inf alone has -inf and 0.  The maximum is subtracted first: beside
    the type's lowest value even 64 bits lose ln of the sum."""
    m = z.double().amax(1, keepdim=True)
    y = (z.double() - torch.where(m == -math.inf, 0.0, m)) / T
    lp = torch.where(m == -math.inf, -math.inf, y - torch.logsumexp(y, 1, keepdim=True))
    return lp, torch.exp(lp)


def entropy(lp, p):
    return -torch.where(p > 0, p * lp, 0.0).sum(1)


def order(z, k):
    """Tokens of the k greatest logits, the lower one first among equals."""
    return torch.sort(z.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :k]


def grad(z, T, targets, ids, g, gH, gl, ga):
    """The gradient, and the sum of its terms' sizes (what an error is relative to)."""
    lp, p = softmax(z, T)
    H = entropy(lp, p)[:, None]
    empty = ~(p.sum(1) > 0)
    rows = z.shape[0]
    at = torch.arange(rows)
    out, size = torch.zeros_like(p), torch.zeros_like(p)

    def named(tokens, value):
        value = torch.where((tokens < 0) | empty, 0.0, value.double())
        t = tokens.clamp(min=0).long()
        out.index_put_((at, t), value, accumulate=True)
        size.index_put_((at, t), value.abs(), accumulate=True)
        out.sub_(value[:, None] * p)
        size.add_(value.abs()[:, None] * p)

    if g is not None:
        named(targets, g)
    if ga is not None:
        for j in range(ids.shape[1]):
            named(ids[:, j], ga[:, j])
    if gl is not None:
        out += gl.double()[:, None] * p
        size += gl.double().abs()[:, None] * p
    if gH is not None:
        part = torch.where(p > 0, p * (lp + H), 0.0)
        out -= gH.double()[:, None] * part
        # ln p + H is formed from its parts
        size += gH.double().abs()[:, None] * torch.where(p > 0, p * (lp.abs() + 2 * H + 20), 0.0)
    # an exponential's argument d = (z - max) / T is rounded: |d| steps
    d = (z.double() - z.double().amax(1, keepdim=True)) / T
    size = size * (1 + torch.nan_to_num(d, nan=0.0, neginf=0.0).abs().clamp(max=200))
    return out / T, size / T


def distill(z, T, ids, x, tail):
    """loss, gradient and the sizes of the loss' and the gradient's terms."""
    lp, p = softmax(z, T)
    rows, V = z.shape
    loss, size = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    grad_, gsize = torch.zeros_like(p), torch.zeros_like(p)
    d = (z.double() - z.double().amax(1, keepdim=True)) / T
    far = 1 + torch.nan_to_num(d, nan=0.0, neginf=0.0).abs().clamp(max=200)
    for r in range(rows):
        keep, seen = [], set()
        for j in range(ids.shape[1]):
            v = int(ids[r, j])
            if v < 0 or v >= V or (tail and v in seen):
                continue
            seen.add(v)
            keep.append(j)
        if not keep:
            continue
        v = ids[r, keep].long()
        xs = x[r, keep].double()
        if tail:
            lq = xs
        else:
            if bool((xs == -math.inf).all()):
                continue
            lq = xs / T - torch.logsumexp(xs / T, 0)
        q = torch.exp(lq)
        rest = max(0.0, 1.0 - float(q.sum())) if tail else 0.0
        named = torch.zeros(V, dtype=torch.bool)
        named[v] = True
        if rest <= 2.0 ** -20 and not bool((lp[r][~named] > -math.inf).any()):
            rest = 0.0  # the rounding of the teacher's values, where the student has no other token
        there = q > 0
        loss[r] = (q[there] * (lq[there] - lp[r, v[there]])).sum()
        size[r] = (q[there] * (lq[there].abs() + torch.nan_to_num(lp[r, v[there]], neginf=0.0).abs() + 1)).sum()
        if bool((z[r] == -math.inf).all()):
            continue
        total = float(q.sum()) + rest
        grad_[r] = total * p[r]
        gsize[r] = total * p[r]
        grad_[r].index_put_((v,), -q, accumulate=True)
        gsize[r].index_put_((v,), q, accumulate=True)
        if tail and rest > 0:
            other = ~named
            if bool((lp[r][other] > -math.inf).any()):
                top = lp[r][other].amax()
                near = lp[r][other] - top  # (beside the type's lowest value the sum's logarithm would be lost)
                lt = top + torch.logsumexp(near, 0)
                within = torch.softmax(near, 0)
                loss[r] += rest * (math.log(rest) - lt)
                size[r] += rest * (abs(math.log(rest)) + lt.abs() + 1) + 4 * 2.0 ** -24 / SUM(V) * (lt.abs() + 20)
                share = rest * within
                grad_[r][other] -= share
                # the rest is 1 less a sum: off by a few steps of 1
                gsize[r][other] += share + within * 4 * 2.0 ** -24 / SUM(V)
            else:
                loss[r] = math.inf
    return loss, grad_ / T, size, gsize * far / T


def close(got, want, allowed, what=""):
    """Values that are finite in the kernels' type within `allowed`, others equal."""
    got, want = got.detach().cpu().double(), want.double()
    want = torch.where(want.abs() > torch.finfo(torch.float32).max, torch.sign(want) * math.inf, want)
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    other = ~fine & ~torch.isnan(want)
    assert torch.equal(got[other], want[other]), what
    over = ((got - want).abs() - allowed)[fine]
    assert not len(over) or float(over.max()) <= 0, f"{what}: over by {float(over.max()):.3e}"
