"""Log probabilities of given tokens, entropy and alternatives, and their gradient, against 64 bits (GPU)."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

SHAPES = [(1, 1, 1), (3, 2, 2), (5, 7, 7), (4, 8, 1), (9, 9, 5), (33, 127, 127), (6, 128, 128), (700, 255, 20),
          (2, 2047, 32), (3, 2049, 33), (11, 4099, 64), (1, 16385, 65), (2, 50257, 128), (40, 32001, 20), (1, 152064, 20),
          (5, 128256, 64)]
KINDS = ["normal", "ties", "equal", "ascending", "descending", "masked", "lowest", "sharp", "far"]


def _check(estp, ctx, z, T, k, targets, view=None):
    x = R.padded(z) if view is None else view
    lp = ctx.token_logprobs(x, targets.cuda(), top_k=k, temperature=T)
    ctx.sync_status()
    rows, V = z.shape
    ref, p = R.softmax(z, T)
    H = R.entropy(ref, p)
    ids = R.order(z, k)
    assert torch.equal(lp.top_ids.cpu().long(), ids)
    tol = R.SUM(V)
    at = torch.arange(rows)
    want = torch.where(targets < 0, 0.0, ref[at, targets.clamp(min=0).long()])
    big = lambda y: tol + 2.0 ** -22 * torch.nan_to_num(y, neginf=0.0).abs()  # noqa: E731
    R.close(lp.logprob, want, big(want), "logprob")
    top = torch.take_along_dim(ref, ids, 1)
    R.close(lp.top_logprobs, top, big(top), "top_logprobs")
    # ln s, and t with the error of the sums and of d, both relative to the entropy's parts
    R.close(lp.entropy, H, 2 * tol * (2 + H), "entropy")
    m = z.double().amax(1)
    R.close(lp.norm[:, 0], m, torch.zeros(rows), "max")
    s = torch.exp((z.double() - torch.where(m == -math.inf, 0.0, m)[:, None]) / T).sum(1)
    R.close(lp.norm[:, 1], s, s * tol, "sum")
    return lp


def _targets(rows, V, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (rows,), generator=g).int()
    t[::7] = -1
    t[1::7] = V - 1
    return t


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,V,k", SHAPES)
def test_shapes(cuda_lib, dtype, rows, V, k):
    z = R.logits("normal", rows, V, dtype, seed=rows + V)
    _check(cuda_lib, cuda_lib.Context(0), z, 1.0, k, _targets(rows, V, 1))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["normal", "ties", "masked", "equal"])
@pytest.mark.parametrize("rows,V,k", [(228, 4099, 9), (229, 4099, 9), (250, 30011, 70), (500, 9001, 20), (2500, 1500, 30), (4000, 77, 5)])
def test_rows_cut_in_every_way(cuda_lib, dtype, kind, rows, V, k):
    """Blocks a row, pieces of whole rows, equal pieces that begin and end inside rows, several rows a piece."""
    z = R.logits(kind, rows, V, dtype, seed=V + rows)
    _check(cuda_lib, cuda_lib.Context(0), z, 1.0, k, _targets(rows, V, 3))


@pytest.mark.parametrize("T", [1e-6, 1e-3, 1e4, 1e30])
def test_extreme_temperatures(cuda_lib, T):
    for kind in ("normal", "masked"):
        _check(cuda_lib, cuda_lib.Context(0), R.logits(kind, 9, 3001, F32), T, 8, _targets(9, 3001, 3))


def test_a_long_row(cuda_lib):
    """Two million logits: many blocks a row."""
    for rows in (1, 3):
        _check(cuda_lib, cuda_lib.Context(0), R.logits("normal", rows, (1 << 21) + 3, BF), 1.0, 20, _targets(rows, 1 << 21, 3))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,V,k,T", [(13, 300, 20, 0.5), (6, 5003, 100, 1.0), (2, 40001, 40, 3.0)])
def test_kinds(cuda_lib, dtype, kind, rows, V, k, T):
    z = R.logits(kind, rows, V, dtype, seed=V)
    _check(cuda_lib, cuda_lib.Context(0), z, T, k, _targets(rows, V, 2))


def test_without_alternatives_or_targets(cuda_lib):
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", 21, 3001, BF)
    x = R.padded(z, extra=3)
    a = ctx.token_logprobs(x, top_k=5)
    b = ctx.token_logprobs(x, _targets(21, 3001, 3).cuda())
    ctx.sync_status()
    assert a.logprob is None and b.top_ids is None and b.top_logprobs is None
    ref, p = R.softmax(z, 1.0)
    for lp in (a, b):  # (their sums are joined in another order)
        R.close(lp.entropy, R.entropy(ref, p), 2 * R.SUM(3001) * 10, "entropy")
    R.close(a.lse, torch.logsumexp(z.double(), 1), R.SUM(3001) + 2.0 ** -22 * 20, "lse")
    c = ctx.token_logprobs(x, top_k=3, V=1000)
    ref, p = R.softmax(z[:, :1000], 1.0)
    assert torch.equal(c.top_ids.cpu().long(), R.order(z[:, :1000], 3))
    R.close(c.entropy, R.entropy(ref, p), 2 * R.SUM(1000) * 8, "entropy of the first columns")


def test_no_rows(cuda_lib):
    ctx = cuda_lib.Context(0)
    x = torch.zeros(0, 64, dtype=BF, device="cuda")
    lp = ctx.token_logprobs(x, torch.zeros(0, dtype=torch.int32, device="cuda"), top_k=4)
    assert lp.logprob.shape == (0,) and lp.top_ids.shape == (0, 4)
    assert ctx.token_logprobs_grad(x, None, lp).shape == (0, 64)
    ctx.sync_status()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("V", [77, 20000])
def test_rows_with_nan_or_infinity(cuda_lib, dtype, bad, V):
    """Such a row gives NaN and no alternatives; its neighbours are as they were."""
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", 6, V, dtype)
    clean = ctx.token_logprobs(R.padded(z), _targets(6, V, 5).cuda(), top_k=9)
    y = z.clone()
    y[1, 3] = bad
    y[4, V - 1] = bad
    y[5, :] = bad
    got = ctx.token_logprobs(R.padded(y), _targets(6, V, 5).cuda(), top_k=9)
    ctx.sync_status()
    for r in range(6):
        for name in ("logprob", "entropy", "top_logprobs"):
            a, b = getattr(clean, name)[r], getattr(got, name)[r]
            if r in (1, 4, 5):
                assert bool(torch.isnan(b).all()) or (name == "logprob" and _targets(6, V, 5)[r] < 0)
            else:
                assert torch.equal(a, b)
        assert torch.equal(got.top_ids[r], clean.top_ids[r] if r not in (1, 4, 5) else torch.full_like(clean.top_ids[r], -1))
        assert bool(torch.isnan(got.norm[r, 1])) == (r in (1, 4, 5))


def test_a_target_past_the_vocabulary(cuda_lib):
    ctx = cuda_lib.Context(0)
    x = R.padded(R.logits("normal", 4, 100, F32))
    t = torch.tensor([3, 100, -5, 2 ** 30], dtype=torch.int32, device="cuda")
    lp = ctx.token_logprobs(x, t)
    with pytest.raises(cuda_lib.EstpError) as e:
        ctx.sync_status()
    assert e.value.status == cuda_lib.ESTP_ERR_INVALID_ARG
    got = lp.logprob.cpu()
    assert math.isnan(got[1]) and math.isnan(got[3]) and got[2] == 0 and got[0] < 0
    out = ctx.token_logprobs_grad(x, t, lp, grad_logprob=torch.ones(4, device="cuda"))
    with pytest.raises(cuda_lib.EstpError):
        ctx.sync_status()
    assert not out[1].any() and not out[2].any() and not out[3].any() and out[0].any()


# ------------------------------------------------------------------------ gradient
def _grad_check(ctx, z, T, k, which, seed=0, duplicate=False):
    rows, V = z.shape
    g = torch.Generator().manual_seed(seed)
    x = R.padded(z)
    t = _targets(rows, V, 4)
    lp = ctx.token_logprobs(x, t.cuda(), top_k=k, temperature=T)
    ids = None
    if k:
        if duplicate:  # the same alternatives again, none, and the target among them
            lp.top_ids[:, k // 2:] = lp.top_ids[:, : k - k // 2]
            lp.top_ids[::2, 0] = -1
            lp.top_ids[1::2, 0] = t.cuda()[1::2].clamp(min=0)
        ids = lp.top_ids.cpu()
    up = {n: torch.randn(rows, generator=g) if n in which else None for n in ("logprob", "entropy", "lse")}
    top = torch.randn(rows, k, generator=g) if k and "top" in which else None
    dev = lambda y: None if y is None else y.cuda()  # noqa: E731
    out = ctx.token_logprobs_grad(x, t.cuda(), lp, grad_logprob=dev(up["logprob"]), grad_entropy=dev(up["entropy"]),
                                  grad_lse=dev(up["lse"]), grad_top=dev(top))
    ctx.sync_status()
    want, size = R.grad(z, T, t, ids, up["logprob"], up["entropy"], up["lse"], top)
    R.close(out, want, (2 * R.SUM(V) + 2.0 ** -21) * size + R.HALF[z.dtype] * want.abs() + 1e-37, "gradient")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,V,k", [(1, 1, 1), (5, 7, 3), (9, 9, 9), (300, 255, 20), (3, 8191, 64), (2, 8193, 128), (3, 40961, 5),
                                      (1, 152064, 20)])
def test_gradient_shapes(cuda_lib, dtype, rows, V, k):
    _grad_check(cuda_lib.Context(0), R.logits("normal", rows, V, dtype, seed=V), 1.0, k, ("logprob", "entropy", "lse", "top"))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["ties", "equal", "masked", "lowest", "sharp", "far"])
@pytest.mark.parametrize("T", [0.6, 2.0])
def test_gradient_kinds(cuda_lib, dtype, kind, T):
    _grad_check(cuda_lib.Context(0), R.logits(kind, 14, 1003, dtype), T, 12, ("logprob", "entropy", "top"))


@pytest.mark.parametrize("which", [("logprob",), ("entropy",), ("lse",), ("top",), ()])
def test_gradient_of_one_output(cuda_lib, which):
    _grad_check(cuda_lib.Context(0), R.logits("normal", 8, 2000, F32), 1.0, 6, which)


@pytest.mark.parametrize("k", [2, 40, 128])
def test_gradient_of_repeated_alternatives(cuda_lib, k):
    _grad_check(cuda_lib.Context(0), R.logits("normal", 9, 5001, F32), 1.0, k, ("logprob", "top"), duplicate=True)


def test_gradient_agrees_with_differences(cuda_lib):
    """Against central differences of the 64-bit definition: step 1e-5, their error about 1e-9."""
    ctx, rows, V, k, T = cuda_lib.Context(0), 2, 37, 4, 0.7
    z = R.logits("normal", rows, V, F32, seed=8)
    t = torch.tensor([5, 36], dtype=torch.int32)
    g = torch.Generator().manual_seed(1)
    up = [torch.randn(rows, generator=g) for _ in range(3)]
    top = torch.randn(rows, k, generator=g)
    x = R.padded(z)
    lp = ctx.token_logprobs(x, t.cuda(), top_k=k, temperature=T)
    out = ctx.token_logprobs_grad(x, t.cuda(), lp, up[0].cuda(), up[1].cuda(), up[2].cuda(), top.cuda()).cpu().double()
    ids = lp.top_ids.cpu().long()

    def value(y):
        ref, p = R.softmax(y, T)
        return (up[0].double() * ref[torch.arange(rows), t.long()] + up[1].double() * R.entropy(ref, p)
                + up[2].double() * torch.logsumexp(y / T, 1) + (top.double() * torch.take_along_dim(ref, ids, 1)).sum(1))

    for v in range(V):
        step = torch.zeros(rows, V, dtype=torch.float64)
        step[:, v] = 1e-5
        slope = (value(z.double() + step) - value(z.double() - step)) / 2e-5
        assert torch.allclose(out[:, v], slope, rtol=1e-5, atol=2e-6)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_gradient_in_place_leaves_the_padding(cuda_lib, dtype):
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", 30, 5005, dtype)
    x = R.padded(z, extra=2, fill=7.0)
    t = _targets(30, 5005, 6).cuda()
    lp = ctx.token_logprobs(x, t, top_k=10)
    g, a = torch.randn(30, device="cuda"), torch.randn(30, 10, device="cuda")
    want = ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, grad_entropy=g, grad_top=a)
    assert want.shape == (30, 5005) and want.stride(0) * want.element_size() % 16 == 0
    wide = torch.full((30, 5016), 3.0, dtype=dtype, device="cuda")
    ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, grad_entropy=g, grad_top=a, out=wide)
    assert torch.equal(wide[:, :5005], want) and bool((wide[:, 5005:] == 3).all())
    got = ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, grad_entropy=g, grad_top=a, out=x)
    ctx.sync_status()
    assert got is x and torch.equal(x, want)
    base = x._base
    assert bool((base[:, 5005:] == 7).all())


def test_rows_without_weight_get_zeros(cuda_lib):
    """A padding row, NaN in it or not, adds nothing to a gradient."""
    ctx = cuda_lib.Context(0)
    z = R.logits("normal", 5, 900, BF)
    z[1] = math.nan
    z[3, 7] = math.inf
    t = torch.tensor([1, -1, 2, -1, -1], dtype=torch.int32, device="cuda")
    x = R.padded(z)
    lp = ctx.token_logprobs(x, t)
    out = ctx.token_logprobs_grad(x, t, lp, grad_logprob=torch.ones(5, device="cuda"))
    ctx.sync_status()
    assert not out[1].any() and not out[3].any() and not out[4].any()
    assert torch.isfinite(out).all() and out[0].any() and out[2].any()


def test_repeated_calls_give_the_same_bits(cuda_lib):
    ctx = cuda_lib.Context(0)
    x = R.padded(R.logits("ties", 50, 30000, BF))
    t = _targets(50, 30000, 1).cuda()
    a = ctx.token_logprobs(x, t, top_k=50)
    ga = ctx.token_logprobs_grad(x, t, a, grad_logprob=a.entropy, grad_top=a.top_logprobs)
    for _ in range(3):
        b = ctx.token_logprobs(x, t, top_k=50)
        for n in ("logprob", "entropy", "norm", "top_ids", "top_logprobs"):
            assert torch.equal(getattr(a, n), getattr(b, n)), n
        assert torch.equal(ga, ctx.token_logprobs_grad(x, t, b, grad_logprob=b.entropy, grad_top=b.top_logprobs))


def test_rows_past_32_bit_offsets(cuda_lib):
    """The last rows of logits of more than 2^32 bytes."""
    ctx = cuda_lib.Context(0)
    rows, V = 17000, 128256
    x = torch.zeros(rows, V, dtype=BF, device="cuda")
    z = R.logits("normal", 3, V, BF)
    x[-3:] = z.cuda()
    t = torch.zeros(rows, dtype=torch.int32, device="cuda")
    t[-3:] = torch.tensor([7, V - 1, 0], dtype=torch.int32)
    lp = ctx.token_logprobs(x, t, top_k=4)
    want = _check(cuda_lib, ctx, z, 1.0, 4, t[-3:].cpu())
    R.close(lp.logprob[-3:], want.logprob.cpu(), 2 * R.SUM(V), "last rows")
    assert torch.equal(lp.top_ids[-3:], want.top_ids)
    assert torch.equal(lp.top_ids[: rows - 3].cpu(), torch.arange(4, dtype=torch.int32).expand(rows - 3, 4))
    g = torch.zeros(rows, device="cuda")
    g[-1] = 1.0
    ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, out=x)
    ctx.sync_status()
    ref, size = R.grad(z[-1:], 1.0, t[-1:].cpu(), None, torch.ones(1), None, None, None)
    R.close(x[-1:], ref, (2 * R.SUM(V) + 2.0 ** -21) * size + 2.0 ** -8 * ref.abs() + 1e-37, "last row's gradient")
    assert not x[:-1].any()
