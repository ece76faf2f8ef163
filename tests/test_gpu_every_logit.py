"""Every logit of a row counts, and once: rows of 0 and -inf, whose exponentials are 1 and 0 and whose sums are whole numbers
below 2^24, so that fp32 holds them exactly and a single 16-byte unit left out or read twice shows (GPU)."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
LENGTHS = [(1, 152064), (3, (1 << 21) + 3), (40, 128256), (61, 50257), (228, 9001), (229, 9001), (500, 152064), (1000, 30011), (2500, 1500),
           (9000, 257)]


def _rows(rows, V, dtype, masked, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.zeros(rows, V, dtype=dtype, device="cuda")
    if masked:
        z.masked_fill_(torch.rand(rows, V, generator=g, device="cuda") < 0.4, -math.inf)
        z[:, 0] = 0
    return R.padded(z, fill=0.0), (z == 0)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("masked", [False, True], ids=["whole", "masked"])
@pytest.mark.parametrize("rows,V", LENGTHS)
def test_sums_are_counts(cuda_lib, dtype, masked, rows, V):
    ctx = cuda_lib.Context(0)
    z, here = _rows(rows, V, dtype, masked, V)
    count = here.sum(1)
    ln = count.double().log()
    t = torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(1)).int().cuda()
    k = min(V, 33)
    # the first k that are not masked
    first = torch.where(here, torch.arange(V, device="cuda"), V).sort(1).values[:, :k]
    assert bool((first < V).all())
    for top in (0, k):
        lp = ctx.token_logprobs(z, t, top_k=top, temperature=0.75)
        ctx.sync_status()
        assert torch.equal(lp.norm[:, 0], torch.zeros(rows, device="cuda"))
        assert not int((lp.norm[:, 1].long() != count).sum()) and not int((lp.norm[:, 1].frac() != 0).sum())
        # a logarithm, off by a unit of the last place
        assert float(((lp.entropy.double() - ln).abs() - 2.0 ** -22 * ln).max()) <= 0
        want = torch.where(here.gather(1, t[:, None].long())[:, 0], -ln, -math.inf)
        R.close(lp.logprob, want.cpu(), 2.0 ** -22 * ln.cpu())
        if top:
            assert not int((lp.top_ids != first).sum())
            R.close(lp.top_logprobs, -ln[:, None].expand(rows, k).cpu(), 2.0 ** -22 * ln[:, None].cpu())
        # every element of the gradient is written: p = 1 / count where there is a token
        g = torch.full((rows,), 3.0, device="cuda")
        out = torch.full((rows, V + -V % 8), 9.0, dtype=dtype, device="cuda")
        ctx.token_logprobs_grad(z, None, lp, grad_lse=g, out=out)
        ctx.sync_status()
        value = (3 / 0.75 / count.double())[:, None]
        for r in range(0, rows, 100):
            s = slice(r, r + 100)
            want = torch.where(here[s], value[s], 0.0)
            assert float(((out[s, :V].double() - want).abs() - (R.HALF[dtype] + 2.0 ** -21) * want).max()) <= 0
        assert bool((out[:, V:] == 9).all())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("masked", [False, True], ids=["whole", "masked"])
@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("rows,V,K", [(1, 152064, 40), (40, 128256, 8), (500, 152064, 20), (600, 30011, 70), (2500, 1500, 30), (9000, 257, 5),
                                      (4, 409700, 12), (300, 98304, 33)])
def test_losses_are_logarithms_of_counts(cuda_lib, dtype, masked, tail, rows, V, K):
    """The teacher's K tokens have 1 / K each, of 1 or of 0.75.  What is off: q by two units of its last place (2^-22 relative; 1 / K
    by a rounding), ln q by one, and where a rest is 1 less their sum, that too; the sums are exact, and what follows
    them is formed in two floats.  A unit left out would change the loss by Q of its share of the count."""
    ctx, T = cuda_lib.Context(0), 1.25
    z, here = _rows(rows, V, dtype, masked, V + K)
    g = torch.Generator(device="cuda").manual_seed(K)
    step = V // K
    ids = torch.randint(0, step, (rows, K), generator=g, device="cuda") + step * torch.arange(K, device="cuda")
    z.scatter_(1, ids, 0.0)
    here.scatter_(1, ids, True)
    count = here.sum(1).double()
    x = torch.full((rows, K), math.log(0.75 / K) if tail else 2.5, device="cuda")
    lq = x.double() if tail else torch.full_like(x, -math.log(K), dtype=torch.float64)
    q = lq.exp()
    Q = q.sum(1)
    rest = 1 - Q if tail else torch.zeros(rows, device="cuda")
    ln = count.log()
    want = (q * lq).sum(1) + Q * ln
    size = Q * (lq.abs() + (lq + ln[:, None]).abs()).amax(1)
    if tail:
        other = ((count - K) / count).log()
        want = want + rest * (rest.log() - other)
        size = size + Q * ((rest.log() - other).abs() + 1)
    allowed = 2.0 ** -22 * size + 2.0 ** -24 * want.abs()
    assert float((allowed - Q * (16 // z.element_size()) / count).max()) < 0
    alone = ctx.distill_loss(z, ids.int(), x, temperature=T, tail=tail, grads=False)
    out = torch.full((rows, V + -V % 8), 9.0, dtype=dtype, device="cuda")
    loss, _ = ctx.distill_loss(z, ids.int(), x, temperature=T, tail=tail, out=out)
    ctx.sync_status()
    for got in (loss, alone):
        assert float(((got.double() - want).abs() - allowed).max()) <= 0
    for r in range(0, rows, 100):
        s = slice(r, r + 100)
        p = torch.where(here[s], 1 / count[s, None], 0.0)
        spread = (rest[s] / (count[s] - K)).double()[:, None] if tail else 0.0
        grad = (p - torch.where(here[s], spread, 0.0)).scatter(1, ids[s], p.gather(1, ids[s]) - q[s]) / T
        size = (p + torch.where(here[s], spread, 0.0)).scatter(1, ids[s], p.gather(1, ids[s]) + q[s]) / T
        off = (out[s, :V].double() - grad).abs() - R.HALF[dtype] * grad.abs() - 2.0 ** -20 * size
        assert float(off.max()) <= 0
    assert bool((out[:, V:] == 9).all())
