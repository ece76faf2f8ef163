"""Attention over a paged KV cache against its definition in 64 bits (GPU).

Tolerances.  A score q.k of d products in fp32 is off by at most d 2^-24 sum |q_i k_i|, for
N(0,1) entries (sum about 0.64 d) and scale d^-1/2 below e_s = 0.64 d^1.5 2^-24: 6e-5 at d = 128.
A probability is then off by the factor e^(2 e_s), and ex2 and the sums add some 2^-20:
1.3e-4 relative in the worst case, 10 times less as products round to both sides.
  lse      |err| <= e_s + 2^-20 |lse|, taken as 2e-5 + 2e-6 |lse| (two scores in a hundred thousand)
  weights  2e-4 relative to what the slot received, plus fp32 rounding of the sum it is added to
  out      bf16: half an ulp of the result, 2^-8 |o|, and 2e-4 max |v|; fp32: 2e-4 max |v|
"""
import math

import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _check(estp, ctx, cache, Q, kn, vn, counts, sees, use_tree=True, row_weight=None, accumulate=True, scale=None):
    d, Hkv = cache.head_dim, cache.Hkv
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    scale = 1 / math.sqrt(d) if scale is None else scale
    ref_o, ref_lse, ref_wn, gave = R.attention(cache, Q, kn, vn, cu, scale, sees, row_weight)
    before, was = cache.weight.clone(), [x.clone() for x in (cache.k, cache.v, cache.position, cache.length)]
    words = -(-max(max(counts), 1) // 64)
    out, lse, wn = ctx.cache_attention(cache, Q, kn, vn, torch.from_numpy(cu).cuda(), max(counts), scale=scale,
                                       tree_mask=R.bits_of(sees, words) if use_tree else None,
                                       row_weight=row_weight, accumulate=accumulate, details=True)
    ctx.sync_status()
    o, l = R.host(out), R.host(lse)
    v_new = np.zeros(1) if vn is None else R.host(vn)
    vmax = max([float(np.abs(v_new[np.isfinite(v_new)]).max())]
               + [float(np.abs(R.host(cache.v)[R.slots(cache, b, T)]).max()) for b, T in enumerate(cache.length.tolist()) if T])
    ok = np.isfinite(ref_o)
    assert np.array_equal(np.isfinite(o), ok)
    tol = 2e-4 * vmax + (2.0 ** -8 * np.abs(ref_o[ok]) if cache.dtype == BF else 0)
    assert np.all(np.abs(o[ok] - ref_o[ok]) <= tol), np.abs(o[ok] - ref_o[ok]).max()
    none = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(l), none)
    fine = np.isfinite(ref_lse)
    assert np.all(np.abs(l[fine] - ref_lse[fine]) <= 2e-5 + 2e-6 * np.abs(ref_lse[fine]))
    assert np.all(o[none.T] == 0)
    if wn is not None:
        ok = np.isfinite(ref_wn)
        assert np.all(np.abs(R.host(wn)[ok] - ref_wn[ok]) <= 2e-4 * np.abs(ref_wn[ok]) + 1e-9)
    for b, T in enumerate(cache.length.tolist()):
        pg, of = R.slots(cache, b, T)
        for g in range(Hkv):
            old, new = R.host(before)[pg, g, of], R.host(cache.weight)[pg, g, of]
            want = old + (gave[b][:, g] if accumulate else 0)
            ok = np.isfinite(want)
            assert np.all(np.abs(new[ok] - want[ok]) <= 2e-4 * gave[b][ok, g] + 2.0 ** -23 * np.abs(want[ok]) + 1e-9)
    # nothing else is written
    used = torch.zeros_like(cache.weight, dtype=torch.bool)
    for b, T in enumerate(cache.length.tolist()):
        pg, of = R.slots(cache, b, T)
        used[torch.from_numpy(pg).long().cuda(), :, torch.from_numpy(of).cuda()] = True
    assert torch.equal(cache.weight[~used].isnan(), before[~used].isnan())
    for x, y in zip((cache.k, cache.v, cache.position, cache.length), was):
        assert torch.equal(x.nan_to_num(), y.nan_to_num())
    return out, lse, wn


def _rows(rng, n, heads, d, dtype):
    return torch.from_numpy(rng.standard_normal((n, heads, d))).to(dtype).cuda()


CASES = [
    # lens, counts, Hq, Hkv, d, page
    ([1], [1], 1, 1, 64, 8),
    ([0], [1], 8, 2, 128, 16),
    ([127], [1], 28, 4, 128, 16),
    ([128], [1], 8, 8, 64, 128),
    ([129], [2], 32, 8, 128, 64),
    ([5, 0, 300, 257], [1, 1, 1, 1], 8, 8, 128, 32),
    ([40, 700, 0, 1025], [3, 1, 4, 0], 14, 2, 64, 16),
    ([1000, 3], [17, 9], 16, 2, 128, 256),
    ([260, 90], [64, 33], 14, 2, 128, 16),
    ([100], [128], 4, 1, 64, 8),
    ([2500], [128], 8, 1, 128, 512),
    ([33, 520], [5, 128], 8, 1, 64, 32),
    ([777], [4], 64, 1, 128, 16),
    ([4000], [1], 7, 1, 128, 8),
    # many tiles a CTA in every kernel: several turns of the rings, several sequences a CTA
    ([9000, 12000, 700, 8000], [1, 1, 1, 1], 64, 16, 128, 64),
    ([9000, 7000, 500, 8000], [3, 4, 1, 4], 64, 16, 128, 128),
    ([9000, 7000, 500, 8000], [7, 8, 5, 8], 64, 16, 128, 64),
    ([9000, 7000, 500, 8000], [7, 8, 5, 8], 64, 16, 64, 32),
    ([5000, 4000, 500, 3000], [30, 20, 9, 17], 64, 16, 128, 64),
    ([5000, 4000, 500, 3000], [70, 40, 9, 100], 32, 8, 128, 64),
    ([5000, 4000, 500, 3000], [70, 40, 9, 100], 32, 8, 64, 16),
    # more sequences than a warp has lanes
    ([37 * i % 300 for i in range(70)], [1 - (i % 9 == 4) for i in range(70)], 12, 3, 64, 16),
    ([53 * i % 700 for i in range(40)], [i % 6 for i in range(40)], 12, 3, 128, 32),
    ([71 * i % 400 for i in range(36)], [i * 5 % 41 for i in range(36)], 8, 2, 128, 64),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,counts,Hq,Hkv,d,page", CASES)
def test_matches_definition(cuda_lib, lens, counts, Hq, Hkv, d, page, dtype):
    rng = np.random.default_rng(sum(lens) + Hq * d)
    ctx = cuda_lib.Context(0)
    cache = R.make_cache(cuda_lib, rng, lens, Hkv, d, page, dtype)
    n = sum(counts)
    Q, kn, vn = _rows(rng, n, Hq, d, dtype), _rows(rng, n, Hkv, d, dtype), _rows(rng, n, Hkv, d, dtype)
    sees = [R.tree(rng, c) for c in counts]
    c = torch.from_numpy(rng.uniform(0, 1, n).astype(np.float32)).cuda()
    c[::3] = 0  # rows that do not count
    _check(cuda_lib, ctx, cache, Q, kn, vn, counts, sees, row_weight=c)
    # a chain without a mask, every row counted
    chain = [np.tril(np.ones((m, m), bool)) for m in counts]
    _check(cuda_lib, ctx, cache, Q, kn, vn, counts, chain, use_tree=False)
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_nothing(cuda_lib, dtype, d):
    rng = np.random.default_rng(d)
    ctx = cuda_lib.Context(0)
    cache = R.make_cache(cuda_lib, rng, [0, 30, 0], 2, d, 16, dtype)
    counts = [5, 2, 3]
    Q, kn, vn = _rows(rng, 10, 6, d, dtype), _rows(rng, 10, 2, d, dtype), _rows(rng, 10, 2, d, dtype)
    sees = [R.tree(rng, c) for c in counts]
    sees[0][1] = False  # not even itself
    sees[0][:, 1] = False
    sees[1][0] = False  # the cache only
    sees[2][:] = False
    _check(cuda_lib, ctx, cache, Q, kn, vn, counts, sees)
    # without drafts of their own: a sequence without slots gives zeros
    out, lse, wn = _check(cuda_lib, ctx, cache, Q, None, None, counts, sees, use_tree=False)
    assert wn is None
    assert torch.all(out[:5] == 0) and torch.all(lse[:, 7:] == -math.inf)
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_hidden_drafts_hold_anything(cuda_lib, dtype, bad):
    """K and V of a hidden draft do not reach the rows that do not see it; rows that do see it get
    what the definition gives."""
    rng = np.random.default_rng(5)
    ctx = cuda_lib.Context(0)
    counts = [6, 40]
    cache = R.make_cache(cuda_lib, rng, [20, 150], 2, 128, 16, dtype)
    n = sum(counts)
    Q, kn, vn = _rows(rng, n, 8, 128, dtype), _rows(rng, n, 2, 128, dtype), _rows(rng, n, 2, 128, dtype)
    sees = [R.tree(rng, c) for c in counts]
    for b, j in ((0, 3), (1, 17)):
        sees[b][:, j] = False  # no row sees it, nor it itself
        at = j + (6 if b else 0)
        kn[at], vn[at] = bad, bad
    _check(cuda_lib, ctx, cache, Q, kn, vn, counts, sees)
    vn[6 + 39, 1, 5] = bad  # the last draft's own V: its row alone sees it
    with np.errstate(invalid="ignore"):
        out, _, _ = _check(cuda_lib, ctx, cache, Q, kn, vn, counts, sees)
    assert torch.isfinite(out[: 6 + 39]).all() and not torch.isfinite(out[6 + 39, 4:, 5]).any()
    assert torch.isfinite(out[6 + 39, 4:, 6]).all() and torch.isfinite(out[6 + 39, :4]).all()
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 12, 70])
def test_strided_inputs(cuda_lib, dtype, n):
    """Head-major pages, and rows that are slices of a fused projection."""
    rng = np.random.default_rng(n)
    ctx = cuda_lib.Context(0)
    d, Hq, Hkv = 128, 6, 3
    cache = R.make_cache(cuda_lib, rng, [300, 77], Hkv, d, 32, dtype, head_major=True)
    fused = _rows(rng, 2 * n, Hq + 2 * Hkv, d, dtype)
    Q, kn, vn = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    _check(cuda_lib, ctx, cache, Q, kn, vn, [n, n], [R.tree(rng, n), R.tree(rng, n)])
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [6.0, 40.0])
def test_peaked_scores(cuda_lib, dtype, size):
    """Scores far apart (one key takes nearly all), growing along the cache so that the running
    maximum moves on in every tile.  Scores up to some 500 carry an fp32 error of 500 2^-22."""
    rng = np.random.default_rng(int(size))
    ctx = cuda_lib.Context(0)
    cache = R.make_cache(cuda_lib, rng, [900], 2, 64, 16, dtype)
    pg, of = R.slots(cache, 0, 900)
    grow = torch.linspace(0, size, 900, device="cuda").to(dtype)
    ids = torch.from_numpy(pg).long().cuda(), torch.from_numpy(of).cuda()
    base = cache.k[ids][:1]
    cache.k[ids] = (cache.k[ids].float() * 0.1 + base.float() * grow[:, None, None].float()).to(dtype)
    Q = (base[0][:, None].float().expand(2, 4, 64).reshape(1, 8, 64) * 1.0).to(dtype)
    kn, vn = _rows(rng, 1, 2, 64, dtype), _rows(rng, 1, 2, 64, dtype)
    cu = np.array([0, 1], np.int32)
    ref_o, ref_lse, _, gave = R.attention(cache, Q, kn, vn, cu, 0.125, [np.ones((1, 1), bool)])
    before = R.host(cache.weight)
    out, lse, _ = ctx.cache_attention(cache, Q, kn, vn, torch.from_numpy(cu).cuda(), 1, scale=0.125, accumulate=True, details=True)
    ctx.sync_status()
    top = float(np.abs(ref_lse).max())
    e = 4e-4 + top * 2.0 ** -20  # of a probability
    assert np.all(np.abs(R.host(lse) - ref_lse) <= 2e-5 + 2e-6 * np.abs(ref_lse))
    assert np.all(np.abs(R.host(out) - ref_o) <= e * 4 + (2.0 ** -8 * np.abs(ref_o) if dtype == BF else 0))
    got = R.host(cache.weight)[pg, :, of] - before[pg, :, of]
    assert np.all(np.abs(got - gave[0]) <= e * gave[0] + 2.0 ** -22 * (before[pg, :, of] + gave[0]) + 1e-9)
    ctx.close()


@pytest.mark.parametrize("n", [1, 24])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_same_bits_on_another_stream_and_in_a_graph(cuda_lib, dtype, n):
    rng = np.random.default_rng(n)
    ctx = cuda_lib.Context(0)
    cache = R.make_cache(cuda_lib, rng, [1500, 333, 64], 4, 128, 64, dtype)
    counts = [n, 1, n]
    rows = sum(counts)
    Q, kn, vn = _rows(rng, rows, 28, 128, dtype), _rows(rng, rows, 4, 128, dtype), _rows(rng, rows, 4, 128, dtype)
    cu = torch.tensor([0, n, n + 1, 2 * n + 1], dtype=torch.int32, device="cuda")
    w0 = cache.weight.clone()

    def call(out=None):
        return ctx.cache_attention(cache, Q, kn, vn, cu, n, accumulate=True, out=out)

    ref = call()
    torch.cuda.synchronize()
    w1 = cache.weight.clone()
    side = torch.cuda.Stream()
    cache.weight.copy_(w0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = call()
    side.synchronize()
    assert torch.equal(again, ref) and torch.equal(cache.weight.nan_to_num(), w1.nan_to_num())
    out = torch.empty_like(ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out)
    for _ in range(2):
        out.fill_(float("nan"))
        cache.weight.copy_(w0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(cache.weight.nan_to_num(), w1.nan_to_num())
    ctx.sync_status()
    del g
    ctx.close()


def test_shared_pages_without_weights(cuda_lib):
    """Two sequences read one prefix: the same pages in both tables."""
    rng = np.random.default_rng(9)
    ctx = cuda_lib.Context(0)
    base = R.make_cache(cuda_lib, rng, [200], 2, 128, 32, BF)
    table = base.page_table.expand(2, -1).contiguous()
    length = torch.tensor([200, 70], dtype=torch.int32, device="cuda")
    cache = cuda_lib.KVCache(base.k, base.v, table, length, length.clone())
    assert cache.max_slots == 2 * table.shape[1] * 32
    Q, kn, vn = _rows(rng, 2, 4, 128, BF), _rows(rng, 2, 2, 128, BF), _rows(rng, 2, 2, 128, BF)
    ref, _, _, _ = R.attention(cache, Q, kn, vn, [0, 1, 2], 128 ** -0.5, [np.ones((1, 1), bool)] * 2)
    out = ctx.cache_attention(cache, Q, kn, vn, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), 1)
    ctx.sync_status()
    assert np.all(np.abs(R.host(out) - ref) <= 2.0 ** -8 * np.abs(ref) + 2e-4 * 5)
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_offsets_past_32_bits(cuda_lib, dtype):
    """A pool whose K has more than 2^32 bytes and 2^31 elements: its last pages are used."""
    rng = np.random.default_rng(1)
    ctx = cuda_lib.Context(0)
    page, Hkv, d = 256, 8, 128
    n_pages = (1 << 31) // (page * Hkv * d) + 8
    k = torch.zeros(n_pages, page, Hkv, d, dtype=dtype, device="cuda")
    v = torch.zeros_like(k)
    weight = torch.zeros(n_pages, Hkv, page, device="cuda")
    ids = [n_pages - 1, 0, n_pages - 3]
    for i in ids:
        k[i], v[i] = torch.randn(page, Hkv, d, device="cuda").to(dtype), torch.randn(page, Hkv, d, device="cuda").to(dtype)
    length = torch.tensor([600], dtype=torch.int32, device="cuda")
    small = cuda_lib.KVCache(k[ids].contiguous(), v[ids].contiguous(), torch.arange(3, dtype=torch.int32, device="cuda")[None],
                             length, length.clone(), torch.zeros(3, Hkv, page, device="cuda"))
    big = cuda_lib.KVCache(k, v, torch.tensor([ids], dtype=torch.int32, device="cuda"), length, length.clone(), weight, max_slots=600)
    Q, kn, vn = _rows(rng, 1, 8, d, dtype), _rows(rng, 1, 8, d, dtype), _rows(rng, 1, 8, d, dtype)
    cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    a = ctx.cache_attention(small, Q, kn, vn, cu, 1, accumulate=True)
    b = ctx.cache_attention(big, Q, kn, vn, cu, 1, accumulate=True)
    ctx.sync_status()
    assert torch.equal(a, b) and torch.equal(small.weight, weight[ids])
    assert a.abs().max() > 0
    ctx.close()


def test_lengths_the_device_refuses(cuda_lib):
    """Lengths, row counts and pages that do not fit are recorded, and nothing is written."""
    estp = cuda_lib
    rng = np.random.default_rng(2)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, [50, 20], 2, 64, 16, BF)
    Q, kn, vn = _rows(rng, 2, 4, 64, BF), _rows(rng, 2, 2, 64, BF), _rows(rng, 2, 2, 64, BF)
    good = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    w0 = cache.weight.clone()

    def refused(cu=good, most=1):
        ctx.cache_attention(cache, Q, kn, vn, cu, most, accumulate=True)
        with pytest.raises(estp.EstpError) as e:
            ctx.sync_status()
        assert e.value.status == estp.ESTP_ERR_INVALID_ARG

    for cu in ([0, 2, 2], [0, 2, 1], [1, 1, 2], [0, 1, 1]):
        refused(torch.tensor(cu, dtype=torch.int32, device="cuda"))
    for bad in (-1, 10 ** 6):
        cache.length[1] = bad
        refused()
    cache.length[1] = 20
    cache.max_slots = 69
    refused()
    cache.max_slots = 70
    ctx.cache_attention(cache, Q, kn, vn, good, 1)
    ctx.sync_status()
    assert torch.equal(w0.nan_to_num(), cache.weight.nan_to_num())
    was = cache.page_table.clone()
    for bad in (-1, cache.k.shape[0]):
        cache.page_table[0, 1] = bad
        refused()
    cache.page_table.copy_(was)
    ctx.close()


def test_refusals(cuda_lib):
    estp = cuda_lib
    rng = np.random.default_rng(2)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, [50, 20], 2, 64, 16, BF)
    Q, kn, vn = _rows(rng, 2, 4, 64, BF), _rows(rng, 2, 2, 64, BF), _rows(rng, 2, 2, 64, BF)
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")

    def status(f):
        with pytest.raises(estp.EstpError) as e:
            f()
        return e.value.status

    bad, no = estp.ESTP_ERR_INVALID_ARG, estp.ESTP_ERR_UNSUPPORTED
    call = ctx.cache_attention
    assert status(lambda: call(cache, Q, kn, vn, cu, 3)) == bad                       # more than the rows
    assert status(lambda: call(cache, Q, kn, vn, cu, 0)) == bad
    assert status(lambda: call(cache, Q, kn, vn, cu, 1, scale=0.0)) == bad
    assert status(lambda: call(cache, Q, kn, vn, cu, 1, scale=math.inf)) == bad
    assert status(lambda: call(cache, Q[:, :3], kn, vn, cu, 1)) == bad                # 3 heads over 2
    big = _rows(rng, 200, 4, 64, BF)
    assert status(lambda: call(cache, big, None, None, cu, 129)) == no
    wide = _rows(rng, 100, 64, 64, BF)
    assert status(lambda: call(cache, wide, None, None, cu, 33)) == no                # 33 x 32 query heads
    bare = estp.KVCache(cache.k, cache.v, cache.page_table, cache.length, cache.seen)
    assert status(lambda: call(bare, Q, kn, vn, cu, 1, accumulate=True)) == bad
    assert status(lambda: call(cache, big, None, None, cu, 65, tree_mask=torch.zeros(200, 1, dtype=torch.int64, device="cuda"))) == bad
    for f in (lambda: call(cache, Q.float(), kn, vn, cu, 1), lambda: call(cache, Q, kn[:1], vn[:1], cu, 1),
              lambda: call(cache, Q, kn, vn, cu[:2], 1), lambda: call(cache, Q, kn, vn, cu.long(), 1),
              lambda: call(cache, Q, kn, vn, cu, 1, row_weight=torch.ones(3, device="cuda")),
              lambda: call(cache, Q, kn, vn, cu, 1, tree_mask=torch.zeros(3, 1, dtype=torch.int64, device="cuda")),
              lambda: estp.KVCache(cache.k, cache.v[:1], cache.page_table, cache.length, cache.seen),
              lambda: estp.KVCache(cache.k, cache.v, cache.page_table.long(), cache.length, cache.seen),
              lambda: estp.KVCache(cache.k, cache.v, cache.page_table, cache.length[:1], cache.seen),
              lambda: estp.KVCache(cache.k, cache.v, cache.page_table, cache.length, cache.seen, cache.weight[:1])):
        with pytest.raises(ValueError):
            f()
    odd = torch.zeros(4, 12, 2, 64, dtype=BF, device="cuda")
    assert status(lambda: call(estp.KVCache(odd, odd, cache.page_table, cache.length, cache.seen), Q, kn, vn, cu, 1)) == bad
    thin = torch.zeros(4, 16, 2, 32, dtype=BF, device="cuda")
    q32 = _rows(rng, 2, 4, 32, BF)
    assert status(lambda: call(estp.KVCache(thin, thin, cache.page_table, cache.length, cache.seen), q32, None, None, cu, 1)) == no
    # nothing to do
    empty = call(cache, Q[:0], kn[:0], vn[:0], torch.zeros(3, dtype=torch.int32, device="cuda"), 0)
    assert empty.shape == (0, 4, 64)
    ctx.sync_status()
    ctx.close()


def test_checked_build_agrees(cuda_lib):
    estp = cuda_lib
    res = []
    for library in (estp.lib, estp.load_library(estp.CHECKS_LIB_PATH)):
        rng = np.random.default_rng(4)
        ctx = estp.Context(0, library=library)
        for dtype in (BF, F32):
            cache = R.make_cache(estp, rng, [500, 64, 3], 2, 128, 16, dtype)
            Q, kn, vn = _rows(rng, 10, 14, 128, dtype), _rows(rng, 10, 2, 128, dtype), _rows(rng, 10, 2, 128, dtype)
            cu = torch.tensor([0, 1, 8, 10], dtype=torch.int32, device="cuda")
            out, lse, wn = ctx.cache_attention(cache, Q, kn, vn, cu, 7, accumulate=True, details=True)
            ctx.sync_status()
            res.append((out, lse, wn, cache.weight.nan_to_num()))
        ctx.close()
    for a, b in zip(res[:2], res[2:]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("n", [1, 60])
def test_wait_runs_out_then_context_recovers(cuda_lib, n):
    """A bounded wait of the tensor-core kernels that runs out is recorded, and the next call is right."""
    rng = np.random.default_rng(n)
    ctx = cuda_lib.Context(0)
    cache = R.make_cache(cuda_lib, rng, [700, 90], 2, 128, 16, BF)
    Q, kn, vn = _rows(rng, 2 * n, 8, 128, BF), _rows(rng, 2 * n, 2, 128, BF), _rows(rng, 2 * n, 2, 128, BF)
    cu = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    ctx.set_wait_limit(2)
    ctx.cache_attention(cache, Q, kn, vn, cu, n)
    with pytest.raises(cuda_lib.EstpError) as e:
        ctx.sync_status()
    assert e.value.status == cuda_lib.ESTP_ERR_TIMEOUT
    ctx.set_wait_limit(0)
    ctx.sync_status()
    _check(cuda_lib, ctx, cache, Q, kn, vn, [n, n], [R.tree(rng, n), R.tree(rng, n)])
    ctx.close()
