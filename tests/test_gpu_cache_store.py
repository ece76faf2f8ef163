"""Rows into a paged KV cache and slots out of it: exact against the definition (GPU)."""
import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _cu(counts):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()


def _same(t, a):
    x = R.host(t)
    assert np.array_equal(x, a, equal_nan=True) if x.dtype.kind == "f" else np.array_equal(x, a)


def _append_ref(cache, kn, vn, counts, weight, rows, fresh):
    k, v, w, pos = host4 = [R.host(t) for t in (cache.k, cache.v, cache.weight, cache.position)]
    length, seen = R.host(cache.length), R.host(cache.seen)
    table, page = cache.page_table.cpu().numpy(), cache.k.shape[1]
    kn, vn, weight = R.host(kn), R.host(vn), None if weight is None else R.host(weight)
    src = np.arange(sum(counts)) if rows is None else rows.cpu().numpy()
    e = 0
    for b, n in enumerate(counts):
        if fresh:
            length[b] = seen[b] = 0
        for i in range(n):
            s = length[b] + i
            p, o = table[b, s // page], s % page
            k[p, o], v[p, o] = kn[src[e]], vn[src[e]]
            w[p, :, o] = 0 if weight is None else weight[src[e]]
            pos[p, :, o] = seen[b] + i
            e += 1
        length[b] += n
        seen[b] += n
    return (*host4, length, seen)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,counts,Hkv,d,page", [
    ([0], [1], 1, 64, 8),
    ([7, 8, 9], [1, 1, 1], 2, 128, 8),
    ([0, 100, 31], [130, 0, 33], 3, 64, 32),
    ([5] * 70, [0, 1, 2, 0, 3, 9, 1] * 10, 4, 128, 16),
    ([16], [300], 8, 128, 256),
])
def test_append(cuda_lib, dtype, lens, counts, Hkv, d, page):
    rng = np.random.default_rng(len(lens) + d)
    ctx = cuda_lib.Context(0)
    n = sum(counts)
    for kind in ("plain", "rows", "fresh", "strided"):
        cache = R.make_cache(cuda_lib, rng, lens, Hkv, d, page, dtype, spare=max(counts) + 1, head_major=kind == "strided")
        cache.seen += 11
        fused = torch.from_numpy(rng.standard_normal((n + 4, 2 * Hkv + 1, d))).to(dtype).cuda()
        kn, vn = fused[:, :Hkv], fused[:, Hkv:2 * Hkv]
        if kind != "strided":
            kn, vn = kn.contiguous(), vn.contiguous()
        weight = None if kind == "fresh" else torch.from_numpy(rng.exponential(size=(n + 4, Hkv)).astype(np.float32)).cuda()
        rows = torch.from_numpy(rng.integers(0, n + 4, n + 2).astype(np.int32)).cuda() if kind == "rows" else None
        want = _append_ref(cache, kn, vn, counts, weight, rows, kind == "fresh")
        ctx.cache_append(cache, kn, vn, _cu(counts), weight=weight, rows=rows, fresh=kind == "fresh")
        ctx.sync_status()
        for t, a in zip((cache.k, cache.v, cache.weight, cache.position, cache.length, cache.seen), want):
            _same(t, a)
    ctx.close()


def test_append_that_does_not_fit(cuda_lib):
    """The sequence keeps its length, the others get their rows, and the status says so."""
    estp = cuda_lib
    rng = np.random.default_rng(3)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, [30, 30], 2, 64, 16, F32, cap=32)
    kn = torch.randn(5, 2, 64, device="cuda")
    ctx.cache_append(cache, kn, kn, _cu([3, 2]))
    with pytest.raises(estp.EstpError) as e:
        ctx.sync_status()
    assert e.value.status == estp.ESTP_ERR_INVALID_ARG
    assert cache.length.tolist() == [30, 32] and cache.seen.tolist() == [30, 32]
    # rows outside k_new, and a list of counts that falls
    rows = torch.tensor([5, -1], dtype=torch.int32, device="cuda")
    cache.length.fill_(0)
    k0 = cache.k.clone()
    for args in ((_cu([1, 1]), rows), (torch.tensor([0, 2, 1], dtype=torch.int32, device="cuda"), None)):
        ctx.cache_append(cache, kn, kn, args[0], rows=args[1])
        with pytest.raises(estp.EstpError):
            ctx.sync_status()
    ctx.close()
    assert k0.shape == cache.k.shape


def _evict_check(ctx, cache, budget, recent, sinks):
    want = R.evict(cache, budget, recent, sinks)
    seen = cache.seen.clone()
    ctx.cache_evict(cache, budget, recent=recent, sinks=sinks)
    ctx.sync_status()
    for t, a in zip((cache.k, cache.v, cache.weight, cache.position, cache.length), want):
        _same(t, a)
    assert torch.equal(seen, cache.seen)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,Hkv,d,page,budget,recent,sinks", [
    ([2], 1, 64, 8, 1, 0, 0),
    ([2], 1, 64, 8, 1, 1, 0),
    ([10, 0, 9, 33], 2, 128, 8, 9, 3, 2),
    ([100, 64, 65, 1], 3, 64, 16, 64, 0, 4),
    ([1025] * 5, 4, 128, 16, 1024, 32, 4),
    ([700, 1500, 300], 2, 64, 64, 100, 100, 0),
    ([3000], 8, 128, 256, 2500, 10, 1),
    ([20000], 1, 64, 32, 4000, 64, 4),
    ([400, 50], 2, 64, 16, 1000, 0, 0),
])
def test_evict(cuda_lib, dtype, lens, Hkv, d, page, budget, recent, sinks):
    rng = np.random.default_rng(sum(lens) + d)
    ctx = cuda_lib.Context(0)
    cache = R.make_cache(cuda_lib, rng, lens, Hkv, d, page, dtype)
    _evict_check(ctx, cache, budget, recent, sinks)
    # a second time nothing is left to drop; to half of it, with positions out of order now
    _evict_check(ctx, cache, budget, recent, sinks)
    if budget > 1:
        _evict_check(ctx, cache, -(-budget // 2), recent // 2, sinks // 2)
    ctx.close()


@pytest.mark.parametrize("values", [[1.0], [0.0, -0.0], [3.0, 3.0, float("nan")], [float("inf"), float("-inf"), float("nan"), -1.0, 2.0],
                                    [1e-45, 0.0, -1e-45, 1.0, 1.0000001]])
@pytest.mark.parametrize("n,budget,recent,sinks", [(70, 33, 5, 2), (3000, 1000, 0, 0), (9000, 8000, 100, 4)])
def test_ties_and_odd_weights(cuda_lib, values, n, budget, recent, sinks):
    """Equal weights go by the slot, zeros of both signs are equal, NaN goes first."""
    rng = np.random.default_rng(n)
    ctx = cuda_lib.Context(0)
    cache = R.make_cache(cuda_lib, rng, [n, n // 2], 2, 64, 16, BF)
    w = torch.from_numpy(rng.choice(np.array(values, np.float32), cache.weight.shape)).cuda()
    cache.weight.copy_(w)
    _evict_check(ctx, cache, budget, recent, sinks)
    ctx.close()


def test_more_slots_than_fit_in_shared_memory(cuda_lib):
    rng = np.random.default_rng(0)
    ctx = cuda_lib.Context(0)
    n, page = 450_001, 64
    per = -(-n // page)
    k = torch.randn(per, page, 1, 64, device="cuda", dtype=torch.float32).to(BF)
    table = torch.from_numpy(rng.permutation(per).astype(np.int32)).cuda()[None]
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    weight = torch.from_numpy(rng.integers(0, 1000, (per, 1, page)).astype(np.float32)).cuda()
    position = torch.from_numpy(rng.integers(0, n, (per, 1, page)).astype(np.int32)).cuda()
    cache = cuda_lib.KVCache(k, k.clone(), table, length, length.clone(), weight, position)
    _evict_check(ctx, cache, 150_000, 1000, 4)
    ctx.close()


def test_evict_in_a_graph(cuda_lib):
    """A step at the budget (a row enters, a slot goes), captured and replayed."""
    rng = np.random.default_rng(8)
    ctx = cuda_lib.Context(0)
    caches = []
    for _ in range(2):
        rng = np.random.default_rng(8)
        caches.append(R.make_cache(cuda_lib, rng, [64, 64], 2, 64, 16, BF, spare=2))
    kn = torch.randn(2, 2, 64, device="cuda").to(BF)
    cu = _cu([1, 1])

    def step(c):
        ctx.cache_append(c, kn, kn, cu)
        ctx.cache_evict(c, 64, recent=8, sinks=2)

    for c in caches:
        step(c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(caches[1])
    for _ in range(5):
        step(caches[0])
        g.replay()
    torch.cuda.synchronize()
    ctx.sync_status()
    for n in ("k", "v", "weight", "position", "length", "seen"):
        assert torch.equal(getattr(caches[0], n).nan_to_num(), getattr(caches[1], n).nan_to_num())
    assert caches[0].length.tolist() == [64, 64] and caches[0].seen.tolist() == [70, 70]
    del g
    ctx.close()


def test_evict_refuses(cuda_lib):
    estp = cuda_lib
    rng = np.random.default_rng(2)
    ctx = estp.Context(0)
    cache = R.make_cache(estp, rng, [50], 2, 64, 16, BF)
    bare = estp.KVCache(cache.k, cache.v, cache.page_table, cache.length, cache.seen)
    for f in (lambda: ctx.cache_evict(cache, 0), lambda: ctx.cache_evict(cache, 10, recent=8, sinks=3),
              lambda: ctx.cache_evict(cache, 10, recent=-1), lambda: ctx.cache_evict(bare, 10)):
        with pytest.raises(estp.EstpError) as e:
            f()
        assert e.value.status == estp.ESTP_ERR_INVALID_ARG
    cache.length[0] = 10 ** 7
    ctx.cache_evict(cache, 10)
    with pytest.raises(estp.EstpError):
        ctx.sync_status()
    kn = torch.zeros(3, 2, 64, dtype=BF, device="cuda")
    for f in (lambda: ctx.cache_append(cache, kn.float(), kn.float(), _cu([3])), lambda: ctx.cache_append(cache, kn, kn[:2], _cu([3])),
              lambda: ctx.cache_append(cache, kn, kn, _cu([1, 2])), lambda: ctx.cache_append(cache, kn, kn, _cu([3]), weight=torch.zeros(2, 2, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    ctx.close()
