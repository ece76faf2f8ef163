"""The cache as a serving program uses it (GPU): a ragged batch of prompts is prefilled with the
fused forward, its importance becomes the cache's weights, the cache is cut to a budget, and
steps of drafted trees follow: attention, the accepted path appended, eviction.  Every step is
checked against the same loop in 64 bits on the host."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu


def test_prefill_evict_and_decode(cuda_lib):
    estp = cuda_lib
    rng = np.random.default_rng(0)
    ctx = estp.Context(0)
    Hq, Hkv, d, page, budget, recent, sinks = 8, 2, 128, 16, 96, 24, 4
    lens = [150, 61, 97]
    n, B = sum(lens), len(lens)
    bf = torch.bfloat16
    rand = lambda m, h: torch.from_numpy(rng.standard_normal((m, h, d))).to(bf).cuda()  # noqa: E731
    Q, K, V = rand(n, Hq), rand(n, Hkv), rand(n, Hkv)
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    ctx.attn_forward_importance(Q, K, V, cu, max(lens), divisor="none")
    S = ctx.attn_importance_finalize(1, n)  # mean over the heads of the attention each token received
    per = -(-(max(lens) + 16) // page)
    n_pages = per * B
    nan = float("nan")
    cache = estp.KVCache(torch.full((n_pages, page, Hkv, d), nan, dtype=bf, device="cuda"),
                         torch.full((n_pages, page, Hkv, d), nan, dtype=bf, device="cuda"),
                         torch.from_numpy(rng.permutation(n_pages).reshape(B, per).astype(np.int32)).cuda(),
                         torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"),
                         torch.full((n_pages, Hkv, page), nan, device="cuda"),
                         torch.full((n_pages, Hkv, page), -1, dtype=torch.int32, device="cuda"))
    ctx.cache_append(cache, K, V, cu, weight=(S[:, None] * (Hq // Hkv)).expand(-1, Hkv).contiguous(), fresh=True)
    ctx.sync_status()
    assert cache.length.tolist() == lens and cache.seen.tolist() == lens
    for b, T in enumerate(lens):  # the tokens as they were, weights summing to the attention given
        pg, of = R.slots(cache, b, T)
        assert np.array_equal(R.host(cache.k)[pg, of], R.host(K[cu[b]:cu[b + 1]]))
        total = R.host(cache.weight)[pg, :, of].sum(0)
        assert np.all(np.abs(total - T * Hq / Hkv) <= 1e-3 * T * Hq / Hkv)

    def evict():
        want = R.evict(cache, budget, recent, sinks)
        ctx.cache_evict(cache, budget, recent=recent, sinks=sinks)
        ctx.sync_status()
        for t, a in zip((cache.k, cache.v, cache.weight, cache.position, cache.length), want):
            assert np.array_equal(R.host(t), a, equal_nan=True) if t.is_floating_point() else np.array_equal(R.host(t), a)

    evict()
    for step in range(4):
        counts = [int(c) for c in rng.integers(1, 9, B)]
        m = sum(counts)
        q, k, v = rand(m, Hq), rand(m, Hkv), rand(m, Hkv)
        sees = [R.tree(rng, c) for c in counts]
        prob = torch.from_numpy(rng.uniform(0.1, 1, m).astype(np.float32)).cuda()
        cu_rows = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        want, _, _, gave = R.attention(cache, q, k, v, cu_rows, 1 / math.sqrt(d), sees, prob)
        before = R.host(cache.weight)
        out, lse, w = ctx.cache_attention(cache, q, k, v, torch.from_numpy(cu_rows).cuda(), max(counts),
                                          tree_mask=R.bits_of(sees, 1), row_weight=prob, accumulate=True, details=True)
        ctx.sync_status()
        assert np.all(np.abs(R.host(out) - want) <= 2.0 ** -8 * np.abs(want) + 2e-4 * 5)
        for b, T in enumerate(cache.length.tolist()):
            pg, of = R.slots(cache, b, T)
            grown = R.host(cache.weight)[pg, :, of] - before[pg, :, of]
            assert np.all(np.abs(grown - gave[b]) <= 2e-4 * gave[b] + 2.0 ** -22 * before[pg, :, of] + 1e-9)
        # the path to one accepted node of every tree enters the cache
        path = [np.flatnonzero(s[int(rng.integers(0, len(s)))]) + lo for s, lo in zip(sees, cu_rows)]
        accepted = torch.from_numpy(np.concatenate(path).astype(np.int32)).cuda()
        cu_acc = torch.from_numpy(np.concatenate([[0], np.cumsum([len(p) for p in path])]).astype(np.int32)).cuda()
        held, seen = cache.length.tolist(), cache.seen.tolist()
        ctx.cache_append(cache, k, v, cu_acc, weight=w, rows=accepted)
        ctx.sync_status()
        for b, p in enumerate(path):
            pg, of = (x[held[b]:] for x in R.slots(cache, b, held[b] + len(p)))
            assert np.array_equal(R.host(cache.v)[pg, of], R.host(v)[p])
            assert np.array_equal(R.host(cache.weight)[pg, :, of], R.host(w)[p])
            assert cache.seen[b] == seen[b] + len(p)
        evict()
        assert max(cache.length.tolist()) <= budget
    ctx.close()
