"""Plain 64-bit definitions of the cache operators on host data, and small caches to try them on."""
import numpy as np
import torch


def make_cache(estp, rng, lens, Hkv, d, page, dtype, spare=2, cap=None, poison=True, head_major=False, holes=3):
    """A KVCache of sequences of `lens` slots, on pages in random order; unused slots hold NaN."""
    B = len(lens)
    per = max(1, -(-(max(lens) + spare if cap is None else cap) // page))
    n_pages = B * per + holes
    shape = (n_pages, Hkv, page, d) if head_major else (n_pages, page, Hkv, d)
    fill = float("nan") if poison else 0.0
    k = torch.full(shape, fill, dtype=dtype, device="cuda")
    v = torch.full(shape, fill, dtype=dtype, device="cuda")
    if head_major:
        k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
    weight = torch.full((n_pages, Hkv, page), fill, device="cuda")
    position = torch.full((n_pages, Hkv, page), -7, dtype=torch.int32, device="cuda")
    table = torch.from_numpy(rng.permutation(n_pages)[: B * per].reshape(B, per).astype(np.int32)).cuda()
    for b, T in enumerate(lens):
        slot = np.arange(T)
        pg = table[b, torch.from_numpy(slot // page).cuda()].long()
        of = torch.from_numpy(slot % page).cuda()
        k[pg, of] = torch.from_numpy(rng.standard_normal((T, Hkv, d))).to(dtype).cuda()
        v[pg, of] = torch.from_numpy(rng.standard_normal((T, Hkv, d))).to(dtype).cuda()
        weight[pg, :, of] = torch.from_numpy(rng.exponential(size=(T, Hkv)).astype(np.float32)).cuda()
        position[pg, :, of] = torch.from_numpy(slot.astype(np.int32)).cuda()[:, None].expand(T, Hkv)
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return estp.KVCache(k, v, table, length, length.clone(), weight, position)


def slots(cache, b, T):
    """Page and offset arrays of the first T slots of sequence b."""
    page = cache.k.shape[1]
    at = np.arange(T)
    return cache.page_table[b].cpu().numpy()[at // page], at % page


def host(t):
    """An array of doubles (whole numbers stay)."""
    t = t.detach().cpu()
    return t.double().numpy() if t.is_floating_point() else t.numpy().copy()


def attention(cache, Q, k_new, v_new, cu, scale, sees, row_weight=None):
    """out, lse, weight_new and what every slot received [per b: (T, Hkv)], in 64 bits.
    sees[b]: bool [n_b, n_b]."""
    k, v, q = host(cache.k), host(cache.v), host(Q)
    Hq, d, Hkv = q.shape[1], q.shape[2], k.shape[2]
    rep = Hq // Hkv
    out, lse = np.zeros(q.shape), np.full((Hq, q.shape[0]), -np.inf)
    w_new, gave = np.zeros((q.shape[0], Hkv)), []
    c = np.ones(q.shape[0]) if row_weight is None else host(row_weight)
    for b, T in enumerate(cache.length.tolist()):
        lo, hi = cu[b], cu[b + 1]
        pg, of = slots(cache, b, T)
        K, V = k[pg, of], v[pg, of]
        got = np.zeros((T, Hkv))
        for i in range(lo, hi):
            mine = np.flatnonzero(sees[b][i - lo]) if k_new is not None else np.zeros(0, int)
            Ki = K if not len(mine) else np.concatenate([K, host(k_new[lo:hi])[mine]])
            Vi = V if not len(mine) else np.concatenate([V, host(v_new[lo:hi])[mine]])
            if not len(Ki):
                continue
            for h in range(Hq):
                g = h // rep
                z = scale * (Ki[:, g] @ q[i, h])
                m = z.max()
                e = np.exp(z - m)
                lse[h, i] = m + np.log(e.sum())
                p = e / e.sum()
                out[i, h] = p @ Vi[:, g]
                if c[i] != 0:
                    got[:, g] += c[i] * p[:T]
                    w_new[lo + mine, g] += c[i] * p[T:]
        gave.append(got)
    return out, lse, w_new, gave


def evict(cache, budget, recent, sinks):
    """The cache's arrays after an eviction (k, v, weight, position, length)."""
    k, v, w, pos = host(cache.k), host(cache.v), cache.weight.cpu().numpy().copy(), host(cache.position)
    length, seen = host(cache.length), host(cache.seen)
    for b, n in enumerate(length.tolist()):
        if n <= budget:
            continue
        pg, of = slots(cache, b, n)
        at = np.arange(n)
        for g in range(k.shape[2]):
            p, x = pos[pg, g, of], w[pg, g, of].astype(np.float64)
            safe = (p < sinks) | (p >= seen[b] - recent)
            rank = np.where(np.isnan(x), -np.inf, x)
            order = np.lexsort((at, np.isnan(x) & ~safe, -rank, ~safe))
            # among the safe ones all rank alike
            order = np.concatenate([np.sort(order[: safe.sum()]), order[safe.sum():]])[:budget]
            keep = np.zeros(n, bool)
            keep[order] = True
            dst, src = at[(at < budget) & ~keep], at[(at >= budget) & keep]
            for t in (k, v):
                t[pg[dst], of[dst], g] = t[pg[src], of[src], g]
            for t in (w, pos):
                t[pg[dst], g, of[dst]] = t[pg[src], g, of[src]]
        length[b] = budget
    return k, v, w, pos, length


def bits_of(sees, words):
    """uint64 words (as int64) of bool matrices, one after another."""
    rows = []
    for s in sees:
        for r in s:
            m = sum(1 << int(j) for j in np.flatnonzero(r))
            rows.append([m >> 64 * w & (1 << 64) - 1 for w in range(words)])
    return torch.from_numpy(np.array(rows, dtype=np.uint64).reshape(-1, words).view(np.int64)).cuda()


def tree(rng, n):
    """Ancestors (and self) of a random tree of n nodes."""
    s = np.zeros((n, n), bool)
    for i in range(n):
        up = int(rng.integers(-1, i)) if i else -1
        if up >= 0:
            s[i] = s[up]
        s[i, i] = True
    return s
