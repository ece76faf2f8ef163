"""The calls on a paged KV cache whose speed this library is held to: their sizes, inputs,
plain forms and 64-bit references.

Three operators, as a serving program uses them after the prefill:
  attention  the rows of one decoding step (a single token a sequence, or a tree of drafted
             tokens) attend to the cache and to the drafts they descend from; every cached
             slot's accumulated attention weight grows by what the rows gave it
  append     rows enter the cache (a whole prompt with the prefill's importance as weights)
  evict      rows enter the cache and it is cut back to its budget: of each KV head the slots
             of the least weight go, and kept rows from the tail fill the freed slots

``listed()`` names the cases, ``draw()`` gives further ones of the same ranges, ``prepare()``
makes what a program holds before the call, ``run()`` makes the call, ``exact()`` evaluates the
definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False  # set by the tool that measures: False runs the plain forms

DEVICE = "cuda:0"
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------- cases
def _attention(name, dtype, B, T_lo, T_hi, Hq, Hkv, d, page, n_lo=1, n_hi=1, sinks=0):
    """One layer's attention of n_lo..n_hi rows a sequence over T_lo..T_hi cached slots; more
    than one row is a tree of drafts, each row counted with its draft probability."""
    return {"name": name, "op": "attention", "dtype": dtype, "B": B, "T_lo": T_lo, "T_hi": T_hi,
            "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "n_lo": n_lo, "n_hi": n_hi, "sinks": sinks}


def _append(name, dtype, B, T_lo, T_hi, Hkv, d, page):
    """Prompts of T_lo..T_hi tokens enter a cache whose sequences were empty."""
    return {"name": name, "op": "append", "dtype": dtype, "B": B, "T_lo": T_lo, "T_hi": T_hi,
            "Hkv": Hkv, "d": d, "page": page}


def _evict(name, dtype, B, budget, more, Hkv, d, page, recent, sinks, fresh=False):
    """`more` rows a sequence enter, then every sequence is cut to `budget` slots.  fresh: the
    rows are a whole prompt that enters an empty sequence; else they follow `budget` slots."""
    return {"name": name, "op": "evict", "dtype": dtype, "B": B, "budget": budget, "more": more,
            "Hkv": Hkv, "d": d, "page": page, "recent": recent, "sinks": sinks, "fresh": fresh}


def listed():
    return [
        # the smallest step: one token after a single 128-token prompt, fp32, one KV head a
        # query head; launches and latency are what it costs
        _attention("decode_f32_T128", "f32", 1, 128, 128, 8, 8, 64, 16),
        # one token of an ordinary ragged serving batch, 28/4 heads
        _attention("decode_varlen16", "bf16", 16, 256, 2048, 28, 4, 128, 16),
        # one token of a single long-context request with attention sinks: few rows, a long
        # axis to split
        _attention("decode_long32k", "bf16", 1, 32768, 32768, 28, 4, 128, 64, sinks=4),
        # one token of each of 256 rollouts, 32/8 heads: the largest call
        _attention("decode_rl256", "bf16", 256, 128, 4096, 32, 8, 128, 64),
        # small draft trees (odd sizes) of 8 long sequences, 64/8 heads
        _attention("tree17_8x8k", "bf16", 8, 8192, 8192, 64, 8, 128, 128, 9, 17, sinks=4),
        # wide draft trees, up to 64 nodes x 7 query heads on one KV head
        _attention("tree64_varlen6", "bf16", 6, 256, 4096, 28, 4, 128, 32, 40, 64),
        # draft trees in fp32, head size 64, two query heads a KV head
        _attention("tree9_f32", "f32", 3, 500, 1500, 16, 8, 64, 16, 3, 9),
        # the prompts of the ragged batch enter the cache with their importance
        _append("append_varlen16", "bf16", 16, 256, 2048, 4, 128, 16),
        # a single short fp32 prompt enters the cache
        _append("append_f32_T128", "f32", 1, 128, 128, 8, 64, 16),
        # a decoding step at the budget: one token enters, one slot of each KV head goes
        _evict("evict_step16", "bf16", 16, 1024, 1, 4, 128, 16, 32, 4),
        # a prompt chunk pushes out as many of the oldest tokens' slots
        _evict("evict_chunk8", "bf16", 8, 4096, 1000, 8, 128, 64, 1024, 4),
        # long prompts enter and are cut to an eighth of their length
        _evict("evict_prompt4x32k", "bf16", 4, 4096, 32768, 4, 128, 64, 256, 4, fresh=True),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges, at most the largest listed one's work."""
    op = rng.choice(["attention"] * 4 + ["append"] + ["evict"] * 2)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    Hkv = rng.choice([1, 2, 4, 8])
    d = rng.choice([64, 128])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    if op == "attention":
        rep = rng.choice([1, 2, 4, 7, 8])
        T_hi = _between(rng, 2, 32768)
        T_lo = max(1, int(T_hi * rng.uniform(0.1, 1.0)))
        # K and V at most 0.5 GB (0.13 GB in fp32, whose steps are not the large ones)
        slots = (1 << 29 if dtype == "bf16" else 1 << 27) // (2 * Hkv * d * (2 if dtype == "bf16" else 4))
        B = _between(rng, 1, max(1, min(256, slots // T_hi)))
        n_hi = 1 if rng.random() < 0.5 else _between(rng, 2, 64 if dtype == "bf16" else 16)
        while n_hi > 1 and 4 * d * Hkv * rep * n_hi * B * T_hi > 2e11:
            n_hi = max(1, n_hi // 2)
        n_lo = max(1, int(n_hi * rng.uniform(0.3, 1.0)))
        return _attention(None, dtype, B, T_lo, T_hi, Hkv * rep, Hkv, d, page, n_lo, n_hi,
                          rng.choice([0, 4]))
    if op == "append":
        T_hi = _between(rng, 1, 8192)
        B = _between(rng, 1, max(1, min(64, 131072 // T_hi)))
        return _append(None, dtype, B, max(1, int(T_hi * rng.uniform(0.1, 1.0))), T_hi, Hkv, d, page)
    budget = _between(rng, 40, 4096)
    fresh = rng.random() < 0.4
    more = budget + _between(rng, 1, 8 * budget) if fresh else _between(rng, 1, budget // 2)
    recent = rng.randint(1, budget // 2) if fresh else rng.randint(more, budget - 8)
    B = _between(rng, 1, max(1, min(64, 131072 // (budget + more))))
    return _evict(None, dtype, B, budget, more, Hkv, d, page, recent, rng.choice([0, 1, 4]), fresh)


# ------------------------------------------------------------------------ inputs
def _lengths(lo, hi, n):
    """n sizes of [lo, hi], the same ones whatever the seed: outputs of one case are of one shape."""
    rng = random.Random("%d %d %d" % (lo, hi, n))
    return [hi] if n == 1 else [rng.randint(lo, hi) for _ in range(n)]


def _cu(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=DEVICE)


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(dtype)


def _pages(gen, case, dtype, capacity, B, filled):
    """A pool of pages in random order and the page table of B sequences of `capacity` slots,
    with K, V and weights everywhere and positions as an append would have left them."""
    per = -(-capacity // case["page"])
    n = per * B + 3
    page, Hkv, d = case["page"], case["Hkv"], case["d"]
    table = torch.randperm(n, generator=gen, device=DEVICE)[: per * B].reshape(B, per)
    k = torch.empty(n, page, Hkv, d, dtype=dtype, device=DEVICE).normal_(generator=gen)
    v = torch.empty(n, page, Hkv, d, dtype=dtype, device=DEVICE).normal_(generator=gen)
    # a token's accumulated weight: most get little, few get much
    weight = torch.empty(n, Hkv, page, device=DEVICE).exponential_(generator=gen) ** 2
    position = torch.zeros(n, Hkv, page, dtype=torch.int32, device=DEVICE)
    slot = torch.arange(per * page, dtype=torch.int32, device=DEVICE).reshape(1, per, 1, page)
    position[table.reshape(-1)] = slot.expand(B, per, Hkv, page).reshape(B * per, Hkv, page).contiguous()
    if case.get("sinks") and case["op"] == "attention":  # the first tokens draw much of the attention
        first = table[:, 0]
        k[first, : min(case["sinks"], page)] *= 8
    return {"k": k, "v": v, "weight": weight, "position": position,
            "table": table.to(torch.int32).contiguous(),
            "length": torch.tensor(filled, dtype=torch.int32, device=DEVICE),
            "seen": torch.tensor(filled, dtype=torch.int32, device=DEVICE)}


def _trees(rng, counts):
    """Ancestor bits of random draft trees: row i of a sequence sees draft j where j is i or one
    of its ancestors; int64 [rows, words]."""
    words = -(-max(counts) // 64)
    rows = []
    for n in counts:
        masks = []
        for i in range(n):
            up = rng.randint(max(-1, i - 6), i - 1) if i else -1
            masks.append((masks[up] if up >= 0 else 0) | 1 << i)
        rows += [[m >> 64 * w & (1 << 64) - 1 for w in range(words)] for m in masks]
    bits = np.array(rows, dtype=np.uint64).view(np.int64)
    return torch.from_numpy(bits).to(DEVICE)


def prepare(case, seed):
    rng = random.Random(seed)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype = _TYPES[case["dtype"]]
    B, Hkv, d = case["B"], case["Hkv"], case["d"]
    if case["op"] == "attention":
        lens = _lengths(case["T_lo"], case["T_hi"], B)
        counts = _lengths(case["n_lo"], case["n_hi"], B)
        rows, most = sum(counts), max(counts)
        s = _pages(gen, case, dtype, max(lens), B, lens)
        s.update(case=case, max_len=max(lens), max_rows=most, cu=_cu(counts),
                 q=_normal(gen, (rows, case["Hq"], d), dtype),
                 k_new=_normal(gen, (rows, Hkv, d), dtype), v_new=_normal(gen, (rows, Hkv, d), dtype),
                 tree=None, row_weight=None, scale=1.0 / math.sqrt(d))
        if most > 1:
            s["tree"] = _trees(rng, counts)
            s["row_weight"] = torch.rand(rows, generator=gen, device=DEVICE)
        return s
    if case["op"] == "append":
        counts = _lengths(case["T_lo"], case["T_hi"], B)
        s = _pages(gen, case, dtype, max(counts), B, [0] * B)
        s.update(case=case, max_rows=max(counts), fresh=True)
    else:
        # a sequence at its budget, or an empty one that a whole prompt enters
        fresh = case["fresh"]
        held = 0 if fresh else case["budget"]
        counts = [case["more"]] * B
        s = _pages(gen, case, dtype, held + case["more"], B, [held] * B)
        s.update(case=case, max_rows=case["more"], max_len=held + case["more"], fresh=fresh)
    rows = sum(counts)
    s.update(cu=_cu(counts), k_new=_normal(gen, (rows, Hkv, d), dtype), v_new=_normal(gen, (rows, Hkv, d), dtype),
             weight_new=torch.empty(rows, Hkv, device=DEVICE).exponential_(generator=gen) ** 2)
    return s


# ------------------------------------------------------------------- plain forms
def _slots(s, most):
    """Pages and offsets [B, most] of the first `most` slots of each sequence."""
    page = s["k"].shape[1]
    at = torch.arange(most, device=DEVICE)
    return s["table"].long()[:, at // page], (at % page).expand(s["table"].shape[0], most)


def _padded(s):
    """Packed row of (sequence, i), i < max_rows, and which of them exist."""
    cu = s["cu"].long()
    i = torch.arange(s["max_rows"], device=DEVICE)
    there = i < (cu[1:] - cu[:-1])[:, None]
    return torch.where(there, cu[:-1, None] + i, 0), there


def _plain_attention(s):
    case = s["case"]
    Hkv, d, rep = case["Hkv"], case["d"], case["Hq"] // case["Hkv"]
    B, L, N = s["length"].shape[0], s["max_len"], s["max_rows"]
    page, off = _slots(s, L)
    at, there = _padded(s)
    held = torch.arange(L, device=DEVICE) < s["length"][:, None]
    K = s["k"][page, off].float()
    V = torch.where(held[:, :, None, None], s["v"][page, off].float(), 0.0)
    K = torch.cat([K, s["k_new"][at].float()], 1)
    V = torch.cat([V, torch.where(there[:, :, None, None], s["v_new"][at].float(), 0.0)], 1)
    Q = s["q"][at].float().reshape(B, N, Hkv, rep, d)
    j = torch.arange(N, device=DEVICE)
    if s["tree"] is None:
        sees = (j[None, :] <= j[:, None]).expand(B, N, N)
    else:
        sees = (s["tree"][at][:, :, j // 64] >> (j % 64) & 1).bool()
    sees = torch.cat([held[:, None, :].expand(B, N, L), sees & there[:, None, :]], 2) & there[:, :, None]
    z = torch.einsum("bnghd,bjgd->bghnj", Q, K) * s["scale"]
    z = torch.where(sees[:, None, None], z, -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    p = e / torch.where(total == 0, 1.0, total)
    o = torch.einsum("bghnj,bjgd->bnghd", p, V).reshape(B, N, Hkv * rep, d)
    c = torch.ones(B, N, device=DEVICE) if s["row_weight"] is None else s["row_weight"][at]
    w = torch.einsum("bghnj,bn->bgj", p, torch.where(there, c, 0.0))
    rows = s["q"].shape[0]
    spot = torch.where(there, at, rows).reshape(-1)  # rows that do not exist land past the end
    out = torch.empty(rows + 1, Hkv * rep, d, dtype=s["q"].dtype, device=DEVICE)
    out[spot] = o.reshape(B * N, Hkv * rep, d).to(out.dtype)
    lse_out = torch.empty(Hkv * rep, rows + 1, device=DEVICE)
    lse_out[:, spot] = lse.reshape(B, Hkv * rep, N).transpose(0, 1).reshape(Hkv * rep, B * N)
    w_new = torch.empty(rows + 1, Hkv, device=DEVICE)
    w_new[spot] = w[:, :, L:].transpose(1, 2).reshape(B * N, Hkv)
    size = s["weight"].shape[2]
    flat = (page[:, None, :] * Hkv + torch.arange(Hkv, device=DEVICE)[None, :, None]) * size + off[:, None, :]
    s["weight"].view(-1).scatter_add_(0, flat.reshape(-1), torch.where(held[:, None, :], w[:, :, :L], 0.0).reshape(-1))
    return {"out": out[:rows], "lse": lse_out[:, :rows], "weight_new": w_new[:rows], "weight": s["weight"]}


def _plain_append(s):
    cu = s["cu"].long()
    rows = s["k_new"].shape[0]
    start = torch.zeros_like(s["length"]) if s["fresh"] else s["length"]
    seen = torch.zeros_like(s["seen"]) if s["fresh"] else s["seen"]
    r = torch.arange(rows, device=DEVICE)
    b = torch.searchsorted(cu, r, right=True) - 1
    i = r - cu[b]
    size = s["k"].shape[1]
    slot = start.long()[b] + i
    page, off = s["table"].long()[b, slot // size], slot % size
    s["k"][page, off] = s["k_new"]
    s["v"][page, off] = s["v_new"]
    s["weight"][page, :, off] = s["weight_new"]
    s["position"][page, :, off] = (seen.long()[b] + i).int()[:, None].expand(rows, s["k"].shape[2])
    n = (cu[1:] - cu[:-1]).int()
    s["length"].copy_(start + n)
    s["seen"].copy_(seen + n)


def _plain_evict(s):
    case = s["case"]
    budget, L, Hkv = case["budget"], s["max_len"], case["Hkv"]
    page, off = _slots(s, L)
    head = torch.arange(Hkv, device=DEVICE)[None, :, None]
    at = torch.arange(L, device=DEVICE)
    held = at < s["length"][:, None, None]
    w, pos = s["weight"][page[:, None], head, off[:, None]], s["position"][page[:, None], head, off[:, None]]
    kept_anyway = (pos < case["sinks"]) | (pos >= s["seen"][:, None, None] - case["recent"])
    w = torch.where(held, torch.where(kept_anyway, math.inf, w), -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :budget]
    keep = torch.zeros_like(held.expand_as(w)).scatter(-1, order, True) & held
    hole, tail = ~keep & (at < budget) & held, keep & (at >= budget)
    most = min(budget, L - budget)
    dst = torch.sort(hole.int(), dim=-1, descending=True, stable=True).indices[..., :most]
    src = torch.sort(tail.int(), dim=-1, descending=True, stable=True).indices[..., :most]
    moved = torch.arange(most, device=DEVICE) < tail.sum(-1, keepdim=True)
    dst_page, dst_off = page[:, None].expand(-1, Hkv, -1).gather(-1, dst), off[:, None].expand(-1, Hkv, -1).gather(-1, dst)
    src_page, src_off = page[:, None].expand(-1, Hkv, -1).gather(-1, src), off[:, None].expand(-1, Hkv, -1).gather(-1, src)
    for x in (s["k"], s["v"]):
        x[dst_page, dst_off, head] = torch.where(moved[..., None], x[src_page, src_off, head], x[dst_page, dst_off, head])
    for x in (s["weight"], s["position"]):
        x[dst_page, head, dst_off] = torch.where(moved, x[src_page, head, src_off], x[dst_page, head, dst_off])
    s["length"].clamp_(max=budget)


# --------------------------------------------------------------------- the calls
_ctx = None


def _own_run(s):
    import paper_2608_15592_gb300 as estp
    global _ctx
    if _ctx is None:
        _ctx = estp.Context(0)
    cache = s.get("cache")
    if cache is None:
        cache = s["cache"] = estp.KVCache(s["k"], s["v"], s["table"], s["length"], s["seen"], s["weight"], s["position"])
    if s["case"]["op"] == "attention":
        out, lse, w_new = _ctx.cache_attention(cache, s["q"], s["k_new"], s["v_new"], s["cu"], s["max_rows"], scale=s["scale"],
                                               tree_mask=s["tree"], row_weight=s["row_weight"], accumulate=True, details=True)
        return {"out": out, "lse": lse, "weight_new": w_new, "weight": s["weight"]}
    _ctx.cache_append(cache, s["k_new"], s["v_new"], s["cu"], weight=s["weight_new"], fresh=s["fresh"])
    if s["case"]["op"] == "evict":
        _ctx.cache_evict(cache, s["case"]["budget"], recent=s["case"]["recent"], sinks=s["case"]["sinks"])
    return _whole(s)


def _whole(s):
    return {n: s[n] for n in ("k", "v", "weight", "position", "length", "seen")}


def run(state):
    if own:
        return _own_run(state)
    if state["case"]["op"] == "attention":
        return _plain_attention(state)
    _plain_append(state)
    if state["case"]["op"] == "evict":
        _plain_evict(state)
    return _whole(state)


# -------------------------------------------------------------------------- work
def work(case):
    es, Hkv, d, B = 2 if case["dtype"] == "bf16" else 4, case["Hkv"], case["d"], case["B"]
    row = 2 * d * es + 8  # K and V, weight, position of one slot of one KV head
    if case["op"] == "attention":
        lens, counts = _lengths(case["T_lo"], case["T_hi"], B), _lengths(case["n_lo"], case["n_hi"], B)
        slots, rows = sum(lens), sum(counts)
        io = rows * (case["Hq"] * (2 * d * es + 4) + Hkv * (2 * d * es + 4))
        pairs = sum(n * (t + 1) for n, t in zip(counts, lens))  # a draft sees itself and a few before it
        # every slot's K and V read, its weight read and written
        return {"bytes": slots * Hkv * (2 * d * es + 8) + io, "flops": 4 * d * case["Hq"] * pairs}
    if case["op"] == "append":
        rows = sum(_lengths(case["T_lo"], case["T_hi"], B))
        return {"bytes": rows * Hkv * (2 * 2 * d * es + 4 + 8), "flops": 0}
    more, budget = case["more"], case["budget"]
    held = 0 if case["fresh"] else budget
    # the rows that enter are read and written once; every slot's weight and position are read; at
    # the budget as many rows move as entered, of a fresh prompt those kept from past the budget
    moved = min(more, budget) if not case["fresh"] else budget * (more - budget) / more
    return {"bytes": B * Hkv * (more * (2 * 2 * d * es + 4 + 8) + (held + more) * 8 + moved * 2 * row), "flops": 0}


# -------------------------------------------------------------------------- exact
def exact(case, seed):
    s = prepare(case, seed)
    size, Hkv = case["page"], case["Hkv"]
    if case["op"] == "attention":
        rep, d = case["Hq"] // Hkv, case["d"]
        cu, lens = s["cu"].tolist(), s["length"].tolist()
        rows = cu[-1]
        out = torch.zeros(rows, case["Hq"], d, dtype=torch.float64, device=DEVICE)
        lse = torch.zeros(case["Hq"], rows, dtype=torch.float64, device=DEVICE)
        w_new = torch.zeros(rows, Hkv, dtype=torch.float64, device=DEVICE)
        weight = s["weight"].double()
        bits = None if s["tree"] is None else s["tree"].cpu().numpy().view(np.uint64)
        for b, T in enumerate(lens):
            lo, hi = cu[b], cu[b + 1]
            n = hi - lo
            ids = s["table"][b, : -(-T // size)].long()
            K = torch.cat([s["k"][ids].reshape(-1, Hkv, d)[:T], s["k_new"][lo:hi]]).double()
            V = torch.cat([s["v"][ids].reshape(-1, Hkv, d)[:T], s["v_new"][lo:hi]]).double()
            if bits is None:
                seen = np.tril(np.ones((n, n), dtype=bool))
            else:
                seen = np.array([[bool(int(bits[lo + i, j // 64]) >> j % 64 & 1) for j in range(n)] for i in range(n)])
            hidden = torch.from_numpy(~seen).to(DEVICE)
            c = torch.ones(n, dtype=torch.float64, device=DEVICE) if s["row_weight"] is None else s["row_weight"][lo:hi].double()
            for g in range(Hkv):
                total = torch.zeros(T + n, dtype=torch.float64, device=DEVICE)
                for h in range(g * rep, (g + 1) * rep):
                    z = s["q"][lo:hi, h].double() @ K[:, g].T * s["scale"]
                    z[:, T:][hidden] = -math.inf
                    lse[h, lo:hi] = torch.logsumexp(z, 1)
                    p = torch.exp(z - lse[h, lo:hi, None])
                    out[lo:hi, h] = p @ V[:, g]
                    total += c @ p
                w_new[lo:hi, g] = total[T:]
                grown = weight[ids, g].reshape(-1)
                grown[:T] += total[:T]
                weight[ids, g] = grown.reshape(-1, size)
        return {"out": out, "lse": lse, "weight_new": w_new, "weight": weight}
    if case["B"] * Hkv * (case.get("more", 0) + case.get("budget", 0)) > 4 << 20:
        return None
    # copies of given values: the tables that result, head by head on the host
    cu, table = s["cu"].tolist(), s["table"].cpu().numpy()
    k, v = s["k"].double().cpu().numpy(), s["v"].double().cpu().numpy()
    kn, vn = s["k_new"].double().cpu().numpy(), s["v_new"].double().cpu().numpy()
    w, pos, wn = s["weight"].cpu().numpy().astype(np.float64), s["position"].cpu().numpy(), s["weight_new"].cpu().numpy()
    length, seen = s["length"].cpu().numpy(), s["seen"].cpu().numpy()
    for b in range(case["B"]):
        n = cu[b + 1] - cu[b]
        t0, p0 = (0, 0) if s["fresh"] else (int(length[b]), int(seen[b]))
        slot = t0 + np.arange(n)
        pg, of = table[b, slot // size], slot % size
        k[pg, of], v[pg, of] = kn[cu[b]: cu[b + 1]], vn[cu[b]: cu[b + 1]]
        w[pg, :, of] = wn[cu[b]: cu[b + 1]]
        pos[pg, :, of] = (p0 + np.arange(n, dtype=np.int32))[:, None]
        length[b], seen[b] = t0 + n, p0 + n
        if case["op"] == "append" or length[b] <= case["budget"]:
            continue
        at = np.arange(length[b])
        pg, of = table[b, at // size], at % size
        for g in range(Hkv):
            safe = (pos[pg, g, of] < case["sinks"]) | (pos[pg, g, of] >= seen[b] - case["recent"])
            order = np.lexsort((at, -w[pg, g, of], ~safe))[: case["budget"]]
            kept = np.zeros(length[b], dtype=bool)
            kept[order] = True
            dst, src = at[(at < case["budget"]) & ~kept], at[(at >= case["budget"]) & kept]
            for x in (k, v):
                x[pg[dst], of[dst], g] = x[pg[src], of[src], g]
            for x in (w, pos):
                x[pg[dst], g, of[dst]] = x[pg[src], g, of[src]]
        length[b] = case["budget"]
    return {"k": k, "v": v, "weight": w, "position": pos, "length": length, "seen": seen}
