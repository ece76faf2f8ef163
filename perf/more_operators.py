"""The calls on a model's token distributions whose speed this library is held to: their sizes,
inputs, plain forms and 64-bit references.

Three operators on logits [rows, V], as scoring, policy-gradient and distillation programs use them:
  logprobs  log probability of each row's given token, the row's entropy, the greatest logit and the
            sum of exponentials (what the gradient needs), and the top alternatives
  grad      the gradient of those with respect to the logits
  distill   the divergence from a teacher of whom the top logits are known, by itself or with the
            gradient with respect to the student's logits

``listed()`` names the cases, ``draw()`` gives further ones of the same ranges, ``prepare()``
makes what a program holds before the call, ``run()`` makes the call, ``exact()`` evaluates the
definition in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # set by the tool that measures: False runs the plain forms

DEVICE = "cuda:0"
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------- cases
def _logprobs(name, dtype, rows, V, top=0, T=1.0, masked=0.0):
    """Scores of given tokens with entropy, and `top` alternatives; `masked`: the share of the
    vocabulary that a constrained decoder rules out (-inf), a whole row among several."""
    return {"name": name, "op": "logprobs", "dtype": dtype, "rows": rows, "V": V, "top": top, "T": T, "masked": masked}


def _grad(name, dtype, rows, V, top=0, T=1.0, entropy=True, masked=0.0):
    """Gradient of the log probabilities (of `top` alternatives too) and of the entropy."""
    return {"name": name, "op": "grad", "dtype": dtype, "rows": rows, "V": V, "top": top, "T": T,
            "entropy": entropy, "masked": masked}


def _distill(name, dtype, rows, V, K, T=1.0, tail=False, grads=True):
    """Divergence from K teacher logits a row (tail: from K log probabilities and their rest)."""
    return {"name": name, "op": "distill", "dtype": dtype, "rows": rows, "V": V, "K": K, "T": T,
            "tail": tail, "grads": grads}


def listed():
    return [
        # one decoded token with its 20 alternatives, as a serving program reports them: latency
        _logprobs("logprobs_decode1", "bf16", 1, 152064, top=20),
        # a decoding batch under a grammar: nine tenths of an odd vocabulary masked, fp32, 5 alternatives
        _logprobs("logprobs_masked61_f32", "f32", 61, 50257, top=5, T=0.7, masked=0.9),
        # a teacher scores a chunk of ragged prompts for distillation: 64 alternatives a token
        _logprobs("logprobs_top64", "bf16", 1537, 152064, top=64),
        # the sampled tokens of rollouts scored under the policy that is trained, no alternatives
        _logprobs("logprobs_rl4096", "bf16", 4096, 128256),
        # policy gradient with an entropy bonus over the same tokens: the largest call
        _grad("grad_rl4096", "bf16", 4096, 128256, T=1.0),
        # a short sequence: the gradient of a handful of rows
        _grad("grad_33", "bf16", 33, 152064, entropy=False),
        # fp32 logits of an odd vocabulary, gradients of alternatives too, sampled with a temperature
        _grad("grad_top_f32", "f32", 501, 32001, top=8, T=0.8),
        # a student's training step: loss and gradient, the teacher's top 64 renormalised
        _distill("distill_train", "bf16", 2048, 128256, 64, T=2.0),
        # the same with the teacher's remaining mass as one bucket
        _distill("distill_tail", "bf16", 1021, 152064, 32, tail=True),
        # a small fp32 student
        _distill("distill_small_f32", "f32", 130, 32000, 16, tail=True),
        # validation: the loss alone
        _distill("distill_eval", "bf16", 1024, 152064, 100, grads=False),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges, at most the largest listed one's work."""
    op = rng.choice(["logprobs", "grad", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    V = rng.choice([32000, 128256, 152064, _between(rng, 1000, 262144), _between(rng, 1000, 262144)])
    most = (1 << 28) // V  # rows of a case, half of that in fp32
    rows = _between(rng, 1, max(1, min(8192, most if dtype == "bf16" else most // 2)))
    T = rng.choice([1.0, 1.0, 0.6, 2.0])
    masked = rng.choice([0.0, 0.0, 0.5, 0.99])
    if op == "logprobs":
        return _logprobs(None, dtype, rows, V, rng.choice([0, 1, 5, 20, 64, 128]), T, masked)
    if op == "grad":
        return _grad(None, dtype, rows, V, rng.choice([0, 0, 5, 20]), T, rng.random() < 0.5, masked)
    return _distill(None, dtype, rows, V, rng.choice([1, 8, 20, 64, 128]), T, rng.random() < 0.5, rng.random() < 0.7)


# ------------------------------------------------------------------------ inputs
_CHUNK = 1 << 26  # logits that are made (or looked at in 64 bits) at a time


def _chunks(rows, V):
    step = max(1, _CHUNK // V)
    return [(lo, min(rows, lo + step)) for lo in range(0, rows, step)]


def _padded_rows(rows, V, dtype):
    """[rows, V] whose rows start on 16 bytes; what lies between them is no logit."""
    per = 16 // _SIZE[dtype]
    wide = torch.full((rows, -(-V // per) * per), 30.0, dtype=_TYPES[dtype], device=DEVICE)
    return wide[:, :V]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rows, V, T, op = case["rows"], case["V"], case["T"], case["op"]
    uniform = lambda *shape: torch.rand(shape, generator=gen, device=DEVICE)  # noqa: E731
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEVICE)  # noqa: E731
    logits = _padded_rows(rows, V, case["dtype"])
    target = torch.empty(rows, dtype=torch.int32, device=DEVICE)
    K = case.get("K", 0)
    ids = torch.empty(rows, K, dtype=torch.int32, device=DEVICE)
    teacher = torch.empty(rows, K, device=DEVICE)
    for lo, hi in _chunks(rows, V):
        n = hi - lo
        # rows from flat to sharp, half of them sure of one token
        x = normal(n, V) * (1.0 + 2.0 * uniform(n, 1))
        sure = torch.randint(0, V, (n, 1), generator=gen, device=DEVICE)
        x.scatter_add_(1, sure, torch.where(uniform(n, 1) < 0.5, 6.0 + 8.0 * uniform(n, 1), 0.0))
        if case.get("masked"):
            x = torch.where(uniform(n, V) < case["masked"], -math.inf, x)
        x = x.to(_TYPES[case["dtype"]])
        if case.get("masked") and lo <= rows // 2 < hi and rows >= 4:
            x[rows // 2 - lo] = -math.inf  # a mask that leaves a row empty
        logits[lo:hi] = x
        if op == "distill":
            z = x.float() * 0.9 + 0.8 * normal(n, V)
            top = torch.topk(z, K, dim=1)
            ids[lo:hi] = top.indices.int()
            teacher[lo:hi] = (top.values / T - torch.logsumexp(z / T, 1, keepdim=True)) if case["tail"] else top.values
        else:  # the sampled token
            noise = -torch.log(-torch.log(uniform(n, V).clamp_(1e-20, 1 - 1e-7)))
            target[lo:hi] = torch.argmax(x.float() / T + noise, dim=1).int()
    s = {"case": case, "logits": logits}
    if op == "distill":
        if rows >= 8:  # rows with fewer alternatives, and one without any (padding)
            ids[::7, (K + 1) // 2:] = -1
            ids[rows // 2] = -1
        s.update(ids=ids, teacher=teacher, weight=(0.5 + uniform(rows)) / rows)
        return s
    if rows >= 8:
        target[::11] = -1  # prompt tokens that are not scored
    s["target"] = target
    if op == "grad":
        norm, entropy, top_ids = [], [], []
        for lo, hi in _chunks(rows, V):
            z = logits[lo:hi].double()
            m = z.amax(1)
            m0 = torch.where(m == -math.inf, 0.0, m)
            e = torch.exp((z - m0[:, None]) / T)
            total = e.sum(1)
            log = torch.log(torch.where(total == 0, 1.0, total))
            lp = (z - m0[:, None]) / T - log[:, None]
            p = e / torch.where(total == 0, 1.0, total)[:, None]
            entropy.append(-torch.where(p > 0, p * lp, 0.0).sum(1).float())
            norm.append(torch.stack([m, total], 1).float())
            if case["top"]:
                top_ids.append(torch.topk(z, case["top"], dim=1).indices.int())
        s.update(norm=torch.cat(norm), entropy=torch.cat(entropy), g_logprob=normal(rows) / rows,
                 g_entropy=0.05 * normal(rows) / rows if case["entropy"] else None, top_ids=None, top_logprobs=None, g_top=None)
        if case["top"]:
            s["top_ids"] = torch.cat(top_ids)
            s["g_top"] = normal(rows, case["top"]) / rows
    return s


# ------------------------------------------------------------------- plain forms
def _statistics(z, T):
    """Greatest logit, the same with 0 for an empty row, exponentials, their sum, log of the sum."""
    m = z.amax(1)
    m0 = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp((z - m0[:, None]) / T)
    total = e.sum(1)
    return m, m0, e, total, torch.log(torch.where(total == 0, 1.0, total))


def _plain_logprobs(s):
    T, k = s["case"]["T"], s["case"]["top"]
    z = s["logits"].float()
    m, m0, e, total, log = _statistics(z, T)
    lp = (z - m0[:, None]) / T - log[:, None]
    entropy = -torch.where(e > 0, e * lp, 0.0).sum(1) / torch.where(total == 0, 1.0, total)
    t = s["target"].long()
    picked = lp.gather(1, t.clamp(min=0)[:, None])[:, 0]
    out = {"logprob": torch.where(t < 0, 0.0, picked), "entropy": entropy, "norm": torch.stack([m, total], 1)}
    if k:
        # whole-number keys: the greater logit first, among equals the lower token
        bits = (z + 0.0).view(torch.int32)
        order = (bits ^ (bits >> 31 & 0x7FFFFFFF)).long()
        key = order * (1 << 32) + (z.shape[1] - 1 - torch.arange(z.shape[1], device=DEVICE))
        ids = torch.topk(key, k, dim=1).indices
        out["top_ids"] = ids.int()
        out["top_logprobs"] = lp.gather(1, ids)
    return out


def _plain_grad(s):
    T = s["case"]["T"]
    z = s["logits"].float()
    m, total = s["norm"][:, 0], s["norm"][:, 1]
    m0, some = torch.where(m == -math.inf, 0.0, m), torch.where(total == 0, 1.0, total)
    lp = (z - m0[:, None]) / T - torch.log(some)[:, None]
    p = torch.exp((z - m0[:, None]) / T) / some[:, None]
    t = s["target"].long()
    there = total > 0
    g = torch.where((t >= 0) & there, s["g_logprob"], 0.0)
    pull = g
    if s["g_top"] is not None:
        pull = pull + torch.where(there[:, None], s["g_top"], 0.0).sum(1)
    dz = -pull[:, None] * p
    if s["g_entropy"] is not None:
        dz = dz - torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0) * s["g_entropy"][:, None]
    dz.scatter_add_(1, t.clamp(min=0)[:, None], g[:, None])
    if s["g_top"] is not None:
        dz.scatter_add_(1, s["top_ids"].long(), torch.where(there[:, None], s["g_top"], 0.0))
    return {"grad": (dz / T).to(s["logits"].dtype)}


def _plain_distill(s):
    case = s["case"]
    T = case["T"]
    z = s["logits"].float()
    m, m0, e, total, log = _statistics(z, T)
    some, ids = s["ids"] >= 0, s["ids"].long().clamp(min=0)
    x = torch.where(some, s["teacher"], -math.inf)
    if case["tail"]:
        q = torch.exp(x)
        rest = torch.where(some.any(1), (1.0 - q.double().sum(1)).clamp(min=0.0).float(), 0.0)
    else:
        top = x.amax(1, keepdim=True)
        q = torch.exp((x - torch.where(top == -math.inf, 0.0, top)) / T)
        q = q / torch.where(some.any(1), q.sum(1), 1.0)[:, None]
        rest = torch.zeros_like(m)
    lp = ((z - m0[:, None]) / T - log[:, None]).gather(1, ids)
    loss = torch.where(q > 0, q * (torch.log(torch.where(q > 0, q, 1.0)) - lp), 0.0).sum(1)
    spot = torch.where(some, ids, z.shape[1])  # entries that are none land past the end
    inside = torch.zeros(z.shape[0], z.shape[1] + 1, dtype=torch.bool, device=DEVICE).scatter_(1, spot, True)[:, :-1]
    outside = torch.where(inside, 0.0, e).sum(1)
    if case["tail"]:
        part = torch.log(torch.where(rest > 0, rest, 1.0)) - (torch.log(outside) - log)
        loss = loss + torch.where(rest > 0, rest * part, 0.0)
    if not case["grads"]:
        return {"loss": loss}
    p = e / total[:, None]
    dz = p * (q.sum(1) + rest)[:, None]
    if case["tail"]:
        # rest * p / p_tail with both sums over the same exponentials
        dz = dz - torch.where(inside | (rest == 0)[:, None], 0.0, e * (rest / outside)[:, None])
    wide = torch.cat([dz, torch.zeros_like(m)[:, None]], 1).scatter_add_(1, spot, -q)
    return {"loss": loss, "grad": (wide[:, :-1] * (s["weight"] / T)[:, None]).to(s["logits"].dtype)}


# --------------------------------------------------------------------- the calls
_ctx = None


def _own_run(s):
    import paper_2608_15592_gb300 as estp
    global _ctx
    if _ctx is None:
        _ctx = estp.Context(0)
    case = s["case"]
    if case["op"] == "logprobs":
        lp = _ctx.token_logprobs(s["logits"], s["target"], top_k=case["top"], temperature=case["T"])
        out = {"logprob": lp.logprob, "entropy": lp.entropy, "norm": lp.norm}
        if case["top"]:
            out.update(top_ids=lp.top_ids, top_logprobs=lp.top_logprobs)
        return out
    if case["op"] == "grad":
        lp = estp.TokenLogprobs(None, s["entropy"], s["norm"], s["top_ids"], None, case["T"])
        return {"grad": _ctx.token_logprobs_grad(s["logits"], s["target"], lp, grad_logprob=s["g_logprob"],
                                                 grad_entropy=s["g_entropy"], grad_top=s["g_top"])}
    if not case["grads"]:
        return {"loss": _ctx.distill_loss(s["logits"], s["ids"], s["teacher"], temperature=case["T"], tail=case["tail"],
                                          grads=False)}
    loss, grad = _ctx.distill_loss(s["logits"], s["ids"], s["teacher"], temperature=case["T"], tail=case["tail"],
                                   row_weight=s["weight"])
    return {"loss": loss, "grad": grad}


def run(state):
    if own:
        return _own_run(state)
    return {"logprobs": _plain_logprobs, "grad": _plain_grad, "distill": _plain_distill}[state["case"]["op"]](state)


# -------------------------------------------------------------------------- work
def work(case):
    rows, n = case["rows"], case["rows"] * case["V"]
    read = n * _SIZE[case["dtype"]]
    if case["op"] == "logprobs":
        # scale, exponential, two sums and a comparison an element
        return {"bytes": read + rows * (4 + 16 + 8 * case["top"]), "flops": 6 * n}
    if case["op"] == "grad":
        return {"bytes": 2 * read + rows * (20 + 8 * case["top"]), "flops": 6 * n}
    return {"bytes": (2 if case["grads"] else 1) * read + rows * (8 + 8 * case["K"]), "flops": (9 if case["grads"] else 5) * n}


# -------------------------------------------------------------------------- exact
def _exact_logprobs(s, lo, hi):
    T, k = s["case"]["T"], s["case"]["top"]
    raw = s["logits"][lo:hi]
    y = raw.double() / T
    lse = torch.logsumexp(y, 1)
    empty = lse == -math.inf
    lp = torch.where(empty[:, None], -math.inf, y - lse[:, None])
    p = torch.exp(lp)
    t = s["target"][lo:hi].long()
    at = torch.arange(hi - lo, device=DEVICE)
    out = {"logprob": torch.where(t < 0, 0.0, lp[at, t.clamp(min=0)]), "entropy": -torch.nan_to_num(p * lp, nan=0.0).sum(1),
           "norm": torch.stack([raw.double().amax(1), torch.where(empty, 0.0, torch.exp(lse - y.amax(1)))], 1)}
    if k:
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :k]
        out.update(top_ids=order, top_logprobs=torch.take_along_dim(lp, order, 1))
    return out


def _exact_grad(s, lo, hi):
    T = s["case"]["T"]
    y = s["logits"][lo:hi].double() / T
    lse = torch.logsumexp(y, 1)
    empty = lse == -math.inf
    lp = torch.where(empty[:, None], -math.inf, y - lse[:, None])
    p = torch.exp(lp)
    H = -torch.nan_to_num(p * lp, nan=0.0).sum(1)
    grad = torch.zeros_like(p)
    at = torch.arange(hi - lo, device=DEVICE)
    t = s["target"][lo:hi].long()
    terms = [(t.clamp(min=0), torch.where(t < 0, 0.0, s["g_logprob"][lo:hi].double()))]
    for j in range(s["case"]["top"]):
        terms.append((s["top_ids"][lo:hi, j].long(), s["g_top"][lo:hi, j].double()))
    for token, g in terms:  # d ln p_t / dz = ([v = t] - p) / T
        g = torch.where(empty, 0.0, g)
        grad -= g[:, None] * p
        grad[at, token] += g
    if s["g_entropy"] is not None:
        grad -= s["g_entropy"][lo:hi].double()[:, None] * torch.nan_to_num(p * (lp + H[:, None]), nan=0.0)
    return {"grad": grad / T}


def _exact_distill(s, lo, hi):
    case = s["case"]
    T = case["T"]
    y = s["logits"][lo:hi].double() / T
    ids, x = s["ids"][lo:hi], s["teacher"][lo:hi].double()
    n, V = y.shape
    lp = y - torch.logsumexp(y, 1, keepdim=True)
    p = torch.exp(lp)
    q = torch.zeros(n, V, dtype=torch.float64, device=DEVICE)  # the teacher over the vocabulary
    row, col = torch.nonzero(ids >= 0, as_tuple=True)
    value = torch.exp(x) if case["tail"] else torch.softmax(torch.where(ids >= 0, x / T, -math.inf), 1)
    q[row, ids[row, col].long()] = value[row, col]
    named = torch.zeros(n, V, dtype=torch.bool, device=DEVICE)
    named[row, ids[row, col].long()] = True
    loss = (torch.special.xlogy(q, q) - q * lp).sum(1)
    grad = p * q.sum(1, keepdim=True) - q
    if case["tail"]:
        rest = torch.where(named.any(1), 1.0 - q.sum(1), 0.0).clamp(min=0.0)
        other = torch.where(named, -math.inf, lp)
        log_tail = torch.logsumexp(other, 1)
        loss += torch.where(rest > 0, rest * (torch.log(torch.where(rest > 0, rest, 1.0)) - log_tail), 0.0)
        grad += rest[:, None] * (p - torch.exp(other - log_tail[:, None]))
    if not case["grads"]:
        return {"loss": loss}
    return {"loss": loss, "grad": grad * (s["weight"][lo:hi].double() / T)[:, None]}


def exact(case, seed):
    s = prepare(case, seed)
    form = {"logprobs": _exact_logprobs, "grad": _exact_grad, "distill": _exact_distill}[case["op"]]
    if case["rows"] * case["V"] > 1 << 28 and case["op"] != "logprobs":
        return None  # the gradient in 64 bits beside its parts
    parts = [form(s, lo, hi) for lo, hi in _chunks(case["rows"], case["V"])]
    return {name: torch.cat([part[name] for part in parts]) for name in parts[0]}
