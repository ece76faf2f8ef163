"""README's loop of a cache from the prompt on, run as it stands (GPU): the prompt's weights that it appends
are on the scale on which cache_attention goes on adding to them.  A weight of (KV head, token) is the sum,
undivided, of the attention that the query heads of the KV head gave the token; the importance has the mean
over all heads, so each KV head starts from the mean over the heads times its Hq / Hkv."""
import os
import re

import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2608_15592_gb300 as estp
from gpu_util import assert_importance

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


class _Recorder:
    """A context that keeps the weights each append is given."""

    def __init__(self, ctx):
        self.ctx, self.appended = ctx, []

    def __getattr__(self, name):
        return getattr(self.ctx, name)

    def cache_append(self, *args, **kw):
        self.appended.append(kw["weight"].clone())
        return self.ctx.cache_append(*args, **kw)


def test_loop_keeps_one_scale(cuda_lib):
    blocks = re.findall(r"```python\n(.*?)```", open(README).read(), flags=re.S)
    code, = [b for b in blocks if "estp.KVCache(" in b]
    rng = np.random.default_rng(0)
    Hq, Hkv, d, page = 8, 2, 128, 16
    lens, drafts = [150, 61, 197], [3, 1, 5]
    sumT, m, B = sum(lens), sum(drafts), len(lens)
    rand = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, d))).to(torch.bfloat16).cuda()  # noqa: E731
    ints = lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)).cuda()  # noqa: E731
    Q, K, V = rand(sumT, Hq), rand(sumT, Hkv), rand(sumT, Hkv)
    cu = ints(np.concatenate([[0], np.cumsum(lens)]))
    ctx = _Recorder(cuda_lib.Context(0))
    ctx.attn_importance(Q, K, cu, max(lens))
    S = ctx.attn_importance_finalize(1, sumT)  # the pooling's
    per = -(-(max(lens) + 16) // page)
    pool = torch.full((B * per, page, Hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    have = dict(
        estp=estp, ctx=ctx, Q=Q, K=K, V=V, S=S, cu=cu, max_seqlen=max(lens), sumT=sumT, Hq=Hq, Hkv=Hkv, budget=96,
        k_pages=pool, v_pages=pool.clone(), page_table=ints(rng.permutation(B * per).reshape(B, per)),
        length=ints([0] * B), seen=ints([0] * B), weight=torch.full((B * per, Hkv, page), float("nan"), device="cuda"),
        position=torch.full((B * per, Hkv, page), -1, dtype=torch.int32, device="cuda"),
        q=rand(m, Hq), k=rand(m, Hkv), v=rand(m, Hkv), cu_rows=ints([0, 3, 4, 9]), max_rows=5,
        bits=R.bits_of([R.tree(rng, n) for n in drafts], 1), draft_prob=torch.ones(m, device="cuda"),
        accepted=ints([0, 3, 4, 5]), cu_accepted=ints([0, 1, 2, 4]))
    exec(code, have)
    ctx.sync_status()
    first, second = ctx.appended
    want = np.zeros((sumT, Hkv))
    lo = 0
    for T in lens:
        for h in range(Hq):
            q, k = R.host(Q)[lo:lo + T, h], R.host(K)[lo:lo + T, h // (Hq // Hkv)]
            z = np.where(np.tril(np.ones((T, T), bool)), q @ k.T / np.sqrt(d), -np.inf)
            p = np.exp(z - z.max(1, keepdims=True))
            want[lo:lo + T] += ((p / p.sum(1, keepdims=True)).sum(0) / Hkv)[:, None]
        lo += T
    assert_importance(first.cpu().numpy(), want)
    # a draft gives each of the KV head's query heads a probability, as a token of the prompt did
    assert torch.all(second >= 0) and torch.all(second <= max(drafts) * Hq // Hkv)
    assert have["cache"].length.tolist() == [97, 62, 98] and have["cache"].seen.tolist() == [151, 62, 199]
    ctx.close()
