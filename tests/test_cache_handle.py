"""KVCache follows its tensors: what a program replaces is what the next call gets.  The kernels are handed
addresses and sizes of one struct, which is read here as the library reads it; no GPU is needed for that."""
import ctypes

import pytest
import torch

import paper_2608_15592_gb300 as estp


def _tensors(n_pages=6, page=8, Hkv=2, d=64, B=2, per=3, dtype=torch.bfloat16):
    return {"k": torch.zeros(n_pages, page, Hkv, d, dtype=dtype), "v": torch.zeros(n_pages, page, Hkv, d, dtype=dtype),
            "page_table": torch.zeros(B, per, dtype=torch.int32), "length": torch.zeros(B, dtype=torch.int32),
            "seen": torch.zeros(B, dtype=torch.int32), "weight": torch.zeros(n_pages, Hkv, page),
            "position": torch.zeros(n_pages, Hkv, page, dtype=torch.int32)}


class _Recorder:
    """A library whose calls keep what they are given."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, estp._KVCache.from_buffer_copy(ctypes.string_at(args[1], ctypes.sizeof(estp._KVCache))), args))
            return estp.ESTP_OK
        return call


def _context():
    ctx = estp.Context.__new__(estp.Context)
    ctx._lib, ctx._h = _Recorder(), None
    return ctx


class _Stream:
    cuda_stream = 0


def _evict(ctx, cache):
    ctx.cache_evict(cache, 4, stream=_Stream())
    return ctx._lib.calls[-1]


def _same(c, t):
    assert (c.k, c.v, c.page_table) == (t["k"].data_ptr(), t["v"].data_ptr(), t["page_table"].data_ptr())
    assert (c.weight, c.position) == tuple(None if t[n] is None else t[n].data_ptr() for n in ("weight", "position"))
    assert (c.n_pages, c.page_size, c.Hkv, c.head_dim) == tuple(t["k"].shape)
    assert (c.page_stride, c.slot_stride, c.head_stride) == t["k"].stride()[:3]
    assert c.max_pages == t["page_table"].shape[1]


def test_a_longer_page_table_is_used():
    t = _tensors()
    ctx, cache = _context(), estp.KVCache(**t)
    _same(_evict(ctx, cache)[1], t)
    assert cache.max_slots == 48
    t["page_table"] = torch.zeros(2, 5, dtype=torch.int32)
    cache.page_table = t["page_table"]
    _same(_evict(ctx, cache)[1], t)
    assert cache.max_slots == 48  # the pool's
    cache.weight = t["weight"] = None
    _same(_evict(ctx, cache)[1], t)
    assert cache.max_slots == 80


@pytest.mark.parametrize("name", ["k", "v", "weight", "position"])
def test_every_replaced_array_is_used(name):
    t = _tensors()
    ctx, cache = _context(), estp.KVCache(**t)
    t[name] = t[name].clone()
    setattr(cache, name, t[name])
    _same(_evict(ctx, cache)[1], t)


def test_a_larger_pool_replaced_array_by_array():
    ctx, cache = _context(), estp.KVCache(**_tensors())
    t = _tensors(n_pages=20, B=3, per=7, dtype=torch.float32)
    for name, x in t.items():
        setattr(cache, name, x)
    _, c, args = _evict(ctx, cache)
    _same(c, t)
    assert c.dtype == estp.ESTP_F32 and cache.B == 3 and args[2] == t["length"].data_ptr() and args[5] == 3
    assert cache.max_slots == 160


@pytest.mark.parametrize("name,value", [
    ("length", torch.zeros(1, dtype=torch.int32)), ("length", torch.zeros(2, dtype=torch.int64)),
    ("seen", torch.zeros(3, dtype=torch.int32)), ("seen", torch.zeros(2)),
    ("page_table", torch.zeros(2, 3, dtype=torch.int64)), ("page_table", torch.zeros(3, 3, dtype=torch.int32)),
    ("page_table", torch.zeros(3, 2, dtype=torch.int32).T), ("weight", torch.zeros(5, 2, 8)),
    ("position", torch.zeros(6, 2, 8)), ("k", torch.zeros(6, 8, 2, 64)),
])
def test_a_replacement_that_does_not_fit_is_refused(name, value):
    ctx, cache = _context(), estp.KVCache(**_tensors())
    setattr(cache, name, value)
    kn = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    q, cu = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: ctx.cache_evict(cache, 4, stream=_Stream()),
                 lambda: ctx.cache_append(cache, kn, kn, cu, stream=_Stream()),
                 lambda: ctx.cache_attention(cache, q, kn, kn, cu, 1, stream=_Stream())):
        with pytest.raises(ValueError):
            call()
    assert ctx._lib.calls == []


def test_a_bound_of_the_slots_stays():
    cache = estp.KVCache(**_tensors(), max_slots=20)
    cache.page_table = torch.zeros(2, 9, dtype=torch.int32)
    assert cache.max_slots == 20
    cache.max_slots = 30
    assert cache.max_slots == 30


def _new(n, Hkv, d=64, extra=0):
    """Rows of a wider array, n of them."""
    return torch.zeros(n, Hkv + extra, d, dtype=torch.bfloat16)[:, :Hkv]


@pytest.mark.parametrize("n,Hkv", [(1, 2), (0, 2), (1, 1)])
def test_strides_that_are_never_stepped_by_need_not_agree(n, Hkv):
    """One row: K from a fused projection, V of its own (a batch of one in decoding)."""
    ctx, cache = _context(), estp.KVCache(**_tensors(B=1, Hkv=Hkv))
    kn, vn, q = _new(n, Hkv, extra=5), _new(n, Hkv), _new(n, 2 * Hkv)
    cu = torch.zeros(2, dtype=torch.int32)
    ctx.cache_append(cache, kn, vn, cu, stream=_Stream())
    ctx.cache_attention(cache, q, kn, vn, cu, 1, stream=_Stream())
    ctx.cache_attention(cache, q, vn, kn, cu, 1, stream=_Stream())
    assert [c[2][9] for c in ctx._lib.calls[:1]] == [Hkv * 64] and [c[2][10] for c in ctx._lib.calls[1:]] == [Hkv * 64] * 2


def test_rows_of_one_head():
    """A single KV head: the heads' stride is never stepped by, the rows' is."""
    ctx, cache = _context(), estp.KVCache(**_tensors(Hkv=1))
    cu = torch.zeros(3, dtype=torch.int32)
    wide = torch.zeros(3, 128, dtype=torch.bfloat16)
    kn = wide[:, :64].unsqueeze(1)                   # strides 128, 64, 1
    vn = wide[:, 64:].reshape(3, 1, 64).as_strided((3, 1, 64), (128, 7, 1))
    ctx.cache_append(cache, kn, vn, cu, stream=_Stream())
    assert ctx._lib.calls[-1][2][9] == 128


@pytest.mark.parametrize("kn,vn", [(_new(2, 2, extra=1), _new(2, 2)), (_new(2, 2), _new(3, 2)), (_new(2, 2), _new(2, 2).float()),
                                   (_new(2, 2), torch.zeros(2, 64, 2, dtype=torch.bfloat16).transpose(1, 2)),
                                   (torch.zeros(1, 64, 2, dtype=torch.bfloat16).transpose(1, 2), _new(1, 2)),
                                   (_new(1, 2), torch.zeros(1, 64, 2, dtype=torch.bfloat16).transpose(1, 2))])
def test_rows_that_do_not_agree_are_refused(kn, vn):
    ctx, cache = _context(), estp.KVCache(**_tensors(B=1))
    with pytest.raises(ValueError):
        ctx.cache_append(cache, kn, vn, torch.zeros(2, dtype=torch.int32), stream=_Stream())
    assert ctx._lib.calls == []
