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
