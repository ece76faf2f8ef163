"""What the calls on rows of logits refuse, before any work is enqueued (CPU): the C entry points on a context
that is never looked into, and the binding's own checks."""
import ctypes

import pytest
import torch

import paper_2608_15592_gb300 as estp

BF = estp.ESTP_BF16


class _Library:
    """estp.lib for a context that was not created (there is no GPU here): a zeroed one."""

    def __init__(self):
        self.room = ctypes.create_string_buffer(4096)
        self.ctx = ctypes.addressof(self.room)


P = 4096  # an address that is aligned and never read


def _logprobs(**change):
    a = dict(ctx=_Library().ctx, z=P, dtype=BF, rows=4, V=100, ld=104, targets=P, T=1.0, k=5, lp=P, H=P, norm=P, ids=P, tops=P)
    a.update(change)
    return estp.lib.estp_token_logprobs(a["ctx"], a["z"], a["dtype"], a["rows"], a["V"], a["ld"], a["targets"], a["T"], a["k"],
                                        a["lp"], a["H"], a["norm"], a["ids"], a["tops"], None)


def _grad(**change):
    a = dict(ctx=_Library().ctx, z=P, dtype=BF, rows=4, V=100, ld=104, norm=P, H=P, targets=P, T=1.0, k=5, ids=P, g=P, gH=P, gl=P,
             ga=P, out=1 << 20, ldo=104)
    a.update(change)
    return estp.lib.estp_token_logprobs_grad(a["ctx"], a["z"], a["dtype"], a["rows"], a["V"], a["ld"], a["norm"], a["H"],
                                             a["targets"], a["T"], a["k"], a["ids"], a["g"], a["gH"], a["gl"], a["ga"],
                                             a["out"], a["ldo"], None)


def _distill(**change):
    a = dict(ctx=_Library().ctx, z=P, dtype=BF, rows=4, V=100, ld=104, ids=P, x=P, K=5, T=1.0, tail=0, w=P, loss=P, out=1 << 20, ldo=104)
    a.update(change)
    return estp.lib.estp_distill_loss(a["ctx"], a["z"], a["dtype"], a["rows"], a["V"], a["ld"], a["ids"], a["x"], a["K"], a["T"],
                                      a["tail"], a["w"], a["loss"], a["out"], a["ldo"], None)


ALL = [dict(ctx=None), dict(dtype=7), dict(rows=-1), dict(V=0), dict(ld=96), dict(ld=103), dict(z=P + 2), dict(z=None), dict(T=0.0),
       dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-9)]


@pytest.mark.parametrize("change", ALL, ids=str)
@pytest.mark.parametrize("call", [_logprobs, _grad, _distill])
def test_refused_by_all(call, change):
    assert call(**change) == estp.ESTP_ERR_INVALID_ARG
    assert estp.lib.estp_last_error(None)


@pytest.mark.parametrize("change", [dict(k=-1), dict(k=101), dict(targets=None), dict(ids=None), dict(norm=P + 4)], ids=str)
def test_refused_log_probabilities(change):
    assert _logprobs(**change) == estp.ESTP_ERR_INVALID_ARG


GRAD_PLACES = [dict(out=P + 8), dict(ldo=99), dict(ldo=103), dict(out=P, ldo=112), dict(out=P + 16), dict(out=P + 208),
               dict(z=1 << 20, out=(1 << 20) - 3 * 208 - 192)]


@pytest.mark.parametrize("change", [dict(norm=None), dict(norm=P + 4), dict(out=None), dict(targets=None), dict(H=None), dict(ids=None),
                                    dict(k=0), dict(k=101)] + GRAD_PLACES, ids=str)
def test_refused_gradients(change):
    assert _grad(**change) == estp.ESTP_ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(K=0), dict(ids=None), dict(x=None), dict(loss=None)] + GRAD_PLACES, ids=str)
def test_refused_distillation(change):
    assert _distill(**change) == estp.ESTP_ERR_INVALID_ARG


def test_unsupported():
    assert _logprobs(k=129, V=1000, ld=1000) == estp.ESTP_ERR_UNSUPPORTED
    assert _grad(k=129, V=1000, ld=1000, ldo=1000) == estp.ESTP_ERR_UNSUPPORTED
    assert _distill(K=129, V=1000, ld=1000, ldo=1000) == estp.ESTP_ERR_UNSUPPORTED
    for call in (_logprobs, _grad, _distill):
        big = (1 << 26) + 8
        assert call(V=big, ld=big, ldo=big) == estp.ESTP_ERR_UNSUPPORTED


def test_no_rows_is_no_work():
    for call in (_logprobs, _grad, _distill):
        assert call(rows=0, z=None) == estp.ESTP_OK


def _context():
    ctx = estp.Context.__new__(estp.Context)
    ctx._lib, ctx._h, ctx.device = estp.lib, None, -1  # a CPU tensor's get_device()
    return ctx


def test_the_binding_refuses():
    ctx, x = _context(), torch.zeros(4, 96, dtype=torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int32)
    norm, g = torch.zeros(4, 2), torch.zeros(4)
    lp = estp.TokenLogprobs(None, g, norm, None, None)
    bad = [
        lambda: ctx.token_logprobs(x[0], t),
        lambda: ctx.token_logprobs(x.t(), t),
        lambda: ctx.token_logprobs(x, t.long()),
        lambda: ctx.token_logprobs(x, t[:3]),
        lambda: ctx.token_logprobs(x, t, V=97),
        lambda: ctx.token_logprobs(x, t, V=0),
        lambda: ctx.token_logprobs_grad(x, t, lp, grad_logprob=g.double()),
        lambda: ctx.token_logprobs_grad(x, t, lp, grad_logprob=g[:2]),
        lambda: ctx.token_logprobs_grad(x, t, lp, grad_top=torch.zeros(4, 3)),
        lambda: ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, out=torch.zeros(4, 96)),
        lambda: ctx.token_logprobs_grad(x, t, lp, grad_logprob=g, out=torch.zeros(4, 90, dtype=torch.bfloat16)),
        lambda: ctx.token_logprobs_grad(x, t, estp.TokenLogprobs(None, g, norm[:3], None, None), grad_logprob=g),
        lambda: ctx.distill_loss(x, torch.zeros(4, 3), torch.zeros(4, 3)),
        lambda: ctx.distill_loss(x, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 2)),
        lambda: ctx.distill_loss(x, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3), row_weight=g[:1]),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ctx.token_logprobs(torch.zeros(4, 96, dtype=torch.float16), t)
    ctx.device = 0
    with pytest.raises(ValueError):
        ctx.token_logprobs(x, t)
