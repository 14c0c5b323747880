"""The class losses refuse arguments that do not fit, before anything is launched.  CPU only (see test_gate_validation)."""
import ctypes
import math

import pytest
import torch

from paper_2308_10037_b200 import api
from test_gate_validation import BF, F64, I32, I64, L, NULL, P, ctx, dead, fake   # noqa: F401 (fixtures)

X, Y, R = (6, 8), 6, 6


def test_well_formed_calls_get_through(ctx):
    x, y, r = fake(X), fake(Y, I64), fake(R)
    ctx.logp(x, y)
    ctx.logp(fake(X, BF), fake(Y, I32), scale=0.5, ignore_id=0)
    ctx.logp_grad(x, y, r, r)
    ctx.logp_grad(x, y, r, r, out=fake(X))
    ctx.policy_loss(x, y, r)
    ctx.policy_loss(fake(X, BF), y, r, r, r, r, kl_coef=0.1, norm=3.0, grad=False)
    ctx.pref_loss(x, y, fake(5, I32), fake(4), fake(2))
    ctx.pref_loss(fake(X, BF), y, fake(5, I64), average=True)
    ctx.distill_loss(x, fake((6, 2), I32), fake((6, 2)))
    ctx.distill_loss(fake(X, BF), fake((6, 2), I64), fake((6, 2), BF), r, r)
    assert ctx.rec.calls == ["lr_logp", "lr_logp_bf16", "lr_logp_grad", "lr_logp_grad", "lr_policy_loss", "lr_policy_loss_bf16", "lr_pref_loss",
                             "lr_pref_loss_bf16", "lr_distill_loss", "lr_distill_loss_bf16"]


CALLS = {
    "logits of doubles": lambda c: c.logp(fake(X, F64), fake(Y, I64)),
    "logits of half": lambda c: c.policy_loss(fake(X, torch.float16), fake(Y, I64), fake(R)),
    "logits transposed": lambda c: c.logp(fake((8, 6)).t(), fake(Y, I64)),
    "logits of three dimensions": lambda c: c.logp(fake((2, 3, 8)), fake(Y, I64)),
    "logits on another device": lambda c: c.logp(fake(X, index=1), fake(Y, I64)),
    "targets of floats": lambda c: c.logp(fake(X), fake(Y)),
    "fewer targets": lambda c: c.logp(fake(X), fake(5, I64)),
    "targets of two dimensions": lambda c: c.logp(fake(X), fake((2, 3), I64)),
    "targets on another device": lambda c: c.logp(fake(X), fake(Y, I64, 1)),
    "no lse": lambda c: c.logp_grad(fake(X), fake(Y, I64), None, fake(R)),
    "lse too short": lambda c: c.logp_grad(fake(X), fake(Y, I64), fake(5), fake(R)),
    "dlogp of bfloat16": lambda c: c.logp_grad(fake(X), fake(Y, I64), fake(R), fake(R, BF)),
    "gradient of another type": lambda c: c.logp_grad(fake(X), fake(Y, I64), fake(R), fake(R), out=fake(X, BF)),
    "gradient of another shape": lambda c: c.policy_loss(fake(X), fake(Y, I64), fake(R), out=fake((6, 9))),
    "no advantages": lambda c: c.policy_loss(fake(X), fake(Y, I64), None),
    "advantages too long": lambda c: c.policy_loss(fake(X), fake(Y, I64), fake(7)),
    "weights of another shape": lambda c: c.policy_loss(fake(X), fake(Y, I64), fake(R), weights=fake((6, 1))),
    "older scores that are strided": lambda c: c.policy_loss(fake(X), fake(Y, I64), fake(R), fake((6, 2))[:, 0]),
    "norm of zero": lambda c: c.policy_loss(fake(X), fake(Y, I64), fake(R), norm=0.0),
    "norm below zero": lambda c: c.distill_loss(fake(X), fake((6, 2), I32), fake((6, 2)), norm=-1.0),
    "norm that is no number": lambda c: c.pref_loss(fake(X), fake(Y, I64), fake(5, I32), norm=math.nan),
    "an even number of offsets": lambda c: c.pref_loss(fake(X), fake(Y, I64), fake(4, I32)),
    "no offsets": lambda c: c.pref_loss(fake(X), fake(Y, I64), fake(0, I32)),
    "offsets of floats": lambda c: c.pref_loss(fake(X), fake(Y, I64), fake(5)),
    "reference of pairs": lambda c: c.pref_loss(fake(X), fake(Y, I64), fake(5, I32), fake(2)),
    "weights of sequences": lambda c: c.pref_loss(fake(X), fake(Y, I64), fake(5, I32), weights=fake(4)),
    "classes of other rows": lambda c: c.distill_loss(fake(X), fake((5, 2), I32), fake((5, 2))),
    "teacher of another width": lambda c: c.distill_loss(fake(X), fake((6, 2), I32), fake((6, 3))),
    "teacher of half": lambda c: c.distill_loss(fake(X), fake((6, 2), I32), fake((6, 2), torch.float16)),
    "teacher's lse too short": lambda c: c.distill_loss(fake(X), fake((6, 2), I32), fake((6, 2)), fake(5)),
}


@pytest.mark.parametrize("what", CALLS)
def test_binding_refuses(ctx, what):
    with pytest.raises((TypeError, ValueError)):
        CALLS[what](ctx)
    assert ctx.rec.calls == []


def at(a):
    return ctypes.c_void_p(a)


def logp(L, c, x=P, ld=64, T=4, V=64, y=P, ib=8, scale=1.0, lp=P, lse=P):
    return L.lr_logp(c, x, ld, T, V, y, ib, -100, scale, lp, lse, NULL)


def logp_grad(L, c, x=P, ld=64, T=4, V=64, y=P, ib=8, scale=1.0, lse=P, g=P, d=at(1 << 20), ldd=64):
    return L.lr_logp_grad(c, x, ld, T, V, y, ib, -100, scale, lse, g, d, ldd, NULL)


def policy(L, c, x=P, ld=64, T=4, V=64, y=P, ib=8, o=(-100, 1.0, 0.2, 0.2, 0.0, 0.0, 1.0), adv=P, old=NULL, w=NULL, stats=P, d=at(1 << 20), ldd=64):
    return L.lr_policy_loss(c, x, ld, T, V, y, ib, ctypes.byref(api.LrPolicyOpt(*o)) if o else None, adv, old, NULL, w, stats, NULL, d, ldd, NULL)


def pref(L, c, x=P, ld=64, T=4, V=64, y=P, f=P, ob=4, pairs=1, o=(-100, 1.0, 0.1, 0.0, 0.0, 0, 0.0, 1.0), loss=P, h=P, d=at(1 << 20), ldd=64):
    return L.lr_pref_loss(c, x, ld, T, V, y, 8, f, ob, pairs, ctypes.byref(api.LrPrefOpt(*o)) if o else None, NULL, NULL, loss, h, NULL, d, ldd, NULL)


def distill(L, c, x=P, ld=64, T=4, V=64, ids=P, K=2, t=P, tb=4, o=(-1, 1.0, 0.0, 1.0), loss=P, d=at(1 << 20), ldd=64):
    return L.lr_distill_loss(c, x, ld, T, V, ids, 4, K, t, tb, ctypes.byref(api.LrDistillOpt(*o)) if o else None, NULL, NULL, loss, NULL, d, ldd, NULL)


@pytest.mark.parametrize("f", [logp, logp_grad, policy, pref, distill])
def test_c_entry_points_refuse_what_they_share(L, dead, f):
    assert f(L, None) == api.LR_ERR_NULL
    assert f(L, dead, x=NULL) == api.LR_ERR_NULL
    assert f(L, dead, T=-1) == api.LR_ERR_SHAPE
    assert f(L, dead, T=1 << 31) == api.LR_ERR_SHAPE
    assert f(L, dead, V=0) == api.LR_ERR_SHAPE
    assert f(L, dead, V=(1 << 24) + 1, ld=1 << 25) == api.LR_ERR_SHAPE
    assert f(L, dead, ld=63) == api.LR_ERR_SHAPE
    assert f(L, dead, ld=(1 << 40) + 1) == api.LR_ERR_SHAPE
    assert f(L, dead, x=at(258)) == api.LR_ERR_ALIGNMENT
    if f is not logp:
        assert f(L, dead, ldd=63) == api.LR_ERR_SHAPE
        assert f(L, dead, ldd=(1 << 40) + 1) == api.LR_ERR_SHAPE
        # the logits' own memory at another pitch, or shifted within their rows; columns beside them are another matter
        assert f(L, dead, d=P, ldd=65) == api.LR_ERR_VALUE
        assert f(L, dead, d=at(256 + 4)) == api.LR_ERR_VALUE
        assert f(L, dead, ld=200, ldd=200, d=at(256 + 63 * 4)) == api.LR_ERR_VALUE


def test_c_entry_points_refuse_their_own(L, dead):
    nan, inf = math.nan, math.inf
    for s in (0.0, -1.0, nan, inf):
        assert logp(L, dead, scale=s) == api.LR_ERR_VALUE and logp_grad(L, dead, scale=s) == api.LR_ERR_VALUE
        assert policy(L, dead, o=(-100, s, 0.2, 0.2, 0.0, 0.0, 1.0)) == api.LR_ERR_VALUE
        assert pref(L, dead, o=(-100, s, 0.1, 0.0, 0.0, 0, 0.0, 1.0)) == api.LR_ERR_VALUE
        assert distill(L, dead, o=(-1, s, 0.0, 1.0)) == api.LR_ERR_VALUE
    assert logp(L, dead, ib=2) == api.LR_ERR_VALUE and logp(L, dead, y=NULL) == api.LR_ERR_NULL and logp(L, dead, lp=NULL) == api.LR_ERR_NULL
    assert logp(L, dead, y=at(260)) == api.LR_ERR_ALIGNMENT and logp(L, dead, lse=at(257)) == api.LR_ERR_ALIGNMENT
    assert logp_grad(L, dead, lse=NULL) == api.LR_ERR_NULL and logp_grad(L, dead, g=NULL) == api.LR_ERR_NULL and logp_grad(L, dead, d=NULL) == api.LR_ERR_NULL
    assert policy(L, dead, o=None) == api.LR_ERR_NULL and policy(L, dead, adv=NULL) == api.LR_ERR_NULL and policy(L, dead, stats=NULL) == api.LR_ERR_NULL
    assert policy(L, dead, old=at(257)) == api.LR_ERR_ALIGNMENT and policy(L, dead, w=at(257)) == api.LR_ERR_ALIGNMENT
    for bad in ((-0.1, 0.2, 0.0, 0.0, 1.0), (0.2, -0.1, 0.0, 0.0, 1.0), (nan, 0.2, 0.0, 0.0, 1.0), (0.2, nan, 0.0, 0.0, 1.0), (0.2, 0.2, nan, 0.0, 1.0),
                (0.2, 0.2, inf, 0.0, 1.0), (0.2, 0.2, 0.0, -1.0, 1.0), (0.2, 0.2, 0.0, nan, 1.0), (0.2, 0.2, 0.0, inf, 1.0), (0.2, 0.2, 0.0, 0.0, nan)):
        assert policy(L, dead, o=(-100, 1.0, *bad)) == api.LR_ERR_VALUE
    assert pref(L, dead, o=None) == api.LR_ERR_NULL and pref(L, dead, f=NULL) == api.LR_ERR_NULL and pref(L, dead, loss=NULL) == api.LR_ERR_NULL
    assert pref(L, dead, h=NULL) == api.LR_ERR_NULL and pref(L, dead, ob=2) == api.LR_ERR_VALUE
    assert pref(L, dead, pairs=-1) == api.LR_ERR_SHAPE and pref(L, dead, pairs=(1 << 24) + 1) == api.LR_ERR_SHAPE
    assert pref(L, dead, f=at(260), ob=8) == api.LR_ERR_ALIGNMENT
    for bad in ((nan, 0.0, 0.0, 0, 0.0, 1.0), (0.1, inf, 0.0, 0, 0.0, 1.0), (0.1, 0.0, -0.1, 0, 0.0, 1.0), (0.1, 0.0, 1.1, 0, 0.0, 1.0),
                (0.1, 0.0, nan, 0, 0.0, 1.0), (0.1, 0.0, 0.0, 0, -1.0, 1.0), (0.1, 0.0, 0.0, 0, 0.0, inf)):
        assert pref(L, dead, o=(-100, 1.0, *bad)) == api.LR_ERR_VALUE
    assert distill(L, dead, o=None) == api.LR_ERR_NULL and distill(L, dead, ids=NULL) == api.LR_ERR_NULL and distill(L, dead, t=NULL) == api.LR_ERR_NULL
    assert distill(L, dead, loss=NULL) == api.LR_ERR_NULL and distill(L, dead, tb=8) == api.LR_ERR_VALUE
    assert distill(L, dead, K=0) == api.LR_ERR_SHAPE and distill(L, dead, K=1025) == api.LR_ERR_SHAPE
    assert distill(L, dead, t=at(257)) == api.LR_ERR_ALIGNMENT
    assert distill(L, dead, o=(-1, 1.0, nan, 1.0)) == api.LR_ERR_VALUE and distill(L, dead, o=(-1, 1.0, 0.0, nan)) == api.LR_ERR_VALUE
