"""The token-gate calls refuse arguments that do not fit, before anything is launched: the binding (with the library replaced by a
recorder and CUDA tensors imitated by CPU tensors that nothing dereferences) and the C entry points (through a context
that is never used: every refusal comes before the device is touched).  CPU only."""
import ctypes
import math

import pytest
import torch

from paper_2308_10037_b200 import api
from test_api_validation import FakeCuda, Recorder


def fake(shape, dtype=torch.float32, index=0):
    return FakeCuda(torch.zeros(shape, dtype=dtype), index)


@pytest.fixture
def ctx(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(api, "lib", lambda: rec)
    monkeypatch.setattr(api.Context, "_stream", lambda self: 0)
    empty = torch.empty_strided
    monkeypatch.setattr(torch, "empty_strided", lambda *a, device=None, **k: FakeCuda(empty(*a, **k)))
    c = api.Context.__new__(api.Context)
    c._h, c.device, c.n_max = ctypes.c_void_p(1), 0, 4096
    c.rec = rec
    yield c
    c._h = ctypes.c_void_p()


I32, I64, I8, BF, F64 = torch.int32, torch.int64, torch.int8, torch.bfloat16, torch.float64


def test_well_formed_calls_get_through(ctx):
    ids, x = fake(6, I64), fake((6, 8))
    ctx.embed(fake((5, 8)), ids)
    ctx.embed(fake((5, 8), BF), fake((2, 3), I32), scale=2.0)
    ctx.embed_grad(ids, x, 5)
    ctx.embed_grad(ids, fake((6, 8), BF), 5, out=fake((5, 8)), accumulate=True)
    ctx.route(x, 2, bias=fake(8), groups=2, top_groups=1)
    ctx.route(fake((6, 8), BF), 2, score="softmax")
    ctx.route_grad(x, fake((6, 2), I32), fake((6, 2)))
    q, s = fake((6, 8), I8), fake((6, 1))
    ctx.ckpt8_save(x)
    ctx.ckpt8_load(q, s, dtype=BF)
    ctx.ckpt8_grad(q, s, fake((6, 3)))
    assert ctx.rec.calls == ["lr_embed", "lr_embed_bf16", "lr_embed_grad", "lr_embed_grad_bf16", "lr_route", "lr_route_bf16",
                             "lr_route_grad", "lr_ckpt8_save", "lr_ckpt8_load_bf16", "lr_ckpt8_grad"]


CALLS = {
    "table of doubles": lambda c: c.embed(fake((5, 8), F64), fake(6, I64)),
    "table on the CPU": lambda c: c.embed(torch.zeros(5, 8), fake(6, I64)),
    "table of one dimension": lambda c: c.embed(fake(40), fake(6, I64)),
    "table transposed": lambda c: c.embed(fake((8, 5)).t(), fake(6, I64)),
    "table expanded": lambda c: c.embed(fake((1, 8)).expand(5, 8), fake(6, I64)),
    "table without columns": lambda c: c.embed(fake((5, 0)), fake(6, I64)),
    "tokens of floats": lambda c: c.embed(fake((5, 8)), fake(6)),
    "tokens on another device": lambda c: c.embed(fake((5, 8)), fake(6, I64, 1)),
    "table on another device": lambda c: c.embed(fake((5, 8), index=1), fake(6, I64)),
    "out of another shape": lambda c: c.embed(fake((5, 8)), fake(6, I64), out=fake((5, 8))),
    "out of another type": lambda c: c.embed(fake((5, 8)), fake(6, I64), out=fake((6, 8), BF)),
    "fewer rows than tokens": lambda c: c.embed_grad(fake(6, I64), fake((5, 8)), 5),
    "accumulate into nothing": lambda c: c.embed_grad(fake(6, I64), fake((6, 8)), 5, accumulate=True),
    "gradient of another shape": lambda c: c.embed_grad(fake(6, I64), fake((6, 8)), 5, out=fake((4, 8))),
    "gradient in bfloat16": lambda c: c.embed_grad(fake(6, I64), fake((6, 8)), 5, out=fake((5, 8), BF)),
    "gradient that is a slice": lambda c: c.embed_grad(fake(6, I64), fake((6, 8)), 5, out=fake((5, 9))[:, :8]),
    "unknown score": lambda c: c.route(fake((6, 8)), 2, score="tanh"),
    "bias too short": lambda c: c.route(fake((6, 8)), 2, bias=fake(7)),
    "bias of another type": lambda c: c.route(fake((6, 8)), 2, bias=fake(8, BF)),
    "logits of half": lambda c: c.route(fake((6, 8), torch.float16), 2),
    "ids for other rows": lambda c: c.route_grad(fake((6, 8)), fake((5, 2), I32), fake((5, 2))),
    "weights of another k": lambda c: c.route_grad(fake((6, 8)), fake((6, 2), I32), fake((6, 3))),
    "ids of 64 bits": lambda c: c.route_grad(fake((6, 8)), fake((6, 2), I64), fake((6, 2))),
    "gradient of another type": lambda c: c.route_grad(fake((6, 8)), fake((6, 2), I32), fake((6, 2)), out=fake((6, 8), BF)),
    "rows of integers": lambda c: c.ckpt8_save(fake((6, 8), I32)),
    "kept rows of another type": lambda c: c.ckpt8_load(fake((6, 8), torch.uint8), fake((6, 1))),
    "too few scales": lambda c: c.ckpt8_load(fake((6, 129), I8), fake((6, 1))),
    "load into doubles": lambda c: c.ckpt8_load(fake((6, 8), I8), fake((6, 1)), out=fake((6, 8), F64)),
    "load as doubles": lambda c: c.ckpt8_load(fake((6, 8), I8), fake((6, 1)), dtype=F64),
    "dz of other rows": lambda c: c.ckpt8_grad(fake((6, 8), I8), fake((6, 1)), fake((5, 3))),
    "grad_w too short": lambda c: c.ckpt8_grad(fake((6, 8), I8), fake((6, 1)), fake((6, 3)), grad_w=fake((2, 8))),
    "grad_b too short": lambda c: c.ckpt8_grad(fake((6, 8), I8), fake((6, 1)), fake((6, 3)), grad_b=fake(2)),
    "accumulate into one of two": lambda c: c.ckpt8_grad(fake((6, 8), I8), fake((6, 1)), fake((6, 3)), grad_w=fake((3, 8)), accumulate=True),
}


@pytest.mark.parametrize("what", CALLS)
def test_binding_refuses(ctx, what):
    with pytest.raises((TypeError, ValueError)):
        CALLS[what](ctx)
    assert ctx.rec.calls == []


# ---- the C entry points ----------------------------------------------------------------------------------

P, NULL = ctypes.c_void_p(256), None


@pytest.fixture(scope="module")
def L():
    from paper_2308_10037_b200 import build
    build.build()
    return api.lib()


@pytest.fixture(scope="module")
def dead():
    """Memory in place of a context: the refusals below come before anything of it is looked at."""
    buf = ctypes.create_string_buffer(4096)
    yield ctypes.cast(buf, ctypes.c_void_p)


def opt(k=2, groups=1, top=1, score=0, renorm=1, factor=1.0):
    return ctypes.byref(api.LrRouteOpt(k, groups, top, score, renorm, factor))


def route(L, c, logits=P, ld=64, T=4, E=64, o=None, bias=NULL, ids=P, w=P, counts=P):
    return L.lr_route(c, logits, ld, T, E, opt() if o is None else o, bias, ids, w, counts, NULL)


def test_c_refuses_routing(L, dead):
    assert route(L, None) == api.LR_ERR_NULL
    assert L.lr_route(dead, P, 64, 4, 64, None, NULL, P, P, P, NULL) == api.LR_ERR_NULL
    for bad in (dict(logits=NULL), dict(ids=NULL), dict(w=NULL)):
        assert route(L, dead, **bad) == api.LR_ERR_NULL
    for bad in (dict(T=-1), dict(T=2 ** 31), dict(E=0), dict(E=1025, ld=1025), dict(ld=63), dict(o=opt(k=0)), dict(o=opt(k=33)),
                dict(E=4, o=opt(k=5)), dict(o=opt(groups=0)), dict(o=opt(groups=5, top=5)), dict(o=opt(groups=64, top=64)), dict(o=opt(groups=4, top=5)),
                dict(o=opt(groups=4, top=0)), dict(o=opt(k=17, groups=4, top=1))):
        assert route(L, dead, **bad) == api.LR_ERR_SHAPE, bad
    for bad in (dict(o=opt(score=2)), dict(o=opt(score=-1)), dict(o=opt(factor=math.nan)), dict(o=opt(factor=math.inf))):
        assert route(L, dead, **bad) == api.LR_ERR_VALUE
    odd = ctypes.c_void_p(257)
    for bad in (dict(logits=odd), dict(ids=odd), dict(w=odd), dict(counts=odd), dict(bias=odd)):
        assert route(L, dead, **bad) == api.LR_ERR_ALIGNMENT
    assert L.lr_route_bf16(dead, odd, 64, 4, 64, opt(), NULL, P, P, P, NULL) == api.LR_ERR_ALIGNMENT
    grad = lambda c=dead, x=P, ld=64, E=64, ids=P, g=P, d=P, ldd=64: L.lr_route_grad(c, x, ld, 4, E, opt(), ids, g, d, ldd, NULL)
    assert grad(c=None) == grad(x=NULL) == grad(ids=NULL) == grad(g=NULL) == grad(d=NULL) == api.LR_ERR_NULL
    assert grad(ldd=63) == grad(ld=2) == api.LR_ERR_SHAPE
    assert grad(d=odd) == grad(x=odd) == grad(ids=odd) == grad(g=odd) == api.LR_ERR_ALIGNMENT
    assert L.lr_route_grad(dead, NULL, 64, 0, 64, opt(), NULL, NULL, NULL, 64, NULL) == api.LR_OK     # no rows: nothing to do


def test_c_refuses_token_rows(L, dead):
    odd = ctypes.c_void_p(257)
    look = lambda c=dead, t=P, ld=8, ids=P, ib=8, T=4, V=9, n=8, s=1.0, o=P, ldo=8: L.lr_embed(c, t, ld, ids, ib, T, V, n, s, o, ldo, NULL)
    assert look(c=None) == look(t=NULL) == look(ids=NULL) == look(o=NULL) == api.LR_ERR_NULL
    assert look(T=-1) == look(T=2 ** 31) == look(V=0) == look(V=2 ** 31) == look(n=0) == look(ld=7) == look(ldo=7) == api.LR_ERR_SHAPE
    assert look(ib=2) == look(s=math.inf) == look(s=math.nan) == api.LR_ERR_VALUE
    assert look(t=odd) == look(o=odd) == look(ids=ctypes.c_void_p(260)) == api.LR_ERR_ALIGNMENT
    assert look(T=0, t=NULL, ids=NULL, o=NULL) == api.LR_OK
    grad = lambda c=dead, ids=P, ib=4, d=P, ld=8, T=4, V=9, n=8, s=1.0, g=P: L.lr_embed_grad(c, ids, ib, d, ld, T, V, n, s, -1, 0, g, NULL)
    assert grad(c=None) == grad(ids=NULL) == grad(d=NULL) == grad(g=NULL) == api.LR_ERR_NULL
    assert grad(T=-1) == grad(T=2 ** 31) == grad(V=0) == grad(n=0) == grad(ld=7) == api.LR_ERR_SHAPE
    assert grad(ib=1) == grad(s=math.nan) == api.LR_ERR_VALUE
    assert grad(d=odd) == grad(g=odd) == grad(ids=odd) == api.LR_ERR_ALIGNMENT


def test_c_refuses_kept_rows(L, dead):
    odd = ctypes.c_void_p(257)
    save = lambda c=dead, x=P, ld=8, T=4, n=8, q=P, ldq=8, s=P: L.lr_ckpt8_save(c, x, ld, T, n, q, ldq, s, NULL)
    load = lambda c=dead, x=P, ld=8, T=4, n=8, q=P, ldq=8, s=P: L.lr_ckpt8_load(c, q, ldq, s, T, n, x, ld, NULL)
    for f in (save, load):
        assert f(c=None) == f(x=NULL) == f(q=NULL) == f(s=NULL) == api.LR_ERR_NULL
        assert f(T=-1) == f(n=0) == f(n=2 ** 24 + 1) == f(ld=7) == f(ldq=7) == api.LR_ERR_SHAPE
        assert f(x=odd) == f(s=odd) == api.LR_ERR_ALIGNMENT
        assert f(T=0, x=NULL, q=NULL, s=NULL) == api.LR_OK
    grad = lambda c=dead, q=P, ldq=8, s=P, T=4, n=8, z=P, ldz=3, C=3, w=P, b=P: L.lr_ckpt8_grad(c, q, ldq, s, T, n, z, ldz, C, 0, w, b, NULL)
    assert grad(c=None) == grad(q=NULL) == grad(s=NULL) == grad(z=NULL) == grad(w=NULL) == api.LR_ERR_NULL
    assert grad(T=-1) == grad(n=0) == grad(ldq=7) == grad(C=0) == grad(C=65537, ldz=65537) == grad(ldz=2) == api.LR_ERR_SHAPE
    assert grad(s=odd) == grad(z=odd) == grad(w=odd) == grad(b=odd) == api.LR_ERR_ALIGNMENT
