"""The token-gate operators against plain implementations in float64: token rows and their gradient, routing and its
gradient, rows kept in 8 bits and the gradient taken from them.

Tolerances, with u = 2^-24 (fp32 rounding) and derived from the operations, not from a run:
  lookup            one product rounded once: 2u relative in fp32 (scale itself is rounded too), 2^-8 in bfloat16
  sum of L rows     a chain of L rounded additions and one product: (L + 3) u times the sum of the magnitudes
  routing weights   exp of a rounded difference |x| <= 20 (20u + 4u), a sum of up to 1024 terms in a tree of lanes (<= 40u),
                    a quotient: 80u relative
  routing gradient  the same probabilities in a difference of two terms, each at most factor * sum |g|: 160u of that; bfloat16
                    output adds 2^-8 relative
  8-bit rows        s: two roundings; q: |q - 127 x / a| <= 1/2 + 127 * 4u; read back: bit for bit q * s rounded
  8-bit gradient    T products of three factors summed in fp32: rounding errors of partial sums add like sqrt(T) at worst for
                    random signs of the errors: (8 + sqrt(T)) u times the sum of the magnitudes
"""
import math

import numpy as np
import pytest
import torch

from paper_2308_10037_b200 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    from paper_2308_10037_b200 import build
    build.build()
    c = api.Context(n_max=64, device=0)
    yield c
    assert c.device_status() == 0
    assert c.check_guards() == 0                    # no kernel wrote outside the scratch
    c.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rnd(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=gen(seed), device="cuda").to(dtype)


def strided(t, extra, shift):
    """The same values as a slice of a wider matrix, starting `shift` elements into its rows."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan") if t.is_floating_point() else 99, dtype=t.dtype, device=t.device)
    view = wide[:, shift:shift + t.shape[1]]
    view.copy_(t)
    return view


def close(got, want, bound):
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    off = (got - want).abs()
    assert bool((off <= bound).all()), f"worst {float((off - bound).max()):.3e} over its bound, largest error {float(off.max()):.3e}"


# ---- token rows ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,n", [(1, 1, 1), (3, 7, 5), (17, 100, 64), (33, 50, 130), (5, 9, 1000), (300, 40, 1028), (2, 4, 5001), (1000, 31, 8)])
def test_embed(ctx, dt, T, V, n):
    table = rnd(V, n, seed=T, dtype=DT[dt])
    ids = torch.randint(0, V, (T,), generator=gen(1), device="cuda")
    want = table.double()[ids] * 1.7
    for i in (ids, ids.int()):
        got = ctx.embed(table, i, scale=1.7)
        assert got.dtype == table.dtype
        close(got, want, (2 * U if dt == "f32" else 2.0 ** -8) * want.abs())
    assert torch.equal(ctx.embed(table, ids), table[ids])                    # scale 1: the rows themselves
    assert torch.equal(ctx.embed(strided(table, 3, 1), ids, scale=1.7), ctx.embed(table, ids, scale=1.7))
    out = strided(torch.zeros(T, n, dtype=DT[dt], device="cuda"), 5, 2)
    ctx.embed(table, ids, scale=1.7, out=out)
    assert torch.equal(out, ctx.embed(table, ids, scale=1.7))


def test_embed_shapes_and_tokens_outside_the_table(ctx):
    table = rnd(10, 12)
    assert ctx.embed(table, torch.zeros((2, 3), dtype=torch.int64, device="cuda")).shape == (2, 3, 12)
    assert ctx.embed(table, torch.zeros(0, dtype=torch.int32, device="cuda")).shape == (0, 12)
    assert ctx.device_status() == 0
    ids = torch.tensor([3, -1, 10, 2 ** 40, 9], device="cuda")
    got = ctx.embed(table, ids)
    assert torch.equal(got[[0, 4]], table[[3, 9]]) and bool((got[1:4] == 0).all())
    assert ctx.device_status() == api.LR_ERR_VALUE
    assert ctx.device_status() == 0


def test_embed_offsets_beyond_32_bits(ctx):
    V, n = 1_100_000, 2048                                                   # 2.25e9 elements
    table = torch.empty(V, n, dtype=torch.bfloat16, device="cuda")
    table[-3:] = rnd(3, n, dtype=torch.bfloat16)
    ids = torch.tensor([V - 1, V - 3], device="cuda")
    assert torch.equal(ctx.embed(table, ids), table[ids])


def grad_reference(ids, dout, V, scale, pad=-1, base=None):
    """(gradient, sum of magnitudes, number of rows) per table row in float64."""
    ids = ids.long()
    keep = (ids >= 0) & (ids < V) & (ids != pad)
    d = dout.double()[keep] * scale
    z = torch.zeros(V, dout.shape[1], dtype=torch.float64, device="cuda")
    want = z.clone().index_add_(0, ids[keep], d)
    mag = z.index_add_(0, ids[keep], d.abs())
    count = torch.bincount(ids[keep], minlength=V).double()[:, None]
    return want if base is None else want + base.double(), mag if base is None else mag + base.double().abs(), count


def skewed(T, V, seed):
    """Token numbers of which a few are frequent."""
    r = torch.rand(T, generator=gen(seed), device="cuda", dtype=torch.float64)
    return ((V + 1) ** r).long().clamp_(1, V) - 1


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,n", [(1, 1, 1), (2, 3, 5), (16, 1, 8), (63, 2, 130), (64, 300, 64), (65, 5, 257), (1000, 70000, 12), (1023, 3, 33),
                                   (1024, 40, 1000), (5000, 1, 40), (8192, 20, 24), (9001, 300, 520), (40000, 70000, 16)])
def test_embed_grad(ctx, dt, T, V, n):
    ids = skewed(T, V, T)
    dout = rnd(T, n, seed=n, dtype=DT[dt])
    want, mag, count = grad_reference(ids, dout, V, 1.3)
    got = ctx.embed_grad(ids, dout, V, scale=1.3)
    assert got.dtype == torch.float32
    close(got, want, (count + 3) * U * mag)
    assert torch.equal(ctx.embed_grad(ids.int(), dout, V, scale=1.3), got)   # the same bits again, from 32-bit tokens
    assert torch.equal(ctx.embed_grad(ids, strided(dout, 8, 3), V, scale=1.3)[0], got[0]) or n % 4 == 0
    base = rnd(V, n, seed=9)
    into = base.clone()
    ctx.embed_grad(ids, dout, V, scale=1.3, out=into, accumulate=True)
    want, mag, count = grad_reference(ids, dout, V, 1.3, base=base)
    close(into, want, (count + 4) * U * mag)
    untouched = torch.bincount(ids, minlength=V) == 0
    assert torch.equal(into[untouched], base[untouched])


@pytest.mark.parametrize("R", [16, 32, 64])
def test_embed_grad_runs_around_the_chunk_borders(ctx, R):
    # runs that start and end at, just before and just after borders of the chunks of R positions, short and long ones
    T0 = {16: 500, 32: 4000, 64: 9000}[R]
    lengths = [1, R - 1, R, R + 1, 2 * R - 1, 2 * R, 2 * R + 1, 1, 3 * R, 1, 4 * R + 1, R - 2, 5 * R - 1]
    lengths = [x for x in lengths]
    lengths.append(max(1, T0 - sum(lengths)))
    ids = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
    perm = torch.randperm(ids.numel(), generator=gen(3), device="cuda")
    for order in (ids, ids[perm], ids.flip(0)):
        dout = rnd(order.numel(), 20, seed=R)
        want, mag, count = grad_reference(order, dout, len(lengths) + 1, 1.0)
        close(ctx.embed_grad(order.contiguous(), dout, len(lengths) + 1), want, (count + 3) * U * mag)


def test_embed_grad_padding_and_tokens_outside(ctx):
    V, n = 50, 36
    ids = torch.randint(0, V, (3000,), generator=gen(4), device="cuda")
    ids[::3] = 7
    dout = rnd(3000, n)
    dout[ids == 7] = float("nan")                                            # what padding carries is not looked at
    want, mag, count = grad_reference(ids, torch.nan_to_num(dout), V, 2.0, pad=7)
    got = ctx.embed_grad(ids, dout, V, scale=2.0, padding_id=7)
    close(got, want, (count + 3) * U * mag)
    assert bool((got[7] == 0).all()) and ctx.device_status() == 0
    ids[5], ids[6] = -4, V
    dout[5:7] = float("inf")
    want, mag, count = grad_reference(ids, torch.nan_to_num(dout, posinf=0.0), V, 2.0, pad=7)
    close(ctx.embed_grad(ids, dout, V, scale=2.0, padding_id=7), want, (count + 3) * U * mag)
    assert ctx.device_status() == api.LR_ERR_VALUE
    every = torch.full((100,), 7, device="cuda")                             # no position with a gradient
    assert bool((ctx.embed_grad(every, dout[:100], V, padding_id=7) == 0).all())
    none = ctx.embed_grad(every[:0], dout[:0], V)
    assert none.shape == (V, n) and bool((none == 0).all())


@pytest.mark.parametrize("V", [255, 256, 511, 512, 65535, 65536, (1 << 18) - 1, 1 << 18, (1 << 24) - 1, 1 << 24])
def test_embed_grad_around_the_passes_of_the_sort(ctx, V):
    ids = torch.randint(0, V, (20000,), generator=gen(5), device="cuda")
    ids[:4] = torch.tensor([0, V - 1, V - 1, V // 2], device="cuda")
    dout = rnd(20000, 1, seed=2)
    want, mag, count = grad_reference(ids, dout, V, 1.0)
    close(ctx.embed_grad(ids, dout, V), want, (count + 3) * U * mag)


def test_embed_grad_is_the_derivative_of_embed(ctx):
    # <dout, embed(table + d) - embed(table)> = <grad, d> for any direction d (the lookup is linear)
    V, n, T = 90, 24, 700
    ids = skewed(T, V, 8)
    dout, d = rnd(T, n, seed=3), rnd(V, n, seed=4)
    lhs = (dout.double() * (d.double()[ids] * 0.75)).sum()
    grad = ctx.embed_grad(ids, dout, V, scale=0.75)
    rhs = (grad.double() * d.double()).sum()
    mag = grad_reference(ids, dout, V, 0.75)[1]
    assert abs(lhs - rhs) <= ((torch.bincount(ids, minlength=V)[:, None] + 3) * U * mag * d.double().abs()).sum()


# ---- routing ---------------------------------------------------------------------------------------------

def route_reference(logits, k, bias, groups, top, score, renorm, factor):
    """(ids, weights, choice values) of plain loops in float64, by the definition in the header."""
    x = logits.double().cpu().numpy()
    T, E = x.shape
    b = np.zeros(E) if bias is None else bias.double().cpu().numpy()
    ids, w, choice = np.full((T, k), -1), np.zeros((T, k)), np.full((T, E), -np.inf)
    for t in range(T):
        r = x[t]
        if np.isnan(r).any() or (score == "softmax" and np.isposinf(r).any()):
            w[t] = np.nan
            continue
        with np.errstate(over="ignore"):
            if score == "sigmoid":
                p = 1 / (1 + np.exp(-r))
            else:
                p = np.exp(r - r.max()) if np.isfinite(r.max()) else np.zeros(E)
                p = p / max(p.sum(), 1e-300)
        c = (p if score == "sigmoid" else r) + b
        c[np.isneginf(r) | np.isneginf(c) | np.isnan(c)] = -np.inf
        choice[t] = c
        gs = E // groups
        worth = []
        for g in range(groups):
            v = sorted((v for v in c[g * gs:(g + 1) * gs] if v > -np.inf), reverse=True)
            worth.append(-np.inf if not v else v[0] if score == "softmax" or len(v) == 1 else v[0] + v[1])
        kept = sorted(range(groups), key=lambda g: (-worth[g], g))[:top]
        able = [e for e in range(E) if e // gs in kept and c[e] > -np.inf]
        sel = sorted(able, key=lambda e: (-c[e], e))[:k]
        if renorm and sel:
            # ratios of the chosen p from their logarithms, so that they are right where the p underflow
            with np.errstate(over="ignore"):
                log_p = -np.logaddexp(0.0, -r[sel]) if score == "sigmoid" else r[sel]
                rel = np.exp(log_p - log_p.max())
        for i, e in enumerate(sel):
            ids[t, i] = e
            w[t, i] = factor * (rel[i] / rel.sum() if renorm else p[e])
    return ids, w, choice


def grid_logits(T, E, seed, dtype):
    """Logits on a grid of eighths: equal ones are exactly equal, different ones have clearly different probabilities."""
    return (torch.randint(-24, 25, (T, E), generator=gen(seed), device="cuda").float() / 8).to(dtype)


ROUTES = [(1, 1, 1, 1, 1), (5, 8, 3, 1, 1), (9, 8, 8, 1, 1), (33, 60, 6, 4, 2), (40, 64, 6, 8, 3), (100, 100, 4, 5, 5), (70, 128, 8, 2, 1),
          (50, 160, 6, 8, 3), (64, 256, 8, 8, 4), (20, 257, 32, 1, 1), (30, 384, 8, 32, 16), (21, 512, 1, 1, 1), (10, 999, 9, 3, 2), (12, 1024, 8, 16, 2),
          (25, 32, 4, 32, 7), (8, 96, 12, 3, 1)]


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k,groups,top", ROUTES)
def test_route_ties_go_to_the_lowest_index(ctx, T, E, k, groups, top, score, dt):
    x = grid_logits(T, E, E + k, DT[dt])
    for renorm, factor in ((True, 1.0), (False, 2.5)):
        ids, w, counts = ctx.route(x, k, groups=groups, top_groups=top, score=score, renorm=renorm, factor=factor)
        rid, rw, _ = route_reference(x, k, None, groups, top, score, renorm, factor)
        # group sums of two sigmoids can differ by less than fp32 resolves where the pairs differ: such rows are left out by construction
        # of the grid only for single values, so compare rows whose kept groups are clear
        clear = np.ones(T, bool) if score == "softmax" or groups == 1 or top == groups else _clear_groups(x, groups, top)
        assert clear.mean() > 0.5
        assert np.array_equal(ids.cpu().numpy()[clear], rid[clear])
        close(w[torch.from_numpy(clear).cuda()], torch.from_numpy(rw[clear]).cuda(), 80 * U * torch.from_numpy(np.abs(rw[clear])).cuda())
        assert np.array_equal(counts.cpu().numpy(), np.bincount(ids.cpu().numpy().ravel(), minlength=E))
        ids2 = ctx.route(strided(x, 3, 1), k, groups=groups, top_groups=top, score=score, renorm=renorm, factor=factor)[0]
        assert torch.equal(ids, ids2)


def _clear_groups(x, groups, top):
    p = torch.sigmoid(x.double()).reshape(x.shape[0], groups, -1)
    worth = p.topk(min(2, p.shape[2]), dim=2)[0].sum(2).sort(dim=1, descending=True)[0]
    gap = worth[:, top - 1] - worth[:, top]
    return ((gap > 1e-5) | (gap == 0)).cpu().numpy()    # equal pairs of logits: a tie in any precision


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,groups,top", ROUTES)
def test_route_with_a_bias(ctx, T, E, k, groups, top, score):
    x = rnd(T, E, seed=T + E) * 2
    bias = rnd(E, seed=3) * 0.1
    ids, w, counts = ctx.route(x, k, bias=bias, groups=groups, top_groups=top, score=score, factor=1.5)
    rid, rw, choice = route_reference(x, k, bias, groups, top, score, True, 1.5)
    got = ids.cpu().numpy()
    same = (got == rid).all(axis=1)
    for t in np.flatnonzero(~same):                 # only where two choice values are closer than fp32 resolves
        srt = np.sort(choice[t])[::-1]
        assert np.min(srt[:-1] - srt[1:]) < 1e-6
    assert same.mean() >= 0.9 or T < 10
    m = torch.from_numpy(same).cuda()
    close(w[m], torch.from_numpy(rw).cuda()[m], 80 * U * torch.from_numpy(np.abs(rw)).cuda()[m])
    assert np.array_equal(counts.cpu().numpy(), np.bincount(got.ravel(), minlength=E))


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("groups,top", [(1, 1), (4, 2)])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_masked_and_extreme_rows(ctx, score, groups, top, renorm):
    E, k = 32, 5
    low = torch.finfo(torch.float32).min
    x = rnd(14, E, seed=1)
    x[0] = -math.inf                                # a mask that leaves nothing
    x[1] = -math.inf
    x[1, 9] = 0.5                                   # one expert left
    x[2, 1:] = -math.inf
    x[3] = low                                      # the type's lowest value is a number, not a mask
    x[4] = low
    x[4, 20:22] = torch.tensor([1.0, 2.0])
    x[5, 3] = math.nan
    x[6, 3] = math.inf
    x[7] = torch.finfo(torch.float32).max
    x[8] = 0.0
    x[8, ::2] = -0.0                                # equal to +0: the lowest index
    x[9, 4:] = -math.inf                            # four left, all in one or in half a group
    x[10] = 80.0                                    # saturated sigmoids: all ties
    x[11] = -120.0                                  # underflowing sigmoids
    bias = torch.zeros(E, device="cuda")
    bias[30] = -math.inf                            # a mask for all rows
    for b in (None, bias):
        ids, w, counts = ctx.route(x, k, bias=b, groups=groups, top_groups=top, score=score, renorm=renorm)
        rid, rw, _ = route_reference(x, k, b, groups, top, score, renorm, 1.0)
        got, gw = ids.cpu().numpy(), w.double().cpu().numpy()
        clear = np.ones(14, bool)
        if score == "sigmoid":
            clear[[12, 13]] = groups == 1           # random rows: covered elsewhere when groups are close
        assert np.array_equal(got[:12], rid[:12])
        nan = np.isnan(rw)
        assert np.array_equal(np.isnan(gw), nan)
        ok = ~nan & clear[:, None]
        assert (np.abs(gw - rw)[ok] <= 80 * U * np.abs(rw[ok]) + 2.0 ** -120).all()
        assert counts.sum().item() == (got >= 0).sum()
        # the gradient of those rows is finite wherever the weights are
        g = rnd(14, k, seed=2)
        d = ctx.route_grad(x, ids, g, score=score, renorm=renorm)
        rows = ~nan.any(axis=1)
        assert bool(torch.isfinite(d[torch.from_numpy(rows).cuda()]).all())
        assert bool((d[0] == 0).all())


def test_route_counts_over_many_ctas_and_calls(ctx):
    x = rnd(30001, 64, seed=5)
    for _ in range(3):                              # the running counts are left at zero for the next call
        ids, _, counts = ctx.route(x, 4, score="softmax")
        assert torch.equal(counts, torch.bincount(ids.flatten().long(), minlength=64).int())
    ids, w, counts = ctx.route(x[:0], 4)
    assert ids.shape == (0, 4) and bool((counts == 0).all())


def grad_formula(x, ids, g, score, renorm, factor):
    """dL/dlogits in float64 by automatic differentiation of the definition, with ids of -1 left out."""
    x = x.double().clone().requires_grad_(True)
    p = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, dim=1)
    have = ids >= 0
    c = p.gather(1, ids.clamp(min=0).long()) * have
    w = c / c.sum(1, keepdim=True) if renorm else c
    (w * factor * g.double()).sum().backward()
    return x.grad


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (7, 8, 8), (33, 60, 6), (100, 100, 2), (64, 128, 8), (50, 257, 32), (1000, 64, 4), (9, 1000, 8)])
def test_route_grad(ctx, T, E, k, score, dt):
    x = (rnd(T, E, seed=E) * 2).to(DT[dt])
    g = rnd(T, k, seed=k)
    for renorm in (True, False):
        ids = ctx.route(x, k, score=score, renorm=renorm)[0]
        ids[0, k - 1] = -1 if k > 1 else ids[0, 0]
        got = ctx.route_grad(x, ids, g, score=score, renorm=renorm, factor=2.0)
        want = grad_formula(x, ids, g, score, renorm, 2.0)
        bound = 160 * U * 2.0 * g.double().abs().sum(1, keepdim=True) + (2.0 ** -8 * want.abs() if dt == "bf16" else 0.0)
        assert got.dtype == x.dtype
        close(got, want, bound)
        out = strided(torch.zeros_like(x), 4, 3)
        ctx.route_grad(strided(x, 5, 2), ids, g, score=score, renorm=renorm, factor=2.0, out=out)
        assert torch.equal(out, got)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_grad_against_differences(ctx, score, renorm):
    T, E, k, h = 6, 20, 4, 1e-6
    x, g = rnd(T, E, seed=11), rnd(T, k, seed=12)
    ids = ctx.route(x, k, score=score)[0]
    got = ctx.route_grad(x, ids, g, score=score, renorm=renorm).double()

    def loss(z):
        p = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, dim=1)
        c = p.gather(1, ids.long())
        return ((c / c.sum(1, keepdim=True) if renorm else c) * g.double()).sum(1)

    for e in range(E):
        step = torch.zeros(T, E, dtype=torch.float64, device="cuda")
        step[:, e] = h
        diff = (loss(x.double() + step) - loss(x.double() - step)) / (2 * h)
        # central difference: h^2 |f'''| <= 1e-11 and rounding 2^-53 |f| / h <= 1e-8
        close(got[:, e], diff, 160 * U * g.double().abs().sum(1) + 1e-8)


# ---- rows in 8 bits --------------------------------------------------------------------------------------

CKPT = [(1, 1), (3, 7), (5, 128), (4, 129), (9, 136), (2, 1000), (17, 1024), (6, 4100), (100, 64), (33, 255), (2, 16391)]


def padded_groups(x):
    return torch.nn.functional.pad(x.double(), (0, -x.shape[1] % 128)).unflatten(1, (-1, 128))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,n", CKPT)
def test_ckpt8_round_trip(ctx, dt, T, n):
    x = (rnd(T, n, seed=n) * torch.exp(rnd(T, n, seed=n + 1))).to(DT[dt])
    q, s = ctx.ckpt8_save(x)
    assert q.shape == (T, n) and s.shape == (T, (n + 127) // 128)
    g = padded_groups(x)
    a = g.abs().amax(2)
    close(s, a / 127, 2 * U * a / 127)
    t = g * (127 / a)[:, :, None]
    off = (padded_groups(q) - t).abs()
    assert bool((off <= 0.5 + 127 * 4 * U).all())
    back32 = (padded_groups(q).float() * s[:, :, None]).flatten(1)[:, :n]
    for d in (torch.float32, torch.bfloat16):
        assert torch.equal(ctx.ckpt8_load(q, s, dtype=d), back32.to(d))
    q2, s2 = ctx.ckpt8_save(strided(x, 3, 1))       # another alignment, the same result
    assert torch.equal(q2, q) and torch.equal(s2, s)
    odd = strided(q, 5, 3)
    out = strided(torch.zeros(T, n, device="cuda"), 1, 1)
    ctx.ckpt8_load(odd, s, out=out)
    assert torch.equal(out, back32)


def test_ckpt8_special_values(ctx):
    x = rnd(8, 300)
    x[0] = 0
    x[1, :128] = 1e-38                              # 127 / a would overflow: kept as zeros
    x[2, 130] = math.inf
    x[3, 299] = math.nan
    x[4, 5] = -3e38
    x[5] = torch.finfo(torch.float32).max
    q, s = ctx.ckpt8_save(x)
    back = ctx.ckpt8_load(q, s)
    assert bool((back[0] == 0).all()) and bool((back[1, :128] == 0).all()) and bool((s[0] == 0).all())
    assert bool(torch.isnan(back[2, 128:256]).all()) and bool(torch.isfinite(back[2, :128]).all())
    assert bool(torch.isnan(back[3, 256:]).all()) and bool(torch.isfinite(back[3, :256]).all())
    assert back[4, 5].item() == pytest.approx(-3e38, rel=1e-6)
    assert bool(torch.isfinite(back[5]).all())
    e, f = ctx.ckpt8_save(x[:0])
    assert e.shape == (0, 300) and f.shape == (0, 3) and ctx.ckpt8_load(e, f).shape == (0, 300)


def test_ckpt8_offsets_beyond_32_bits(ctx):
    T, n = 70_000, 65_536                           # 4.6e9 elements
    q = torch.zeros(T, n, dtype=torch.int8, device="cuda")
    s = torch.zeros(T, n // 128, device="cuda")
    x = rnd(2, n, dtype=torch.bfloat16)
    q2, s2 = ctx.ckpt8_save(x)
    q[-2:], s[-2:] = q2, s2
    out = torch.empty(T, n, dtype=torch.bfloat16, device="cuda")
    ctx.ckpt8_load(q, s, out=out)
    assert torch.equal(out[-2:], ctx.ckpt8_load(q2, s2, dtype=torch.bfloat16)) and bool((out[:2] == 0).all())
    q3, s3 = ctx.ckpt8_save(out)
    assert torch.equal(s3[:2], s[:2]) and bool((q3[:2] == 0).all()) and int((q3[-2:].int() - q2.int()).abs().max()) <= 1
    dz = torch.zeros(T, 1, device="cuda")
    dz[-1] = 1.0
    gw, _ = ctx.ckpt8_grad(q, s, dz)
    close(gw, ctx.ckpt8_load(q2, s2)[1:].double(), 4 * U * ctx.ckpt8_load(q2, s2)[1:].double().abs())


GRADS = [(1, 1, 1), (1, 128, 3), (2, 130, 1), (31, 64, 2), (33, 200, 5), (100, 129, 8), (1000, 300, 9), (257, 1000, 16), (500, 256, 17), (64, 512, 64),
         (700, 136, 100), (2000, 96, 1), (3001, 384, 40), (129, 1040, 128), (50, 33, 300), (4097, 256, 64), (5000, 48, 4)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,n,C", GRADS)
def test_ckpt8_grad(ctx, dt, T, n, C):
    q, s = ctx.ckpt8_save(rnd(T, n, seed=n))
    dz = (rnd(T, C, seed=C) * torch.exp(2 * rnd(T, 1, seed=3))).to(DT[dt])
    x = (padded_groups(q) * s.double()[:, :, None]).flatten(1)[:, :n]
    want, mag = dz.double().t() @ x, dz.double().abs().t() @ x.abs()
    wb, mb = dz.double().sum(0), dz.double().abs().sum(0)
    rel = (8 + math.sqrt(T)) * U
    gw, gb = ctx.ckpt8_grad(q, s, dz)
    close(gw, want, rel * mag)
    close(gb, wb, rel * mb)
    assert all(torch.equal(a, b) for a, b in zip(ctx.ckpt8_grad(q, s, dz), (gw, gb)))
    base_w, base_b = rnd(C, n, seed=5), rnd(C, seed=6)
    aw, ab = base_w.clone(), base_b.clone()
    ctx.ckpt8_grad(q, s, dz, aw, ab, accumulate=True)
    close(aw, want + base_w.double(), rel * mag + U * (want + base_w.double()).abs())
    close(ab, wb + base_b.double(), rel * mb + U * (wb + base_b.double()).abs())
    ow, ob = ctx.ckpt8_grad(strided(q, 3, 1), s, strided(dz, 2, 1))
    close(ow, want, rel * mag)
    close(ob, wb, rel * mb)


@pytest.mark.parametrize("C", [2, 16, 17, 40, 50])
@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("T", [32, 33, 64, 65, 96, 511, 512, 513, 544, 545, 577, 1024, 1025, 1057, 1537, 5000])
def test_ckpt8_grad_many_rows_per_cta(ctx, T, shift, C):
    # one CTA per block of columns for all rows: every number of stages, turns of the rings and sets of warps
    n = 300
    q, s = ctx.ckpt8_save(rnd(T, n, seed=n))
    dz = rnd(T, C, seed=C)
    x = (padded_groups(q) * s.double()[:, :, None]).flatten(1)[:, :n]
    want, mag = dz.double().t() @ x, dz.double().abs().t() @ x.abs()
    rel = (8 + math.sqrt(T)) * U
    ctx.set_sm_limit(1)
    try:
        gw, gb = ctx.ckpt8_grad(strided(q, 5, shift) if shift else q, s, dz)
    finally:
        ctx.set_sm_limit(0)
    close(gw, want, rel * mag)
    close(gb, dz.double().sum(0), rel * dz.double().abs().sum(0))


def test_ckpt8_grad_wide_range_of_dz(ctx):
    # rows whose gradient differs by many orders of magnitude: the small ones must not be lost where they stand alone
    T, n, C = 300, 256, 20
    q, s = ctx.ckpt8_save(rnd(T, n))
    dz = torch.zeros(T, C, device="cuda")
    for c in range(C):
        dz[c::C, c] = rnd(T // C, seed=c) * 10.0 ** (2 * c - 30)
    x = (padded_groups(q) * s.double()[:, :, None]).flatten(1)[:, :n]
    want, mag = dz.double().t() @ x, dz.double().abs().t() @ x.abs()
    close(ctx.ckpt8_grad(q, s, dz)[0], want, (8 + math.sqrt(T)) * U * mag + 2.0 ** -126)


def test_ckpt8_grad_is_the_derivative_of_the_layer(ctx):
    # <dz, X dW^T + db> = <grad_w, dW> + <grad_b, db>
    T, n, C = 400, 200, 24
    q, s = ctx.ckpt8_save(rnd(T, n))
    x = ctx.ckpt8_load(q, s).double()
    dz, dW, db = rnd(T, C, seed=1), rnd(C, n, seed=2).double(), rnd(C, seed=3).double()
    lhs = (dz.double() * (x @ dW.t() + db)).sum()
    gw, gb = ctx.ckpt8_grad(q, s, dz)
    mag = dz.double().abs().t() @ x.abs()
    tol = (8 + math.sqrt(T)) * U * ((mag * dW.abs()).sum() + (dz.double().abs().sum(0) * db.abs()).sum())
    assert abs(lhs - (gw.double() * dW).sum() - (gb.double() * db).sum()) <= tol


def test_ckpt8_grad_of_no_rows(ctx):
    q, s = ctx.ckpt8_save(rnd(0, 40))
    gw, gb = ctx.ckpt8_grad(q, s, rnd(0, 3))
    assert gw.shape == (3, 40) and bool((gw == 0).all()) and bool((gb == 0).all())


# ---- streams ---------------------------------------------------------------------------------------------

def test_calls_run_on_the_current_stream(ctx):
    table, ids, dout = rnd(500, 64), skewed(5000, 500, 1), rnd(5000, 64, seed=2)
    x = rnd(5000, 64, seed=3)
    want = (ctx.embed(table, ids, 2.0), ctx.embed_grad(ids, dout, 500), *ctx.route(x, 4), *ctx.ckpt8_save(x))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = torch.empty_like(x)
        torch.cuda._sleep(20_000_000)               # the inputs come late on this stream
        late.copy_(x)
        got = (ctx.embed(table, ids, 2.0), ctx.embed_grad(ids, dout, 500), *ctx.route(late, 4), *ctx.ckpt8_save(late))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_default_contexts_of_two_streams_do_not_share_scratch(ctx):
    # the module's functions keep a context per stream: calls that overlap on the GPU must not meet in one scratch
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    work = []
    for i, st in enumerate(streams):
        ids, dout, x = skewed(20000, 3000, i), rnd(20000, 128, seed=i + 2), rnd(20000, 96, seed=i + 4)
        q, s = ctx.ckpt8_save(dout)
        want = (ctx.embed_grad(ids, dout, 3000), ctx.route(x, 4)[2], *ctx.ckpt8_grad(q, s, x))
        work.append((st, ids, dout, x, q, s, want))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (st, ids, dout, x, q, s, _) in enumerate(work):
            with torch.cuda.stream(st):
                got[i].append((api.lr_embed_grad(ids, dout, 3000), api.lr_route(x, 4)[2], *api.lr_ckpt8_grad(q, s, x)))
    torch.cuda.synchronize()
    for g, w in zip(got, work):
        assert all(torch.equal(a, b) for one in g for a, b in zip(one, w[-1]))


def test_calls_can_be_captured(ctx):
    ids, dout, x = skewed(5000, 500, 1), rnd(5000, 64, seed=2), rnd(5000, 64, seed=3)
    grad, dz = torch.empty(500, 64, device="cuda"), rnd(5000, 40, seed=4)
    gw, gb = torch.empty(40, 64, device="cuda"), torch.empty(40, device="cuda")
    q, s = ctx.ckpt8_save(x)
    ctx.embed_grad(ids, dout, 500, out=grad)        # the scratch grows outside the capture
    ctx.ckpt8_grad(q, s, dz, gw, gb)
    want = [t.clone() for t in (grad, gw, gb)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.embed_grad(ids, dout, 500, out=grad)
        ctx.ckpt8_grad(q, s, dz, gw, gb)
    ctx.embed_grad(skewed(60000, 500, 2), rnd(60000, 64, seed=5), 500)   # another call makes the scratch grow in between
    for t in (grad, gw, gb):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((grad, gw, gb), want))
    # the module's functions: the capture borrows the context of the warm-up
    api.lr_embed_grad(ids, dout, 500, out=grad)
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2):
        api.lr_embed_grad(ids, dout, 500, out=grad)
    grad.zero_()
    graph2.replay()
    torch.cuda.synchronize()
    assert torch.equal(grad, want[0])


# ---- the operators together ------------------------------------------------------------------------------

def test_token_gate_step_matches_automatic_differentiation(ctx):
    from paper_2308_10037_b200.examples import token_gate
    m = token_gate.TokenGate(vocab=300, n=48, experts=12, k=3, ctx=ctx, seed=3)
    tokens = torch.randint(0, 300, (700,), generator=gen(9), device="cuda")
    y = (torch.rand(700, generator=gen(10), device="cuda") < 0.5).float()
    X, logits, ids, *_ = m.forward(tokens)
    loss, _, (dtable, dW, db, da) = m.step(tokens, y)
    p = [t.double().clone().requires_grad_(True) for t in (m.table, m.W, m.b, m.a)]
    z64 = (p[0] * m.scale)[tokens] @ p[1].t() + p[2]
    c = torch.sigmoid(z64).gather(1, ids.long())
    ref = torch.nn.functional.binary_cross_entropy_with_logits(((c / c.sum(1, keepdim=True)) * p[3][ids.long()]).sum(1), y.double())
    ref.backward()
    # rows of about 1 in fp32, sums over 48 columns and 700 tokens: 1e-5 covers the roundings; the gate's own gradient sees rows that are
    # off by half a step of 8 bits, a/254 with a about 2.5 times the rows' size, independently from row to row: 1 % of its norm
    assert abs(loss.item() - ref.item()) <= 1e-5
    for got, want, bound in ((dtable, p[0].grad, 1e-5), (dW, p[1].grad, 1e-2), (db, p[2].grad, 1e-5), (da, p[3].grad, 1e-5)):
        assert (got.double() - want).norm() <= bound * want.norm()


def test_token_gate_learns(ctx):
    from paper_2308_10037_b200.examples import token_gate
    _, losses, counts, _ = token_gate.train(120, ctx=ctx)
    assert losses[-10:].mean() < 0.5 < losses[:5].mean()     # 0.69 at the start, 0.33 is the planted noise's
    assert counts.sum().item() == 4096 * 2
