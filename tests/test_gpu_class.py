"""The losses over a vocabulary's classes against plain implementations in float64, whose gradients come from automatic differentiation
and from differences.

Tolerances, with u = 2^-24 (fp32 rounding), R the largest distance of a row's scaled logits from their maximum, derived from the operations:
  a term of a row    2^a with a = (x - top) * c: the difference, c and the product are rounded, each is u |a| in a, |a| <= R / ln 2; the power
                     itself is good to 2^-22: (3R + 4) u relative
  a row's sum        a thread's chain of at most 32 + V / (32 * 64) terms, then trees and the other warps: at most 100 additions here:
                     (3R + 104) u relative; lse and lp, the rest of which is fp64 but for a logarithm good to 2u, are off by that: (3R + 110) u =: L
  p                  its term and the sum: (6R + 115) u relative =: P
  a row's factor g   policy: |r A| L + kl_coef e^(ref-lp) L;  preference: |dloss/dh| <= beta, curvature <= 1/4, both over a sum of n rows
  a gradient         (p + [target]) times the error of g, |g| (P p + [target] L), three roundings of products, and half a step of its type
"""
import math

import pytest
import torch

from paper_2308_10037_b200 import api
from test_gpu_gate import DT, U, ctx, gen, rnd, strided   # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu
HALF = {"f32": U, "bf16": 2.0 ** -8}
SHAPES = [(1, 1), (1, 2), (3, 3), (2, 7), (5, 8), (4, 31), (6, 64), (3, 257), (2, 1000), (17, 1003), (7, 4097), (300, 12), (2, 32000), (2, 50021),
          (1, 131072), (2, 200003), (1500, 40)]


def logits(T, V, dt, seed=0, spread=3.0, shift=0.0):
    x = rnd(T, V, seed=seed + T + V) * spread + shift
    x[torch.arange(T, device="cuda"), torch.randint(0, V, (T,), generator=gen(seed + 1), device="cuda")] += 6.0
    return x.to(DT[dt])


def targets(T, V, seed=0, drop=0.0, ignore=-100):
    y = torch.randint(0, V, (T,), generator=gen(seed + 2), device="cuda")
    if drop:
        y[torch.rand(T, generator=gen(seed + 3), device="cuda") < drop] = ignore
    return y


def log_softmax(x, scale):
    return torch.log_softmax(x * scale, 1)


def spread_of(x, scale):
    """R: finite distances from the row's maximum."""
    l = x.double() * scale
    d = l.amax(1, keepdim=True) - l
    d = d[torch.isfinite(d)]
    return float(d.max()) if d.numel() else 0.0


def errs(x, scale):
    R = spread_of(x, scale)
    return (3 * R + 110) * U, (6 * R + 115) * U


def close(got, want, bound):
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    bound = torch.as_tensor(bound, dtype=torch.float64, device=got.device).expand(got.shape)
    same = (got == want) | (got.isnan() & want.isnan())
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= bound)
    assert not bool(bad.any()), f"{int(bad.sum())} off, worst {float((off - bound).max()):.3e} over its bound, largest error {float(off.max()):.3e}"


def onehot(y, V):
    hot = torch.zeros(len(y), V, dtype=torch.float64, device="cuda")
    rows = (y >= 0) & (y < V)
    hot[rows, y[rows]] = 1.0
    return hot


def grad_bound(x, scale, y, g, g_err, dt, want):
    """Of dlogits = scale * g * (onehot - p) for a row factor g that is off by g_err."""
    L, P = errs(x, scale)
    p = torch.exp(log_softmax(x.double(), scale)).nan_to_num(0.0)
    hot = onehot(y, x.shape[1])
    g, g_err = g.abs()[:, None], g_err[:, None]
    return scale * ((p + hot) * g_err + g * (P * p + (L + 4 * U) * hot + 4 * U * p)) + 1.01 * HALF[dt] * want.abs() + 1e-38


# ---- log-probabilities -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", SHAPES)
def test_logp_and_its_gradient(ctx, dt, T, V):
    scale = 1.3 if T % 2 else 1.0
    x, y = logits(T, V, dt), targets(T, V, drop=0.3)
    x[y == -100] = float("nan")                     # rows that do not count are not read
    lp = log_softmax(x.double(), scale)
    live = y >= 0
    want = torch.where(live, lp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    lse = torch.where(live, torch.logsumexp(x.double() * scale, 1), 0.0)
    got, got_lse = ctx.logp(x, y, scale=scale)
    L, P = errs(x, scale)
    close(got, want, L + U * want.abs())
    close(got_lse, lse, L + 2 * U * lse.abs())
    again = ctx.logp(x, y.int(), scale=scale)
    assert torch.equal(again[0], got) and torch.equal(again[1], got_lse)

    g = rnd(T, seed=5)
    d = ctx.logp_grad(x, y, got_lse, g, scale=scale)
    assert d.dtype == x.dtype
    # the gradient is that of the lse it is given
    p = torch.exp(x.double() * scale - got_lse.double()[:, None])
    want = torch.where(live[:, None], scale * g.double()[:, None] * (onehot(y, V) - p), 0.0)
    p = p.nan_to_num(0.0)
    bound = scale * g.double().abs()[:, None] * (P * p + 4 * U * (p + onehot(y, V))) + 1.01 * HALF[dt] * want.abs() + 1e-38
    close(d, want, bound)
    assert torch.equal(ctx.logp_grad(x, y.int(), got_lse, g, scale=scale), d)
    # a slice of a wider matrix whose other columns are NaN, into a slice at another offset, and in place
    for shift in (0, 1, 3):
        xs = strided(x, 11, shift)
        close(ctx.logp(xs, y, scale=scale)[0], got, 2 * L + 2 * U * got.double().abs())     # (sums in another order)
        out = strided(torch.full((T, V), 7.0, dtype=DT[dt], device="cuda"), 13, 2)
        ctx.logp_grad(xs, y, got_lse, g, scale=scale, out=out)
        assert torch.equal(out, d)
        base = out._base if out._base is not None else out
        assert bool(base.view(-1)[:2].isnan().all())                                        # nothing beside the slice is written
        assert torch.equal(ctx.logp_grad(xs, y, got_lse, g, scale=scale), d)
    assert torch.equal(ctx.logp_grad(x, y, got_lse, g, scale=scale, out=x), d) and torch.equal(x, d)


def test_logp_far_from_zero_and_masked(ctx):
    V = 5000
    for shift in (1000.0, -3000.0):
        x = (rnd(4, V, seed=1) * 3 + shift).contiguous()
        y = targets(4, V)
        lp = log_softmax(x.double(), 1.0).gather(1, y[:, None])[:, 0]
        close(ctx.logp(x, y)[0], lp, errs(x, 1.0)[0] + U * lp.abs())
        close(ctx.logp(x, y)[1], torch.logsumexp(x.double(), 1), 2 * U * abs(shift) + errs(x, 1.0)[0])
    x = rnd(6, V, seed=2)
    x[:, ::2] = -math.inf                           # half of the classes masked
    x[1] = -math.inf
    x[1, 7] = 3.0                                   # one class left
    x[2] = -math.inf                                # none left
    x[3, 5] = math.nan
    x[4, 5] = math.inf
    x[5, 0] = torch.finfo(torch.float32).min        # the lowest value is no infinity
    y = torch.tensor([1, 7, 7, 1, 1, 0], device="cuda")
    for dt in ("f32", "bf16"):
        xx = x.to(DT[dt])
        if dt == "bf16":
            xx[5, 0] = torch.finfo(torch.bfloat16).min
        want = log_softmax(xx.double(), 1.0).gather(1, y[:, None])[:, 0]
        got, lse = ctx.logp(xx, y)
        assert bool(got[2:5].isnan().all()) and bool(want[2:5].isnan().all())
        assert float(got[1]) == 0.0                 # the one term is 1
        close(got[[0, 1]], want[[0, 1]], 1e-5)
        close(got[5:], want[5:], 4 * U * want[5:].abs())
        d = ctx.logp_grad(xx, y, lse, torch.ones(6, device="cuda"))
        assert bool((d[0, ::2] == 0).all()) and float(d[1].abs().max()) <= 115 * U + HALF[dt] and bool(d[3].isnan().all())
        assert float(d[5, 0]) == 1.0


@pytest.mark.parametrize("V", [40, 3000, 50021])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rows_far_out(ctx, dt, V):
    """Rows at the type's lowest or highest value, at the values that programs mask with, and far from zero with differences of their own."""
    lowest = torch.finfo(DT[dt]).min
    rows = [torch.full((V,), v) for v in (lowest, -lowest, -1e9, -1e30, -1e4, 0.0, -65504.0)]
    rows += [torch.full((V,), lowest), torch.full((V,), -1e9), torch.full((V,), lowest)]
    rows[7][3] = 2.0                                # all but one masked
    rows[8][5:9] = torch.tensor([1.0, 2.0, 3.0, 4.0])
    rows[9][::2] = -1e30                            # one mask above another
    x = torch.stack(rows).to(DT[dt]).cuda()
    T = len(rows)
    y = torch.full((T,), 7, device="cuda")
    y[7], y[9] = 3, 4
    want = log_softmax(x.double(), 1.0).gather(1, y[:, None])[:, 0]
    lp, lse = ctx.logp(x, y)
    close(lp, want, 110 * U + 2 * U * want.abs())
    close(lse, torch.logsumexp(x.double(), 1), 110 * U + 2 * U * torch.logsumexp(x.double(), 1).abs())
    adv, one = torch.linspace(-1, 1, T, device="cuda"), torch.ones(T, device="cuda")
    stats, _, d = ctx.policy_loss(x, y, adv)
    ref = policy_reference(x, y, adv, None, None, one, 1.0, 0.2, 0.2, 0.0, None, 1.0)
    p = torch.softmax(x.double(), 1)
    close(d, ref[2], adv.double().abs()[:, None] / T * (p + onehot(y, V)) * 230 * U + 1.01 * HALF[dt] * ref[2].abs() + 1e-38)
    ids = torch.stack([torch.arange(3, 9, device="cuda")] * T)
    t = rnd(T, 6)
    loss, kl, dd = ctx.distill_loss(x, ids, t)
    want = distill_reference(x, ids, t, None, one, 1.0, None, 1.0)
    close(kl, want[1], 300 * U + 8 * U * (want[1].abs() + want[5]))
    q = torch.zeros(T, V, dtype=torch.float64, device="cuda").scatter_add_(1, ids, want[3])
    close(dd, want[2], (p * 230 * U + q * 14 * U) / T + 1.01 * HALF[dt] * want[2].abs() + 1e-38)


def test_policy_loss_of_unlikely_rows(ctx):
    """Ratios beyond fp32, targets without probability, an advantage of zero."""
    x = rnd(6, 50, seed=1)
    x[0, 3] = x[1, 3] = -math.inf
    y = torch.full((6,), 3, device="cuda")
    adv = torch.tensor([1.0, -1.0, 0.0, 1.0, 0.0, -2.0], device="cuda")
    lp = ctx.logp(x, y)[0]
    old = torch.stack([torch.tensor(-3.0), torch.tensor(-3.0), torch.tensor(-200.0), torch.tensor(-200.0), torch.tensor(200.0), torch.tensor(150.0)]).cuda()
    stats, got, d = ctx.policy_loss(x, y, adv, old)
    assert torch.equal(got, lp) and float(got[0]) == -math.inf
    assert bool(torch.isfinite(d).all()) and bool(torch.isfinite(stats).all())
    assert bool((d[2] == 0).all()) and bool((d[3] == 0).all()) and bool((d[4] == 0).all())      # no advantage; held by the clip; no advantage
    # -min(r A, r' A) with r' = r held in [0.8, 1.2]: row 3 (r huge) -1.2; rows 1 and 5 (r = 0, A = -1 and -2: r A = 0 > r' A) 0.8 and 1.6; these
    # three are held; row 0 (r = 0, A = 1) and the rows without an advantage 0
    assert abs(float(stats[1]) - (-1.2 + 0.8 + 1.6) / 6) < 1e-6
    assert abs(float(stats[3]) - 3 / 6) < 1e-6


def test_targets_outside_the_classes(ctx):
    x = rnd(5, 100)
    y = torch.tensor([3, -1, 100, 2 ** 40, -100], device="cuda")
    lp, lse = ctx.logp(x, y)
    assert bool((lp[1:] == 0).all()) and bool((lse[1:] == 0).all()) and float(lp[0]) < 0
    assert ctx.device_status() == api.LR_ERR_VALUE
    d = ctx.logp_grad(x, y, lse, torch.ones(5, device="cuda"))
    assert bool((d[1:] == 0).all()) and bool((d[0] != 0).any())
    assert ctx.device_status() == api.LR_ERR_VALUE
    stats, lp2, d2 = ctx.policy_loss(x, y, torch.ones(5, device="cuda"))
    assert torch.equal(lp2, lp) and bool((d2[1:] == 0).all()) and float(stats[1]) == -1.0     # one row counts
    assert ctx.device_status() == api.LR_ERR_VALUE
    ctx.logp(x, torch.tensor([3, 7, 7, 99, 0], device="cuda"), ignore_id=7)
    assert ctx.device_status() == 0


# ---- policy loss -----------------------------------------------------------------------------------------

def policy_reference(x, y, adv, old, ref, w, scale, low, high, kl_coef, norm, factor):
    """(stats, lp, dlogits, row factor g, its sensitivity) in float64."""
    x = x.double().clone()
    live = (y >= 0) & (w != 0)
    x[~live] = 0.0
    x.requires_grad_(True)
    lp = log_softmax(x, scale).gather(1, y.clamp(min=0)[:, None])[:, 0]
    ratio = torch.exp(lp - (old.double() if old is not None else lp.detach()))
    held = ratio.clamp(1 - low, 1 + high)
    first = -torch.minimum(ratio * adv.double(), held * adv.double())
    d = ref.double() - lp if ref is not None else torch.zeros_like(lp)
    kl = torch.exp(d) - d - 1
    wl = torch.where(live, w.double(), 0.0)
    n = float(wl.sum()) if norm is None else norm
    inv = 1.0 / n if n else 0.0
    loss = factor * ((first + kl_coef * kl) * wl).sum() * inv
    clipped = (ratio * adv.double() > held * adv.double()).double()
    stats = torch.stack([loss, (first * wl).sum() * inv, (kl * wl).sum() * inv, (clipped * wl).sum() * inv]).detach()
    (dx,) = torch.autograd.grad(loss, x)
    with torch.no_grad():
        share = wl.abs() * abs(inv * factor)
        size = share * ((ratio * adv.double()).abs() + (abs(kl_coef) * torch.exp(d) if ref is not None else 0.0) + abs(kl_coef))
        cancel = (((first.abs() + kl.abs() * abs(kl_coef)) * wl.abs()).sum() * abs(inv) * abs(factor), (first.abs() * wl.abs()).sum() * abs(inv),
                  ((kl.abs() + torch.exp(d)) * wl.abs()).sum() * abs(inv), clipped.sum() * 0)
    return stats, torch.where(live, lp, 0.0).detach(), dx, size, cancel


def ratios(lp, seed):
    """Older log-probabilities that put the ratio well away from the borders 0.8 and 1.25."""
    r = torch.tensor([0.5, 0.7, 0.95, 1.0, 1.1, 1.4, 1.9], device="cuda", dtype=torch.float64)
    return (lp - torch.log(r[torch.randint(0, 7, lp.shape, generator=gen(seed), device="cuda")])).float()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", SHAPES)
def test_policy_loss(ctx, dt, T, V):
    scale = 0.7 if T % 3 == 0 else 1.0
    x, y, adv = logits(T, V, dt), targets(T, V, drop=0.25), rnd(T, seed=3)
    lp = log_softmax(x.double(), scale).gather(1, y.clamp(min=0)[:, None])[:, 0]
    old, ref = ratios(lp, 4), (lp + 0.4 * rnd(T, seed=6)).float()
    w = rnd(T, seed=8).abs()
    w[::5] = 0.0
    x[(y < 0) | (w == 0)] = float("nan")
    one = torch.ones(T, device="cuda")
    for old_, ref_, w_, kl_coef, norm, factor in [(old, ref, w, 0.1, None, 1.0), (old, None, None, 0.0, 37.0, 2.5), (None, ref, w, 0.3, None, -1.5)]:
        xx = x if w_ is not None else torch.where((y < 0)[:, None], x, logits(T, V, dt))
        stats, want_lp, want, size, cancel = policy_reference(xx, y, adv, old_, ref_, one if w_ is None else w_, scale, 0.2, 0.25, kl_coef, norm, factor)
        got, got_lp, d = ctx.policy_loss(xx, y, adv, old_, ref_, w_, scale=scale, clip_low=0.2, clip_high=0.25, kl_coef=kl_coef, norm=norm,
                                         factor=factor)
        clean = torch.where(((y < 0) | ((one if w_ is None else w_) == 0))[:, None], 0.0, xx.float())
        L, P = errs(clean, scale)
        close(got_lp, want_lp, L + U * want_lp.abs())
        for i in range(4):
            close(got[i], stats[i], (L + 8 * U) * float(cancel[i]) + 4 * U * float(stats[i].abs()) + 1e-38)
        live = ((y >= 0) & ((one if w_ is None else w_) != 0)).double()
        close(d, want, grad_bound(clean, scale, y, size * live, size * live * (L + 8 * U), dt, want))
        got2, lp2, none = ctx.policy_loss(xx, y.int(), adv, old_, ref_, w_, scale=scale, clip_low=0.2, clip_high=0.25, kl_coef=kl_coef, norm=norm,
                                          factor=factor, grad=False)
        assert none is None and torch.equal(got2, got) and torch.equal(lp2, got_lp)
    # a slice, into a slice at another offset, and in place
    args = (y, adv, old, ref, w)
    kw = dict(scale=scale, kl_coef=0.1)
    stats, _, d = ctx.policy_loss(x, *args, **kw)
    again = ctx.policy_loss(x, *args, **kw)
    assert torch.equal(again[0], stats) and torch.equal(again[2], d)
    xs = strided(x, 5, 3)
    out = strided(torch.zeros(T, V, dtype=DT[dt], device="cuda"), 9, 4)
    assert ctx.policy_loss(xs, *args, out=out, **kw)[2] is out
    fresh = ctx.policy_loss(xs, *args, **kw)[2]
    assert torch.equal(fresh, out)
    inplace = ctx.policy_loss(xs, *args, out=xs, **kw)[2]
    assert torch.equal(inplace, out)


def test_policy_loss_where_nothing_counts(ctx):
    x, adv = torch.full((5, 300), math.nan, device="cuda"), rnd(5)
    y = torch.full((5,), -100, device="cuda")
    for yy, w in ((y, None), (targets(5, 300), torch.zeros(5, device="cuda"))):
        stats, lp, d = ctx.policy_loss(x, yy, adv, weights=w)
        assert bool((stats == 0).all()) and bool((lp == 0).all()) and bool((d == 0).all())
    stats, lp, d = ctx.policy_loss(x[:0], y[:0], adv[:0])
    assert bool((stats == 0).all()) and lp.shape == (0,) and d.shape == (0, 300)
    assert ctx.logp(x[:0], y[:0])[0].shape == (0,) and ctx.logp_grad(x[:0], y[:0], adv[:0], adv[:0]).shape == (0, 300)
    loss, rows, d = ctx.distill_loss(x, torch.zeros(5, 4, dtype=torch.int64, device="cuda"), torch.zeros(5, 4, device="cuda"),
                                     weights=torch.zeros(5, device="cuda"))
    assert float(loss) == 0 and bool((rows == 0).all()) and bool((d == 0).all())
    loss, h, s, d = ctx.pref_loss(x, y, torch.tensor([0, 2, 5], device="cuda"))
    assert abs(float(loss) - math.log(2)) < 4 * U and float(h) == 0 and bool((s == 0).all()) and bool((d == 0).all())
    loss, h, s, d = ctx.pref_loss(x, y, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert float(loss) == 0 and h.shape == (0,) and s.shape == (0,) and bool((d == 0).all())
    loss, h, s, d = ctx.pref_loss(x[:0], y[:0], torch.zeros(3, dtype=torch.int32, device="cuda"), margin=1.0)
    assert abs(float(loss) - math.log1p(math.e)) < 8 * U and d.shape == (0, 300)


def test_policy_clip_options(ctx):
    T, V = 64, 200
    x, y, adv = logits(T, V, "f32"), targets(T, V), rnd(T, seed=2)
    lp = log_softmax(x.double(), 1.0).gather(1, y[:, None])[:, 0]
    old = ratios(lp, 9)
    free, _, d = ctx.policy_loss(x, y, adv, old, clip_low=math.inf, clip_high=math.inf)
    assert float(free[3]) == 0.0
    want = policy_reference(x, y, adv, old, None, torch.ones(T, device="cuda"), 1.0, 1e9, 1e9, 0.0, None, 1.0)
    close(free[:2], want[0][:2], 1e-4)
    held = ctx.policy_loss(x, y, adv, old, clip_low=0.0, clip_high=0.0)[0]
    want = policy_reference(x, y, adv, old, None, torch.ones(T, device="cuda"), 1.0, 0.0, 0.0, 0.0, None, 1.0)
    r = torch.exp(lp - old.double())
    sure = ((r - 1).abs() > 1e-3)
    assert abs(float(held[3]) - float(((r > 1) & (adv > 0) | (r < 1) & (adv < 0))[sure].sum()) / T) <= float((~sure).sum()) / T + 1e-6


# ---- preference loss -------------------------------------------------------------------------------------

def pref_reference(x, y, offsets, ref, w, beta, margin, smoothing, average, scale, norm, factor):
    o = [int(v) for v in offsets.tolist()]
    P = len(o) // 2
    rows = torch.arange(len(y), device="cuda")
    live = (y >= 0) & (rows >= o[0]) & (rows < o[-1])
    x = torch.where(live[:, None], x.double(), 0.0).requires_grad_(True)
    lp = torch.where(live, log_softmax(x, scale).gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    n = torch.tensor([max(1, int(live[a:z].sum())) for a, z in zip(o, o[1:])], dtype=torch.float64, device="cuda")
    s = torch.stack([lp[a:z].sum() if z > a else zero for a, z in zip(o, o[1:])])
    if average:
        s = s / n
    d = s - (ref.double() if ref is not None else 0.0)
    h = beta * (d[:P] - d[P:]) - margin
    ls = torch.nn.functional.logsigmoid             # (softplus has exp(h) in its derivative: not a number beyond h = 709)
    each = -(1 - smoothing) * ls(h) - smoothing * ls(-h)
    wl = torch.ones(P, dtype=torch.float64, device="cuda") if w is None else w.double()
    total = float(wl.sum()) if norm is None else norm
    inv = 1.0 / total if total else 0.0
    loss = factor * (each * wl).sum() * inv
    (dx,) = torch.autograd.grad(loss, x)
    return loss.detach().view(1), h.detach(), s.detach(), dx, n, wl, inv


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V,lens", [(7, (1, 1)), (1, (2, 3)), (33, (4, 0, 5, 6)), (1000, (3, 9, 0, 2, 8, 1)), (4099, (20, 1, 30, 2)),
                                    (130, (150, 300, 299, 1, 0, 2, 77, 500)), (50021, (3, 4)), (200003, (1, 1))])
def test_pref_loss(ctx, dt, V, lens):
    first, behind = (2, 3) if V % 2 else (0, 0)     # rows before the first sequence and behind the last
    o = torch.tensor([first, *lens], device="cuda").cumsum(0)
    T, P = int(o[-1]) + behind, len(lens) // 2
    x, y = logits(T, V, dt), targets(T, V, drop=0.2)
    x[(y < 0)] = math.nan
    x[:first] = math.nan
    x[T - behind:] = math.nan
    ref, w = rnd(2 * P, seed=3) * 3, rnd(P, seed=4).abs() + 0.1
    clean = torch.where(x.isnan(), 0.0, x.float())
    for beta, margin, smoothing, average, r, ww, norm, factor, scale in [
            (0.1, 0.0, 0.0, False, ref, None, None, 1.0, 1.0), (2.0, 0.5, 0.1, True, None, w, None, 1.0, 0.8),
            (0.3, 0.0, 0.3, False, ref, w, 5.0, -2.0, 1.0)]:
        loss, h, s, want, n, wl, inv = pref_reference(x, y, o, r, ww, beta, margin, smoothing, average, scale, norm, factor)
        got, gh, gs, d = ctx.pref_loss(x, y, o, r, ww, beta=beta, margin=margin, smoothing=smoothing, average=average, scale=scale, norm=norm,
                                       factor=factor)
        L, _ = errs(clean, scale)
        size = torch.tensor(lens, dtype=torch.float64, device="cuda")
        s_err = L * (torch.ones_like(size) if average else size)
        close(gs, s, s_err + 2 * U * s.abs())
        h_err = beta * (s_err[:P] + s_err[P:])
        close(gh, h, h_err + 4 * U * (h.abs() + abs(margin)))
        close(got, loss, abs(factor) * abs(inv) * (wl * h_err).sum() + 4 * U * loss.abs())
        owner = torch.bucketize(torch.arange(T, device="cuda"), o[1:], right=True).clamp(max=2 * P - 1)
        rows = torch.arange(T, device="cuda")
        inside = ((rows >= o[0]) & (rows < o[-1]) & (y >= 0)).double()
        each = (wl * abs(inv) * abs(factor) * beta).repeat(2) / (n if average else 1.0)
        g = each[owner] * inside
        g_err = g * (h_err.repeat(2)[owner] / 4 + 6 * U)
        close(d, want, grad_bound(clean, scale, y, g, g_err, dt, want))
        again = ctx.pref_loss(x, y.int(), o.int(), r, ww, beta=beta, margin=margin, smoothing=smoothing, average=average, scale=scale, norm=norm,
                              factor=factor)
        assert all(torch.equal(a, b) for a, b in zip(again, (got, gh, gs, d)))
        quiet = ctx.pref_loss(x, y, o, r, ww, beta=beta, margin=margin, smoothing=smoothing, average=average, scale=scale, norm=norm,
                              factor=factor, grad=False)
        assert quiet[3] is None and torch.equal(quiet[0], got)
    mine = x.clone()
    got = ctx.pref_loss(mine, y, o, ref)[3]
    assert torch.equal(ctx.pref_loss(mine, y, o, ref, out=mine)[3], got) and torch.equal(mine, got)


def test_pref_saturates_without_overflow(ctx):
    """h of hundreds either way: the loss is |h| or 0, the gradient's factor beta or 0."""
    x, y = rnd(40, 50) * 2, targets(40, 50)
    o = torch.tensor([0, 20, 40], device="cuda")
    for r in (torch.tensor([1e4, 0.0]), torch.tensor([0.0, 1e4]), torch.tensor([3e38, 0.0])):
        ref = r.cuda()
        loss, h, s, d = ctx.pref_loss(x, y, o, ref, beta=1.0)
        want = pref_reference(x, y, o, ref, None, 1.0, 0.0, 0.0, False, 1.0, None, 1.0)
        close(loss, want[0], 1e-6 * want[0].abs() + 1e-38)
        close(d, want[3], 1e-4)


def test_pref_bad_offsets_read_nothing(ctx):
    x, y = rnd(10, 50), targets(10, 50)
    for o in ([0, 11, 10], [-3, 5, 10], [0, 7, 5], [0, 2 ** 40, 10], [5, 3, 2 ** 62]):
        loss, h, s, d = ctx.pref_loss(x, y, torch.tensor(o, device="cuda"))
        assert ctx.device_status() == api.LR_ERR_VALUE
        assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(d).all())
    assert ctx.device_status() == 0


# ---- distillation ----------------------------------------------------------------------------------------

def distill_reference(x, ids, t, tlse, w, scale, norm, factor, ignore=-1):
    V = x.shape[1]
    live = w != 0
    x = torch.where(live[:, None], x.double(), 0.0).requires_grad_(True)
    here = (ids >= 0) & (ids < V) & (t != -math.inf)
    z = torch.where(here, t.double() * scale, -math.inf)
    lse = tlse.double()[:, None] if tlse is not None else torch.logsumexp(z, 1, keepdim=True)
    logq = z - lse
    q = torch.where(here, torch.exp(logq), 0.0)
    lp = log_softmax(x, scale).gather(1, ids.clamp(0, V - 1).long())
    rows = torch.where(q > 0, q * (logq - lp), 0.0).sum(1)
    wl = torch.where(live, w.double(), 0.0)
    total = float(wl.sum()) if norm is None else norm
    inv = 1.0 / total if total else 0.0
    loss = factor * torch.where(live, rows * wl, 0.0).sum() * inv
    (dx,) = torch.autograd.grad(loss, x)
    mass = (q * (logq.abs().nan_to_num(0.0, 0.0, 0.0) + lp.abs())).sum(1).detach()
    return loss.detach().view(1), torch.where(live, rows, 0.0).detach(), dx, q.detach(), wl * abs(inv), mass


@pytest.mark.parametrize("dt,tt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (3, 2, 1), (2, 7, 7), (5, 8, 3), (4, 300, 33), (6, 1003, 64), (2, 4097, 256), (1, 5000, 1024), (40, 130, 5),
                                   (2, 50021, 8), (1, 131072, 64), (2, 200003, 31)])
def test_distill_loss(ctx, dt, tt, T, V, K):
    x = logits(T, V, dt)
    ids = torch.stack([torch.randperm(V, generator=gen(s), device="cuda")[:K] for s in range(T)])
    t = (3 * rnd(T, K, seed=2)).to(DT[tt])
    w = rnd(T, seed=8).abs() + 0.2
    if T > 2:
        w[1] = 0.0
        x[1] = math.nan
        t[2, 0] = -math.inf                         # absent
    if K > 2:
        ids[0, 1] = -1                              # absent, as are all the others in the last row
        ids[0, 2] = ids[0, 0]                       # named twice
    if T > 3:
        ids[-1] = -1
    one = torch.ones(T, device="cuda")
    for scale, part, ww, norm, factor in [(1.0, False, w, None, 1.0), (0.5, True, w, 3.0, 4.0), (1.2, False, w, None, -1.0)]:
        tlse = (torch.logsumexp(t.float() * scale, 1) + 0.3).nan_to_num(0.0, neginf=0.0) if part else None
        loss, rows, want, q, wl, mass = distill_reference(x, ids, t, tlse, ww, scale, norm, factor)
        got, gr, d = ctx.distill_loss(x, ids, t, tlse, ww, scale=scale, norm=norm, factor=factor)
        clean = torch.where((ww == 0)[:, None], 0.0, x.float())
        L, P = errs(clean, scale)
        Q = q.sum(1)
        close(gr, rows, Q * L + 8 * U * mass + U * rows.abs())
        close(got, loss, abs(factor) * float((wl * (Q * L + 8 * U * mass)).sum()) + 4 * U * float(loss.abs()))
        p = torch.exp(log_softmax(clean.double(), scale))
        qv = torch.zeros_like(p).scatter_add_(1, ids.clamp(0, V - 1).long(), q)
        gain = (wl * abs(factor) * scale)[:, None]
        close(d, want, gain * (Q[:, None] * p * (P + 6 * U) + qv * (K + 8) * U) + 1.01 * HALF[dt] * want.abs() + 1e-38)
        again = ctx.distill_loss(x, ids.int(), t, tlse, ww, scale=scale, norm=norm, factor=factor)
        assert all(torch.equal(a, b) for a, b in zip(again, (got, gr, d)))
        quiet = ctx.distill_loss(x, ids, t, tlse, ww, scale=scale, norm=norm, factor=factor, grad=False)
        assert quiet[2] is None and torch.equal(quiet[0], got) and torch.equal(quiet[1], gr)
    assert ctx.device_status() == 0
    got = ctx.distill_loss(torch.where(x.isnan(), 0.0, x.float()).to(x.dtype), ids, t)      # no weights: every row counts
    want = distill_reference(torch.where(x.isnan(), 0.0, x.float()), ids, t, None, one, 1.0, None, 1.0)
    close(got[0], want[0], errs(torch.where(x.isnan(), 0.0, x.float()), 1.0)[0] * 2 + 1e-6 * float(want[0].abs()))
    xs = strided(x, 7, 5)
    out = strided(torch.zeros(T, V, dtype=DT[dt], device="cuda"), 6, 1)
    ctx.distill_loss(xs, ids, t, weights=w, out=out)
    assert torch.equal(out, ctx.distill_loss(xs, ids, t, weights=w, out=xs)[2])


def test_distill_classes_outside_and_absent(ctx):
    x, t = rnd(3, 20), rnd(3, 4, seed=1)
    ids = torch.tensor([[1, 2, 3, 20], [4, -5, 6, 7], [-7, -7, -7, -7]], device="cuda")
    got = ctx.distill_loss(x, ids, t, ignore_id=-7)
    assert ctx.device_status() == api.LR_ERR_VALUE
    want = distill_reference(x, ids, t, None, torch.ones(3, device="cuda"), 1.0, None, 1.0)
    close(got[1], want[1], 1e-5)
    close(got[2], want[2], 1e-5)
    assert float(got[1][2]) == 0 and bool((got[2][2] == 0).all())
    ctx.distill_loss(x, ids.clamp(-7, 19).masked_fill(ids == -5, -7), t, ignore_id=-7)
    assert ctx.device_status() == 0
    x[0, 1] = -math.inf                             # a class of the teacher that the student masks: the loss is infinite, the gradient finite
    loss, rows, d = ctx.distill_loss(x, ids.clamp(0, 19), t)
    assert float(rows[0]) == math.inf and float(loss) == math.inf and bool(torch.isfinite(d).all()) and float(d[0, 1]) < 0


# ---- differences, offsets, streams, graphs ---------------------------------------------------------------

def test_gradients_against_differences(ctx):
    """<gradient, v> against differences of the 64-bit losses along random directions v; a central difference over 2h of a loss with a third
    derivative of a few is off by h^2, h = 1e-4, and by 1e-16 / h."""
    T, V, K = 12, 90, 5
    x, y = logits(T, V, "f32"), targets(T, V, drop=0.2)
    lp = log_softmax(x.double(), 1.0).gather(1, y.clamp(min=0)[:, None])[:, 0]
    adv, old, ref, w = rnd(T, seed=1), ratios(lp, 2), (lp + 0.3).float(), torch.ones(T, device="cuda")
    o, sref = torch.tensor([0, 3, 5, 9, 12], device="cuda"), rnd(4, seed=3)
    ids, t = torch.randint(0, V, (T, K), generator=gen(4), device="cuda"), rnd(T, K, seed=5)
    losses = {
        "policy": (lambda z: policy_reference(z, y, adv, old, ref, w, 1.0, 0.2, 0.25, 0.1, None, 1.0)[0][0],
                   ctx.policy_loss(x, y, adv, old, ref, clip_low=0.2, clip_high=0.25, kl_coef=0.1)[2]),
        "pref": (lambda z: pref_reference(z, y, o, sref, None, 0.5, 0.1, 0.1, False, 1.0, None, 1.0)[0][0],
                 ctx.pref_loss(x, y, o, sref, beta=0.5, margin=0.1, smoothing=0.1)[3]),
        "distill": (lambda z: distill_reference(z, ids, t, None, w, 1.0, None, 1.0)[0][0], ctx.distill_loss(x, ids, t)[2]),
    }
    for name, (f, d) in losses.items():
        for s in range(5):
            v = rnd(T, V, seed=100 + s).double()
            diff = (f(x.double() + 1e-4 * v) - f(x.double() - 1e-4 * v)) / 2e-4
            dot = (d.double() * v).sum()
            L, P = errs(x, 1.0)
            assert abs(float(diff - dot)) <= 2 * (L + P) * float((d.double() * v).abs().sum()) + 1e-6 + P, name


def test_offsets_beyond_32_bits(ctx):
    """Rows that start past 2^31 elements."""
    V, T = 200_000, 11_000                          # 2.2e9 elements of bfloat16
    x = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    tail = logits(3, V, "bf16")
    x[-3:] = tail
    y = torch.full((T,), -100, device="cuda")
    y[-3:] = targets(3, V)
    adv = rnd(T)
    lp, lse = ctx.logp(x, y)
    assert torch.equal(lp[-3:], ctx.logp(tail, y[-3:])[0]) and bool((lp[:-3] == 0).all())
    want = ctx.policy_loss(tail, y[-3:], adv[-3:])
    got = ctx.policy_loss(x, y, adv, out=x)         # the gradient replaces the logits
    assert torch.equal(got[0], want[0]) and torch.equal(x[-3:], want[2]) and bool((x[:-3].amax(1) == 0).all())


def test_a_step_of_them_together(ctx):
    """Scores of a reference and of the acting policy, then the three losses on them: the results of separate 64-bit passes."""
    T, V, P = 60, 777, 3
    new, refx, oldx = (logits(T, V, "bf16", seed=s) for s in (0, 50, 90))
    y, adv = targets(T, V, drop=0.2), rnd(T, seed=1)
    ref, ref_lse = ctx.logp(refx, y)
    old, _ = ctx.logp(oldx, y)
    o = torch.tensor([0, 12, 20, 33, 41, 50, 60], device="cuda")
    seq_ref = ctx.pref_loss(refx, y, o, grad=False)[2]
    top = refx.float().topk(16, 1)
    stats, lp, d1 = ctx.policy_loss(new, y, adv, old, ref, kl_coef=0.05, clip_low=0.2, clip_high=0.25)
    _, h, s, d2 = ctx.pref_loss(new, y, o, seq_ref)
    _, _, d3 = ctx.distill_loss(new, top[1], top[0], torch.logsumexp(refx.float(), 1))
    one = torch.ones(T, device="cuda")
    want = [policy_reference(new, y, adv, old, ref, one, 1.0, 0.2, 0.25, 0.05, None, 1.0)[2],
            pref_reference(new, y, o, pref_reference(refx, y, o, None, None, 0.1, 0, 0, False, 1.0, None, 1.0)[2], None, 0.1, 0, 0, False, 1.0,
                           None, 1.0)[3],
            distill_reference(new, top[1], top[0], torch.logsumexp(refx.double(), 1), one, 1.0, None, 1.0)[2]]
    for got, w in zip((d1, d2, d3), want):
        assert float((got.double() - w).norm()) <= 2.0 ** -8 * float(w.norm())
    # the gradient written by hand through logp_grad is the policy's: no clip, no reference
    free = ctx.policy_loss(new, y, adv, old, clip_low=math.inf, clip_high=math.inf)
    lp, lse = ctx.logp(new, y)
    g = torch.where(y >= 0, -adv * torch.exp(lp - old) / (y >= 0).sum(), 0.0)
    mine = ctx.logp_grad(new, y, lse, g)
    assert float((mine.double() - free[2].double()).norm()) <= 2.0 ** -7 * float(free[2].double().norm())


def all_calls(c, x, y, adv, o, ids, t):
    lp, lse = api.lr_logp(x, y, ctx=c)
    return (lp, lse, api.lr_logp_grad(x, y, lse, adv, ctx=c), *api.lr_policy_loss(x, y, adv, lp.detach() + 0.1, kl_coef=0.1, ctx=c),
            *api.lr_pref_loss(x, y, o, ctx=c), *api.lr_distill_loss(x, ids, t, weights=adv.abs(), ctx=c))


def problem(i, T=500, V=3001, dt="bf16"):
    x, y = logits(T, V, dt, seed=i), targets(T, V, seed=i, drop=0.3)
    o = torch.tensor([0, 100, 220, 300, 500], device="cuda")
    return x, y, rnd(T, seed=i), o, torch.randint(0, V, (T, 12), generator=gen(i), device="cuda"), rnd(T, 12, seed=i)


@pytest.mark.parametrize("shared", [False, True])
def test_graphs_and_streams(ctx, shared):
    c = ctx if shared else None
    work = [problem(i) for i in range(3)]
    want = [[t.clone() for t in all_calls(c, *w)] for w in work]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for w in work[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(all_calls(c, *w))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
        eager = all_calls(c, *work[2])
    torch.cuda.synchronize()
    for got, exp in zip((*outs, eager), want):
        assert all(torch.equal(a, b) for a, b in zip(got, exp))
    assert ctx.check_guards() == 0
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        side = all_calls(None, *work[0])
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(side, want[0]))
