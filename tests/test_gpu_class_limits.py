"""The losses over a vocabulary's classes where a number is infinite, absent or out of its place.  Tolerances as in test_gpu_class."""
import math

import pytest
import torch

from paper_2308_10037_b200 import api
from test_gpu_class import (DT, HALF, U, close, ctx, distill_reference, errs, gen, log_softmax, logits, onehot, rnd, strided, targets)   # noqa: F401

pytestmark = pytest.mark.gpu
# rows by a warp, several to a warp, by a CTA that looks at them on its way, from its own list, from a kernel's list, and by clusters
WAYS = [(5, 130), (1300, 60), (9, 9000), (310, 4500), (4500, 4200), (2, 50021)]


# ---- a teacher's classes ---------------------------------------------------------------------------------

def kinds_of_classes(T, V, K, ignore, seed=0):
    """A teacher's lists that are padded with `ignore`, a class like any other: some lists hold it here and there, one holds nothing else."""
    ids = torch.randint(0, V, (T, K), generator=gen(seed), device="cuda")
    ids[torch.rand(T, K, generator=gen(seed + 1), device="cuda") < 0.4] = ignore
    ids[0, K // 2:] = ignore
    ids[T // 2] = ignore
    return ids


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", WAYS)
def test_a_class_of_the_vocabulary_that_is_ignored(ctx, dt, T, V):
    K, scale = 12, 0.8
    x, t, one = logits(T, V, dt), 3 * rnd(T, K, seed=2), torch.ones(T, device="cuda")
    for ignore in (0, V - 1, V // 2):
        ids = kinds_of_classes(T, V, K, ignore)
        gone = ids.masked_fill(ids == ignore, -1)
        for tlse in (None, torch.logsumexp(t * scale, 1) + 0.2):
            loss, rows, want, q, wl, mass = distill_reference(x, gone, t, tlse, one, scale, None, 1.0)
            got, gr, d = ctx.distill_loss(x, ids, t, tlse, scale=scale, ignore_id=ignore)
            L, P = errs(x, scale)
            Q = q.sum(1)
            close(gr, rows, Q * L + 8 * U * mass + U * rows.abs())
            close(got, loss, float((wl * (Q * L + 8 * U * mass)).sum()) + 4 * U * float(loss.abs()))
            p = torch.softmax(x.double() * scale, 1)
            qv = torch.zeros_like(p).scatter_add_(1, gone.clamp(min=0), q)
            close(d, want, scale * wl[:, None] * (Q[:, None] * p * (P + 6 * U) + qv * (K + 8) * U) + 1.01 * HALF[dt] * want.abs() + 1e-38)
            assert float(gr[T // 2]) == 0.0 and bool((d[T // 2] == 0).all())
            quiet = ctx.distill_loss(x, ids.int(), t, tlse, scale=scale, ignore_id=ignore, grad=False)
            assert torch.equal(quiet[0], got) and torch.equal(quiet[1], gr)
            other = ctx.distill_loss(x, gone, t, tlse, scale=scale)
            assert all(torch.equal(a, b) for a, b in zip(other, (got, gr, d)))
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", WAYS)
def test_rows_without_a_teacher(ctx, dt, T, V):
    """A row of which all classes are absent has loss and gradient 0, whatever its logits hold; its neighbours do not see it."""
    K = 5
    x, t = logits(T, V, dt), rnd(T, K, seed=2)
    ids = torch.randint(0, V, (T, K), generator=gen(3), device="cuda")
    none = torch.zeros(T, dtype=torch.bool, device="cuda")
    none[::3] = True
    ids[none] = -1
    ids[0], t[0] = 1, -math.inf                     # the other way to be absent
    want = ctx.distill_loss(x, ids, t)
    for junk in (math.nan, math.inf, -math.inf):
        xx = x.clone()
        xx[none] = junk
        if T > 3:
            xx[3] = x[3]
            xx[3, V // 2] = junk
        got = ctx.distill_loss(xx, ids, t)
        assert bool((got[2][none] == 0).all()) and bool((got[1][none] == 0).all())
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- an infinite log-probability -------------------------------------------------------------------------

def pref_by_hand(x, y, o, ref, w, beta, margin, smoothing, average=False, scale=1.0):
    """(loss, margins, seq_logp, dlogits, each row's coefficient) in float64 from the definition: a term of a loss whose factor is 0 is left out; a
    sequence whose own offsets fall or leave the rows is empty; a row that several sequences hold counts in each."""
    T, P = len(y), len(o) // 2
    lp = log_softmax(x.double(), scale).gather(1, y.clamp(0, x.shape[1] - 1)[:, None])[:, 0]
    live = (y >= 0) & (y < x.shape[1])
    lp = torch.where(live, lp, 0.0)
    rows = [range(a, z) if 0 <= a <= z <= T else range(0) for a, z in zip(o, o[1:])]
    n = [max(1, int(live[r.start:r.stop].sum())) if average else 1 for r in rows]
    s = [lp[r.start:r.stop].sum() / m if len(r) else torch.zeros((), dtype=torch.float64, device="cuda") for r, m in zip(rows, n)]
    s = torch.stack(s)
    d = s - (ref.double() if ref is not None else 0.0)
    h = beta * (d[:P] - d[P:]) - margin
    wl = torch.ones(P, dtype=torch.float64, device="cuda") if w is None else w.double()
    inv = 1.0 / float(wl.sum()) if float(wl.sum()) else 0.0
    loss, coef = 0.0, torch.zeros(T, dtype=torch.float64, device="cuda")
    for i in range(P):
        if float(wl[i]) == 0.0:
            continue
        hi, each = float(h[i]), 0.0
        soft = math.nan if hi != hi else math.log1p(math.exp(-abs(hi)))
        if smoothing < 1:
            each += (1 - smoothing) * (max(-hi, 0.0) + soft)
        if smoothing > 0:
            each += smoothing * (max(hi, 0.0) + soft)
        right = math.nan if hi != hi else 1 / (1 + math.exp(-hi)) if hi > -700 else 0.0
        wrong = math.nan if hi != hi else 1 / (1 + math.exp(hi)) if hi < 700 else 0.0
        loss += float(wl[i]) * each * inv
        g = float(wl[i]) * inv * beta * (smoothing * right - (1 - smoothing) * wrong)
        for j, sign in ((i, 1.0), (i + P, -1.0)):
            coef[rows[j].start:rows[j].stop] += sign * g / n[j]
    coef = torch.where(live, coef, 0.0)
    p = torch.softmax(x.double() * scale, 1)
    dx = torch.where((coef != 0)[:, None], scale * coef[:, None] * (onehot(y, x.shape[1]) - p), 0.0)
    return torch.tensor([loss], dtype=torch.float64, device="cuda"), h, s, dx, coef


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 5000, 50021])
def test_a_sequence_without_probability(ctx, dt, V):
    """A target on a masked class: the pair's margin is infinite.  A rejected answer that cannot be is rejected for good (loss 0, no gradient); a
    preferred one has an infinite loss and the largest gradient."""
    o = [0, 4, 7, 12, 15, 20, 22]
    T = o[-1]
    x, y = logits(T, V, dt), targets(T, V, drop=0.1)
    y[[5, 13, 16]] = 3
    ref = rnd(6, seed=4)
    for mask_at, smoothing, w in [((13,), 0.0, None), ((13,), 0.2, None), ((5,), 0.0, None), ((5,), 0.1, None), ((5,), 1.0, None), ((16,), 0.0, None),
                                  ((5, 13), 0.0, None), ((5,), 0.0, torch.tensor([1.0, 0.0, 2.0], device="cuda"))]:
        xx = x.clone()
        for at in mask_at:
            xx[at, 3] = -math.inf
        loss, h, s, want, coef = pref_by_hand(xx, y, o, ref, w, 0.3, 0.1, smoothing)
        got, gh, gs, d = ctx.pref_loss(xx, y, torch.tensor(o, device="cuda"), ref, w, beta=0.3, margin=0.1, smoothing=smoothing)
        L, P = errs(xx, 1.0)
        fine = s.isfinite()
        assert torch.equal(gs[~fine].double(), s[~fine]) and torch.equal(gh[~h.isfinite()].double(), h[~h.isfinite()])
        close(gs[fine], s[fine], 6 * L + 2 * U * s[fine].abs())
        if math.isfinite(float(loss)):
            close(got, loss, 0.3 * 12 * L + 4 * U * loss.abs())
        else:
            assert float(got) == float(loss)
        p = torch.softmax(xx.double(), 1)
        c = coef.abs()[:, None]
        close(d, want, c * ((p + onehot(y, V)) * (0.3 * 12 * L + 6 * U) + P * p + (L + 8 * U) * onehot(y, V)) + 1.01 * HALF[dt] * want.abs() + 1e-38)


def test_margins_beyond_fp32(ctx):
    """h past fp32's largest number, by a reference and by classes at the type's lowest value."""
    x, y = rnd(40, 50) * 2, targets(40, 50)
    o = [0, 20, 40]
    for r, beta in (([3e38, -3e38], 2.0), ([-3e38, 3e38], 2.0), ([math.inf, 0.0], 0.5), ([0.0, math.inf], 0.5), ([200.0, 0.0], 1.0), ([0.0, 200.0], 1.0)):
        ref = torch.tensor(r, device="cuda")
        loss, h, s, want, coef = pref_by_hand(x, y, o, ref, None, beta, 0.0, 0.0)
        got, gh, gs, d = ctx.pref_loss(x, y, torch.tensor(o, device="cuda"), ref, beta=beta)
        close(gh, h.float(), 1e-6 * h.abs().nan_to_num(0.0, posinf=0.0) + 1e-4)
        close(got, loss.float(), 1e-5 * loss.abs().nan_to_num(0.0, posinf=0.0) + 1e-38)
        close(d, want, 1e-4 * want.abs() + 1e-6 * coef.abs()[:, None] + 1e-38)
    low = torch.finfo(torch.float32).min
    x[25, 3], y[25] = low, 3
    x[30, 3], y[30] = low, 3
    got, gh, gs, d = ctx.pref_loss(x, y, torch.tensor(o, device="cuda"), beta=2.0)
    assert float(gh) == math.inf and float(got) == 0.0 and bool((d == 0).all())
    got, gh, gs, d = ctx.pref_loss(x, y, torch.tensor([0, 0, 40], device="cuda"), beta=-2.0)
    assert float(gh) == -math.inf and float(got) == math.inf and bool(torch.isfinite(d).all()) and bool((d != 0).any())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(6, 50), (1200, 50), (6, 5000), (160, 5000), (6, 50021)])
def test_a_reference_that_is_far_off(ctx, dt, T, V):
    """exp(ref - lp) past fp32, and a target without probability under a reference that has one."""
    x, y, adv = logits(T, V, dt), torch.full((T,), 3, device="cuda"), rnd(T, seed=1)
    x[0, 3] = -math.inf                             # no probability
    x[1, 3] = -300.0                                # hardly one
    x[2, :2] = -math.inf                            # masked classes beside the target
    x[1, 5:9] = -math.inf
    ref = torch.full((T,), -2.0, device="cuda")
    ref[2] = 200.0
    ref[3] = -math.inf                              # the reference has none: a loss, but no gradient of its own
    ref[4:] = ctx.logp(x, y)[0][4:] + 0.2
    plain = ctx.policy_loss(x, y, adv)
    stats, lp, d = ctx.policy_loss(x, y, adv, None, ref)            # watched only
    assert torch.equal(stats[:2], plain[0][:2]) and torch.equal(d, plain[2]) and float(stats[2]) == math.inf
    assert bool(torch.isfinite(d).all())
    stats, lp, d = ctx.policy_loss(x, y, adv, None, ref, kl_coef=0.1, norm=1.0)
    assert float(stats[0]) == math.inf and float(stats[2]) == math.inf and torch.equal(stats[1:2], ctx.policy_loss(x, y, adv, norm=1.0)[0][1:2])
    assert bool(torch.isfinite(d).all())
    assert bool((d[0] >= 0).sum() >= V - 1) and float(d[0, 3]) < -1e37 and bool((d[1, 5:9] == 0).all()) and bool((d[2, :2] == 0).all())
    # what is finite is as before: without rows 0 to 3
    rest = ctx.policy_loss(x[4:], y[4:], adv[4:], None, ref[4:], kl_coef=0.1, norm=1.0)
    L, P = errs(x[4:], 1.0)
    size = (adv[4:].double().abs() + 0.1 * math.exp(0.2) + 0.1)[:, None] * (torch.softmax(x[4:].double(), 1) + onehot(y[4:], V))
    close(d[4:], rest[2], 2 * (L + P) * size + 2.0 ** -7 * (dt == "bf16") * rest[2].double().abs() + 1e-38)
    # beyond fp32 whatever the norm, with advantages above 1, both signs and a large factor
    old = torch.full((T,), -400.0, device="cuda")
    d = ctx.policy_loss(x, y, torch.full((T,), -3.0, device="cuda"), old, ref, kl_coef=7.0, norm=1e-3, factor=100.0)[2]
    assert bool(torch.isfinite(d).all()) and bool((d[1, 5:9] == 0).all())


# ---- offsets ---------------------------------------------------------------------------------------------

def check_offsets(ctx, T, V, dt, o, average=False):
    x, y = logits(T, V, dt), targets(T, V, drop=0.2)
    junk = logits(T, V, dt, seed=7, spread=30.0)
    ctx.pref_loss(junk, targets(T, V), torch.tensor([0, T // 2, T], device="cuda"))          # other values where the call works
    bad = any(not 0 <= a <= z <= T for a, z in zip(o, o[1:]))
    inside = torch.zeros(T, dtype=torch.bool, device="cuda")
    for a, z in zip(o, o[1:]):
        if 0 <= a <= z <= T:
            inside[a:z] = True
    x[~inside] = math.nan                           # rows outside all sequences do not count
    clean = torch.where(inside[:, None], x.float(), 0.0).to(x.dtype)
    loss, h, s, want, coef = pref_by_hand(clean, torch.where(inside, y, -100), o, None, None, 0.05, 0.0, 0.1, average)
    got, gh, gs, d = ctx.pref_loss(x, y, torch.tensor(o, device="cuda"), beta=0.05, smoothing=0.1, average=average)
    assert ctx.device_status() == (api.LR_ERR_VALUE if bad else 0)
    L, P = errs(clean, 1.0)
    most = max([z - a for a, z in zip(o, o[1:]) if 0 <= a <= z <= T], default=0)
    s_err = L * (1 if average else most)
    close(gs, s, s_err + 2 * U * s.abs())
    close(gh, h, 0.1 * s_err + 4 * U * h.abs())
    close(got, loss, 0.1 * s_err + 4 * U * loss.abs())
    p = torch.softmax(clean.double(), 1)
    c = coef.abs()[:, None]
    # the coefficient of a row of two sequences is a difference: its parts are at most beta / P
    part = (0.05 / (len(o) // 2)) * inside.double()[:, None]
    close(d, want, part * (p + onehot(y, V)) * (0.1 * s_err + 12 * U) + c * (P * p + (L + 8 * U) * onehot(y, V)) + 1.01 * HALF[dt] * want.abs() + 1e-38)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", WAYS)
@pytest.mark.parametrize("average", [False, True])
def test_a_sequence_counts_by_its_own_offsets(ctx, dt, T, V, average):
    """Only a sequence whose own offsets fall or leave the rows is empty."""
    a, b, c = T // 5, T // 2, T - T // 4
    for o in ([0, c, b], [b, 0, T], [0, b, T + 1], [-1, b, T], [0, c, 0], [a, b, c], [0, b, c, a, a], [c, a, b, T, b], [T, 0, 0, b, b]):
        check_offsets(ctx, T, V, dt, o, average)


@pytest.mark.parametrize("T,V", [(1300, 60), (900, 4200), (5000, 4200)])
def test_many_sequences_with_rows_outside(ctx, T, V):
    """More sequences than a warp looks through for the rows between the first and the last."""
    n = 2 * 140
    edges = torch.linspace(T // 6, T - T // 6, n + 1).long().tolist()
    check_offsets(ctx, T, V, "f32", edges)
    fall = list(edges)
    fall[n], fall[3] = edges[n - 3], T + 5          # the last falls, two others leave the rows
    check_offsets(ctx, T, V, "f32", fall)


@pytest.mark.parametrize("T,V", WAYS)
def test_rows_of_two_sequences(ctx, T, V):
    """Where falling offsets make sequences overlap, a row counts in each of them."""
    a, b, c = T // 5, T // 2, T - T // 4
    for o in ([0, c, a, b, T], [0, T, 0, T, T], [a, T, 0, c, c]):
        check_offsets(ctx, T, V, "f32", o)


# ---- numbers that fp32 does not hold ---------------------------------------------------------------------

@pytest.mark.parametrize("scale", [1e-38, 3e-39, 1e-41])
@pytest.mark.parametrize("V", [50, 5000, 200003])
def test_scales_that_make_every_class_alike(ctx, scale, V):
    """lse / scale is past fp32's largest number: the gradient is that of equal classes all the same, and so is a teacher's q."""
    T, K = 3, 4
    x, y = logits(T, V, "f32"), targets(T, V)
    got, lse = ctx.logp(x, y, scale=scale)
    close(got, torch.full((T,), -math.log(V), device="cuda"), 110 * U + U * math.log(V))
    g = rnd(T, seed=1) * 1e37
    s = float(torch.tensor(scale, dtype=torch.float32))
    gt = (g.double() * s)[:, None]
    p = torch.exp(x.double() * s - lse.double()[:, None])
    want = gt * (onehot(y, V) - p)
    d = ctx.logp_grad(x, y, lse, g, scale=scale)
    # the exponent is at most log2(V) < 18, and rounded like every term's (3 * 18 u); (x - 2^128) c is off by 2^128 times half a step of c, which below
    # fp32's normal numbers is 2^-150: 2^-22 = 4 u
    close(d, want, gt.abs() * ((54 + 4 + 115) * U * p + 8 * U * onehot(y, V)) + 2e-38 + U * want.abs())
    t = rnd(T, K, seed=2)
    ids = torch.stack([torch.arange(K, device="cuda")] * T)
    tlse = torch.full((T,), 9.0, device="cuda")
    kl = ctx.distill_loss(x, ids, t, tlse, scale=scale)[1]
    q = torch.exp(t.double() * s - 9.0)
    close(kl, (q * (math.log(V) - 9.0)).sum(1), float(q.sum(1).max()) * (110 + 60) * U * (9.0 + math.log(V)))


# ---- the gradient in place of the logits -----------------------------------------------------------------

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(3, 50021), (20, 131072), (60, 40000), (300, 128000)])
def test_rows_of_a_cluster_in_place(ctx, dt, T, V):
    """CTAs that share a row read each other's part of it only as long as it holds logits: the same bits in place and beside, targets at
    the ends of the row, in its middle and in its unaligned edges."""
    x = strided(logits(T, V, dt), 3, 1)
    y = targets(T, V, drop=0.1)
    y[::4], y[1::4] = 0, V - 1
    adv, old = rnd(T, seed=1), ctx.logp(x, y)[0] + 0.1
    ids = torch.randint(0, V, (T, 40), generator=gen(5), device="cuda")
    ids[:, 0], ids[:, 1] = 0, V - 1
    t = rnd(T, 40, seed=6)
    stats, lp, d = ctx.policy_loss(x, y, adv, old, clip_low=1.0, clip_high=9.0)
    loss, kl, dd = ctx.distill_loss(x, ids, t)
    for _ in range(10):
        mine = strided(x, 3, 1)
        got = ctx.policy_loss(mine, y, adv, old, clip_low=1.0, clip_high=9.0, out=mine)
        assert torch.equal(got[0], stats) and torch.equal(got[1], lp) and torch.equal(mine, d)
        mine = strided(x, 3, 1)
        got = ctx.distill_loss(mine, ids, t, out=mine)
        assert torch.equal(got[0], loss) and torch.equal(got[1], kl) and torch.equal(mine, dd)


# ---- errors that add up ----------------------------------------------------------------------------------

def nearly_exact_scale():
    """A scale near 1 whose product with log2(e) fp32 holds to 1e-10: the exponents are then off by their own rounding alone."""
    s = torch.arange(-2 ** 14, 2 ** 14, dtype=torch.float64) * 2.0 ** -23 + 1.0
    c = s * math.log2(math.e)
    off = (c.float().double() / c - 1).abs()
    assert float(off.min()) < 1e-10
    return float(s[off.argmin()])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V,scale", [(500, None), (4096, None), (9001, None), (9001, 1.0), (9001, 0.7), (32003, 1.25)])
def test_errors_of_a_long_sequence_cancel(ctx, dt, V, scale):
    """The mean signed error of lp over many rows, of terms of every size and of equal ones: an error that all rows share would add up over a
    sequence.  lp is rounded to half a step of 2^-20 (3e-7 in the mean square), its sum and logarithm less: 4 / sqrt(8192) of it is 1.3e-8; the
    powers' mean error is 3e-9, and 3e-8 in the few terms above 1/2; the scale's 1e-9 (long rows: any scale's, short ones: of one that is nearly
    exact).  3e-8 in all; an uncorrected power gives 5e-8."""
    scale = float(torch.tensor(scale or nearly_exact_scale(), dtype=torch.float32))
    T = 8192
    y = torch.randint(0, V, (T,), generator=gen(1), device="cuda")
    kinds = {"random": 2.5 * rnd(T, V, seed=2), "near one another": 0.3 * rnd(T, V, seed=5), "of one value": rnd(T, 1, seed=3).expand(T, V).contiguous()}
    kinds["ties beside masked classes"] = kinds["of one value"].clone()
    count = torch.randint(2, V + 1, (T, 1), generator=gen(4), device="cuda")
    kinds["ties beside masked classes"][torch.arange(V, device="cuda") >= count] = -math.inf
    for name, x in kinds.items():
        x = x.to(DT[dt])
        at = y if name in ("random", "near one another") else y % 2
        want = torch.cat([torch.log_softmax(p.double() * scale, 1).gather(1, i[:, None])[:, 0] for p, i in zip(x.split(512), at.split(512))])
        off = float((ctx.logp(x, at, scale=scale)[0].double() - want).mean())
        if name == "of one value":                  # (one number for all rows: its own rounding)
            assert abs(off) <= 0.5 * 2.0 ** -20 + 1e-7
        else:
            assert abs(off) <= 3e-8, (name, off)


@pytest.mark.parametrize("part", [False, True])
@pytest.mark.parametrize("V,K", [(900, 200), (40000, 200), (40000, 1024)])
def test_the_divergence_has_the_bits_of_its_terms(ctx, V, K, part):
    """Errors of the rows' divergences over 400 rows, student and teacher far apart, in the mean square and relative to the sum of the magnitudes m
    (10 or more times the mass).  An entry's power is off by 1u in the mean square, which the few entries that matter average to 0.5u; the student's
    log-sum-exp by a logarithm good to 1u and by scale * log2(e) in fp32, u / 2 of a distance of up to 15: 0.8u of m in all; the result's own
    rounding is less than 0.3u of m.  Together 1u; 1.2u is asked for.  A teacher's exponent held in fp32 alone, 5 to 20 in size, is off by u / 2
    of itself from scale * log2(e) alone, for all entries alike: 2u of m and more where nothing divides it away."""
    T, scale = 400, 0.9
    x, t = 2.5 * rnd(T, V, seed=1), -20 * torch.rand(T, K, generator=gen(2), device="cuda") + 40 * rnd(T, 1, seed=3)
    ids = torch.stack([torch.randperm(V, generator=gen(10 + i), device="cuda")[:K] for i in range(T)])
    s = float(torch.tensor(scale, dtype=torch.float32))
    z = t.double() * s
    tlse = (torch.logsumexp(z, 1) + 0.3).float() if part else None
    logq = z - (tlse.double()[:, None] if part else torch.logsumexp(z, 1, keepdim=True))
    lp = torch.log_softmax(x.double() * s, 1).gather(1, ids)
    want = (logq.exp() * (logq - lp)).sum(1)
    m = (logq.exp() * (logq.abs() + lp.abs())).sum(1)
    off = (ctx.distill_loss(x, ids, t, tlse, scale=scale, grad=False)[1].double() - want) / m
    assert float(off.square().mean().sqrt()) <= 1.2 * U


# ---- the clip's borders ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(1, 3), (1200, 20), (2, 9000)])
def test_rows_next_to_the_borders_of_the_clip(ctx, dt, T, V):
    """Rows whose one class has log-probability 0, so that the ratio is exp(-old) to all bits: older scores one fp32 step after the other across
    the logarithms of both borders, which are far closer to each other than fp32 ratios are."""
    x = torch.full((T, V), -math.inf, device="cuda").to(DT[dt])
    x[:, V // 2] = 1.0
    y = torch.full((T,), V // 2, device="cuda")
    clip_low, clip_high = 0.2, 0.25
    low, high = (float(torch.tensor(c, dtype=torch.float32)) for c in (clip_low, clip_high))
    for border, sign in ((math.log1p(high), 1.0), (math.log1p(-low), -1.0)):
        old = torch.tensor(-border, dtype=torch.float32)
        steps = [old]
        for _ in range(5):
            steps = [torch.nextafter(steps[0], torch.tensor(-10.0))] + steps + [torch.nextafter(steps[-1], torch.tensor(10.0))]
        for o in steps:
            stats = ctx.policy_loss(x, y, torch.full((T,), sign, device="cuda"), torch.full((T,), float(o), device="cuda"), clip_low=clip_low,
                                    clip_high=clip_high)[0]
            past = -float(o) > border if sign > 0 else -float(o) < border
            assert float(stats[3]) == float(past), (float(o), border)
            assert float(ctx.policy_loss(x, y, torch.full((T,), -sign, device="cuda"), torch.full((T,), float(o), device="cuda"), clip_low=clip_low,
                                         clip_high=clip_high)[0][3]) == 0.0
