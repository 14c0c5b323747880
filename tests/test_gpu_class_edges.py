"""The losses over a vocabulary's classes at the edges of what their documentation allows: very many rows, one class named by a whole row, few
SMs, launches that do not overlap, host threads, first calls that are captured.  Tolerances as in test_gpu_class."""
import math
import threading

import pytest
import torch

from paper_2308_10037_b200 import api
from test_gpu_class import (DT, HALF, U, close, ctx, distill_reference, errs, gen, log_softmax, logits, onehot, policy_reference,   # noqa: F401
                            pref_reference, rnd, targets)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,dt", [(300_000, 17, "f32"), (1_200_000, 5, "bf16"), (5000, 9000, "bf16"), (40_000, 3000, "bf16")])
def test_many_rows(ctx, T, V, dt):
    """More rows than warps, and more than one turn of the kernels that look the rows over."""
    x, y = logits(T, V, dt), targets(T, V, drop=0.4)
    live = y >= 0
    lp = torch.where(live, log_softmax(x.double(), 1.0).gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    L, P = errs(x, 1.0)
    got, lse = ctx.logp(x, y)
    close(got, lp, L + U * lp.abs())
    adv, w = rnd(T, seed=1), rnd(T, seed=2).abs()
    w[::7] = 0.0
    stats, lp2, d = ctx.policy_loss(x, y, adv, weights=w)
    n = torch.where(live, w.double(), 0.0).sum()
    g = torch.where(live, -adv.double() * w.double() / n, 0.0)
    counts = live & (w != 0)
    close(lp2, torch.where(counts, lp, 0.0), L + U * lp.abs())
    close(stats[0], g.sum(), 4 * U * float(g.abs().sum()) + 4 * U * float(g.sum().abs()))
    p = torch.softmax(x.double(), 1)
    hot = onehot(y, V)
    want = g[:, None] * (hot - p)
    close(d, want, g.abs()[:, None] * ((P + 8 * U) * p + (L + 8 * U) * hot) + 1.01 * HALF[dt] * want.abs() + 1e-38)
    again = ctx.policy_loss(x, y, adv, weights=w)
    assert all(torch.equal(a, b) for a, b in zip(again, (stats, lp2, d)))


@pytest.mark.parametrize("V", [900, 20_011])
def test_a_class_named_by_the_whole_row(ctx, V):
    T, K = 5, 1024
    x, t = logits(T, V, "f32"), rnd(T, K, seed=1)
    ids = torch.full((T, K), 13, device="cuda")
    ids[1] = torch.arange(K, device="cuda") % 31
    ids[2, 5:] = -1
    ids[3] = torch.arange(K, device="cuda") * 7 % V                          # (different where V is large enough)
    loss, kl, d = ctx.distill_loss(x, ids, t)
    want = distill_reference(x, ids, t, None, torch.ones(T, device="cuda"), 1.0, None, 1.0)
    L, P = errs(x, 1.0)
    close(kl, want[1], L + 8 * U * want[5] + U * want[1].abs())
    p = torch.softmax(x.double(), 1)
    q = torch.zeros_like(p).scatter_add_(1, ids.clamp(min=0), want[3])
    close(d, want[2], (p * (P + 6 * U) + q * (K + 8) * U) / T + 1.01 * U * want[2].abs() + 1e-38)


@pytest.mark.parametrize("sms,overlap", [(1, True), (10, True), (0, False)])
def test_few_sms_and_launches_one_after_the_other(sms, overlap):
    c = api.Context(n_max=1, device=0)
    c.set_sm_limit(sms)
    c.set_overlap(overlap)
    for T, V in ((300, 30_000), (40, 130_001), (700, 300)):
        x, y, adv = logits(T, V, "bf16"), targets(T, V, drop=0.3), rnd(T, seed=1)
        one = torch.ones(T, device="cuda")
        L, P = errs(x, 1.0)
        stats, lp, d = c.policy_loss(x, y, adv)
        want = policy_reference(x, y, adv, None, None, one, 1.0, 0.2, 0.2, 0.0, None, 1.0)
        close(lp, want[1], L + U * want[1].abs())
        p, size = torch.softmax(x.double(), 1), want[3][:, None]
        close(d, want[2], size * ((P + 8 * U) * p + (L + 8 * U) * onehot(y, V)) + 1.01 * HALF["bf16"] * want[2].abs() + 1e-38)
        o = torch.tensor([0, T // 3, T], device="cuda")
        loss, h, s, d = c.pref_loss(x, y, o)
        want = pref_reference(x, y, o, None, None, 0.1, 0.0, 0.0, False, 1.0, None, 1.0)
        close(s, want[2], L * T + 2 * U * want[2].abs())
        close(h, want[1], 0.1 * L * 2 * T + 4 * U * want[1].abs())
    assert c.device_status() == 0 and c.check_guards() == 0
    c.close()


def test_first_calls_that_are_captured():
    """A context's first call, and sizes that no call has had before: whatever is looked up or set once is looked up in the capture."""
    c = api.Context(n_max=1, device=0)
    T, V, K = 310, 21_111, 77
    x, y, t = logits(T, V, "f32"), targets(T, V, drop=0.2), rnd(T, K, seed=4)
    ids = torch.stack([torch.randperm(V, generator=gen(s), device="cuda")[:K] for s in range(T)])
    o, adv = torch.tensor([0, 100, 160, 200, 310], device="cuda"), rnd(T, seed=3)

    def calls():
        lp, lse = c.logp(x, y)
        return (lp, lse, c.logp_grad(x, y, lse, adv), *c.policy_loss(x, y, adv, weights=adv.abs()), *c.pref_loss(x, y, o), *c.distill_loss(x, ids, t))

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = calls()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    got = [v.clone() for v in got]
    assert all(torch.equal(a, b) for a, b in zip(got, calls()))
    x.mul_(0.5)                                     # the graph reads its inputs anew
    g.replay()
    fresh = calls()
    torch.cuda.synchronize()
    assert not torch.equal(fresh[0], got[0])
    del g
    c.close()


def test_threads_on_one_stream():
    """Host threads that share the default context: each call is enqueued as a whole."""
    T, V = 600, 9001
    work = [(logits(T, V, "bf16", seed=i), targets(T, V, seed=i, drop=0.2), rnd(T, seed=i)) for i in range(4)]
    o = torch.tensor([0, 150, 300, 450, 600], device="cuda")
    want = [(*api.lr_policy_loss(*w), *api.lr_pref_loss(w[0], w[1], o)) for w in work]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(4)

    def run(i):
        start.wait()
        for _ in range(20):
            got = (*api.lr_policy_loss(*work[i]), *api.lr_pref_loss(work[i][0], work[i][1], o))
            torch.cuda.current_stream().synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                wrong.append(i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == []


def test_slices_of_one_matrix_beside_each_other(ctx):
    """Logits and gradient as column blocks of one matrix; rows of a matrix that ends with its memory."""
    T, V = 37, 4000
    both = torch.zeros(T, 2 * V, device="cuda")
    both[:, :V] = logits(T, V, "f32")
    y, adv = targets(T, V), rnd(T, seed=2)
    want = ctx.policy_loss(both[:, :V], y, adv)[2]
    ctx.policy_loss(both[:, :V], y, adv, out=both[:, V:])
    assert torch.equal(both[:, V:], want)
    with pytest.raises(api.LrError):
        ctx.policy_loss(both[:, :V], y, adv, out=both[:, 10:V + 10])
    for V in (1, 5, 4097, 70_001):                  # the last row ends at the end of an allocation of its own size
        for dt in ("f32", "bf16"):
            x = torch.empty(3, V, dtype=DT[dt], device="cuda")
            x.copy_(logits(3, V, dt))
            close(ctx.logp(x, targets(3, V))[0], log_softmax(x.double(), 1.0).gather(1, targets(3, V)[:, None])[:, 0], 1e-4)
    assert ctx.check_guards() == 0


def test_scales_and_factors_at_their_ends(ctx):
    x, y, adv = logits(4, 700, "f32"), targets(4, 700), rnd(4, seed=1)
    for scale in (1e-6, 1e-30, 50.0, 1e6):
        lp = log_softmax(x.double(), float(torch.tensor(scale)))[torch.arange(4), y]
        close(ctx.logp(x, y, scale=scale)[0], lp, 2e-4 + 8 * U * lp.abs())
    for bad in (3e38, math.inf, -1.0, math.nan):
        with pytest.raises(api.LrError):
            ctx.logp(x, y, scale=bad)
    assert bool((ctx.policy_loss(x, y, adv, factor=0.0)[2] == 0).all())
    a, b = ctx.policy_loss(x, y, adv, norm=2.0), ctx.policy_loss(x, y, adv, norm=1.0, factor=0.5)
    assert torch.equal(a[2], b[2]) and float(a[0][0]) == float(b[0][0])
