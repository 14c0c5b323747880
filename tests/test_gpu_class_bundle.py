"""Many short rows, which share warps: the same checks and tolerances as for any rows (test_gpu_class), at row lengths around where a lane holds one,
two, four and eight groups of 16 bytes, and rows of every kind beside one another."""
import math

import pytest
import torch

from test_gpu_class import close, errs, log_softmax, logits, targets, test_logp_and_its_gradient, test_policy_loss as check_policy
from test_gpu_gate import DT, ctx, gen, rnd, strided   # noqa: F401 (ctx is a fixture)

check_logp = test_logp_and_its_gradient
del test_logp_and_its_gradient
pytestmark = pytest.mark.gpu
SHAPES = [(1185, 1), (1191, 9), (2501, 128), (1300, 131), (1186, 255), (2402, 257), (1188, 512), (1187, 515), (4801, 1000), (1203, 1024), (1189, 1030)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", SHAPES)
def test_many_short_rows(ctx, dt, T, V):
    check_logp(ctx, dt, T, V)
    check_policy(ctx, dt, T, V)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 250, 700])
def test_rows_of_every_kind_beside_one_another(ctx, dt, V):
    """Masked classes, rows without a class, infinities, NaN, the lowest value, weights of 0, targets that do not count: none touches its
    neighbours, and each is as it is in a call of a few rows."""
    T = 1200
    x, y = logits(T, V, dt), targets(T, V, drop=0.2)
    kind = torch.randint(0, 9, (T,), generator=gen(8), device="cuda")
    x[kind == 0, : V // 2] = -math.inf
    x[kind == 1] = -math.inf
    x[kind == 2] = torch.finfo(x.dtype).min
    x[kind == 3, V // 3] = math.nan
    x[kind == 4, V // 5] = math.inf
    x[kind == 5] = (rnd(T, V, seed=9)[kind == 5] * 3 - 2000).to(x.dtype)
    w = torch.rand(T, generator=gen(10), device="cuda") + 0.5
    w[kind == 6] = 0.0
    adv = rnd(T, seed=11)
    x = strided(x, 5, 1)
    _, logp, d = ctx.policy_loss(x, y, adv, weights=w, norm=100.0)
    live = (y >= 0) & (w != 0)
    assert bool((logp[~live] == 0).all()) and bool((d[~live] == 0).all())
    lp = torch.where(live, log_softmax(x.double(), 1.0).gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    plain = live & ((kind == 2) | (kind > 4))
    close(logp[plain], lp[plain], errs(x[plain], 1.0)[0] + 2.0 ** -24 * lp[plain].abs())
    close(d[~plain].isnan().any(1), lp[~plain].isnan() | lp[~plain].isinf() & (kind[~plain] == 1), 0.0)
    for first in range(0, T, 400):                  # by a warp per row
        part = slice(first, first + 400)
        one = ctx.policy_loss(x[part], y[part], adv[part], weights=w[part], norm=100.0)
        close(logp[part], one[1], 2 * errs(x[plain], 1.0)[0] + 2.0 ** -23 * one[1].double().abs().nan_to_num(0.0, posinf=0.0, neginf=0.0))
        want = one[2].double()
        close(d[part], want, (1e-4 + 2 * torch.finfo(x.dtype).eps) * want.abs().nan_to_num(0.0) + 1e-38)
