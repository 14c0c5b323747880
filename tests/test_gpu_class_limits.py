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
