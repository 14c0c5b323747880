"""Edges of the token-gate calls: saturated scores, tokens outside the table, refusals, status words, new contexts."""
import pytest
import torch

from paper_2308_10037_b200 import api
from test_gpu_gate import DT, U, close, ctx, gen, rnd   # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_grad_of_saturated_sigmoids(ctx, dt, renorm):
    # relative to the derivative itself, not to the largest one: both sigmoids take an exp (2 ulp) and a quotient, the weights a sum more
    x = (torch.arange(-80, 81, device="cuda").float() / 2)[:, None] + torch.tensor([0.0, 0.25, -0.5], device="cuda")
    x = torch.cat([x, 2 * x]).to(DT[dt])
    T = x.shape[0]
    ids = torch.tensor([[2, 0]], dtype=torch.int32, device="cuda").repeat(T, 1)
    g = rnd(T, 2, seed=1)
    z = x.double().gather(1, ids.long())
    p, rest = torch.sigmoid(z), torch.sigmoid(-z)
    lg = torch.nn.functional.logsigmoid(z)
    w = torch.softmax(lg, 1)
    G = g.double()
    if renorm:
        d = 2.5 * (G - (G * w).sum(1, keepdim=True)) * w * rest
        bound = 160 * U * 2.5 * G.abs().sum(1, keepdim=True) * w * rest
    else:
        d = 2.5 * G * p * rest
        bound = 40 * U * d.abs()
    want = torch.zeros_like(x, dtype=torch.float64).scatter_(1, ids.long(), d)
    room = torch.zeros_like(want).scatter_(1, ids.long(), bound)
    got = ctx.route_grad(x, ids, g, score="sigmoid", renorm=renorm, factor=2.5)
    close(got, want, room + (2.0 ** -8 * want.abs() if dt == "bf16" else 0.0) + 2.0 ** -126)


@pytest.mark.parametrize("T", [3, 3000])
def test_tokens_outside_the_table_are_reported_whatever_the_padding(ctx, T):
    V, n = 20, 12
    dout = rnd(T, n)
    assert ctx.device_status() == 0
    for token, padding, status in ((-1, -1, api.LR_ERR_VALUE), (V + 5, V + 5, api.LR_ERR_VALUE), (-4, -1, api.LR_ERR_VALUE), (7, 7, 0)):
        ids = torch.full((T,), 3, device="cuda")
        ids[T // 2] = token
        got = ctx.embed_grad(ids, dout, V, padding_id=padding)
        assert ctx.device_status() == status, token
        want = dout.double().sum(0) - dout[T // 2].double()
        close(got[3], want, (T + 3) * U * dout.double().abs().sum(0))
        assert int((got != 0).any(dim=1).sum()) == 1


def test_a_refused_embed_grad_launches_nothing(ctx):
    n = 65535 * 256 + 1
    out, dout = torch.full((1, n), 7.0, device="cuda"), torch.ones(1, n, device="cuda")
    before = ctx.launch_count()
    with pytest.raises(api.LrError) as e:
        ctx.embed_grad(torch.zeros(1, dtype=torch.int64, device="cuda"), dout, 1, out=out)
    assert e.value.code == api.LR_ERR_SHAPE
    assert ctx.launch_count() == before and bool((out == 7.0).all())


def test_a_token_outside_the_table_does_not_hide_a_wait_that_ran_out(ctx):
    table, outside = rnd(4, 8), torch.tensor([9], device="cuda")
    assert ctx.device_status() == 0
    for first in (True, False):                     # whichever was reported first
        if first:
            ctx.embed(table, outside)
        ctx.selftest_wait(arm=False, limit_ms=20)
        if not first:
            ctx.embed_grad(outside, rnd(1, 8), 4)
        assert [ctx.device_status() for _ in range(3)] == [api.LR_ERR_TIMEOUT, api.LR_ERR_VALUE, 0]
