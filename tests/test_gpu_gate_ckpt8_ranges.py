"""The gradient taken from rows kept in 8 bits where dz and the scales differ widely between rows, and where values are not finite.

Every element of the gradient is held to (8 + sqrt(T)) u times its own sum of magnitudes sum_t |dz[t,c] s[t,g] q[t,j]|, u = 2^-24: a
chain of T rounded products and additions whose rounding errors add up like sqrt(T).  So a row that is masked (dz = 0), or
whose q is zero in a column, must not cost that column's other rows any bits, whatever its scale or dz."""
import math

import pytest
import torch

from test_gpu_gate import DT, U, close, ctx, gen, padded_groups, rnd   # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


def wanted(q, s, dz):
    x = (padded_groups(q) * s.double()[:, :, None]).flatten(1)[:, :q.shape[1]]
    return dz.double().t() @ x, dz.double().abs().t() @ x.abs()


def check(ctx, q, s, dz):
    T = q.shape[0]
    want, mag = wanted(q, s, dz)
    assert float(want.abs().max()) < 3e38 and float(mag.max()) < 3e38
    for rows in (q, strided_bytes(q)):              # as a tensor-map copy reads it, and rows of any alignment
        gw, gb = ctx.ckpt8_grad(rows, s, dz)
        assert bool(torch.isfinite(gw).all()) and bool(torch.isfinite(gb).all())
        close(gw, want, (8 + math.sqrt(T)) * U * mag)
        close(gb, dz.double().sum(0), (8 + math.sqrt(T)) * U * dz.double().abs().sum(0))


def strided_bytes(q):
    wide = torch.zeros(q.shape[0], q.shape[1] + 5, dtype=torch.int8, device="cuda")
    wide[:, 3:3 + q.shape[1]] = q
    return wide[:, 3:3 + q.shape[1]]


CLASSES = [1, 2, 20, 64, 100]


@pytest.mark.parametrize("C", CLASSES)
@pytest.mark.parametrize("T", [64, 1000, 4096])
@pytest.mark.parametrize("times", [1e2, 1e4, 1e6, 1e10, 1e20])
def test_a_masked_row_with_a_large_scale(ctx, T, C, times):
    q, s = ctx.ckpt8_save(rnd(T, 300, seed=T))
    dz = rnd(T, C, seed=C) * 1e-3
    s[T // 3] *= times
    dz[T // 3] = 0
    check(ctx, q, s, dz)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("C", CLASSES)
def test_large_scales_stand_beside_small_dz(ctx, C, dt):
    T = 2000
    q, s = ctx.ckpt8_save(rnd(T, 260, seed=1))
    size = torch.exp(rnd(T, 1, seed=2) * 6)         # about 1e-8 .. 1e8
    dz = (rnd(T, C, seed=C) * 1e-3 / size).to(DT[dt])
    check(ctx, q, s * size, dz)


@pytest.mark.parametrize("C", CLASSES)
@pytest.mark.parametrize("ratio", [1e-2, 1e-4, 1e-6])
def test_columns_that_only_rows_with_a_small_dz_reach(ctx, C, ratio):
    # column j is nonzero in every fifth row; the five sets of rows have gradients of five magnitudes
    T, n = 1500, 256
    x = rnd(T, n, seed=3)
    band = torch.arange(T, device="cuda") % 5
    x *= (torch.arange(n, device="cuda")[None, :] % 5 == band[:, None])
    q, s = ctx.ckpt8_save(x)
    check(ctx, q, s, rnd(T, C, seed=C) * (ratio ** band.double())[:, None].float())


@pytest.mark.parametrize("C", CLASSES)
def test_magnitudes_whose_product_is_out_of_range_in_different_rows(ctx, C):
    T = 500
    q, s = ctx.ckpt8_save(rnd(T, 256, seed=4))
    dz = rnd(T, C, seed=C)
    s[7], dz[7] = 1e-10, 1e25
    s[300], dz[300] = 1e16, 0
    check(ctx, q, s, dz)
    dz = rnd(T, C, seed=C) * 1e-3                   # near the largest finite sums
    s.copy_(torch.rand(s.shape, generator=gen(5), device="cuda") + 0.5)
    s[100] = 2e36
    dz[100] = 1.0
    check(ctx, q, s, dz)


@pytest.mark.parametrize("C", [1, 2, 40, 64])
@pytest.mark.parametrize("T", [32, 512, 1024, 5000])
def test_long_chains_of_one_sign(ctx, T, C):
    # every addition rounds the same way where sums are cut off instead of rounded
    x = torch.rand(T, 200, generator=gen(6), device="cuda") + 0.5
    q, s = ctx.ckpt8_save(x)
    dz = torch.rand(T, C, generator=gen(7), device="cuda") + 0.5
    ctx.set_sm_limit(1)                             # all rows in one chain
    try:
        check(ctx, q, s, dz)
    finally:
        ctx.set_sm_limit(0)
    check(ctx, q, s, dz)


@pytest.mark.parametrize("C", [1, 2, 40, 64])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_reach_what_they_enter_and_nothing_else(ctx, C, bad):
    T, n = 600, 300
    q, s = ctx.ckpt8_save(rnd(T, n, seed=8))
    dz = rnd(T, C, seed=C)
    dz[211, C // 2] = bad
    gw, gb = ctx.ckpt8_grad(q, s, dz)
    here = torch.arange(C, device="cuda") == C // 2
    assert torch.equal(torch.isfinite(gw), ~here[:, None].expand(C, n)) and torch.equal(torch.isfinite(gb), ~here)
    dz = rnd(T, C, seed=C)
    s[500, 1] = bad                                 # columns 128 .. 255
    gw, gb = ctx.ckpt8_grad(q, s, dz)
    here = (torch.arange(n, device="cuda") // 128 == 1)[None, :]
    assert torch.equal(torch.isfinite(gw), ~here.expand(C, n)) and bool(torch.isfinite(gb).all())
